// The norm of many changes together, and the changes scaled down to a bound.
#include "bp_blocks_internal.h"
#include "bp_pieces.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kValues = kClipTile / kThreads;   // of a thread and tile
constexpr int kBlocksPerSm = 8;

// The sum of squares of a thread's values: in float32 where that neither overflows nor loses any that count, else of
// the values times a power of two.
template <int N>
__device__ __forceinline__ double squares(const float (&v)[N]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
    if (s >= 1e-25f && s <= 1e37f) return (double)s;
    const bool large = !(s < 1.f);   // (a NaN too: it stays one)
    const float by = large ? 0x1p-70f : 0x1p100f;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(v[i] * by, v[i] * by, s);
    return (double)s * (large ? 0x1p140 : 0x1p-200);
}

// The block's sum, in one order, in every thread.
__device__ __forceinline__ double block_sum(double x, double* part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
    for (int w = 1; w < kWarps; ++w) x += part[w];
    return x;
}

// A chunk's values in 16-byte pieces: `head` values before the first whole piece, `pieces` pieces, `tail` values
// behind them.
template <class T>
struct Split {
    static constexpr int V = 16 / (int)sizeof(T);
    const T* in;
    long long pieces;
    int head, tail;
    __device__ __forceinline__ explicit Split(const ClipChunk& c) {
        in = (const T*)c.in;
        head = (int)min((long long)((16 - ((uintptr_t)in & 15)) & 15) / (long long)sizeof(T), (long long)c.count);
        pieces = ((long long)c.count - head) / V;
        tail = (int)((long long)c.count - head - pieces * V);
    }
};

template <class T>
__device__ __forceinline__ double chunk_squares(const ClipChunk& c) {
    constexpr int V = Split<T>::V, J = kValues / V;
    const Split<T> s(c);
    const T* body = s.in + s.head;
    double sum = 0.0;
    for (long long b = 0; b < s.pieces; b += kThreads * J) {
        Piece<T, V> p[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const long long at = b + j * kThreads + threadIdx.x;
            p[j].u = make_uint4(0u, 0u, 0u, 0u);
            if (at < s.pieces) p[j].load_rw(body + at * V);
        }
        float v[kValues];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float x[V];
            p[j].values(x);
#pragma unroll
            for (int i = 0; i < V; ++i) v[j * V + i] = x[i];
        }
        sum += squares(v);
    }
    const int edge = (int)threadIdx.x;
    if (edge < s.head + s.tail) {
        const float v[1] = {to_f32(edge < s.head ? s.in[edge] : body[s.pieces * V + edge - s.head])};
        sum += squares(v);
    }
    return sum;
}

template <class T>
__device__ __forceinline__ void scale_chunk(const ClipChunk& c, float by) {
    constexpr int V = Split<T>::V, J = kValues / V;
    const Split<T> s(c);
    const T* body = s.in + s.head;
    T* out = (T*)c.out;
    const bool whole = (((uintptr_t)c.in ^ (uintptr_t)c.out) & 15) == 0;   // pieces of one are pieces of the other
    for (long long b = 0; b < s.pieces; b += kThreads * J) {
        Piece<T, V> p[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const long long at = b + j * kThreads + threadIdx.x;
            if (at < s.pieces) p[j].load_rw(body + at * V);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const long long at = b + j * kThreads + threadIdx.x;
            if (at >= s.pieces) continue;
            float x[V];
            p[j].values(x);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] *= by;
            T* to = out + s.head + at * V;
            if (whole) {
                p[j].set(x);
                p[j].store(to);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) to[i] = from_f32<T>(x[i]);
            }
        }
    }
    const int edge = (int)threadIdx.x;
    if (edge < s.head + s.tail) {
        const long long at = edge < s.head ? edge : s.head + s.pieces * V + edge - s.head;
        out[at] = from_f32<T>(to_f32(s.in[at]) * by);
    }
}

// Squares of every blocks-th chunk, summed up by block.  Bound by reading the values once.
__global__ void __launch_bounds__(kThreads) k_clip_norm(ClipArgs g) {
    __shared__ double part[kWarps];
    pdl_launch();
    double sum = 0.0;
    for (int i = blockIdx.x; i < g.n_chunks; i += gridDim.x) {
        const ClipChunk c = g.chunks[i];
        sum += c.dtype == BP_BF16 ? chunk_squares<__nv_bfloat16>(c) : chunk_squares<float>(c);
    }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) g.partial[blockIdx.x] = sum;
}

// What the values are multiplied by, the same in every block: 1 where nothing is clipped.
__device__ __forceinline__ float clip_factor(const ClipArgs& g, double total) {
    const double norm = sqrt(total);
    const bool finite = norm <= 1.7e308;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (g.norm != nullptr) *g.norm = (float)norm;
        if (!finite) atomicOr(g.flags, kFlagNonfinite);
    }
    return finite && norm > (double)g.max_norm ? (float)((double)g.max_norm / norm) : 1.f;
}

__global__ void __launch_bounds__(kThreads) k_clip_scale(ClipArgs g, int blocks) {
    __shared__ double part[kWarps];
    pdl_wait();
    double sum = 0.0;
    for (int i = threadIdx.x; i < blocks; i += kThreads) sum += __ldcg(g.partial + i);
    const float by = clip_factor(g, block_sum(sum, part));
    if (!g.write || (by == 1.f && g.in_place)) return;
    for (int i = blockIdx.x; i < g.n_chunks; i += gridDim.x) {
        const ClipChunk c = g.chunks[i];
        if (by == 1.f && c.in == c.out) continue;
        if (c.dtype == BP_BF16) scale_chunk<__nv_bfloat16>(c, by);
        else scale_chunk<float>(c, by);
    }
}

}  // namespace

int clip_blocks(int num_sms) { return num_sms * kBlocksPerSm; }

cudaError_t clip_run(const ClipArgs& a, int num_sms, cudaStream_t s) {
    const int blocks = max(1, min(a.n_chunks, clip_blocks(num_sms)));
    k_clip_norm<<<blocks, kThreads, 0, s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_pdl(k_clip_scale, a.write ? blocks : 1, 1, kThreads, 0, s, a, blocks);
}

}  // namespace bp
