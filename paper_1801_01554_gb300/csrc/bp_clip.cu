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

// The block's sum, in one order, in every thread: each warp's first where the block has its SM to itself; by one warp
// where it shares it, as a float64 sum is 16 cycles of the SM's unit for every warp that takes part.
__device__ __forceinline__ double block_sum_alone(double x, double* part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
    for (int w = 1; w < kWarps; ++w) x += part[w];
    return x;
}
__device__ __forceinline__ double block_sum(double x, double* part) {   // part [kThreads]
    part[threadIdx.x] = x;
    __syncthreads();
    if (threadIdx.x < 32) {
#pragma unroll
        for (int w = 1; w < kWarps; ++w) x += part[w * 32 + threadIdx.x];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (threadIdx.x == 0) part[0] = x;
    }
    __syncthreads();
    return part[0];
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

// What values are multiplied by: `by`, or `far` where the factor is below float32's normal numbers, which have fewer bits the
// smaller they are, and then none (a bound of 1e-9 for a norm of 1e38 takes a factor of 1e-47 to values of 1e-9); else 0.
struct Factor {
    float by;
    double far;
};
template <class T>
__device__ __forceinline__ void scale_far(const ClipChunk& c, double far) {
    const T* in = (const T*)c.in;
    T* out = (T*)c.out;
    for (unsigned i = threadIdx.x; i < c.count; i += kThreads) out[i] = from_f32<T>((float)((double)to_f32(in[i]) * far));
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

// Squares of every blocks-th chunk, summed up by block; the block that comes last adds up the blocks' sums, in their
// order.  Bound by reading the values once.
__global__ void __launch_bounds__(kThreads) k_clip_norm(ClipArgs g) {
    __shared__ double part[kThreads];
    __shared__ bool last;
    pdl_launch();
    double sum = 0.0;
    for (int i = blockIdx.x; i < g.n_chunks; i += gridDim.x) {
        const ClipChunk c = g.chunks[i];
        sum += c.dtype == BP_BF16 ? chunk_squares<__nv_bfloat16>(c) : chunk_squares<float>(c);
    }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) {
        g.partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(g.arrived, 1u) == gridDim.x - 1;
        if (last) *g.arrived = 0u;   // for the next call
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) sum += __ldcg(g.partial + i);
    __syncthreads();
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) *g.total = sum;
}

// What the values are multiplied by, the same in every block: 1 where nothing is clipped.  The root is float32's, of the sum
// times an even power of two (float64's root and quotient take some 2 us).
__device__ __forceinline__ Factor clip_factor(const ClipArgs& g, double total) {
    const bool finite = total <= 1.7e308;   // (not a NaN)
    const int half = total > 0.0 && finite ? (((__double2hiint(total) >> 20) & 0x7ff) - 1023) >> 1 : 0;
    // total * 4^-half lies in [1, 4): a normal number, as sums of squares are none or at least 2^-298
    const double m = __hiloint2double(__double2hiint(total) - (half << 21), __double2loint(total));
    const float root = finite ? sqrtf((float)(total > 0.0 ? m : 0.0)) : (float)total, norm = ldexpf(root, half);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (g.norm != nullptr) *g.norm = norm;
        if (!finite) atomicOr(g.flags, kFlagNonfinite);
    }
    Factor f{1.f, 0.0};
    if (finite && norm > g.max_norm) {   // (infinity is above every bound)
        f.by = ldexpf(g.max_norm / root, -half);
        if (f.by < 0x1p-126f && g.max_norm > 0.f) f.far = ldexp((double)g.max_norm / (double)root, -half);
    }
    return f;
}

__device__ __forceinline__ void scale(const ClipArgs& g, int i, const Factor& f) {
    const ClipChunk c = g.chunks[i];
    if (f.by == 1.f && c.in == c.out) return;
    if (f.far != 0.0) {
        if (c.dtype == BP_BF16) scale_far<__nv_bfloat16>(c, f.far);
        else scale_far<float>(c, f.far);
    } else if (c.dtype == BP_BF16) {
        scale_chunk<__nv_bfloat16>(c, f.by);
    } else {
        scale_chunk<float>(c, f.by);
    }
}

// Bound by reading the values again and writing them.  (Of 1 GB that the norm has read L2 keeps nothing to speak of: the same time
// from the last chunk to the first.)
__global__ void __launch_bounds__(kThreads) k_clip_scale(ClipArgs g) {
    pdl_wait();
    const Factor f = clip_factor(g, __ldcg(g.total));
    if (!g.write || (f.by == 1.f && g.in_place)) return;
    for (int i = blockIdx.x; i < g.n_chunks; i += gridDim.x) scale(g, i, f);
}

// Few chunks: one launch of one cluster, a CTA a chunk, whose values stay in registers while the CTAs read one
// another's sums.
constexpr int kFewCtas = kClipFew;
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <class T>
__device__ __forceinline__ void clip_chunk(const ClipArgs& g, const ClipChunk& c, double* part, double* mine) {
    constexpr int V = Split<T>::V, J = kValues / V;
    const Split<T> s(c);
    const T* body = s.in + s.head;
    T* out = (T*)c.out;
    const bool whole = (((uintptr_t)c.in ^ (uintptr_t)c.out) & 15) == 0, edge = (int)threadIdx.x < s.head + s.tail;
    const long long edge_at = (int)threadIdx.x < s.head ? (long long)threadIdx.x : s.pieces * V + (long long)threadIdx.x;
    Piece<T, V> p[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const long long at = j * kThreads + threadIdx.x;
        p[j].u = make_uint4(0u, 0u, 0u, 0u);
        if (at < s.pieces) p[j].load_rw(body + at * V);
    }
    const float e[1] = {edge ? to_f32(s.in[edge_at]) : 0.f};
    float v[J * V];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        float x[V];
        p[j].values(x);
#pragma unroll
        for (int i = 0; i < V; ++i) v[j * V + i] = x[i];
    }
    const double sum = block_sum_alone(squares(v) + squares(e), part);
    if (threadIdx.x == 0) *mine = sum;
    cluster_sync();
    double sums[kFewCtas], total = 0.0;
#pragma unroll
    for (int r = 0; r < kFewCtas; ++r) {
        unsigned a;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(mine)), "r"(r));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(sums[r]) : "r"(a) : "memory");
    }
#pragma unroll
    for (int r = 0; r < kFewCtas; ++r) total += sums[r];
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // this CTA has read the sums
    const Factor f = clip_factor(g, total);
    const float by = f.by;
    if (g.write && f.far != 0.0) {
        scale_far<T>(c, f.far);
    } else if (g.write && !(by == 1.f && c.in == c.out)) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const long long at = j * kThreads + threadIdx.x;
            if (at >= s.pieces) continue;
            float x[V];
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = v[j * V + i] * by;
            T* to = out + s.head + at * V;
            if (whole) {
                p[j].set(x);
                p[j].store(to);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) to[i] = from_f32<T>(x[i]);
            }
        }
        if (edge) out[edge_at] = from_f32<T>(e[0] * by);
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // no CTA leaves while another reads its sum
}
__global__ void __launch_bounds__(kThreads) k_clip_few(ClipArgs g, __grid_constant__ const ClipFew few) {
    __shared__ double part[kWarps];
    __shared__ double mine;
    const ClipChunk c = few.chunks[blockIdx.x];   // (empty ones behind the last)
    if (c.dtype == BP_BF16) clip_chunk<__nv_bfloat16>(g, c, part, &mine);
    else clip_chunk<float>(g, c, part, &mine);
}

cudaLaunchConfig_t few_config(cudaLaunchAttribute* at, cudaStream_t s) {
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = kFewCtas;
    at->val.clusterDim.y = at->val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(kFewCtas);
    c.blockDim = dim3(kThreads);
    c.stream = s;
    c.attrs = at;
    c.numAttrs = 1;
    return c;
}

}  // namespace

// Whether the device holds a cluster of kFewCtas, so that calls of as many chunks, of a tile at most, go to k_clip_few.
cudaError_t clip_setup(int n_chunks, bool tiles, int* few) {
    *few = 0;
    cudaError_t e = cudaFuncSetAttribute(k_clip_few, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess || n_chunks > kFewCtas || !tiles) return e;
    cudaLaunchAttribute at;
    const cudaLaunchConfig_t c = few_config(&at, nullptr);
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, k_clip_few, &c) == cudaSuccess) *few = clusters > 0;
    else cudaGetLastError();
    return cudaSuccess;
}

int clip_blocks(int num_sms) { return num_sms * kBlocksPerSm; }

cudaError_t clip_run(const ClipArgs& a, const ClipFew& few, int num_sms, cudaStream_t s) {
    if (a.few) {
        cudaLaunchAttribute at;
        const cudaLaunchConfig_t c = few_config(&at, s);
        return cudaLaunchKernelEx(&c, k_clip_few, a, few);
    }
    const int blocks = max(1, min(a.n_chunks, clip_blocks(num_sms)));
    k_clip_norm<<<blocks, kThreads, 0, s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_pdl(k_clip_scale, a.write ? blocks : 1, 1, kThreads, 0, s, a);
}

}  // namespace bp
