// Changes of the experts' biases: the sums of a group's delta rows.
//
// Bound by reading the deltas once (16,384 rows of 4,096 bfloat16: 134 MB, 20 us at the measured copy
// rate).  A warp reads rows in pieces of up to 16 bytes a lane; a CTA of eight warps takes a run of a
// group's rows by 32 pieces of columns, its warps every eighth row.  Groups of many rows are cut into
// runs, so that few groups fill the SMs too; the runs' sums go to scratch and the last CTA to arrive adds
// them in the runs' order, so that the result does not depend on which CTA that was.
#include "bp_experts_device.cuh"

namespace bp {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

// V columns a lane: 16 bytes of bfloat16, one float32.  The loads are volatile so that a batch of them is
// under way before the first is added: ptxas sinks plain ones to their uses.
template <class T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
    static constexpr int V = 8;
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    }
    __device__ __forceinline__ void add(float (&s)[V]) const {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[2 * i] += __uint_as_float(w[i] << 16);
            s[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <>
struct Piece<float> {
    static constexpr int V = 1;
    float x;
    __device__ __forceinline__ void load(const float* p) { asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(x) : "l"(p)); }
    __device__ __forceinline__ void add(float (&s)[V]) const { s[0] += x; }
};

template <class T>
__global__ void __launch_bounds__(kThreads) k_sums(SumsArgs g) {
    constexpr int V = Piece<T>::V, B = 8;
    __shared__ float part[kWarps][32 * V];
    __shared__ int last;
    const int e = blockIdx.y, runs = gridDim.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n0 = blockIdx.x * 32 * V, n = n0 + lane * V;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    const int per = (hi - lo + runs - 1) / runs, r0 = lo + blockIdx.z * per, r1 = min(hi, r0 + per);
    float s[V] = {};
    if (n < g.N) {
        const T* d = (const T*)g.d + n;
        Piece<T> p[B];
        int r = r0 + warp;
        for (; r + (B - 1) * kWarps < r1; r += B * kWarps) {
#pragma unroll
            for (int i = 0; i < B; ++i) p[i].load(d + (size_t)(r + i * kWarps) * g.N);
#pragma unroll
            for (int i = 0; i < B; ++i) p[i].add(s);
        }
        if (r < r1) {   // fewer than B left: the last row again in place of those past it
#pragma unroll
            for (int i = 0; i < B; ++i) p[i].load(d + (size_t)min(r + i * kWarps, r1 - 1) * g.N);
#pragma unroll
            for (int i = 0; i < B; ++i)
                if (r + i * kWarps < r1) p[i].add(s);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) part[warp][lane * V + i] = s[i];
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * V; c += kThreads) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) x += part[w][c];
        if (n0 + c >= g.N) continue;
        if (runs > 1) {
            g.scratch[((size_t)blockIdx.z * gridDim.y + e) * g.N + n0 + c] = x;
        } else {
            float* p = g.S + (size_t)e * g.N + n0 + c;
            *p = g.accumulate ? *p + x : x;
        }
    }
    if (runs == 1) return;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned* count = g.arrived + (size_t)e * gridDim.x + blockIdx.x;
        last = atomicAdd(count, 1u) == (unsigned)runs - 1;
        if (last) *count = 0;   // for the next call
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int c = threadIdx.x; c < 32 * V && n0 + c < g.N; c += kThreads) {
        float x = 0.f;
        for (int z = 0; z < runs; ++z) x += __ldcg(&g.scratch[((size_t)z * gridDim.y + e) * g.N + n0 + c]);
        float* p = g.S + (size_t)e * g.N + n0 + c;
        *p = g.accumulate ? *p + x : x;
    }
}

}  // namespace

// Runs of a group: CTAs for every SM several times over, of at least 64 rows on average.
int sums_runs(int n_rows, int n_groups, int N, int dtype, int num_sms) {
    const int cols = 32 * (dtype == BP_F32 ? 1 : 8), tiles = (N + cols - 1) / cols;
    int runs = 1;
    while (runs < kMaxSumRuns && (long long)tiles * n_groups * runs < 6 * num_sms && n_rows / ((long long)n_groups * runs) >= 128) runs *= 2;
    return runs;
}

cudaError_t group_sums(const SumsArgs& a, int dtype, int num_sms, cudaStream_t s) {
    const int cols = 32 * (dtype == BP_F32 ? 1 : 8);
    const dim3 grid((a.N + cols - 1) / cols, a.groups.n_groups, sums_runs(a.groups.n_rows, a.groups.n_groups, a.N, dtype, num_sms));
    // not a dependent launch: started beside the change's last tiles, it cost more than it
    // gained (gradients of 1,001 patterns: 46 and 48 us, this way 41 and 44)
    if (dtype == BP_F32) k_sums<float><<<grid, kThreads, 0, s>>>(a);
    else k_sums<__nv_bfloat16><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace bp
