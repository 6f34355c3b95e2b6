// Device helpers that the two routers share: order of floats, and the rows of a block's choices.
#pragma once

#include "bp_experts_device.cuh"

namespace bp {

// Ascending whole numbers for ascending floats; 0 for NaN and for -infinity, which are never
// chosen.  (x + 0 turns -0 into +0, so that the two tie.)
__device__ __forceinline__ unsigned order_of(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    if (!(x > -INFINITY)) return 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned o) {
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A block's patterns that chose expert e, as bits: bits[e * kWords + word].
template <int kWords>
__device__ __forceinline__ int rank_of(const unsigned* bits, int e, int p) {
    int r = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const unsigned m = p >= 32 * (w + 1) ? 0xffffffffu : p > 32 * w ? (1u << (p - 32 * w)) - 1u : 0u;
        r += __popc(bits[e * kWords + w] & m);
    }
    return r;
}
template <int kWords>
__device__ __forceinline__ int count_of(const unsigned* bits, int e) {
    int r = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) r += __popc(bits[e * kWords + w]);
    return r;
}

// Rows of a block's choices: base[e] is the row of the block's first pattern with expert e.
template <int kWords>
__device__ __forceinline__ void place_rows(const RouteArgs& g, const unsigned* bits, const int* base, int p0, int np) {
    for (int i = threadIdx.x; i < np * g.k; i += blockDim.x) {
        const int p = i / g.k, e = g.expert[(size_t)p0 * g.k + i];
        int at = -1;
        if (e >= 0) {
            at = base[e] + rank_of<kWords>(bits, e, p);
            g.source[at] = p0 + p;
        }
        g.place[(size_t)p0 * g.k + i] = at;
    }
}

// Exclusive sums of cnt[0 .. E) by the block, and the total.
__device__ __forceinline__ int block_scan(int* cnt, int E, int* warp_tot) {
    int carry = 0;
    for (int b = 0; b < E; b += blockDim.x) {
        const int i = b + threadIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
        const int x = i < E ? cnt[i] : 0;
        int s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        __syncthreads();
        if (lane == 31) warp_tot[w] = s;
        __syncthreads();
        int before = carry;
        for (int v = 0; v < (int)blockDim.x / 32; ++v) {
            if (v < w) before += warp_tot[v];
            carry += warp_tot[v];
        }
        if (i < E) cnt[i] = before + s - x;
    }
    __syncthreads();
    return carry;
}

}  // namespace bp
