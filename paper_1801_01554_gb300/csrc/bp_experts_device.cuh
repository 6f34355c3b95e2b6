// Device helpers that the kernels of the expert and adapter layers share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "bp_experts_internal.h"

namespace bp {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// The rows of group g, clamped to [0, n_rows] and to ascending order.
__device__ __forceinline__ void group_rows(const int* offsets, int n_rows, int g, int& lo, int& hi, int* flags) {
    if (offsets == nullptr) {
        lo = 0;
        hi = n_rows;
        return;
    }
    const int a = offsets[g], b = offsets[g + 1];
    lo = min(max(a, 0), n_rows);
    hi = min(max(b, lo), n_rows);
    if (lo != a || hi != b) atomicOr(flags, kFlagBounds);
}

// A row's source, row 0 where it is out of range.
__device__ __forceinline__ int source_row(const int* source, int r, int n, int* flags) {
    if (source == nullptr) return r;
    const int s = source[r];
    if ((unsigned)s < (unsigned)n) return s;
    atomicOr(flags, kFlagBounds);
    return 0;
}

// The adapter of request i, -1 for none.
__device__ __forceinline__ int request_adapter(const Requests& q, int i, int* flags) {
    const int a = q.adapter[i];
    if (a >= -1 && a < q.n_adapters) return a;
    atomicOr(flags, kFlagBounds);
    return -1;
}

// The first request that ends after row r (n_requests if none): offsets ascend.
__device__ __forceinline__ int first_request(const Requests& q, int r) {
    int lo = 0, hi = q.n_requests;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (q.offsets[mid + 1] > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// The `tile`-th block of TM rows of the groups, by one converged warp: group and first row, or
// g = -1 past the last one.  Every lane gets the result.
template <int TM>
__device__ __forceinline__ void find_tile(const RowGroups& q, int tile, int& g, int& row0, int& end, int* flags) {
    const int lane = threadIdx.x & 31;
    for (int base = 0; base < q.n_groups; base += 32) {
        int lo = 0, hi = 0;
        if (base + lane < q.n_groups) group_rows(q.offsets, q.n_rows, base + lane, lo, hi, flags);
        const int tiles = (hi - lo + TM - 1) / TM;
        int sum = tiles;   // inclusive
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += x;
        }
        const unsigned past = __ballot_sync(0xffffffffu, sum > tile);
        if (past != 0) {
            const int l = __ffs(past) - 1;
            g = base + l;
            const int before = __shfl_sync(0xffffffffu, sum - tiles, l);
            row0 = __shfl_sync(0xffffffffu, lo, l) + (tile - before) * TM;
            end = __shfl_sync(0xffffffffu, hi, l);
            return;
        }
        tile -= __shfl_sync(0xffffffffu, sum, 31);
    }
    g = -1;
    row0 = end = 0;
}

// d += a b: 16 x 16 bfloat16 (rows of k) by 16 x 8 (columns of k), float32 sums.
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// acc += A B over one warp's steps of 32 of K (first, first + step, ..), A of NA tiles of 16 rows, B of
// NB tiles of 8 columns, both with k contiguous; a and b point at this lane's rows (lane / 4, and 8
// further for a[.][1]) and its eight values of k, 8 (lane % 4), or are NULL for rows whose sums are not
// kept; `any` is a row that they may read instead.  The eight values stand for the four pairs of k that
// two MMAs want, the same eight in both operands, so that the sum over k is only taken in another order.
template <int NA, int NB>
__device__ __forceinline__ void step_products(float (&acc)[NA][NB][4], const uint4 (&x)[NA][2], const uint4 (&y)[NB]) {
#pragma unroll
    for (int m = 0; m < NA; ++m)
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            mma_16816(acc[m][c], x[m][0].x, x[m][1].x, x[m][0].y, x[m][1].y, y[c].x, y[c].y);
            mma_16816(acc[m][c], x[m][0].z, x[m][1].z, x[m][0].w, x[m][1].w, y[c].z, y[c].w);
        }
}

// Loads straight into registers, B steps under way.  No load hangs on a condition but in the last,
// short step.
// PART > 0: after PART steps a sum is added to the total by rounding to nearest, because mma.sync truncates
// as it accumulates (a sum of positive products comes out 7e-8 of itself too small for every 16 of them).
template <int NA, int NB, int B, int PART = 0>
__device__ __forceinline__ void direct_products(float (&total)[NA][NB][4], const __nv_bfloat16* (&a)[NA][2],
                                                const __nv_bfloat16* (&b)[NB], const __nv_bfloat16* any, int K, int first,
                                                int step) {
    const int k8 = (threadIdx.x & 3) * 8, whole = K / 32;
#pragma unroll
    for (int m = 0; m < NA; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) a[m][h] = a[m][h] != nullptr ? a[m][h] : any + k8;
#pragma unroll
    for (int c = 0; c < NB; ++c) b[c] = b[c] != nullptr ? b[c] : any + k8;
    int k = first, steps = 0;
    float acc[NA][NB][4] = {};
    auto add = [&] {
#pragma unroll
        for (int m = 0; m < NA; ++m)
#pragma unroll
            for (int c = 0; c < NB; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) total[m][c][i] += acc[m][c][i], acc[m][c][i] = 0.f;
    };
    auto load = [](const __nv_bfloat16* p) {   // volatile: ptxas may not sink it to its use
        uint4 u;
        asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
        return u;
    };
    auto batch = [&](auto count) {
        constexpr int n = decltype(count)::value;
        uint4 x[n][NA][2], y[n][NB];
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int at = (k + i * step) * 32;
#pragma unroll
            for (int m = 0; m < NA; ++m) x[i][m][0] = load(a[m][0] + at), x[i][m][1] = load(a[m][1] + at);
#pragma unroll
            for (int c = 0; c < NB; ++c) y[i][c] = load(b[c] + at);
        }
#pragma unroll
        for (int i = 0; i < n; ++i) step_products<NA, NB>(acc, x[i], y[i]);
        k += n * step;
    };
    while (k + (B - 1) * step < whole) {
        batch(std::integral_constant<int, B>{});
        if constexpr (PART > 0) {
            static_assert(PART % B == 0);
            steps += B;
            if (steps % PART == 0) add();
        }
    }
    while (k < whole) batch(std::integral_constant<int, 1>{});
    if (k == whole && k * 32 < K) {   // this warp has the rest of K
        const bool in = k * 32 + k8 < K;
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        uint4 x[NA][2], y[NB];
#pragma unroll
        for (int m = 0; m < NA; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[m][h] = in ? *reinterpret_cast<const uint4*>(a[m][h] + k * 32) : zero;
#pragma unroll
        for (int c = 0; c < NB; ++c) y[c] = in ? *reinterpret_cast<const uint4*>(b[c] + k * 32) : zero;
        step_products<NA, NB>(acc, x, y);
    }
    add();
}

// Loads through S steps of shared memory by cp.async, each lane reading back what it copied itself: no
// barriers, and more under way than registers would hold where a step is many pieces (61 rows of
// 4096-4096: 14 us against 17; of few pieces the copies cost more than they hide, 9.5 against 6).
// `ring`: this warp's ring_bytes<NA, NB, S>() of shared memory.
template <int NA, int NB, int S>
constexpr int ring_bytes() { return S * (2 * NA + NB) * 512; }
template <int NA, int NB, int S>
__device__ __forceinline__ void ring_products(float (&acc)[NA][NB][4], const __nv_bfloat16* (&a)[NA][2],
                                              const __nv_bfloat16* (&b)[NB], const __nv_bfloat16* any, int K, int first,
                                              int step, void* ring) {
    constexpr int P = 2 * NA + NB;
    const int lane = threadIdx.x & 31, k8 = (lane & 3) * 8;
    uint4* mine = reinterpret_cast<uint4*>(ring) + lane;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine);
    const int steps = first * 32 < K ? ((K + 31) / 32 - first + step - 1) / step : 0;
    auto copy = [&](int i) {
        const int k = (first + i * step) * 32;
        const bool in = i < steps && k + k8 < K;
        const uint32_t at = to + (i % S) * P * 512;
        auto piece = [&](int p, const __nv_bfloat16* src) {   // zeros where nothing is to be read
            const bool read = in && src != nullptr;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + p * 512), "l"(read ? src + k : any),
                         "r"(read ? 16 : 0)
                         : "memory");
        };
#pragma unroll
        for (int m = 0; m < NA; ++m) piece(2 * m, a[m][0]), piece(2 * m + 1, a[m][1]);
#pragma unroll
        for (int c = 0; c < NB; ++c) piece(2 * NA + c, b[c]);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) copy(i);
    for (int i = 0; i < steps; ++i) {
        copy(i + S - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
        const uint4* from = mine + (i % S) * P * 32;
        uint4 x[NA][2], y[NB];
#pragma unroll
        for (int m = 0; m < NA; ++m) x[m][0] = from[2 * m * 32], x[m][1] = from[(2 * m + 1) * 32];
#pragma unroll
        for (int c = 0; c < NB; ++c) y[c] = from[(2 * NA + c) * 32];
        step_products<NA, NB>(acc, x, y);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// What block t of kTileRows rows holds (see kTileRows).
// (a converged warp asks)
__device__ __forceinline__ int2 tile_info(const Requests& q, int t, int* flags) {
    const int row0 = t * kTileRows, end = min(row0 + kTileRows, q.n_rows), first = first_request(q, row0);
    int count = 0;
    for (int base = first; base < q.n_requests; base += 32) {
        const int i = base + (threadIdx.x & 31);
        int lo = q.n_rows, hi = q.n_rows, a = -1;
        if (i < q.n_requests) {
            group_rows(q.offsets, q.n_rows, i, lo, hi, flags);
            a = request_adapter(q, i, flags);
        }
        const unsigned whole = __ballot_sync(0xffffffffu, hi > lo && lo <= row0 && hi >= end);
        if (whole != 0) {
            const int l = __ffs(whole) - 1;
            return make_int2(__shfl_sync(0xffffffffu, a, l), base + l);
        }
        count += __popc(__ballot_sync(0xffffffffu, hi > lo && lo < end && a >= 0));
        if (2 * count > q.rank) return make_int2(kTileByRow, first);
        if (__any_sync(0xffffffffu, lo >= end)) break;
    }
    return make_int2(count > 0 ? kTileMixed : -1, first);
}

// Rows outside every request: zeros in low [n_rows, rank] and in the terms [n_rows, pitch], if any
// (pitch at least the rank).
__device__ __forceinline__ void zero_outside(const Requests& q, int thread, int threads, float* low, __nv_bfloat16* terms,
                                             int pitch) {
    const int lo = q.n_requests > 0 ? min(max(q.offsets[0], 0), q.n_rows) : q.n_rows;
    const int hi = q.n_requests > 0 ? min(max(q.offsets[q.n_requests], lo), q.n_rows) : q.n_rows;
    for (long long i = thread; i < (long long)(lo + q.n_rows - hi) * pitch; i += threads) {
        const long long k = i / pitch, row = k < lo ? k : k - lo + hi;
        const int j = (int)(i - k * pitch);
        if (terms != nullptr) terms[row * pitch + j] = __float2bfloat16_rn(0.f);
        if (j < q.rank) low[row * q.rank + j] = 0.f;
    }
}

// Most blocks of TM rows that n_rows rows in n_groups groups can make.
inline int max_tiles(long long n_rows, long long n_groups, int TM) {
    const long long t = n_rows / TM + n_groups;
    return (int)(t < n_rows ? t : n_rows);
}

}  // namespace bp
