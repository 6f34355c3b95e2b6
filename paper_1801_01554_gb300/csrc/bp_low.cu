// The low-rank products of the adapter layers in bfloat16: low = scale_a P_a x for the rows of
// every request, on mma.sync.
//
// A product with so few columns is bound by reading x (and, of requests of one row, by reading
// their adapters): 16,384 rows of 4,096 are 134 MB and 20 us at the measured copy rate, the
// 2 * 64 * 16,384 * 4,096 flops of rank 64 a fraction of that on mma.sync, whose 16-row tiles fit
// short requests where a tcgen05 tile would hold 128 rows.  A CTA takes up to 64 rows of one
// request.  Warps share K and, from 32 on, the rank; their sums are added in shared memory in a
// fixed order.
#include "bp_experts_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kRows = 64, kThreads = 256, kWarps = kThreads / 32;
// Steps of 32 of a warp's sum in one part (direct_products): the sums are float32 results.
constexpr int kPart = 16;

// The unit-th run of up to kRows rows of one request; the whole block calls it.  Request, first row
// and end, or request -1 past the last unit.
__device__ __forceinline__ void find_unit(const Requests& q, int unit, int (&where)[3], int* warp_tot, int* flags) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) where[0] = -1;
    for (int base = 0; base < q.n_requests; base += kThreads) {
        const int i = base + threadIdx.x;
        int lo = 0, hi = 0;
        if (i < q.n_requests) group_rows(q.offsets, q.n_rows, i, lo, hi, flags);
        const int units = (hi - lo + kRows - 1) / kRows;
        int sum = units;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
        }
        __syncthreads();
        if (lane == 31) warp_tot[warp] = sum;
        __syncthreads();
        int before = 0, total = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += warp_tot[w];
            total += warp_tot[w];
        }
        const int first = before + sum - units;
        if (unit >= first && unit < first + units) {
            where[0] = i;
            where[1] = lo + (unit - first) * kRows;
            where[2] = min(hi, where[1] + kRows);
        }
        if (unit < total) break;
        unit -= total;
    }
    __syncthreads();
}

// A row's terms: x rounded to bfloat16, the rest rounded, ..; three add up to x but for 2^-25 of it.
__device__ __forceinline__ void store_terms(bf16* terms, int stride, int n_terms, float x) {
    for (int t = 0; t < n_terms; ++t) {
        const bf16 h = __float2bfloat16_rn(x);
        terms[t * stride] = h;
        const float f = __bfloat162float(h);
        x = isfinite(f) ? x - f : 0.f;
    }
}

// Rows of one request in low and in the terms, from their sums [rows, pitch] in shared memory (NULL:
// zeros), by the whole block: eight ranks of a row a thread, a term's in one 16-byte store.  (A value at a
// time from the registers of the warp that has the sums: 24 us for 66 rows of rank 16, where the sums
// take 8.)
__device__ __forceinline__ void store_rows_low(const LowArgs& g, int row0, int rows, const float* sums, int pitch, float scale_low,
                                               float scale_terms) {
    const int r = g.req.rank, per = g.n_terms > 0 ? g.terms_stride / 8 : (r + 7) / 8;
    for (int i = threadIdx.x; i < rows * per; i += kThreads) {
        const int m = i / per, j0 = i % per * 8;
        const size_t row = row0 + m;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = sums != nullptr && j0 + j < r ? sums[m * pitch + j0 + j] : 0.f;
            if (j0 + j < r) g.low[row * r + j0 + j] = scale_low * v[j];
            v[j] *= scale_terms;
        }
        for (int t = 0; t < g.n_terms; ++t) {
            __align__(16) bf16 h[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[j] = __float2bfloat16_rn(v[j]);
                const float f = __bfloat162float(h[j]);
                v[j] = isfinite(f) ? v[j] - f : 0.f;
            }
            *reinterpret_cast<uint4*>((bf16*)g.terms + (row * g.n_terms + t) * g.terms_stride + j0) = *reinterpret_cast<const uint4*>(h);
        }
    }
}

template <int MT, int NT>
__device__ __forceinline__ void low_rows(const LowArgs& g, float scale_low, float scale_terms, int row0, int rows, int adapter,
                                         int rank_warps, float* red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = g.req.rank;
    const int kw = warp / rank_warps, nw = warp - kw * rank_warps, k_warps = kWarps / rank_warps;   // this warp's share
    const int j0 = nw * NT * 8;
    const int gr = lane >> 2, k8 = (lane & 3) * 8;
    const bf16 *in = (const bf16*)g.in + (size_t)row0 * g.K, *P = (const bf16*)g.P + (size_t)adapter * r * g.K;
    const bf16 *x[MT][2], *p[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[m][h] = 16 * m + 8 * h + gr < rows ? in + (size_t)(16 * m + 8 * h + gr) * g.K + k8 : nullptr;
#pragma unroll
    for (int n = 0; n < NT; ++n) p[n] = j0 + 8 * n + gr < r ? P + (size_t)(j0 + 8 * n + gr) * g.K + k8 : nullptr;
    float acc[MT][NT][4] = {};
    direct_products<MT, NT, (MT == 1 ? 4 : 2), kPart>(acc, x, p, in, g.K, kw, k_warps);
    for (int s = k_warps / 2; s >= 1; s >>= 1) {
        __syncthreads();
        float* at = red + (size_t)((kw % s) * rank_warps + nw) * MT * NT * 128 + lane;
        if (kw >= s && kw < 2 * s) {
#pragma unroll
            for (int i = 0; i < MT * NT * 4; ++i) at[i * 32] = acc[i / (NT * 4)][i / 4 % NT][i % 4];
        }
        __syncthreads();
        if (kw < s) {
#pragma unroll
            for (int i = 0; i < MT * NT * 4; ++i) acc[i / (NT * 4)][i / 4 % NT][i % 4] += at[i * 32];
        }
    }
    // the sums by rows, for the whole block
    const int pitch = rank_warps * NT * 8;
    __syncthreads();
    if (kw == 0) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * m + (lane >> 2) + 8 * (i >> 1), j = j0 + 8 * n + 2 * (lane & 3) + (i & 1);
                    red[row * pitch + j] = acc[m][n][i];
                }
    }
    __syncthreads();
    store_rows_low(g, row0, rows, red, pitch, scale_low, scale_terms);
}

// NT: eights of the rank of a warp.
template <int NT>
__global__ void __launch_bounds__(kThreads, 1) k_low(LowArgs g, int rank_warps, int tiles) {
    __shared__ int where[3];
    __shared__ int warp_tot[kWarps];
    __shared__ float red[kWarps / 2 * (kRows / 16) * NT * 128];
    static_assert(kRows * 4 * NT * 8 <= kWarps / 2 * (kRows / 16) * NT * 128, "room for the sums by rows");
    const Requests& q = g.req;
    pdl_launch();
    if (g.tiles != nullptr)
        for (int t = blockIdx.x + gridDim.x * (threadIdx.x >> 5); t < tiles; t += gridDim.x * kWarps) {
            const int2 info = tile_info(q, t, g.flags);
            if ((threadIdx.x & 31) == 0) g.tiles[t] = info;
        }
    if (blockIdx.x == 0)
        zero_outside(q, threadIdx.x, kThreads, g.low, g.n_terms > 0 ? (bf16*)g.terms : nullptr,
                     g.n_terms > 0 ? g.n_terms * g.terms_stride : q.rank);
    find_unit(q, blockIdx.x, where, warp_tot, g.flags);
    if (where[0] < 0) return;
    const int row0 = where[1], rows = where[2] - where[1], adapter = request_adapter(q, where[0], g.flags);
    if (adapter < 0) {
        store_rows_low(g, row0, rows, nullptr, 0, 0.f, 0.f);
        return;
    }
    const float c = g.scale != nullptr ? g.scale[adapter] : 1.f, scale_low = g.scaled_low ? c : 1.f;
    if (rows <= 16) low_rows<1, NT>(g, scale_low, c, row0, rows, adapter, rank_warps, red);
    else low_rows<kRows / 16, NT>(g, scale_low, c, row0, rows, adapter, rank_warps, red);
}

// The terms of given float32 rows [n_rows, rank].
__global__ void __launch_bounds__(kThreads) k_terms(const float* low, int n_rows, int rank, bf16* terms, int stride, int n_terms) {
    const long long n = (long long)n_rows * stride;
    for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
        const long long row = i / stride;
        const int j = (int)(i - row * stride);
        store_terms(terms + row * n_terms * stride + j, stride, n_terms, j < rank ? low[row * rank + j] : 0.f);
    }
}

}  // namespace

cudaError_t low_product(const LowArgs& a, cudaStream_t s) {
    const int tiles = (a.req.n_rows + kTileRows - 1) / kTileRows;
    int units = max_tiles(a.req.n_rows, a.req.n_requests, kRows);
    if (units < 1) units = 1;
    if (a.req.rank <= 16) {
        k_low<2><<<units, kThreads, 0, s>>>(a, 1, tiles);
    } else {
        const int w = a.req.rank <= 32 ? 1 : a.req.rank <= 64 ? 2 : 4;
        k_low<4><<<units, kThreads, 0, s>>>(a, w, tiles);
    }
    return cudaGetLastError();
}

cudaError_t low_terms(const float* low, int n_rows, int rank, void* terms, int stride, int n_terms, int num_sms, cudaStream_t s) {
    const long long want = ((long long)n_rows * stride + kThreads - 1) / kThreads;
    k_terms<<<(int)(want < 8 * num_sms ? want : 8 * num_sms), kThreads, 0, s>>>(low, n_rows, rank, (bf16*)terms, stride, n_terms);
    return cudaGetLastError();
}

}  // namespace bp
