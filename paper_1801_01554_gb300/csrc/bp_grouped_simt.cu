// Products of rows with the weights of their group, in float32 FMAs: the expert and adapter
// layers of float32, and of bfloat16 where no tensor-core kernel takes the call.
//
// Each kernel is a 64 x 64 tile by 256 threads (4 x 4 sums a thread) over K in steps of 16
// staged in shared memory as float32.  What differs between the products is where an operand's
// element lies, which the kernels pass as functions; operands are read along whichever of their
// dimensions is contiguous.
#include "bp_experts_device.cuh"

namespace bp {
namespace {

using bf16 = __nv_bfloat16;

constexpr int TM = 64, TN = 64, TK = 16, kThreads = 256;

struct Tile {
    float a[TK][TM + 4];
    float b[TK][TN + 4];
};

// acc += A B^T over k in [0, K): a(m, k) and b(n, k) give the operands' elements (0 outside).
// KFAST: the operand's k is contiguous in memory.
template <bool A_KFAST, bool B_KFAST, class FA, class FB>
__device__ __forceinline__ void accumulate(Tile& t, float (&acc)[4][4], int K, FA a, FB b) {
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    for (int k0 = 0; k0 < K; k0 += TK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM * TK / kThreads; ++i) {
            const int e = tid + i * kThreads;
            const int ak = A_KFAST ? e % TK : e / TM, am = A_KFAST ? e / TK : e % TM;
            const int bk = B_KFAST ? e % TK : e / TN, bn = B_KFAST ? e / TK : e % TN;
            t.a[ak][am] = k0 + ak < K ? a(am, k0 + ak) : 0.f;
            t.b[bk][bn] = k0 + bk < K ? b(bn, k0 + bk) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < TK; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(&t.a[k][4 * ty]);
            const float4 y = *reinterpret_cast<const float4*>(&t.b[k][4 * tx]);
            const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
        }
    }
}

template <class T, bool BACK>
__global__ void __launch_bounds__(kThreads) k_rows_simt(RowsArgs g) {
    __shared__ __align__(16) Tile t;
    __shared__ int where[3];
    __shared__ int src[TM];
    if (threadIdx.x < 32) {
        int e, row0, end;
        find_tile<TM>(g.groups, blockIdx.x, e, row0, end, g.flags);
        if (threadIdx.x == 0) where[0] = e, where[1] = row0, where[2] = end;
    }
    __syncthreads();
    const int e = where[0], row0 = where[1], rows = min(TM, where[2] - where[1]), n0 = blockIdx.y * TN;
    if (e < 0) return;
    if (threadIdx.x < TM)
        src[threadIdx.x] = threadIdx.x < rows ? source_row(BACK ? nullptr : g.source, row0 + threadIdx.x, g.n_in_rows, g.flags) : 0;
    __syncthreads();
    const T* in = (const T*)g.in;
    const T* W = (const T*)g.W + (size_t)e * g.N * g.K;
    float acc[4][4] = {};
    auto fa = [&](int m, int k) { return m < rows ? to_f32(in[(size_t)src[m] * g.K + k]) : 0.f; };
    if (BACK)
        accumulate<true, false>(t, acc, g.K, fa, [&](int n, int k) {
            return n0 + n < g.N ? to_f32(W[(size_t)k * g.N + n0 + n]) : 0.f;
        });
    else
        accumulate<true, true>(t, acc, g.K, fa, [&](int n, int k) {
            return n0 + n < g.N ? to_f32(W[(size_t)(n0 + n) * g.K + k]) : 0.f;
        });
    if (g.low != nullptr) {   // the requests that overlap the tile, one after another
        const int r = g.req.rank;
        for (int i = first_request(g.req, row0); i < g.req.n_requests; ++i) {
            int lo, hi;
            group_rows(g.req.offsets, g.req.n_rows, i, lo, hi, g.flags);
            if (lo >= row0 + rows) break;
            const int ad = request_adapter(g.req, i, g.flags);
            if (ad < 0 || hi <= lo) continue;
            const float c = g.scale != nullptr ? g.scale[ad] : 1.f;
            const T* P = (const T*)g.P + (size_t)ad * r * g.N;
            float part[4][4] = {};   // apart: other requests' rows must not meet this adapter's values, not times 0
            accumulate<true, false>(
                t, part, r, [&](int m, int k) { return m < rows ? c * g.low[(size_t)(row0 + m) * r + k] : 0.f; },
                [&](int n, int k) { return n0 + n < g.N ? to_f32(P[(size_t)k * g.N + n0 + n]) : 0.f; });
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int row = row0 + 4 * (threadIdx.x >> 4) + p;
                if (row >= lo && row < hi) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[p][q] += part[p][q];
                }
            }
        }
    }
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = 4 * ty + i, row = row0 + m;
        if (m >= rows) continue;
        const T* x = nullptr;
        if (BACK && g.squash) x = (const T*)g.x + (size_t)source_row(g.x_source, row, g.n_x, g.flags) * g.N;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + 4 * tx + j;
            if (n >= g.N) continue;
            float v = acc[i][j];
            if (!BACK) {
                if (g.bias != nullptr) v += g.bias[(size_t)e * g.N + n];
                if (g.squash) v = __fdividef(1.f, 1.f + expf(-v));
            } else if (g.squash) {
                const float a = to_f32(x[n]);
                v *= a * (1.f - a);
            }
            ((T*)g.out)[(size_t)row * g.N + n] = from_f32<T>(v);
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) k_low_simt(LowArgs g) {
    __shared__ __align__(16) Tile t;
    const int row0 = blockIdx.x * TM, rows = min(TM, g.req.n_rows - row0), n0 = blockIdx.y * TN, r = g.req.rank;
    const T* in = (const T*)g.in;
    float acc[4][4] = {};
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = first_request(g.req, row0); i < g.req.n_requests; ++i) {
        int lo, hi;
        group_rows(g.req.offsets, g.req.n_rows, i, lo, hi, g.flags);
        if (lo >= row0 + rows) break;
        const int ad = request_adapter(g.req, i, g.flags);
        if (ad < 0 || hi <= lo) continue;
        const float c = g.scaled_low && g.scale != nullptr ? g.scale[ad] : 1.f;
        const T* P = (const T*)g.P + (size_t)ad * r * g.K;
        float part[4][4] = {};
        accumulate<true, true>(
            t, part, g.K,
            [&](int m, int k) {
                const int row = row0 + m;
                return m < rows && row >= lo && row < hi ? to_f32(in[(size_t)row * g.K + k]) : 0.f;
            },
            [&](int n, int k) { return n0 + n < r ? to_f32(P[(size_t)(n0 + n) * g.K + k]) : 0.f; });
#pragma unroll
        for (int p = 0; p < 4; ++p) {   // a row is in one request
            const int row = row0 + 4 * ty + p;
            if (row >= lo && row < hi) {
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] = c * part[p][q];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * ty + i < rows && n0 + 4 * tx + j < r) g.low[(size_t)(row0 + 4 * ty + i) * r + n0 + 4 * tx + j] = acc[i][j];
}

__device__ __forceinline__ void store_change(float* G, int M, int N, int m0, int n0, const float (&acc)[4][4], float c,
                                             int accumulate) {
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 4 * ty + i, n = n0 + 4 * tx + j;
            if (m >= M || n >= N) continue;
            float* p = G + (size_t)m * N + n;
            *p = accumulate ? *p + c * acc[i][j] : c * acc[i][j];
        }
}

template <class T>
__global__ void __launch_bounds__(kThreads) k_change_simt(ChangeArgs g) {
    __shared__ __align__(16) Tile t;
    const int e = blockIdx.z, m0 = blockIdx.y * TM, n0 = blockIdx.x * TN;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    const T *a = (const T*)g.a, *b = (const T*)g.b;
    float acc[4][4] = {};
    accumulate<false, false>(
        t, acc, hi - lo, [&](int m, int k) { return m0 + m < g.M ? to_f32(a[(size_t)(lo + k) * g.M + m0 + m]) : 0.f; },
        [&](int n, int k) {
            return n0 + n < g.N ? to_f32(b[(size_t)source_row(g.source, lo + k, g.n_b, g.flags) * g.N + n0 + n]) : 0.f;
        });
    store_change(g.G + (size_t)e * g.M * g.N, g.M, g.N, m0, n0, acc, 1.f, g.accumulate);
}

template <class T>
__global__ void __launch_bounds__(kThreads) k_low_change_simt(LowChangeArgs g) {
    __shared__ __align__(16) Tile t;
    const int ad = blockIdx.z, m0 = blockIdx.y * TM, n0 = blockIdx.x * TN, r = g.req.rank;
    const T* b = (const T*)g.b;
    float acc[4][4] = {};
    for (int i = 0; i < g.req.n_requests; ++i) {   // the adapter's requests, in order
        if (request_adapter(g.req, i, g.flags) != ad) continue;
        int lo, hi;
        group_rows(g.req.offsets, g.req.n_rows, i, lo, hi, g.flags);
        accumulate<false, false>(
            t, acc, hi - lo, [&](int m, int k) { return m0 + m < r ? g.low[(size_t)(lo + k) * r + m0 + m] : 0.f; },
            [&](int n, int k) { return n0 + n < g.N ? to_f32(b[(size_t)(lo + k) * g.N + n0 + n]) : 0.f; });
    }
    store_change(g.G + (size_t)ad * r * g.N, r, g.N, m0, n0, acc, g.scale != nullptr ? g.scale[ad] : 1.f, g.accumulate);
}

// 32 columns by 8 slices of the group's rows; the slices are added in order.
template <class T>
__global__ void __launch_bounds__(kThreads) k_sums_simt(SumsArgs g) {
    __shared__ float part[8][32];
    const int e = blockIdx.y, c = threadIdx.x & 31, k = threadIdx.x >> 5, n = blockIdx.x * 32 + c;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    const T* d = (const T*)g.d;
    float s = 0.f;
    if (n < g.N)
        for (int r = lo + k; r < hi; r += 8) s += to_f32(d[(size_t)r * g.N + n]);
    part[k][c] = s;
    __syncthreads();
    if (k == 0 && n < g.N) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][c];
        float* p = g.S + (size_t)e * g.N + n;
        *p = g.accumulate ? *p + s : s;
    }
}

int blocks(long long n, int per) { return (int)((n + per - 1) / per); }

}  // namespace

cudaError_t simt_rows(const RowsArgs& a, int dtype, bool back, cudaStream_t s) {
    const dim3 grid(max_tiles(a.groups.n_rows, a.groups.n_groups, TM), blocks(a.N, TN));
    if (dtype == BP_F32) {
        if (back) k_rows_simt<float, true><<<grid, kThreads, 0, s>>>(a);
        else k_rows_simt<float, false><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (back) k_rows_simt<bf16, true><<<grid, kThreads, 0, s>>>(a);
        else k_rows_simt<bf16, false><<<grid, kThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t simt_low(const LowArgs& a, int dtype, cudaStream_t s) {
    const dim3 grid(blocks(a.req.n_rows, TM), blocks(a.req.rank, TN));
    if (dtype == BP_F32) k_low_simt<float><<<grid, kThreads, 0, s>>>(a);
    else k_low_simt<bf16><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_change(const ChangeArgs& a, int dtype, cudaStream_t s) {
    const dim3 grid(blocks(a.N, TN), blocks(a.M, TM), a.groups.n_groups);
    if (dtype == BP_F32) k_change_simt<float><<<grid, kThreads, 0, s>>>(a);
    else k_change_simt<bf16><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_low_change(const LowChangeArgs& a, int dtype, cudaStream_t s) {
    const dim3 grid(blocks(a.N, TN), blocks(a.req.rank, TM), a.req.n_adapters);
    if (dtype == BP_F32) k_low_change_simt<float><<<grid, kThreads, 0, s>>>(a);
    else k_low_change_simt<bf16><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_sums(const SumsArgs& a, int dtype, cudaStream_t s) {
    const dim3 grid(blocks(a.N, 32), a.groups.n_groups);
    if (dtype == BP_F32) k_sums_simt<float><<<grid, kThreads, 0, s>>>(a);
    else k_sums_simt<bf16><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace bp
