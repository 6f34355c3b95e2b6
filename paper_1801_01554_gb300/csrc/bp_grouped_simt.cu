// Products of rows with the weights of their group in float32 FMAs: the expert and adapter layers
// of float32.
//
// Each kernel is a tile of 16 P x 16 P by 256 threads (P x P sums a thread) over K, staged in two
// shared-memory buffers: a step's loads are under way while the step before is multiplied.  What
// differs between the products is where an operand's element lies, which the kernels pass as
// functions; operands are read along whichever of their dimensions is contiguous, a float at a time
// (rows of 203 floats start on no 16-byte boundary).  P = 8 where there are tiles for every SM:
// a thread then reads 16 floats of shared memory for 64 FMAs, and the FMA pipe is the bound; P = 4 reads
// twice as many for each, but cuts small products into enough tiles.  Sums run over at most
// kSum values of k at a time, which are added up apart, so that a long sum's error stays that of
// short ones (65,536 rows in one chain: ten times it).
#include "bp_experts_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256;
constexpr int kSum = 512;

template <int P>
struct Tile {
    static constexpr int T = 16 * P, K = P == 8 ? 16 : 32;
    float a[2][K][T + 4];
    float b[2][K][T + 4];
};

// total += A B^T over k in [0, K): a(m, k) and b(n, k) give the operands' elements (0 outside).
// A_KFAST, B_KFAST: the operand's k is contiguous in memory.
template <int P, bool A_KFAST, bool B_KFAST, class FA, class FB>
__device__ __forceinline__ void accumulate(Tile<P>& t, float (&total)[P][P], int K, FA a, FB b) {
    constexpr int T = Tile<P>::T, TK = Tile<P>::K, L = T * TK / kThreads;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    float ra[L], rb[L], acc[P][P];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = tid + i * kThreads;
            const int ak = A_KFAST ? e % TK : e / T, am = A_KFAST ? e / TK : e % T;
            const int bk = B_KFAST ? e % TK : e / T, bn = B_KFAST ? e / TK : e % T;
            ra[i] = k0 + ak < K ? a(am, k0 + ak) : 0.f;
            rb[i] = k0 + bk < K ? b(bn, k0 + bk) : 0.f;
        }
    };
    auto store = [&](int s) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = tid + i * kThreads;
            t.a[s][A_KFAST ? e % TK : e / T][A_KFAST ? e / TK : e % T] = ra[i];
            t.b[s][B_KFAST ? e % TK : e / T][B_KFAST ? e / TK : e % T] = rb[i];
        }
    };
    auto fresh = [&] {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) acc[i][j] = 0.f;
    };
    auto add = [&] {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) total[i][j] += acc[i][j];
    };
    if (K <= 0) return;
    fresh();
    __syncthreads();   // an earlier call's last step is read
    load(0);
    store(0);
    __syncthreads();
    for (int k0 = 0, s = 0; k0 < K; k0 += TK, s ^= 1) {
        if (k0 + TK < K) load(k0 + TK);
#pragma unroll
        for (int k = 0; k < TK; ++k) {
            float x[P], y[P];   // rows and columns 4 tx .., and 64 further
#pragma unroll
            for (int h = 0; h < P / 4; ++h) {
                *reinterpret_cast<float4*>(&x[4 * h]) = *reinterpret_cast<const float4*>(&t.a[s][k][64 * h + 4 * ty]);
                *reinterpret_cast<float4*>(&y[4 * h]) = *reinterpret_cast<const float4*>(&t.b[s][k][64 * h + 4 * tx]);
            }
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < P; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
        }
        if ((k0 / TK) % (kSum / TK) == kSum / TK - 1) {
            add();
            fresh();
        }
        if (k0 + TK < K) store(s ^ 1);
        __syncthreads();
    }
    add();
}
// Row (or column) of a tile that sum i of a thread is for; w: its ty (tx).
__device__ __forceinline__ int tile_at(int w, int i) { return 64 * (i / 4) + 4 * w + i % 4; }

template <int P, bool BACK>
__global__ void __launch_bounds__(kThreads) k_rows_simt(RowsArgs g) {
    constexpr int T = Tile<P>::T;
    __shared__ __align__(16) Tile<P> t;
    __shared__ int where[3];
    __shared__ int src[T];
    if (threadIdx.x < 32) {
        int e, row0, end;
        find_tile<T>(g.groups, blockIdx.x, e, row0, end, g.flags);
        if (threadIdx.x == 0) where[0] = e, where[1] = row0, where[2] = end;
    }
    __syncthreads();
    const int e = where[0], row0 = where[1], rows = min(T, where[2] - where[1]), n0 = blockIdx.y * T;
    if (e < 0) return;
    if (threadIdx.x < T)
        src[threadIdx.x] = threadIdx.x < rows ? source_row(BACK ? nullptr : g.source, row0 + threadIdx.x, g.n_in_rows, g.flags) : 0;
    __syncthreads();
    const float* in = (const float*)g.in;
    const float* W = (const float*)g.W + (size_t)e * g.N * g.K;
    float acc[P][P] = {};
    auto fa = [&](int m, int k) { return m < rows ? in[(size_t)src[m] * g.K + k] : 0.f; };
    if (BACK)
        accumulate<P, true, false>(t, acc, g.K, fa, [&](int n, int k) { return n0 + n < g.N ? W[(size_t)k * g.N + n0 + n] : 0.f; });
    else
        accumulate<P, true, true>(t, acc, g.K, fa, [&](int n, int k) { return n0 + n < g.N ? W[(size_t)(n0 + n) * g.K + k] : 0.f; });
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    if (g.low != nullptr) {
        const int r = g.req.rank, first = first_request(g.req, row0);
        int lo = 0, hi = 0;
        if (first < g.req.n_requests) group_rows(g.req.offsets, g.req.n_rows, first, lo, hi, g.flags);
        if (first < g.req.n_requests && lo <= row0 && hi >= row0 + rows) {   // one request: a product like the other
            const int ad = request_adapter(g.req, first, g.flags);
            if (ad >= 0) {
                const float c = g.scale != nullptr ? g.scale[ad] : 1.f;
                const float* A = (const float*)g.P + (size_t)ad * r * g.N;
                accumulate<P, true, false>(
                    t, acc, r, [&](int m, int k) { return m < rows ? c * g.low[(size_t)(row0 + m) * r + k] : 0.f; },
                    [&](int n, int k) { return n0 + n < g.N ? A[(size_t)k * g.N + n0 + n] : 0.f; });
            }
        } else if (first < g.req.n_requests) {
            // several: each row with its own adapter's values and no others (0 times an infinity is not 0)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int m = tile_at(ty, i), row = row0 + m;
                if (m >= rows) continue;
                const int q = first_request(g.req, row);
                if (q >= g.req.n_requests) continue;
                group_rows(g.req.offsets, g.req.n_rows, q, lo, hi, g.flags);
                const int ad = row >= lo && row < hi ? request_adapter(g.req, q, g.flags) : -1;
                if (ad < 0) continue;
                const float c = g.scale != nullptr ? g.scale[ad] : 1.f;
                const float *low = g.low + (size_t)row * r, *A = (const float*)g.P + (size_t)ad * r * g.N + n0;
                int at[P];   // columns past the last one read the last one
#pragma unroll
                for (int j = 0; j < P; ++j) at[j] = min(tile_at(tx, j), g.N - 1 - n0);
#pragma unroll 4
                for (int k = 0; k < r; ++k) {
                    const float u = c * low[k];
#pragma unroll
                    for (int j = 0; j < P; ++j) acc[i][j] = fmaf(u, A[(size_t)k * g.N + at[j]], acc[i][j]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int m = tile_at(ty, i), row = row0 + m;
        if (m >= rows) continue;
        const float* x = nullptr;
        if (BACK && g.squash) x = (const float*)g.x + (size_t)source_row(g.x_source, row, g.n_x, g.flags) * g.N;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int n = n0 + tile_at(tx, j);
            if (n >= g.N) continue;
            float v = acc[i][j];
            if (!BACK) {
                if (g.bias != nullptr) v += g.bias[(size_t)e * g.N + n];
                if (g.squash) v = __fdividef(1.f, 1.f + expf(-v));
            } else if (g.squash) {
                v *= x[n] * (1.f - x[n]);
            }
            ((float*)g.out)[(size_t)row * g.N + n] = v;
        }
    }
}

// Blocks of up to 64 rows of one request.
__global__ void __launch_bounds__(kThreads) k_low_simt(LowArgs g) {
    __shared__ __align__(16) Tile<4> t;
    __shared__ int where[3];
    const int r = g.req.rank, n0 = blockIdx.y * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    if (blockIdx.x == 0 && blockIdx.y == 0) zero_outside(g.req, threadIdx.x, kThreads, g.low, nullptr, r);
    if (threadIdx.x < 32) {
        int q, row0, end;
        find_tile<64>(RowGroups{g.req.offsets, g.req.n_requests, g.req.n_rows}, blockIdx.x, q, row0, end, g.flags);
        if (threadIdx.x == 0) where[0] = q, where[1] = row0, where[2] = end;
    }
    __syncthreads();
    if (where[0] < 0) return;
    const int row0 = where[1], rows = min(64, where[2] - row0), ad = request_adapter(g.req, where[0], g.flags);
    float acc[4][4] = {};
    if (ad >= 0) {
        const float *in = (const float*)g.in + (size_t)row0 * g.K, *A = (const float*)g.P + (size_t)ad * r * g.K;
        accumulate<4, true, true>(
            t, acc, g.K, [&](int m, int k) { return m < rows ? in[(size_t)m * g.K + k] : 0.f; },
            [&](int n, int k) { return n0 + n < r ? A[(size_t)(n0 + n) * g.K + k] : 0.f; });
    }
    const float c = ad >= 0 && g.scaled_low && g.scale != nullptr ? g.scale[ad] : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (tile_at(ty, i) < rows && n0 + tile_at(tx, j) < r)
                g.low[(size_t)(row0 + tile_at(ty, i)) * r + n0 + tile_at(tx, j)] = c * acc[i][j];
}

template <int P>
__device__ __forceinline__ void store_change(float* G, int M, int N, int m0, int n0, const float (&acc)[P][P], float c,
                                             int accumulate) {
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int m = m0 + tile_at(ty, i), n = n0 + tile_at(tx, j);
            if (m >= M || n >= N) continue;
            float* p = G + (size_t)m * N + n;
            *p = accumulate ? *p + c * acc[i][j] : c * acc[i][j];
        }
}

template <int P>
__global__ void __launch_bounds__(kThreads) k_change_simt(ChangeArgs g) {
    constexpr int T = Tile<P>::T;
    __shared__ __align__(16) Tile<P> t;
    const int e = blockIdx.z, m0 = blockIdx.y * T, n0 = blockIdx.x * T;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    const float *a = (const float*)g.a, *b = (const float*)g.b;
    float acc[P][P] = {};
    accumulate<P, false, false>(
        t, acc, hi - lo, [&](int m, int k) { return m0 + m < g.M ? a[(size_t)(lo + k) * g.M + m0 + m] : 0.f; },
        [&](int n, int k) {
            return n0 + n < g.N ? b[(size_t)source_row(g.source, lo + k, g.n_b, g.flags) * g.N + n0 + n] : 0.f;
        });
    store_change<P>(g.G + (size_t)e * g.M * g.N, g.M, g.N, m0, n0, acc, 1.f, g.accumulate);
}

__global__ void __launch_bounds__(kThreads) k_low_change_simt(LowChangeArgs g) {
    __shared__ __align__(16) Tile<4> t;
    const int ad = blockIdx.z, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, r = g.req.rank;
    const float* b = (const float*)g.b;
    float acc[4][4] = {};
    for (int base = 0; base < g.req.n_requests; base += 32) {   // the adapter's requests, in order
        const int i = base + (threadIdx.x & 31);
        unsigned mine = __ballot_sync(0xffffffffu, i < g.req.n_requests && g.req.adapter[i] == ad);
        for (; mine != 0; mine &= mine - 1) {
            int lo, hi;
            group_rows(g.req.offsets, g.req.n_rows, base + __ffs(mine) - 1, lo, hi, g.flags);
            accumulate<4, false, false>(
                t, acc, hi - lo, [&](int m, int k) { return m0 + m < r ? g.low[(size_t)(lo + k) * r + m0 + m] : 0.f; },
                [&](int n, int k) { return n0 + n < g.N ? b[(size_t)(lo + k) * g.N + n0 + n] : 0.f; });
        }
    }
    store_change<4>(g.G + (size_t)ad * r * g.N, r, g.N, m0, n0, acc, g.scale != nullptr ? g.scale[ad] : 1.f, g.accumulate);
}

int blocks(long long n, int per) { return (int)((n + per - 1) / per); }

}  // namespace

cudaError_t simt_rows(const RowsArgs& a, bool back, int num_sms, cudaStream_t s) {
    // the groups' sizes are on the device: full tiles are what they make if all are as large
    const long long busy = a.groups.n_groups < a.groups.n_rows ? a.groups.n_groups : a.groups.n_rows;
    const bool large = busy * blocks(a.groups.n_rows, busy * 128) * blocks(a.N, 128) >= num_sms && a.groups.n_rows >= 64 * busy;
    const int T = large ? 128 : 64;
    const dim3 grid(max_tiles(a.groups.n_rows, a.groups.n_groups, T), blocks(a.N, T));
    if (large) {
        if (back) k_rows_simt<8, true><<<grid, kThreads, 0, s>>>(a);
        else k_rows_simt<8, false><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (back) k_rows_simt<4, true><<<grid, kThreads, 0, s>>>(a);
        else k_rows_simt<4, false><<<grid, kThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t simt_low(const LowArgs& a, cudaStream_t s) {
    const int units = max_tiles(a.req.n_rows, a.req.n_requests, 64);
    k_low_simt<<<dim3(units > 0 ? units : 1, blocks(a.req.rank, 64)), kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_change(const ChangeArgs& a, int num_sms, cudaStream_t s) {
    const bool large = (long long)a.groups.n_groups * blocks(a.M, 128) * blocks(a.N, 128) >= num_sms;
    const int T = large ? 128 : 64;
    const dim3 grid(blocks(a.N, T), blocks(a.M, T), a.groups.n_groups);
    if (large) k_change_simt<8><<<grid, kThreads, 0, s>>>(a);
    else k_change_simt<4><<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_low_change(const LowChangeArgs& a, cudaStream_t s) {
    const dim3 grid(blocks(a.N, 64), blocks(a.req.rank, 64), a.req.n_adapters);
    k_low_change_simt<<<grid, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace bp
