// Products of rows with the weights of their group in float32 FMAs: the expert and adapter layers
// of float32.
//
// Each kernel is a tile of 16 P x 16 P by 256 threads (P x P sums a thread) over K, through a ring of
// four steps in shared memory that cp.async fills three steps ahead.  What differs between the products
// is where an operand's element lies, which the kernels pass as functions; operands are read along
// whichever of their dimensions is contiguous, a float at a time (rows of 203 floats start on no 16-byte
// boundary).  P = 8 where there are tiles for every SM: a thread then reads 16 floats of shared memory
// for 64 FMAs, and the FMA pipe is the bound; P = 4 and 2 read two and four times as many for each, but
// cut small products into enough tiles (128 rows of 203-120 in each of 8 groups: 48 tiles of P = 4 take a
// third of the SMs).  Sums run over at most kSum values of k at a time, which are added up apart, so that
// a long sum's error stays that of short ones (65,536 rows in one chain: ten times it).
#include "bp_experts_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256;
constexpr int kSum = 512;
constexpr int kLowP = 2;   // of the products that are as narrow as an adapter's rank

constexpr int kRing = 4;
template <int P>
struct Step {
    static constexpr int T = 16 * P, K = P == 8 ? 16 : 32;
    float a[K][T + 4];
    float b[K][T + 4];
};
template <int P>
constexpr int kSmem = kRing * sizeof(Step<P>);

// total += A B^T over k in [0, K): a(m, k) and b(n, k) point at the operands' elements (NULL: 0).
// A_KFAST, B_KFAST: the operand's k is contiguous in memory.  `any`: an address that may be named.
template <int P, bool A_KFAST, bool B_KFAST, class FA, class FB>
__device__ __forceinline__ void accumulate(Step<P>* ring, float (&total)[P][P], int K, const float* any, FA a, FB b) {
    constexpr int T = Step<P>::T, TK = Step<P>::K, L = T * TK / kThreads;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, steps = (K + TK - 1) / TK;
    float acc[P][P];
    auto copy = [&](int step) {
        Step<P>& t = ring[step % kRing];
        auto one = [&](float* to, const float* from) {
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                         "l"(from != nullptr ? from : any), "r"(from != nullptr ? 4 : 0)
                         : "memory");
        };
        if (step < steps) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int e = tid + i * kThreads;
                const int ak = A_KFAST ? e % TK : e / T, am = A_KFAST ? e / TK : e % T;
                const int bk = B_KFAST ? e % TK : e / T, bn = B_KFAST ? e / TK : e % T;
                one(&t.a[ak][am], step * TK + ak < K ? a(am, step * TK + ak) : nullptr);
                one(&t.b[bk][bn], step * TK + bk < K ? b(bn, step * TK + bk) : nullptr);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
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
    __syncthreads();   // an earlier call's last step is read
    fresh();
#pragma unroll 1
    for (int i = 0; i < kRing - 1; ++i) copy(i);
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
        __syncthreads();   // step i is there for all, and step i - 1 is read
        copy(i + kRing - 1);
        const Step<P>& t = ring[i % kRing];
#pragma unroll
        for (int k = 0; k < TK; ++k) {
            float x[P], y[P];   // (tile_at)
            if constexpr (P == 2) {
                *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(&t.a[k][2 * ty]);
                *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(&t.b[k][2 * tx]);
            } else {
#pragma unroll
                for (int h = 0; h < P / 4; ++h) {
                    *reinterpret_cast<float4*>(&x[4 * h]) = *reinterpret_cast<const float4*>(&t.a[k][64 * h + 4 * ty]);
                    *reinterpret_cast<float4*>(&y[4 * h]) = *reinterpret_cast<const float4*>(&t.b[k][64 * h + 4 * tx]);
                }
            }
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int q = 0; q < P; ++q) acc[p][q] = fmaf(x[p], y[q], acc[p][q]);
        }
        if (i % (kSum / TK) == kSum / TK - 1) {
            add();
            fresh();
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    add();
}
// Row (or column) of a tile that sum i of a thread is for; w: its ty (tx).
template <int P>
__device__ __forceinline__ int tile_at(int w, int i) {
    constexpr int V = P < 4 ? P : 4;
    return 16 * V * (i / V) + V * w + i % V;
}

template <int P, bool BACK>
__global__ void __launch_bounds__(kThreads) k_rows_simt(RowsArgs g) {
    constexpr int T = Step<P>::T;
    extern __shared__ __align__(16) uint8_t smem[];
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
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
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    auto of_layer = [&] {
        auto fa = [&](int m, int k) { return m < rows ? in + (size_t)src[m] * g.K + k : nullptr; };
        if (BACK)
            accumulate<P, true, false>(t, acc, g.K, W, fa, [&](int n, int k) { return n0 + n < g.N ? W + (size_t)k * g.N + n0 + n : nullptr; });
        else
            accumulate<P, true, true>(t, acc, g.K, W, fa, [&](int n, int k) { return n0 + n < g.N ? W + (size_t)(n0 + n) * g.K + k : nullptr; });
    };
    if (g.low == nullptr) {
        of_layer();
    } else {
        const int r = g.req.rank, first = first_request(g.req, row0);
        int lo = 0, hi = 0;
        if (first < g.req.n_requests) group_rows(g.req.offsets, g.req.n_rows, first, lo, hi, g.flags);
        if (first < g.req.n_requests && lo <= row0 && hi >= row0 + rows) {   // one request: a product like the other
            const int ad = request_adapter(g.req, first, g.flags);
            if (ad >= 0) {
                const float c = g.scale != nullptr ? g.scale[ad] : 1.f;
                const float* A = (const float*)g.P + (size_t)ad * r * g.N;
                accumulate<P, true, false>(
                    t, acc, r, A, [&](int m, int k) { return m < rows ? g.low + (size_t)(row0 + m) * r + k : nullptr; },
                    [&](int n, int k) { return n0 + n < g.N ? A + (size_t)k * g.N + n0 + n : nullptr; });
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int j = 0; j < P; ++j) acc[i][j] *= c;
            }
        } else if (first < g.req.n_requests) {
            // several: each row with its own adapter's values and no others (0 times an infinity is not 0)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int m = tile_at<P>(ty, i), row = row0 + m;
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
                for (int j = 0; j < P; ++j) at[j] = min(tile_at<P>(tx, j), g.N - 1 - n0);
#pragma unroll 4
                for (int k = 0; k < r; ++k) {
                    const float u = c * low[k];
#pragma unroll
                    for (int j = 0; j < P; ++j) acc[i][j] = fmaf(u, A[(size_t)k * g.N + at[j]], acc[i][j]);
                }
            }
        }
        of_layer();
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int m = tile_at<P>(ty, i), row = row0 + m;
        if (m >= rows) continue;
        const float* x = nullptr;
        if (BACK && g.squash) x = (const float*)g.x + (size_t)source_row(g.x_source, row, g.n_x, g.flags) * g.N;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int n = n0 + tile_at<P>(tx, j);
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

// Blocks of up to 32 rows of one request.
__global__ void __launch_bounds__(kThreads) k_low_simt(LowArgs g) {
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int P = kLowP, T = Step<P>::T;
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
    __shared__ int where[3];
    const int r = g.req.rank, n0 = blockIdx.y * T, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    if (blockIdx.x == 0 && blockIdx.y == 0) zero_outside(g.req, threadIdx.x, kThreads, g.low, nullptr, r);
    if (threadIdx.x < 32) {
        int q, row0, end;
        find_tile<T>(RowGroups{g.req.offsets, g.req.n_requests, g.req.n_rows}, blockIdx.x, q, row0, end, g.flags);
        if (threadIdx.x == 0) where[0] = q, where[1] = row0, where[2] = end;
    }
    __syncthreads();
    if (where[0] < 0) return;
    const int row0 = where[1], rows = min(T, where[2] - row0), ad = request_adapter(g.req, where[0], g.flags);
    float acc[P][P] = {};
    if (ad >= 0) {
        const float *in = (const float*)g.in + (size_t)row0 * g.K, *A = (const float*)g.P + (size_t)ad * r * g.K;
        accumulate<P, true, true>(
            t, acc, g.K, A, [&](int m, int k) { return m < rows ? in + (size_t)m * g.K + k : nullptr; },
            [&](int n, int k) { return n0 + n < r ? A + (size_t)(n0 + n) * g.K + k : nullptr; });
    }
    const float c = ad >= 0 && g.scaled_low && g.scale != nullptr ? g.scale[ad] : 1.f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (tile_at<P>(ty, i) < rows && n0 + tile_at<P>(tx, j) < r)
                g.low[(size_t)(row0 + tile_at<P>(ty, i)) * r + n0 + tile_at<P>(tx, j)] = c * acc[i][j];
}

template <int P>
__device__ __forceinline__ void store_change(float* G, int M, int N, int m0, int n0, const float (&acc)[P][P], float c,
                                             int accumulate) {
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int m = m0 + tile_at<P>(ty, i), n = n0 + tile_at<P>(tx, j);
            if (m >= M || n >= N) continue;
            float* p = G + (size_t)m * N + n;
            *p = accumulate ? *p + c * acc[i][j] : c * acc[i][j];
        }
}

template <int P>
__global__ void __launch_bounds__(kThreads) k_change_simt(ChangeArgs g) {
    constexpr int T = Step<P>::T;
    extern __shared__ __align__(16) uint8_t smem[];
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
    const int e = blockIdx.z, m0 = blockIdx.y * T, n0 = blockIdx.x * T;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    const float *a = (const float*)g.a, *b = (const float*)g.b;
    float acc[P][P] = {};
    accumulate<P, false, false>(
        t, acc, hi - lo, a, [&](int m, int k) { return m0 + m < g.M ? a + (size_t)(lo + k) * g.M + m0 + m : nullptr; },
        [&](int n, int k) {
            return n0 + n < g.N ? b + (size_t)source_row(g.source, lo + k, g.n_b, g.flags) * g.N + n0 + n : nullptr;
        });
    store_change<P>(g.G + (size_t)e * g.M * g.N, g.M, g.N, m0, n0, acc, 1.f, g.accumulate);
}

__global__ void __launch_bounds__(kThreads) k_low_change_simt(LowChangeArgs g) {
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int P = kLowP, T = Step<P>::T;
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
    const int ad = blockIdx.z, m0 = blockIdx.y * T, n0 = blockIdx.x * T, r = g.req.rank;
    const float* b = (const float*)g.b;
    float acc[P][P] = {};
    for (int base = 0; base < g.req.n_requests; base += 32) {   // the adapter's requests, in order
        const int i = base + (threadIdx.x & 31);
        unsigned mine = __ballot_sync(0xffffffffu, i < g.req.n_requests && g.req.adapter[i] == ad);
        for (; mine != 0; mine &= mine - 1) {
            int lo, hi;
            group_rows(g.req.offsets, g.req.n_rows, base + __ffs(mine) - 1, lo, hi, g.flags);
            accumulate<P, false, false>(
                t, acc, hi - lo, b, [&](int m, int k) { return m0 + m < r ? g.low + (size_t)(lo + k) * r + m0 + m : nullptr; },
                [&](int n, int k) { return n0 + n < g.N ? b + (size_t)(lo + k) * g.N + n0 + n : nullptr; });
        }
    }
    store_change<P>(g.G + (size_t)ad * r * g.N, r, g.N, m0, n0, acc, g.scale != nullptr ? g.scale[ad] : 1.f, g.accumulate);
}

int blocks(long long n, int per) { return (int)((n + per - 1) / per); }

}  // namespace

template <class K>
static cudaError_t allow(K k, int bytes) {
    return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int P>
static cudaError_t setup_tile() {
    cudaError_t e;
    if ((e = allow(k_rows_simt<P, false>, kSmem<P>)) != cudaSuccess) return e;
    if ((e = allow(k_rows_simt<P, true>, kSmem<P>)) != cudaSuccess) return e;
    return allow(k_change_simt<P>, kSmem<P>);
}
cudaError_t simt_setup() {
    cudaError_t e;
    if ((e = setup_tile<2>()) != cudaSuccess) return e;
    if ((e = setup_tile<4>()) != cudaSuccess) return e;
    if ((e = setup_tile<8>()) != cudaSuccess) return e;
    if ((e = allow(k_low_simt, kSmem<kLowP>)) != cudaSuccess) return e;
    return allow(k_low_change_simt, kSmem<kLowP>);
}

// The widest tiles of which there is one for every SM.
template <class Tiles>
static int pick_tile(int num_sms, Tiles tiles) {
    return tiles(128) >= num_sms ? 8 : tiles(64) >= num_sms ? 4 : 2;
}

cudaError_t simt_rows(const RowsArgs& a, bool back, int num_sms, cudaStream_t s) {
    // the groups' sizes are on the device: taken for even
    const long long busy = a.groups.n_groups < a.groups.n_rows ? a.groups.n_groups : a.groups.n_rows;
    const int p = pick_tile(num_sms, [&](int T) { return a.groups.n_rows / T < busy && T > 64 ? 0 : busy * blocks(a.groups.n_rows, busy * T) * blocks(a.N, T); });
    const dim3 grid(max_tiles(a.groups.n_rows, a.groups.n_groups, 16 * p), blocks(a.N, 16 * p));
    auto go = [&](auto k, int bytes) { k<<<grid, kThreads, bytes, s>>>(a); };
    if (p == 8) back ? go(k_rows_simt<8, true>, kSmem<8>) : go(k_rows_simt<8, false>, kSmem<8>);
    else if (p == 4) back ? go(k_rows_simt<4, true>, kSmem<4>) : go(k_rows_simt<4, false>, kSmem<4>);
    else back ? go(k_rows_simt<2, true>, kSmem<2>) : go(k_rows_simt<2, false>, kSmem<2>);
    return cudaGetLastError();
}

cudaError_t simt_low(const LowArgs& a, cudaStream_t s) {
    const int units = max_tiles(a.req.n_rows, a.req.n_requests, 16 * kLowP);
    k_low_simt<<<dim3(units > 0 ? units : 1, blocks(a.req.rank, 16 * kLowP)), kThreads, kSmem<kLowP>, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_change(const ChangeArgs& a, int num_sms, cudaStream_t s) {
    const int p = pick_tile(num_sms, [&](int T) { return (long long)a.groups.n_groups * blocks(a.M, T) * blocks(a.N, T); });
    const dim3 grid(blocks(a.N, 16 * p), blocks(a.M, 16 * p), a.groups.n_groups);
    if (p == 8) k_change_simt<8><<<grid, kThreads, kSmem<8>, s>>>(a);
    else if (p == 4) k_change_simt<4><<<grid, kThreads, kSmem<4>, s>>>(a);
    else k_change_simt<2><<<grid, kThreads, kSmem<2>, s>>>(a);
    return cudaGetLastError();
}

cudaError_t simt_low_change(const LowChangeArgs& a, cudaStream_t s) {
    const dim3 grid(blocks(a.N, 16 * kLowP), blocks(a.req.rank, 16 * kLowP), a.req.n_adapters);
    k_low_change_simt<<<grid, kThreads, kSmem<kLowP>, s>>>(a);
    return cudaGetLastError();
}

}  // namespace bp
