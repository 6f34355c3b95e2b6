// Products of rows with the weights of their group in float32 FMAs: the expert and adapter layers
// of float32.
//
// Each kernel is a tile of 16 P x 16 P by 256 threads (P x P sums a thread) over K, through a ring of
// four steps in shared memory that cp.async fills three steps ahead.  What differs between the products
// is where an operand's rows start, which the kernels pass as functions; an operand is copied along
// whichever of its dimensions is contiguous and kept as it lies, k by k or row by row, so that its copies
// are 16 bytes wide where rows start on 16-byte boundaries (those of 203 floats do not: 4 bytes).  P = 8
// where there are tiles for every SM: a thread then reads 16 floats of shared memory for 64 FMAs, and the
// FMA pipe is the bound; P = 4 and 2 read two and four times as many for each, but cut small products
// into enough tiles (128 rows of 203-120 in each of 8 groups: 48 tiles of P = 4 take a third of the
// SMs).  Sums run over at most kSum values of k at a time, which are added up apart, so that a long sum's
// error stays that of short ones (65,536 rows in one chain: ten times it).
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
    static constexpr int kRowPitch = K + 4, kColPitch = T + 4;   // of an operand kept by rows; by k
    static constexpr int kFloats = T * kRowPitch > K * kColPitch ? T * kRowPitch : K * kColPitch;
    float a[kFloats];
    float b[kFloats];
};
template <int P>
constexpr int kSmem = kRing * sizeof(Step<P>);

// Row (column) of a tile that sum i of a thread is for, w its ty (tx): of an operand kept by rows w + 16 i
// (a quarter warp's 16-byte reads then hit all banks), of one kept by k runs of four.
template <int P, bool KFAST>
__device__ __forceinline__ int tile_at(int w, int i) {
    constexpr int V = P < 4 ? P : 4;
    return KFAST ? w + 16 * i : 16 * V * (i / V) + V * w + i % V;
}

// One operand's part of step `step`.  KFAST: row(m) is where row m's k lie (NULL: zeros); else row(k) is
// where k's columns lie, of which `cols` are there.
template <int P, bool KFAST, bool WIDE, class F>
__device__ __forceinline__ void copy_operand(float* to, int step, int K, int cols, const float* any, F row) {
    constexpr int T = Step<P>::T, TK = Step<P>::K, V = WIDE ? 4 : 1, L = T * TK / V / kThreads;
    constexpr int kPer = (KFAST ? TK : T) / V;   // copies along the contiguous dimension
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(to);
    const int fast = threadIdx.x % kPer * V;
    const bool in = KFAST ? step * TK + fast < K : fast < cols;
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int slow = threadIdx.x / kPer + i * (kThreads / kPer);
        const float* p = nullptr;
        if (in && (KFAST || step * TK + slow < K)) p = row(KFAST ? slow : step * TK + slow);
        const uint32_t at = base + (slow * (KFAST ? Step<P>::kRowPitch : Step<P>::kColPitch) + fast) * 4;
        const float* from = p != nullptr ? p + (KFAST ? step * TK + fast : fast) : any;
        const int n = p != nullptr ? 4 * V : 0;
        if constexpr (WIDE)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(n) : "memory");
        else
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at), "l"(from), "r"(n) : "memory");
    }
}
// KN values of k of a thread's rows (columns).
template <int P, bool KFAST, int KN>
__device__ __forceinline__ void read_operand(float (&x)[KN][P], const float* t, int k, int w) {
    if constexpr (KFAST) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float4 f = *reinterpret_cast<const float4*>(t + tile_at<P, true>(w, i) * Step<P>::kRowPitch + k);
            x[0][i] = f.x, x[1][i] = f.y, x[2][i] = f.z, x[3][i] = f.w;
        }
    } else {
        constexpr int V = P < 4 ? P : 4;
#pragma unroll
        for (int j = 0; j < KN; ++j)
#pragma unroll
            for (int i = 0; i < P; i += V) {
                const float* p = t + (k + j) * Step<P>::kColPitch + tile_at<P, false>(w, i);
                if constexpr (V == 4) *reinterpret_cast<float4*>(&x[j][i]) = *reinterpret_cast<const float4*>(p);
                else *reinterpret_cast<float2*>(&x[j][i]) = *reinterpret_cast<const float2*>(p);
            }
    }
}

// total += A B^T over k in [0, K).  WIDE: both operands' rows start on 16-byte boundaries, K is a
// multiple of 4 if they are contiguous along it, their columns are if not.
template <int P, bool A_KFAST, bool B_KFAST, bool WIDE, class FA, class FB>
__device__ __forceinline__ void accumulate(Step<P>* ring, float (&total)[P][P], int K, const float* any, int a_cols, FA a,
                                           int b_cols, FB b) {
    constexpr int TK = Step<P>::K, KN = 4;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, steps = (K + TK - 1) / TK;
    float acc[P][P];
    auto copy = [&](int step) {
        if (step < steps) {
            copy_operand<P, A_KFAST, WIDE>(ring[step % kRing].a, step, K, a_cols, any, a);
            copy_operand<P, B_KFAST, WIDE>(ring[step % kRing].b, step, K, b_cols, any, b);
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
#pragma unroll(P == 8 ? 2 : 4)
        for (int k = 0; k < TK; k += KN) {
            float x[KN][P], y[KN][P];
            read_operand<P, A_KFAST, KN>(x, t.a, k, ty);
            read_operand<P, B_KFAST, KN>(y, t.b, k, tx);
#pragma unroll
            for (int j = 0; j < KN; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int q = 0; q < P; ++q) acc[p][q] = fmaf(x[j][p], y[j][q], acc[p][q]);
        }
        if (i % (kSum / TK) == kSum / TK - 1) {
            add();
            fresh();
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    add();
}

template <int P, bool BACK, bool WIDE>
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
        auto fa = [&](int m) { return m < rows ? in + (size_t)src[m] * g.K : nullptr; };
        if (BACK)
            accumulate<P, true, false, WIDE>(t, acc, g.K, W, 0, fa, g.N - n0, [&](int k) { return W + (size_t)k * g.N + n0; });
        else
            accumulate<P, true, true, WIDE>(t, acc, g.K, W, 0, fa, 0, [&](int n) { return n0 + n < g.N ? W + (size_t)(n0 + n) * g.K : nullptr; });
    };
    // this thread's rows and columns
    auto row_of = [&](int i) { return tile_at<P, true>(ty, i); };
    auto col_of = [&](int j) { return tile_at<P, !BACK>(tx, j); };
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
                float part[P][P] = {};   // by tile_at<P, false> along the columns
                accumulate<P, true, false, false>(
                    t, part, r, A, 0, [&](int m) { return m < rows ? g.low + (size_t)(row0 + m) * r : nullptr; }, g.N - n0,
                    [&](int k) { return A + (size_t)k * g.N + n0; });
                if (!BACK) {   // to the columns of the layer's product, through shared memory
                    float* turn = reinterpret_cast<float*>(smem);
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < P; ++i)
#pragma unroll
                        for (int j = 0; j < P; ++j) turn[row_of(i) * (T + 1) + tile_at<P, false>(tx, j)] = part[i][j];
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < P; ++i)
#pragma unroll
                        for (int j = 0; j < P; ++j) part[i][j] = turn[row_of(i) * (T + 1) + col_of(j)];
                }
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int j = 0; j < P; ++j) acc[i][j] = c * part[i][j];
            }
        } else if (first < g.req.n_requests) {
            // several: each row with its own adapter's values and no others (0 times an infinity is not 0)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const int m = row_of(i), row = row0 + m;
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
                for (int j = 0; j < P; ++j) at[j] = min(col_of(j), g.N - 1 - n0);
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
        const int m = row_of(i), row = row0 + m;
        if (m >= rows) continue;
        const float* x = nullptr;
        if (BACK && g.squash) x = (const float*)g.x + (size_t)source_row(g.x_source, row, g.n_x, g.flags) * g.N;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int n = n0 + col_of(j);
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
        accumulate<P, true, true, false>(
            t, acc, g.K, A, 0, [&](int m) { return m < rows ? in + (size_t)m * g.K : nullptr; }, 0,
            [&](int n) { return n0 + n < r ? A + (size_t)(n0 + n) * g.K : nullptr; });
    }
    const float c = ad >= 0 && g.scaled_low && g.scale != nullptr ? g.scale[ad] : 1.f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (tile_at<P, true>(ty, i) < rows && n0 + tile_at<P, true>(tx, j) < r)
                g.low[(size_t)(row0 + tile_at<P, true>(ty, i)) * r + n0 + tile_at<P, true>(tx, j)] = c * acc[i][j];
}

// Share z of `shares` of rows [lo, hi).
__device__ __forceinline__ void share_rows(int& lo, int& hi, int z, int shares) {
    const int per = (hi - lo + shares - 1) / shares;
    lo = min(lo + z * per, hi);
    hi = min(lo + per, hi);
}

// A tile of changes [groups][M, N] from the block's sums; with several shares they go to scratch
// [shares][groups][M, N], and the last block to arrive adds the shares' in their order.
template <int P>
__device__ __forceinline__ void store_change(const ChangeShares& s, int z, int groups, int e, float* G, int M, int N, int m0, int n0,
                                             float (&acc)[P][P], float c, int accumulate) {
    __shared__ int last;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const size_t plane = (size_t)groups * M * N;
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const int m = m0 + tile_at<P, false>(ty, i), n = n0 + tile_at<P, false>(tx, j);
                if (m < M && n < N) f(acc[i][j], ((size_t)e * M + m) * N + n);
            }
    };
    if (s.shares > 1) {
        each([&](float& x, size_t at) { s.scratch[z * plane + at] = x; });
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned* count = s.arrived + ((size_t)e * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
            last = atomicAdd(count, 1u) == (unsigned)s.shares - 1;
            if (last) *count = 0u;
        }
        __syncthreads();
        if (!last) return;
        __threadfence();
        each([&](float& x, size_t) { x = 0.f; });
        for (int k = 0; k < s.shares; ++k) each([&](float& x, size_t at) { x += __ldcg(&s.scratch[k * plane + at]); });
    }
    each([&](float& x, size_t at) { G[at] = accumulate ? G[at] + c * x : c * x; });
}

template <int P, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_change_simt(ChangeArgs g, ChangeShares sh) {
    constexpr int T = Step<P>::T;
    extern __shared__ __align__(16) uint8_t smem[];
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
    const int E = g.groups.n_groups, z = blockIdx.z / E, e = blockIdx.z - z * E, m0 = blockIdx.y * T, n0 = blockIdx.x * T;
    int lo, hi;
    group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
    share_rows(lo, hi, z, sh.shares);
    const float *a = (const float*)g.a, *b = (const float*)g.b;
    float acc[P][P] = {};
    accumulate<P, false, false, WIDE>(
        t, acc, hi - lo, a, g.M - m0, [&](int k) { return a + (size_t)(lo + k) * g.M + m0; }, g.N - n0,
        [&](int k) { return b + (size_t)source_row(g.source, lo + k, g.n_b, g.flags) * g.N + n0; });
    store_change<P>(sh, z, E, e, g.G, g.M, g.N, m0, n0, acc, 1.f, g.accumulate);
}

__global__ void __launch_bounds__(kThreads) k_low_change_simt(LowChangeArgs g, ChangeShares sh) {
    constexpr int P = kLowP, T = Step<P>::T;
    extern __shared__ __align__(16) uint8_t smem[];
    Step<P>* t = reinterpret_cast<Step<P>*>(smem);
    const int n_ad = g.req.n_adapters, z = blockIdx.z / n_ad, ad = blockIdx.z - z * n_ad;
    const int m0 = blockIdx.y * T, n0 = blockIdx.x * T, r = g.req.rank;
    const float* b = (const float*)g.b;
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)   // adapters out of range belong to no block
        for (int i = threadIdx.x; i < g.req.n_requests; i += kThreads) request_adapter(g.req, i, g.flags);
    float acc[P][P] = {};
    for (int base = 0; base < g.req.n_requests; base += 32) {   // the adapter's requests, in order
        const int i = base + (threadIdx.x & 31);
        unsigned mine = __ballot_sync(0xffffffffu, i < g.req.n_requests && g.req.adapter[i] == ad);
        for (; mine != 0; mine &= mine - 1) {
            int lo, hi;
            group_rows(g.req.offsets, g.req.n_rows, base + __ffs(mine) - 1, lo, hi, g.flags);
            share_rows(lo, hi, z, sh.shares);
            if (hi <= lo) continue;
            accumulate<P, false, false, false>(
                t, acc, hi - lo, b, r - m0, [&](int k) { return g.low + (size_t)(lo + k) * r + m0; }, g.N - n0,
                [&](int k) { return b + (size_t)(lo + k) * g.N + n0; });
        }
    }
    store_change<P>(sh, z, n_ad, ad, g.G, r, g.N, m0, n0, acc, g.scale != nullptr ? g.scale[ad] : 1.f, g.accumulate);
}

int blocks(long long n, int per) { return (int)((n + per - 1) / per); }

}  // namespace

template <class K>
static cudaError_t allow(K k, int bytes) {
    return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int P, bool WIDE>
static cudaError_t setup_tile() {
    cudaError_t e;
    if ((e = allow(k_rows_simt<P, false, WIDE>, kSmem<P>)) != cudaSuccess) return e;
    if ((e = allow(k_rows_simt<P, true, WIDE>, kSmem<P>)) != cudaSuccess) return e;
    return allow(k_change_simt<P, WIDE>, kSmem<P>);
}
cudaError_t simt_setup() {
    cudaError_t e;
    if ((e = setup_tile<2, false>()) != cudaSuccess) return e;
    if ((e = setup_tile<4, false>()) != cudaSuccess) return e;
    if ((e = setup_tile<8, false>()) != cudaSuccess) return e;
    if ((e = setup_tile<8, true>()) != cudaSuccess) return e;
    if ((e = allow(k_low_simt, kSmem<kLowP>)) != cudaSuccess) return e;
    return allow(k_low_change_simt, kSmem<kLowP>);
}

// The widest tiles of which there is one for every SM.
template <class Tiles>
static int pick_tile(int num_sms, Tiles tiles) {
    return tiles(128) >= num_sms ? 8 : tiles(64) >= num_sms ? 4 : 2;
}

// Whether both operands' rows start on 16-byte boundaries.
static bool wide(const void* a, const void* b, int a_row, int b_row) {
    return (((uintptr_t)a | (uintptr_t)b) & 15) == 0 && a_row % 4 == 0 && b_row % 4 == 0;
}

cudaError_t simt_rows(const RowsArgs& a, bool back, int num_sms, cudaStream_t s) {
    // the groups' sizes are on the device: taken for even
    const long long busy = a.groups.n_groups < a.groups.n_rows ? a.groups.n_groups : a.groups.n_rows;
    const int p = pick_tile(num_sms, [&](int T) { return a.groups.n_rows / T < busy && T > 64 ? 0 : busy * blocks(a.groups.n_rows, busy * T) * blocks(a.N, T); });
    const dim3 grid(max_tiles(a.groups.n_rows, a.groups.n_groups, 16 * p), blocks(a.N, 16 * p));
    auto go = [&](auto k, int bytes) { k<<<grid, kThreads, bytes, s>>>(a); };
    if (p == 8 && wide(a.in, a.W, a.K, back ? a.N : a.K))
        back ? go(k_rows_simt<8, true, true>, kSmem<8>) : go(k_rows_simt<8, false, true>, kSmem<8>);
    else if (p == 8) back ? go(k_rows_simt<8, true, false>, kSmem<8>) : go(k_rows_simt<8, false, false>, kSmem<8>);
    else if (p == 4) back ? go(k_rows_simt<4, true, false>, kSmem<4>) : go(k_rows_simt<4, false, false>, kSmem<4>);
    else back ? go(k_rows_simt<2, true, false>, kSmem<2>) : go(k_rows_simt<2, false, false>, kSmem<2>);
    return cudaGetLastError();
}

cudaError_t simt_low(const LowArgs& a, cudaStream_t s) {
    const int units = max_tiles(a.req.n_rows, a.req.n_requests, 16 * kLowP);
    k_low_simt<<<dim3(units > 0 ? units : 1, blocks(a.req.rank, 16 * kLowP)), kThreads, kSmem<kLowP>, s>>>(a);
    return cudaGetLastError();
}

// Shares of every group's rows: while tiles for four blocks an SM are wanting and a busy group has 128
// rows for each (the groups' sizes are on the device: taken for even).
static int change_shares(long long tiles, int groups, int busy, int n_rows, int num_sms) {
    int shares = 1;
    while (shares < 64 && tiles * groups * shares * 2 <= 4 * num_sms && n_rows / (2ll * busy * shares) >= 128) shares *= 2;
    return shares;
}
// Of any call of a layer: tiles of all shares are at most four an SM where there are several.
size_t simt_change_scratch(int groups, int least_busy, size_t cells, int max_rows, int num_sms) {
    size_t shares = 1;
    while (shares < 64 && max_rows / (2ll * least_busy * (long long)shares) >= 128) shares *= 2;
    const size_t most = (size_t)4 * num_sms * 128 * 128, all = shares * groups * cells;
    return shares == 1 ? 0 : all < most ? all : most;
}
size_t simt_change_counts(int num_sms) { return (size_t)4 * num_sms; }

cudaError_t simt_change(const ChangeArgs& a, const ChangeShares& room, int num_sms, cudaStream_t s) {
    const int E = a.groups.n_groups;
    const int p = pick_tile(num_sms, [&](int T) { return (long long)E * blocks(a.M, T) * blocks(a.N, T); }), T = 16 * p;
    ChangeShares sh = room;
    sh.shares = change_shares((long long)blocks(a.M, T) * blocks(a.N, T), E, E, a.groups.n_rows, num_sms);
    const dim3 grid(blocks(a.N, T), blocks(a.M, T), E * sh.shares);
    if (p == 8 && wide(a.a, a.b, a.M, a.N)) k_change_simt<8, true><<<grid, kThreads, kSmem<8>, s>>>(a, sh);
    else if (p == 8) k_change_simt<8, false><<<grid, kThreads, kSmem<8>, s>>>(a, sh);
    else if (p == 4) k_change_simt<4, false><<<grid, kThreads, kSmem<4>, s>>>(a, sh);
    else k_change_simt<2, false><<<grid, kThreads, kSmem<2>, s>>>(a, sh);
    return cudaGetLastError();
}

cudaError_t simt_low_change(const LowChangeArgs& a, const ChangeShares& room, int num_sms, cudaStream_t s) {
    constexpr int T = 16 * kLowP;
    const int n_ad = a.req.n_adapters, busy = a.req.n_requests < 1 ? 1 : n_ad < a.req.n_requests ? n_ad : a.req.n_requests;
    const int x = blocks(a.N, T), y = blocks(a.req.rank, T);
    ChangeShares sh = room;
    sh.shares = change_shares((long long)x * y, n_ad, busy, a.req.n_rows, num_sms);
    k_low_change_simt<<<dim3(x, y, n_ad * sh.shares), kThreads, kSmem<kLowP>, s>>>(a, sh);
    return cudaGetLastError();
}

}  // namespace bp
