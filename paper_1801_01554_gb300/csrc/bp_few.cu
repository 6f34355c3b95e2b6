// The forward product of a few rows with bfloat16 weights: single patterns through their experts,
// single rows of many requests through a shared layer and their adapters.
//
// The time is that of reading the weights once: five patterns of two experts each of 1024-2048 read
// 42 MB, 6.3 us at the measured copy rate.  So the weights are streamed into mma.sync, 16 units by
// 32 of K a step and warp, 16 bytes a lane (direct_products); the rows, which every CTA reads again,
// come from L2.  Eight warps share K, their sums are added in
// shared memory in order, and eight units of a row leave as one 16-byte store.
//
// Behind an adapter's low-rank product the launch is a dependent one that streams the weights while
// that product runs, and waits for it before it reads low.
#include "bp_experts_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kWarps = 8;
// Beside the warps that stream, one that looks up the rows' adapters.
constexpr int few_threads(bool low) { return 32 * (kWarps + (low ? 1 : 0)); }

// Steps under way where they go through shared memory.
constexpr int kRing = 4;
template <int MU, int NT>
constexpr bool kThroughRing = MU * NT > 2;
template <int MU, int NT>
constexpr int few_smem() {
    constexpr int ring = kThroughRing<MU, NT> ? kWarps * ring_bytes<MU, NT, kRing>() : 0, sums = kWarps * 8 * NT * (16 * MU + 4) * 4;
    return ring > sums ? ring : sums;
}

// The slot-th group that has rows, by a converged warp; false if there are not so many.
__device__ __forceinline__ bool busy_group(const RowGroups& q, int slot, int& g, int& lo, int& hi, int* flags) {
    const int lane = threadIdx.x & 31;
    for (int base = 0; base < q.n_groups; base += 32) {
        int l = 0, h = 0;
        if (base + lane < q.n_groups) group_rows(q.offsets, q.n_rows, base + lane, l, h, flags);
        unsigned m = __ballot_sync(0xffffffffu, h > l);
        if (slot < __popc(m)) {
            for (; slot > 0; --slot) m &= m - 1;
            const int at = __ffs(m) - 1;
            g = base + at;
            lo = __shfl_sync(0xffffffffu, l, at);
            hi = __shfl_sync(0xffffffffu, h, at);
            return true;
        }
        slot -= __popc(m);
    }
    return false;
}

// MU tiles of 16 units by NT of 8 rows a pass.  LOW: one group of all rows, the adapters' part added.
template <int MU, int NT, bool LOW>
__global__ void __launch_bounds__(few_threads(LOW)) k_few(RowsArgs a) {
    constexpr int U = 16 * MU, R = 8 * NT, kThreads = few_threads(LOW);
    extern __shared__ __align__(16) uint8_t smem[];   // the warps' rings; then their sums [kWarps][R][U + 4]
    float* red = reinterpret_cast<float*>(smem);
    __shared__ int s_adapter[R];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, k8 = (lane & 3) * 8;
    int g = 0, lo = 0, hi = a.groups.n_rows;
    if (!LOW && !busy_group(a.groups, blockIdx.y, g, lo, hi, a.flags)) return;
    const int u0 = blockIdx.x * U, K = a.K, N = a.N;
    const bf16* W = (const bf16*)a.W + ((size_t)g * N + u0) * K;
    const bf16* X = (const bf16*)a.in;
    for (int row0 = lo; row0 < hi; row0 += R) {
        __syncthreads();   // the pass before has read red
        float acc[MU][NT][4] = {};
        if (!LOW || warp < kWarps) {
            const bf16 *x[NT], *w[MU][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int row = row0 + 8 * n + gr;
                x[n] = row < hi ? X + (size_t)source_row(a.source, row, a.n_in_rows, a.flags) * K + k8 : nullptr;
            }
#pragma unroll
            for (int m = 0; m < MU; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int u = 16 * m + 8 * h + gr;
                    w[m][h] = u0 + u < N ? W + (size_t)u * K + k8 : nullptr;
                }
            if constexpr (kThroughRing<MU, NT>)
                ring_products<MU, NT, kRing>(acc, w, x, W, K, warp, kWarps, smem + warp * ring_bytes<MU, NT, kRing>());
            else
                direct_products<MU, NT, 8>(acc, w, x, W, K, warp, kWarps);
        } else {
            for (int i = lane; i < R; i += 32) {
                int ad = -1;
                const int row = row0 + i, q = row < hi ? first_request(a.req, row) : a.req.n_requests;
                if (q < a.req.n_requests) {
                    int l, h;
                    group_rows(a.req.offsets, a.req.n_rows, q, l, h, a.flags);
                    if (row >= l && row < h) ad = request_adapter(a.req, q, a.flags);
                }
                s_adapter[i] = ad;
            }
        }
        __syncthreads();   // every warp is done with its ring
        if (!LOW || warp < kWarps) {
#pragma unroll
            for (int m = 0; m < MU; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int u = 16 * m + gr + 8 * (i >> 1), row = 8 * n + 2 * (lane & 3) + (i & 1);
                        red[(warp * R + row) * (U + 4) + u] = acc[m][n][i];
                    }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < R * U / 8; i += kThreads) {   // eight units of a row
            const int row = row0 + i / (U / 8), u = i % (U / 8) * 8, n = u0 + u;
            if (row >= hi || n >= N) continue;   // N is a multiple of 8
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4* p = reinterpret_cast<const float4*>(&red[(w * R + row - row0) * (U + 4) + u]);
                const float4 p0 = p[0], p1 = p[1];
                v[0] += p0.x, v[1] += p0.y, v[2] += p0.z, v[3] += p0.w;
                v[4] += p1.x, v[5] += p1.y, v[6] += p1.z, v[7] += p1.w;
            }
            if (LOW) {
                const int ad = s_adapter[row - row0], r = a.req.rank;
                const bf16* P = (const bf16*)a.P + (size_t)max(ad, 0) * r * N + n;
                constexpr int B = 8;   // the first of the adapter's rows arrive while low is waited for
                uint4 p[B];
#pragma unroll
                for (int j = 0; j < B; ++j)
                    p[j] = ad >= 0 && j < r ? *reinterpret_cast<const uint4*>(P + (size_t)j * N) : make_uint4(0u, 0u, 0u, 0u);
                pdl_wait();
                if (ad >= 0) {
                    const float c = a.scale != nullptr ? a.scale[ad] : 1.f;
                    const float* low = a.low + (size_t)row * r;
                    float s[8] = {};
                    for (int j0 = 0; j0 < r; j0 += B) {
                        uint4 now[B];
                        float t[B];
#pragma unroll
                        for (int j = 0; j < B; ++j) {
                            now[j] = p[j];
                            t[j] = j0 + j < r ? low[j0 + j] : 0.f;
                            if (j0 + B + j < r) p[j] = *reinterpret_cast<const uint4*>(P + (size_t)(j0 + B + j) * N);
                        }
#pragma unroll
                        for (int j = 0; j < B; ++j) {
                            if (j0 + j >= r) break;
                            const uint32_t pw[4] = {now[j].x, now[j].y, now[j].z, now[j].w};
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                s[2 * q] = fmaf(t[j], __uint_as_float(pw[q] << 16), s[2 * q]);
                                s[2 * q + 1] = fmaf(t[j], __uint_as_float(pw[q] & 0xffff0000u), s[2 * q + 1]);
                            }
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = fmaf(c, s[q], v[q]);
                }
            }
            if (a.bias != nullptr) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] += a.bias[(size_t)g * N + n + q];
            }
            if (a.squash) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = sigmoid_fast(v[q]);
            }
            __align__(16) __nv_bfloat162 o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = __floats2bfloat162_rn(v[2 * q], v[2 * q + 1]);
            *reinterpret_cast<uint4*>((bf16*)a.out + (size_t)row * N + n) = *reinterpret_cast<const uint4*>(o);
        }
    }
}

template <int MU, int NT, bool LOW>
cudaError_t launch(const RowsArgs& a, int slots, cudaStream_t s) {
    const dim3 grid((a.N + 16 * MU - 1) / (16 * MU), slots);
    constexpr int threads = few_threads(LOW), smem = few_smem<MU, NT>();
    if (LOW) return launch_pdl(k_few<MU, NT, LOW>, grid.x, 1, threads, smem, s, a);
    k_few<MU, NT, LOW><<<grid, threads, smem, s>>>(a);
    return cudaGetLastError();
}

template <int MU, int NT, bool LOW>
cudaError_t setup() {
    return cudaFuncSetAttribute(k_few<MU, NT, LOW>, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem<MU, NT>());
}

}  // namespace

cudaError_t few_setup() {
    cudaError_t e;
    if ((e = setup<1, 1, false>()) != cudaSuccess) return e;
    if ((e = setup<1, 2, false>()) != cudaSuccess) return e;
    if ((e = setup<1, 1, true>()) != cudaSuccess) return e;
    if ((e = setup<1, 2, true>()) != cudaSuccess) return e;
    if ((e = setup<2, 4, true>()) != cudaSuccess) return e;
    return setup<2, 8, true>();
}

// A warp's sum is one chain of mma.sync, which truncates: up to 128 steps of 16 of K, as in a part of the
// tcgen05 products.
static bool few_sums(int K) { return K <= 128 * 16 * kWarps; }

bool few_with_adapters(int n_rows, int K) { return n_rows <= 64 && few_sums(K); }

// us of the experts' forward here / on tcgen05, weights from DRAM: 8 rows of 1024-1024 of 16 experts 12.0 /
// 13.3, of 4096-4096 63.1 / 63.4; 12 of 1024-2048 of 16 16.4 / 18.4 (their 29 MB in L2: 10 of them 9.6 /
// 12.4), 16 of 2048-2048 of 16 32.8 / 28.7; 32 of 512-512 of 8 8.2 / 10.2, of 4096-256 18.4 / 26.6, of
// 1024-2048 20.5 / 16.2; 48 of 2048-2048 of 16 51 / 37; 512 of 512-512 in one of 128 76 / 16 (16 rows a
// pass: larger groups read their weights again); 64 of 4096-256 of 16 20.5 / 26.6.  So: up to 8 rows; to 16
// where their experts' weights may lie in L2; to 32 or 64 where their units are so few that tcgen05 tiles leave
// SMs idle; of one expert up to two passes (32 of 4096-4096 30.7 / 34.8, 64 51 / 35).
bool few_experts(int n_rows, int n_groups, int N, int K) {
    if (!few_sums(K)) return false;
    if (n_groups == 1) return n_rows <= 32;
    const int busy = n_groups < n_rows ? n_groups : n_rows;   // at most: their sizes are on the device
    const long long units = (long long)busy * N;
    return n_rows <= 4 * busy && (n_rows <= 8 || (n_rows <= 16 && units * K <= 1 << 25) || (n_rows <= 32 && units <= 8192) ||
                                  (n_rows <= 64 && units <= 4096));
}

}  // namespace bp

// What few_experts says, for tests.
extern "C" int bp_internal_few_experts(int n_rows, int n_experts, int n_in, int n_out) {
    return bp::few_experts(n_rows, n_experts, n_out, n_in) ? 1 : 0;
}

namespace bp {

cudaError_t few_rows(const RowsArgs& a, cudaStream_t s) {
    const int n = a.groups.n_rows;
    if (a.low != nullptr) {
        if (n <= 8) return launch<1, 1, true>(a, 1, s);
        if (n <= 16) return launch<1, 2, true>(a, 1, s);
        if (n <= 32) return launch<2, 4, true>(a, 1, s);
        return launch<2, 8, true>(a, 1, s);
    }
    const int slots = a.groups.n_groups < n ? a.groups.n_groups : n;
    return n <= 8 ? launch<1, 1, false>(a, slots, s) : launch<1, 2, false>(a, slots, s);
}

}  // namespace bp
