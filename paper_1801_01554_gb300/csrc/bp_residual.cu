// The stream between blocks: a block's output is normed, gated, scaled and added, and the sum is normed again; with the
// gradients.  Rows are independent but for the sums of the weights' and gates' gradients.
#include "bp_blocks_internal.h"
#include "bp_pieces.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {
constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32;   // of a worker
constexpr int kSums = 16;        // of the reductions between two barriers, at most
constexpr int kRed = 32 * kSums;
// Warps of a block, one block an SM: as many as its registers are enough for (64, 80 or 128 a thread).
constexpr int block_warps(bool back, bool mean, int v, int c) { return back || v * c > 8 || (mean && c > 1) ? 16 : mean ? 24 : 32; }
constexpr int kWorkerRows = 4;   // the backward pass has a worker for every so many rows, up to the device's: their sums by column are joined at the end
// Rows whose sums by column are added up in registers; then they go on to float64 sums.  (A worker may have millions of rows: 3,290 equal
// ones in one float32 sum were off by 3e-5, as every addition rounds the same way.  300,000 rows of 1,024 bfloat16 units take 585 us going
// back, 572 without float64 sums; calls of fewer rows a worker reach none.)
constexpr int kRunRows = 128;

// A worker is `warps` warps that take a row at a time, a thread C pieces of V columns; a block has one or more.
// (With narrow rows a worker is a warp, whose reductions need no barrier.)
struct Worker {
    int id, warps, tid, threads;   // id: in the block
    float* red;
    __device__ __forceinline__ Worker(int warps_, float* shared) : warps(warps_) {
        threads = warps * 32;
        id = threadIdx.x / threads;
        tid = threadIdx.x - id * threads;
        red = shared + id * warps * kSums;
    }
    __device__ __forceinline__ void sync() const {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(threads) : "memory");
    }
};

// Sums of the worker's N values, in one order, in every thread: each warp gives its part before the worker's barrier,
// and takes the sums after it.  (Two places, used in turn, so that one barrier a reduction is enough.)  A step that
// halves the lanes of a sum also halves the sums of a lane (M, N rounded up to a power of two, to one), which takes M + 4
// shuffles and as many to hand them out, not 5 N.
template <int N>
struct Sums {
    static constexpr int M = N <= 1 ? 1 : N <= 4 ? 4 : 16, L = 32 / M;   // lanes of a sum, in the end
    static_assert(N <= M && M <= kSums, "");
    float* at;
    int turn = 0;
    float mine = 0.f;
    __device__ __forceinline__ explicit Sums(const Worker& w, int place = 0) : at(w.red + place * w.warps) {}
    __device__ __forceinline__ void give(const float (&v)[N], const Worker& w) {
        const int lane = threadIdx.x & 31;
        float x[M];
#pragma unroll
        for (int i = 0; i < M; ++i) x[i] = i < N ? v[i < N ? i : 0] : 0.f;
#pragma unroll
        for (int h = M / 2, bit = 16; h >= 1; h /= 2, bit /= 2) {
            const bool upper = lane & bit;
#pragma unroll
            for (int i = 0; i < h; ++i) {
                const float send = upper ? x[i] : x[i + h], keep = upper ? x[i + h] : x[i];
                x[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
            }
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
        if (w.warps > 1) {
            if (lane % L == 0) at[turn * kRed + (w.tid >> 5) * M + lane / L] = x[0];
        } else {
            mine = x[0];
        }
    }
    __device__ __forceinline__ void take(float (&v)[N], const Worker& w) {
        const int lane = threadIdx.x & 31;
        float x = mine;
        if (w.warps > 1) {
            x = 0.f;
            for (int i = lane % L; i < w.warps; i += L) x += at[turn * kRed + i * M + lane / L];
#pragma unroll
            for (int o = (L < kMaxWarps ? L : kMaxWarps) / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            turn ^= 1;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, x, i * L);
    }
};

// Two float32 operations an instruction, over a thread's P values (one at a time where P is 1).
__device__ __forceinline__ unsigned long long pair(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(unsigned long long x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ unsigned long long fma_pair(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long mul_pair(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// One value for all places, or a value each.
struct Same {
    float x;
    __device__ __forceinline__ float operator[](int) const { return x; }
};
template <int P, class A, class B>
__device__ __forceinline__ void mul(float (&d)[P], const A& a, const B& b) {
    if constexpr (P == 1) d[0] = a[0] * b[0];
    else
#pragma unroll
        for (int i = 0; i < P; i += 2) unpair(mul_pair(pair(a[i], a[i + 1]), pair(b[i], b[i + 1])), d[i], d[i + 1]);
}
template <int P, class A, class B, class D>
__device__ __forceinline__ void fma(float (&d)[P], const A& a, const B& b, const D& c) {
    if constexpr (P == 1) d[0] = fmaf(a[0], b[0], c[0]);
    else
#pragma unroll
        for (int i = 0; i < P; i += 2)
            unpair(fma_pair(pair(a[i], a[i + 1]), pair(b[i], b[i + 1]), pair(c[i], c[i + 1])), d[i], d[i + 1]);
}
template <int P>
__device__ __forceinline__ void sub(float (&d)[P], const float (&a)[P], float b) {   // a - b, exact where a times 1 is
    fma(d, a, Same{1.f}, Same{-b});
}
template <int P, class A>
__device__ __forceinline__ float dot(const A& a, const float (&b)[P]) {
    if constexpr (P == 1) return a[0] * b[0];
    else {
        unsigned long long s = mul_pair(pair(a[0], a[1]), pair(b[0], b[1]));
#pragma unroll
        for (int i = 2; i < P; i += 2) s = fma_pair(pair(a[i], a[i + 1]), pair(b[i], b[i + 1]), s);
        float x, y;
        unpair(s, x, y);
        return x + y;
    }
}

// A thread's columns: C pieces of V, the worker's width apart.
template <int V, int C>
struct Columns {
    int width, tid, threads;
    __device__ __forceinline__ Columns(int width_, const Worker& w) : width(width_), tid(w.tid), threads(w.threads) {}
    __device__ __forceinline__ int at(int j) const { return (j * threads + tid) * V; }
    __device__ __forceinline__ bool in(int j) const { return at(j) < width; }
};

// A value a column; 0 past the row's end, which keeps what is there out of every sum.
template <int V, int C>
__device__ __forceinline__ void load_floats(const Columns<V, C>& cols, const float* p, float none, float (&out)[V * C]) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) out[j * V + i] = !cols.in(j) ? 0.f : p != nullptr ? __ldg(p + cols.at(j) + i) : none;
}
template <class T, int V, int C>
__device__ __forceinline__ void values(const Piece<T, V> (&p)[C], float (&out)[V * C]) {
#pragma unroll
    for (int j = 0; j < C; ++j) {
        float x[V];
        p[j].values(x);
#pragma unroll
        for (int i = 0; i < V; ++i) out[j * V + i] = x[i];
    }
}
template <class T, int V, int C>
__device__ __forceinline__ void round_to(const float (&x)[V * C], Piece<T, V> (&p)[C]) {
#pragma unroll
    for (int j = 0; j < C; ++j) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = x[j * V + i];
        p[j].set(y);
    }
}
template <class T, int V, int C, int M>
__device__ __forceinline__ void store_row(const Columns<V, C>& cols, const Piece<T, V> (&p)[M], T* to, int j0 = 0) {
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (cols.in(j0 + i)) p[i].store(to + (j0 + i) * cols.threads * V);
}

// Rows on their way: S rows of N arrays, each thread's pieces in places of its own in shared memory, so that a thread
// waits for its own copies alone.
template <class T, int V, int C, int N, int S>
struct Ring {
    static constexpr int kBytes = V * (int)sizeof(T);
    unsigned base;
    int lanes;
    __device__ __forceinline__ Ring(const void* shared) : base(smem_u32(shared) + threadIdx.x * kBytes), lanes(blockDim.x * kBytes) {}
    __device__ __forceinline__ unsigned place(unsigned slot, int n, int j) const { return slot + (n * C + j) * lanes; }
    __device__ __forceinline__ void step(unsigned& slot) const {
        slot += N * C * lanes;
        if (slot == base + S * N * C * lanes) slot = base;
    }
    // Pieces of array n from p on.
    __device__ __forceinline__ void ask(const Columns<V, C>& cols, const T* p, unsigned slot, int n) const {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!cols.in(j)) continue;
            const T* from = p + j * cols.threads * V;
            if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place(slot, n, j)), "l"(from) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(place(slot, n, j)), "l"(from) : "memory");
        }
    }
    __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ static void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory"); }   // for the first of S rows
    // The row's pieces from the j0-th on; zeros for an array that is not there and past the row's end.
    template <int M>
    __device__ __forceinline__ void take(const Columns<V, C>& cols, bool there, unsigned slot, int n, Piece<T, V> (&out)[M], int j0 = 0) const {
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const int j = j0 + i;
            out[i].u = make_uint4(0u, 0u, 0u, 0u);
            if (!there || !cols.in(j)) continue;
            uint4& u = out[i].u;
            if constexpr (kBytes == 16)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(place(slot, n, j)) : "memory");
            else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(u.x) : "r"(place(slot, n, j)) : "memory");
        }
    }
};
// Stages.  Three rows are enough to keep the memory busy (16,384 rows of 4,096 bfloat16 units, forward: 2 stages 100.0 us,
// 3 98.5, 6 as 4: what more of them take from the L1 cache is missed); what fits beside wide rows' weights going back.
template <class T, int V, int C>
constexpr int stages(bool back) {
    constexpr int bytes = V * C * (int)sizeof(T);
    return back && V * C >= 16 ? (bytes <= 32 ? 2 : 1) : 3;
}
// Shared memory of a thread: the stages, and going back the weights of 16 values.
template <class T, int V, int C>
constexpr int thread_bytes(bool back) {
    return stages<T, V, C>(back) * (back ? 4 : 2) * C * V * (int)sizeof(T) + (back && V * C >= 16 ? 2 * V * C * 4 : 0);
}

// Rows that share a row of gates: of row r, the gates' row (-1: none) and the first row from r on that is not of it.
struct Stretch {
    int seg, end;
};
__device__ __forceinline__ Stretch stretch_of(const ResidualArgs& g, int r) {
    if (g.offsets == nullptr || g.n_gates == 0) return {0, g.n};
    int lo = 0, hi = g.n_gates;
    while (lo < hi) {   // the first range that ends after r
        const int mid = (lo + hi) >> 1;
        if (__ldg(g.offsets + mid + 1) > r) hi = mid;
        else lo = mid + 1;
    }
    if (lo == g.n_gates) return {-1, g.n};
    const int first = __ldg(g.offsets + lo);
    if (first > r) return {-1, min(first, g.n)};
    return {lo, min(__ldg(g.offsets + lo + 1), g.n)};
}
__device__ __forceinline__ void check_offsets(const ResidualArgs& g) {
    if (g.offsets == nullptr || g.n_gates == 0) return;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i <= g.n_gates; i += (long long)gridDim.x * blockDim.x) {
        const int x = __ldg(g.offsets + i), y = i < g.n_gates ? __ldg(g.offsets + i + 1) : g.n;
        if (x < 0 || x > y || y > g.n) atomicOr(g.flags, kFlagBounds);
    }
}
__device__ __forceinline__ int first_row(const ResidualArgs& g, int worker) { return (int)((long long)g.n * worker / g.workers); }

// scale * gate of a stretch, by column.
template <int V, int C>
__device__ __forceinline__ void load_gate(const ResidualArgs& g, const Columns<V, C>& cols, int seg, float (&k)[V * C]) {
    load_floats(cols, g.n_gates > 0 && seg >= 0 ? g.gate + (size_t)seg * g.width : nullptr, seg < 0 ? 0.f : 1.f, k);
#pragma unroll
    for (int i = 0; i < V * C; ++i) k[i] *= g.scale;
}

// Mean and 1 / sqrt of a row, in the same two steps as Sums.  MEAN: each warp's mean first and the squared differences from it,
// then the warps' means and differences from theirs, so that nothing cancels where the mean is far from 0.
template <bool MEAN, int V, int C>
struct NormStats {
    Sums<1> sums;
    float* at;
    int turn = 0;
    float mean_w = 0.f, m2_w = 0.f;        // of this warp
    float values_w = 0.f, each_w = 0.f;    // how many values it has, and one over that
    __device__ __forceinline__ NormStats(const Worker& w, int place, int width) : sums(w, place), at(w.red + place * w.warps) {
        if constexpr (MEAN) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < C; ++j) n += max(0, min(32 * V, width - (j * w.threads + (w.tid & ~31)) * V));
            values_w = (float)n;
            each_w = n > 0 ? 1.f / values_w : 0.f;
        }
    }
    __device__ __forceinline__ static float warp_sum(float x, int lanes) {
        for (int o = lanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        return x;
    }
    __device__ __forceinline__ void give(const Columns<V, C>& cols, const float (&v)[V * C], const Worker& w) {
        if constexpr (MEAN) {
            const float s = dot(Same{1.f}, v);   // (columns past the row's end are 0)
            mean_w = warp_sum(s, 32) * each_w;
            float d[V * C];
            sub(d, v, mean_w);
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (!cols.in(j))
#pragma unroll
                    for (int i = 0; i < V; ++i) d[j * V + i] = 0.f;
            m2_w = warp_sum(dot(d, d), 32);
            float* to = at + turn * kRed + (w.tid >> 5) * 4;
            if (w.warps > 1 && (threadIdx.x & 31) == 0) to[0] = mean_w, to[1] = m2_w, to[2] = values_w;
        } else {
            const float s[1] = {dot(v, v)};
            sums.give(s, w);
        }
    }
    __device__ __forceinline__ void take(const ResidualArgs& g, int kind, const Worker& w, float& mean, float& rinv) {
        if constexpr (MEAN) {
            float m = mean_w, m2 = m2_w;
            if (w.warps > 1) {
                const int lane = threadIdx.x & 31;
                const float* from = at + turn * kRed + lane * 4;
                const bool in = lane < w.warps;
                const float m_w = in ? from[0] : 0.f, n_w = in ? from[2] : 0.f;
                m = warp_sum(m_w * n_w, kMaxWarps) * g.each;
                m = __shfl_sync(0xffffffffu, m, 0);
                const float d = m_w - m;
                m2 = warp_sum((in ? from[1] : 0.f) + n_w * d * d, kMaxWarps);
                m2 = __shfl_sync(0xffffffffu, m2, 0);
                turn ^= 1;
            }
            const float var = m2 * g.each + (kind == BP_NORM_LAYER ? 0.f : m * m);
            mean = kind == BP_NORM_LAYER ? m : 0.f;
            rinv = rsqrtf(var + g.eps);
        } else {
            float s[1];
            sums.take(s, w);
            mean = 0.f;
            rinv = rsqrtf(fmaf(s[0], g.each, g.eps));
        }
    }
};

// A worker takes consecutive rows, a thread the same columns of each, whose weights stay in its registers; rows ahead
// are on their way in shared memory.  MEAN: a norm takes means off.  FULL: every operand and both norms are there, known
// to the compiler.  Bound by reading X and F once and writing Y and H once.
template <class T, int V, int C, bool MEAN, bool FULL>
__global__ void __maxnreg__(65536 / (32 * block_warps(false, MEAN, V, C)) / 8 * 8) k_residual(ResidualArgs g) {
    constexpr int P = V * C, S = stages<T, V, C>(false);
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float red[2 * kRed];
    Worker w(g.worker_warps, red);
    const Columns<V, C> cols(g.width, w);
    const Ring<T, V, C, 2, S> ring(room);
    const int mine = blockIdx.x * g.workers_a_block + w.id;
    check_offsets(g);
    if (mine >= g.workers) return;
    const int r0 = first_row(g, mine), r1 = first_row(g, mine + 1), n = r1 - r0;
    const bool block = FULL || g.F != nullptr, normed_out = FULL || (block && g.norm_out != BP_NORM_NONE);
    const bool gives_y = FULL || g.Y != nullptr, gives_h = FULL || g.H != nullptr;
    const bool normed_in = FULL || (g.norm_in != BP_NORM_NONE && (gives_h || g.stats != nullptr));
    const size_t at = (size_t)r0 * g.width + cols.at(0);   // this thread's first value
    const T *X = (const T*)g.X + at, *F = (const T*)g.F + at;
    T *Y = (T*)g.Y + at, *H = (T*)g.H + at;
    float* stats = g.stats != nullptr && w.tid < 4 ? g.stats + (size_t)r0 * 4 + w.tid : nullptr;
    unsigned slot = ring.base;
    int left = n;   // rows to ask for
    const auto ask = [&] {
        if (left > 0) {
            ring.ask(cols, X, slot, 0);
            if (block) ring.ask(cols, F, slot, 1);
        }
        --left;
        X += g.width, F += g.width;
        ring.commit();
        ring.step(slot);
    };
#pragma unroll
    for (int i = 0; i < S; ++i) ask();
    float k[P], wi[P], kb[MEAN ? P : 1], bi[MEAN ? P : 1];   // k: scale * gate * w_out, kb: scale * gate * b_out
    load_floats(cols, g.wi, 1.f, wi);
    if constexpr (MEAN) load_floats(cols, g.bi, 0.f, bi);
    NormStats<MEAN, V, C> of_f(w, 0, g.width), of_y(w, 4, g.width);
    int end = r0;   // of the stretch, or ~end of one that no range has (which takes no further register)
    for (int r = r0; r < r1; ++r) {
        if (r >= (end ^ (end >> 31))) {
            const Stretch now = stretch_of(g, r);
            end = now.seg >= 0 ? now.end : ~now.end;
            load_gate(g, cols, now.seg, k);
            if constexpr (MEAN) {
                load_floats(cols, g.bo, 0.f, kb);
                mul(kb, kb, k);
            }
            float wo[P];
            load_floats(cols, g.wo, 1.f, wo);
            mul(k, k, wo);
        }
        float y[P], mf = 0.f, rf = 1.f, my = 0.f, ry = 1.f;
        Piece<T, V> p[C];
        ring.wait();
        ring.take(cols, true, slot, 0, p);
        values<T, V, C>(p, y);
        if (block) {
            float u[P];
            ring.take(cols, true, slot, 1, p);
            values<T, V, C>(p, u);
            if (normed_out) {
                of_f.give(cols, u, w);
                w.sync();
                of_f.take(g, g.norm_out, w, mf, rf);
            }
            if constexpr (MEAN) sub(u, u, mf);
            mul(u, u, Same{rf});
            fma(y, k, u, y);
            if constexpr (MEAN) fma(y, kb, Same{1.f}, y);
            round_to<T, V, C>(y, p);
            if (end < 0) ring.take(cols, true, slot, 0, p);   // a row of no range is x, also where f is not a number
            values<T, V, C>(p, y);
        } else {
            round_to<T, V, C>(y, p);
        }
        if (gives_y) store_row<T>(cols, p, Y);
        if (normed_in) {
            of_y.give(cols, y, w);
            w.sync();
            of_y.take(g, g.norm_in, w, my, ry);
        }
        if (gives_h) {
            if constexpr (MEAN) sub(y, y, my);
            mul(y, y, Same{ry});
            if constexpr (MEAN) fma(y, wi, y, bi);
            else mul(y, wi, y);
            round_to<T, V, C>(y, p);
            store_row<T>(cols, p, H);
        }
        if (stats != nullptr) {
            *stats = w.tid == 0 ? mf : w.tid == 1 ? rf : w.tid == 2 ? my : ry;
            stats += 4;
        }
        ask();   // (the row's values are in registers)
        Y += g.width, H += g.width;
    }
}

// Gradients.  With f^ and y^ the normed rows, e = w_in dH, k = scale gate w_out:
//   dy = dY + r_y (e - mean(e) - y^ mean(e y^)),   dF = r_f (k dy - mean(k dy) - f^ mean(k dy f^))
// (means of e and k dy for BP_NORM_LAYER only).  dy is linear in the first two means, so those of k dy are
// sums that need not wait for them: one reduction a row.  The sums by column stay in registers over a
// run of a worker's rows: of dy f^ and dy (what gates and output weights want, by stretch where gates are by range), of dH y^
// and dH.  Bound by reading Y, F, dY and dH once and writing dX and dF once.
template <class T, int V, int C, bool MEAN, bool FULL>
__global__ void __launch_bounds__(kMaxThreads) k_residual_backward(ResidualArgs g) {
    constexpr int P = V * C, N = MEAN ? 10 : 4, S = stages<T, V, C>(true);
    extern __shared__ __align__(16) unsigned char room[];
    __shared__ float red[2 * kRed];
    pdl_launch();
    Worker w(g.worker_warps, red);
    const Columns<V, C> cols(g.width, w);
    const Ring<T, V, C, 4, S> ring(room);
    const int mine = blockIdx.x * g.workers_a_block + w.id;
    check_offsets(g);
    const bool live = mine < g.workers;
    const int r0 = live ? first_row(g, mine) : 0, r1 = live ? first_row(g, mine + 1) : 0;
    const bool has_f = FULL || g.F != nullptr, has_y = FULL || g.dY != nullptr, has_h = FULL || g.dH != nullptr;
    const bool gives_x = FULL || g.dX != nullptr, gives_f = FULL || g.dF != nullptr;
    const size_t at = (size_t)r0 * g.width + cols.at(0);   // this thread's first value
    const T *Y = (const T*)g.Y + at, *F = (const T*)g.F + at, *dY = (const T*)g.dY + at, *dH = (const T*)g.dH + at;
    T *dX = (T*)g.dX + at, *dF = (T*)g.dF + at;
    unsigned slot = ring.base;
    int left = r1 - r0;   // rows to ask for
    const auto ask = [&] {
        if (left > 0) {
            if (has_h) ring.ask(cols, Y, slot, 0);
            if (has_f) ring.ask(cols, F, slot, 1);
            if (has_y) ring.ask(cols, dY, slot, 2);
            if (has_h) ring.ask(cols, dH, slot, 3);
        }
        --left;
        Y += g.width, F += g.width, dY += g.width, dH += g.width;
        ring.commit();
        ring.step(slot);
    };
#pragma unroll
    for (int i = 0; i < S; ++i) ask();
    const bool out_normed = FULL || g.norm_out != BP_NORM_NONE;
    const float layer_in = g.norm_in == BP_NORM_LAYER ? 1.f : 0.f, layer_out = g.norm_out == BP_NORM_LAYER ? 1.f : 0.f;
    const bool by_range = g.n_gates > 0 && g.offsets != nullptr;
    // 16 values a thread are taken 8 at a time, twice a row, and their weights lie in shared memory: all at once they
    // would take more registers than there are.
    constexpr bool WIDE = P >= 16;
    constexpr int Q = WIDE ? 8 : P, Z = P / Q, JC = Q / V;   // values of a part, parts, pieces of a part
    float k_all[WIDE ? 1 : Q], wi_all[WIDE ? 1 : Q];
    float* const own = reinterpret_cast<float*>(room + (size_t)S * 4 * P * sizeof(T) * blockDim.x) + threadIdx.x;   // (WIDE)
    const auto keep = [&](const float (&x)[P], float (&to)[WIDE ? 1 : Q], int first) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            if constexpr (WIDE) own[(first + c) * blockDim.x] = x[c];
            else to[c] = x[c];
        }
    };
    const auto kept = [&](const float (&from)[WIDE ? 1 : Q], int first, int z, float (&x)[Q]) {
#pragma unroll
        for (int c = 0; c < Q; ++c) {
            if constexpr (WIDE) x[c] = own[(first + z * Q + c) * blockDim.x];
            else x[c] = from[c];
        }
    };
    {
        float x[P];
        load_floats(cols, g.wi, 1.f, x);
        keep(x, wi_all, P);
    }
    float A[Z][Q] = {}, B[MEAN ? Z : 1][MEAN ? Q : 1] = {}, CI[Z][Q] = {}, D[MEAN ? Z : 1][MEAN ? Q : 1] = {};
    // What there is of earlier rows: sums of A and B, of C and D, and of W and WB; and whether a stretch ends at `stop`.
    enum : unsigned { kRanOut = 1u, kRanIn = 2u, kWeights = 4u, kEnds = 8u };
    unsigned state = kEnds;
    const auto each_column = [&](const auto& f) {   // f(value, its place in a row of sums by worker)
#pragma unroll
        for (int c = 0; c < P; ++c)
            if (cols.in(c / V)) f(c, (size_t)mine * g.width + cols.at(c / V) + c % V);
    };
    const auto to_run = [&](auto& acc, double* run, bool ran) {
        each_column([&](int c, size_t at) {
            run[at] = (ran ? run[at] : 0.0) + (double)acc[c / Q][c % Q];
            acc[c / Q][c % Q] = 0.f;
        });
    };
    const auto with_run = [&](auto& acc, const double* run, bool ran) {
        if (ran) each_column([&](int c, size_t at) { acc[c / Q][c % Q] = (float)(run[at] + (double)acc[c / Q][c % Q]); });
    };
    // Gates by range: the sums of a stretch to its record, and times scale * gate to this worker's part of the weights'
    // gradients.
    const auto flush = [&](int seg, bool last) {
        float q[P];
        load_gate(g, cols, seg, q);
        const auto take = [&](auto& acc, const double* run, const float* gates, float* records, const float* weights, double* weights_run, float* out) {
            with_run(acc, run, state & kRanOut);
            each_column([&](int c, size_t at) {
                const float x = seg >= 0 ? acc[c / Q][c % Q] : 0.f;
                acc[c / Q][c % Q] = 0.f;
                if (seg >= 0 && gates != nullptr) records[at + (size_t)seg * g.width] = x;
                if (weights == nullptr) return;
                const double sum = (state & kWeights ? weights_run[at] : 0.0) + (double)(q[c] * x);
                if (last) out[at] = (float)sum;
                else weights_run[at] = sum;
            });
        };
        take(A, g.A_run, g.Ggate, g.A, g.Gwo, g.W_run, g.W);
        if constexpr (MEAN) take(B, g.B_run, g.Ggate, g.B, g.Gbo, g.WB_run, g.WB);
        state = (state & ~kRanOut) | kWeights;
    };
    Sums<N> sums(w);
    float next[4] = {};   // the row's statistics
    const auto load_stats = [&](int r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = __ldg(g.stats + (size_t)r * 4 + i);
    };
    if (r0 < r1) load_stats(r0);
    int stop = r0, seg = 0;   // stop: the row that begins a stretch or a run
    for (int r = r0; r < r1; ++r) {
        if (r == stop) {
            const Stretch now = stretch_of(g, r);
            const int of_run = (r - r0) % kRunRows, run_end = r + kRunRows - of_run;
            if (state & kEnds) {
                if (r > r0) flush(seg, false);
                float x[P], wo[P];
                load_gate(g, cols, now.seg, x);
                load_floats(cols, g.wo, 1.f, wo);
                mul(x, x, wo);
                keep(x, k_all, 0);
            } else {
                to_run(A, g.A_run, state & kRanOut);
                if constexpr (MEAN) to_run(B, g.B_run, state & kRanOut);
                state |= kRanOut;
            }
            if (r > r0 && of_run == 0) {
                to_run(CI, g.C_run, state & kRanIn);
                if constexpr (MEAN) to_run(D, g.D_run, state & kRanIn);
                state |= kRanIn;
            }
            seg = now.seg;
            stop = min(now.end, run_end);
            state = now.end <= run_end ? state | kEnds : state & ~kEnds;
        }
        const bool none = seg < 0;   // a row of no range has no part in f's gradients, also where f is not a number
        const float mf = next[0], rf = next[1], my = next[2], ry = next[3];
        if (r + 1 < r1) load_stats(r + 1);
        ring.wait();
        float yv[Q], fv[Q], av[Q], bv[Q], k[Q], wi[Q], s[N];
        const auto load = [&](int z) {
            Piece<T, V> y[JC], f[JC], a[JC], b[JC];
            ring.take(cols, has_h, slot, 0, y, z * JC);
            ring.take(cols, has_f, slot, 1, f, z * JC);
            ring.take(cols, has_y, slot, 2, a, z * JC);
            ring.take(cols, has_h, slot, 3, b, z * JC);
            values<T, V, JC>(y, yv), values<T, V, JC>(f, fv), values<T, V, JC>(a, av), values<T, V, JC>(b, bv);
            if constexpr (MEAN) sub(yv, yv, my), sub(fv, fv, mf);
            kept(k_all, 0, z, k), kept(wi_all, P, z, wi);
        };
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            load(z);
            float e[Q], t[Q];
            mul(e, bv, wi);
            mul(t, k, fv);
            const auto add = [&](int i, float x) { s[i] = z == 0 ? x : s[i] + x; };
            add(0, dot(e, yv)), add(1, dot(t, av)), add(2, dot(t, e)), add(3, dot(t, yv));
            if constexpr (MEAN) {
                const Same one{1.f};
                add(4, dot(one, e)), add(5, dot(one, t)), add(6, dot(k, av)), add(7, dot(k, e)), add(8, dot(k, yv)), add(9, dot(one, k));
            }
        }
        sums.give(s, w);
        w.sync();
        sums.take(s, w);
        const float c1 = ry * s[0] * g.each;
        float c0 = 0.f, d0 = 0.f, d1 = 0.f;
        if constexpr (MEAN) c0 = layer_in * s[4] * g.each;
        if (out_normed) {
            float x = s[2] - c1 * ry * s[3];
            if constexpr (MEAN) {
                x -= c0 * s[5];
                d0 = layer_out * (s[6] + ry * (s[7] - c0 * s[9] - c1 * ry * s[8])) * g.each;
            }
            d1 = rf * (s[1] + ry * x) * g.each;
        }
#pragma unroll
        for (int z = 0; z < Z; ++z) {
            if constexpr (WIDE) load(z);
            mul(yv, yv, Same{ry});
            mul(fv, fv, Same{rf});
            fma(CI[z], bv, yv, CI[z]);
            if constexpr (MEAN) fma(D[z], bv, Same{1.f}, D[z]);
            mul(bv, bv, wi);
            fma(av, bv, Same{ry}, av);
            fma(av, yv, Same{-ry * c1}, av);   // dy
            if constexpr (MEAN) sub(av, av, ry * c0);
            fma(A[z], av, fv, A[z]);
            if constexpr (MEAN) fma(B[z], av, Same{1.f}, B[z]);
            Piece<T, V> p[JC];
            if (gives_x) {
                round_to<T, V, JC>(av, p);
                store_row<T>(cols, p, dX, z * JC);
            }
            if (gives_f) {
                mul(av, av, k);
                mul(av, av, Same{rf});
                fma(av, fv, Same{-rf * d1}, av);
                if constexpr (MEAN) sub(av, av, rf * d0);
                round_to<T, V, JC>(av, p);
                if (none)
#pragma unroll
                    for (int i = 0; i < JC; ++i) p[i].u = make_uint4(0u, 0u, 0u, 0u);
                store_row<T>(cols, p, dF, z * JC);
            }
        }
        ask();   // (the row's values are in registers)
        dX += g.width, dF += g.width;
    }
    if (by_range && live && (g.Gwo != nullptr || g.Gbo != nullptr || g.Ggate != nullptr)) flush(seg, true);
    with_run(A, g.A_run, state & kRanOut);
    with_run(CI, g.C_run, state & kRanIn);
    if constexpr (MEAN) {
        with_run(B, g.B_run, state & kRanOut);
        with_run(D, g.D_run, state & kRanIn);
    }
    // The block's sums over its rows.
    const auto put = [&](const auto& acc, float* to) {
        if (g.workers_a_block == 1) {
#pragma unroll
            for (int c = 0; c < P; ++c)
                if (cols.in(c / V)) to[(size_t)blockIdx.x * g.width + cols.at(c / V) + c % V] = acc[c / Q][c % Q];
            return;
        }
        float* part = reinterpret_cast<float*>(room);
        __syncthreads();
#pragma unroll
        for (int c = 0; c < P; ++c)
            if (cols.in(c / V)) part[w.id * g.width + cols.at(c / V) + c % V] = acc[c / Q][c % Q];
        __syncthreads();
        for (int c = threadIdx.x; c < g.width; c += blockDim.x) {
            float x = part[c];
            for (int i = 1; i < g.workers_a_block; ++i) x += part[i * g.width + c];
            to[(size_t)blockIdx.x * g.width + c] = x;
        }
    };
    if (!by_range) {
        if (g.Gwo != nullptr || g.Ggate != nullptr) put(A, g.A);
        if constexpr (MEAN)
            if (g.Gbo != nullptr || g.Ggate != nullptr) put(B, g.B);
    }
    if (g.Gwi != nullptr) put(CI, g.C);
    if constexpr (MEAN)
        if (g.Gbi != nullptr) put(D, g.D);
}

// The blocks' and workers' sums, added up in their order: blocks (x) of 32 columns by (y) output weights, biases and one row
// of gates for all; input weights and biases; then the rows of gates by range.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(kJoinWarps * 32) k_residual_join(ResidualArgs g) {
    __shared__ float part[2][kJoinWarps][33];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const bool in = col < g.width, by_range = g.n_gates > 0 && g.offsets != nullptr;
    const bool layer = g.B != nullptr;
    const int job = blockIdx.y;
    const float *from = nullptr, *from2 = nullptr;
    int lo = 0, hi = (int)((g.workers + g.workers_a_block - 1) / g.workers_a_block);   // blocks
    if (job == 0) {
        if (by_range) hi = g.workers;
        if (g.Gwo != nullptr || (!by_range && g.Ggate != nullptr)) from = by_range ? g.W : g.A;
        if (layer && (g.Gbo != nullptr || (!by_range && g.Ggate != nullptr))) from2 = by_range ? g.WB : g.B;
    } else if (job == 1) {
        if (g.Gwi != nullptr) from = g.C;
        if (g.Gbi != nullptr) from2 = g.D;
    } else {
        from = g.A;
        from2 = layer && g.bo != nullptr ? g.B : nullptr;
    }
    if (from == nullptr && from2 == nullptr) return;
    const auto give = [&](float* out, size_t at, float x) {
        if (out != nullptr) out[at] = g.accumulate ? out[at] + x : x;
    };
    for (int seg = job - 2; seg < g.n_gates; seg += (int)gridDim.y - 2) {
        if (job >= 2) {
            const int a = min(max(__ldg(g.offsets + seg), 0), g.n), b = min(max(__ldg(g.offsets + seg + 1), a), g.n);
            lo = hi = 0;
            if (b > a) {   // the records of the workers that hold rows a and b - 1, and those between
                lo = (int)((((long long)a + 1) * g.workers - 1) / g.n) + seg;
                hi = (int)(((long long)b * g.workers - 1) / g.n) + seg + 1;
            }
        }
        float s = 0.f, s2 = 0.f;
        if (in) {
#pragma unroll 4
            for (int r = lo + warp; r < hi; r += kJoinWarps) {
                if (from != nullptr) s += __ldcg(from + (size_t)r * g.width + col);
                if (from2 != nullptr) s2 += __ldcg(from2 + (size_t)r * g.width + col);
            }
        }
        part[0][warp][lane] = s;
        part[1][warp][lane] = s2;
        __syncthreads();
        if (warp == 0 && in) {
            s = s2 = 0.f;
            for (int w = 0; w < kJoinWarps; ++w) s += part[0][w][lane], s2 += part[1][w][lane];
            const float wo = g.wo != nullptr ? __ldg(g.wo + col) : 1.f, bo = g.bo != nullptr ? __ldg(g.bo + col) : 0.f;
            if (job == 1) {
                give(g.Gwi, col, s);
                give(g.Gbi, col, s2);
            } else if (job == 0) {
                const float k = by_range ? 1.f : g.scale * (g.n_gates > 0 ? __ldg(g.gate + col) : 1.f);
                give(g.Gwo, col, k * s);
                give(g.Gbo, col, k * s2);
                if (!by_range) give(g.Ggate, col, g.scale * (bo * s2 + wo * s));
            } else {
                give(g.Ggate, (size_t)seg * g.width + col, g.scale * (bo * s2 + wo * s));
            }
        }
        if (job < 2) return;
        __syncthreads();
    }
}

// How rows of `width` are shared out: pieces of v values, c of them a thread, `warps` a worker, `workers` a block; one block
// an SM.  Going forward, 8 values a thread where a row has them for more than
// 32 threads (16,000 rows of 600 float32 units, layer norms: 39 us, 50 with 4), 16 above 2,048 units: what a thread does once a row (its part of
// two reductions, addresses) is a third of its instructions then (16,384 rows of 4,096 bfloat16 units: 88.7 us, 6.05 TB/s;
// 98.5 us with 8).  Backward that would take more registers than 512 threads have, and half the threads are no faster
// (143 us, 5.6 TB/s, with 8 values and 512 threads; the same with 16 and 256).
struct Shape {
    int v, c, warps, workers;
};
Shape shape_of(int width, int size, bool pieces, bool back, bool mean) {
    Shape s;
    s.v = pieces ? 16 / size : 1;
    const int nv = (width + s.v - 1) / s.v;
    s.c = 1;
    while (!back && (nv + s.c - 1) / s.c > 32 && s.c * s.v < 8) s.c *= 2;
    while ((nv + s.c - 1) / s.c > (back ? kMaxThreads : kMaxThreads / 2) && s.c * s.v < 16) s.c *= 2;
    s.warps = ((nv + s.c - 1) / s.c + 31) / 32;
    s.workers = min(s.warps > 1 ? 15 : 32, block_warps(back, mean, s.v, s.c) / s.warps);   // (15: barriers)
    return s;
}

bool pieces16(const ResidualArgs& a) {
    const uintptr_t p = (uintptr_t)a.X | (uintptr_t)a.F | (uintptr_t)a.Y | (uintptr_t)a.H | (uintptr_t)a.dY | (uintptr_t)a.dH |
                        (uintptr_t)a.dX | (uintptr_t)a.dF;
    return (p & 15) == 0 && a.width % 4 == 0;
}

bool takes_means(const ResidualArgs& a) { return a.norm_out == BP_NORM_LAYER || a.norm_in == BP_NORM_LAYER; }

// What to do with the kernels of a shape: launch one, or set up both.
struct Launch {
    const ResidualArgs* a;
    bool back;
    cudaStream_t s;
    template <class T, int V, int C>
    cudaError_t shape() const {
        const bool mean = takes_means(*a);
        const int threads = a->workers_a_block * a->worker_warps * 32, blocks = (a->workers + a->workers_a_block - 1) / a->workers_a_block;
        const int bytes = thread_bytes<T, V, C>(back) * threads;
        const bool norms = a->F != nullptr && a->norm_out != BP_NORM_NONE && a->norm_in != BP_NORM_NONE;
        const bool full = V > 1 && norms && (back ? a->dY != nullptr && a->dH != nullptr && a->dX != nullptr && a->dF != nullptr : a->H != nullptr);
        const auto go = [&](auto k) { k<<<blocks, threads, bytes, s>>>(*a); };
        if (back) {
            if (mean) full ? go(k_residual_backward<T, V, C, true, (V > 1)>) : go(k_residual_backward<T, V, C, true, false>);
            else full ? go(k_residual_backward<T, V, C, false, (V > 1)>) : go(k_residual_backward<T, V, C, false, false>);
        } else {
            if (mean) full ? go(k_residual<T, V, C, true, (V > 1)>) : go(k_residual<T, V, C, true, false>);
            else full ? go(k_residual<T, V, C, false, (V > 1)>) : go(k_residual<T, V, C, false, false>);
        }
        return cudaGetLastError();
    }
};
struct Setup {
    template <class T, int V, int C>
    cudaError_t shape() const {
        const auto most = [](bool back, bool mean) { return thread_bytes<T, V, C>(back) * block_warps(back, mean, V, C) * 32; };
        const auto set = [](auto k, int bytes) { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); };
        cudaError_t e = cudaSuccess;
        const auto both = [&](auto full, auto mean) {
            if (e == cudaSuccess) e = set(k_residual<T, V, C, decltype(mean)::value, decltype(full)::value>, most(false, decltype(mean)::value));
            if (e == cudaSuccess) e = set(k_residual_backward<T, V, C, decltype(mean)::value, decltype(full)::value>, most(true, decltype(mean)::value));
        };
        both(std::false_type{}, std::false_type{}), both(std::false_type{}, std::true_type{});
        if constexpr (V > 1) both(std::true_type{}, std::false_type{}), both(std::true_type{}, std::true_type{});
        return e;
    }
};
template <class F>
cudaError_t with_shape(const F& f, int dtype, const Shape& h) {
    if (dtype == BP_BF16) return h.c == 1 ? f.template shape<__nv_bfloat16, 8, 1>() : f.template shape<__nv_bfloat16, 8, 2>();
    if (h.v == 4) return h.c == 1 ? f.template shape<float, 4, 1>() : h.c == 2 ? f.template shape<float, 4, 2>() : f.template shape<float, 4, 4>();
    switch (h.c) {
        case 1: return f.template shape<float, 1, 1>();
        case 2: return f.template shape<float, 1, 2>();
        case 4: return f.template shape<float, 1, 4>();
        case 8: return f.template shape<float, 1, 8>();
        default: return f.template shape<float, 1, 16>();
    }
}
Shape shape_of(const ResidualArgs& a, bool back) {
    return shape_of(a.width, a.dtype == BP_F32 ? 4 : 2, a.dtype == BP_BF16 || pieces16(a), back, takes_means(a));
}

}  // namespace

int residual_workers(int num_sms, int width, int dtype) {
    const Shape s = shape_of(width, dtype == BP_F32 ? 4 : 2, true, true, true);
    if (dtype == BP_BF16) return num_sms * s.workers;
    return num_sms * max(s.workers, shape_of(width, 4, false, true, true).workers);   // a call's rows may be whole pieces or not
}

cudaError_t residual_setup(int width, int dtype) {
    const int size = dtype == BP_F32 ? 4 : 2;
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < 4 && e == cudaSuccess; ++i)   // rows in whole pieces or not, either direction
        if ((i & 1) == 0 || dtype == BP_F32) e = with_shape(Setup{}, dtype, shape_of(width, size, (i & 1) == 0, i >= 2, true));
    return e;
}

cudaError_t residual_forward(ResidualArgs a, cudaStream_t s) {
    const Shape h = shape_of(a, false);
    const int blocks = a.num_sms;
    a.worker_warps = h.warps;
    a.workers = min(a.n, blocks * h.workers);
    a.workers_a_block = (a.workers + blocks - 1) / blocks;
    return with_shape(Launch{&a, false, s}, a.dtype, h);
}

cudaError_t residual_backward(ResidualArgs a, cudaStream_t s) {
    const Shape h = shape_of(a, true);
    a.worker_warps = h.warps;
    a.workers = min((a.n + kWorkerRows - 1) / kWorkerRows, a.num_sms * h.workers);
    a.workers_a_block = (a.workers + a.num_sms - 1) / a.num_sms;
    const cudaError_t e = with_shape(Launch{&a, true, s}, a.dtype, h);
    if (e != cudaSuccess) return e;
    const bool weights = a.Gwo != nullptr || a.Gbo != nullptr || a.Gwi != nullptr || a.Gbi != nullptr;
    if (!weights && a.Ggate == nullptr) return cudaSuccess;
    const int ranges = a.Ggate != nullptr && a.offsets != nullptr ? min(a.n_gates, 4096) : 0;
    return launch_pdl(k_residual_join, (a.width + 31) / 32, 2 + ranges, kJoinWarps * 32, 0, s, a);
}

}  // namespace bp
