// The stream between blocks: a block's output is normed, gated, scaled and added, and the sum is normed again; with the
// gradients.  Rows are independent but for the sums of the weights' and gates' gradients.
#include "bp_blocks_internal.h"
#include "bp_pieces.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32;

// Sums of the block's values, in one order, in every thread.  The two halves of `red` are used in turn, so
// that one barrier a call is enough.
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (*red)[kMaxWarps * 8], int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    float* at = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) at[(threadIdx.x >> 5) * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = at[i];
    for (int w = 1; w < warps; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += at[w * N + i];
}

// Number, mean and sum of squared differences from it, of two sets together: no cancellation where the mean
// is far from 0.
struct Moments {
    float n, mean, m2;
    __device__ __forceinline__ void join(float n2, float mean2, float m22) {
        const float all = n + n2;
        if (all == 0.f) return;
        const float d = mean2 - mean, part = n2 / all;
        mean += d * part;
        m2 += m22 + d * d * n * part;
        n = all;
    }
};
__device__ __forceinline__ void block_moments(Moments& m, float (*red)[kMaxWarps * 8], int& turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        m.join(__shfl_xor_sync(0xffffffffu, m.n, o), __shfl_xor_sync(0xffffffffu, m.mean, o), __shfl_xor_sync(0xffffffffu, m.m2, o));
    m.n = __shfl_sync(0xffffffffu, m.n, 0);   // (joined in another order, other lanes have other last bits)
    m.mean = __shfl_sync(0xffffffffu, m.mean, 0);
    m.m2 = __shfl_sync(0xffffffffu, m.m2, 0);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    float* at = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
        const int w = threadIdx.x >> 5;
        at[w * 3] = m.n, at[w * 3 + 1] = m.mean, at[w * 3 + 2] = m.m2;
    }
    __syncthreads();
    m = {at[0], at[1], at[2]};
    for (int w = 1; w < warps; ++w) m.join(at[w * 3], at[w * 3 + 1], at[w * 3 + 2]);
}

// A thread's columns: C pieces of V, the block's width apart.
template <int V, int C>
struct Columns {
    int width;
    __device__ __forceinline__ int at(int j) const { return (j * (int)blockDim.x + (int)threadIdx.x) * V; }
    __device__ __forceinline__ bool in(int j) const { return at(j) < width; }
};

template <int V, int C>
__device__ __forceinline__ void load_floats(const Columns<V, C>& cols, const float* p, float none, float (&out)[V * C]) {
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) out[j * V + i] = p != nullptr && cols.in(j) ? __ldg(p + cols.at(j) + i) : none;
}

template <class T, int V, int C>
__device__ __forceinline__ void load_row(const Columns<V, C>& cols, const void* p, long long row, Piece<T, V> (&out)[C]) {
#pragma unroll
    for (int j = 0; j < C; ++j) {
        out[j].u = make_uint4(0u, 0u, 0u, 0u);
        if (p != nullptr && cols.in(j)) out[j].load_rw((const T*)p + (size_t)row * cols.width + cols.at(j));
    }
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
__device__ __forceinline__ int first_row(const ResidualArgs& g, int cta) { return (int)((long long)g.n * cta / (int)gridDim.x); }

// scale * gate of a stretch, by column.
template <int V, int C>
__device__ __forceinline__ void load_gate(const ResidualArgs& g, const Columns<V, C>& cols, int seg, float (&k)[V * C]) {
    load_floats(cols, g.n_gates > 0 && seg >= 0 ? g.gate + (size_t)seg * g.width : nullptr, seg < 0 ? 0.f : 1.f, k);
#pragma unroll
    for (int i = 0; i < V * C; ++i) k[i] *= g.scale;
}

template <bool MEAN, int V, int C>
__device__ __forceinline__ void norm_stats(const ResidualArgs& g, const Columns<V, C>& cols, const float (&v)[V * C], int kind,
                                           float (*red)[kMaxWarps * 8], int& turn, float& mean, float& rinv) {
    if constexpr (MEAN) {
        Moments m{0.f, 0.f, 0.f};
        float sum = 0.f;
        int n = 0;
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (cols.in(j)) {
                n += V;
#pragma unroll
                for (int i = 0; i < V; ++i) sum += v[j * V + i];
            }
        m.n = (float)n;
        m.mean = n > 0 ? sum / m.n : 0.f;
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (cols.in(j))
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = v[j * V + i] - m.mean;
                    m.m2 += d * d;
                }
        block_moments(m, red, turn);
        const float var = m.m2 / m.n + (kind == BP_NORM_LAYER ? 0.f : m.mean * m.mean);
        mean = kind == BP_NORM_LAYER ? m.mean : 0.f;
        rinv = 1.f / sqrtf(var + g.eps);
    } else {
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < V * C; ++i) s[0] = fmaf(v[i], v[i], s[0]);   // (columns past the row's end are 0)
        block_sums(s, red, turn);
        mean = 0.f;
        rinv = 1.f / sqrtf(s[0] / (float)g.width + g.eps);
    }
}

// A block takes consecutive rows, a thread the same columns of each, whose weights stay in its registers; the next row is
// under way while one is worked on.  MEAN: a norm takes means off.  Bound by reading X and F once and writing Y
// and H once.
template <class T, int V, int C, bool MEAN>
__global__ void __launch_bounds__(kMaxThreads) k_residual(ResidualArgs g) {
    constexpr int P = V * C;
    __shared__ float red[2][kMaxWarps * 8];
    int turn = 0;
    const Columns<V, C> cols{g.width};
    const int r0 = first_row(g, blockIdx.x), r1 = first_row(g, blockIdx.x + 1);
    const bool block = g.F != nullptr, normed_in = g.norm_in != BP_NORM_NONE && (g.H != nullptr || g.stats != nullptr);
    check_offsets(g);
    float wo[P], wi[P], bo[MEAN ? P : 1], bi[MEAN ? P : 1], k[P];
    load_floats(cols, g.wo, 1.f, wo);
    load_floats(cols, g.wi, 1.f, wi);
    if constexpr (MEAN) {
        load_floats(cols, g.bo, 0.f, bo);
        load_floats(cols, g.bi, 0.f, bi);
    }
    Piece<T, V> x[C], f[C];
    load_row(cols, g.X, r0, x);
    load_row(cols, g.F, r0, f);
    Stretch now{0, r0};
    for (int r = r0; r < r1; ++r) {
        if (r >= now.end) {
            now = stretch_of(g, r);
            load_gate(g, cols, now.seg, k);
        }
        Piece<T, V> xn[C], fn[C];
        if (r + 1 < r1) {
            load_row(cols, g.X, r + 1, xn);
            load_row(cols, g.F, r + 1, fn);
        }
        float y[P], u[P], mf = 0.f, rf = 1.f, my = 0.f, ry = 1.f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float a[V], b[V];
            x[j].values(a);
            f[j].values(b);
#pragma unroll
            for (int i = 0; i < V; ++i) y[j * V + i] = a[i], u[j * V + i] = b[i];
        }
        if (block) {
            if (g.norm_out != BP_NORM_NONE) norm_stats<MEAN>(g, cols, u, g.norm_out, red, turn, mf, rf);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                float a[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = j * V + i;
                    float h = (u[c] - mf) * rf * wo[c];
                    if constexpr (MEAN) h += bo[c];
                    a[i] = cols.in(j) ? fmaf(k[c], h, y[c]) : 0.f;
                }
                x[j].set(a);
                x[j].values(a);
#pragma unroll
                for (int i = 0; i < V; ++i) y[j * V + i] = a[i];
            }
        }
        if (g.Y != nullptr)
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (cols.in(j)) x[j].store((T*)g.Y + (size_t)r * g.width + cols.at(j));
        if (normed_in) norm_stats<MEAN>(g, cols, y, g.norm_in, red, turn, my, ry);
        if (g.H != nullptr) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                if (!cols.in(j)) continue;
                float h[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = j * V + i;
                    h[i] = (y[c] - my) * ry * wi[c];
                    if constexpr (MEAN) h[i] += bi[c];
                }
                Piece<T, V> p;
                p.set(h);
                p.store((T*)g.H + (size_t)r * g.width + cols.at(j));
            }
        }
        if (g.stats != nullptr && threadIdx.x < 4)
            g.stats[(size_t)r * 4 + threadIdx.x] = threadIdx.x == 0 ? mf : threadIdx.x == 1 ? rf : threadIdx.x == 2 ? my : ry;
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = xn[j], f[j] = fn[j];
    }
}

// Gradients.  With f^ and y^ the normed rows, e = w_in dH, k = scale gate w_out:
//   dy = dY + r_y (e - mean(e) - y^ mean(e y^)),   dF = r_f (k dy - mean(k dy) - f^ mean(k dy f^))
// (means of e and k dy for BP_NORM_LAYER only).  dy is linear in the first two means, so those of k dy are
// sums that need not wait for them: one reduction a row.  The sums by column stay in registers over a
// block's rows: of dy f^ and dy by stretch (what gates and output weights want), of dH y^ and dH.
// Bound by reading Y, F, dY and dH once and writing dX and dF once.
template <class T, int V, int C, bool MEAN>
__global__ void __launch_bounds__(kMaxThreads) k_residual_backward(ResidualArgs g) {
    constexpr int P = V * C, S = MEAN ? 8 : 3;
    __shared__ float red[2][kMaxWarps * 8];
    int turn = 0;
    pdl_launch();
    const Columns<V, C> cols{g.width};
    const int r0 = first_row(g, blockIdx.x), r1 = first_row(g, blockIdx.x + 1);
    const bool out_normed = g.norm_out != BP_NORM_NONE;
    const float layer_in = g.norm_in == BP_NORM_LAYER ? 1.f : 0.f, layer_out = g.norm_out == BP_NORM_LAYER ? 1.f : 0.f;
    const float each = 1.f / (float)g.width;
    const bool sum_out = g.Gwo != nullptr || g.Gbo != nullptr || g.Ggate != nullptr;
    check_offsets(g);
    float k[P], wi[P];
    load_floats(cols, g.wi, 1.f, wi);
    float A[P] = {}, B[MEAN ? P : 1] = {}, CI[P] = {}, D[MEAN ? P : 1] = {};
    bool fresh = true;   // nothing of this block in W and WB
    // The sums of a stretch: to its record, and times scale * gate to this block's part of the weights' gradients.
    const auto flush = [&](int seg) {
        if (!sum_out) return;
        float q[P];
        load_gate(g, cols, seg, q);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!cols.in(j)) continue;
            const size_t w = (size_t)blockIdx.x * g.width + cols.at(j);
            const size_t rec = (size_t)(blockIdx.x + max(seg, 0)) * g.width + cols.at(j);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = j * V + i;
                if (seg >= 0 && g.Ggate != nullptr) g.A[rec + i] = A[c];
                if (g.Gwo != nullptr) g.W[w + i] = (fresh ? 0.f : g.W[w + i]) + q[c] * A[c];
                if constexpr (MEAN) {
                    if (seg >= 0 && g.Ggate != nullptr && g.bo != nullptr) g.B[rec + i] = B[c];
                    if (g.Gbo != nullptr) g.WB[w + i] = (fresh ? 0.f : g.WB[w + i]) + q[c] * B[c];
                }
            }
        }
        fresh = false;
#pragma unroll
        for (int c = 0; c < P; ++c) {
            A[c] = 0.f;
            if constexpr (MEAN) B[c] = 0.f;
        }
    };
    Piece<T, V> y[C], f[C], a[C], b[C];
    const auto load = [&](int r, Piece<T, V>(&y)[C], Piece<T, V>(&f)[C], Piece<T, V>(&a)[C], Piece<T, V>(&b)[C]) {
        load_row(cols, g.dH != nullptr ? g.Y : nullptr, r, y);
        load_row(cols, g.F, r, f);
        load_row(cols, g.dY, r, a);
        load_row(cols, g.dH, r, b);
    };
    load(r0, y, f, a, b);
    Stretch now{0, r0};
    for (int r = r0; r < r1; ++r) {
        if (r >= now.end) {
            if (r > r0) flush(now.seg);
            now = stretch_of(g, r);
            load_gate(g, cols, now.seg, k);
            float wo[P];
            load_floats(cols, g.wo, 1.f, wo);
#pragma unroll
            for (int c = 0; c < P; ++c) k[c] *= wo[c];
        }
        Piece<T, V> yn[C], fn[C], an[C], bn[C];
        if (r + 1 < r1) load(r + 1, yn, fn, an, bn);
        const float* st = g.stats + (size_t)r * 4;
        const float mf = __ldg(st), rf = __ldg(st + 1), my = __ldg(st + 2), ry = __ldg(st + 3);
        float s[S] = {};
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!cols.in(j)) continue;
            float yv[V], fv[V], av[V], bv[V];
            y[j].values(yv), f[j].values(fv), a[j].values(av), b[j].values(bv);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = j * V + i;
                const float e = bv[i] * wi[c], yh = (yv[i] - my) * ry, fh = (fv[i] - mf) * rf, base = av[i] + ry * e;
                s[0] = fmaf(e, yh, s[0]);
                s[1] = fmaf(k[c] * base, fh, s[1]);
                s[2] = fmaf(k[c] * yh, fh, s[2]);
                if constexpr (MEAN) {
                    s[3] += e;
                    s[4] = fmaf(k[c], fh, s[4]);
                    s[5] = fmaf(k[c], base, s[5]);
                    s[6] = fmaf(k[c], yh, s[6]);
                    s[7] += k[c];
                }
            }
        }
        block_sums(s, red, turn);
        const float c1 = s[0] * each;
        float c0 = 0.f, d0 = 0.f, d1 = 0.f;
        if constexpr (MEAN) c0 = layer_in * s[3] * each;
        if (out_normed) {
            d1 = s[1] - ry * c1 * s[2];
            if constexpr (MEAN) {
                d1 -= ry * c0 * s[4];
                d0 = layer_out * (s[5] - ry * (c0 * s[7] + c1 * s[6])) * each;
            }
            d1 *= each;
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!cols.in(j)) continue;
            float yv[V], fv[V], av[V], bv[V], dx[V], df[V];
            y[j].values(yv), f[j].values(fv), a[j].values(av), b[j].values(bv);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = j * V + i;
                const float e = bv[i] * wi[c], yh = (yv[i] - my) * ry, fh = (fv[i] - mf) * rf;
                const float dy = av[i] + ry * (e - c0 - yh * c1);
                dx[i] = dy;
                df[i] = rf * (k[c] * dy - d0 - fh * d1);
                A[c] = fmaf(dy, fh, A[c]);
                CI[c] = fmaf(bv[i], yh, CI[c]);
                if constexpr (MEAN) {
                    B[c] += dy;
                    D[c] += bv[i];
                }
            }
            Piece<T, V> p;
            const size_t at = (size_t)r * g.width + cols.at(j);
            if (g.dX != nullptr) {
                p.set(dx);
                p.store((T*)g.dX + at);
            }
            if (g.dF != nullptr) {
                p.set(df);
                p.store((T*)g.dF + at);
            }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = yn[j], f[j] = fn[j], a[j] = an[j], b[j] = bn[j];
    }
    flush(now.seg);
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if (!cols.in(j)) continue;
        const size_t w = (size_t)blockIdx.x * g.width + cols.at(j);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (g.Gwi != nullptr) g.C[w + i] = CI[j * V + i];
            if constexpr (MEAN)
                if (g.Gbi != nullptr) g.D[w + i] = D[j * V + i];
        }
    }
}

// The blocks' sums, added up in the blocks' order: blocks (x) of 32 columns by (y) the four sums of weights and
// biases, then the rows of gates.
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(kJoinWarps * 32) k_residual_join(ResidualArgs g) {
    __shared__ float part[2][kJoinWarps][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const bool in = col < g.width;
    const int job = blockIdx.y;
    float *out = nullptr, *from = nullptr, *from2 = nullptr;
    int lo = 0, hi = g.ctas, seg = 0;
    if (job < 4) {
        out = job == 0 ? g.Gwo : job == 1 ? g.Gbo : job == 2 ? g.Gwi : g.Gbi;
        from = job == 0 ? g.W : job == 1 ? g.WB : job == 2 ? g.C : g.D;
    }
    for (int it = 0;; ++it) {
        if (job >= 4) {   // gates, a block several rows of them
            seg = job - 4 + it * ((int)gridDim.y - 4);
            if (seg >= g.n_gates) return;
            out = g.Ggate;
            from = g.A, from2 = g.bo != nullptr ? g.B : nullptr;
            int a = 0, b = g.n;
            if (g.offsets != nullptr) {
                a = min(max(__ldg(g.offsets + seg), 0), g.n);
                b = min(max(__ldg(g.offsets + seg + 1), a), g.n);
            }
            lo = hi = 0;
            if (b > a) {   // the blocks that hold rows a and b - 1
                lo = (int)((((long long)a + 1) * g.ctas - 1) / g.n) + seg;
                hi = (int)(((long long)b * g.ctas - 1) / g.n) + seg + 1;
            }
        } else if (it > 0) {
            return;
        }
        if (out == nullptr) return;
        float s = 0.f, s2 = 0.f;
        if (in) {
#pragma unroll 4
            for (int r = lo + warp; r < hi; r += kJoinWarps) {
                s += __ldcg(from + (size_t)r * g.width + col);
                if (from2 != nullptr) s2 += __ldcg(from2 + (size_t)r * g.width + col);
            }
        }
        part[0][warp][lane] = s;
        part[1][warp][lane] = s2;
        __syncthreads();
        if (warp == 0 && in) {
            for (int w = 1; w < kJoinWarps; ++w) s += part[0][w][lane], s2 += part[1][w][lane];
            float* to = out + col;
            if (job >= 4) {
                to += (size_t)seg * g.width;
                s *= g.wo != nullptr ? __ldg(g.wo + col) : 1.f;
                if (from2 != nullptr) s = fmaf(__ldg(g.bo + col), s2, s);
                s *= g.scale;
            }
            *to = g.accumulate ? *to + s : s;
        }
        __syncthreads();
    }
}

// Threads and pieces a thread for rows of `width`.
struct Shape {
    int v, c, threads;
};
template <class T>
Shape shape_of(int width, bool pieces) {
    Shape s;
    s.v = pieces ? 16 / (int)sizeof(T) : 1;
    const int nv = (width + s.v - 1) / s.v;
    s.c = 1;
    while ((nv + s.c - 1) / s.c > kMaxThreads) s.c *= s.v == 1 ? 4 : 2;
    s.threads = ((nv + s.c - 1) / s.c + 31) / 32 * 32;
    return s;
}

bool pieces16(const ResidualArgs& a) {
    const uintptr_t p = (uintptr_t)a.X | (uintptr_t)a.F | (uintptr_t)a.Y | (uintptr_t)a.H | (uintptr_t)a.dY | (uintptr_t)a.dH |
                        (uintptr_t)a.dX | (uintptr_t)a.dF;
    return (p & 15) == 0 && a.width % 4 == 0;
}

template <class T, int V, int C>
cudaError_t run(const ResidualArgs& a, bool back, int threads, cudaStream_t s) {
    const bool mean = a.norm_out == BP_NORM_LAYER || a.norm_in == BP_NORM_LAYER;
    if (!back) {
        if (mean) k_residual<T, V, C, true><<<a.ctas, threads, 0, s>>>(a);
        else k_residual<T, V, C, false><<<a.ctas, threads, 0, s>>>(a);
    } else if (mean) {
        k_residual_backward<T, V, C, true><<<a.ctas, threads, 0, s>>>(a);
    } else {
        k_residual_backward<T, V, C, false><<<a.ctas, threads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t run_shape(ResidualArgs& a, bool back, cudaStream_t s) {
    const bool f32 = a.dtype == BP_F32, pieces = !f32 || pieces16(a);
    const Shape h = f32 ? shape_of<float>(a.width, pieces) : shape_of<__nv_bfloat16>(a.width, true);
    a.ctas = min(a.n, residual_ctas(a.num_sms, h.threads));
    if (!f32) {
        if (h.c == 1) return run<__nv_bfloat16, 8, 1>(a, back, h.threads, s);
        return run<__nv_bfloat16, 8, 2>(a, back, h.threads, s);
    }
    if (h.v == 4) {
        if (h.c == 1) return run<float, 4, 1>(a, back, h.threads, s);
        if (h.c == 2) return run<float, 4, 2>(a, back, h.threads, s);
        return run<float, 4, 4>(a, back, h.threads, s);
    }
    if (h.c == 1) return run<float, 1, 1>(a, back, h.threads, s);
    if (h.c == 4) return run<float, 1, 4>(a, back, h.threads, s);
    return run<float, 1, 16>(a, back, h.threads, s);
}

}  // namespace

int residual_ctas(int num_sms, int threads) { return num_sms * max(1, min(16, 1024 / threads)); }
int residual_most_ctas(int num_sms, int width, int dtype) {
    if (dtype == BP_BF16) return residual_ctas(num_sms, shape_of<__nv_bfloat16>(width, true).threads);
    // a call's rows may be whole pieces or not
    return max(residual_ctas(num_sms, shape_of<float>(width, true).threads), residual_ctas(num_sms, shape_of<float>(width, false).threads));
}

cudaError_t residual_forward(ResidualArgs a, cudaStream_t s) { return run_shape(a, false, s); }

cudaError_t residual_backward(ResidualArgs a, cudaStream_t s) {
    const cudaError_t e = run_shape(a, true, s);
    if (e != cudaSuccess) return e;
    const bool weights = a.Gwo != nullptr || a.Gbo != nullptr || a.Gwi != nullptr || a.Gbi != nullptr, gates = a.Ggate != nullptr;
    if (!weights && !gates) return cudaSuccess;
    return launch_pdl(k_residual_join, (a.width + 31) / 32, 4 + (gates ? min(a.n_gates, 4096) : 0), kJoinWarps * 32, 0, s, a);
}

}  // namespace bp
