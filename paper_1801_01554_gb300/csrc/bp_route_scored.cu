// The router by scores: k experts of each pattern by softmax or sigmoid scores and a bias, within the pattern's best
// groups of experts, their gates, and the gates' gradient.
#include <cmath>

#include "bp_route_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256, kBackThreads = 256;
constexpr int kOneBlock = 64;    // patterns of a call that one block takes (256 of 128 experts: 41 us in one block, 17 us in several)
constexpr float kNone = -INFINITY;

// A warp takes a pattern: each group of experts has 32 / (groups, rounded up to a power of two) lanes, a lane
// `per` consecutive experts of its group.  So the lowest index among equals is the first lane's first.
struct Share {
    int first, count, group, group_lanes;
};
__device__ __forceinline__ Share share_of(const ScoredArgs& g) {
    const int lane = threadIdx.x & 31, size = g.E / g.n_groups, sub = lane % g.group_lanes;
    Share s;
    s.group = lane / g.group_lanes;
    s.group_lanes = g.group_lanes;
    s.first = s.group * size + sub * g.per;
    s.count = s.group < g.n_groups ? min(max(size - sub * g.per, 0), g.per) : 0;
    return s;
}

// float64 values as whole numbers that ascend with them (the float64 unit is slow, 16 cycles a warp's operation,
// comparisons too).
using Order64 = unsigned long long;
__device__ __forceinline__ Order64 order64(double x) {
    const Order64 u = (Order64)__double_as_longlong(x + 0.0);   // (-0 and 0 are equal)
    if (!(x > -INFINITY)) return 0ull;
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ double value64(Order64 o) {
    return __longlong_as_double((long long)((o >> 63) ? (o & 0x7fffffffffffffffull) : ~o));
}
// What is below every value: of an expert that is closed.
template <class F>
constexpr F kClosed = kNone;
template <>
constexpr Order64 kClosed<Order64> = 0ull;
__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ Order64 plus(Order64 a, Order64 b) { return order64(value64(a) + value64(b)); }
// The largest value of the warp.
__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ Order64 warp_max(Order64 x) {
    const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(x >> 32));
    const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(x >> 32) == hi ? (unsigned)x : 0u);
    return ((Order64)hi << 32) | lo;
}

// A lane's two largest values and where they are, ties to the lowest index.
template <class F, int PER>
struct Best {
    F v1, v2;
    int at1, at2;
    bool known2;   // v2 is the second largest (and not: was taken)
    __device__ __forceinline__ void start() { v1 = v2 = kClosed<F>, at1 = at2 = 0, known2 = true; }
    __device__ __forceinline__ void see(F x, int i) {
        const bool first = x > v1, second = x > v2;
        v2 = first ? v1 : second ? x : v2;
        at2 = first ? at1 : second ? i : at2;
        v1 = first ? x : v1;
        at1 = first ? i : at1;
    }
    __device__ __forceinline__ void scan(const F (&c)[PER]) {
        start();
#pragma unroll
        for (int i = 0; i < PER; ++i) see(c[i], i);
    }
    // Without the largest one.
    __device__ __forceinline__ void pop(const F (&c)[PER]) {
        if (known2) {
            v1 = v2, at1 = at2, known2 = false;
            return;
        }
        const F last = v1;
        const int last_at = at1;
        start();
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (c[i] < last || (c[i] == last && i > last_at)) see(c[i], i);
    }
};

// What the lane's group is worth: its largest value, or the sum of its two largest.
template <class F>
__device__ __forceinline__ F group_worth(const ScoredArgs& g, const Share& s, F m1, F m2) {   // a lane's two largest
    for (int d = 1; d < s.group_lanes; d <<= 1) {
        const F p1 = __shfl_xor_sync(0xffffffffu, m1, d), p2 = __shfl_xor_sync(0xffffffffu, m2, d);
        m2 = max(min(m1, p1), max(m2, p2));
        m1 = max(m1, p1);
    }
    return g.group_top == 2 && m2 > kClosed<F> ? plus(m1, m2) : m1;   // (kClosed: a group with none open)
}
// Whether the lane's group is one of the open ones, those of largest worth, ties to the lowest index.  A group's lanes compare it
// with some of the others each.
template <class F>
__device__ __forceinline__ bool group_stays(const ScoredArgs& g, const Share& s, F worth) {
    const int sub = (threadIdx.x & 31) & (s.group_lanes - 1);
    int above = 0;
    for (int h0 = 0; h0 < g.n_groups; h0 += s.group_lanes) {
        const int h = h0 + sub;
        const F w = __shfl_sync(0xffffffffu, worth, (h * s.group_lanes) & 31);
        above += h < g.n_groups && (w > worth || (w == worth && h < s.group));
    }
    for (int d = 1; d < s.group_lanes; d <<= 1) above += __shfl_xor_sync(0xffffffffu, above, d);
    return above < g.open_groups;
}

// The largest of the warp's values left, ties to the lowest index: lane j of [j0, j1) gets the expert (or keeps -1: none) and
// value of the j-th one.
template <class F, int PER>
__device__ __forceinline__ void take_largest(const Share& s, const F (&c)[PER], Best<F, PER>& b, int j0, int j1, int& mine, F& value) {
    const int lane = threadIdx.x & 31;
    for (int j = j0; j < j1; ++j) {
        const F most = warp_max(b.v1);
        if (!(most > kClosed<F>)) break;
        const int owner = __ffs(__ballot_sync(0xffffffffu, b.v1 == most)) - 1;
        const int e = __shfl_sync(0xffffffffu, s.first + b.at1, owner);
        if (lane == j) mine = e, value = most;
        if (lane == owner) b.pop(c);
    }
}

__device__ __forceinline__ double warp_sum64(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The choice in float64, for a pattern whose scores lie too near to one another for float32.
template <class T, int PER>
__device__ __noinline__ int choose64(const ScoredArgs& g, const T* z) {
    const Share s = share_of(g);
    const bool soft = g.scores == BP_SCORES_SOFTMAX;
    float v[PER], peak = kNone;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = i < s.count ? to_f32(z[s.first + i]) : kNone;
        peak = fmaxf(peak, v[i]);   // (not a NaN's)
    }
    double up[PER], total = 1.0;
    if (soft) {
        peak = warp_max(peak);   // (a number: a pattern that comes here has an open expert)
        total = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            up[i] = v[i] == peak ? 1.0 : v[i] > kNone ? exp((double)v[i] - (double)peak) : 0.0;
            total += up[i];
        }
        total = warp_sum64(total);
    }
    Order64 c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = 0ull;
        if (!(v[i] > kNone)) continue;
        double p = soft ? up[i] / total : 1.0 / (1.0 + exp(-(double)v[i]));
        if (g.bias != nullptr) p += (double)g.bias[s.first + i];
        c[i] = order64(p);
    }
    Best<Order64, PER> best;
    best.scan(c);
    if (g.n_groups > 1 && !group_stays(g, s, group_worth(g, s, best.v1, best.v2))) best.start();
    int mine = -1;
    Order64 value;
    take_largest(s, c, best, 0, g.r.k, mine, value);
    return mine;
}

// The experts of a list (lane j < n its j-th) by their float64 values, for sigmoid scores: lane j gets the j-th.
template <class T>
__device__ __forceinline__ int order_list(const ScoredArgs& g, const T* z, int mine, int n) {
    const int lane = threadIdx.x & 31;
    Order64 o = 0ull;
    if (lane < n) {
        double p = 1.0 / (1.0 + exp(-(double)to_f32(z[mine])));
        if (g.bias != nullptr) p += (double)g.bias[mine];
        o = order64(p);
    }
    int place = 0;
    for (int j = 0; j < n; ++j) {
        const Order64 x = __shfl_sync(0xffffffffu, o, j);
        const int e = __shfl_sync(0xffffffffu, mine, j);
        place += x > o || (x == o && e < mine);
    }
    int sorted = -1;
    for (int j = 0; j < n; ++j) {
        const int at = __shfl_sync(0xffffffffu, place, j), e = __shfl_sync(0xffffffffu, mine, j);
        if (lane == at) sorted = e;
    }
    return sorted;
}

// Gate of a chosen expert of logit z (live), by lane; every lane takes part.
__device__ __forceinline__ float share_of_chosen(const ScoredArgs& g, float z, bool live) {
    // Renormalised scores: a factor that all have in common drops out, which keeps them apart from zero.
    const float a = g.scores == BP_SCORES_SIGMOID ? fminf(z, 0.f) : z;
    const unsigned most = __reduce_max_sync(0xffffffffu, live ? order_of(a) : 0u);
    const float m = value_of(most);
    float w = 0.f;
    if (live) {
        w = a == m ? 1.f : expf(a - m);
        if (g.scores == BP_SCORES_SIGMOID) w /= 1.f + expf(-fabsf(z));
    }
    const float total = warp_sum(w);
    return live ? w / total : 0.f;
}

// e^x and 1 / x with the errors that k_route_scored counts.
__device__ __forceinline__ float fast_exp(float x) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A lane's logits, in 16-byte pieces where each lane has whole ones (`pieces`).
template <class T, int PER>
__device__ __forceinline__ void load_logits(const T* z, const Share& s, bool pieces, float (&v)[PER]) {
    constexpr int V = 16 / (int)sizeof(T);
    if constexpr (PER >= V) {
        if (pieces) {
#pragma unroll
            for (int i = 0; i < PER; i += V) {
                uint4 u = make_uint4(0u, 0u, 0u, 0u);
                if (i < s.count) u = __ldg(reinterpret_cast<const uint4*>(z + s.first + i));
                const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float x = sizeof(T) == 4 ? __uint_as_float(w[j % 4]) : __uint_as_float((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
                    v[i + j] = i < s.count ? x : kNone;
                }
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = i < s.count ? to_f32(z[s.first + i]) : kNone;
}

// A choice in float32, and again in float64 where two scores that it tells apart (or two groups) are nearer
// than float32 can: the choice is that of float64 scores.  Errors of float32 scores, with x log2(e) half a unit off,
// 2^x and a quotient two units each:  e^x is off by |x| 9e-8 + 3e-7 of itself, so that a sigmoid s is by
// s (1 - s) (|x| 9e-8 + 3e-7) + s 3e-7, at most 5e-7, and of itself at most 1e-5 (|x| up to 88); a softmax 1e-5 of itself (its
// difference from the peak is half a unit off too, |x| 6e-8, and a sum of 512 terms 2^-19).  Scores below e^-88 are
// as good as none.
template <class T, int PER, bool ONE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kThreads && PER <= 8 ? 4 : 1) k_route_scored(ScoredArgs g) {
    constexpr int kPatterns = ONE ? kOneBlock : kRoutePatterns, kWords = kPatterns / 32;
    __shared__ unsigned bits[BP_MAX_EXPERTS * kWords];
    __shared__ int base[ONE ? BP_MAX_EXPERTS : 1];
    __shared__ int warp_tot[32];
    __shared__ float2 lists[THREADS / 32][32];   // a warp's values and experts
    pdl_launch();
    const int p0 = blockIdx.x * kPatterns, np = min(kPatterns, g.r.n - p0), E = g.E;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Share s = share_of(g);
    const bool soft = g.scores == BP_SCORES_SOFTMAX;
    const T* z = (const T*)g.r.logits + (size_t)(p0 + warp) * E;
    float v[PER];
    if (warp < np) load_logits(z, s, g.pieces, v);
    for (int i = threadIdx.x; i < E * kWords; i += THREADS) bits[i] = 0u;
    float b[PER], b_most = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        b[i] = g.bias != nullptr && i < s.count ? __ldg(g.bias + s.first + i) : 0.f;
        if (!(b[i] > kNone)) b[i] = kNone;   // (no bias of its own: closed)
        else b_most = fmaxf(b_most, fabsf(b[i]));
    }
    b_most = warp_max(b_most);
    __syncthreads();
    for (int p = warp; p < np; p += THREADS / 32) {
        bool nan = false;
        float c[PER], peak = 0.f, total = 1.f, most = 1.f;   // most: the largest score, at most
#pragma unroll
        for (int i = 0; i < PER; ++i) nan |= v[i] != v[i];
        nan = __any_sync(0xffffffffu, nan);
        if (soft) {
            peak = v[0];
#pragma unroll
            for (int i = 1; i < PER; ++i) peak = fmaxf(peak, v[i]);   // (not a NaN's)
            peak = warp_max(peak);
            total = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = v[i] == peak ? 1.f : fast_exp(v[i] - peak);
                total += v[i] > kNone ? c[i] : 0.f;
            }
            total = warp_sum(total);
            most = fast_reciprocal(total);
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = v[i] > kNone ? fmaf(c[i], most, b[i]) : kNone;
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) c[i] = v[i] > kNone ? fast_reciprocal(1.f + fast_exp(-v[i])) + b[i] : kNone;
        }
        const float unit = soft ? 1e-5f : 5e-7f;   // (of `most`: of itself, 1e-5)
        const float err = unit * most + 1.2e-7f * (1.f + b_most);   // of any score and its bias
        bool near = false, near_groups = false, open = true;
        float m1 = c[0], m2 = kNone;   // the lane's two largest
#pragma unroll
        for (int i = 1; i < PER; ++i) {
            m2 = fmaxf(m2, fminf(m1, c[i]));
            m1 = fmaxf(m1, c[i]);
        }
        if (g.n_groups > 1) {
            const float worth = group_worth(g, s, m1, m2);
            const bool real = s.group < g.n_groups;
            open = group_stays(g, s, worth);
            const float kept = -warp_max(real && open ? -worth : kNone), left = warp_max(real && !open ? worth : kNone);
            near = near_groups = left > kNone && !(kept - left > 6.f * err);   // (a worth is off by 2 err, and by its sum's rounding)
            if (!open) m1 = kNone;
        }
        // The values from the (k + 3)-th largest lane's largest on: as many as are wanted, and some more (so that the last choice
        // is hardly ever too near to what is not among them).  They go to a lane each, in the experts' order, and from there to the place that they have by size.
        float least = kNone;
        {
            float t = m1;
            for (int j = 0; j < g.r.k + 3; ++j) {
                least = warp_max(t);
                if (!(least > kNone)) break;
                t = t == least ? kNone : t;
            }
        }
        unsigned found = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) found |= open && c[i] > kNone && c[i] >= least ? 1u << i : 0u;
        int upto = __popc(found);
        const int own = upto;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        int taken = __shfl_sync(0xffffffffu, upto, 31);   // entries of the list
        const bool listed = taken <= 32;                   // the list has them all
        bool whole = !(least > kNone);                     // there are no others
        int mine = -1;
        float value = kNone;
        if (listed) {
            int at = upto - own;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (found >> i & 1) lists[warp][at++] = make_float2(c[i], __int_as_float(s.first + i));
            __syncwarp();
            const float2 entry = lane < taken ? lists[warp][lane] : make_float2(kNone, 0.f);
            int place = 0;
            for (int j = 0; j < taken; ++j) {
                const float x = __shfl_sync(0xffffffffu, entry.x, j);
                place += x > entry.x || (x == entry.x && j < lane);
            }
            __syncwarp();
            if (lane < taken) lists[warp][place] = entry;
            __syncwarp();
            if (lane < taken) value = lists[warp][lane].x, mine = __float_as_int(lists[warp][lane].y);
            __syncwarp();
        } else {   // more of them: one after another
            Best<float, PER> best;
            best.scan(c);
            if (!open) best.start();
            taken = g.r.k + 9;
            whole = false;
            take_largest(s, c, best, 0, taken, mine, value);
        }
        // Whether the choice can be told from the list.  Equal logits with equal biases are equal in float64 too; where
        // the last choice has such equals behind it, what comes after them has to be far enough away.
        if (!near) {
            const float next = __shfl_down_sync(0xffffffffu, value, 1);
            const bool close = lane < taken - 1 && next > kNone &&
                               !(value - next > (g.bias != nullptr ? 2.f * err : 2e-5f * value + 1e-36f));
            if (__any_sync(0xffffffffu, close)) {
                const float logit = mine >= 0 ? to_f32(z[mine]) : 0.f, bias = mine >= 0 && g.bias != nullptr ? __ldg(g.bias + mine) : 0.f;
                const float next_logit = __shfl_down_sync(0xffffffffu, logit, 1), next_bias = __shfl_down_sync(0xffffffffu, bias, 1);
                const bool same = logit == next_logit && bias == next_bias;
                const unsigned last = 1u << (g.r.k - 1), unlike = __ballot_sync(0xffffffffu, close && !same);
                const unsigned run = __ballot_sync(0xffffffffu, close && same) & ~(last - 1);   // of equals, from the last choice on
                const unsigned behind = (run + last) & ~run;                                     // the first place that is not
                near = (unlike & ((last - 1) | behind)) != 0 || (!whole && behind >= 1u << (taken - 1));
            }
        }
        if (near) {
            // The list again by float64 scores, where float32 can tell that it has every expert of the choice (sigmoid scores: they are
            // each their own); else all experts.
            const float kth = __shfl_sync(0xffffffffu, value, g.r.k - 1);
            if (!near_groups && !soft && listed && (whole || kth - least > 2.f * err)) mine = order_list(g, z, mine, taken);
            else mine = choose64<T, PER>(g, z);
        }
        if (lane >= g.r.k) mine = -1;
        const bool live = mine >= 0;
        const float logit = live ? to_f32(z[mine]) : kNone;
        z += (size_t)(THREADS / 32) * E;
        if (p + THREADS / 32 < np) load_logits(z, s, g.pieces, v);
        float gate;
        if (g.renormalise) gate = share_of_chosen(g, logit, live);
        else if (soft) gate = live ? (logit == peak ? 1.f : expf(logit - peak)) / total : 0.f;
        else gate = live ? 1.f / (1.f + expf(-logit)) : 0.f;
        if (live) atomicOr(&bits[mine * kWords + (p >> 5)], 1u << (p & 31));
        if (lane < g.r.k) {
            const size_t i = (size_t)(p0 + p) * g.r.k + lane;
            g.r.expert[i] = mine;
            g.r.gate[i] = !live ? 0.f : nan ? NAN : g.scale * gate;
        }
    }
    __syncthreads();
    if constexpr (!ONE) {
        for (int e = threadIdx.x; e < E; e += THREADS) g.r.hist[(size_t)e * (gridDim.x + 1) + blockIdx.x] = count_of<kWords>(bits, e);
    } else {
        for (int e = threadIdx.x; e < E; e += THREADS) base[e] = count_of<kWords>(bits, e);
        __syncthreads();
        const int rows = block_scan(base, E, warp_tot);
        for (int e = threadIdx.x; e < E; e += THREADS) g.r.offsets[e] = base[e];
        if (threadIdx.x == 0) g.r.offsets[E] = rows;
        for (int i = rows + threadIdx.x; i < g.r.n * g.r.k; i += THREADS) g.r.source[i] = -1;
        place_rows<kWords>(g.r, bits, base, p0, np);
    }
}

// Gradient of the gates by the logits, a warp a pattern, its row put together in shared memory.  Reads the chosen
// logits, and all of them for a softmax over all; writes every place.
template <class T>
__global__ void __launch_bounds__(kBackThreads) k_route_scored_backward(ScoredArgs g, const float* dgate, T* dz) {
    __shared__ float rows[kBackThreads / 32][BP_MAX_EXPERTS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = g.E;
    const long long p = (long long)blockIdx.x * (kBackThreads / 32) + warp;
    if (p >= g.r.n) return;
    float* row = rows[warp];
    const T* z = (const T*)g.r.logits + (size_t)p * E;
    const int e = lane < g.r.k ? g.r.expert[(size_t)p * g.r.k + lane] : -1;
    const bool live = (unsigned)e < (unsigned)E, soft = g.scores == BP_SCORES_SOFTMAX;
    const float logit = live ? to_f32(z[e]) : -INFINITY;
    const float u = live ? g.scale * dgate[(size_t)p * g.r.k + lane] : 0.f;
    float share, d, rest = 0.f;   // of the chosen; rest: what a score of a softmax over all is multiplied by
    float peak = 0.f, total = 1.f;
    if (soft && !g.renormalise) {
        float m = -INFINITY;
        bool nan = false;
        for (int i = lane; i < E; i += 32) {
            const float x = to_f32(z[i]);
            row[i] = x;
            m = fmaxf(m, x);
            nan |= x != x;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        peak = __any_sync(0xffffffffu, nan) ? NAN : m;
        float sum = 0.f;
        for (int i = lane; i < E; i += 32) {
            const float x = row[i] == peak ? 1.f : row[i] == -INFINITY ? 0.f : expf(row[i] - peak);
            row[i] = x;
            sum += x;
        }
        total = warp_sum(sum);
        share = live ? (logit == peak ? 1.f : expf(logit - peak)) / total : 0.f;
        const float pull = warp_sum(share * u);
        rest = __any_sync(0xffffffffu, live) ? -pull / total : 0.f;
        d = share * (u - pull);
    } else {
        for (int i = lane; i < E; i += 32) row[i] = 0.f;
        if (g.renormalise) {
            share = share_of_chosen(g, logit, live);
            d = share * (u - warp_sum(share * u));
        } else {
            share = live ? 1.f / (1.f + expf(-logit)) : 0.f;
            d = share * u;
        }
        if (!soft) d *= 1.f / (1.f + expf(logit));   // 1 - sigmoid
    }
    __syncwarp();
    if (rest != 0.f)
        for (int i = lane; i < E; i += 32) row[i] *= rest;
    else if (soft && !g.renormalise)
        for (int i = lane; i < E; i += 32) row[i] = 0.f;
    __syncwarp();
    if (live) row[e] = d;
    __syncwarp();
    T* out = dz + (size_t)p * E;
    for (int i = lane; i < E; i += 32) out[i] = from_f32<T>(row[i]);
}

template <class T, int PER>
cudaError_t launch(const ScoredArgs& a, int blocks, cudaStream_t s) {
    constexpr int kMany = PER <= 8 ? 1024 : 512;
    if (a.r.n <= kOneBlock) k_route_scored<T, PER, true, kMany><<<1, kMany, 0, s>>>(a);
    else if (blocks <= a.num_sms) k_route_scored<T, PER, false, kMany><<<blocks, kMany, 0, s>>>(a);   // a pattern a warp
    else k_route_scored<T, PER, false, kThreads><<<blocks, kThreads, 0, s>>>(a);
    return cudaGetLastError();
}
template <class T>
cudaError_t launch(const ScoredArgs& a, int blocks, cudaStream_t s) {
    if (a.per <= 1) return launch<T, 1>(a, blocks, s);
    if (a.per <= 2) return launch<T, 2>(a, blocks, s);
    if (a.per <= 4) return launch<T, 4>(a, blocks, s);
    if (a.per <= 8) return launch<T, 8>(a, blocks, s);
    if (a.per <= 16) return launch<T, 16>(a, blocks, s);
    return launch<T, 32>(a, blocks, s);
}

}  // namespace

cudaError_t route_scored_forward(ScoredArgs a, cudaStream_t s) {
    a.group_lanes = 32;
    while (32 / a.group_lanes < a.n_groups) a.group_lanes /= 2;
    a.per = (a.E / a.n_groups + a.group_lanes - 1) / a.group_lanes;
    const int size = a.r.dtype == BP_F32 ? 4 : 2, whole = 16 / size;   // rows of which every lane has whole 16-byte pieces, or none
    a.pieces = a.per % whole == 0 && a.E / a.n_groups % whole == 0 && ((uintptr_t)a.r.logits & 15) == 0;
    const bool one = a.r.n <= kOneBlock;
    const int blocks = one ? 1 : (a.r.n + kRoutePatterns - 1) / kRoutePatterns;
    const cudaError_t e = a.r.dtype == BP_F32 ? launch<float>(a, blocks, s) : launch<__nv_bfloat16>(a, blocks, s);
    return one || e != cudaSuccess ? e : route_order(a.r, s);
}

cudaError_t route_scored_backward(const ScoredArgs& a, const float* dgate, void* dlogits, cudaStream_t s) {
    const int per = kBackThreads / 32, blocks = (a.r.n + per - 1) / per;
    if (a.r.dtype == BP_F32) k_route_scored_backward<float><<<blocks, kBackThreads, 0, s>>>(a, dgate, (float*)dlogits);
    else k_route_scored_backward<__nv_bfloat16><<<blocks, kBackThreads, 0, s>>>(a, dgate, (__nv_bfloat16*)dlogits);
    return cudaGetLastError();
}

}  // namespace bp
