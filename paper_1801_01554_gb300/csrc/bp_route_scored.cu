// The router by scores: k experts of each pattern by softmax or sigmoid scores and a bias, within the pattern's best
// groups of experts, their gates, and the gates' gradient.
#include <cmath>

#include "bp_route_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256, kBackThreads = 256;
constexpr int kOneBlock = 256;   // patterns of a call that one block takes

// A warp takes a pattern: each group of experts has 32 / (groups, rounded up to a power of two) lanes, a lane
// `per` consecutive experts of its group.  So the lowest index among equals is the first lane's first.
struct Share {
    int first, count, group, group_lanes;
    bool leads;   // the first lane of a group
};
__device__ __forceinline__ Share share_of(const ScoredArgs& g) {
    const int lane = threadIdx.x & 31, size = g.E / g.n_groups, sub = lane % g.group_lanes;
    Share s;
    s.group = lane / g.group_lanes;
    s.group_lanes = g.group_lanes;
    s.first = s.group * size + sub * g.per;
    s.count = s.group < g.n_groups ? min(max(size - sub * g.per, 0), g.per) : 0;
    s.leads = s.group < g.n_groups && sub == 0;
    return s;
}

using bp::order_of;
__device__ __forceinline__ double order_value(unsigned long long o) {
    return __longlong_as_double((long long)((o >> 63) ? (o & 0x7fffffffffffffffull) : ~o));
}
__device__ __forceinline__ unsigned long long order_of(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    if (!(x > -INFINITY)) return 0ull;
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ float order_value(unsigned o) { return value_of(o); }
__device__ __forceinline__ unsigned warp_most(unsigned x) { return __reduce_max_sync(0xffffffffu, x); }
__device__ __forceinline__ unsigned long long warp_most(unsigned long long x) {
    const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(x >> 32));
    const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(x >> 32) == hi ? (unsigned)x : 0u);
    return ((unsigned long long)hi << 32) | lo;
}

// Closes the groups beyond the open ones of largest value.  With err > 0: whether two groups on either side
// are nearer to one another than that.
template <class F, class K, int PER>
__device__ __forceinline__ bool close_groups(const ScoredArgs& g, const Share& s, K (&o)[PER], F err) {
    F m1 = -INFINITY, m2 = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const F x = o[i] != 0 ? (F)order_value(o[i]) : (F)-INFINITY;
        m2 = max(m2, min(m1, x));
        m1 = max(m1, x);
    }
    for (int d = 1; d < s.group_lanes; d <<= 1) {
        const F p1 = __shfl_xor_sync(0xffffffffu, m1, d), p2 = __shfl_xor_sync(0xffffffffu, m2, d);
        m2 = max(min(m1, p1), max(m2, p2));
        m1 = max(m1, p1);
    }
    const F worth = g.group_top == 2 && m2 > (F)-INFINITY ? m1 + m2 : m1;   // (-infinity: a group with none open)
    int above = 0;
    for (int h = 0; h < g.n_groups; ++h) {
        const F w = __shfl_sync(0xffffffffu, worth, h * s.group_lanes);
        above += w > worth || (w == worth && h < s.group);
    }
    const bool stays = above < g.open_groups;
    bool near = false;
    if (err > (F)0) {
        const K kept = warp_most(s.leads && stays ? ~order_of(worth) : (K)0);    // the least of those that stay
        const K left = warp_most(s.leads && !stays ? order_of(worth) : (K)0);
        near = left != 0 && !((F)order_value((K)~kept) - (F)order_value(left) > err);
    }
    if (!stays)
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = 0;
    return near;
}

// The `rounds` largest of the warp's values, ties to the lowest index: lane j gets the j-th one's expert (-1: none) and order.
template <class K, int PER>
__device__ __forceinline__ void take_largest(const Share& s, K (&o)[PER], int rounds, int& mine, K& order) {
    const int lane = threadIdx.x & 31;
    mine = -1;
    order = 0;
    K best = 0;
    int at = 0;
    const auto again = [&] {
        best = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (o[i] > best) best = o[i], at = i;
    };
    again();
    for (int j = 0; j < rounds; ++j) {
        const K most = warp_most(best);
        if (most == 0) break;
        const int owner = __ffs(__ballot_sync(0xffffffffu, best == most)) - 1;
        const int e = __shfl_sync(0xffffffffu, s.first + at, owner);
        if (lane == j) mine = e, order = most;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (i == at) o[i] = 0;
            again();
        }
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
    unsigned long long o[PER];
    double v[PER], peak = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = i < s.count ? (double)to_f32(z[s.first + i]) : -INFINITY;
        if (v[i] > peak) peak = v[i];
    }
    double total = 1.0;
    if (g.scores == BP_SCORES_SOFTMAX) {
        peak = order_value(warp_most(order_of(peak)));   // (a pattern with an open expert: there is one)
        total = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) total += v[i] > -INFINITY ? (v[i] == peak ? 1.0 : exp(v[i] - peak)) : 0.0;
        total = warp_sum64(total);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        o[i] = 0;
        if (!(v[i] > -INFINITY)) continue;
        const double p = g.scores == BP_SCORES_SOFTMAX ? (v[i] == peak ? 1.0 : exp(v[i] - peak)) / total : 1.0 / (1.0 + exp(-v[i]));
        o[i] = order_of(g.bias != nullptr ? p + (double)g.bias[s.first + i] : p);
    }
    if (g.n_groups > 1) close_groups<double>(g, s, o, 0.0);
    int mine;
    unsigned long long order;
    take_largest(s, o, g.r.k, mine, order);
    return mine;
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

// A choice in float32, and again in float64 where two scores that it tells apart (or two groups) are nearer
// than float32 can: the choice is that of float64 scores.  Errors of float32 scores: a sigmoid 2^-21 of itself
// (expf 2 units, a sum and a quotient); a softmax 1e-5 of itself (its difference from the peak half a unit of up to 90,
// 2^-17.5; a sum of 512 terms 2^-19), and nothing that matters below e^-90.
template <class T, int PER, bool ONE>
__global__ void __launch_bounds__(ONE ? (PER <= 8 ? 1024 : 512) : kThreads) k_route_scored(ScoredArgs g) {
    constexpr int kBlock = ONE ? (PER <= 8 ? 1024 : 512) : kThreads;
    constexpr int kPatterns = ONE ? kOneBlock : kRoutePatterns, kWords = kPatterns / 32;
    __shared__ unsigned bits[BP_MAX_EXPERTS * kWords];
    __shared__ int base[ONE ? BP_MAX_EXPERTS : 1];
    __shared__ int warp_tot[32];
    pdl_launch();
    const int p0 = blockIdx.x * kPatterns, np = min(kPatterns, g.r.n - p0), E = g.E;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < E * kWords; i += kBlock) bits[i] = 0u;
    __syncthreads();
    const Share s = share_of(g);
    const bool soft = g.scores == BP_SCORES_SOFTMAX;
    float b[PER], b_most = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        b[i] = g.bias != nullptr && i < s.count ? g.bias[s.first + i] : 0.f;
        b_most = fmaxf(b_most, fabsf(b[i]));
    }
    b_most = value_of(__reduce_max_sync(0xffffffffu, order_of(b_most)));
    for (int p = warp; p < np; p += kBlock / 32) {
        const T* z = (const T*)g.r.logits + (size_t)(p0 + p) * E;
        float v[PER];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = i < s.count ? to_f32(z[s.first + i]) : -INFINITY;
            nan |= v[i] != v[i];
        }
        nan = __any_sync(0xffffffffu, nan);
        unsigned o[PER];
        float peak = 0.f, total = 1.f, most = 1.f;   // most: the largest score, at most
        if (soft) {
            unsigned top = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) top = max(top, order_of(v[i]));
            peak = value_of(__reduce_max_sync(0xffffffffu, top));
            total = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                o[i] = __float_as_uint(v[i] == peak ? 1.f : v[i] > -INFINITY ? expf(v[i] - peak) : 0.f);
                total += __uint_as_float(o[i]);
            }
            total = warp_sum(total);
            most = 1.f / total;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const float score = soft ? __uint_as_float(o[i]) / total : 1.f / (1.f + expf(-v[i]));
            o[i] = v[i] > -INFINITY ? order_of(score + b[i]) : 0u;
        }
        const float unit = soft ? 1e-5f : 5e-7f;
        const float err = unit * most + 1.2e-7f * (1.f + b_most);   // of any score and its bias
        bool near = false;
        if (g.n_groups > 1) near = close_groups<float>(g, s, o, 6.f * err);
        int mine;
        unsigned order;
        take_largest(s, o, g.r.k + 1, mine, order);
        float logit = mine >= 0 ? to_f32(z[mine]) : -INFINITY;
        {   // each choice against the next one; equal logits with equal biases are equal in float64 too
            const float bias = mine >= 0 && g.bias != nullptr ? g.bias[mine] : 0.f;
            const int next = __shfl_down_sync(0xffffffffu, mine, 1);
            const unsigned next_order = __shfl_down_sync(0xffffffffu, order, 1);
            const float next_logit = __shfl_down_sync(0xffffffffu, logit, 1), next_bias = __shfl_down_sync(0xffffffffu, bias, 1);
            if (lane < g.r.k && next >= 0 && !(logit == next_logit && bias == next_bias)) {
                const float x = value_of(order);
                near |= !(x - value_of(next_order) > (g.bias != nullptr ? 2.f * err : 2.f * unit * x + 1e-36f));
            }
        }
        if (__any_sync(0xffffffffu, near)) {
            mine = choose64<T, PER>(g, z);
            logit = mine >= 0 ? to_f32(z[mine]) : -INFINITY;
        }
        if (lane >= g.r.k) mine = -1;
        const bool live = mine >= 0;
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
        for (int e = threadIdx.x; e < E; e += kBlock) g.r.hist[(size_t)e * (gridDim.x + 1) + blockIdx.x] = count_of<kWords>(bits, e);
    } else {
        for (int e = threadIdx.x; e < E; e += kBlock) base[e] = count_of<kWords>(bits, e);
        __syncthreads();
        const int rows = block_scan(base, E, warp_tot);
        for (int e = threadIdx.x; e < E; e += kBlock) g.r.offsets[e] = base[e];
        if (threadIdx.x == 0) g.r.offsets[E] = rows;
        for (int i = rows + threadIdx.x; i < g.r.n * g.r.k; i += kBlock) g.r.source[i] = -1;
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
    if (blocks == 1 && a.r.n <= kOneBlock) k_route_scored<T, PER, true><<<1, PER <= 8 ? 1024 : 512, 0, s>>>(a);
    else k_route_scored<T, PER, false><<<blocks, kThreads, 0, s>>>(a);
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
