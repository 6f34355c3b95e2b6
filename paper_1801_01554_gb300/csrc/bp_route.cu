// The router (choice of k experts, gates, order of the rows by expert) and the mix of the
// experts' outputs, with their gradients.
#include <cmath>

#include "bp_experts_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

// A call of up to kOneBlock patterns is one block of 1,024 threads, which orders its rows too: one
// launch.  Longer ones take blocks of kRoutePatterns patterns, four a warp, and two more launches for
// the order (16,384 patterns of 64 experts: 128 patterns a block took 21 us for the choice alone).
constexpr int kOneBlock = 256, kOneThreads = 1024;
constexpr int kRouteThreads = 256;

// Ascending whole numbers for ascending floats; 0 for NaN and for -infinity, which are never
// chosen.  (x + 0 turns -0 into +0, so that the two tie.)
__device__ __forceinline__ unsigned order_of(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    if (!(x > -INFINITY)) return 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned o) {
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A block's patterns that chose expert e, as bits: bits[e * kWords + word].
template <int kWords>
__device__ __forceinline__ int rank_of(const unsigned* bits, int e, int p) {
    int r = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const unsigned m = p >= 32 * (w + 1) ? 0xffffffffu : p > 32 * w ? (1u << (p - 32 * w)) - 1u : 0u;
        r += __popc(bits[e * kWords + w] & m);
    }
    return r;
}
template <int kWords>
__device__ __forceinline__ int count_of(const unsigned* bits, int e) {
    int r = 0;
#pragma unroll
    for (int w = 0; w < kWords; ++w) r += __popc(bits[e * kWords + w]);
    return r;
}

// Rows of a block's choices: base[e] is the row of the block's first pattern with expert e.
template <int kWords>
__device__ __forceinline__ void place_rows(const RouteArgs& g, const unsigned* bits, const int* base, int p0, int np) {
    for (int i = threadIdx.x; i < np * g.k; i += blockDim.x) {
        const int p = i / g.k, e = g.expert[(size_t)p0 * g.k + i];
        int at = -1;
        if (e >= 0) {
            at = base[e] + rank_of<kWords>(bits, e, p);
            g.source[at] = p0 + p;
        }
        g.place[(size_t)p0 * g.k + i] = at;
    }
}

// Exclusive sums of cnt[0 .. E) by the block, and the total.
__device__ __forceinline__ int block_scan(int* cnt, int E, int* warp_tot) {
    int carry = 0;
    for (int b = 0; b < E; b += blockDim.x) {
        const int i = b + threadIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
        const int x = i < E ? cnt[i] : 0;
        int s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        __syncthreads();
        if (lane == 31) warp_tot[w] = s;
        __syncthreads();
        int before = carry;
        for (int v = 0; v < (int)blockDim.x / 32; ++v) {
            if (v < w) before += warp_tot[v];
            carry += warp_tot[v];
        }
        if (i < E) cnt[i] = before + s - x;
    }
    __syncthreads();
    return carry;
}

// A warp a pattern, lane l with the logits of experts l, l + 32, ..: k times the largest one
// left (by its order, then by the lowest index).
template <class T, int PER, bool ONE>
__global__ void __launch_bounds__(ONE ? kOneThreads : kRouteThreads) k_route(RouteArgs g) {
    constexpr int kPatterns = ONE ? kOneBlock : kRoutePatterns, kThreads = ONE ? kOneThreads : kRouteThreads;
    constexpr int kWords = kPatterns / 32;
    __shared__ unsigned bits[BP_MAX_EXPERTS * kWords];
    __shared__ int base[ONE ? BP_MAX_EXPERTS : 1];
    __shared__ int warp_tot[32];
    pdl_launch();
    const int p0 = blockIdx.x * kPatterns, np = min(kPatterns, g.n - p0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < g.E * kWords; i += kThreads) bits[i] = 0u;
    __syncthreads();
    for (int p = warp; p < np; p += kThreads / 32) {
        const T* z = (const T*)g.logits + (size_t)(p0 + p) * g.E;
        unsigned o[PER];
        float v[PER];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane + 32 * i;
            v[i] = e < g.E ? to_f32(z[e]) : -INFINITY;
            nan |= v[i] != v[i];
            o[i] = order_of(v[i]);
        }
        nan = __any_sync(0xffffffffu, nan);
        int mine = -1;         // lane j keeps choice j
        float logit = -INFINITY, peak = 0.f;
        for (int j = 0; j < g.k; ++j) {
            unsigned best = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) best = max(best, o[i]);
            best = __reduce_max_sync(0xffffffffu, best);
            if (best == 0) break;
            unsigned at = 0xffffffffu;
#pragma unroll
            for (int i = PER - 1; i >= 0; --i)
                if (o[i] == best) at = lane + 32 * i;
            at = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (at == lane + 32 * i) o[i] = 0u;
            if (j == 0) peak = value_of(best);
            if (lane == j) {
                mine = (int)at;
                logit = value_of(best);
            }
            if (lane == 0) atomicOr(&bits[at * kWords + (p >> 5)], 1u << (p & 31));
        }
        float up = mine >= 0 ? expf(logit - peak) : 0.f, total;
        if (g.gates == BP_GATES_ALL) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) total += lane + 32 * i < g.E ? expf(v[i] - peak) : 0.f;
            total = warp_sum(total);
        } else {
            total = warp_sum(up);
        }
        if (lane < g.k) {
            const size_t i = (size_t)(p0 + p) * g.k + lane;
            g.expert[i] = mine;
            g.gate[i] = mine < 0 ? 0.f : nan ? NAN : up / total;
        }
    }
    __syncthreads();
    if constexpr (!ONE) {
        for (int e = threadIdx.x; e < g.E; e += kThreads) g.hist[(size_t)e * (gridDim.x + 1) + blockIdx.x] = count_of<kWords>(bits, e);
    } else {
        for (int e = threadIdx.x; e < g.E; e += kThreads) base[e] = count_of<kWords>(bits, e);
        __syncthreads();
        const int total = block_scan(base, g.E, warp_tot);
        for (int e = threadIdx.x; e < g.E; e += kThreads) g.offsets[e] = base[e];
        if (threadIdx.x == 0) g.offsets[g.E] = total;
        for (int i = total + threadIdx.x; i < g.n * g.k; i += kThreads) g.source[i] = -1;
        place_rows<kWords>(g, bits, base, p0, np);
    }
}

// An expert's counts, block after block, turned into its rows before each block, and their total
// behind them: hist is [E, blocks + 1], a CTA an expert.
__global__ void __launch_bounds__(kRouteThreads) k_route_columns(RouteArgs g, int blocks) {
    __shared__ int warp_tot[32];
    __shared__ int cnt[kRouteThreads];
    pdl_launch();
    pdl_wait();
    int* h = g.hist + (size_t)blockIdx.x * (blocks + 1);
    int carry = 0;
    for (int b = 0; b < blocks; b += kRouteThreads) {
        const int i = b + threadIdx.x;
        cnt[threadIdx.x] = i < blocks ? h[i] : 0;
        const int total = block_scan(cnt, kRouteThreads, warp_tot);
        if (i < blocks) h[i] = carry + cnt[threadIdx.x];
        carry += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) h[blocks] = carry;
}

// Rows of every block's choices, from the counts.
__global__ void __launch_bounds__(kRouteThreads) k_route_place(RouteArgs g) {
    constexpr int kWords = kRoutePatterns / 32;
    __shared__ unsigned bits[BP_MAX_EXPERTS * kWords];
    __shared__ int base[BP_MAX_EXPERTS];
    __shared__ int warp_tot[32];
    const int p0 = blockIdx.x * kRoutePatterns, np = min(kRoutePatterns, g.n - p0);
    for (int i = threadIdx.x; i < g.E * kWords; i += kRouteThreads) bits[i] = 0u;
    pdl_wait();
    const int* h = g.hist;
    for (int e = threadIdx.x; e < g.E; e += kRouteThreads) base[e] = h[(size_t)e * (gridDim.x + 1) + gridDim.x];
    __syncthreads();
    for (int i = threadIdx.x; i < np * g.k; i += kRouteThreads) {
        const int p = i / g.k, e = g.expert[(size_t)p0 * g.k + i];
        if (e >= 0) atomicOr(&bits[e * kWords + (p >> 5)], 1u << (p & 31));
    }
    const int total = block_scan(base, g.E, warp_tot);
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < g.E; e += kRouteThreads) g.offsets[e] = base[e];
        if (threadIdx.x == 0) g.offsets[g.E] = total;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < g.E; e += kRouteThreads) base[e] += h[(size_t)e * (gridDim.x + 1) + blockIdx.x];
    __syncthreads();
    for (int i = p0 * g.k + threadIdx.x; i < (p0 + np) * g.k; i += kRouteThreads)
        if (i >= total) g.source[i] = -1;
    place_rows<kWords>(g, bits, base, p0, np);
}

// Gradient of the gates: dz = p (.. ) for every expert with gates over all, for the chosen ones else.
template <class T>
__global__ void __launch_bounds__(kRouteThreads) k_route_backward(RouteArgs g, const float* dgate, T* dz) {
    const int p = blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (p >= g.n) return;
    const size_t c = (size_t)p * g.k + lane;
    const int e = lane < g.k ? g.expert[c] : -1;
    const float gate = e >= 0 ? g.gate[c] : 0.f;
    const float own = e >= 0 ? gate * dgate[c] : 0.f;   // g_j dg_j
    const float pull = warp_sum(own);
    const T* z = (const T*)g.logits + (size_t)p * g.E;
    T* out = dz + (size_t)p * g.E;
    float peak = 0.f, total = 1.f;
    const bool any = __any_sync(0xffffffffu, e >= 0);
    if (g.gates == BP_GATES_ALL && any) {
        float m = -INFINITY;
        bool nan = false;
        for (int i = lane; i < g.E; i += 32) {
            const float x = to_f32(z[i]);
            m = fmaxf(m, x);
            nan |= x != x;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        peak = __any_sync(0xffffffffu, nan) ? NAN : m;
        float s = 0.f;
        for (int i = lane; i < g.E; i += 32) s += expf(to_f32(z[i]) - peak);
        total = warp_sum(s);
    }
    for (int b = 0; b < g.E; b += 32) {
        const int i = b + lane;
        float d = 0.f;
        if (g.gates == BP_GATES_ALL && any && i < g.E) d = -(expf(to_f32(z[i]) - peak) / total) * pull;
        for (int j = 0; j < g.k; ++j) {   // the choice that names this expert, if any
            const int ej = __shfl_sync(0xffffffffu, e, j);
            const float oj = __shfl_sync(0xffffffffu, own, j), gj = __shfl_sync(0xffffffffu, gate, j);
            if (ej == i && ej >= 0) d += g.gates == BP_GATES_ALL ? oj : oj - gj * pull;
        }
        if (i < g.E) out[i] = from_f32<T>(d);
    }
}

// ------------------------------------------------------------ mix
// V values a lane and step: 16 bytes of a row where rows are whole 16-byte pieces.
template <class T, int V>
struct Piece {
    float v[V];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (V == 1) {
            v[0] = to_f32(*p);
        } else if constexpr (sizeof(T) == 4) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (V == 1) {
            *p = from_f32<T>(v[0]);
        } else if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            __align__(16) __nv_bfloat162 h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(h);
        }
    }
};

constexpr int kMixThreads = 256;

// `warps` warps a pattern, each on every warps-th run of 32 V columns.
template <class T, int V>
__global__ void __launch_bounds__(kMixThreads) k_mix(MixArgs g) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = kMixThreads / 32 / g.warps;
    const int t = blockIdx.x * per + warp / g.warps, part = warp % g.warps;
    if (t >= g.n) return;
    int row = -1;
    float gate = 0.f;
    if (lane < g.k) {
        row = g.place[(size_t)t * g.k + lane];
        if ((unsigned)row >= (unsigned)g.n_rows) row = -1;
        gate = g.gate == nullptr ? 1.f : g.gate[(size_t)t * g.k + lane];
    }
    const T* H = (const T*)g.H;
    for (int c = (part * 32 + lane) * V; c - lane * V < g.N; c += g.warps * 32 * V) {
        Piece<T, V> y{}, h;
        for (int j = 0; j < g.k; ++j) {
            const int r = __shfl_sync(0xffffffffu, row, j);
            const float w = __shfl_sync(0xffffffffu, gate, j);
            if (r < 0 || c >= g.N) continue;
            h.load(H + (size_t)r * g.N + c);
#pragma unroll
            for (int i = 0; i < V; ++i) y.v[i] = fmaf(w, h.v[i], y.v[i]);
        }
        if (c < g.N) y.store((T*)g.Y + (size_t)t * g.N + c);
    }
}

template <class T, int V>
__global__ void __launch_bounds__(kMixThreads) k_mix_backward(MixArgs g) {
    __shared__ float dots[kMixThreads / 32][BP_MAX_CHOICES];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = kMixThreads / 32 / g.warps;
    const int t = blockIdx.x * per + warp / g.warps, part = warp % g.warps;
    const bool live = t < g.n;
    int row = -1;
    float gate = 0.f;
    if (live && lane < g.k) {
        row = g.place[(size_t)t * g.k + lane];
        if ((unsigned)row >= (unsigned)g.n_rows) row = -1;
        gate = g.gate == nullptr ? 1.f : g.gate[(size_t)t * g.k + lane];
    }
    const T *H = (const T*)g.H, *D = (const T*)g.D;
    float mine = 0.f;   // lane j: this warp's part of choice j's product
    constexpr int C = 2;   // choices that share a read of D
    for (int j0 = 0; j0 < g.k; j0 += C) {
        int r[C];
        float w[C], dot[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            r[j] = __shfl_sync(0xffffffffu, row, j0 + j);   // (k is at most 16; lanes from k on hold -1)
            w[j] = __shfl_sync(0xffffffffu, gate, j0 + j);
            dot[j] = 0.f;
        }
        for (int c = (part * 32 + lane) * V; c < g.N; c += g.warps * 32 * V) {
            Piece<T, V> d, h[C], o;
            if (live) d.load(D + (size_t)t * g.N + c);
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (r[j] >= 0 && g.dgate != nullptr) h[j].load(H + (size_t)r[j] * g.N + c);
#pragma unroll
            for (int j = 0; j < C; ++j) {
                if (r[j] < 0) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) o.v[i] = w[j] * d.v[i];
                o.store((T*)g.dH + (size_t)r[j] * g.N + c);
                if (g.dgate != nullptr) {
#pragma unroll
                    for (int i = 0; i < V; ++i) dot[j] = fmaf(h[j].v[i], d.v[i], dot[j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const float x = warp_sum(dot[j]);
            if (lane == j0 + j) mine = x;
        }
    }
    if (g.dgate == nullptr) return;
    if (lane < g.k) dots[warp][lane] = mine;
    __syncthreads();
    if (live && part == 0 && lane < g.k) {
        float s = 0.f;
        for (int w = 0; w < g.warps; ++w) s += dots[warp + w][lane];
        g.dgate[(size_t)t * g.k + lane] = s;
    }
}

template <class T, bool ONE>
cudaError_t launch_route(const RouteArgs& a, int blocks, cudaStream_t s) {
    constexpr int threads = ONE ? kOneThreads : kRouteThreads;
    if (a.E <= 32) k_route<T, 1, ONE><<<blocks, threads, 0, s>>>(a);
    else if (a.E <= 64) k_route<T, 2, ONE><<<blocks, threads, 0, s>>>(a);
    else if (a.E <= 128) k_route<T, 4, ONE><<<blocks, threads, 0, s>>>(a);
    else k_route<T, BP_MAX_EXPERTS / 32, ONE><<<blocks, threads, 0, s>>>(a);
    return cudaGetLastError();
}

// Whether rows of N values at these addresses are whole 16-byte pieces.
bool pieces(const MixArgs& a, int size) {
    const uintptr_t p = (uintptr_t)a.H | (uintptr_t)a.Y | (uintptr_t)a.D | (uintptr_t)a.dH;
    return (p & 15) == 0 && (size_t)a.N * size % 16 == 0;
}

int device_sms() {
    int dev = 0, n = 1;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

// Warps of a pattern: as many as its row has pieces for, while patterns are few.
int mix_warps(int n, int N, int per_warp) {
    static const int num_sms = device_sms();   // (no handle keeps it)
    int w = 1;
    while (w < kMixThreads / 32 && w * per_warp < N && (long long)n * w < 16 * num_sms) w *= 2;
    return w;
}

}  // namespace

cudaError_t route_forward(const RouteArgs& a, cudaStream_t s) {
    const bool f32 = a.dtype == BP_F32;
    if (a.n <= kOneBlock) return f32 ? launch_route<float, true>(a, 1, s) : launch_route<bf16, true>(a, 1, s);
    const int blocks = (a.n + kRoutePatterns - 1) / kRoutePatterns;
    cudaError_t e = f32 ? launch_route<float, false>(a, blocks, s) : launch_route<bf16, false>(a, blocks, s);
    if (e == cudaSuccess) e = launch_pdl(k_route_columns, a.E, 1, kRouteThreads, 0, s, a, blocks);
    if (e == cudaSuccess) e = launch_pdl(k_route_place, blocks, 1, kRouteThreads, 0, s, a);
    return e;
}

cudaError_t route_backward(const RouteArgs& a, const float* dgate, void* dlogits, cudaStream_t s) {
    const int per = kRouteThreads / 32, blocks = (a.n + per - 1) / per;
    if (a.dtype == BP_F32) k_route_backward<float><<<blocks, kRouteThreads, 0, s>>>(a, dgate, (float*)dlogits);
    else k_route_backward<bf16><<<blocks, kRouteThreads, 0, s>>>(a, dgate, (bf16*)dlogits);
    return cudaGetLastError();
}

template <class T, bool BACK>
static cudaError_t launch_mix(MixArgs a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool wide = sizeof(T) == 2 || pieces(a, sizeof(T));   // bfloat16 rows always are (bp_mix's checks)
    a.warps = mix_warps(a.n, a.N, 32 * (wide ? V : 1));
    const int per = kMixThreads / 32 / a.warps, blocks = (a.n + per - 1) / per;
    if (wide) {
        if constexpr (BACK) k_mix_backward<T, V><<<blocks, kMixThreads, 0, s>>>(a);
        else k_mix<T, V><<<blocks, kMixThreads, 0, s>>>(a);
    } else if constexpr (sizeof(T) == 4) {
        if constexpr (BACK) k_mix_backward<T, 1><<<blocks, kMixThreads, 0, s>>>(a);
        else k_mix<T, 1><<<blocks, kMixThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}
cudaError_t mix_forward(const MixArgs& a, cudaStream_t s) {
    return a.dtype == BP_F32 ? launch_mix<float, false>(a, s) : launch_mix<bf16, false>(a, s);
}
cudaError_t mix_backward(const MixArgs& a, cudaStream_t s) {
    return a.dtype == BP_F32 ? launch_mix<float, true>(a, s) : launch_mix<bf16, true>(a, s);
}

}  // namespace bp
