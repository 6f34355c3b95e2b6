// Embeddings: rows of a table by token, and the pooled change of every token's row.
#include "bp_blocks_internal.h"
#include "bp_pieces.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// ------------------------------------------------------------ lookup
// A warp takes up to kLook pieces a lane of one row, or several short rows.  Bound by reading the rows that
// are named and writing n.
constexpr int kLook = 4;

template <class T, int V>
__global__ void __launch_bounds__(kThreads) k_embed(EmbedArgs g, int lanes, int chunks) {
    const int lane = threadIdx.x & 31, nv = g.width / V;
    const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const long long row = w / chunks * (32 / lanes) + lane / lanes;
    if (row >= g.n) return;
    const int id = g.ids[row];
    const bool ok = (unsigned)id < (unsigned)g.n_tokens;
    if (!ok && id != -1) atomicOr(g.flags, kFlagBounds);
    const int v0 = (int)(w % chunks) * lanes * kLook + lane % lanes;
    const T* in = (const T*)g.table + (size_t)(ok ? id : 0) * g.width;
    T* out = (T*)g.Y + (size_t)row * g.width;
    Piece<T, V> p[kLook];
#pragma unroll
    for (int i = 0; i < kLook; ++i)
        if (ok && v0 + i * lanes < nv) p[i].load(in + (size_t)(v0 + i * lanes) * V);
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
        if (v0 + i * lanes >= nv) break;
        float v[V] = {};
        if (ok) {
            p[i].values(v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] *= g.scale;
        }
        p[i].set(v);
        p[i].store(out + (size_t)(v0 + i * lanes) * V);
    }
}

// ------------------------------------------------------------ ids in order
// A stable radix sort of (token, place) by one cluster, which takes two passes of up to nine bits for up to
// 2^18 - 1 tokens, three beyond.  Each warp has a run of the ids; a pass counts every warp's digits in shared memory, adds the
// counts up over the warps, the cluster's CTAs (distributed shared memory) and the digits, and moves each id behind
// those before it.  Up to kHold times 32 ids a warp stay in registers within a pass, and go out by way of the CTA's shared memory,
// where they are put in order first: scattered words cost a CTA 32 cycles a warp's store, runs of them a few.  The ids lie in L2
// between passes.  No launch waits for another one's progress: the cluster's barrier is the hardware's.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kMaxDigits = 512;
constexpr int kMostCtas = 16;
constexpr int kHold = 8;
constexpr int kSortBytes = (kSortWarps + 3) * kMaxDigits * 4 + kSortWarps * kHold * 32 * 8;

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_rank() {
    int r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ int cluster_size() {
    int r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned of_cta(const unsigned* p, int cta) {   // a word of another CTA's shared memory
    unsigned a, v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ unsigned key_of(IdPlace x) { return (unsigned)(x >> 32); }
__device__ __forceinline__ int place_of(IdPlace x) { return (int)(unsigned)x; }

__global__ void __launch_bounds__(kSortThreads) k_sort(EmbedArgs g, int passes, int bits) {
    extern __shared__ __align__(16) IdPlace sorted[];   // [warps * kHold * 32] the CTA's ids in order
    unsigned* const sm = reinterpret_cast<unsigned*>(sorted + kSortWarps * kHold * 32);
    const int D = 1 << bits;
    unsigned* total = sm;              // [D] of this CTA
    unsigned* base = total + D;        // [D] where this CTA's ids of a digit go, less `own`
    unsigned* own = base + D;          // [D] this CTA's ids of lower digits
    unsigned* count = own + D;         // [warps, D]
    __shared__ unsigned scan[2][kSortWarps];
    pdl_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ctas = cluster_size(), rank = cluster_rank();
    const int shares = ctas * kSortWarps, per = (int)(((long long)g.n + shares * 32 - 1) / (shares * 32)) * 32;
    const long long first = (long long)(rank * kSortWarps + warp) * per;
    const int lo = (int)min(first, (long long)g.n), hi = (int)min(first + per, (long long)g.n);
    const bool held = per <= kHold * 32;
    unsigned* mine = count + (size_t)warp * D;
    for (int pass = 0; pass < passes; ++pass) {
        const IdPlace* in = g.ids_in_order[(pass + 1) & 1];
        IdPlace* out = g.ids_in_order[pass & 1];
        const int shift = pass * bits;
        const auto load = [&](int i) -> IdPlace {
            if (pass > 0) return __ldcg(in + i);
            const int id = __ldg(g.ids + i);
            if ((unsigned)id < (unsigned)g.n_tokens) return (IdPlace)(unsigned)id << 32 | (unsigned)i;
            if (id != -1) atomicOr(g.flags, kFlagBounds);
            return (IdPlace)(unsigned)g.n_tokens << 32 | (unsigned)i;   // behind every token
        };
        const auto digit = [&](IdPlace x) { return (key_of(x) >> shift) & (unsigned)(D - 1); };
        // How many ids of a lane's digit this warp has had before it; its ids are counted.
        const auto see = [&](unsigned d, bool live) -> unsigned {
            const unsigned peers = __match_any_sync(0xffffffffu, live ? d : 0xffffffffu);
            const unsigned before = live ? mine[d] : 0u;
            __syncwarp();
            if (live && lane == __ffs(peers) - 1) mine[d] = before + __popc(peers);
            __syncwarp();
            return before + __popc(peers & ((1u << lane) - 1u));
        };
        IdPlace x[kHold];
        unsigned before[kHold];
        if (held) {
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                const int i = lo + 32 * j + lane;
                x[j] = i < hi ? load(i) : 0ull;
            }
        }
        for (int i = threadIdx.x; i < kSortWarps * D; i += kSortThreads) count[i] = 0u;
        __syncthreads();
        if (held) {
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                before[j] = 0;
                if (lo + 32 * j < hi) before[j] = see(digit(x[j]), lo + 32 * j + lane < hi);
            }
        } else {
            for (int b = lo; b < hi; b += 32) {
                const bool live = b + lane < hi;
                see(live ? digit(load(b + lane)) : 0u, live);
            }
        }
        __syncthreads();
        unsigned of_own = 0, ahead = 0, all = 0;
        if (threadIdx.x < D) {
            for (int w0 = 0; w0 < kSortWarps; w0 += 8) {
                unsigned c[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) c[w] = count[(size_t)(w0 + w) * D + threadIdx.x];
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    count[(size_t)(w0 + w) * D + threadIdx.x] = of_own;
                    of_own += c[w];
                }
            }
            total[threadIdx.x] = of_own;
        }
        cluster_sync();
        if (threadIdx.x < D) {
            unsigned c[kMostCtas];
#pragma unroll
            for (int r = 0; r < kMostCtas; ++r) c[r] = r < ctas ? of_cta(total + threadIdx.x, r) : 0u;
#pragma unroll
            for (int r = 0; r < kMostCtas; ++r) {
                if (r < rank) ahead += c[r];
                all += c[r];
            }
        }
        unsigned s = all, t = of_own;   // digits up to this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned a = __shfl_up_sync(0xffffffffu, s, o), b = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) s += a, t += b;
        }
        if (lane == 31) scan[0][warp] = s, scan[1][warp] = t;
        __syncthreads();
        if (threadIdx.x < D) {
            for (int w = 0; w < warp; ++w) s += scan[0][w], t += scan[1][w];
            own[threadIdx.x] = t - of_own;
            base[threadIdx.x] = ahead + (s - all) - (t - of_own);
        }
        __syncthreads();
        if (held) {
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                if (lo + 32 * j + lane < hi) {
                    const unsigned d = digit(x[j]);
                    sorted[own[d] + mine[d] + before[j]] = x[j];
                }
            }
            __syncthreads();
            const long long cta_first = (long long)rank * kSortWarps * per;
            const int here = (int)(min(cta_first + (long long)kSortWarps * per, (long long)g.n) - min(cta_first, (long long)g.n));
            for (int i = threadIdx.x; i < here; i += kSortThreads) {
                const IdPlace y = sorted[i];
                out[base[digit(y)] + i] = y;
            }
        } else {
            for (int b = lo; b < hi; b += 32) {   // (mine goes on from the ids of the warps before)
                const bool live = b + lane < hi;
                const IdPlace y = live ? load(b + lane) : 0ull;
                const unsigned d = digit(y), r = see(d, live);
                if (live) out[base[d] + own[d] + r] = y;
            }
        }
        cluster_sync();   // the ids are there for the next pass; no CTA leaves while another reads its counts
    }
}

// ------------------------------------------------------------ changes
// The keys come from a launch that this one may overlap until pdl_wait: ordinary loads behind it, and never read-only ones, whose
// data must not change while a kernel runs.  (From L2 alone 40,001 ids of 1,024 units take 89.5 us, with the lookup, not 88.2.)
// keys[0, n) ascend: the first indexes whose keys are at least k1 and k2, by a converged warp.
__device__ __forceinline__ void warp_lower_bounds(const IdPlace* keys, int n, unsigned k1, unsigned k2, int& first, int& second) {
    const int lane = threadIdx.x & 31;
    int lo[2] = {0, 0}, hi[2] = {n, n};
    const unsigned k[2] = {k1, k2};
    while (lo[0] < hi[0] || lo[1] < hi[1]) {
        unsigned key[2];
        int step[2];
        long long at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            step[i] = max(1, (int)(((long long)hi[i] - lo[i] + 31) / 32));
            at[i] = lo[i] + (long long)(lane + 1) * step[i] - 1;
            key[i] = at[i] < hi[i] ? key_of(keys[at[i]]) : 0xffffffffu;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned m = __ballot_sync(0xffffffffu, at[i] >= hi[i] || key[i] >= k[i]);
            if (lo[i] >= hi[i]) continue;
            if (m == 0) {
                lo[i] = hi[i];
                continue;
            }
            const int f = __ffs(m) - 1;
            hi[i] = (int)min((long long)hi[i], lo[i] + (long long)(f + 1) * step[i] - 1);
            lo[i] += f * step[i];
        }
    }
    first = lo[0], second = lo[1];
}

constexpr int kZeroTokens = 16;   // tokens of a warp that writes zeros
// Pieces that are added up one after another.  (A plain sum of all of them is off by more the more there are: 32,768 pieces of equal
// rows by up to 1.8e-4, as every addition rounds the same way.  By 32 it is 2^-24 times 31 for the piece and for each of log32.)
constexpr int kChain = 32;

// A warp takes kEmbedTile sorted ids and 32 C pieces of their rows (two a lane for bfloat16: 40,001 rows of 1,024 units in 46 us,
// 48 with one), and adds up runs of equal tokens in registers.
// A run of at most kEmbedTile ids is summed by the tile that it starts in, also past that tile's end, and is stored at
// once.  A longer one is cut at the tiles' ends: its pieces go to scratch, and the warp whose piece comes
// last adds them up in an order of their own, so that sums do not depend on which that is.  Further warps write the zeros of
// tokens without ids.  Bound by reading D once and writing G once.
template <class T, int V, int C>
__global__ void __launch_bounds__(kThreads, 2) k_embed_sums(EmbedArgs g, const IdPlace* keys, long long sum_warps, int slabs) {
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    pdl_wait();
    const int n = g.n, N = g.width;
    if (w >= sum_warps) {   // zeros
        if (g.accumulate) return;
        const long long t0 = (w - sum_warps) * kZeroTokens;
        if (t0 >= g.n_tokens) return;
        const int last = (int)min(t0 + kZeroTokens, (long long)g.n_tokens);
        int at, end;
        warp_lower_bounds(keys, n, (unsigned)t0, (unsigned)last, at, end);
        unsigned m = 0;   // tokens that have ids
        if (end - at <= 128) {
            for (; at < end; at += 32)
                m |= __reduce_or_sync(0xffffffffu, at + lane < end ? 1u << (key_of(keys[at + lane]) - (unsigned)t0) : 0u);
        } else {
            bool there = false;
            if (t0 + lane < last) {
                const unsigned t = (unsigned)(t0 + lane);
                int lo = at, hi = end;
                while (lo < hi) {
                    const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
                    if (key_of(keys[mid]) < t) lo = mid + 1;
                    else hi = mid;
                }
                there = lo < end && key_of(keys[lo]) == t;
            }
            m = __ballot_sync(0xffffffffu, there);
        }
        m = ~m & ((1u << (last - (int)t0)) - 1u);
        while (m != 0) {
            float* row = g.G + (size_t)(t0 + __ffs(m) - 1) * N;
            m &= m - 1;
            if constexpr (V > 1) {
                for (int c = lane * 4; c < N; c += 128) *reinterpret_cast<float4*>(row + c) = make_float4(0.f, 0.f, 0.f, 0.f);
            } else {
                for (int c = lane; c < N; c += 32) row[c] = 0.f;
            }
        }
        return;
    }
    constexpr unsigned kNone = 0xffffffffu;
    const int tile = (int)(w / slabs), slab = (int)(w % slabs), t0 = tile * kEmbedTile;
    const unsigned tokens = (unsigned)g.n_tokens;
    const auto at = [&](int i) { return i < n ? keys[i] : (IdPlace)kNone << 32; };
    const IdPlace here = at(t0 + lane), after = at(t0 + 32 + lane);
    const unsigned kp = tile > 0 ? key_of(at(t0 - 32 + lane)) : kNone, kc = key_of(here), kn = key_of(after);
    const int pc = place_of(here), pn = place_of(after);
    const unsigned first = __shfl_sync(0xffffffffu, kc, 0), last = __shfl_sync(0xffffffffu, kc, 31);
    if (first >= tokens) return;   // ids of no token, behind all others
    // the rows [a, b) of this tile (from 32 on: the next one's); long runs at its ends
    int a = 0, b = __popc(__ballot_sync(0xffffffffu, kc < tokens));
    int head = 0, tail = 32;       // rows [0, head) and [tail, 32) are pieces of longer runs
    const int came = __clz(~__ballot_sync(0xffffffffu, kp == first));   // ids of the first run before this tile (32: or more)
    const unsigned of_first = __ballot_sync(0xffffffffu, kc == first), of_last = __ballot_sync(0xffffffffu, kc == last);
    const int lead = of_first == 0xffffffffu ? 32 : __ffs(~of_first) - 1;
    if (came > 0) {
        const bool lng = came == 32 || __shfl_sync(0xffffffffu, kc, (32 - came) & 31) == first;
        if (lng) head = lead;
        else a = lead;
    }
    if (last < tokens && __shfl_sync(0xffffffffu, kn, 0) == last && head < 32) {   // the last run goes on
        const int start = 32 - __clz(~of_last);
        if (__shfl_sync(0xffffffffu, kn, start & 31) == last) {
            tail = start;
        } else {
            const unsigned more = __ballot_sync(0xffffffffu, kn == last);
            b = 32 + __ffs(~more) - 1;   // (at most 31 more)
        }
    }
    constexpr int B = C > 1 ? 4 : 16, J = V == 1 ? 16 : 64 / (V * C);   // rows, and pieces of a run, under way
    const int c0 = (slab * 32 * C + lane) * V;   // and every 32 V columns on
    bool in[C];
#pragma unroll
    for (int c = 0; c < C; ++c) in[c] = c0 + c * 32 * V < N;
    const T* D = (const T*)g.D + c0;
    float acc[C][V] = {};
    const auto write = [&](unsigned token) {
        float* p = g.G + (size_t)token * N + c0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!in[c]) continue;
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = acc[c][i] * g.scale;
            if (g.accumulate) {
                float x[V];
                load_floats_l2<V>(p + c * 32 * V, x);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += x[i];
            }
            store_floats<V>(p + c * 32 * V, v);
        }
    };
    // A piece of a long run: to its slot, and all of the run's pieces to G if it is the last one.
    const auto join = [&](unsigned token, int slot) {
        const auto piece_of = [&](int at, int c) { return g.partial + (size_t)at * N + c0 + c * 32 * V; };
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (in[c]) store_floats<V>(piece_of(slot, c), acc[c]);
        int s, e;
        warp_lower_bounds(keys, n, token, token + 1, s, e);
        const int from = s / kEmbedTile, to = (e - 1) / kEmbedTile;
        __threadfence();
        __syncwarp();
        unsigned mine = 0;
        if (lane == 0) {
            unsigned* count = g.arrived + (size_t)from * slabs + slab;
            mine = atomicAdd(count, 1u);
            if (mine == (unsigned)(to - from)) *count = 0;   // for the next call
        }
        mine = __shfl_sync(0xffffffffu, mine, 0);
        if (mine != (unsigned)(to - from)) return;
        __threadfence();
        // kChain at a time, each sum in the place of its first piece, until one is left: a lane reads what it wrote.
        const int pieces = to - from + 1;
        const auto place_of_piece = [&](int q) { return q == 0 ? 2 * from + 1 : 2 * (from + q); };
        for (int step = 1; step < pieces; step *= kChain) {
            for (int q0 = 0; q0 < pieces; q0 += step * kChain) {
                const int end = min(pieces, q0 + step * kChain);
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (in[c]) load_floats_l2<V>(piece_of(place_of_piece(q0), c), acc[c]);
                for (int q = q0 + step; q < end; q += J * step) {
                    float x[J][C][V] = {};
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int c = 0; c < C; ++c)
                            if (q + j * step < end && in[c]) load_floats_l2<V>(piece_of(2 * (from + q + j * step), c), x[j][c]);
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int c = 0; c < C; ++c)
#pragma unroll
                            for (int i = 0; i < V; ++i) acc[c][i] += x[j][c][i];
                }
                if (step * kChain >= pieces) break;   // the last sum
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (in[c]) store_floats<V>(piece_of(place_of_piece(q0), c), acc[c]);
            }
        }
        write(token);
    };
    unsigned now = kNone;
    const auto row_key = [&](int r) { return r < 32 ? __shfl_sync(0xffffffffu, kc, r) : __shfl_sync(0xffffffffu, kn, r & 31); };
    const auto row_place = [&](int r) { return r < 32 ? __shfl_sync(0xffffffffu, pc, r) : __shfl_sync(0xffffffffu, pn, r & 31); };
    for (int r0 = a; r0 < b; r0 += B) {
        Piece<T, V> x[B][C];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int p = row_place(min(r0 + j, b - 1));
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (in[c]) x[j][c].load(D + (size_t)p * N + c * 32 * V);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int r = r0 + j;
            if (r >= b) break;
            const unsigned k = row_key(r);
            if (k != now) {
                if (now != kNone) {
                    if (r == head) join(now, 2 * tile);
                    else write(now);
                }
                now = k;
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[c][i] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (!in[c]) continue;
                float v[V];
                x[j][c].values(v);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[c][i] += v[i];
            }
        }
    }
    if (now == kNone) return;
    if (head == b) join(now, 2 * tile);
    else if (tail < 32) join(now, 2 * tile + 1);
    else write(now);
}

// Few ids of few tokens: a block a token and slab of columns, which looks the ids through for its own, in order, and shares
// out their rows to its warps, 32 rows a sum and the sums in order.  One launch, no order of all ids.
constexpr int kFewThreads = 1024, kFewWarps = kFewThreads / 32;
constexpr int kFewIds = 4096, kFewChunks = kFewIds / kFewThreads;   // of a call; of a warp, 32 at a time

template <class T, int V>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(EmbedArgs g) {
    constexpr int B = V == 1 ? 32 : V == 4 ? 8 : 4;   // rows under way
    __shared__ unsigned short list[kFewIds];
    __shared__ int counts[kFewWarps];
    __shared__ __align__(16) float part[kFewWarps][32 * V];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, N = g.width, token = blockIdx.x, chunks = (g.n + kFewThreads - 1) / kFewThreads;
    const bool checks = blockIdx.x == 0 && blockIdx.y == 0;
    int id[kFewChunks];
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) {
        const int i = (warp * chunks + j) * 32 + lane;
        id[j] = j < chunks && i < g.n ? __ldg(g.ids + i) : -1;
    }
    unsigned found[kFewChunks];
    int count = 0;
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) {
        if (checks && ((unsigned)id[j] >= (unsigned)g.n_tokens) && id[j] != -1) atomicOr(g.flags, kFlagBounds);
        found[j] = __ballot_sync(0xffffffffu, id[j] == token);
        count += __popc(found[j]);
    }
    if (lane == 0) counts[warp] = count;
    __syncthreads();
    int before = lane < warp ? counts[lane] : 0, rows = counts[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        before += __shfl_xor_sync(0xffffffffu, before, o);
        rows += __shfl_xor_sync(0xffffffffu, rows, o);
    }
#pragma unroll
    for (int j = 0; j < kFewChunks; ++j) {
        if (found[j] >> lane & 1) list[before + __popc(found[j] & ((1u << lane) - 1u))] = (unsigned short)((warp * chunks + j) * 32 + lane);
        before += __popc(found[j]);
    }
    __syncthreads();
    if (rows == 0 && g.accumulate) return;
    const int c0 = ((int)blockIdx.y * 32 + lane) * V;
    const bool in_row = c0 < N;
    const T* D = (const T*)g.D + c0;
    float sum[V] = {};
    const int groups = (rows + 31) / 32, q1 = groups * (warp + 1) / kFewWarps;
    for (int q = groups * warp / kFewWarps; q < q1; ++q) {
        const int end = min(rows, q * 32 + 32);
        float acc[V] = {};
        for (int r0 = q * 32; r0 < end; r0 += B) {
            Piece<T, V> x[B];
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (in_row && r0 + j < end) x[j].load(D + (size_t)list[r0 + j] * N);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (!in_row || r0 + j >= end) break;
                float v[V];
                x[j].values(v);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += v[i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += acc[i];
    }
    store_floats<V>(&part[warp][lane * V], sum);
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * V; c += kFewThreads) {
        const int col = (int)blockIdx.y * 32 * V + c;
        if (col >= N) break;
        float x = 0.f;
#pragma unroll 8
        for (int w = 0; w < kFewWarps; ++w) x += part[w][c];
        x *= g.scale;
        float* to = g.G + (size_t)token * N + col;
        *to = g.accumulate ? *to + x : x;
    }
}
// Whether a call is for it.  Its time grows with its blocks, by 13 us a thousand, that of the next kernel with the ids, by 5 us a
// thousand; at the limit they are about as fast (of 256 units, bfloat16: 1,000 ids of 300 tokens take 5.6 us, by the next
// kernel 7.8; of 500 8.5 and 8.2; 4,000 of 1,000 15 and 21; 100 of 256 4.7 and 3.6).  3,584 ids of 29 tokens and 15 units take
// 5 us, by the sort 18.
bool is_few(const EmbedArgs& a, int slabs) { return a.n <= kFewIds && 4 * (long long)a.n_tokens * slabs <= a.n + 256; }

template <class T, int V>
bool few(const EmbedArgs& a, cudaStream_t s, cudaError_t& e) {
    const int slabs = (a.width + 32 * V - 1) / (32 * V);
    if (!is_few(a, slabs)) return false;
    k_embed_few<T, V><<<dim3(a.n_tokens, slabs), kFewThreads, 0, s>>>(a);
    e = cudaGetLastError();
    return true;
}

// Few ids of many tokens: zeros everywhere first, then a block an id, which looks all ids through for its token.  The block
// of every 32nd id of a token (the first one, mostly the only one, among them) adds up the rows of it and the 31 behind it;
// more than 32 are joined as pieces, as in k_embed_sums, in the slots that the ids' order would give them.  Its time grows with
// the ids: 100 of 2,000 tokens and 256 units take 4 us, 1,000 10, 4,000 24; by the sort 21, 23 and 23.
constexpr int kScanIds = 4096;

__global__ void __launch_bounds__(kThreads) k_zero(float* G, long long n) {
    pdl_launch();
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x, all = (long long)gridDim.x * kThreads;
    if (((uintptr_t)G & 15) == 0) {
        for (long long j = i; j < n / 4; j += all) reinterpret_cast<float4*>(G)[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n % 4) G[n / 4 * 4 + i] = 0.f;
    } else {
        for (long long j = i; j < n; j += all) G[j] = 0.f;
    }
}

template <class T, int V>
__global__ void __launch_bounds__(kThreads) k_embed_scan(EmbedArgs g, int slabs) {
    constexpr int kEach = kScanIds / kThreads, B = 8;   // ids of a thread; rows, and pieces, under way
    __shared__ int list[kEmbedTile];
    __shared__ unsigned of_warp[3][kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = g.n, N = g.width, i = blockIdx.x;
    const int token = __ldg(g.ids + i);
    if ((unsigned)token >= (unsigned)g.n_tokens) {
        if (token != -1 && threadIdx.x == 0) atomicOr(g.flags, kFlagBounds);
        pdl_wait();   // (no block is gone before the zeros are there: the stream goes on behind this kernel)
        return;
    }
    // A warp takes a run of the ids, 32 at a time: of this token, before this id; of lower tokens.
    const int chunks = (n + kThreads - 1) / kThreads, first = warp * chunks * 32;
    unsigned same[kEach], all = 0, before = 0, lower = 0;
    int id[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int at = first + j * 32 + lane;
        id[j] = j < chunks && at < n ? __ldg(g.ids + at) : -1;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        same[j] = __ballot_sync(0xffffffffu, id[j] == token);
        all += __popc(same[j]);
        const int left = i - (first + j * 32);   // ids of the 32 that come before this one
        before += __popc(same[j] & (left <= 0 ? 0u : left >= 32 ? 0xffffffffu : (1u << left) - 1u));
        lower += (unsigned)id[j] < (unsigned)token;
    }
    lower = __reduce_add_sync(0xffffffffu, lower);
    if (lane == 0) of_warp[0][warp] = all, of_warp[1][warp] = before, of_warp[2][warp] = lower;
    __syncthreads();
    unsigned at = 0;   // the token's ids of the warps before
    all = before = lower = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) at += of_warp[0][w];
        all += of_warp[0][w];
        before += of_warp[1][w];
        lower += of_warp[2][w];
    }
    if (before % kEmbedTile != 0) {
        pdl_wait();
        return;
    }
    const int rows = (int)min(all - before, (unsigned)kEmbedTile);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {   // the places of the rows
        const unsigned rank = at + __popc(same[j] & ((1u << lane) - 1u)) - before;
        if ((same[j] >> lane & 1) && rank < (unsigned)kEmbedTile) list[rank] = first + j * 32 + lane;
        at += __popc(same[j]);
    }
    __syncthreads();
    pdl_wait();
    for (int slab = warp; slab < slabs; slab += kWarps) {
        const int c0 = (slab * 32 + lane) * V;
        const bool in_row = c0 < N;
        const T* D = (const T*)g.D + c0;
        float acc[V] = {};
        for (int r0 = 0; r0 < rows; r0 += B) {
            Piece<T, V> x[B];
#pragma unroll
            for (int j = 0; j < B; ++j)
                if (in_row && r0 + j < rows) x[j].load(D + (size_t)list[r0 + j] * N);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (!in_row || r0 + j >= rows) break;
                float v[V];
                x[j].values(v);
#pragma unroll
                for (int c = 0; c < V; ++c) acc[c] += v[c];
            }
        }
        if (all > kEmbedTile) {
            const int pieces = (int)(all + kEmbedTile - 1) / kEmbedTile, from = (int)lower / kEmbedTile;
            const auto piece_of = [&](int p) { return g.partial + (size_t)(p == 0 ? 2 * from + 1 : 2 * (((int)lower + p * kEmbedTile) / kEmbedTile)) * N + c0; };
            if (in_row) store_floats<V>(piece_of((int)before / kEmbedTile), acc);
            __threadfence();
            __syncwarp();
            unsigned mine = 0;
            if (lane == 0) {
                unsigned* arrived = g.arrived + (size_t)from * slabs + slab;
                mine = atomicAdd(arrived, 1u);
                if (mine == (unsigned)pieces - 1) *arrived = 0;   // for the next call
            }
            mine = __shfl_sync(0xffffffffu, mine, 0);
            if (mine != (unsigned)pieces - 1) continue;
            __threadfence();
            if (in_row) {
                load_floats_l2<V>(piece_of(0), acc);
                for (int p = 1; p < pieces; p += B) {
                    float x[B][V] = {};
#pragma unroll
                    for (int j = 0; j < B; ++j)
                        if (p + j < pieces) load_floats_l2<V>(piece_of(p + j), x[j]);
#pragma unroll
                    for (int j = 0; j < B; ++j)
#pragma unroll
                        for (int c = 0; c < V; ++c) acc[c] += x[j][c];
                }
            }
        }
        if (in_row) {
            float* to = g.G + (size_t)token * N + c0;
#pragma unroll
            for (int c = 0; c < V; ++c) acc[c] *= g.scale;
            if (g.accumulate) {
                float x[V];
                load_floats_l2<V>(to, x);
#pragma unroll
                for (int c = 0; c < V; ++c) acc[c] += x[c];
            }
            store_floats<V>(to, acc);
        }
    }
}

template <class T, int V>
cudaError_t scan(const EmbedArgs& a, cudaStream_t s) {
    if (!a.accumulate) {
        const long long values = (long long)a.n_tokens * a.width, blocks = (values / 4 + kThreads - 1) / kThreads;
        k_zero<<<(unsigned)max(1ll, min(blocks, 2048ll)), kThreads, 0, s>>>(a.G, values);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    const int slabs = (a.width + 32 * V - 1) / (32 * V);
    if (!a.accumulate) return launch_pdl(k_embed_scan<T, V>, a.n, 1, kThreads, 0, s, a, slabs);
    k_embed_scan<T, V><<<a.n, kThreads, 0, s>>>(a, slabs);
    return cudaGetLastError();
}

int sort_bits(int n_tokens, int& passes) {
    int bits = 1;
    while ((n_tokens >> bits) != 0) ++bits;   // tokens and n_tokens itself
    passes = (bits + 8) / 9;
    return (bits + passes - 1) / passes;
}

template <class T, int V>
cudaError_t lookup(const EmbedArgs& a, cudaStream_t s) {
    const int nv = a.width / V;
    int lanes = 1;
    while (lanes < 32 && lanes < nv) lanes *= 2;
    const int chunks = (nv + lanes * kLook - 1) / (lanes * kLook), rows = 32 / lanes;
    const long long warps = (long long)((a.n + rows - 1) / rows) * chunks;
    k_embed<T, V><<<(unsigned)((warps + kWarps - 1) / kWarps), kThreads, 0, s>>>(a, lanes, chunks);
    return cudaGetLastError();
}

template <class T, int V, int C>
cudaError_t sums(const EmbedArgs& a, int passes, cudaStream_t s) {
    const int tiles = (a.n + kEmbedTile - 1) / kEmbedTile, slabs = (a.width + 32 * V * C - 1) / (32 * V * C);
    const long long sum_warps = (long long)tiles * slabs;
    const long long zero_warps = a.accumulate ? 0 : (a.n_tokens + kZeroTokens - 1) / kZeroTokens;
    const long long blocks = (sum_warps + zero_warps + kWarps - 1) / kWarps;
    if (blocks == 0) return cudaSuccess;
    const int at = (passes - 1) & 1;
    return launch_pdl(k_embed_sums<T, V, C>, (int)blocks, 1, kThreads, 0, s, a, (const IdPlace*)a.ids_in_order[at], sum_warps, slabs);
}

bool pieces16(const void* a, const void* b, int width) { return (((uintptr_t)a | (uintptr_t)b) & 15) == 0 && width % 4 == 0; }

}  // namespace

size_t embed_counts(int max_ids, int width, int dtype) {
    const size_t slab = dtype == BP_BF16 ? 256 : 32;
    return ((size_t)max_ids + kEmbedTile - 1) / kEmbedTile * ((width + slab - 1) / slab);
}

namespace {
cudaLaunchConfig_t sort_config(int ctas, cudaLaunchAttribute* at, cudaStream_t s) {
    at->id = cudaLaunchAttributeClusterDimension;
    at->val.clusterDim.x = ctas;
    at->val.clusterDim.y = at->val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(ctas);
    c.blockDim = dim3(kSortThreads);
    c.dynamicSmemBytes = kSortBytes;
    c.stream = s;
    c.attrs = at;
    c.numAttrs = 1;
    return c;
}
}  // namespace

// The CTAs of a cluster that sorts: 16 where the device has room for them, else the 8 that any has.
cudaError_t embed_setup(int* sort_ctas) {
    cudaError_t e = cudaFuncSetAttribute(k_sort, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortBytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_sort, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at;
    const cudaLaunchConfig_t c = sort_config(kMostCtas, &at, nullptr);
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, k_sort, &c);
    *sort_ctas = e == cudaSuccess && clusters > 0 ? kMostCtas : 8;
    if (e != cudaSuccess) cudaGetLastError();
    return cudaSuccess;
}

cudaError_t embed_forward(const EmbedArgs& a, cudaStream_t s) {
    if (a.dtype == BP_BF16) return lookup<__nv_bfloat16, 8>(a, s);
    return pieces16(a.table, a.Y, a.width) ? lookup<float, 4>(a, s) : lookup<float, 1>(a, s);
}

cudaError_t embed_backward(const EmbedArgs& a, cudaStream_t s) {
    const bool pieces = a.dtype == BP_BF16 || pieces16(a.D, a.G, a.width);
    cudaError_t few_status = cudaSuccess;
    if (a.dtype == BP_BF16 ? few<__nv_bfloat16, 8>(a, s, few_status) : pieces ? few<float, 4>(a, s, few_status) : few<float, 1>(a, s, few_status))
        return few_status;
    if (a.n > 0 && a.n <= kScanIds)
        return a.dtype == BP_BF16 ? scan<__nv_bfloat16, 8>(a, s) : pieces ? scan<float, 4>(a, s) : scan<float, 1>(a, s);
    int passes = 1;
    const int bits = sort_bits(a.n_tokens, passes);
    if (a.n > 0) {
        cudaLaunchAttribute at;
        const cudaLaunchConfig_t c = sort_config(a.sort_ctas, &at, s);
        const cudaError_t e = cudaLaunchKernelEx(&c, k_sort, a, passes, bits);
        if (e != cudaSuccess) return e;
    }
    if (a.dtype == BP_BF16) return a.width > 256 ? sums<__nv_bfloat16, 8, 2>(a, passes, s) : sums<__nv_bfloat16, 8, 1>(a, passes, s);
    return pieces ? sums<float, 4, 1>(a, passes, s) : sums<float, 1, 1>(a, passes, s);
}

}  // namespace bp
