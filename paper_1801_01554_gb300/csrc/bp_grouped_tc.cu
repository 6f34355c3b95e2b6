// Products of rows with the weights of their group on the tensor cores, in bfloat16 with float32
// sums: the expert layers, and the adapter layers' shared product with the adapters' part added.
//
//   forward  out[r, n]  = sum over k of in[src(r), k] W_g[n, k]     both operands along K
//   back     out[r, n]  = sum over k of in[r, k] W_g[k, n]          W as an MN-major operand
//   change   G_g[m, n]  = sum over the group's rows of a[r, m] b[r, n]   both MN-major
//   up       low[r, j]  = scale_a * sum over k of in[r, k] P_a[j, k], a the adapter of the row's request
//   low      G_a[j, n]  = scale_a * sum over the rows of the adapter's requests of low[r, j] b[r, n]
//            (of A and of B in one launch: twice the tiles to balance the SMs with)
//
// One persistent CTA per SM: a warp that issues TMA copies into a ring of stages, a warp that
// issues tcgen05.mma (128 rows x BN columns x 64 of K a stage) into TMEM, eight epilogue warps.
// The tensor cores bound the large products: 16,384 rows of 4096-4096 in 8 ragged groups take 336 us forward
// and 340 back (1.63 PFLOP/s, 86% of the measured burst rate), their changes 404 (1.36 PFLOP/s; 350 without
// the 537 MB that they write); few rows a group are bound by reading the weights (240 rows of 4096-1024
// in 32 groups: 44 us, the 268 MB at the measured copy rate 40).
//
// The groups' ends lie on the device: each CTA turns them into first tiles in shared memory and
// finds the group of a tile by bisection, so that no host knows the sizes and no list is written.
//
// Ragged groups need no padded copy of the rows.  A tile that runs over its group's end computes
// the next group's rows too and does not store them; in a change, where rows are summed, the
// stage's foreign rows are set to zero in shared memory in both operands (0 times a foreign
// infinity would not be 0).  W's maps have a dimension of their own for the group, past whose
// edges the copy engine fills in zeros.  Rows that the forward product reads through an index are
// gathered by four more warps, eight lanes a row, with cp.async into the swizzled stage (gathered by the
// copy engine, four rows an instruction, a K block waited for its 32 instructions: 539 us for 32,768
// rows of 2048-2048 against 181 without an index; copied into order first: 224).  A change, whose
// epilogue wants the registers of such warps, takes rows that are copied into order first.
//
// The adapters' part of a tile whose rows all belong to one request is K beyond the layer's own:
// the rows of low as two bfloat16 terms (its rounding and the rest) times the adapter's rows.  In
// a tile of several requests each request's part is a sum of its own for all of the tile's rows, of
// which the epilogue adds the request's rows (as one product with the other requests' rows at zero,
// an adapter's infinity would reach them); with more requests than half the rank the epilogue
// takes the rows one by one instead.  In the low form the terms lie side by side along
// M (three: as exact as float32), so that a rank of up to 32 costs one product and one of 64 two
// instead of three; the epilogue warps of the other terms pass their sums on through shared
// memory.  Its K blocks run over the adapter's requests in order.
#include <mutex>

#include "bp_experts_device.cuh"
#include "bp_tc_device.cuh"

namespace bp {
namespace {

constexpr int kEpiWarps = 8;         // two per TMEM lane quarter, each on half of the columns
constexpr int kEpiThreads = 32 * kEpiWarps;
constexpr int kThreads = 64 + kEpiThreads;   // warp 0 copies, warp 1 MMA, warps 2.. epilogue
constexpr int kGatherWarps = 4;              // of a forward product with an index, behind them
constexpr int threads_of(bool gather) { return kThreads + (gather ? 32 * kGatherWarps : 0); }

// LOW_WIDE: the low form of ranks above 64.
enum Form : int { FORWARD = 0, BACK = 1, CHANGE = 2, LOW = 3, UP = 4, LOW_WIDE = 5 };
constexpr bool is_low(int form) { return form == LOW || form == LOW_WIDE; }

struct TcArgs {
    RowGroups groups;
    int num_n, num_m;        // tiles along N; along M of a change
    int M, N, K;             // M: rows of a change; K: not of a change
    const bf16* in;          // forward with an index: rows [n_in_rows, K]
    const int* source;
    int n_in_rows;
    const float* bias;
    int squash;
    const bf16* x;
    const int* x_source;
    int n_x;
    bf16* out;
    float* G;
    int accumulate;
    int sectors;             // G starts on a 32-byte boundary
    // adapters
    int2* tiles;               // per 128 rows: adapter or kind, first request; or NULL
    int rank16;                // 16-wide pieces of the rank
    int n_terms, stride;       // bfloat16 terms of low, and their pitch (32, 64 or 128)
    Requests req;
    const float* low;
    const bf16* P;
    const float* scale;
    // of the low form: a second product's changes G2 [n_adapters, rank, N2], whose tiles follow the first's
    int N2, num_n2;            // (num_n2 0: none)
    float* G2;
    const float* scale2;
    int sectors2;
    int num_sms;
    int runs;                  // of the low form: most shares of an adapter's rows, of which the sums go to
    float* scratch;            // [runs, n_adapters, rank, N], and behind it the second's
    unsigned* arrived;         // of every warp's part of a tile; zeros, left so
    // up
    float* low_out;
    bf16* terms;
    int scaled_low, wide_low;   // low with the scale; in 16-byte pieces
    int max_items;
    int* flags;
};

constexpr int kBarBytes = 384;
// An operand A of the low form holds all terms: up to four blocks of 64 columns, six of ranks above 64.
constexpr int low_blocks(int form) { return form == LOW_WIDE ? 6 : 4; }

template <int BN, int FORM>
struct Cfg {
    static constexpr int kStages = BN == 256 ? 4 : FORM == LOW_WIDE ? 3 : FORM == LOW ? (BN == 128 ? 4 : 5) : BN == 128 ? 6 : 8;
    static constexpr int kABytes = is_low(FORM) ? low_blocks(FORM) * BK * 64 * 2 : BM * BK * 2;
    static constexpr int kBBytes = BN * BK * 2;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kRingBytes = kStages * kStageBytes;
    static constexpr int kOutBytes = kEpiWarps * 32 * 32 * 2;   // a 32 x 32 bf16 block per epilogue warp
    static constexpr int kBiasBytes = kEpiWarps * (BN / 2) * 4;   // a warp's half of the tile's biases
    static constexpr int kGroupBytes = (3 * BP_MAX_EXPERTS + 32) * 4;
    static constexpr int kSmemBytes = 1024 + kRingBytes + kOutBytes + kBiasBytes + kGroupBytes + kBarBytes;
};

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
        "l"((unsigned long long)map), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}
// Products that the low form takes for all terms: 128 of their columns each.
__host__ __device__ __forceinline__ int low_sets(const TcArgs& g) { return (g.n_terms * g.stride + BM - 1) / BM; }

// A tile: rows [row0, end) of a forward or back product, of group g; of a change, all rows of the
// group and the block mb of M.
struct Item {
    int g, row0, end, mb, nb;
    int kbs;        // K blocks
    int kb0, kb1;   // of the low form: of the adapter's
    int run, shares;
    bool second;    // of the low form: the second product
    int adapter;    // whose low-rank K follows; of an up product, the rows'; -1, or a kind of tile
    int request;    // the tile's first
};

// The requests with an adapter that have rows in a tile, in order.
struct TileRequests {
    const TcArgs& g;
    const Item& w;
    int at;
    __device__ bool next(int& lo, int& hi, int& adapter) {
        for (; at < g.req.n_requests; ++at) {
            group_rows(g.req.offsets, g.req.n_rows, at, lo, hi, g.flags);
            if (lo >= w.end) return false;
            if (hi <= lo) continue;
            adapter = request_adapter(g.req, at, g.flags);
            if (adapter < 0) continue;
            ++at;
            return true;
        }
        return false;
    }
};

// The stretches of rows that a change sums over, K blocks kb0 to kb1 of them: the group's, or of the
// low form those of the requests of adapter w.g in order, which the whole warp looks for.
struct RequestTable {   // of the requests, in shared memory; adapter NULL: too many, read where they are
    const int *adapter, *lo, *hi;
};
template <int FORM>
struct Stretches {
    const TcArgs& g;
    const Item& w;
    const RequestTable& table;
    int at, seen;   // next request; K blocks before it
    __device__ bool request(int& lo, int& hi) {
        const int lane = threadIdx.x & 31;
        const int* adapter = table.adapter != nullptr ? table.adapter : g.req.adapter;
        while (at < g.req.n_requests) {
            const int base = at & ~31, i = base + lane;
            const bool mine = i >= at && i < g.req.n_requests && adapter[i] == w.g;
            const unsigned m = __ballot_sync(0xffffffffu, mine);
            if (m == 0) {
                at = base + 32;
                continue;
            }
            const int r = base + __ffs(m) - 1;
            at = r + 1;
            if (table.adapter != nullptr) lo = table.lo[r], hi = table.hi[r];
            else group_rows(g.req.offsets, g.req.n_rows, r, lo, hi, g.flags);
            if (hi > lo) return true;
        }
        return false;
    }
    __device__ bool next(int& lo, int& hi) {
        if constexpr (!is_low(FORM)) {
            lo = w.row0;
            hi = w.end;
            return at++ == 0 && hi > lo;
        } else {
            while (seen < w.kb1 && request(lo, hi)) {
                const int blocks = (hi - lo + BK - 1) / BK, s = max(w.kb0 - seen, 0), e = min(w.kb1 - seen, blocks);
                seen += blocks;
                if (s >= e) continue;
                hi = min(hi, lo + e * BK);
                lo += s * BK;
                return true;
            }
            return false;
        }
    }
};

// Row blocks of a group are swept 16 at a time over all column blocks (row block fastest), so
// that the tiles in flight share rows and weights in L2 (16: as square as 152 tiles of
// 128 x 256 get).
__device__ __forceinline__ void sweep(int tile, int num_m, int num_n, int& mb, int& nb) {
    constexpr int kRun = 16;
    const int run = tile / (kRun * num_n), first = run * kRun, m = min(num_m - first, kRun);
    const int local = tile - run * kRun * num_n;
    mb = first + local % m;
    nb = local / m;
}

template <int FORM>
struct Schedule {
    const TcArgs& g;
    const int *lo, *hi, *tile0;   // per group, in shared memory: first row, end; first row block (n_groups + 1)
    const RequestTable table;
    __device__ int table_blocks(int i) const {   // K blocks of a request
        int l, h;
        if (table.adapter != nullptr) l = table.lo[i], h = table.hi[i];
        else group_rows(g.req.offsets, g.req.n_rows, i, l, h, g.flags);
        return (h - l + BK - 1) / BK;
    }
    __device__ int items() const {
        if (is_low(FORM)) return g.req.n_adapters * (g.num_n + g.num_n2) * g.runs;
        if (FORM == UP) return g.max_items;
        return FORM == CHANGE ? g.groups.n_groups * g.num_m * g.num_n : tile0[g.groups.n_groups] * g.num_n;
    }
    __device__ Item item(int it) const {
        Item w;
        if (is_low(FORM)) {
            // all tiles' first shares, then their second ones, ..: those that there are lie together
            const int first = g.req.n_adapters * g.num_n, tiles = first + g.req.n_adapters * g.num_n2;
            w.run = g.runs == 1 ? 0 : it / tiles;
            int tile = it - w.run * tiles;
            w.second = tile >= first;
            if (w.second) tile -= first;
            const int num_n = w.second ? g.num_n2 : g.num_n;
            w.g = tile / num_n;
            w.nb = tile - w.g * num_n;
            w.mb = w.row0 = w.end = 0;
            w.adapter = w.request = -1;
            Stretches<LOW> all{g, w, table, 0, 0};
            int lo, hi, blocks = 0;
            while (all.request(lo, hi)) blocks += (hi - lo + BK - 1) / BK;
            // as many shares as an adapter has times an SM's part of all K blocks, to the nearest; one of few
            // rows is left whole (another share costs what 10 K blocks do)
            w.shares = 1;
            if (g.runs > 1 && blocks >= 16) {
                int all_blocks = 0;
                for (int i = threadIdx.x & 31; i < g.req.n_requests; i += 32)
                    if ((table.adapter != nullptr ? table.adapter : g.req.adapter)[i] >= 0) all_blocks += table_blocks(i);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) all_blocks += __shfl_xor_sync(0xffffffffu, all_blocks, o);
                const int part = max((int)((long long)all_blocks * (g.num_n + g.num_n2) / g.num_sms), 8);
                w.shares = min(max((2 * blocks + part) / (2 * part), 1), g.runs);
            }
            const int share = blocks / w.shares, more = blocks - share * w.shares;   // the first `more` shares have one more
            w.kb0 = w.run * share + min(w.run, more);
            w.kb1 = w.run < w.shares ? w.kb0 + share + (w.run < more ? 1 : 0) : w.kb0;
            w.kbs = w.kb1 - w.kb0;
            return w;
        }
        if (FORM == UP) {   // (the whole warp asks)
            int end;
            find_tile<BM>(RowGroups{g.req.offsets, g.req.n_requests, g.req.n_rows}, it, w.request, w.row0, end, g.flags);
            w.g = w.nb = w.mb = 0;
            w.end = min(end, w.row0 + BM);
            w.adapter = w.request >= 0 ? request_adapter(g.req, w.request, g.flags) : -1;
            w.kbs = w.adapter >= 0 ? (g.K + BK - 1) / BK : 0;
            return w;
        }
        if (FORM == CHANGE) {
            const int per = g.num_m * g.num_n;
            w.g = it / per;
            sweep(it - w.g * per, g.num_m, g.num_n, w.mb, w.nb);
            w.row0 = lo[w.g];
            w.end = hi[w.g];
            w.kbs = (w.end - w.row0 + BK - 1) / BK;
            w.adapter = w.request = -1;
            return w;
        }
        int a = 0, b = g.groups.n_groups;   // the last group whose first tile is not past `it`, with tiles
        while (b - a > 1) {
            const int mid = (a + b) >> 1;
            if (tile0[mid] * g.num_n <= it) a = mid;
            else b = mid;
        }
        w.g = a;
        int mb;
        sweep(it - tile0[a] * g.num_n, tile0[a + 1] - tile0[a], g.num_n, mb, w.nb);
        w.mb = tile0[a] + mb;
        w.row0 = lo[a] + mb * BM;
        w.kbs = (g.K + BK - 1) / BK;
        const int2 t = g.tiles != nullptr ? g.tiles[mb] : make_int2(-1, 0);
        w.adapter = t.x;
        w.request = t.y;
        w.end = min(hi[a], w.row0 + BM);
        return w;
    }
};

// Rows of one K block of an MN-major operand's 64-wide blocks from `from` up to `to` set to zero.
__device__ __forceinline__ void zero_rows(uint8_t* block, int blocks, int from, int to) {
    const int lane = threadIdx.x & 31, per = (to - from) * 8;   // 16-byte pieces of a block's rows
    for (int i = lane; i < blocks * per; i += 32) {
        const int b = i / per, p = i - b * per;
        *reinterpret_cast<uint4*>(block + b * kMnBlockBytes + from * 128 + p * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Stores a warp's 32 x 32 block of float32 sums as bfloat16 rows (see bp_tc_device.cuh).
__device__ __forceinline__ void store_rows(bf16* out, int N, int row0, int end, int n0, const float (&v)[32], uint4* sS4) {
    const int lane = threadIdx.x & 31, piece = lane & 3;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        __align__(16) __nv_bfloat162 h[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] = __floats2bfloat162_rn(v[8 * k + 2 * q], v[8 * k + 2 * q + 1]);
        *piece_at(sS4, lane, k) = *reinterpret_cast<const uint4*>(h);
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = 8 * j + (lane >> 2);
        const uint4 u = *piece_at(sS4, r, piece);
        if (row0 + r < end && n0 + piece * 8 < N)
            *reinterpret_cast<uint4*>(out + (size_t)(row0 + r) * N + n0 + piece * 8) = u;
    }
    __syncwarp();   // the block may be rewritten
}

// Stores a warp's 32 x 16 block of float32 changes.  The block turns in shared memory (16-byte pieces
// permuted by row), after which four lanes hold 64 bytes of a row: whole sectors.  Stored by rows as
// TMEM gives them, 16 bytes a lane and row, a 128 x 256 tile took 20,000 clocks.
__device__ __forceinline__ void store_change(float* G, int M, int N, int m0, int n0, const float (&v)[16], int accumulate,
                                             float4* sF) {
    const int lane = threadIdx.x & 31, piece = lane & 3, n = n0 + 4 * piece;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        sF[lane * 4 + (k ^ ((lane >> 1) & 3))] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 8 * j + (lane >> 2), m = m0 + row;
        float4 o = sF[row * 4 + (piece ^ ((row >> 1) & 3))];
        if (m < M && n < N) {   // N is a multiple of 8
            float4* p = reinterpret_cast<float4*>(G + (size_t)m * N + n);
            if (accumulate) {
                const float4 old = *p;
                o.x += old.x, o.y += old.y, o.z += old.z, o.w += old.w;
            }
            __stcs(p, o);
        }
    }
    __syncwarp();   // the block may be rewritten
}

// The same straight from a lane's row, a sector (32 bytes, and so aligned) an instruction.
__device__ __forceinline__ void store_sectors(float* p, const float (&v)[16], int cols) {
#pragma unroll
    for (int c = 0; c < 16; c += 8)
        if (c < cols)   // cols is a multiple of 8
            asm volatile("st.global.L1::no_allocate.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + c), "f"(v[c]),
                         "f"(v[c + 1]), "f"(v[c + 2]), "f"(v[c + 3]), "f"(v[c + 4]), "f"(v[c + 5]), "f"(v[c + 6]), "f"(v[c + 7])
                         : "memory");
}

// The same for 16 columns of low [n_rows, rank], rows below `end`; in 16-byte pieces if they are whole.
__device__ __forceinline__ void store_low(float* low, int rank, int row0, int end, int j0, const float (&v)[16], int wide,
                                          float4* sF) {
    const int lane = threadIdx.x & 31, piece = lane & 3, j = j0 + 4 * piece;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        sF[lane * 4 + (k ^ ((lane >> 1) & 3))] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        const float4 o = sF[r * 4 + (piece ^ ((r >> 1) & 3))];
        if (row0 + r >= end || j >= rank) continue;
        float* p = low + (size_t)(row0 + r) * rank + j;
        if (wide) {
            *reinterpret_cast<float4*>(p) = o;
        } else {
            p[0] = o.x;
            if (j + 1 < rank) p[1] = o.y;
            if (j + 2 < rank) p[2] = o.z;
            if (j + 3 < rank) p[3] = o.w;
        }
    }
    __syncwarp();   // the block may be rewritten
}

// scale_a * sum over j of low[row, j] P_a[j, n0 .. n0 + 31] added to a row's sums (a: the adapter of
// the row's request).
__device__ __forceinline__ void add_low(const TcArgs& g, int row, int adapter, int n0, float (&v)[32]) {
    if (adapter < 0) return;
    const int r = g.req.rank;
    const float c = g.scale != nullptr ? g.scale[adapter] : 1.f;
    const float* low = g.low + (size_t)row * r;
    const bf16* P = g.P + (size_t)adapter * r * g.N;
    int at[4];   // columns past the last ones read the last ones: their sums are not kept
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = min(n0 + 8 * k, g.N - 8);
    constexpr int B = 2;   // rows of the adapter under way (volatile: ptxas would sink the loads)
    for (int j0 = 0; j0 < r; j0 += B) {
        uint4 p[B][4];
        float u[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int row_of = min(j0 + j, r - 1);
            u[j] = j0 + j < r ? c * low[row_of] : 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(p[j][k].x), "=r"(p[j][k].y), "=r"(p[j][k].z), "=r"(p[j][k].w)
                             : "l"(P + (size_t)row_of * g.N + at[k]));
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
            if (j0 + j >= r) break;   // (0 times an infinity is not 0)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t w[4] = {p[j][k].x, p[j][k].y, p[j][k].z, p[j][k].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v[8 * k + 2 * q] = fmaf(u[j], __uint_as_float(w[q] << 16), v[8 * k + 2 * q]);
                    v[8 * k + 2 * q + 1] = fmaf(u[j], __uint_as_float(w[q] & 0xffff0000u), v[8 * k + 2 * q + 1]);
                }
            }
        }
    }
}

// K blocks of one sum of a change in TMEM.  The tensor cores truncate as they accumulate, so that
// a sum's error grows with its length; these sums are added in registers, rounding to nearest.
// 2-norm error against float64 of the changes of 4096 x 4096 weights by 2,048 rows a group: 3.0e-7 in sums
// of 8 K blocks, 1.4e-6 of 32 (float32 FMAs in one library product: 4.0e-7).  A drained sum costs the
// epilogue about 500 clocks, which run beside the next sum's MMAs (8 K blocks of 128 x 256: 4,200); sums
// of 32 are 2% faster.  (An adapter's change has up to two products a K block and few columns to drain;
// with sums of two K blocks its error is 5e-7.)
constexpr int kChain = 8, kLowChain = 2;
// And of outputs and hidden deltas, which leave as bfloat16 (an adapter's K of up to 16 steps comes on top):
// the sum of positive products comes out too small by 1e-7 a step of 16, 1.6e-3 over 2^18 products in one
// accumulator, 1.2e-5 in parts of 32 K blocks.  The next part's accumulator takes the last one's sum in, for
// which the MMAs wait once a part: 16,384 rows of 4096-4096 take 1% longer.
constexpr int kRowChain = 32;

template <int BN, int FORM, bool GATHER = false>
__global__ void __launch_bounds__(threads_of(GATHER), 1)
    k_grouped(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ CUtensorMap map_low, const __grid_constant__ CUtensorMap map_p,
              const __grid_constant__ TcArgs g) {
    using C = Cfg<BN, FORM>;
    constexpr int S = C::kStages;
    constexpr bool kLow = is_low(FORM), kChange = FORM == CHANGE || kLow;
    constexpr bool kFinds = kLow || FORM == UP;   // the warp looks for requests together
    constexpr bool kAMn = kChange, kBMn = FORM != FORWARD && FORM != UP;
    constexpr int kChainBlocks = kLow ? kLowChain : kChain;
    constexpr int kAcc = 2;   // the epilogue of a sum overlaps the next one's MMAs
    constexpr int kTmemCols = kAcc * BN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    bf16* stage_out = reinterpret_cast<bf16*>(ring + C::kRingBytes);
    float* bias_s = reinterpret_cast<float*>(ring + C::kRingBytes + C::kOutBytes);   // [kEpiWarps][BN / 2]
    int* s_lo = reinterpret_cast<int*>(ring + C::kRingBytes + C::kOutBytes + C::kBiasBytes);
    int* s_hi = s_lo + BP_MAX_EXPERTS;
    int* s_tile0 = s_hi + BP_MAX_EXPERTS;
    uint64_t* full = reinterpret_cast<uint64_t*>(ring + C::kRingBytes + C::kOutBytes + C::kBiasBytes + C::kGroupBytes);
    uint64_t* empty = full + S;
    uint64_t* tfull = empty + S;
    uint64_t* tempty = tfull + kAcc;
    uint64_t* drain = tempty + kAcc;   // used only when a wait ran out
    uint64_t* xfull = drain + 1;       // of the low form: a warp's block of sums is there for another one; is read
    uint64_t* xempty = xfull + kEpiWarps;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(xempty + kEpiWarps);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    static_assert((2 * S + 2 * kAcc + 1 + 2 * kEpiWarps) * 8 + 8 <= kBarBytes, "room for the barriers");

    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    pdl_launch();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], GATHER ? 1 + kGatherWarps : 1);
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < kAcc; ++a) {
            mbar_init(&tfull[a], 1);
            mbar_init(&tempty[a], kEpiThreads);
        }
        mbar_init(drain, 1);
        for (int e = 0; e < kEpiWarps; ++e) {
            mbar_init(&xfull[e], 32);
            mbar_init(&xempty[e], 32);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_a);
        prefetch_map(&map_b);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();   // every thread, before its first access to what earlier kernels wrote or still read
    if (kLow) {
        // the table of requests; of more than it holds block 0 reports those out of range
        const bool fits = g.req.n_requests <= BP_MAX_EXPERTS;
        if (fits || blockIdx.x == 0)
            for (int i = threadIdx.x; i < g.req.n_requests; i += kThreads) {
                int lo, hi;
                group_rows(g.req.offsets, g.req.n_rows, i, lo, hi, g.flags);
                const int adapter = request_adapter(g.req, i, g.flags);
                if (fits) s_lo[i] = lo, s_hi[i] = hi, s_tile0[i] = adapter;
            }
    } else if (warp == 2) {
        // the groups' rows and first row blocks
        int carry = 0;
        for (int base = 0; base < g.groups.n_groups; base += 32) {
            const int e = base + lane;
            int lo = 0, hi = 0;
            if (e < g.groups.n_groups) group_rows(g.groups.offsets, g.groups.n_rows, e, lo, hi, g.flags);
            const int blocks = (hi - lo + BM - 1) / BM;
            int sum = blocks;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += y;
            }
            if (e < g.groups.n_groups) {
                s_lo[e] = lo;
                s_hi[e] = hi;
                s_tile0[e] = carry + sum - blocks;
            }
            carry += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) s_tile0[g.groups.n_groups] = carry;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    if (FORM == UP && warp >= 2) {
        for (int t = blockIdx.x + gridDim.x * (warp - 2); t < (g.req.n_rows + kTileRows - 1) / kTileRows;
             t += gridDim.x * kEpiWarps) {
            const int2 info = tile_info(g.req, t, g.flags);
            if (lane == 0) g.tiles[t] = info;
        }
        if (blockIdx.x == 0) zero_outside(g.req, threadIdx.x - 64, kEpiThreads, g.low_out, g.terms, g.n_terms * g.stride);
        __syncwarp();
    }
    const bool kept = kLow && g.req.n_requests <= BP_MAX_EXPERTS;
    const Schedule<FORM> plan{g, s_lo, s_hi, s_tile0, {kept ? s_tile0 : nullptr, s_lo, s_hi}};
    const int items = plan.items();

    if (warp == 0) {
        // ---------------- copies, by one lane
        const bool leader = elect_one();
        if (kFinds || leader) {
            int stage = 0, issued = 0;
            unsigned phase = 0;
            bool ok = true;
            // The stage's buffer is free and its barrier expects `bytes`.
            auto open = [&](unsigned bytes) {
                if (issued >= S) {
                    ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag, g.flags);
                    if (kFinds) ok = __all_sync(0xffffffffu, ok);
                }
                if (ok && leader) mbar_expect_tx(&full[stage], bytes);
                return ok;
            };
            auto close = [&] {
                ++issued;
                if (++stage == S) { stage = 0; phase ^= 1u; }
            };
            const int a_blocks = kLow ? 2 * low_sets(g) : BM / 64;
            for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
                const Item w = plan.item(it);
                if constexpr (kChange) {
                    Stretches<FORM> rows{g, w, plan.table, 0, 0};
                    int lo, hi;
                    while (ok && rows.next(lo, hi)) {
                        for (int r = lo; r < hi; r += BK) {
                            if (!open(a_blocks * kMnBlockBytes + C::kBBytes)) break;
                            uint8_t *sa = ring + stage * C::kStageBytes, *sb = sa + C::kABytes;
                            if (leader) {
                                const CUtensorMap* ma = kLow && w.second ? &map_low : &map_a;
                                const CUtensorMap* mb = kLow && w.second ? &map_p : &map_b;
                                for (int i = 0; i < a_blocks; ++i)
                                    tma_load_2d(sa + i * kMnBlockBytes, ma, w.mb * BM + 64 * i, r, &full[stage]);
#pragma unroll
                                for (int i = 0; i < BN / 64; ++i)
                                    tma_load_2d(sb + i * kMnBlockBytes, mb, w.nb * BN + 64 * i, r, &full[stage]);
                            }
                            close();
                        }
                    }
                } else {
                    for (int kb = 0; kb < w.kbs; ++kb) {
                        if (!open(GATHER ? C::kBBytes : C::kStageBytes)) break;
                        uint8_t *sa = ring + stage * C::kStageBytes, *sb = sa + C::kABytes;
                        if (!GATHER && leader) tma_load_2d(sa, &map_a, kb * BK, w.row0, &full[stage]);
                        if (FORM == UP) {
                            if (leader) tma_load_3d(sb, &map_b, kb * BK, 0, w.adapter, &full[stage]);
                        } else if (FORM == FORWARD) {
                            tma_load_3d(sb, &map_b, kb * BK, w.nb * BN, w.g, &full[stage]);
                        } else {
#pragma unroll
                            for (int i = 0; i < BN / 64; ++i)
                                tma_load_3d(sb + i * kMnBlockBytes, &map_b, w.nb * BN + 64 * i, kb * BK, w.g, &full[stage]);
                        }
                        close();
                    }
                    if constexpr (FORM != UP && !GATHER) {
                        // the low-rank K of one adapter, up to 4 pieces of 16 of a term a stage
                        auto load_low = [&](int adapter) {
                            for (int t = 0; t < kForwardTerms; ++t)
                                for (int c0 = 0; c0 < g.rank16 && ok; c0 += 4) {
                                    const int n = min(4, g.rank16 - c0);
                                    if (!open(C::kABytes + n * 16 * BN * 2)) break;
                                    uint8_t *sa = ring + stage * C::kStageBytes, *sb = sa + C::kABytes;
                                    tma_load_2d(sa, &map_low, t * g.stride + c0 * 16, w.row0, &full[stage]);
                                    for (int c = 0; c < n; ++c)
                                        for (int i = 0; i < BN / 64; ++i)
                                            tma_load_3d(sb + i * kMnBlockBytes + c * 16 * 128, &map_p, w.nb * BN + 64 * i,
                                                        (c0 + c) * 16, adapter, &full[stage]);
                                    close();
                                }
                        };
                        if (ok && w.adapter >= 0) load_low(w.adapter);
                        if (ok && w.adapter == kTileMixed) {
                            TileRequests all{g, w, w.request};
                            int lo, hi, adapter;
                            while (ok && all.next(lo, hi, adapter)) load_low(adapter);
                        }
                    }
                }
            }
            if (!ok && leader) {
                // let every copy already issued land before the CTA can exit
                for (int n = issued - 1; n >= 0 && n >= issued - S; --n) {   // each stage's last copy
                    const unsigned long long t0 = global_ns();
                    while (!mbar_try_wait(&full[n % S], (unsigned)(n / S) & 1u) && global_ns() - t0 < kWaitNs) {
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA: one lane issues; of a change the warp clears foreign rows
        const bool leader = elect_one();
        if (kChange || kFinds || leader) {
            constexpr uint32_t idesc = idesc_bf16(BM, BN, kAMn, kBMn), idesc_low = idesc_bf16(BM, BN, false, true);
            const uint32_t a0 = desc_lo<kAMn>(smem_u32(ring)), b0 = desc_lo<kBMn>(smem_u32(ring) + C::kABytes);
            int stage = 0, acc = 0;
            unsigned phase = 0, acc_phase = 0;
            bool ok = true, issued_any = false;
            auto wait = [&](uint64_t* bar, unsigned parity) {
                ok = mbar_wait(bar, parity, abort_flag, g.flags);
                if (kChange || kFinds) ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                return ok;
            };
            auto close = [&] {
                if (leader) umma_commit(&empty[stage]);
                issued_any = true;
                if (++stage == S) { stage = 0; phase ^= 1u; }
            };
            auto done = [&] {   // the accumulator's sum is complete
                if (leader) umma_commit(&tfull[acc]);
                if (++acc == kAcc) { acc = 0; acc_phase ^= 1u; }
            };
            for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
                const Item w = plan.item(it);
                if constexpr (kChange) {
                    const int sets = kLow ? low_sets(g) : 1;   // of 128 rows of M
                    Stretches<FORM> rows{g, w, plan.table, 0, 0};
                    int lo, hi, kb = 0;
                    while (ok && rows.next(lo, hi)) {
                        for (int r = lo; r < hi; r += BK, ++kb) {
                            if (kb % kChainBlocks == 0 && !wait(&tempty[acc], acc_phase ^ 1u)) break;
                            if (!wait(&full[stage], phase)) break;
                            const uint32_t tmem_d = tmem_base + (uint32_t)(acc * BN);
                            const uint32_t al = a0 + stage * (C::kStageBytes >> 4), bl = b0 + stage * (C::kStageBytes >> 4);
                            int steps = BK / UMMA_K;
                            const int valid = hi - r;
                            if (valid < BK) {   // (uniform) the run's last rows
                                steps = (valid + UMMA_K - 1) / UMMA_K;
                                uint8_t* sa = ring + stage * C::kStageBytes;
                                zero_rows(sa, 2 * sets, valid, steps * UMMA_K);
                                zero_rows(sa + C::kABytes, BN / 64, valid, steps * UMMA_K);
                                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                                __syncwarp();
                            }
                            if (leader) {
                                for (int t = 0; t < sets; ++t)
#pragma unroll
                                    for (int kk = 0; kk < BK / UMMA_K; ++kk)
                                        if (kk < steps)
                                            umma_bf16<idesc>(tmem_d, al + t * (2 * kMnBlockBytes >> 4) + kk * k_step_units<kAMn>(),
                                                             bl + kk * k_step_units<kBMn>(), kb % kChainBlocks != 0 || t > 0 || kk > 0 ? 1u : 0u);
                            }
                            close();
                            if (kb % kChainBlocks == kChainBlocks - 1 || kb == w.kbs - 1) done();
                        }
                    }
                } else {
                    constexpr int chain = FORM == UP ? kChain : kRowChain;
                    for (int k0 = 0; k0 < w.kbs && ok; k0 += chain) {
                        const int k1 = min(w.kbs, k0 + chain);
                        if (!wait(&tempty[acc], acc_phase ^ 1u)) break;
                        const uint32_t tmem_d = tmem_base + (uint32_t)(acc * BN);
                        for (int kb = k0; kb < k1; ++kb) {
                            if (!wait(&full[stage], phase)) break;
                            const uint32_t al = a0 + stage * (C::kStageBytes >> 4), bl = b0 + stage * (C::kStageBytes >> 4);
                            if (leader) {
                                umma_bf16<idesc>(tmem_d, al, bl, kb > k0 ? 1u : 0u);
#pragma unroll
                                for (int kk = 1; kk < BK / UMMA_K; ++kk)
                                    umma_bf16<idesc>(tmem_d, al + kk * k_step_units<kAMn>(), bl + kk * k_step_units<kBMn>(), 1u);
                            }
                            close();
                        }
                        if constexpr (FORM != UP && !GATHER) {
                            const uint32_t low_b0 = desc_lo<true>(smem_u32(ring) + C::kABytes);
                            auto add_low = [&](bool fresh) {   // into accumulator acc
                                const uint32_t d = tmem_base + (uint32_t)(acc * BN);
                                for (int t = 0; t < kForwardTerms; ++t)
                                    for (int c0 = 0; c0 < g.rank16 && ok; c0 += 4) {
                                        if (!wait(&full[stage], phase)) break;
                                        const uint32_t al = a0 + stage * (C::kStageBytes >> 4), bl = low_b0 + stage * (C::kStageBytes >> 4);
                                        for (int c = 0; c < min(4, g.rank16 - c0); ++c) {
                                            umma_bf16<idesc_low>(d, al + c * k_step_units<false>(), bl + c * k_step_units<true>(), fresh ? 0u : 1u);
                                            fresh = false;
                                        }
                                        close();
                                    }
                            };
                            if (ok && k1 == w.kbs && w.adapter >= 0) add_low(false);
                            if (ok && k1 == w.kbs && w.adapter == kTileMixed) {
                                TileRequests all{g, w, w.request};
                                int lo, hi, adapter;
                                while (ok && all.next(lo, hi, adapter)) {
                                    done();
                                    if (!wait(&tempty[acc], acc_phase ^ 1u)) break;
                                    add_low(true);
                                }
                            }
                        }
                        if (ok) done();
                    }
                }
            }
            if (!ok && issued_any && leader) {
                // let every MMA already issued finish before TMEM is released
                umma_commit(drain);
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(drain, 0) && global_ns() - t0 < kWaitNs) {
                }
            }
        }
    } else if (GATHER && warp >= 2 + kEpiWarps) {
        // ---------------- gather: a warp 32 rows of the tile, eight lanes the 128 bytes of a row in a K block
        const int m0 = (warp - 2 - kEpiWarps) * 32 + (lane >> 3), c = lane & 7;   // rows m0, m0 + 4, ..; piece c
        constexpr int kAhead = S - 2;   // K blocks whose copies are under way when the next one's are issued
        int stage = 0, issued = 0;
        unsigned phase = 0;
        bool ok = true;
        auto signal = [&](int block) {   // this warp's rows of a block are there, for the tensor cores to read
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&full[block % S]);
        };
        for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
            const Item w = plan.item(it);
            // rows past the group's end are zeros, which cost no read (the last row again in their place: a
            // tile of 15 rows took 52 us for 14, its copies all of one line)
            const bf16* from[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = w.row0 + m0 + 4 * i;
                from[i] = row < w.end ? g.in + (size_t)source_row(g.source, row, g.n_in_rows, g.flags) * g.K : nullptr;
            }
            for (int kb = 0; kb < w.kbs; ++kb) {
                if (issued >= S) {
                    ok = mbar_wait(&empty[stage], phase ^ 1u, abort_flag, g.flags);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                }
                const uint32_t to = smem_u32(ring + stage * C::kStageBytes) + m0 * 128;
                const int k = kb * BK + 8 * c;
#pragma unroll
                for (int i = 0; i < 8; ++i) {   // (128-byte swizzle: piece c of row m lies at c ^ (m mod 8))
                    const bool read = k < g.K && from[i] != nullptr;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + 512 * i + ((c ^ ((m0 + 4 * i) & 7)) << 4)),
                                 "l"(read ? from[i] + k : g.in), "r"(read ? 16 : 0)
                                 : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                ++issued;
                if (++stage == S) { stage = 0; phase ^= 1u; }
                if (issued > kAhead) {
                    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
                    signal(issued - 1 - kAhead);
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");   // every copy lands before the CTA can exit
        for (int b = max(issued - kAhead, 0); ok && b < issued; ++b) signal(b);
    } else {
        // ---------------- epilogue warps 2..9
        const int q = warp & 3;                  // TMEM lane quarter this warp may access
        const int ew = warp - 2;
        const int cbeg = (ew >> 2) * (BN / 2);   // this warp's half of the columns
        const uint32_t trow = tmem_base + ((uint32_t)(q * 32) << 16);
        uint4* sS4 = reinterpret_cast<uint4*>(stage_out + ew * 1024);
        int acc = 0;
        unsigned acc_phase = 0, xphase = 0;
        // the warp of this one's half of the columns that has row quarter `quarter`
        auto half_warp = [&](int quarter) { return (ew & 4) + ((quarter + 2) & 3); };
        auto wait_acc = [&] {
            const bool got = mbar_wait(&tfull[acc], acc_phase, abort_flag, g.flags);
            const bool leave = __any_sync(0xffffffffu, !got);
            tc_fence_after();
            return !leave;
        };
        auto free_acc = [&](int a) {
            tc_fence_before();
            mbar_arrive(&tempty[a]);
        };
        auto next_acc = [&] {
            if (++acc == kAcc) { acc = 0; acc_phase ^= 1u; }
        };
        auto release = [&] {
            free_acc(acc);
            next_acc();
        };
        for (int it = blockIdx.x; it < items; it += gridDim.x) {
            const Item w = plan.item(it);
            if constexpr (kChange || FORM == UP) {
                if (kLow && w.run >= w.shares) continue;   // left to the first share
                float part[BN / 2];
#pragma unroll
                for (int c = 0; c < BN / 2; ++c) part[c] = 0.f;
                bool stay = true;
                for (int k0 = 0; k0 < w.kbs; k0 += kChainBlocks) {
                    stay = wait_acc();
                    if (!stay) break;
#pragma unroll
                    for (int i = 0; i < BN / 64; ++i) {
                        float v[32];
                        tmem_ld32(trow + (uint32_t)(acc * BN + cbeg + 32 * i), v);
#pragma unroll
                        for (int c = 0; c < 32; ++c) part[32 * i + c] += v[c];
                    }
                    release();
                }
                if (!stay) break;
                if constexpr (FORM == UP) {
                    if (w.request < 0) continue;
                    const float scale = g.scale != nullptr && w.adapter >= 0 ? g.scale[w.adapter] : 1.f;
                    const int row0 = w.row0 + q * 32;
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 16) {
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = (g.scaled_low ? scale : 1.f) * part[c + i];
                        store_low(g.low_out, g.req.rank, row0, w.end, cbeg + c, v, g.wide_low, reinterpret_cast<float4*>(sS4));
                    }
                    for (int t = 0; t < g.n_terms; ++t) {
#pragma unroll
                        for (int c = 0; c < BN / 2; c += 32) {
                            if (cbeg + c >= g.stride) break;
                            float v[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) {   // part keeps what the terms so far leave
                                const float x = t == 0 ? (cbeg + c + i < g.req.rank ? scale * part[c + i] : 0.f) : part[c + i];
                                v[i] = x;
                                const float h = __bfloat162float(__float2bfloat16_rn(x));
                                part[c + i] = isfinite(h) ? x - h : 0.f;
                            }
                            store_rows(g.terms, g.n_terms * g.stride, row0, w.end, t * g.stride + cbeg + c, v, sS4);
                        }
                    }
                    continue;
                }
                if (kLow && g.stride < BM && w.kbs == 0) {
                    if (q >= g.stride / 32) continue;   // no sums to pass on
                } else if (kLow && g.stride < BM) {
                    // row quarters past the first term's: the same ranks of other terms, passed on to it
                    const int own = g.stride / 32, last = min(4, own * g.n_terms);
                    float* block = reinterpret_cast<float*>(stage_out);   // [warp][16][32]
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 16) {
                        if (q >= own) {
                            if (q < last) {
                                stay = mbar_wait(&xempty[ew], xphase ^ 1u, abort_flag, g.flags);
                                stay = !__any_sync(0xffffffffu, !stay);
                                if (!stay) break;
#pragma unroll
                                for (int i = 0; i < 16; ++i) block[ew * 512 + i * 32 + lane] = part[c + i];
                                mbar_arrive(&xfull[ew]);
                            }
                        } else {
                            for (int from = q + own; from < last; from += own) {
                                const int src = half_warp(from);
                                stay = mbar_wait(&xfull[src], xphase, abort_flag, g.flags);
                                stay = !__any_sync(0xffffffffu, !stay);
                                if (!stay) break;
#pragma unroll
                                for (int i = 0; i < 16; ++i) part[c + i] += block[src * 512 + i * 32 + lane];
                                mbar_arrive(&xempty[src]);
                            }
                            if (!stay) break;
                        }
                        xphase ^= 1u;
                    }
                    if (!stay) break;
                    __syncwarp();
                    if (q >= own) continue;
                }
                const bool second = kLow && w.second;
                const int N = second ? g.N2 : g.N;
                const float* scales = second ? g.scale2 : g.scale;
                const float scale = kLow && scales != nullptr ? scales[w.g] : 1.f;
                const int m0 = w.mb * BM + q * 32;
                float* G = (second ? g.G2 : g.G) + (size_t)w.g * g.M * N;
                if (kLow && w.shares > 1) {
                    // the run's sums to scratch; the last warp to arrive adds the runs' in their order
                    if (m0 >= g.M || w.nb * BN + cbeg >= N) continue;
                    const size_t plane = (size_t)g.req.n_adapters * g.M * N;
                    float* shared_out = g.scratch + (second ? (size_t)g.runs * g.req.n_adapters * g.M * g.N : 0);
                    float* mine = shared_out + w.run * plane + (size_t)w.g * g.M * N;
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 16) {
                        const int n0 = w.nb * BN + cbeg + c;
                        if (n0 >= N) break;
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = part[c + i];
                        store_change(mine, g.M, N, m0, n0, v, 0, reinterpret_cast<float4*>(sS4));
                    }
                    __threadfence();
                    __syncwarp();
                    unsigned before = 0;
                    unsigned* count = g.arrived + (second ? (size_t)g.req.n_adapters * g.num_n * kEpiWarps : 0) +
                                      ((size_t)w.g * (second ? g.num_n2 : g.num_n) + w.nb) * kEpiWarps + ew;
                    if (lane == 0) before = atomicAdd(count, 1u);
                    before = __shfl_sync(0xffffffffu, before, 0);
                    if (before != (unsigned)w.shares - 1) continue;
                    if (lane == 0) *count = 0u;
                    __threadfence();
                    const float* all = shared_out + (size_t)w.g * g.M * N;
                    // pieces of four columns: lane + 32 i of the part's, by rows; all loads of a run under way at once
                    constexpr int kPer = BN / 2 / 4;   // of a row
                    float4 sum[kPer];
#pragma unroll
                    for (int i = 0; i < kPer; ++i) sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    // rows and columns past the last ones read the last ones, so that no load hangs on a condition
                    const float* at = all + (size_t)min(m0 + lane / kPer, g.M - 1) * N + min(w.nb * BN + cbeg + lane % kPer * 4, N - 4);
                    for (int z = 0; z < w.shares; ++z) {
#pragma unroll
                        for (int i = 0; i < kPer; ++i) {
                            const int row = min(32 / kPer * i, max(g.M - 1 - m0 - lane / kPer, 0));
                            const float4 x = __ldcg(reinterpret_cast<const float4*>(at + z * plane + (size_t)row * N));
                            sum[i].x += x.x, sum[i].y += x.y, sum[i].z += x.z, sum[i].w += x.w;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const int m = m0 + (lane + 32 * i) / kPer, n = w.nb * BN + cbeg + (lane + 32 * i) % kPer * 4;
                        if (m >= g.M || n >= N) continue;
                        float4 o = make_float4(scale * sum[i].x, scale * sum[i].y, scale * sum[i].z, scale * sum[i].w);
                        float4* to = reinterpret_cast<float4*>(G + (size_t)m * N + n);
                        if (g.accumulate) {
                            const float4 old = *to;
                            o.x += old.x, o.y += old.y, o.z += old.z, o.w += old.w;
                        }
                        *to = o;
                    }
                    continue;
                }
#pragma unroll
                for (int c = 0; c < BN / 2; c += 16) {
                    const int n0 = w.nb * BN + cbeg + c;
                    if (m0 >= g.M || n0 >= N) break;
                    float v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = scale * part[c + i];
                    if ((second ? g.sectors2 : g.sectors) && !g.accumulate) {
                        if (m0 + lane < g.M) store_sectors(G + (size_t)(m0 + lane) * N + n0, v, N - n0);
                    } else {
                        store_change(G, g.M, N, m0, n0, v, g.accumulate, reinterpret_cast<float4*>(sS4));
                    }
                }
            } else {
                const int m0 = w.row0 + q * 32, row = m0 + lane;
                float* sbias = bias_s + ew * (BN / 2);
                if (FORM == FORWARD) {
                    __syncwarp();   // the tile before is read
                    for (int c = lane; c < BN / 2; c += 32) {
                        const int n = w.nb * BN + cbeg + c;
                        sbias[c] = g.bias != nullptr && n < g.N ? g.bias[(size_t)w.g * g.N + n] : 0.f;
                    }
                    __syncwarp();
                }
                int xr[4] = {0, 0, 0, 0};   // source rows of this lane's pieces (back)
                if (FORM == BACK && g.squash) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = m0 + 8 * j + (lane >> 2);
                        xr[j] = r < w.end ? source_row(g.x_source, r, g.n_x, g.flags) : -1;
                    }
                }
                int adapter = -1;   // of this lane's row, in a tile that is taken row by row
                if (!GATHER && w.adapter == kTileByRow && row < w.end) {
                    const int i = first_request(g.req, row);
                    if (i < g.req.n_requests) {
                        int lo, hi;
                        group_rows(g.req.offsets, g.req.n_rows, i, lo, hi, g.flags);
                        if (row >= lo && row < hi) adapter = request_adapter(g.req, i, g.flags);
                    }
                }
                if (!wait_acc()) break;
                // The next accumulator, with the sums so far added to its own or, in rows that its own are
                // not for, in place of them.
                auto join = [&](bool mine) {
                    const int before = acc;
                    next_acc();
                    if (!wait_acc()) return false;
#pragma unroll 1
                    for (int c = 0; c < BN / 2; c += 16) {
                        float x[16], v[16];
                        tmem_ld16(trow + (uint32_t)(before * BN + cbeg + c), x);
                        tmem_ld16(trow + (uint32_t)(acc * BN + cbeg + c), v);
#pragma unroll
                        for (int k = 0; k < 16; ++k) v[k] = mine ? x[k] + v[k] : x[k];
                        tmem_st16(trow + (uint32_t)(acc * BN + cbeg + c), v);
                    }
                    tmem_wait_st();
                    free_acc(before);
                    return true;
                };
                bool stay = true;
                for (int k0 = kRowChain; k0 < w.kbs && stay; k0 += kRowChain) stay = join(true);
                if (!stay) break;
                if (!GATHER && w.adapter == kTileMixed) {   // each request's sums, for its rows
                    TileRequests all{g, w, w.request};
                    int lo, hi, a;
                    while (stay && all.next(lo, hi, a)) stay = join(row >= lo && row < hi);
                    if (!stay) break;
                }
#pragma unroll 1
                for (int i = 0; i < BN / 64; ++i) {
                    const int c0 = 32 * i, n0 = w.nb * BN + cbeg + c0;
                    if (n0 >= g.N) break;
                    Row32 a;
                    if (FORM == BACK && g.squash) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int n = n0 + (lane & 3) * 8;
                            a.u[j] = xr[j] >= 0 && n < g.N ? *reinterpret_cast<const uint4*>(g.x + (size_t)xr[j] * g.N + n)
                                                           : make_uint4(0u, 0u, 0u, 0u);
                        }
                    }
                    float v[32];
                    tmem_ld32(trow + (uint32_t)(acc * BN + cbeg + c0), v);
                    if (!GATHER && w.adapter == kTileByRow) add_low(g, row, adapter, n0, v);
                    if (FORM == FORWARD) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 f = reinterpret_cast<const float4*>(sbias + c0)[k];
                            v[4 * k] += f.x;
                            v[4 * k + 1] += f.y;
                            v[4 * k + 2] += f.z;
                            v[4 * k + 3] += f.w;
                        }
                        if (g.squash) {
#pragma unroll
                            for (int c = 0; c < 32; ++c) v[c] = sigmoid_fast(v[c]);
                        }
                    } else if (g.squash) {
                        block_to_rows(a, sS4);
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            const float x = row_value(a, c);
                            v[c] = v[c] * x * (1.f - x);
                        }
                    }
                    store_rows(g.out, g.N, m0, w.end, n0, v, sS4);
                }
                release();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    }
}

// Rows read through an index, copied into the groups' order, 16 bytes a thread.
__global__ void __launch_bounds__(256)
    k_gather(const uint4* in, const int* source, int n_src, RowGroups q, int pieces, uint4* out, int* flags) {
    pdl_launch();
    pdl_wait();
    const int first = max(q.offsets[0], 0), end = min(q.offsets[q.n_groups], q.n_rows);
    for (int r = first + blockIdx.x * blockDim.y + threadIdx.y; r < end; r += gridDim.x * blockDim.y) {
        const uint4* from = in + (size_t)source_row(source, r, n_src, flags) * pieces;
        uint4* to = out + (size_t)r * pieces;
        int c = threadIdx.x;
        for (; c + 3 * (int)blockDim.x < pieces; c += 4 * blockDim.x) {
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = from[c + i * blockDim.x];
#pragma unroll
            for (int i = 0; i < 4; ++i) to[c + i * blockDim.x] = v[i];
        }
        for (; c < pieces; c += blockDim.x) to[c] = from[c];
    }
}

// ------------------------------------------------------------ host
PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;

// A row-major bfloat16 matrix, or `planes` of them (planes > 0), copied in boxes of 64 columns.
bool make_map(CUtensorMap* map, const void* base, int rows, int cols, int planes, int box_rows) {
    const int rank = planes > 0 ? 3 : 2;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)cols * rows * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, int FORM, bool GATHER = false>
cudaError_t setup_one() {
    return cudaFuncSetAttribute(k_grouped<BN, FORM, GATHER>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<BN, FORM>::kSmemBytes);
}
template <int BN>
cudaError_t setup_width() {
    cudaError_t e;
    if ((e = setup_one<BN, FORWARD>()) != cudaSuccess) return e;
    if ((e = setup_one<BN, FORWARD, true>()) != cudaSuccess) return e;
    if ((e = setup_one<BN, BACK>()) != cudaSuccess) return e;
    return setup_one<BN, CHANGE>();
}

template <int FORM, bool GATHER = false>
cudaError_t launch(const TcArgs& a, int bn, int items, int num_sms, const CUtensorMap (&m)[4], cudaStream_t s) {
    const int grid = items < num_sms ? items : num_sms;
    if (grid < 1) return cudaSuccess;
    auto go = [&](auto k, int smem) { return launch_pdl(k, grid, 1, threads_of(GATHER), smem, s, m[0], m[1], m[2], m[3], a); };
    if (bn == 64) return go(k_grouped<64, FORM, GATHER>, Cfg<64, FORM>::kSmemBytes);
    if (bn == 128 || is_low(FORM) || FORM == UP) return go(k_grouped<128, FORM, GATHER>, Cfg<128, FORM>::kSmemBytes);
    if constexpr (!is_low(FORM) && FORM != UP) return go(k_grouped<256, FORM, GATHER>, Cfg<256, FORM>::kSmemBytes);
    return cudaErrorInvalidValue;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

constexpr int kShareColumns = 1024;   // an SM
constexpr int kMaxShares = 16, kShareRows = 16 * BK;   // of an adapter; rows that a share is for
struct LowCut {
    int bn, num_n, num_n2, runs;
};

// Tile width for row_tiles blocks of 128 rows: the time of the waves of tiles, at the clocks that
// a K block of 64 takes with every SM busy (530, 330 and 230 for 256, 128 and 64 columns: each SM
// reads A again for every column block) and an epilogue of 800 + 900 a 64 columns, whichever is
// longer, plus the other one once.
int pick_width(long long row_tiles, int N, int kbs, int num_sms) {
    const int bns[3] = {256, 128, 64}, clocks[3] = {530, 330, 230};
    int best = 256;
    double best_t = 0;
    for (int i = 0; i < 3; ++i) {
        const double waves = ceil_div(row_tiles * ceil_div(N, bns[i]), num_sms);
        const double k = (double)kbs * clocks[i], e = 800.0 + 900.0 * bns[i] / 64;
        const double t = waves * (k > e ? k : e) + (k > e ? e : k);
        if (i == 0 || t < best_t) best = bns[i], best_t = t;
    }
    return best;
}

}  // namespace

cudaError_t tc_setup() {
    static std::once_flag once;
    static cudaError_t status;
    std::call_once(once, [] {
        g_encode = tensor_map_encoder();
        status = g_encode == nullptr ? cudaErrorNotSupported : cudaSuccess;
    });
    if (status != cudaSuccess) return status;
    cudaError_t e;
    if ((e = setup_width<64>()) != cudaSuccess) return e;
    if ((e = setup_width<128>()) != cudaSuccess) return e;
    if ((e = setup_width<256>()) != cudaSuccess) return e;
    if ((e = setup_one<64, LOW>()) != cudaSuccess) return e;
    if ((e = setup_one<128, LOW>()) != cudaSuccess) return e;
    if ((e = setup_one<64, LOW_WIDE>()) != cudaSuccess) return e;
    if ((e = setup_one<128, LOW_WIDE>()) != cudaSuccess) return e;
    if ((e = setup_one<64, UP>()) != cudaSuccess) return e;
    return setup_one<128, UP>();
}

cudaError_t tc_gather(const void* in, const int* source, int n_src, const RowGroups& groups, int cols, void* out, int* flags,
                      int num_sms, cudaStream_t s) {
    const int pieces = cols / 8;
    int x = 32;
    while (x < 256 && x * 4 < pieces) x *= 2;   // threads of a row
    const int per = 256 / x, want = ceil_div(groups.n_rows, per);
    return launch_pdl_grid(k_gather, dim3(want < 8 * num_sms ? want : 8 * num_sms), dim3(x, per), 0, s, (const uint4*)in, source, n_src,
                           groups, pieces, (uint4*)out, flags);
}

cudaError_t tc_rows(const RowsArgs& r, bool back, const LowTerms& low, int num_sms, cudaStream_t s) {
    TcArgs a{};
    a.groups = r.groups;
    a.N = r.N;
    a.K = r.K;
    a.in = (const bf16*)r.in;
    a.source = r.source;
    a.n_in_rows = r.n_in_rows;
    a.bias = r.bias;
    a.squash = r.squash;
    a.x = (const bf16*)r.x;
    a.x_source = r.x_source;
    a.n_x = r.n_x;
    a.out = (bf16*)r.out;
    a.flags = r.flags;
    const int E = r.groups.n_groups, kbs = ceil_div(r.K, BK);
    // row blocks: every group's, about as many rows in each (the groups' sizes are on the device)
    const long long busy = E < r.groups.n_rows ? E : r.groups.n_rows;
    const long long row_tiles = busy * ceil_div(r.groups.n_rows, busy * BM);
    const int bn = pick_width(row_tiles, r.N, kbs, num_sms);
    a.num_n = ceil_div(r.N, bn);
    CUtensorMap m[4];
    bool ok = make_map(&m[0], r.in, r.n_in_rows, r.K, 0, BM) &&
              (back ? make_map(&m[1], r.W, r.K, r.N, E, BK) : make_map(&m[1], r.W, r.N, r.K, E, bn));
    m[2] = m[3] = m[0];
    if (r.low != nullptr && r.req.n_requests > 0) {   // (without requests P may be NULL)
        a.tiles = low.tiles;
        a.rank16 = ceil_div(r.req.rank, 16);
        a.stride = low.stride;
        a.req = r.req;
        a.low = r.low;
        a.P = (const bf16*)r.P;
        a.scale = r.scale;
        ok = ok && make_map(&m[2], low.terms, r.groups.n_rows, low.n_terms * low.stride, 0, BM) &&
             make_map(&m[3], r.P, r.req.rank, r.N, r.req.n_adapters, 16);
    }
    if (!ok) return cudaErrorInvalidValue;
    const long long items = (long long)max_tiles(r.groups.n_rows, E, BM) * a.num_n;
    const int n = items < num_sms ? (int)items : num_sms;
    if (back) return launch<BACK>(a, bn, n, num_sms, m, s);
    return r.source != nullptr ? launch<FORWARD, true>(a, bn, n, num_sms, m, s) : launch<FORWARD>(a, bn, n, num_sms, m, s);
}

cudaError_t tc_change(const ChangeArgs& c, int num_sms, cudaStream_t s) {
    TcArgs a{};
    a.groups = c.groups;
    a.M = c.M;
    a.N = c.N;
    a.G = c.G;
    a.accumulate = c.accumulate;
    a.sectors = ((uintptr_t)c.G & 31) == 0;
    a.flags = c.flags;
    a.num_m = ceil_div(c.M, BM);
    const int E = c.groups.n_groups;
    const int bn = pick_width((long long)E * a.num_m, c.N, ceil_div(c.groups.n_rows, (long long)E * BK), num_sms);
    a.num_n = ceil_div(c.N, bn);
    CUtensorMap m[4];
    // without rows nothing is copied and the maps' addresses are not used; G stands in for them
    const bool rows = c.groups.n_rows > 0;
    if (!make_map(&m[0], rows ? c.a : c.G, rows ? c.groups.n_rows : 1, c.M, 0, BK) ||
        !make_map(&m[1], rows ? c.b : c.G, rows ? c.n_b : 1, c.N, 0, BK))
        return cudaErrorInvalidValue;
    m[2] = m[3] = m[0];
    const long long items = (long long)E * a.num_m * a.num_n;
    const int n = items < num_sms ? (int)items : num_sms;
    return launch<CHANGE>(a, bn, n, num_sms, m, s);
}

cudaError_t tc_low(const LowArgs& l, int num_sms, cudaStream_t s) {
    TcArgs a{};
    a.req = l.req;
    a.K = l.K;
    a.num_n = 1;
    a.scale = l.scale;
    a.scaled_low = l.scaled_low;
    a.low_out = l.low;
    a.wide_low = l.req.rank % 4 == 0 && ((uintptr_t)l.low & 15) == 0;
    a.terms = (bf16*)l.terms;
    a.n_terms = l.n_terms;
    a.stride = l.terms_stride;
    a.tiles = l.tiles;
    a.flags = l.flags;
    a.max_items = max_tiles(l.req.n_rows, l.req.n_requests, BM);
    const int bn = l.req.rank <= 64 ? 64 : 128;   // at least the terms' stride: the tile writes them in full
    CUtensorMap m[4];
    if (!make_map(&m[0], l.in, l.req.n_rows, l.K, 0, BM) || !make_map(&m[1], l.P, l.req.rank, l.K, l.req.n_adapters, bn))
        return cudaErrorInvalidValue;
    m[2] = m[3] = m[0];
    return launch<UP>(a, bn, a.max_items < num_sms ? a.max_items : num_sms, num_sms, m, s);
}

// How a low change is cut: 128 columns, 64 where that leaves SMs without a tile, and up to 16 shares of
// an adapter's rows, as many as the device finds that it has times an SM's part (Schedule::item), where
// the busy tiles are no more than the SMs, there are rows for them, the items stay few (each is a look at
// the requests, 0.8 us) and the shares' sums fit their scratch.  A share is an exchange, a store and a
// fence of 5 us beside its 0.5 us a K block: us of both changes of a layer of 16,384 rows, a launch each,
// every adapter in 1 / 2 / 4 / 16 shares: 5 adapters of rank 64 of 4096-4096, 160 tiles, 142 / 194 / 295 /
// 297; one of rank 16, 64 tiles, 233 / 145 / 159 / 268; 4 of 512-512, 32 tiles, 206 / 118 / 75 / 63.
static LowCut low_cut(int n_adapters, int n_requests, int n_rows, int N, int N2, int num_sms) {
    const int busy = n_adapters < n_requests ? n_adapters : n_requests;
    LowCut c;
    c.bn = (long long)busy * (ceil_div(N, 128) + ceil_div(N2, 128)) >= num_sms / 4 ? 128 : 64;
    c.num_n = ceil_div(N, c.bn);
    c.num_n2 = ceil_div(N2, c.bn);
    c.runs = 1;
    const long long tiles = c.num_n + c.num_n2;
    while (c.runs < kMaxShares && n_rows >= 2 * c.runs * kShareRows && c.runs * busy * tiles <= num_sms &&
           2 * c.runs * n_adapters * tiles <= 8 * num_sms && 2ll * c.runs * n_adapters * ((long long)N + N2) <= kShareColumns * num_sms)
        c.runs *= 2;
    return c;
}

// Of any call of a layer: columns of shares, and the warps' parts of 64 of them.
size_t low_change_scratch(int n_adapters, int rank, int columns, int max_rows, int num_sms) {
    if (max_rows < 2 * kShareRows) return 0;
    const size_t most = (size_t)kShareColumns * num_sms, all = (size_t)kMaxShares * n_adapters * columns;
    return rank * (all < most ? all : most);
}
size_t low_change_counts(int n_adapters, int num_sms) {
    return ((size_t)kShareColumns / 64 * num_sms + 2 * n_adapters) * kEpiWarps;
}

cudaError_t tc_low_change(const LowChangeArgs& c, const LowTerms& low, const LowChangeArgs* c2, const LowTerms& low2, int num_sms,
                          cudaStream_t s) {
    TcArgs a{};
    a.req = c.req;
    a.M = c.req.rank;
    a.N = c.N;
    a.G = c.G;
    a.scale = c.scale;
    a.accumulate = c.accumulate;
    a.sectors = ((uintptr_t)c.G & 31) == 0;
    if (c2 != nullptr) {
        a.N2 = c2->N;
        a.G2 = c2->G;
        a.scale2 = c2->scale;
        a.sectors2 = ((uintptr_t)c2->G & 31) == 0;
    }
    a.n_terms = low.n_terms;
    a.stride = low.stride;
    a.flags = c.flags;
    const LowCut cut = low_cut(c.req.n_adapters, c.req.n_requests, c.req.n_rows, c.N, a.N2, num_sms);
    a.num_n = cut.num_n;
    a.num_n2 = cut.num_n2;
    a.runs = cut.runs;
    a.num_sms = num_sms;
    a.scratch = c.scratch;
    a.arrived = c.arrived;
    CUtensorMap m[4];
    auto maps = [&](const LowChangeArgs& x, const LowTerms& l, CUtensorMap* to) {
        const bool rows = x.req.n_rows > 0;   // (tc_change)
        return make_map(&to[0], rows ? l.terms : x.G, rows ? x.req.n_rows : 1, l.n_terms * l.stride, 0, BK) &&
               make_map(&to[1], rows ? x.b : x.G, rows ? x.req.n_rows : 1, x.N, 0, BK);
    };
    if (!maps(c, low, &m[0]) || !maps(c2 != nullptr ? *c2 : c, c2 != nullptr ? low2 : low, &m[2])) return cudaErrorInvalidValue;
    const long long items = (long long)c.req.n_adapters * (a.num_n + a.num_n2) * a.runs;
    const int n = items < num_sms ? (int)items : num_sms;
    return low_sets(a) > low_blocks(LOW) / 2 ? launch<LOW_WIDE>(a, cut.bn, n, num_sms, m, s) : launch<LOW>(a, cut.bn, n, num_sms, m, s);
}

}  // namespace bp
