// Internal declarations of the layers whose weights depend on the pattern
// (include/bp_experts.h): what the API passes to the kernels' launchers.
#pragma once

#include <cuda_runtime.h>

#include "bp_experts.h"
#include "bp_internal.h"

namespace bp {

// Rows in groups: group g's rows are [offsets[g], offsets[g + 1]), offsets on the device.
// offsets NULL: one group of all n_rows rows.
struct RowGroups {
    const int* offsets;
    int n_groups;
    int n_rows;
};

// Requests over the rows of a layer with adapters; adapter[i] in [0, n_adapters) or -1.
struct Requests {
    const int* offsets;
    const int* adapter;
    int n_requests, n_rows, n_adapters, rank;
};

// Rows times the weights of their group.  K-major ("forward"): out[r, n] = sum over k of
// in[src(r), k] W_g[n, k], W [groups, N, K]; the other way ("back"): out[r, n] = sum over k of
// in[r, k] W_g[k, n], W [groups, K, N].  With low != NULL there is one group and
// scale_a * sum over j of low[r, j] P_a[j, n] is added, a the adapter of the row's request.
struct RowsArgs {
    RowGroups groups;
    int N, K;
    const void* in;
    int n_in_rows;          // rows of `in`
    const int* source;      // forward: row of `in` for each row, or NULL
    const void* W;
    const float* bias;      // forward: [groups, N] or NULL
    int squash;             // forward: logistic; back: times x (1 - x)
    const void* x;          // back with squash: the layer's inputs [n_x, N], read through x_source
    const int* x_source;
    int n_x;
    void* out;
    // the adapters' part
    Requests req;
    const float* low;       // [n_rows, rank]
    const void* P;          // [n_adapters, rank, N]
    const float* scale;     // [n_adapters] or NULL
    int* flags;
};

// low[r, j] = scale_a * sum over k of in[r, k] P_a[j, k], a the adapter of the row's request
// (0 without one); P [n_adapters, rank, K].
struct LowArgs {
    Requests req;
    int K;
    const void* in;
    const void* P;
    const float* scale;     // or NULL
    int scaled_low;         // 0: low without the scale
    float* low;
    // bfloat16: the scaled sums as n_terms bfloat16 terms, [n_rows, n_terms, terms_stride] with zeros
    // past the rank, and what every block of kTileRows rows holds (0 and NULL: not
    // wanted)
    void* terms;
    int n_terms, terms_stride;
    int2* tiles;
    int* flags;
};

// Changes of weights: G_g[m, n] (+)= sum over the group's rows of a[r, m] b[src(r), n].
struct ChangeArgs {
    RowGroups groups;
    int M, N;
    const void* a;
    const void* b;
    const int* source;
    int n_b;                // rows of b
    float* G;
    int accumulate;
    int* flags;
};

// Changes of adapters: G_a[j, n] (+)= scale_a * sum over the rows of the adapter's requests of
// low[r, j] b[r, n].
struct LowChangeArgs {
    Requests req;
    int N;
    const float* low;
    const void* b;
    const float* scale;     // or NULL
    float* G;
    int accumulate;
    // bfloat16: sums of shares of the rows, and zeros that count their arrivals (low_change_scratch)
    float* scratch;
    unsigned* arrived;
    int* flags;
};

// Column sums of a group's rows: S_g[n] (+)= sum over the group's rows of d[r, n].  scratch: a plane of
// [groups, N] for each run of rows (sums_runs); arrived: a zero for every block of columns of a group,
// left zero.
struct SumsArgs {
    RowGroups groups;
    int N;
    const void* d;
    float* S;
    int accumulate;
    float* scratch;
    unsigned* arrived;
    int* flags;
};
constexpr int kMaxSumRuns = 16;
int sums_runs(int n_rows, int n_groups, int N, int dtype, int num_sms);
cudaError_t group_sums(const SumsArgs& a, int dtype, int num_sms, cudaStream_t s);   // bp_sums.cu

// float32 FMA kernels (bp_grouped_simt.cu).
cudaError_t simt_setup();
cudaError_t simt_rows(const RowsArgs& a, bool back, int num_sms, cudaStream_t s);
cudaError_t simt_low(const LowArgs& a, cudaStream_t s);
// Rows shared out between blocks: the shares' sums [shares, groups, M, N], and zeros that count their
// arrivals (left zero).
struct ChangeShares {
    float* scratch;
    unsigned* arrived;
    int shares;             // (set by the launchers)
};
// Floats of scratch for changes of `cells` values in each of `groups` groups, at least `least_busy` with rows.
size_t simt_change_scratch(int groups, int least_busy, size_t cells, int max_rows, int num_sms);
size_t simt_change_counts(int num_sms);
cudaError_t simt_change(const ChangeArgs& a, const ChangeShares& room, int num_sms, cudaStream_t s);
cudaError_t simt_low_change(const LowChangeArgs& a, const ChangeShares& room, int num_sms, cudaStream_t s);

// Tensor-core kernels for bfloat16 (bp_grouped_tc.cu).
// The adapters' low-rank sums come as bfloat16 terms (LowArgs).  A block of kTileRows rows is of one
// adapter (x: which), of none (-1), or of several requests, y being the first: whose sums are taken
// apart (kTileMixed), or whose rows are (kTileByRow, where they are more than half the rank: a request's
// sums are 0.85 us of a tile, a rank of a tile by rows 0.2 to 0.8, by its width).
constexpr int kTileRows = 128;
constexpr int kTileMixed = -2, kTileByRow = -3;
constexpr int kForwardTerms = 2;   // of the terms, those that a bfloat16 result can tell: 2^-17
struct LowTerms {
    const void* terms;
    int n_terms, stride;
    int2* tiles;
};
cudaError_t tc_setup();
// Rows read through an index into the groups' order; tc_change and the back product take rows in order.
cudaError_t tc_gather(const void* in, const int* source, int n_src, const RowGroups& groups, int cols, void* out, int* flags,
                      int num_sms, cudaStream_t s);
cudaError_t tc_rows(const RowsArgs& a, bool back, const LowTerms& low, int num_sms, cudaStream_t s);
cudaError_t tc_change(const ChangeArgs& a, int num_sms, cudaStream_t s);
cudaError_t tc_low(const LowArgs& a, int num_sms, cudaStream_t s);
size_t low_change_scratch(int n_adapters, int rank, int columns, int max_rows, int num_sms);   // floats
size_t low_change_counts(int n_adapters, int num_sms);
// One launch of one change, or of two of the same requests (second NULL: one).
cudaError_t tc_low_change(const LowChangeArgs& a, const LowTerms& low, const LowChangeArgs* second, const LowTerms& second_low,
                          int num_sms, cudaStream_t s);

// The forward product of a few rows in bfloat16 (bp_few.cu), rows read through an index too; with low,
// behind low_product, which a dependent launch overlaps.
// Which calls it is for, by rows, groups and weights (its sums are no longer than one chain takes).
bool few_experts(int n_rows, int n_groups, int N, int K);
bool few_with_adapters(int n_rows, int K);
cudaError_t few_setup();
cudaError_t few_rows(const RowsArgs& a, cudaStream_t s);

// Low-rank products of bfloat16 (bp_low.cu).
cudaError_t low_product(const LowArgs& a, cudaStream_t s);
cudaError_t low_terms(const float* low, int n_rows, int rank, void* terms, int stride, int n_terms, int num_sms,
                      cudaStream_t s);

// Router and mix (bp_route.cu).
struct RouteArgs {
    int n, E, k, gates, dtype;
    const void* logits;
    int* expert;
    float* gate;
    int* offsets;
    int* source;
    int* place;
    int* hist;              // [E, blocks of kRoutePatterns + 1]
};
constexpr int kRoutePatterns = 32;   // patterns of a block
cudaError_t route_forward(const RouteArgs& a, cudaStream_t s);
cudaError_t route_backward(const RouteArgs& a, const float* dgate, void* dlogits, cudaStream_t s);
struct MixArgs {
    int n, k, n_rows, N, dtype;
    const void* H;
    const int* place;
    const float* gate;
    void* Y;
    const void* D;
    void* dH;
    float* dgate;
    int warps;              // of a pattern (set by the launcher)
};
cudaError_t mix_forward(const MixArgs& a, cudaStream_t s);
cudaError_t mix_backward(const MixArgs& a, cudaStream_t s);

}  // namespace bp
