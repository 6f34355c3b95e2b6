// Internal declarations of what stands around the layers in a model of blocks (include/bp_blocks.h): what
// the API passes to the kernels' launchers.
#pragma once

#include <cuda_runtime.h>

#include "bp_blocks.h"
#include "bp_internal.h"

namespace bp {

// ------------------------------------------------------------ embedding (bp_embed.cu)
using IdPlace = unsigned long long;   // a token (above) and the place of its id
struct EmbedArgs {
    int n, n_tokens, width, dtype;
    const int* ids;
    float scale;
    const void* table;      // forward
    void* Y;
    const void* D;          // backward
    float* G;
    int accumulate;
    IdPlace* ids_in_order[2];   // [n] each; a pass of the sort reads one and writes the other
    int sort_ctas;
    float* partial;         // [2 * tiles, width] sums of pieces of long runs
    unsigned* arrived;      // a zero for every tile and slab, left zero
    int* flags;
};
constexpr int kEmbedTile = 32;   // sorted ids of a warp
size_t embed_counts(int max_ids, int width, int dtype);   // of `arrived`
cudaError_t embed_setup(int* sort_ctas);
cudaError_t embed_forward(const EmbedArgs& a, cudaStream_t s);
cudaError_t embed_backward(const EmbedArgs& a, cudaStream_t s);

// ------------------------------------------------------------ residual stream (bp_residual.cu)
struct ResidualArgs {
    int n, width, dtype, norm_out, norm_in, num_sms;
    float eps, scale, each;   // each: 1 / width
    const void *X, *F;
    const float *wo, *bo, *gate, *wi, *bi;
    const int* offsets;     // of the gates' rows, or NULL
    int n_gates;
    void *Y, *H;            // forward: written; backward: Y read
    float* stats;
    const void *dY, *dH;    // backward
    void *dX, *dF;
    float *Gwo, *Gbo, *Ggate, *Gwi, *Gbi;
    int accumulate;
    // Sums by column.  A, B: of dy f^ and dy, a row for a block's rows [blocks, width]; gates by range: [workers + gates,
    // width], a row for the rows that a worker w and a range g share, at w + g (pairs of rows in order never share
    // that number), and W, WB [workers, width]: the same times scale * gate, over the worker's rows.  C, D
    // [blocks, width]: of dH y^ and dH.
    float *A, *B, *W, *WB, *C, *D;
    double *A_run, *B_run, *W_run, *WB_run, *C_run, *D_run;   // [workers, width] each: sums of a worker's rows but for the last run of them
    int worker_warps, workers, workers_a_block;   // (set by the launchers)
    int* flags;
};
int residual_workers(int num_sms, int width, int dtype);   // of a backward call, at most
cudaError_t residual_setup(int width, int dtype);
cudaError_t residual_forward(ResidualArgs a, cudaStream_t s);
cudaError_t residual_backward(ResidualArgs a, cudaStream_t s);

// ------------------------------------------------------------ clipping (bp_clip.cu)
struct ClipChunk {
    const void* in;
    void* out;
    unsigned count;
    int dtype;
};
constexpr int kClipFew = 16;
struct ClipFew {
    ClipChunk chunks[kClipFew];   // where there are no more: they go with the launch
};
struct ClipArgs {
    const ClipChunk* chunks;   // of the tensors, in order
    int n_chunks, in_place;    // in_place: every output is its input
    int few;                   // (clip_setup)
    int write;                 // 0: the norm alone
    float max_norm;
    float* norm;               // or NULL
    double* partial;           // [clip_blocks], and one for their sum
    double* total;
    unsigned* arrived;         // a zero, left zero
    int* flags;
};
constexpr int kClipTile = 8192;   // values that a block takes at a time
int clip_blocks(int num_sms);
cudaError_t clip_setup(int n_chunks, bool tiles, int* few);   // tiles: no chunk has more than a tile, and less than 16 bytes before it
cudaError_t clip_run(const ClipArgs& a, const ClipFew& few, int num_sms, cudaStream_t s);

}  // namespace bp
