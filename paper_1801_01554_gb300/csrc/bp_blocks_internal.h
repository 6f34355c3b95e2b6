// Internal declarations of what stands around the layers in a model of blocks (include/bp_blocks.h): what
// the API passes to the kernels' launchers.
#pragma once

#include <cuda_runtime.h>

#include "bp_blocks.h"
#include "bp_internal.h"

namespace bp {

// ------------------------------------------------------------ embedding (bp_embed.cu)
struct EmbedArgs {
    int n, n_tokens, width, dtype;
    const int* ids;
    float scale;
    const void* table;      // forward
    void* Y;
    const void* D;          // backward
    float* G;
    int accumulate;
    // ids in order: two buffers of tokens and of the ids' places, as the passes need them (embed_passes)
    unsigned* keys[2];
    int* places[2];
    float* partial;         // [2 * tiles, width] sums of pieces of long runs
    unsigned* arrived;      // a zero for every tile and slab, left zero
    int* flags;
};
constexpr int kEmbedTile = 32;   // sorted ids of a warp
size_t embed_counts(int max_ids, int width, int dtype);   // of `arrived`
cudaError_t embed_setup();
cudaError_t embed_forward(const EmbedArgs& a, cudaStream_t s);
cudaError_t embed_backward(const EmbedArgs& a, cudaStream_t s);

}  // namespace bp
