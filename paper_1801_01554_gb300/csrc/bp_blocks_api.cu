// C ABI of the embeddings, the residual stream and the clipping of changes (include/bp_blocks.h): argument
// checks, handles and scratch.
#include <cuda_runtime.h>

#include <cmath>
#include <new>

#include "bp_api_checks.h"
#include "bp_blocks_internal.h"

using namespace bp;

struct bp_embedding {
    int device = 0, n_tokens = 0, width = 0, dtype = BP_F32, cap = 0;
    int* flags = nullptr;
    unsigned* keys = nullptr;   // [2, cap]
    int* places = nullptr;      // [2, cap]
    float* partial = nullptr;
    unsigned* arrived = nullptr;
};

namespace {

bp_status check_width(const char* call, int width, int most, int dtype) {
    bp_status st = check_dtype(call, dtype);
    if (st == BP_OK) st = check_range(call, "width", width, 1, most);
    if (st == BP_OK && dtype == BP_BF16 && width % 8 != 0)
        st = fail(BP_ESHAPE, "%s: a bfloat16 width must be a multiple of 8 (got %d)", call, width);
    return st;
}

bp_status check_finite(const char* call, const char* what, float x) {
    if (std::isfinite(x)) return BP_OK;
    return fail(BP_EINVAL, "%s: %s must be finite", call, what);
}

template <class T>
bp_status make_array(T** p, size_t n, const char* call) {
    return n == 0 ? BP_OK : cuda_status(cudaMalloc(p, n * sizeof(T)), call);
}

bp_status make_flags(int* device, int** flags, const char* call) {
    cudaError_t e = cudaGetDevice(device);
    if (e == cudaSuccess) e = cudaMalloc(flags, sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(*flags, 0, sizeof(int));
    return cuda_status(e, call);
}

}  // namespace

extern "C" {

// ------------------------------------------------------------ embedding
bp_status bp_embedding_create(int n_tokens, int width, int dtype, int max_ids, bp_embedding** out) {
    const char* call = "bp_embedding_create";
    set_error_message("");
    if (out == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_range(call, "n_tokens", n_tokens, 1, BP_MAX_TOKENS);
    if (st == BP_OK) st = check_width(call, width, kMaxUnits, dtype);
    if (st == BP_OK) st = check_range(call, "max_ids", max_ids, 1, BP_MAX_IDS);
    if (st != BP_OK) return st;
    bp_embedding* l = new (std::nothrow) bp_embedding();
    if (l == nullptr) return fail(BP_ENOMEM, "%s: out of memory", call);
    l->n_tokens = n_tokens;
    l->width = width;
    l->dtype = dtype;
    l->cap = max_ids;
    const size_t tiles = ((size_t)max_ids + kEmbedTile - 1) / kEmbedTile;
    st = make_flags(&l->device, &l->flags, call);
    if (st == BP_OK) st = cuda_status(embed_setup(), call);
    if (st == BP_OK) st = make_array(&l->keys, 2 * (size_t)max_ids, call);
    if (st == BP_OK) st = make_array(&l->places, 2 * (size_t)max_ids, call);
    if (st == BP_OK) st = make_array(&l->partial, 2 * tiles * width, call);
    if (st == BP_OK) st = make_counts(&l->arrived, embed_counts(max_ids, width, dtype), call);
    if (st == BP_OK) st = layer_ready(call);
    if (st != BP_OK) {
        bp_embedding_destroy(l);
        return st;
    }
    *out = l;
    return BP_OK;
}

void bp_embedding_destroy(bp_embedding* l) {
    if (l == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(l->flags);
    cudaFree(l->keys);
    cudaFree(l->places);
    cudaFree(l->partial);
    cudaFree(l->arrived);
    delete l;
}

static bp_status check_embed(const char* call, const bp_embedding* l, int n, float scale) {
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    bp_status st = check_range(call, "n", n, 0, l->cap);
    if (st == BP_OK) st = check_finite(call, "scale", scale);
    return st;
}

static EmbedArgs embed_args(const bp_embedding* l, const int* ids, int n, float scale) {
    EmbedArgs a{};
    a.n = n, a.n_tokens = l->n_tokens, a.width = l->width, a.dtype = l->dtype, a.ids = ids, a.scale = scale;
    a.keys[0] = l->keys, a.keys[1] = l->keys + l->cap;
    a.places[0] = l->places, a.places[1] = l->places + l->cap;
    a.partial = l->partial, a.arrived = l->arrived, a.flags = l->flags;
    return a;
}

bp_status bp_embed(bp_embedding* l, const void* d_table, const int* d_ids, int n, float scale, void* d_Y, void* stream) {
    const char* call = "bp_embed";
    bp_status st = check_embed(call, l, n, scale);
    if (st != BP_OK) return st;
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    st = check_buffers(call, {{d_table, "d_table", align, n > 0}, {d_ids, "d_ids", 4, n > 0}, {d_Y, "d_Y", align, n > 0}});
    if (st == BP_OK) st = check_device(call, l->device);
    if (st != BP_OK || n == 0) return st;
    EmbedArgs a = embed_args(l, d_ids, n, scale);
    a.table = d_table, a.Y = d_Y;
    return cuda_status(embed_forward(a, (cudaStream_t)stream), call);
}

bp_status bp_embed_backward(bp_embedding* l, const int* d_ids, int n, const void* d_D, float scale, float* d_G, int accumulate,
                            void* stream) {
    const char* call = "bp_embed_backward";
    bp_status st = check_embed(call, l, n, scale);
    if (st != BP_OK) return st;
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    st = check_buffers(call, {{d_ids, "d_ids", 4, n > 0}, {d_D, "d_D", align, n > 0}, {d_G, "d_G", align, true}});
    if (st == BP_OK) st = check_device(call, l->device);
    if (st != BP_OK || (n == 0 && accumulate)) return st;
    EmbedArgs a = embed_args(l, d_ids, n, scale);
    a.D = d_D, a.G = d_G, a.accumulate = accumulate != 0;
    return cuda_status(embed_backward(a, (cudaStream_t)stream), call);
}

bp_status bp_embedding_check(bp_embedding* l, void* stream) {
    const char* call = "bp_embedding_check";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    const bp_status st = check_device(call, l->device);
    return st != BP_OK ? st : read_flags(l->flags, nullptr, 0, stream, call, "an id of a call was out of range");
}

}  // extern "C"
