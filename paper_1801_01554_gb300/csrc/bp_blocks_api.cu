// C ABI of the embeddings, the residual stream and the clipping of changes (include/bp_blocks.h): argument
// checks, handles and scratch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "bp_api_checks.h"
#include "bp_blocks_internal.h"

using namespace bp;

struct bp_embedding {
    int device = 0, n_tokens = 0, width = 0, dtype = BP_F32, cap = 0;
    int* flags = nullptr;
    IdPlace* in_order = nullptr;   // [2, cap]
    int sort_ctas = 1;
    float* partial = nullptr;
    unsigned* arrived = nullptr;
};

struct bp_residual {
    ResidualArgs a{};
    int cap = 0, max_gates = 0, device = 0;
    float* sums = nullptr;
};

struct bp_clip {
    ClipArgs a{};
    int device = 0, num_sms = 1;
    ClipChunk* chunks = nullptr;
    ClipFew few{};
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
    if (st == BP_OK) st = cuda_status(embed_setup(&l->sort_ctas), call);
    if (st == BP_OK) st = make_array(&l->in_order, 2 * (size_t)max_ids, call);
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
    cudaFree(l->in_order);
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
    a.ids_in_order[0] = l->in_order, a.ids_in_order[1] = l->in_order + l->cap;
    a.sort_ctas = l->sort_ctas;
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

// ------------------------------------------------------------ residual stream
bp_status bp_residual_create(int width, int dtype, int max_rows, int max_gates, int norm_out, int norm_in, float eps,
                             bp_residual** out) {
    const char* call = "bp_residual_create";
    set_error_message("");
    if (out == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_width(call, width, BP_MAX_WIDTH, dtype);
    if (st == BP_OK) st = check_range(call, "max_rows", max_rows, 1, kMaxRows);
    if (st == BP_OK) st = check_range(call, "max_gates", max_gates, 0, kMaxRows);
    if (st == BP_OK) st = check_range(call, "norm_out", norm_out, BP_NORM_NONE, BP_NORM_LAYER);
    if (st == BP_OK) st = check_range(call, "norm_in", norm_in, BP_NORM_NONE, BP_NORM_LAYER);
    if (st == BP_OK && !(std::isfinite(eps) && eps > 0.f)) st = fail(BP_EINVAL, "%s: eps must be finite and above 0", call);
    if (st != BP_OK) return st;
    bp_residual* l = new (std::nothrow) bp_residual();
    if (l == nullptr) return fail(BP_ENOMEM, "%s: out of memory", call);
    l->cap = max_rows;
    l->max_gates = max_gates;
    l->a.width = width, l->a.dtype = dtype, l->a.norm_out = norm_out, l->a.norm_in = norm_in, l->a.eps = eps, l->a.each = 1.f / (float)width;
    st = make_flags(&l->device, &l->a.flags, call);
    if (st == BP_OK) st = cuda_status(cudaDeviceGetAttribute(&l->a.num_sms, cudaDevAttrMultiProcessorCount, l->device), call);
    if (st == BP_OK) st = cuda_status(residual_setup(width, dtype), call);
    if (st == BP_OK) {
        const size_t w = width, workers = residual_workers(l->a.num_sms, width, dtype) * w;
        const size_t records = workers + max_gates * w;
        const bool layer = norm_out == BP_NORM_LAYER || norm_in == BP_NORM_LAYER;
        st = make_array(&l->sums, (layer ? 2 : 1) * (records + 8 * workers), call);
        float* p = l->sums;
        const auto take = [&](size_t n) { return p += n, p - n; };
        const auto take64 = [&] { return reinterpret_cast<double*>(take(2 * workers)); };   // (first: 8-byte boundaries)
        if (st == BP_OK) {
            l->a.A_run = take64(), l->a.W_run = take64(), l->a.C_run = take64();
            if (layer) l->a.B_run = take64(), l->a.WB_run = take64(), l->a.D_run = take64();
            l->a.A = take(records), l->a.W = take(workers), l->a.C = take(workers);
            if (layer) l->a.B = take(records), l->a.WB = take(workers), l->a.D = take(workers);
        }
    }
    if (st == BP_OK) st = layer_ready(call);
    if (st != BP_OK) {
        bp_residual_destroy(l);
        return st;
    }
    *out = l;
    return BP_OK;
}

void bp_residual_destroy(bp_residual* l) {
    if (l == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(l->a.flags);
    cudaFree(l->sums);
    delete l;
}

// What both directions check: rows, gates, and operands that the handle's norms do not have.
static bp_status check_residual(const char* call, const bp_residual* l, int n, const void* F, const float* wo, const float* bo,
                                const float* gate, const int* offsets, int n_gates, float scale, const float* wi, const float* bi) {
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL stream_layer", call);
    bp_status st = check_range(call, "n", n, 0, l->cap);
    if (st == BP_OK) st = check_range(call, "n_gates", n_gates, 0, l->max_gates);
    if (st == BP_OK) st = check_finite(call, "scale", scale);
    if (st != BP_OK) return st;
    if ((gate != nullptr) != (n_gates > 0)) return fail(BP_EINVAL, "%s: d_gate and n_gates do not agree", call);
    if (offsets == nullptr && n_gates > 1) return fail(BP_EINVAL, "%s: d_offsets is NULL for %d rows of gates", call, n_gates);
    if (offsets != nullptr && n_gates == 0) return fail(BP_EINVAL, "%s: d_offsets without gates", call);
    const int out = l->a.norm_out, in = l->a.norm_in;
    if ((wo != nullptr && out == BP_NORM_NONE) || (bo != nullptr && out != BP_NORM_LAYER))
        return fail(BP_EINVAL, "%s: the norm of a block's output has no such weight or bias", call);
    if ((wi != nullptr && in == BP_NORM_NONE) || (bi != nullptr && in != BP_NORM_LAYER))
        return fail(BP_EINVAL, "%s: the norm before a block has no such weight or bias", call);
    return check_buffers(call, {{F, "d_F", l->a.dtype == BP_BF16 ? 16 : 4, false}, {wo, "d_wo", 4, false}, {bo, "d_bo", 4, false},
                                {gate, "d_gate", 4, false}, {offsets, "d_offsets", 4, false}, {wi, "d_wi", 4, false},
                                {bi, "d_bi", 4, false}});
}

static ResidualArgs residual_args(const bp_residual* l, int n, const void* F, const float* wo, const float* bo, const float* gate,
                                  const int* offsets, int n_gates, float scale, const float* wi) {
    ResidualArgs a = l->a;
    a.n = n, a.F = F, a.scale = scale, a.wi = wi;
    if (F != nullptr) a.wo = wo, a.bo = bo, a.gate = gate, a.offsets = offsets, a.n_gates = n_gates;
    return a;
}

bp_status bp_residual_forward(bp_residual* l, const void* d_X, const void* d_F, int n, const float* d_wo, const float* d_bo,
                              const float* d_gate, const int* d_offsets, int n_gates, float scale, const float* d_wi,
                              const float* d_bi, void* d_Y, void* d_H, float* d_stats, void* stream) {
    const char* call = "bp_residual_forward";
    bp_status st = check_residual(call, l, n, d_F, d_wo, d_bo, d_gate, d_offsets, n_gates, scale, d_wi, d_bi);
    if (st != BP_OK) return st;
    const int align = l->a.dtype == BP_BF16 ? 16 : 4;
    st = check_buffers(call, {{d_X, "d_X", align, n > 0}, {d_Y, "d_Y", align, n > 0 && d_F != nullptr}, {d_H, "d_H", align, false},
                              {d_stats, "d_stats", 4, false}});
    if (st == BP_OK && d_H != nullptr && l->a.norm_in == BP_NORM_NONE)
        st = fail(BP_EINVAL, "%s: d_H without a norm before the next block", call);
    if (st == BP_OK) st = check_device(call, l->device);
    if (st != BP_OK || n == 0) return st;
    ResidualArgs a = residual_args(l, n, d_F, d_wo, d_bo, d_gate, d_offsets, n_gates, scale, d_wi);
    a.X = d_X, a.bi = d_bi, a.Y = d_Y, a.H = d_H, a.stats = d_stats;
    return cuda_status(residual_forward(a, (cudaStream_t)stream), call);
}

bp_status bp_residual_backward(bp_residual* l, const void* d_Y, const void* d_F, int n, const float* d_wo, const float* d_bo,
                               const float* d_gate, const int* d_offsets, int n_gates, float scale, const float* d_wi,
                               const float* d_stats, const void* d_dY, const void* d_dH, void* d_dX, void* d_dF, float* d_Gwo,
                               float* d_Gbo, float* d_Ggate, float* d_Gwi, float* d_Gbi, int accumulate, void* stream) {
    const char* call = "bp_residual_backward";
    bp_status st = check_residual(call, l, n, d_F, d_wo, d_bo, d_gate, d_offsets, n_gates, scale, d_wi, nullptr);
    if (st != BP_OK) return st;
    const int align = l->a.dtype == BP_BF16 ? 16 : 4, out = l->a.norm_out, in = l->a.norm_in;
    const bool rows = n > 0;
    st = check_buffers(call, {{d_Y, "d_Y", align, rows && d_dH != nullptr}, {d_stats, "d_stats", 4, rows}, {d_dY, "d_dY", align, false},
                              {d_dH, "d_dH", align, false}, {d_dX, "d_dX", align, false}, {d_dF, "d_dF", align, false},
                              {d_Gwo, "d_Gwo", 4, false}, {d_Gbo, "d_Gbo", 4, false}, {d_Ggate, "d_Ggate", 4, false},
                              {d_Gwi, "d_Gwi", 4, false}, {d_Gbi, "d_Gbi", 4, false}});
    if (st != BP_OK) return st;
    if (d_dH != nullptr && in == BP_NORM_NONE) return fail(BP_EINVAL, "%s: d_dH without a norm before the next block", call);
    if (rows && d_F == nullptr && (d_dF != nullptr || d_Gwo != nullptr || d_Gbo != nullptr || d_Ggate != nullptr))
        return fail(BP_EINVAL, "%s: gradients of a block's output without d_F", call);
    if ((d_Gwo != nullptr && out == BP_NORM_NONE) || (d_Gbo != nullptr && out != BP_NORM_LAYER) ||
        (d_Gwi != nullptr && in == BP_NORM_NONE) || (d_Gbi != nullptr && in != BP_NORM_LAYER))
        return fail(BP_EINVAL, "%s: a gradient of a weight or bias that the norms do not have", call);
    if (d_Ggate != nullptr && n_gates == 0) return fail(BP_EINVAL, "%s: d_Ggate without gates", call);
    st = check_device(call, l->device);
    if (st != BP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    if (!rows) {   // sums of no rows
        const size_t row = (size_t)l->a.width * sizeof(float);
        float* const sums[] = {d_Gwo, d_Gbo, d_Gwi, d_Gbi, d_Ggate};
        for (int i = 0; i < 5 && st == BP_OK && !accumulate; ++i)
            if (sums[i] != nullptr) st = cuda_status(cudaMemsetAsync(sums[i], 0, i < 4 ? row : row * n_gates, s), call);
        return st;
    }
    ResidualArgs a = residual_args(l, n, d_F, d_wo, d_bo, d_gate, d_offsets, n_gates, scale, d_wi);
    a.Y = const_cast<void*>(d_Y), a.stats = const_cast<float*>(d_stats), a.dY = d_dY, a.dH = d_dH, a.dX = d_dX, a.dF = d_dF;
    a.Gwo = d_Gwo, a.Gbo = d_Gbo, a.Ggate = d_Ggate, a.Gwi = d_Gwi, a.Gbi = d_Gbi, a.accumulate = accumulate != 0;
    return cuda_status(residual_backward(a, s), call);
}

bp_status bp_residual_check(bp_residual* l, void* stream) {
    const char* call = "bp_residual_check";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL stream_layer", call);
    const bp_status st = check_device(call, l->device);
    return st != BP_OK ? st : read_flags(l->a.flags, nullptr, 0, stream, call, "the gates' offsets of a call do not go up from 0 to its rows");
}

// ------------------------------------------------------------ clipping
namespace {

struct Span {
    uintptr_t first, end;
    int tensor;
};

// Outputs are apart from one another, and from every input but their own, which they may be.
bp_status check_spans(const char* call, const std::vector<Span>& in, std::vector<Span>& out) {
    std::sort(out.begin(), out.end(), [](const Span& a, const Span& b) { return a.first < b.first; });
    for (size_t i = 1; i < out.size(); ++i)
        if (out[i].first < out[i - 1].end)
            return fail(BP_EINVAL, "%s: the outputs of tensors %d and %d overlap", call, out[i - 1].tensor, out[i].tensor);
    for (const Span& s : in) {
        auto o = std::lower_bound(out.begin(), out.end(), s.first, [](const Span& a, uintptr_t x) { return a.end <= x; });
        for (; o != out.end() && o->first < s.end; ++o)
            if (o->tensor != s.tensor || o->first != s.first)
                return fail(BP_EINVAL, "%s: the input of tensor %d overlaps the output of tensor %d", call, s.tensor, o->tensor);
    }
    return BP_OK;
}

}  // namespace

bp_status bp_clip_create(const void* const* h_in, void* const* h_out, const int64_t* h_sizes, const int* h_dtypes, int n,
                         bp_clip** out) {
    const char* call = "bp_clip_create";
    set_error_message("");
    if (out == nullptr || h_in == nullptr || h_sizes == nullptr || h_dtypes == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_range(call, "n", n, 1, BP_MAX_TENSORS);
    if (st != BP_OK) return st;
    constexpr long long kMost = 1ll << 40;
    long long total = 0;
    bool in_place = true;
    for (int i = 0; i < n; ++i) {
        st = check_dtype(call, h_dtypes[i]);
        if (st == BP_OK) st = check_range(call, "a tensor's size", h_sizes[i], 0, kMost);
        if (st == BP_OK) st = check_range(call, "the sizes' sum", total += h_sizes[i], 0, kMost);
        if (st != BP_OK) return st;
        const void* to = h_out != nullptr ? h_out[i] : h_in[i];
        const int align = h_dtypes[i] == BP_BF16 ? 2 : 4;
        const bool some = h_sizes[i] > 0;
        st = check_buffers(call, {{h_in[i], "a tensor's input", align, some}, {to, "a tensor's output", align, some}});
        if (st != BP_OK) return st;
        in_place = in_place && (to == h_in[i] || !some);
    }
    bp_clip* l = nullptr;
    try {
        std::vector<Span> in, to;
        std::vector<ClipChunk> chunks;
        // chunks of whole tiles, from a 16-byte boundary on where a tensor goes on; some 2^16 and one a tensor at most
        const long long chunk = (total / 65536 / kClipTile + 1) * kClipTile;
        for (int i = 0; i < n; ++i) {
            const long long size = h_dtypes[i] == BP_BF16 ? 2 : 4;
            if (h_sizes[i] == 0) continue;
            const char* x = (const char*)h_in[i];
            char* y = h_out != nullptr ? (char*)h_out[i] : const_cast<char*>(x);
            const uintptr_t bytes = (uintptr_t)(h_sizes[i] * size);
            in.push_back({(uintptr_t)x, (uintptr_t)x + bytes, i});
            to.push_back({(uintptr_t)y, (uintptr_t)y + bytes, i});
            const long long head = (long long)((16 - ((uintptr_t)x & 15)) & 15) / size;
            for (long long at = 0; at < h_sizes[i];) {
                const long long count = std::min(h_sizes[i] - at, at == 0 ? head + chunk : chunk);
                chunks.push_back({x + at * size, y + at * size, (unsigned)count, h_dtypes[i]});
                at += count;
            }
        }
        st = check_spans(call, in, to);
        if (st != BP_OK) return st;
        l = new bp_clip();
        l->a.n_chunks = (int)chunks.size();
        l->a.in_place = in_place;
        st = make_flags(&l->device, &l->a.flags, call);
        if (st == BP_OK) st = cuda_status(cudaDeviceGetAttribute(&l->num_sms, cudaDevAttrMultiProcessorCount, l->device), call);
        if (st == BP_OK) st = cuda_status(clip_setup(l->a.n_chunks, chunk == kClipTile, &l->a.few), call);
        if (st == BP_OK) st = make_array(&l->chunks, chunks.size(), call);
        if (st == BP_OK) st = make_array(&l->a.partial, (size_t)clip_blocks(l->num_sms) + 1, call);
        if (st == BP_OK) l->a.total = l->a.partial + clip_blocks(l->num_sms);
        if (st == BP_OK) st = make_counts(&l->a.arrived, 1, call);
        if (st == BP_OK && !chunks.empty())
            st = cuda_status(cudaMemcpy(l->chunks, chunks.data(), chunks.size() * sizeof(ClipChunk), cudaMemcpyHostToDevice), call);
        if (st == BP_OK) st = layer_ready(call);
        l->a.chunks = l->chunks;
        for (size_t i = 0; i < chunks.size() && i < kClipFew; ++i) l->few.chunks[i] = chunks[i];
    } catch (const std::bad_alloc&) {
        st = fail(BP_ENOMEM, "%s: out of memory", call);
    }
    if (st != BP_OK) {
        bp_clip_destroy(l);
        return st;
    }
    *out = l;
    return BP_OK;
}

void bp_clip_destroy(bp_clip* l) {
    if (l == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(l->a.flags);
    cudaFree(l->chunks);
    cudaFree(l->a.partial);
    cudaFree(l->a.arrived);
    delete l;
}

bp_status bp_clip_run(bp_clip* l, float max_norm, float* d_norm, void* stream) {
    const char* call = "bp_clip_run";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL clip", call);
    if (!(max_norm >= 0.f)) return fail(BP_EINVAL, "%s: max_norm must be at least 0", call);
    bp_status st = check_buffers(call, {{d_norm, "d_norm", 4, false}});
    if (st == BP_OK) st = check_device(call, l->device);
    if (st != BP_OK) return st;
    ClipArgs a = l->a;
    a.max_norm = max_norm, a.norm = d_norm, a.write = std::isfinite(max_norm);
    return cuda_status(clip_run(a, l->few, l->num_sms, (cudaStream_t)stream), call);
}

bp_status bp_clip_check(bp_clip* l, void* stream) {
    const char* call = "bp_clip_check";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL clip", call);
    const bp_status st = check_device(call, l->device);
    return st != BP_OK ? st : read_flags(l->a.flags, nullptr, 0, stream, call);
}

}  // extern "C"
