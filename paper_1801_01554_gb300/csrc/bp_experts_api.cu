// C ABI of the router, the mix, and the expert and adapter layers (include/bp_experts.h):
// argument checks, handles and the choice of kernels.
#include <cuda_runtime.h>

#include <climits>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "bp_experts_internal.h"

using namespace bp;

struct bp_router {
    int E = 0, k = 0, dtype = BP_F32, cap = 0, gates = BP_GATES_CHOSEN;
    int* hist = nullptr;
};

struct bp_experts {
    int E = 0, n_in = 0, n_out = 0, dtype = BP_F32, cap = 0, num_sms = 0;
    int* flags = nullptr;
    void* rows = nullptr;   // bfloat16: [cap, n_in] inputs in the rows' order
    float* sums = nullptr;  // bias changes of runs of rows
    unsigned* arrived = nullptr;
    ChangeShares shares{};  // float32: changes of shares of the rows
};

struct bp_adapters {
    int n = 0, rank = 0, n_in = 0, n_out = 0, dtype = BP_F32, cap = 0, max_requests = 0, num_sms = 0;
    int* flags = nullptr;
    float* low = nullptr;   // [cap, rank] v of the backward pass
    float* scratch = nullptr;      // changes of shares of the rows
    unsigned* arrived = nullptr;
    size_t n_counts = 0;
    // bfloat16: u or v as bfloat16 terms, u's for its change, and what row blocks hold
    void* terms = nullptr;
    void* u_terms = nullptr;
    int2* tiles = nullptr;
    int n_terms = 0, stride = 0;
    LowTerms low_terms() const { return {terms, n_terms, stride, tiles}; }
};

namespace {

constexpr int kMaxUnits = 1 << 20;
constexpr int kMaxAdapters = 65535;   // a grid dimension
constexpr int kMaxRows = INT_MAX - 1023;   // kernels round up to tiles of rows and look some rows ahead

bp_status fail(bp_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error_message(buf);
    return st;
}

bp_status cuda_status(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return BP_OK;
    return fail(e == cudaErrorMemoryAllocation ? BP_ENOMEM : BP_ECUDA, "%s: %s (%s)", what, cudaGetErrorName(e),
                cudaGetErrorString(e));
}

// A buffer that a call reads or writes: present unless the call has no rows for it, and aligned.
struct Buffer {
    const void* p;
    const char* name;
    int align;
    bool needed;
};
template <int N>
bp_status check_buffers(const char* call, const Buffer (&b)[N]) {
    for (const Buffer& x : b) {
        if (x.p == nullptr && x.needed) return fail(BP_EINVAL, "%s: %s is NULL", call, x.name);
        if (((uintptr_t)x.p & (uintptr_t)(x.align - 1)) != 0)
            return fail(BP_EINVAL, "%s: %s must be %d-byte aligned", call, x.name, x.align);
    }
    return BP_OK;
}

bp_status check_dtype(const char* call, int dtype) {
    if (dtype == BP_F32 || dtype == BP_BF16) return BP_OK;
    return fail(BP_EINVAL, "%s: unknown dtype %d", call, dtype);
}

bp_status check_range(const char* call, const char* what, long long v, long long lo, long long hi) {
    if (v >= lo && v <= hi) return BP_OK;
    return fail(BP_EINVAL, "%s: %s must be in [%lld, %lld] (got %lld)", call, what, lo, hi, v);
}

bp_status check_units(const char* call, int n_in, int n_out, int dtype) {
    bp_status st = check_range(call, "n_in", n_in, 1, kMaxUnits);
    if (st == BP_OK) st = check_range(call, "n_out", n_out, 1, kMaxUnits);
    if (st == BP_OK && dtype == BP_BF16 && (n_in % 8 != 0 || n_out % 8 != 0))
        st = fail(BP_ESHAPE, "%s: bfloat16 layers need n_in and n_out to be multiples of 8 (got %d and %d)", call,
                  n_in, n_out);
    return st;
}

// A layer's error word (zero once layer_ready has returned); the device's SMs and, for bfloat16, its kernels' set-up.
bp_status make_layer(int dtype, int** flags, int* num_sms, const char* call) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(num_sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = dtype == BP_BF16 ? tc_setup() : simt_setup();
    if (e == cudaSuccess && dtype == BP_BF16) e = few_setup();
    if (e == cudaSuccess) e = cudaMalloc(flags, sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(*flags, 0, sizeof(int));
    return cuda_status(e, call);
}

bp_status make_floats(float** p, size_t n, const char* call) {
    return n == 0 ? BP_OK : cuda_status(cudaMalloc(p, n * sizeof(float)), call);
}

// Zeros that blocks count their arrivals with (there once layer_ready has returned).
bp_status make_counts(unsigned** counts, size_t n, const char* call) {
    cudaError_t e = cudaMalloc(counts, n * sizeof(unsigned));
    if (e == cudaSuccess) e = cudaMemset(*counts, 0, n * sizeof(unsigned));
    return cuda_status(e, call);
}

// The memsets of a new layer run on the legacy default stream, behind what it has queued: waited for, as the
// layer's first call may be on a stream that does not wait for that one.
bp_status layer_ready(const char* call) { return cuda_status(cudaStreamSynchronize(cudaStreamLegacy), call); }

// Waits for the stream, then reports and clears the error word, and after a wait that ran out the counts
// (n_counts of them) that its launch left behind.  All on that stream and waited for: the next call
// may be on any.
bp_status read_flags(int* flags, unsigned* counts, size_t n_counts, void* stream, const char* call) {
    cudaStream_t s = (cudaStream_t)stream;
    int f = 0;
    cudaError_t e = cudaMemcpyAsync(&f, flags, sizeof f, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && f != 0) {
        e = cudaMemsetAsync(flags, 0, sizeof f, s);
        if (e == cudaSuccess && (f & kFlagTimeout) && n_counts > 0) e = cudaMemsetAsync(counts, 0, n_counts * sizeof(unsigned), s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    }
    if (e != cudaSuccess) return cuda_status(e, call);
    if (f & kFlagTimeout)
        return fail(BP_ETIMEOUT, "a bounded device-side wait ran out; the launch stopped early");
    if (f & kFlagBounds)
        return fail(BP_ESTATE, "an offset, source row or adapter of a call was out of range");
    return BP_OK;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------ router
bp_status bp_router_create(int n_experts, int k, int dtype, int max_patterns, int gates, bp_router** out) {
    const char* call = "bp_router_create";
    set_error_message("");
    if (out == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_range(call, "n_experts", n_experts, 1, BP_MAX_EXPERTS);
    if (st == BP_OK) st = check_range(call, "k", k, 1, n_experts < BP_MAX_CHOICES ? n_experts : BP_MAX_CHOICES);
    if (st == BP_OK) st = check_dtype(call, dtype);
    if (st == BP_OK) st = check_range(call, "max_patterns", max_patterns, 1, kMaxRows / k);
    if (st == BP_OK && gates != BP_GATES_CHOSEN && gates != BP_GATES_ALL)
        st = fail(BP_EINVAL, "%s: unknown gates %d", call, gates);
    if (st != BP_OK) return st;
    bp_router* r = new (std::nothrow) bp_router();
    if (r == nullptr) return fail(BP_ENOMEM, "%s: out of memory", call);
    r->E = n_experts;
    r->k = k;
    r->dtype = dtype;
    r->cap = max_patterns;
    r->gates = gates;
    const size_t blocks = ((size_t)max_patterns + kRoutePatterns - 1) / kRoutePatterns;
    st = cuda_status(cudaMalloc(&r->hist, (blocks + 1) * n_experts * sizeof(int)), call);
    if (st != BP_OK) {
        delete r;
        return st;
    }
    *out = r;
    return BP_OK;
}

void bp_router_destroy(bp_router* r) {
    if (r == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(r->hist);
    delete r;
}

bp_status bp_route(bp_router* r, const void* d_logits, int n, int* d_expert, float* d_gate, int* d_offsets,
                   int* d_source, int* d_place, void* stream) {
    const char* call = "bp_route";
    if (r == nullptr) return fail(BP_EINVAL, "%s: NULL router", call);
    bp_status st = check_range(call, "n", n, 0, r->cap);
    const bool rows = n > 0;
    if (st == BP_OK)
        st = check_buffers(call, {{d_logits, "d_logits", r->dtype == BP_BF16 ? 2 : 4, rows},
                                  {d_expert, "d_expert", 4, rows},
                                  {d_gate, "d_gate", 4, rows},
                                  {d_offsets, "d_offsets", 4, true},
                                  {d_source, "d_source", 4, rows},
                                  {d_place, "d_place", 4, rows}});
    if (st != BP_OK) return st;
    const RouteArgs a{n, r->E, r->k, r->gates, r->dtype, d_logits, d_expert, d_gate, d_offsets, d_source, d_place, r->hist};
    return cuda_status(route_forward(a, (cudaStream_t)stream), call);
}

bp_status bp_route_backward(bp_router* r, const void* d_logits, int n, const int* d_expert, const float* d_gate,
                            const float* d_dgate, void* d_dlogits, void* stream) {
    const char* call = "bp_route_backward";
    if (r == nullptr) return fail(BP_EINVAL, "%s: NULL router", call);
    bp_status st = check_range(call, "n", n, 0, r->cap);
    const bool rows = n > 0;
    const int align = r->dtype == BP_BF16 ? 2 : 4;
    if (st == BP_OK)
        st = check_buffers(call, {{d_logits, "d_logits", align, rows},
                                  {d_expert, "d_expert", 4, rows},
                                  {d_gate, "d_gate", 4, rows},
                                  {d_dgate, "d_dgate", 4, rows},
                                  {d_dlogits, "d_dlogits", align, rows}});
    if (st != BP_OK || !rows) return st;
    const RouteArgs a{n, r->E, r->k, r->gates, r->dtype, d_logits, const_cast<int*>(d_expert),
                      const_cast<float*>(d_gate), nullptr, nullptr, nullptr, r->hist};
    return cuda_status(route_backward(a, d_dgate, d_dlogits, (cudaStream_t)stream), call);
}

// ------------------------------------------------------------ mix
static bp_status check_mix(const char* call, int n_rows, int n, int k, int n_out, int dtype) {
    bp_status st = check_dtype(call, dtype);
    if (st == BP_OK) st = check_range(call, "k", k, 1, BP_MAX_CHOICES);
    if (st == BP_OK) st = check_range(call, "n", n, 0, kMaxRows / k);
    if (st == BP_OK) st = check_range(call, "n_rows", n_rows, 0, INT_MAX);
    if (st == BP_OK) st = check_units(call, 8, n_out, dtype);
    return st;
}

bp_status bp_mix(const void* d_H, int n_rows, const int* d_place, const float* d_gate, int n, int k, int n_out,
                 int dtype, void* d_Y, void* stream) {
    const char* call = "bp_mix";
    bp_status st = check_mix(call, n_rows, n, k, n_out, dtype);
    const int align = dtype == BP_BF16 ? 16 : 4;
    if (st == BP_OK)
        st = check_buffers(call, {{d_H, "d_H", align, n > 0 && n_rows > 0},
                                  {d_place, "d_place", 4, n > 0},
                                  {d_gate, "d_gate", 4, false},
                                  {d_Y, "d_Y", align, n > 0}});
    if (st != BP_OK || n == 0) return st;
    MixArgs a{};
    a.n = n, a.k = k, a.n_rows = n_rows, a.N = n_out, a.dtype = dtype;
    a.H = d_H, a.place = d_place, a.gate = d_gate, a.Y = d_Y;
    return cuda_status(mix_forward(a, (cudaStream_t)stream), call);
}

bp_status bp_mix_backward(const void* d_D, const void* d_H, int n_rows, const int* d_place, const float* d_gate, int n,
                          int k, int n_out, int dtype, void* d_dH, float* d_dgate, void* stream) {
    const char* call = "bp_mix_backward";
    bp_status st = check_mix(call, n_rows, n, k, n_out, dtype);
    const int align = dtype == BP_BF16 ? 16 : 4;
    const bool rows = n > 0 && n_rows > 0;
    if (st == BP_OK)
        st = check_buffers(call, {{d_D, "d_D", align, n > 0},
                                  {d_H, "d_H", align, rows && d_dgate != nullptr},
                                  {d_place, "d_place", 4, n > 0},
                                  {d_gate, "d_gate", 4, false},
                                  {d_dH, "d_dH", align, rows},
                                  {d_dgate, "d_dgate", 4, false}});
    if (st != BP_OK || n == 0) return st;
    MixArgs a{};
    a.n = n, a.k = k, a.n_rows = n_rows, a.N = n_out, a.dtype = dtype;
    a.H = d_H, a.place = d_place, a.gate = d_gate, a.D = d_D, a.dH = d_dH, a.dgate = d_dgate;
    return cuda_status(mix_backward(a, (cudaStream_t)stream), call);
}

// ------------------------------------------------------------ experts
bp_status bp_experts_create(int n_experts, int n_in, int n_out, int dtype, int max_rows, bp_experts** out) {
    const char* call = "bp_experts_create";
    set_error_message("");
    if (out == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_range(call, "n_experts", n_experts, 1, BP_MAX_EXPERTS);
    if (st == BP_OK) st = check_dtype(call, dtype);
    if (st == BP_OK) st = check_units(call, n_in, n_out, dtype);
    if (st == BP_OK) st = check_range(call, "max_rows", max_rows, 1, kMaxRows);
    if (st != BP_OK) return st;
    bp_experts* l = new (std::nothrow) bp_experts();
    if (l == nullptr) return fail(BP_ENOMEM, "%s: out of memory", call);
    l->E = n_experts;
    l->n_in = n_in;
    l->n_out = n_out;
    l->dtype = dtype;
    l->cap = max_rows;
    st = make_layer(dtype, &l->flags, &l->num_sms, call);
    if (st == BP_OK && dtype == BP_BF16) st = cuda_status(cudaMalloc(&l->rows, (size_t)max_rows * n_in * 2), call);
    // fewer rows make no more runs
    const size_t planes = sums_runs(max_rows, n_experts, n_out, dtype, l->num_sms), cells = (size_t)n_experts * n_out;
    if (st == BP_OK) st = cuda_status(cudaMalloc(&l->sums, planes * cells * sizeof(float)), call);
    if (st == BP_OK) st = make_counts(&l->arrived, cells, call);
    if (st == BP_OK && dtype == BP_F32) {
        st = make_floats(&l->shares.scratch, simt_change_scratch(n_experts, n_experts, (size_t)n_in * n_out, max_rows, l->num_sms), call);
        if (st == BP_OK) st = make_counts(&l->shares.arrived, simt_change_counts(l->num_sms), call);
    }
    if (st == BP_OK) st = layer_ready(call);
    if (st != BP_OK) {
        bp_experts_destroy(l);
        return st;
    }
    *out = l;
    return BP_OK;
}

void bp_experts_destroy(bp_experts* l) {
    if (l == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(l->flags);
    cudaFree(l->rows);
    cudaFree(l->sums);
    cudaFree(l->arrived);
    cudaFree(l->shares.scratch);
    cudaFree(l->shares.arrived);
    delete l;
}

// bfloat16 inputs that are read through an index: from here on a copy in the rows' order.
static cudaError_t rows_in_order(bp_experts* l, const RowGroups& groups, const void*& X, int& n_x, const int*& source,
                                 cudaStream_t s) {
    if (source == nullptr || l->dtype != BP_BF16) return cudaSuccess;
    const cudaError_t e = tc_gather(X, source, n_x, groups, l->n_in, l->rows, l->flags, l->num_sms, s);
    X = l->rows;
    n_x = groups.n_rows;
    source = nullptr;
    return e;
}

static cudaError_t rows_product(const RowsArgs& a, int dtype, bool back, const LowTerms& low, int num_sms, cudaStream_t s) {
    return dtype == BP_BF16 ? tc_rows(a, back, low, num_sms, s) : simt_rows(a, back, num_sms, s);
}

bp_status bp_experts_forward(bp_experts* l, const void* d_W, const float* d_b, const void* d_X, int n_x,
                             const int* d_source, const int* d_offsets, int n_rows, int squash, void* d_Y,
                             void* stream) {
    const char* call = "bp_experts_forward";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    bp_status st = check_range(call, "n_rows", n_rows, 0, l->cap);
    const bool rows = n_rows > 0;
    if (st == BP_OK && rows) st = check_range(call, "n_x", n_x, d_source != nullptr ? 1 : n_rows, INT_MAX);
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    if (st == BP_OK)
        st = check_buffers(call, {{d_W, "d_W", align, rows},
                                  {d_b, "d_b", 4, false},
                                  {d_X, "d_X", align, rows},
                                  {d_source, "d_source", 4, false},
                                  {d_offsets, "d_offsets", 4, true},
                                  {d_Y, "d_Y", align, rows}});
    if (st != BP_OK || !rows) return st;
    cudaStream_t s = (cudaStream_t)stream;
    RowsArgs a{};
    a.groups = {d_offsets, l->E, n_rows};
    const bool few = l->dtype == BP_BF16 && few_experts(n_rows, l->E, l->n_out, l->n_in);
    a.N = l->n_out;
    a.K = l->n_in;
    a.in = d_X;
    a.n_in_rows = n_x;
    a.source = d_source;
    a.W = d_W;
    a.bias = d_b;
    a.squash = squash;
    a.out = d_Y;
    a.flags = l->flags;
    return cuda_status(few ? few_rows(a, s) : rows_product(a, l->dtype, false, {}, l->num_sms, s), call);
}

bp_status bp_experts_backward(bp_experts* l, const void* d_W, const void* d_X, int n_x, const int* d_source,
                              const int* d_offsets, int n_rows, const void* d_D, int squash, void* d_dX, float* d_GW,
                              float* d_Gb, int accumulate, void* stream) {
    const char* call = "bp_experts_backward";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    bp_status st = check_range(call, "n_rows", n_rows, 0, l->cap);
    const bool rows = n_rows > 0;
    if (st == BP_OK && rows) st = check_range(call, "n_x", n_x, d_source != nullptr ? 1 : n_rows, INT_MAX);
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    const bool needs_x = d_GW != nullptr || (d_dX != nullptr && squash != 0);
    if (st == BP_OK)
        st = check_buffers(call, {{d_W, "d_W", align, rows && d_dX != nullptr},
                                  {d_X, "d_X", align, rows && needs_x},
                                  {d_source, "d_source", 4, false},
                                  {d_offsets, "d_offsets", 4, true},
                                  {d_D, "d_D", align, rows},
                                  {d_dX, "d_dX", align, false},
                                  {d_GW, "d_GW", align, false},
                                  {d_Gb, "d_Gb", 4, false}});
    if (st != BP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    const RowGroups groups{d_offsets, l->E, n_rows};
    if (rows && needs_x) {
        st = cuda_status(rows_in_order(l, groups, d_X, n_x, d_source, s), call);
        if (st != BP_OK) return st;
    }
    if (d_dX != nullptr && rows) {
        RowsArgs a{};
        a.groups = groups;
        a.N = l->n_in;
        a.K = l->n_out;
        a.in = d_D;
        a.n_in_rows = n_rows;
        a.W = d_W;
        a.squash = squash;
        a.x = d_X;
        a.x_source = d_source;
        a.n_x = n_x;
        a.out = d_dX;
        a.flags = l->flags;
        st = cuda_status(rows_product(a, l->dtype, true, {}, l->num_sms, s), call);
    }
    if (st == BP_OK && d_GW != nullptr) {
        const ChangeArgs a{groups, l->n_out, l->n_in, d_D, d_X, d_source, n_x, d_GW, accumulate, l->flags};
        st = cuda_status(l->dtype == BP_BF16 ? tc_change(a, l->num_sms, s) : simt_change(a, l->shares, l->num_sms, s), call);
    }
    if (st == BP_OK && d_Gb != nullptr) {
        const SumsArgs a{groups, l->n_out, d_D, d_Gb, accumulate, l->sums, l->arrived, l->flags};
        st = cuda_status(group_sums(a, l->dtype, l->num_sms, s), call);
    }
    return st;
}

bp_status bp_experts_check(bp_experts* l, void* stream) {
    if (l == nullptr) return fail(BP_EINVAL, "bp_experts_check: NULL layer");
    return read_flags(l->flags, nullptr, 0, stream, "bp_experts_check");   // (its counting launches do not wait)
}

// ------------------------------------------------------------ adapters
bp_status bp_adapters_create(int n_adapters, int rank, int n_in, int n_out, int dtype, int max_rows, int max_requests,
                             bp_adapters** out) {
    const char* call = "bp_adapters_create";
    set_error_message("");
    if (out == nullptr) return fail(BP_EINVAL, "%s: NULL argument", call);
    bp_status st = check_range(call, "n_adapters", n_adapters, 1, kMaxAdapters);
    if (st == BP_OK) st = check_range(call, "rank", rank, 1, BP_MAX_RANK);
    if (st == BP_OK) st = check_dtype(call, dtype);
    if (st == BP_OK) st = check_units(call, n_in, n_out, dtype);
    if (st == BP_OK) st = check_range(call, "max_rows", max_rows, 1, kMaxRows / BP_MAX_RANK);
    if (st == BP_OK) st = check_range(call, "max_requests", max_requests, 1, kMaxRows);
    if (st != BP_OK) return st;
    bp_adapters* l = new (std::nothrow) bp_adapters();
    if (l == nullptr) return fail(BP_ENOMEM, "%s: out of memory", call);
    l->n = n_adapters;
    l->rank = rank;
    l->n_in = n_in;
    l->n_out = n_out;
    l->dtype = dtype;
    l->cap = max_rows;
    l->max_requests = max_requests;
    st = make_layer(dtype, &l->flags, &l->num_sms, call);
    if (st == BP_OK) st = cuda_status(cudaMalloc(&l->low, (size_t)max_rows * rank * sizeof(float)), call);
    if (st == BP_OK && dtype == BP_BF16) {
        l->stride = rank <= 32 ? 32 : rank <= 64 ? 64 : 128;
        l->n_terms = 3;   // 2^-25 of a float32 value is lost; of two terms 2^-17
        const size_t bytes = (size_t)max_rows * l->n_terms * l->stride * 2;
        st = cuda_status(cudaMalloc(&l->terms, bytes), call);
        if (st == BP_OK) st = cuda_status(cudaMalloc(&l->u_terms, bytes), call);
        if (st == BP_OK)
            st = cuda_status(cudaMalloc(&l->tiles, ((size_t)max_rows / kTileRows + 1) * sizeof(int2)), call);
    }
    if (st == BP_OK) {
        const size_t cells = (size_t)rank * (n_in > n_out ? n_in : n_out);
        st = make_floats(&l->scratch, dtype == BP_BF16 ? low_change_scratch(n_adapters, rank, n_in + n_out, max_rows, l->num_sms)
                                                       : simt_change_scratch(n_adapters, 1, cells, max_rows, l->num_sms), call);
    }
    l->n_counts = dtype == BP_BF16 ? low_change_counts(n_adapters, l->num_sms) : simt_change_counts(l->num_sms);
    if (st == BP_OK) st = make_counts(&l->arrived, l->n_counts, call);
    if (st == BP_OK) st = layer_ready(call);
    if (st != BP_OK) {
        bp_adapters_destroy(l);
        return st;
    }
    *out = l;
    return BP_OK;
}

void bp_adapters_destroy(bp_adapters* l) {
    if (l == nullptr) return;
    cudaDeviceSynchronize();
    cudaFree(l->flags);
    cudaFree(l->low);
    cudaFree(l->terms);
    cudaFree(l->u_terms);
    cudaFree(l->tiles);
    cudaFree(l->scratch);
    cudaFree(l->arrived);
    delete l;
}

static cudaError_t low_of(const bp_adapters* l, const Requests& req, int K, const void* in, const void* P, const float* scale,
                          bool forward, float* low, cudaStream_t s) {
    const bool few = forward && few_with_adapters(req.n_rows, K);
    const LowArgs a{req, K, in, P, scale, forward ? 0 : 1, low, l->terms, few ? 0 : l->n_terms, l->stride, few ? nullptr : l->tiles, l->flags};
    if (l->dtype != BP_BF16) return simt_low(a, s);
    if (few) return low_product(a, s);
    return (long long)req.n_rows >= 64ll * req.n_requests && req.n_requests > 0 ? tc_low(a, l->num_sms, s) : low_product(a, s);
}

static bp_status check_requests(const char* call, const bp_adapters* l, int n_requests, int n_rows) {
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    bp_status st = check_range(call, "n_rows", n_rows, 0, l->cap);
    if (st == BP_OK) st = check_range(call, "n_requests", n_requests, 0, l->max_requests);
    return st;
}

bp_status bp_adapters_forward(bp_adapters* l, const void* d_W, const float* d_b, const void* d_A, const void* d_B,
                              const float* d_scale, const void* d_X, const int* d_offsets, const int* d_adapter,
                              int n_requests, int n_rows, int squash, float* d_U, void* d_Y, void* stream) {
    const char* call = "bp_adapters_forward";
    bp_status st = check_requests(call, l, n_requests, n_rows);
    if (st != BP_OK) return st;
    const bool rows = n_rows > 0, some = rows && n_requests > 0;
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    st = check_buffers(call, {{d_W, "d_W", align, rows},
                              {d_b, "d_b", 4, false},
                              {d_A, "d_A", align, some},
                              {d_B, "d_B", align, some},
                              {d_scale, "d_scale", 4, false},
                              {d_X, "d_X", align, rows},
                              {d_offsets, "d_offsets", 4, some},
                              {d_adapter, "d_adapter", 4, some},
                              {d_U, "d_U", 4, rows},
                              {d_Y, "d_Y", align, rows}});
    if (st != BP_OK || !rows) return st;
    cudaStream_t s = (cudaStream_t)stream;
    const Requests req{d_offsets, d_adapter, n_requests, n_rows, l->n, l->rank};
    st = cuda_status(low_of(l, req, l->n_in, d_X, d_A, d_scale, true, d_U, s), call);
    if (st != BP_OK) return st;
    RowsArgs a{};
    a.groups = {nullptr, 1, n_rows};
    a.N = l->n_out;
    a.K = l->n_in;
    a.in = d_X;
    a.n_in_rows = n_rows;
    a.W = d_W;
    a.bias = d_b;
    a.squash = squash;
    a.out = d_Y;
    a.req = req;
    a.low = d_U;
    a.P = d_B;
    a.scale = d_scale;
    a.flags = l->flags;
    if (l->dtype == BP_BF16 && few_with_adapters(n_rows, l->n_in)) return cuda_status(few_rows(a, s), call);
    return cuda_status(rows_product(a, l->dtype, false, l->low_terms(), l->num_sms, s), call);
}

bp_status bp_adapters_backward(bp_adapters* l, const void* d_W, const void* d_A, const void* d_B, const float* d_scale,
                               const void* d_X, const float* d_U, const int* d_offsets, const int* d_adapter,
                               int n_requests, int n_rows, const void* d_D, int squash, void* d_dX, float* d_GA,
                               float* d_GB, int accumulate, void* stream) {
    const char* call = "bp_adapters_backward";
    bp_status st = check_requests(call, l, n_requests, n_rows);
    if (st != BP_OK) return st;
    const bool rows = n_rows > 0, some = rows && n_requests > 0, dx = d_dX != nullptr, ga = d_GA != nullptr,
               gb = d_GB != nullptr;
    const int align = l->dtype == BP_BF16 ? 16 : 4;
    st = check_buffers(call, {{d_W, "d_W", align, rows && dx},
                              {d_A, "d_A", align, some && dx},
                              {d_B, "d_B", align, some && (dx || ga)},
                              {d_scale, "d_scale", 4, false},
                              {d_X, "d_X", align, rows && (ga || (dx && squash != 0))},
                              {d_U, "d_U", 4, some && gb},
                              {d_offsets, "d_offsets", 4, some},
                              {d_adapter, "d_adapter", 4, some},
                              {d_D, "d_D", align, rows},
                              {d_dX, "d_dX", align, false},
                              {d_GA, "d_GA", align, false},
                              {d_GB, "d_GB", align, false}});
    if (st != BP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    const Requests req{d_offsets, d_adapter, rows ? n_requests : 0, n_rows, l->n, l->rank};
    // u's terms first: the launches after it depend on one another one by one
    if (gb && some && l->dtype == BP_BF16)
        st = cuda_status(low_terms(d_U, n_rows, l->rank, l->u_terms, l->stride, l->n_terms, l->num_sms, s), call);
    if (st == BP_OK && rows && (dx || ga)) {
        st = cuda_status(low_of(l, req, l->n_out, d_D, d_B, d_scale, false, l->low, s), call);
    }
    if (st == BP_OK && rows && dx) {
        RowsArgs a{};
        a.groups = {nullptr, 1, n_rows};
        a.N = l->n_in;
        a.K = l->n_out;
        a.in = d_D;
        a.n_in_rows = n_rows;
        a.W = d_W;
        a.squash = squash;
        a.x = d_X;
        a.n_x = n_rows;
        a.out = d_dX;
        a.req = req;
        a.low = l->low;   // v: scaled already
        a.P = d_A;
        a.flags = l->flags;
        st = cuda_status(rows_product(a, l->dtype, true, l->low_terms(), l->num_sms, s), call);
    }
    if (st != BP_OK || (!ga && !gb)) return st;
    const LowChangeArgs of_a{req, l->n_in, l->low, d_X, nullptr, d_GA, accumulate, l->scratch, l->arrived, l->flags};
    const LowChangeArgs of_b{req, l->n_out, d_U, d_D, d_scale, d_GB, accumulate, l->scratch, l->arrived, l->flags};
    if (l->dtype == BP_BF16) {
        const LowTerms v = l->low_terms();
        LowTerms u = v;
        u.terms = l->u_terms;
        return cuda_status(tc_low_change(ga ? of_a : of_b, ga ? v : u, ga && gb ? &of_b : nullptr, u, l->num_sms, s), call);
    }
    const ChangeShares room{l->scratch, l->arrived, 1};
    if (ga) st = cuda_status(simt_low_change(of_a, room, l->num_sms, s), call);
    if (st == BP_OK && gb) st = cuda_status(simt_low_change(of_b, room, l->num_sms, s), call);
    return st;
}

bp_status bp_adapters_check(bp_adapters* l, void* stream) {
    const char* call = "bp_adapters_check";
    if (l == nullptr) return fail(BP_EINVAL, "%s: NULL layer", call);
    return read_flags(l->flags, l->arrived, l->n_counts, stream, call);   // (tcgen05 launches wait)
}

}  // extern "C"
