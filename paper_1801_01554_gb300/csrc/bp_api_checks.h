// What the C entry points of bp_experts.h and bp_blocks.h share: messages, checks of arguments, and
// the error word of a handle.
#pragma once

#include <cuda_runtime.h>

#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "bp_internal.h"

namespace bp {
namespace {

constexpr int kMaxUnits = 1 << 20;
constexpr int kMaxRows = INT_MAX - 1023;   // kernels round up to tiles of rows and look some rows ahead

inline bp_status fail(bp_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error_message(buf);
    return st;
}

inline bp_status cuda_status(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return BP_OK;
    cudaGetLastError();   // reported here: the check of a later launch must not find it again
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
inline bp_status check_buffers(const char* call, const Buffer (&b)[N]) {
    for (const Buffer& x : b) {
        if (x.p == nullptr && x.needed) return fail(BP_EINVAL, "%s: %s is NULL", call, x.name);
        if (((uintptr_t)x.p & (uintptr_t)(x.align - 1)) != 0)
            return fail(BP_EINVAL, "%s: %s must be %d-byte aligned", call, x.name, x.align);
    }
    return BP_OK;
}

inline bp_status check_dtype(const char* call, int dtype) {
    if (dtype == BP_F32 || dtype == BP_BF16) return BP_OK;
    return fail(BP_EINVAL, "%s: unknown dtype %d", call, dtype);
}

inline bp_status check_range(const char* call, const char* what, long long v, long long lo, long long hi) {
    if (v >= lo && v <= hi) return BP_OK;
    return fail(BP_EINVAL, "%s: %s must be in [%lld, %lld] (got %lld)", call, what, lo, hi, v);
}

// A handle's scratch is the device's that was current when it was made.
inline bp_status check_device(const char* call, int device) {
    int now = 0;
    const cudaError_t e = cudaGetDevice(&now);
    if (e != cudaSuccess) return cuda_status(e, call);
    if (now == device) return BP_OK;
    return fail(BP_EINVAL, "%s: the handle belongs to device %d (current: %d)", call, device, now);
}

// Zeros that blocks count their arrivals with (there once layer_ready has returned).
inline bp_status make_counts(unsigned** counts, size_t n, const char* call) {
    cudaError_t e = cudaMalloc(counts, n * sizeof(unsigned));
    if (e == cudaSuccess) e = cudaMemset(*counts, 0, n * sizeof(unsigned));
    return cuda_status(e, call);
}

// The memsets of a new layer run on the legacy default stream, behind what it has queued: waited for, as the
// layer's first call may be on a stream that does not wait for that one.
inline bp_status layer_ready(const char* call) { return cuda_status(cudaStreamSynchronize(cudaStreamLegacy), call); }

// Waits for the stream, then reports and clears the error word, and after a wait that ran out the counts
// (n_counts of them) that its launch left behind.  All on that stream and waited for: the next call
// may be on any.
inline bp_status read_flags(int* flags, unsigned* counts, size_t n_counts, void* stream, const char* call,
                            const char* bounds = "an offset, source row or adapter of a call was out of range") {
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
    if (f & kFlagNonfinite)
        return fail(BP_ENONFINITE, "the norm of a call's values was not finite");
    if (f & kFlagBounds)
        return fail(BP_ESTATE, "%s", bounds);
    return BP_OK;
}

}  // namespace
}  // namespace bp
