// The context of the C ABI and what its entry points share: the current device,
// errors, timing, and the checks of buffers.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <string>
#include <vector>

#include "autoloco.h"
#include "reduce.hpp"

namespace autoloco {

constexpr int kMaxBlocks = 16384;   // scratch sized for this many workgroups

// Partial sums of a small call in host memory, per context (host_adds).
constexpr int kHostPartials = 1024;

}  // namespace autoloco

struct autoloco_ctx {
    int device = 0;
    hipStream_t stream = nullptr;
    int num_cus = 0;
    int grid_limit = 0;
    int occupancy[2][AUTOLOCO_MAX_K + 1] = {};  // resident workgroups per CU, by replica type and k
    int occupancy_bf16p[2][AUTOLOCO_MAX_K + 1] = {};  // the BF16-payload round
    double* partials = nullptr;
    double* sums = nullptr;
    double* host_sums = nullptr;
    double* host_sums_dev = nullptr;  // device view of host_sums (coherent host memory), or null
    // partial sums of small calls that the host adds up itself: after the kMaxSums
    // final sums in the same allocation (null where host_sums_dev is)
    double* host_partials = nullptr;
    double* host_partials_dev = nullptr;
    bool timing = false;
    bool timed_valid = false;
    hipEvent_t ev_start = nullptr, ev_stop = nullptr, ev_mid = nullptr;
    bool adamw_timed = false;     // the last timed call was an AdamW step
    bool adamw_norm_ran = false;  // ... and it ran the norm pass (ev_start..ev_mid)
    std::string err;
};

namespace autoloco {

// Makes the context's device current for the duration of a call.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev != dev) ok = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

inline int fail(autoloco_ctx* ctx, int code, const std::string& msg) {
    if (ctx) ctx->err = msg;
    return code;
}

inline int hip_fail(autoloco_ctx* ctx, hipError_t e, const char* what) {
    return fail(ctx, AUTOLOCO_E_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

// The kernels dereference every buffer on the context's device: host memory
// and memory of another device are rejected before anything is launched.
inline int check_device_ptr(autoloco_ctx* ctx, uintptr_t p, const char* name) {
    hipPointerAttribute_t at;
    std::memset(&at, 0, sizeof(at));
    if (hipPointerGetAttributes(&at, reinterpret_cast<const void*>(p)) != hipSuccess) {
        (void)hipGetLastError();
        return fail(ctx, AUTOLOCO_E_INVALID, std::string(name) + " is not device memory");
    }
    if (at.type == hipMemoryTypeManaged || at.isManaged) return AUTOLOCO_OK;
    if (at.type != hipMemoryTypeDevice) return fail(ctx, AUTOLOCO_E_INVALID, std::string(name) + " is not device memory");
    if (at.device != ctx->device)
        return fail(ctx, AUTOLOCO_E_INVALID, std::string(name) + " is on device " + std::to_string(at.device) +
                                                 ", the context's is " + std::to_string(ctx->device));
    return AUTOLOCO_OK;
}

struct Range {
    uintptr_t lo, hi;
    const char* name;
};

// Largest element count a call accepts: far beyond any device's memory, small
// enough that no byte count or address computed from it overflows.
constexpr int64_t kMaxN = int64_t(1) << 56;
inline const char* const kBadN = "n outside 0..2^56";

// Timing of a call's device work.  The previous timing is dropped before the
// start event of a new launch is recorded, so a call that fails after that
// point leaves no timing (E_STATE) rather than a start and stop of two calls.
inline int timer_start(autoloco_ctx* c) {
    c->timed_valid = false;
    if (!c->timing) return AUTOLOCO_OK;
    const hipError_t e = hipEventRecord(c->ev_start, c->stream);
    if (e != hipSuccess) return hip_fail(c, e, "hipEventRecord");
    return AUTOLOCO_OK;
}

inline int timer_stop(autoloco_ctx* c, bool adamw = false, bool norm_ran = false) {
    if (!c->timing) return AUTOLOCO_OK;
    const hipError_t e = hipEventRecord(c->ev_stop, c->stream);
    if (e != hipSuccess) return hip_fail(c, e, "hipEventRecord");
    c->timed_valid = true;
    c->adamw_timed = adamw;
    c->adamw_norm_ran = norm_ran;
    return AUTOLOCO_OK;
}

// Brings the count sums of the last reduction to host_sums and waits for them:
// with a device view of host_sums the reduction kernel already wrote them there
// (coherent host memory, visible once the stream has finished), else a copy.
inline int sums_to_host(autoloco_ctx* c, size_t count) {
    hipError_t e;
    if (c->host_sums_dev == nullptr &&
        (e = hipMemcpyAsync(c->host_sums, c->sums, sizeof(double) * count, hipMemcpyDeviceToHost, c->stream)) !=
            hipSuccess)
        return hip_fail(c, e, "hipMemcpyAsync");
    if ((e = hipStreamSynchronize(c->stream)) != hipSuccess) return hip_fail(c, e, "hipStreamSynchronize");
    return AUTOLOCO_OK;
}

inline double adamw_clip(double norm_sq, double max_norm) {
    if (max_norm == 0.0) return 1.0;
    const double c = max_norm / (std::sqrt(norm_sq) + 1e-6);
    return c > 1.0 ? 1.0 : c;
}

inline void finish_adamw(const double* sums, int k, double max_norm, autoloco_adamw_stats* out) {
    std::memset(out, 0, sizeof(*out));
    out->k = k;
    bool fin = true;
    for (int i = 0; i < k; ++i) {
        out->grad_norm[i] = std::sqrt(sums[i]);
        out->clip_coef[i] = adamw_clip(sums[i], max_norm);
        fin = fin && std::isfinite(out->grad_norm[i]);
    }
    out->finite = fin ? 1 : 0;
}


// Checks alignment and pairwise overlap of a list of ranges.
inline int check_ranges(autoloco_ctx* ctx, const std::vector<Range>& r) {
    for (const Range& x : r) {
        if (x.lo == 0) return fail(ctx, AUTOLOCO_E_INVALID, std::string("null ") + x.name);
        if (x.lo % 16 != 0) return fail(ctx, AUTOLOCO_E_ALIGN, std::string(x.name) + " not 16-byte aligned");
    }
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = i + 1; j < r.size(); ++j)
            if (r[i].lo < r[j].hi && r[j].lo < r[i].hi)
                return fail(ctx, AUTOLOCO_E_ALIAS, std::string(r[i].name) + " overlaps " + r[j].name);
    for (const Range& x : r) {
        const int st = check_device_ptr(ctx, x.lo, x.name);
        if (st != AUTOLOCO_OK) return st;
    }
    return AUTOLOCO_OK;
}

}  // namespace autoloco
