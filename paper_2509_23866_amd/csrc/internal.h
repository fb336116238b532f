// libdart internal helpers shared by its sources; not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "dart.h"

#pragma GCC visibility push(hidden)

// Makes dev the current device for the caller's scope and restores the
// previous one after.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = prev == dev || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        if (ok) (void)hipSetDevice(prev);
    }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
};

// The device a stream belongs to (the current device for the null stream);
// -1 on a HIP error.
inline int stream_device(hipStream_t stream) {
    int dev = -1;
    if ((stream ? hipStreamGetDevice(stream, &dev) : hipGetDevice(&dev)) != hipSuccess) return -1;
    return dev;
}

// Whether a 1-D launch of blocks workgroups of threads work-items each fits
// the dispatch (at most 2^32 - 1 work-items in the grid).
inline bool grid_fits(int64_t blocks, int64_t threads) {
    return blocks >= 0 && threads > 0 && blocks <= 0xFFFFFFFFll / threads;
}

// DART_OK when work on the stream may wait for the host (the stream is not
// being captured into a graph), DART_ERR_UNSUPPORTED when it is being captured,
// DART_ERR_HIP when HIP cannot tell.
inline dart_status_t may_synchronize(hipStream_t stream) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &cs) != hipSuccess) return DART_ERR_HIP;
    return cs == hipStreamCaptureStatusNone ? DART_OK : DART_ERR_UNSUPPORTED;
}

// The optional validation of device-side preconditions (DART_CHECK=1 in the
// environment).
namespace dart_check {

// One device array to validate.
//   Ids:     n int32 values, each in [0, bound)
//   Offsets: n + 1 int32 values, 0 = v[0] < v[1] < ... < v[n] = bound
//   Mask:    n uint8 values, each 0 or 1
//   Labels:  n int32 values, each below bound
struct Item {
    enum Kind { Ids, Offsets, Mask, Labels } kind;
    const void* ptr;
    int64_t n;
    int64_t bound;
};

// True when DART_CHECK=1 is set (read on every call, so it can be switched at
// run time).
__attribute__((visibility("hidden"))) bool enabled();

// With checks enabled: runs the validation kernels for every item on stream,
// waits for them and returns DART_ERR_INVALID_ARG if any precondition fails
// (DART_ERR_HIP on a HIP error). With checks disabled: DART_OK, nothing runs.
__attribute__((visibility("hidden"))) dart_status_t run(hipStream_t stream,
                                                        std::initializer_list<Item> items);

}  // namespace dart_check

// What the LM head's gradient calls share (lmhead.hip).
namespace lmhead {

// A gradient output: row-major, fp32 or bf16.
struct Grad {
    void* p;
    int64_t ld;
    bool bf16;
    void* row(int64_t r) const {
        return static_cast<char*>(p) + r * ld * (bf16 ? 2 : 4);
    }
};

// One block's dh[rows, d] (+)= dz[rows, cols] W[cols, d] and
// dW[cols, d] (+)= dz[rows, cols]^T h[rows, d], in one launch. A bf16 output
// is never added to (sums over blocks go through fp32). With ksplit > 1 dh_out is
// ksplit fp32 matrices part_stride elements apart, which each get their part of
// the sum. With dh_map row i of dh goes to row dh_map[i] of dh_out. With dyn_rows,
// the block's rows are at most *dyn_rows - dyn_base (read on the device).
// A null dh_out.p or dw_out.p leaves that product out; scale (device memory, may be
// null) is a factor of both. small: in tiles of 128 x 128 in place of 256 x 256 (not with dh_acc).
__attribute__((visibility("hidden"))) dart_status_t launch_bwd_gemms(
    const uint16_t* dz, int64_t ld_dz, int64_t rows, int64_t cols, const uint16_t* w, int64_t ld_w,
    const uint16_t* h, int64_t ld_h, int64_t d, const Grad& dh_out, bool dh_acc, int64_t ksplit,
    int64_t part_stride, const Grad& dw_out, bool dw_acc, hipStream_t stream, const int32_t* dh_map,
    const int32_t* dyn_rows, int64_t dyn_base, const float* scale, bool small);

// dst [rows, cols] in bf16 from fp32 rows of cols elements.
__attribute__((visibility("hidden"))) void launch_to_bf16(const float* src, int64_t rows,
                                                          int64_t cols, const Grad& dst,
                                                          hipStream_t stream);

}  // namespace lmhead

#pragma GCC visibility pop
