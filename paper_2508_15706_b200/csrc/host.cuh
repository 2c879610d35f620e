// Host-side helpers shared by the translation units of libsparseloco.
#pragma once
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "sparseloco.h"

// text of the last CUDA error seen by this thread (sl_last_cuda_error); defined in sparseloco.cu
extern thread_local char sl_cuda_err[256] __attribute__((visibility("hidden")));

namespace {

sl_status cuda_fail(cudaError_t e, const char* what) {
    snprintf(sl_cuda_err, sizeof(sl_cuda_err), "%s: %s", what, cudaGetErrorString(e));
    return SL_ERR_CUDA;
}
#define SL_CUDA(call)                                      \
    do {                                                   \
        cudaError_t e_ = (call);                           \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call); \
    } while (0)

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

sl_status sm_count(int* n) {
    int dev = 0;
    SL_CUDA(cudaGetDevice(&dev));
    SL_CUDA(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
    return SL_OK;
}

inline bool known_dtype(int t) { return t == SL_F32 || t == SL_BF16; }
inline int dtype_bytes(int t) { return t == SL_F32 ? 4 : 2; }
inline bool finite_at_least(double x, double low) { return isfinite(x) && x >= low; }

struct DeviceGuard {
    int prev;
    bool ok;
    explicit DeviceGuard(int dev) : prev(-1), ok(false) {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

}  // namespace
