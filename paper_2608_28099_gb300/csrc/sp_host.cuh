// Host helpers of the entry points that need no handle: errors, and what is known of a device.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include "sp_cache.cuh"

namespace sp {

inline sp_status fail(sp_status st, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error_text(buf);
    return st;
}

inline sp_status launched(cudaError_t e, const char *what) {
    return e == cudaSuccess ? SP_OK : fail(SP_ERR_CUDA, "%s: launch failed: %s", what, cudaGetErrorString(e));
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// SMs of the current device, asked for once a device (a call's launch path).
inline int sm_count() {
    static int known[MAX_DEVICES] = {};
    int dev = 0, n = 152;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        cudaGetLastError();  // (no device: the host-only checks still answer)
        return n;
    }
    if (dev >= 0 && dev < MAX_DEVICES && known[dev]) return known[dev];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && dev >= 0 && dev < MAX_DEVICES)
        known[dev] = n;
    return n;
}

inline bool float_type(int dtype) { return dtype == SP_F32 || dtype == SP_BF16; }

}  // namespace sp
