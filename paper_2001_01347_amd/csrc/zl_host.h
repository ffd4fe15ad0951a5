// Host side that every source of the library shares: the calling thread's last error, the device check.
// Part of the ZipLine library (see zipline.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <atomic>
#include <stdio.h>
#include <string.h>

#include "ebsp_zipline.h"

namespace ebsp_host {

// hidden: one copy in the library, none outside it
__attribute__((visibility("hidden"))) inline thread_local char g_err[256] = "";

inline int fail(int code, const char* msg)
{
    snprintf(g_err, sizeof g_err, "%s", msg);
    return code;
}

// The kernels are built for gfx950 only: refuse any other device by name instead of
// letting a launch fail.  Asked once per device; the answer is kept.
__attribute__((visibility("hidden"))) inline int check_device()
{
    constexpr int KNOWN = 64;
    static std::atomic<signed char> seen[KNOWN];       // 0: not asked yet, 1: gfx950, -1: something else
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return fail(EBSP_ERR_DEVICE, "no current HIP device");
    signed char state = dev >= 0 && dev < KNOWN ? seen[dev].load(std::memory_order_relaxed) : 0;
    if (state == 0) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return fail(EBSP_ERR_DEVICE, "hipGetDeviceProperties failed");
        state = strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? 1 : -1;
        if (dev >= 0 && dev < KNOWN) seen[dev].store(state, std::memory_order_relaxed);
    }
    if (state < 0) return fail(EBSP_ERR_DEVICE, "the current device is not a gfx950 (MI355X): this library has code for nothing else");
    return EBSP_OK;
}

}  // namespace ebsp_host
