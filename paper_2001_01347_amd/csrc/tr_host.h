// Host side that the training operators' sources share: launches, checks of sizes, strides and alignment.
// Part of the ZipLine library (see training.hip, tuning.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "ebsp_training.h"
#include "zl_host.h"
#include "tr_common.h"

#define LAUNCH(kernel, grid, block, ...) LAUNCH_LDS(kernel, grid, block, 0, __VA_ARGS__)
#define LAUNCH_LDS(kernel, grid, block, lds, ...)                                          \
    do {                                                                                   \
        hipLaunchKernelGGL(kernel, grid, block, lds, st, __VA_ARGS__);                       \
        hipError_t e_ = hipGetLastError();                                                 \
        if (e_ != hipSuccess) {                                                            \
            snprintf(g_err, sizeof g_err, "%s: %s", #kernel, hipGetErrorString(e_));       \
            return EBSP_ERR_LAUNCH;                                                        \
        }                                                                                  \
    } while (0)

namespace {

using namespace ebsp_host;

// Sizes up to here keep every product of two of them, in elements, inside 64 bits.
constexpr i64 SIZE_MAX_DIM = 1ll << 31;

inline int element_size(int dtype) { return dtype == EBSP_BF16 || dtype == EBSP_F16 ? 2 : dtype == EBSP_F32 ? 4 : 0; }

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

inline bool stride_ok(i64 ld, i64 length) { return ld >= length && ld < (1ll << 40); }

// A launch of so many workgroups: the runtime counts a grid's threads in 32 bits.
inline bool launchable(i64 blocks, int threads) { return blocks * threads <= 0xffffffffll; }

}  // namespace
