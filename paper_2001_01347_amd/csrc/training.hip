// Training operators next to the barrier search, for MI355X (gfx950, wave64).
//
// Implements the C ABI declared in include/ebsp_training.h.  Device code, by header:
//   tr_common.h    element types, loads and stores at any alignment
//   tr_product.h   tiles of matrix products on the matrix cores
//   tr_gated_ff.h  the gated feed-forward block and its backward pass
// This file: the host side (checks, launches, the C entry points).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "ebsp_training.h"
#include "zl_host.h"
#include "tr_gated_ff.h"

namespace {

using namespace ebsp_host;

#define LAUNCH(kernel, grid, block, ...)                                                   \
    do {                                                                                   \
        hipLaunchKernelGGL(kernel, grid, block, 0, st, __VA_ARGS__);                       \
        hipError_t e_ = hipGetLastError();                                                 \
        if (e_ != hipSuccess) {                                                            \
            snprintf(g_err, sizeof g_err, "%s: %s", #kernel, hipGetErrorString(e_));       \
            return EBSP_ERR_LAUNCH;                                                        \
        }                                                                                  \
    } while (0)

// Sizes up to here keep every product of two of them, in bytes, inside 64 bits.
constexpr i64 SIZE_MAX_DIM = 1ll << 31;

int element_size(int dtype) { return dtype == EBSP_BF16 || dtype == EBSP_F16 ? 2 : dtype == EBSP_F32 ? 4 : 0; }

bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Four neighbouring elements can be stored at once.
int wide_rows(const void* p, i64 ld, int size) { return aligned(p, 4 * size) && ld % 4 == 0; }

i64 padded_units(i64 F, int size)
{
    const i64 n = 16 / size;
    return (F + n - 1) / n * n;
}

int check_sizes(i64 M, i64 K, i64 F, int dtype, int act)
{
    if (!element_size(dtype)) return fail(EBSP_ERR_ARGUMENT, "dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (act < EBSP_ACT_SILU || act > EBSP_ACT_SIGMOID) return fail(EBSP_ERR_ARGUMENT, "act must be one of EBSP_ACT_*");
    if (M < 0 || K < 0 || F < 0 || M >= SIZE_MAX_DIM || K >= SIZE_MAX_DIM || F >= SIZE_MAX_DIM)
        return fail(EBSP_ERR_SHAPE, "invalid shape: M, K and F must be 0 to 2^31 - 1");
    return EBSP_OK;
}

bool stride_ok(i64 ld, i64 length) { return ld >= length && ld < (1ll << 40); }

template <class TL, int PER_N>
int tile_grid(i64 m, i64 n, dim3& grid, int z = 1)
{
    const i64 tiles = ((m + TL::BM - 1) / TL::BM) * ((n + PER_N - 1) / PER_N);
    if (tiles > 0x7fffffffll) return fail(EBSP_ERR_SHAPE, "the result is too large for one call");
    grid = dim3((unsigned)tiles, (unsigned)z);
    return EBSP_OK;
}

template <class T>
int ff_forward(const FfForward& f, hipStream_t st)
{
    using TL = Tile<T, 2, 2, 4, 4>;
    dim3 grid;
    if (int rc = tile_grid<TL, TL::BN / 2>(f.x.index, f.w.index, grid)) return rc;
    LAUNCH((tr_ff_forward_kernel<T, TL>), grid, dim3(TL::NT), f);
    return EBSP_OK;
}

template <class T, Layout LA>
int ff_gradient(const FfGradient& f, int z, hipStream_t st)
{
    using TL = Tile<T, 2, 2, 4, 4>;
    dim3 grid;
    if (int rc = tile_grid<TL, TL::BN>(f.a.index, f.b.index, grid, z)) return rc;
    LAUNCH((tr_ff_gradient_kernel<T, TL, LA>), grid, dim3(TL::NT), f);
    return EBSP_OK;
}

template <class T>
int ff_backward(const void* dh, i64 lddh, const void* x, i64 ldx, const void* wg, i64 ldwg, const void* wu, i64 ldwu, const void* g,
                const void* u, i64 ldg, i64 M, i64 K, i64 F, int act, void* dx, i64 lddx, void* dwg, void* dwu, i64 lddw, void* workspace,
                hipStream_t st)
{
    const i64 ldd = padded_units(F, sizeof(T));
    T* dg = (T*)workspace;
    T* du = dg + M * ldd;
    const i64 chunks = M * (ldd / PER_WORD4<T>);
    if (chunks > 0) {
        const i64 blocks = (chunks + 255) / 256;
        LAUNCH(tr_ff_units_kernel<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), (const T*)dh, lddh, (const T*)g, (const T*)u,
               ldg, dg, du, ldd, M, F, act);
    }
    if (dx && M > 0 && K > 0) {
        FfGradient f = {{{dg, du}, {ldd, ldd}, M, ldd}, {{wg, wu}, {ldwg, ldwu}, K, F}, {dx, nullptr}, {lddx, 0}, {wide_rows(dx, lddx, sizeof(T)), 0}, 2};
        if (int rc = ff_gradient<T, ROWS>(f, 1, st)) return rc;
    }
    if (dwg && F > 0 && K > 0) {
        FfGradient f = {{{dg, du}, {ldd, ldd}, F, M}, {{x, x}, {ldx, ldx}, K, M}, {dwg, dwu}, {lddw, lddw},
                        {wide_rows(dwg, lddw, sizeof(T)), wide_rows(dwu, lddw, sizeof(T))}, 1};
        if (int rc = ff_gradient<T, COLS>(f, 2, st)) return rc;
    }
    return EBSP_OK;
}

}  // namespace

extern "C" {

int ebsp_gated_ff_forward(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu, int64_t M, int64_t K,
                          int64_t F, int32_t dtype, int32_t act, void* h, int64_t ldh, void* g, void* u, int64_t ldg, void* stream)
{
    if (int rc = check_sizes(M, K, F, dtype, act)) return rc;
    if (M == 0 || F == 0) return EBSP_OK;
    if (!h || (K > 0 && (!x || !wg || !wu))) return fail(EBSP_ERR_NULL, "x, wg, wu and h must not be NULL");
    if (!g != !u) return fail(EBSP_ERR_NULL, "g and u must both be given or both be NULL");
    if (!stride_ok(ldx, K) || !stride_ok(ldwg, K) || !stride_ok(ldwu, K) || !stride_ok(ldh, F) || (g && !stride_ok(ldg, F)))
        return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    const int size = element_size(dtype);
    if (!aligned(x, size) || !aligned(wg, size) || !aligned(wu, size) || !aligned(h, size) || !aligned(g, size) || !aligned(u, size))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (int rc = check_device()) return rc;
    FfForward f = {{{x, x}, {ldx, ldx}, M, K}, {{wg, wu}, {ldwg, ldwu}, F, K}, h, g, u, ldh, ldg, act,
                   wide_rows(h, ldh, size), g ? wide_rows(g, ldg, size) && wide_rows(u, ldg, size) : 0};
    hipStream_t st = (hipStream_t)stream;
    return dtype == EBSP_BF16 ? ff_forward<__bf16>(f, st) : dtype == EBSP_F16 ? ff_forward<_Float16>(f, st) : ff_forward<float>(f, st);
}

size_t ebsp_gated_ff_workspace_bytes(int64_t M, int64_t F, int32_t dtype)
{
    const int size = element_size(dtype);
    if (!size || M < 0 || F < 0 || M >= SIZE_MAX_DIM || F >= SIZE_MAX_DIM) return 0;
    return ((size_t)2 * M * padded_units(F, size) * size + 255) / 256 * 256;
}

int ebsp_gated_ff_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu,
                           int64_t ldwu, const void* g, const void* u, int64_t ldg, int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
                           void* dx, int64_t lddx, void* dwg, void* dwu, int64_t lddw, void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_sizes(M, K, F, dtype, act)) return rc;
    if (!dwg != !dwu) return fail(EBSP_ERR_NULL, "dwg and dwu must both be given or both be NULL");
    if (K == 0 || (!dx && !dwg) || (M == 0 && F == 0)) return EBSP_OK;
    const bool units = M > 0 && F > 0;                                       // otherwise the gradients are sums of nothing
    if (units && (!dh || !g || !u || !workspace)) return fail(EBSP_ERR_NULL, "dh, g, u and workspace must not be NULL");
    if (units && ((dx && (!wg || !wu)) || (dwg && !x))) return fail(EBSP_ERR_NULL, "x, wg and wu must not be NULL");
    if (units && (!stride_ok(lddh, F) || !stride_ok(ldg, F))) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if ((units && dwg && !stride_ok(ldx, K)) || (units && dx && (!stride_ok(ldwg, K) || !stride_ok(ldwu, K))) || (dx && !stride_ok(lddx, K)) ||
        (dwg && !stride_ok(lddw, K)))
        return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    const int size = element_size(dtype);
    const void* all[] = {dh, x, wg, wu, g, u, dx, dwg, dwu};
    for (const void* p : all)
        if (!aligned(p, size)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (units && (workspace_bytes < ebsp_gated_ff_workspace_bytes(M, F, dtype) || !aligned(workspace, 256)))
        return fail(EBSP_ERR_WORKSPACE, "workspace too small or not 256-byte aligned (ebsp_gated_ff_workspace_bytes)");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    auto run = dtype == EBSP_BF16 ? ff_backward<__bf16> : dtype == EBSP_F16 ? ff_backward<_Float16> : ff_backward<float>;
    return run(dh, lddh, x, ldx, wg, ldwg, wu, ldwu, g, u, ldg, M, K, F, act, dx, lddx, dwg, dwu, lddw, workspace, st);
}

}  // extern "C"
