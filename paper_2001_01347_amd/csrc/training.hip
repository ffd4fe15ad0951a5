// Training operators next to the barrier search, for MI355X (gfx950, wave64).
//
// Implements the C ABI declared in include/ebsp_training.h.  Device code, by header:
//   tr_common.h    element types, loads and stores at any alignment
//   tr_cut.h       how the feed-forward block is cut up (host only)
//   tr_product.h   tiles of matrix products on the matrix cores
//   tr_gated_ff.h  the gated feed-forward block and its backward pass
//   tr_rows.h      rows of logits
//   tr_distill.h   the distillation loss and its gradient
//   tr_merge.h     the merge of the workers' pushes
// This file: the host side (checks, launches, the C entry points); tuning.hip has the rest of that header, tr_host.h what both share.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "ebsp_training.h"
#include "tr_host.h"
#include "tr_cut.h"
#include "tr_gated_ff.h"
#include "tr_distill.h"
#include "tr_merge.h"

namespace {

// Results of so many elements are refused: their bytes, several buffers of them together, stay inside 64 bits.
constexpr i64 ELEMENTS_MAX = 1ll << 56;

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
    if (M * F >= ELEMENTS_MAX) return fail(EBSP_ERR_SHAPE, "invalid shape: M x F must be below 2^56");
    return EBSP_OK;
}

template <class TL, int PER_N>
int tile_grid(i64 m, i64 n, dim3& grid, int z = 1)
{
    const i64 tiles = ((m + TL::BM - 1) / TL::BM) * ((n + PER_N - 1) / PER_N);
    if (!launchable(tiles, TL::NT)) return fail(EBSP_ERR_SHAPE, "the result is too large for one call");
    grid = dim3((unsigned)tiles, (unsigned)z);
    return EBSP_OK;
}

// Whole 16-byte chunks all along, and offsets inside a tile that fit 31 bits: what loads straight to shared memory need.  The two matrices of COLS share
// their offsets, so their strides have to be the same.
bool operand_direct(const Operand& o, Layout l, int size)
{
    const i64 n = 16 / size;
    if (l == COLS && o.ld[0] != o.ld[1]) return false;
    for (int w = 0; w < 2; ++w)
        if (o.p[w] && (!aligned(o.p[w], 16) || o.ld[w] % n || o.ld[w] * size * 256 > 0x7fffffffll)) return false;
    return (l == ROWS ? o.depth : o.index) % n == 0;
}

template <class T, class TL>
int ff_forward_tiles(const FfForward& f, hipStream_t st)
{
    const bool direct = operand_direct(f.x, ROWS, sizeof(T)) && operand_direct(f.w, ROWS, sizeof(T));
    dim3 grid;
    if (int rc = tile_grid<TL, TL::BN / 2>(f.x.index, f.w.index, grid, f.parts)) return rc;
    if (direct) LAUNCH((tr_ff_forward_kernel<T, TL, true>), grid, dim3(TL::NT), f);
    else LAUNCH((tr_ff_forward_kernel<T, TL, false>), grid, dim3(TL::NT), f);
    if (f.parts == 1) return EBSP_OK;
    const i64 blocks = (f.x.index * (partial_ld(f.w.index) / 4) + 255) / 256;
    LAUNCH(tr_ff_forward_join_kernel<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), f);
    return EBSP_OK;
}

template <class T, int FM>
int ff_few(const FfForward& f, hipStream_t st)
{
    using TF = Few<FM>;
    const i64 blocks = (f.w.index + 15) / 16, rows = (f.x.index + FM * 16 - 1) / (FM * 16);
    if (!launchable(blocks * rows, TF::NT)) return fail(EBSP_ERR_SHAPE, "the result is too large for one call");
    LAUNCH((tr_ff_few_kernel<T, TF>), dim3((unsigned)blocks, (unsigned)rows), dim3(TF::NT), f);
    return EBSP_OK;
}

size_t forward_partial_bytes(i64 M, i64 F, int parts) { return parts > 1 ? ((size_t)2 * parts * M * partial_ld(F) * sizeof(float) + 255) / 256 * 256 : 0; }

template <class T>
int ff_forward(FfForward& f, void* workspace, size_t workspace_bytes, hipStream_t st)
{
    const i64 M = f.x.index, K = f.x.depth, F = f.w.index;
    ForwardCut cut = forward_cut(M, K, F, sizeof(T), true);
    if (workspace_bytes < forward_partial_bytes(M, F, cut.parts)) cut = forward_cut(M, K, F, sizeof(T), false);
    f.partial = (float*)workspace;
    f.parts = cut.parts;
    if (cut.few) return cut.few == 1 ? ff_few<T, 1>(f, st) : cut.few == 2 ? ff_few<T, 2>(f, st) : ff_few<T, 4>(f, st);
    return cut.large ? ff_forward_tiles<T, Tile<T, 2, 4, 8, 4>>(f, st) : ff_forward_tiles<T, Tile<T, 2, 2, 4, 4>>(f, st);
}

template <class T, Layout LA>
bool gradient_direct(const FfGradient& f) { return operand_direct(f.a, LA, sizeof(T)) && operand_direct(f.b, COLS, sizeof(T)); }

template <class T, class TL, Layout LA>
int ff_gradient_tiles(const FfGradient& f, int z, bool launch, hipStream_t st)
{
    const bool direct = gradient_direct<T, LA>(f);
    dim3 grid;
    if (int rc = tile_grid<TL, TL::BN>(f.rows, f.b.index, grid, z * f.parts)) return rc;
    if (!launch) return EBSP_OK;
    if (direct) LAUNCH((tr_ff_gradient_kernel<T, TL, LA, true>), grid, dim3(TL::NT), f);
    else LAUNCH((tr_ff_gradient_kernel<T, TL, LA, false>), grid, dim3(TL::NT), f);
    return EBSP_OK;
}

template <class T, Layout LA>
int ff_gradient(const FfGradient& f, int z, bool launch, hipStream_t st)
{
    if (f.large) return ff_gradient_tiles<T, Tile<T, 2, 4, 8, 4>, LA>(f, z, launch, st);
    return ff_gradient_tiles<T, Tile<T, 2, 2, 4, 4>, LA>(f, z, launch, st);
}

size_t partial_bytes(i64 rows, i64 columns, int z, const Cut& cut)
{
    return cut.parts > 1 ? ((size_t)cut.parts * z * rows * partial_ld(columns) * sizeof(float) + 255) / 256 * 256 : 0;
}

template <class T>
int ff_join(const FfGradient& f, int z, hipStream_t st)
{
    if (f.parts == 1) return EBSP_OK;
    const i64 blocks = (f.rows * (partial_ld(f.b.index) / 4) + 255) / 256;
    LAUNCH(tr_ff_join_kernel<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384), (unsigned)z), dim3(256), f);
    return EBSP_OK;
}

// The launches of one gradient.
template <class T, Layout LA>
int ff_gradient_and_join(const FfGradient& f, int z, bool launch, hipStream_t st)
{
    if (f.rows == 0) return EBSP_OK;
    if (int rc = ff_gradient<T, LA>(f, z, launch, st)) return rc;
    return launch ? ff_join<T>(f, z, st) : EBSP_OK;
}

// Both gradients in one launch, where both have small tiles.
template <class T>
int ff_gradients(const FfGradient& x, const FfGradient& w, bool launch, hipStream_t st)
{
    using TL = Tile<T, 2, 2, 4, 4>;
    const bool direct = gradient_direct<T, ROWS>(x);
    const i64 x_tiles = tiles_of(x.rows, x.b.index, TL::BM, TL::BN), w_tiles = tiles_of(w.rows, w.b.index, TL::BM, TL::BN);
    const i64 x_all = x_tiles * x.parts, w_all = w_tiles * 2 * w.parts, all = x_all + w_all;
    const i64 w_first = w.b.depth / w.parts > 2 * x.b.depth / x.parts ? w_all : 0;       // whose sums are longer
    if (!launchable(all, TL::NT)) return fail(EBSP_ERR_SHAPE, "the result is too large for one call");
    if (!launch) return EBSP_OK;
    if (direct) LAUNCH((tr_ff_gradients_kernel<T, TL, true>), dim3((unsigned)all), dim3(TL::NT), x, w, (u32)x_tiles, (u32)x_all, (u32)w_tiles, (u32)w_first);
    else LAUNCH((tr_ff_gradients_kernel<T, TL, false>), dim3((unsigned)all), dim3(TL::NT), x, w, (u32)x_tiles, (u32)x_all, (u32)w_tiles, (u32)w_first);
    if (int rc = ff_join<T>(x, 1, st)) return rc;
    return ff_join<T>(w, 2, st);
}

template <class T>
int ff_backward(const void* dh, i64 lddh, const void* x, i64 ldx, const void* wg, i64 ldwg, const void* wu, i64 ldwu, const float* g,
                const float* u, i64 ldg, i64 M, i64 K, i64 F, int act, void* dx, i64 lddx, void* dwg, void* dwu, i64 lddw, void* workspace,
                size_t workspace_bytes, hipStream_t st)
{
    const i64 ldd = padded_units(F, sizeof(T));
    T* dg = (T*)workspace;
    T* du = dg + M * ldd;
    constexpr bool F16 = __is_same(T, _Float16);
    const size_t units = ebsp_gated_ff_workspace_bytes(M, F, sizeof(T) == 4 ? EBSP_F32 : F16 ? EBSP_F16 : EBSP_BF16);
    float* partial = (float*)((char*)workspace + units);
    float* largest = F16 && units ? (float*)((char*)workspace + units - RANGE_BYTES) : nullptr;
    float* back = largest ? largest + RANGE_BLOCKS : nullptr;
    Cut cx = dx_cut(M, K, F, sizeof(T)), cw = dw_cut(M, K, F, sizeof(T));
    const size_t px = partial_bytes(M, K, 1, cx), pw = partial_bytes(F, K, 2, cw);
    if (workspace_bytes < units + px + pw) cx.parts = cw.parts = 1;
    float* partial_w = cx.parts > 1 ? (float*)((char*)partial + px) : partial;
    const FfGradient to_x = {{{dg, du}, {ldd, ldd}, M, ldd}, {{wg, wu}, {ldwg, ldwu}, K, F}, {dx, nullptr}, {lddx, 0}, 2, M, partial, cx.parts, cx.large, back};
    const FfGradient to_w = {{{dg, du}, {ldd, ldd}, ldd, M}, {{x, x}, {ldx, ldx}, K, M}, {dwg, dwu}, {lddw, lddw}, 1, F, partial_w, cw.parts, cw.large, back};
    const bool together = dx && dwg && M > 0 && F > 0 && !cx.large && !cw.large && gradient_direct<T, ROWS>(to_x) == gradient_direct<T, COLS>(to_w);
    for (bool launch : {false, true}) {                                      // both grids are looked at before anything is enqueued
        const i64 chunks = M * (ldd / PER_WORD4<T>);
        if (launch && chunks > 0) {
            const i64 blocks = (chunks + 255) / 256, most = F16 ? RANGE_BLOCKS : 16384;
            const dim3 grid((unsigned)(blocks < most ? blocks : most));
            const FfUnits<T> form = {(const T*)dh, lddh, g, u, ldg, dg, du, ldd, M, F, act, largest, back};
            LAUNCH(tr_ff_units_kernel<T>, grid, dim3(256), form);
            if constexpr (F16) LAUNCH(tr_ff_rescale_kernel, grid, dim3(256), form, (int)grid.x);
        }
        if (together) {
            if (int rc = ff_gradients<T>(to_x, to_w, launch, st)) return rc;
            continue;
        }
        if (dx)
            if (int rc = ff_gradient_and_join<T, ROWS>(to_x, 1, launch, st)) return rc;
        if (dwg)
            if (int rc = ff_gradient_and_join<T, COLS>(to_w, 2, launch, st)) return rc;
    }
    return EBSP_OK;
}

// Parts that a row is cut into for its sums: several only where rows are few and long, since they take two launches more.  bf16, loss / loss and
// gradient, us in a graph, in one part and in as many as here: 1 x 32000 7.9 / 14.0 and (16) 7.7 / 13.4; 1 x 128000 13.5 / 25 and (31)
// 8.0 / 14.5; 64 x 128000 14.1 / 28 and (8) 11.1 / 23; 128 x 128000 14.9 / 31.5 and (4) 15.2 / 32.6.
int distill_splits(i64 N, i64 V, int size)
{
    const i64 words = (V * size + 15) / 16;
    if (N > 96 || words <= 4096) return 1;
    const i64 s = 512 / (N > 0 ? N : 1), most = words / 512;
    return (int)(s < most ? s : most);
}

// Parts for a gradient from statistics, which need no scratch: about four workgroups a CU, of no less than 512 words.
int gradient_splits(i64 N, i64 V, int size)
{
    const i64 most = (V * size + 15) / 16 / 512, s = 1024 / (N > 0 ? N : 1) < most ? 1024 / (N > 0 ? N : 1) : most;
    return (int)(s < 1 ? 1 : s);
}

size_t distill_partial_bytes(i64 N, int splits) { return splits > 1 ? ((size_t)N * splits * 3 * sizeof(float) + 255) / 256 * 256 : 0; }

template <class T>
int distill_gradient(Distill d, hipStream_t st)
{
    d.splits = gradient_splits(d.N, d.V, sizeof(T));
    LAUNCH((tr_distill_gradient_kernel<256, T>), dim3((unsigned)(d.N * d.splits)), dim3(256), d);
    return EBSP_OK;
}

template <int NT, class T, bool GRAD>
int distill_rows(const Distill& d, hipStream_t st)
{
    const dim3 rows((unsigned)d.N);
    switch (second_of(d)) {
    case ONE: LAUNCH((tr_distill_row_kernel<NT, T, GRAD, ONE>), rows, dim3(NT), d); break;
    case SQUARE: LAUNCH((tr_distill_row_kernel<NT, T, GRAD, SQUARE>), rows, dim3(NT), d); break;
    default: LAUNCH((tr_distill_row_kernel<NT, T, GRAD, APART>), rows, dim3(NT), d);
    }
    return EBSP_OK;
}

template <class T>
int distill_loss(Distill d, bool grad, hipStream_t st)
{
    if (d.splits == 1) {
        // Workgroups that hold a row, or half of one that would fill a CU's registers.  bf16, loss and gradient, us with 1024 / 512 / 256 / 128 threads:
        // 4096 x 128000 597 / 487 / 599 / -, 4096 x 64000 347 / 212 / 248 / -, 4096 x 32000 276 / 162 / 128 / -, 512 x 16000 - / 17 / 17 / 20,
        // 4096 x 8000 - / 86 / 49 / 42, 4096 x 1000 - / 74 / 37 / 21; f32, 2048 x 128000 514 / 579 / 634 / -.  The loss alone streams what it does not hold:
        // 1024 x 128000 84 / 56 / 53 / 51, 400 x 128000 36 / 25 / 26 / 41, 128 x 128000 17 / 17 / 20 / 29, 4096 x 1000 87 / 38 / 19 / 15.
        const i64 words = (d.V + PER_WORD4<T> - 1) / PER_WORD4<T>;
        if (words <= 1024) return grad ? distill_rows<128, T, true>(d, st) : distill_rows<128, T, false>(d, st);
        if (grad) return words <= 4096 ? distill_rows<256, T, true>(d, st) : words <= 16384 ? distill_rows<512, T, true>(d, st) : distill_rows<1024, T, true>(d, st);
        return words > 2048 && d.N <= 384 ? distill_rows<512, T, false>(d, st) : distill_rows<256, T, false>(d, st);
    }
    LAUNCH((tr_distill_part_kernel<256, T>), dim3((unsigned)(d.N * d.splits)), dim3(256), d);
    LAUNCH((tr_distill_join_kernel<256, T>), dim3((unsigned)d.N), dim3(256), d);
    return grad ? distill_gradient<T>(d, st) : EBSP_OK;
}

int check_distill(const Distill& d, int dtype, int index_bytes)
{
    if (!element_size(dtype) || !element_size(d.top_type)) return fail(EBSP_ERR_ARGUMENT, "dtype and top_dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (index_bytes != 4 && index_bytes != 8) return fail(EBSP_ERR_ARGUMENT, "index_bytes must be 4 or 8");
    if (d.N < 0 || d.N >= SIZE_MAX_DIM || d.V < 1 || d.V >= SIZE_MAX_DIM) return fail(EBSP_ERR_SHAPE, "invalid shape: N must be 0 and V 1 to 2^31 - 1");
    if (d.top < 0 || d.top > TOP_MAX) return fail(EBSP_ERR_SHAPE, "invalid shape: top must be 0 to EBSP_DISTILL_TOP_MAX");
    if (!(d.temperature > 0.f) || d.temperature > FLT_MAX) return fail(EBSP_ERR_ARGUMENT, "temperature must be a positive number");
    if (LOG2E / d.temperature > FLT_MAX) return fail(EBSP_ERR_ARGUMENT, "temperature is too small: its inverse is no number any more");
    if (d.N == 0) return EBSP_OK;
    if (!d.logits || (d.top > 0 && (!d.top_index || !d.top_logit))) return fail(EBSP_ERR_NULL, "logits, top_index and top_logit must not be NULL");
    if (!stride_ok(d.ld, d.V) || (d.top > 0 && !stride_ok(d.ldt, d.top))) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (!aligned(d.logits, element_size(dtype)) || !aligned(d.top_index, index_bytes) || !aligned(d.top_logit, element_size(d.top_type)) ||
        !aligned(d.labels, 8) || !aligned(d.grad, element_size(dtype)) || !aligned(d.dloss, 4) || !aligned(d.loss, 4) || !aligned(d.stats, 4) ||
        !aligned(d.status, 4))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    return EBSP_OK;
}

int check_gradient(const Distill& d)
{
    if (!d.grad || !d.dloss) return fail(EBSP_ERR_NULL, "dloss and dlogits must not be NULL");
    if (!stride_ok(d.ldd, d.V)) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (d.grad == d.logits && d.ldd != d.ld) return fail(EBSP_ERR_ARGUMENT, "a gradient in the logits' place must have their row stride");
    return EBSP_OK;
}

// Shared by the loss alone and with its gradient: the scratch, the launches.
int run_distill(Distill& d, int dtype, bool grad, void* workspace, size_t workspace_bytes, hipStream_t st)
{
    const int size = element_size(dtype);
    d.splits = distill_splits(d.N, d.V, size);
    if (!launchable((i64)d.N * d.splits, 1024)) return fail(EBSP_ERR_SHAPE, "too many rows for one call");
    const size_t need = ebsp_distill_workspace_bytes(d.N, d.V, dtype);
    if (need && !workspace) return fail(EBSP_ERR_NULL, "workspace must not be NULL for this shape");
    if (need && (workspace_bytes < need || !aligned(workspace, 256)))
        return fail(EBSP_ERR_WORKSPACE, "workspace too small or not 256-byte aligned (ebsp_distill_workspace_bytes)");
    if (int rc = check_device()) return rc;
    d.partial = (float*)workspace;
    if (grad && d.splits > 1) d.stats = (float*)((char*)workspace + distill_partial_bytes(d.N, d.splits));
    return dtype == EBSP_BF16 ? distill_loss<__bf16>(d, grad, st) : dtype == EBSP_F16 ? distill_loss<_Float16>(d, grad, st) : distill_loss<float>(d, grad, st);
}

template <class T, int SPLIT>
int merge_split(const Merge& g, hipStream_t st)
{
    const i64 per = (SPLIT == 1 ? 256 : 64) * PER_WORD4<T>;                  // (launchable: n is below 2^34 or, of 4 to a thread, no more than 2^34 - 1024)
    LAUNCH_LDS((tr_merge_kernel<T, SPLIT>), dim3((unsigned)((g.n + per - 1) / per)), dim3(SPLIT == 1 ? 256 : SPLIT * 64), g.P * sizeof(Share), g);
    return EBSP_OK;
}

// The workers are split over a workgroup's waves where the chunks alone make too few waves to keep memory busy.  The rule looks at the chunks and not at the
// workers; of the sizes here it is off at 512 x 1048593 alone, which 16 parts would do in 202.  bf16, us, with 1 / 4 / 16
// parts: 1024 x 65539 322 / 92 / 36, 256 x 200000 (391 waves) 81 / 27 / 20, 64 x 500000 (977) 25 / 14 / 17, 1024 x 524309 (1025) 508 / 200 / 217,
// 64 x 1 M (1954) 27 / 23 / 29, 512 x 1048593 (2049) 292 / 239 / 202, 64 x 2 M (3907) 43 / 43 / 55, 256 x 2 M (4096) 184 / 201 / 211, 16 x 2 M
// 16 / 17 / 33.
template <class T>
int merge(const Merge& g, hipStream_t st)
{
    const i64 waves = (g.n + 64 * PER_WORD4<T> - 1) / (64 * PER_WORD4<T>);
    if (waves < 768 && g.P >= 64) return merge_split<T, 16>(g, st);
    if (waves < 4096 && g.P >= 32) return merge_split<T, 4>(g, st);
    return merge_split<T, 1>(g, st);
}

}  // namespace

extern "C" {

int ebsp_gated_ff_forward(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu, int64_t M, int64_t K,
                          int64_t F, int32_t dtype, int32_t act, void* h, int64_t ldh, float* g, float* u, int64_t ldg,
                          void* stream)
{
    return ebsp_gated_ff_forward_split(x, ldx, wg, ldwg, wu, ldwu, M, K, F, dtype, act, h, ldh, g, u, ldg, nullptr, 0, stream);
}

size_t ebsp_gated_ff_forward_workspace_bytes(int64_t M, int64_t K, int64_t F, int32_t dtype)
{
    const int size = element_size(dtype);
    if (!size || M < 1 || K < 1 || F < 1 || M >= SIZE_MAX_DIM || K >= SIZE_MAX_DIM || F >= SIZE_MAX_DIM) return 0;
    return forward_partial_bytes(M, F, forward_cut(M, K, F, size, true).parts);
}

int ebsp_gated_ff_forward_split(const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu, int64_t ldwu, int64_t M, int64_t K,
                                int64_t F, int32_t dtype, int32_t act, void* h, int64_t ldh, float* g, float* u, int64_t ldg,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    if (int rc = check_sizes(M, K, F, dtype, act)) return rc;
    if (M == 0 || F == 0) return EBSP_OK;
    if (!h || (K > 0 && (!x || !wg || !wu))) return fail(EBSP_ERR_NULL, "x, wg, wu and h must not be NULL");
    if (!g != !u) return fail(EBSP_ERR_NULL, "g and u must both be given or both be NULL");
    if (!stride_ok(ldx, K) || !stride_ok(ldwg, K) || !stride_ok(ldwu, K) || !stride_ok(ldh, F) || (g && !stride_ok(ldg, F)))
        return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    const int size = element_size(dtype);
    if (!aligned(x, size) || !aligned(wg, size) || !aligned(wu, size) || !aligned(h, size) || !aligned(g, 4) || !aligned(u, 4))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (!workspace) workspace_bytes = 0;
    if (!aligned(workspace, 256)) return fail(EBSP_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (int rc = check_device()) return rc;
    FfForward f = {{{x, x}, {ldx, ldx}, M, K}, {{wg, wu}, {ldwg, ldwu}, F, K}, h, g, u, ldh, ldg, act, nullptr, 1};
    hipStream_t st = (hipStream_t)stream;
    auto run = dtype == EBSP_BF16 ? ff_forward<__bf16> : dtype == EBSP_F16 ? ff_forward<_Float16> : ff_forward<float>;
    return run(f, workspace, workspace_bytes, st);
}

size_t ebsp_gated_ff_split_workspace_bytes(int64_t M, int64_t K, int64_t F, int32_t dtype)
{
    const size_t units = ebsp_gated_ff_workspace_bytes(M, F, dtype);
    if (!units || K < 0 || K >= SIZE_MAX_DIM) return units;
    const int size = element_size(dtype);
    return units + partial_bytes(M, K, 1, dx_cut(M, K, F, size)) + partial_bytes(F, K, 2, dw_cut(M, K, F, size));
}

size_t ebsp_gated_ff_workspace_bytes(int64_t M, int64_t F, int32_t dtype)
{
    const int size = element_size(dtype);
    if (!size || M < 0 || F < 0 || M >= SIZE_MAX_DIM || F >= SIZE_MAX_DIM || M * F >= ELEMENTS_MAX) return 0;
    const size_t units = ((size_t)2 * M * padded_units(F, size) * size + 255) / 256 * 256;
    return units && dtype == EBSP_F16 ? units + RANGE_BYTES : units;
}

int ebsp_gated_ff_backward(const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, int64_t ldwg, const void* wu,
                           int64_t ldwu, const float* g, const float* u, int64_t ldg, int64_t M, int64_t K, int64_t F, int32_t dtype, int32_t act,
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
    const void* all[] = {dh, x, wg, wu, dx, dwg, dwu};
    for (const void* p : all)
        if (!aligned(p, size) || !aligned(g, 4) || !aligned(u, 4)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (units && (workspace_bytes < ebsp_gated_ff_workspace_bytes(M, F, dtype) || !aligned(workspace, 256)))
        return fail(EBSP_ERR_WORKSPACE, "workspace too small or not 256-byte aligned (ebsp_gated_ff_workspace_bytes)");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    auto run = dtype == EBSP_BF16 ? ff_backward<__bf16> : dtype == EBSP_F16 ? ff_backward<_Float16> : ff_backward<float>;
    return run(dh, lddh, x, ldx, wg, ldwg, wu, ldwu, g, u, ldg, M, K, F, act, dx, lddx, dwg, dwu, lddw, workspace, workspace_bytes, st);
}

size_t ebsp_distill_workspace_bytes(int64_t N, int64_t V, int32_t dtype)
{
    const int size = element_size(dtype);
    if (!size || N < 1 || N >= SIZE_MAX_DIM || V < 1 || V >= SIZE_MAX_DIM) return 0;
    const int splits = distill_splits(N, V, size);
    return splits > 1 ? distill_partial_bytes(N, splits) + ((size_t)N * 3 * sizeof(float) + 255) / 256 * 256 : 0;
}

int ebsp_distill_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const void* top_index, int32_t index_bytes,
                         const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top, const int64_t* labels, float temperature,
                         float kl_weight, float ce_weight, float* loss, float* stats, int32_t* status, void* workspace, size_t workspace_bytes,
                         void* stream)
{
    Distill d = {logits, ld, N, V, top_index, top_logit, ldt, labels, nullptr, loss, stats, status, nullptr, 0, nullptr, top, top_dtype,
                 index_bytes == 8, 1, temperature, kl_weight, ce_weight};
    if (int rc = check_distill(d, dtype, index_bytes)) return rc;
    if (N == 0) return EBSP_OK;
    if (!loss) return fail(EBSP_ERR_NULL, "loss must not be NULL");
    return run_distill(d, dtype, false, workspace, workspace_bytes, (hipStream_t)stream);
}

int ebsp_distill_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const void* top_index, int32_t index_bytes,
                          const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top, const int64_t* labels, float temperature,
                          float kl_weight, float ce_weight, const float* stats, const float* dloss, void* dlogits, int64_t ldd, void* stream)
{
    Distill d = {logits, ld, N, V, top_index, top_logit, ldt, labels, dloss, nullptr, const_cast<float*>(stats), nullptr, dlogits, ldd, nullptr,
                 top, top_dtype, index_bytes == 8, 1, temperature, kl_weight, ce_weight};
    if (int rc = check_distill(d, dtype, index_bytes)) return rc;
    if (N == 0) return EBSP_OK;
    if (!stats) return fail(EBSP_ERR_NULL, "stats must not be NULL");
    if (int rc = check_gradient(d)) return rc;
    if (!launchable(N * gradient_splits(N, V, element_size(dtype)), 256)) return fail(EBSP_ERR_SHAPE, "too many rows for one call");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    return dtype == EBSP_BF16 ? distill_gradient<__bf16>(d, st) : dtype == EBSP_F16 ? distill_gradient<_Float16>(d, st) : distill_gradient<float>(d, st);
}

int ebsp_distill_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const void* top_index, int32_t index_bytes,
                           const void* top_logit, int32_t top_dtype, int64_t ldt, int32_t top, const int64_t* labels, float temperature,
                           float kl_weight, float ce_weight, const float* dloss, float* loss, void* dlogits, int64_t ldd, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream)
{
    Distill d = {logits, ld, N, V, top_index, top_logit, ldt, labels, dloss, loss, nullptr, status, dlogits, ldd, nullptr, top, top_dtype,
                 index_bytes == 8, 1, temperature, kl_weight, ce_weight};
    if (int rc = check_distill(d, dtype, index_bytes)) return rc;
    if (N == 0) return EBSP_OK;
    if (!loss) return fail(EBSP_ERR_NULL, "loss must not be NULL");
    if (int rc = check_gradient(d)) return rc;
    return run_distill(d, dtype, true, workspace, workspace_bytes, (hipStream_t)stream);
}

int ebsp_merge_pushes(const void* pushes, int64_t stride, int32_t P, int64_t n, int32_t dtype, const int32_t* iters, const float* weights,
                      const float* velocity, float lr, float momentum, int32_t nesterov, float* weights_out, float* velocity_out, void* pull,
                      int32_t pull_dtype, void* stream)
{
    const int size = element_size(dtype);
    if (!size || (pull && !element_size(pull_dtype))) return fail(EBSP_ERR_ARGUMENT, "dtype and pull_dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (P < 1 || P > EBSP_MERGE_WORKERS_MAX) return fail(EBSP_ERR_SHAPE, "invalid shape: P must be 1 to EBSP_MERGE_WORKERS_MAX");
    if (n < 0 || n >= 1ll << 34) return fail(EBSP_ERR_SHAPE, "invalid shape: n must be 0 to 2^34 - 1");
    if (size == 4 && n > (1ll << 34) - 1024) return fail(EBSP_ERR_SHAPE, "invalid shape: n must be 0 to 2^34 - 1024 for pushes in fp32");
    if (n == 0) return EBSP_OK;
    if (!pushes || !iters || !weights || !weights_out) return fail(EBSP_ERR_NULL, "pushes, iters, weights and weights_out must not be NULL");
    if (!velocity != !velocity_out) return fail(EBSP_ERR_NULL, "velocity and velocity_out must both be given or both be NULL");
    if (P > 1 && !stride_ok(stride, n)) return fail(EBSP_ERR_ARGUMENT, "a worker's stride is shorter than its push, or 2^40 and more");
    if (!aligned(pushes, size) || !aligned(iters, 4) || !aligned(weights, 4) || !aligned(velocity, 4) || !aligned(weights_out, 4) ||
        !aligned(velocity_out, 4) || (pull && !aligned(pull, element_size(pull_dtype))))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (int rc = check_device()) return rc;
    const Merge g = {pushes, stride, n, iters, weights, velocity, weights_out, velocity_out, pull, P, pull_dtype, nesterov, lr, momentum};
    hipStream_t st = (hipStream_t)stream;
    return dtype == EBSP_BF16 ? merge<__bf16>(g, st) : dtype == EBSP_F16 ? merge<_Float16>(g, st) : merge<float>(g, st);
}

}  // extern "C"
