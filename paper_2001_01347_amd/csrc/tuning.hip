// Operators of tuning a model on answers, next to those of training.hip, for MI355X (gfx950, wave64).
//
// Implements the rest of the C ABI declared in include/ebsp_training.h.  Device code, by header:
//   tr_common.h    element types, loads and stores at any alignment
//   tr_random.h    the counter-based generator behind dropout
//   tr_norm.h      the residual stream around a block, and dropout
//   tr_rows.h      rows of logits
//   tr_tokens.h    the losses of tokens: log-probabilities, policy and preference loss
// This file: the host side (checks, launches, the C entry points).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <type_traits>

#include "ebsp_training.h"
#include "tr_host.h"
#include "tr_norm.h"
#include "tr_tokens.h"

namespace {

constexpr i64 WIDTH_MAX = 1ll << 30;             // a row's elements are counted in 31 bits
constexpr int HELD_UNITS = 2048;                 // units of eight elements of the widest row that a workgroup holds

// What the last-level cache (256 MB) keeps between two kernels at best.
constexpr i64 LAST_CACHE = 200ll << 20;

bool finite(float x) { return x - x == 0.f; }

int check_random(float p, uint64_t seed, uint64_t offset, const int64_t* rng, Random& r)
{
    if (!(p >= 0.f) || p > 1.f) return fail(EBSP_ERR_ARGUMENT, "p must be 0 to 1");
    if (!aligned(rng, 8)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    r.threshold = (u32)nearbyint((double)p * 65536.);
    r.kept = r.threshold < 65536 ? 65536.f / (float)(65536 - r.threshold) : 0.f;
    r.seed = seed;
    r.offset = offset;
    r.place = rng;
    return EBSP_OK;
}

// The checks that both passes share.
int check_norm(const Norm& a, i64 K, int stream, int dtype)
{
    if (!element_size(dtype)) return fail(EBSP_ERR_ARGUMENT, "dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (stream != dtype && stream != EBSP_F32) return fail(EBSP_ERR_ARGUMENT, "stream_dtype must be dtype or EBSP_F32");
    if (a.M < 0 || a.M >= SIZE_MAX_DIM || K < 0 || K >= WIDTH_MAX) return fail(EBSP_ERR_SHAPE, "invalid shape: M must be 0 to 2^31 - 1 and K 0 to 2^30 - 1");
    if (!finite(a.scale)) return fail(EBSP_ERR_ARGUMENT, "scale must be a finite number");
    return EBSP_OK;
}

int check_norm_operands(const Norm& a, int stream, int dtype)
{
    const i64 K = a.K;
    if (!a.branch && (a.post_weight || a.gate || a.random.threshold))
        return fail(EBSP_ERR_ARGUMENT, "post_weight, gate and dropout need a branch");
    if (!a.weight) return fail(EBSP_ERR_NULL, "weight must not be NULL");
    if ((a.branch && !stride_ok(a.ldb, K)) || (a.gate && a.ldgate != 0 && !stride_ok(a.ldgate, K)))
        return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    const int s = element_size(stream), t = element_size(dtype);
    if (!aligned(a.x, s) || !aligned(a.y, s) || !aligned(a.dy, s) || !aligned(a.dx, s) || !aligned(a.branch, t) || !aligned(a.weight, t) ||
        !aligned(a.post_weight, t) || !aligned(a.gate, t) || !aligned(a.n, t) || !aligned(a.dn, t) || !aligned(a.dbranch, t) || !aligned(a.dgate, t) ||
        !aligned(a.stats, 4))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    return EBSP_OK;
}

// Threads a row and units a thread, by the row's units; TWO: with two units a thread.
template <bool TWO, class F>
int with_group(int units, F&& f)
{
#define GROUP(threads, each) f(std::integral_constant<int, threads>(), std::integral_constant<int, each>())
    if (units <= 8) return GROUP(8, 1);
    if (units <= 16) return GROUP(16, 1);
    if (units <= 32) return GROUP(32, 1);
    if (units <= 64) return GROUP(64, 1);
    if constexpr (TWO) {
        if (units <= 128) return GROUP(64, 2);
        if (units <= 256) return GROUP(128, 2);
        if (units <= 512) return GROUP(256, 2);
        if (units <= 1024) return GROUP(512, 2);
    } else {
        if (units <= 128) return GROUP(128, 1);
        if (units <= 256) return GROUP(256, 1);
        if (units <= 512) return GROUP(512, 1);
        if (units <= 1024) return GROUP(1024, 1);
    }
    return GROUP(1024, 2);
#undef GROUP
}

int group_threads(int units)
{
    const int sizes[] = {8, 16, 32, 64, 128, 256, 512};
    for (int g : sizes)
        if (units <= g) return g;
    return 1024;
}

// How a backward pass is launched.  Every workgroup leaves a row of columns' sums behind, so one a CU takes all rows where there are enough of them.  us of both kernels in a row, on operands that the
// last-level cache does not hold, from y / from x where both are: a 16-bit stream of 64 threads a row and more has 1024 threads with the next row under way (8192 x 4096 86 / 87; 512 threads
// two a CU 89 / 89), of fewer 512, two a CU (100000 x 200 62 / 62, 262144 x 64 52 / 52; with the next row under way 67 / 82 and 54 / 59: from x its registers do not hold that).  With a stream in
// fp32 there are none for it either: 512 threads, two a CU (fp32 4096 x 4096 104, bf16 beside it 8192 x 4096 123; 1024 threads and the next row 187 and 193).  Rows above 8192 have two units a
// thread, which are read again (2048 x 16384 171 / 165, 3000 x 10000 181 / 176, 8192 x 12288 460 / 460, fp32 1024 x 16384 173; held 174 / 178, 197 / 195, 503 / 513 and 235).
// Few rows: as many workgroups as there are CUs before anything else, but long rows, whose columns' sums are long too, two to a workgroup from 128 of them on (operands that the cache
// holds: 512 x 4096 19.8 us, so 16.5; 300 x 12000 50 and 42; four to a workgroup 18.5 and 50).
struct NormCut {
    int threads, blocks;
};

constexpr bool takes_next(bool narrow, int g) { return narrow && g >= WAVE; }

NormCut norm_cut(i64 M, i64 K, bool narrow)
{
    const int units = (int)((K + 7) / 8), g = group_threads(units), big = g == 1024 || takes_next(narrow, g) ? 1024 : 512;
    NormCut c = {M >= 1024 / g * 1024 ? big : g < 256 ? 256 : g, 0};
    const int rows = c.threads / g > 0 ? c.threads / g : 1, most = c.threads == 1024 ? 256 : 512;
    const i64 blocks = (M + rows - 1) / rows;
    const i64 half = (blocks + 1) / 2, some = g < 512 ? blocks : half > 128 ? half : blocks < 128 ? blocks : 128;
    c.blocks = (int)(some < most ? some : most);
    return c;
}

template <class S, class T>
int norm_forward(const Norm& a, hipStream_t st)
{
    const int units = (a.K + 7) / 8;
    if (units > HELD_UNITS) {
        LAUNCH((tr_norm_forward_wide_kernel<S, T, 1024>), dim3((unsigned)a.M), dim3(1024), a);
        return EBSP_OK;
    }
    auto launch = [&](auto group, auto each) {
        constexpr int G = decltype(group)::value, U = decltype(each)::value, NT = G < 256 ? 256 : G;
        LAUNCH((tr_norm_forward_kernel<S, T, G, U, NT>), dim3((unsigned)((a.M + NT / G - 1) / (NT / G))), dim3(NT), a);
        return (int)EBSP_OK;
    };
    // Two units a thread mean half the waves to exchange sums between, one a shorter way through a row.  us with two / one, as above: bf16 8192 x 4096 54 / 59 (beside a stream in fp32 68 / 64),
    // 2048 x 4096 15.6 / 16.2, 512 x 4096 6.9 / 6.7, 128 x 4096 5.6 / 4.7, 1 x 4096 5.0 / 4.2; 1021 x 1003 in fp32 beside fp16 7.9 / 6.5.
    return a.M > 1024 ? with_group<true>(units, launch) : with_group<false>(units, launch);
}

template <class S, class T, bool JOIN>
int norm_backward(const Norm& a, hipStream_t st)
{
    const int units = (a.K + 7) / 8;
    if (a.M > 0) {
        int rc = EBSP_OK;
        if (units > HELD_UNITS)
            LAUNCH((tr_norm_backward_wide_kernel<S, T, JOIN, 1024>), dim3(a.blocks), dim3(1024), a);
        else
            rc = with_group<false>(units, [&](auto group, auto each) {
                constexpr int G = decltype(group)::value, U = decltype(each)::value, SMALL = G < 256 ? 256 : G;
                constexpr bool NARROW = sizeof(S) == 2;
                constexpr int BIG = G == 1024 || takes_next(NARROW, G) ? 1024 : 512;
                constexpr Keep KEEP = U == 2 ? REREAD : takes_next(NARROW, G) ? AHEAD : HOLD;
                if (norm_cut(a.M, a.K, NARROW).threads == BIG) LAUNCH((tr_norm_backward_kernel<S, T, JOIN, G, U, BIG, KEEP>), dim3(a.blocks), dim3(BIG), a);
                else if constexpr (SMALL < BIG) LAUNCH((tr_norm_backward_kernel<S, T, JOIN, G, U, SMALL, KEEP>), dim3(a.blocks), dim3(SMALL), a);
                return (int)EBSP_OK;
            });
        if (rc) return rc;
    }
    const i64 columns = ((i64)a.K + 63) / 64;
    if (a.sums > 0) LAUNCH((tr_norm_columns_kernel<T>), dim3((unsigned)(columns < COLUMN_BLOCKS ? columns : COLUMN_BLOCKS), a.sums), dim3(1024), a);
    return EBSP_OK;
}

template <class T> struct Type { using type = T; };

// The kernels' types: the stream's and the rest's.
template <class F>
int with_types(int stream, int dtype, F&& f)
{
    if (dtype == EBSP_F32) return f(Type<float>(), Type<float>());
    if (dtype == EBSP_BF16) return stream == EBSP_F32 ? f(Type<float>(), Type<__bf16>()) : f(Type<__bf16>(), Type<__bf16>());
    return stream == EBSP_F32 ? f(Type<float>(), Type<_Float16>()) : f(Type<_Float16>(), Type<_Float16>());
}

template <class F>
int with_type(int dtype, F&& f)
{
    return dtype == EBSP_BF16 ? f(Type<__bf16>()) : dtype == EBSP_F16 ? f(Type<_Float16>()) : f(Type<float>());
}

// Units of eight elements that a thread takes one after the other: one where there are few.
int dropout_each(const Dropout& a) { return a.M * ((a.K + 7) / 8) < 256 * 4096 ? 1 : 4; }

i64 dropout_blocks(const Dropout& a)
{
    const i64 per = 256 * dropout_each(a);
    return (a.M * ((a.K + 7) / 8) + per - 1) / per;
}

template <class T>
int dropout(const Dropout& a, hipStream_t st)
{
    // Matrices that the last-level cache does not hold beside their result go past it where no word crosses a line: 8192 x 12288 in bf16 77 us, 73 past it.
    const dim3 blocks((unsigned)dropout_blocks(a));
    if (a.M * a.K * (i64)sizeof(T) > LAST_CACHE / 2 && aligned(a.x, 16) && a.ldx * sizeof(T) % 16 == 0) LAUNCH((tr_dropout_kernel<T, 4, true>), blocks, dim3(256), a);
    else if (dropout_each(a) == 4) LAUNCH((tr_dropout_kernel<T, 4, false>), blocks, dim3(256), a);
    else LAUNCH((tr_dropout_kernel<T, 1, false>), blocks, dim3(256), a);
    return EBSP_OK;
}

// Parts that a row is cut into for its sum: several only where rows are few and long, for they cost a launch or two more.  bf16, us of the loss whole / in parts: 1 x 32000 5.7 / 7.3, 1 x 64000 7.9 / 7.4,
// 1 x 128000 12.1 / 7.4, 48 x 64000 8.2 / 8.3, 48 x 128000 12.7 / 9.3, 96 x 64000 8.3 / 9.2, 96 x 128000 12.8 / 11.1, 128 x 128000 15.4 / 12.0, 200 x 128000 16.9 / 16.4, 256 x 128000 17.1 / 17.9; of the
// loss with its gradient 1 x 64000 11.1 / 10.7, 1 x 128000 18.1 / 11.0, 48 x 64000 11.6 / 13.6, 48 x 128000 18.8 / 16.4, 96 x 128000 19.7 / 24.4, 128 x 128000 20.3 / 28.4: one border for both, at 96.
int token_splits(i64 N, i64 V, int size)
{
    const i64 words = (V * size + 15) / 16;
    if (N > 96 || words <= 4096) return 1;
    const i64 s = 512 / (N > 0 ? N : 1), most = words / 512;
    return (int)(s < most ? s : most);
}

// Parts for a gradient from statistics, which need no scratch, of no less than 512 words: about eight workgroups a CU, four where rows are long.  us with four / eight: 300 x 32000 in bf16 11.1 / 9.8,
// 1000 x 16000 15.6 / 13.6, but logp_train_1024 (64000) 71.8 / 74.5; of no less than 256 words 9.7 and 13.6, but 300 x 8000 5.3 where it takes 4.4.
int token_gradient_splits(i64 N, i64 V, int size)
{
    const i64 words = (V * size + 15) / 16, most = words / 512, each = (words <= 4096 ? 2048 : 1024) / (N > 0 ? N : 1), s = each < most ? each : most;
    return (int)(s < 1 ? 1 : s);
}

size_t padded_bytes(size_t n) { return (n + 255) / 256 * 256; }

size_t token_partial_bytes(i64 N, int splits) { return splits > 1 ? padded_bytes((size_t)N * splits * 2 * sizeof(float)) : 0; }

// Bytes for partial sums, and behind them for `rows` rows of statistics that the caller does not keep.
size_t token_workspace(i64 N, i64 V, int dtype, i64 rows)
{
    const int size = element_size(dtype);
    if (!size || N < 1 || N >= SIZE_MAX_DIM || V < 1 || V >= SIZE_MAX_DIM) return 0;
    return token_partial_bytes(N, token_splits(N, V, size)) + padded_bytes((size_t)rows * 3 * sizeof(float));
}

int check_tokens(const Tokens& d, int dtype)
{
    if (!element_size(dtype)) return fail(EBSP_ERR_ARGUMENT, "dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (d.N < 0 || d.N >= SIZE_MAX_DIM || d.V < 1 || d.V >= SIZE_MAX_DIM) return fail(EBSP_ERR_SHAPE, "invalid shape: N must be 0 and V 1 to 2^31 - 1");
    if (!(d.temperature > 0.f) || d.temperature > FLT_MAX) return fail(EBSP_ERR_ARGUMENT, "temperature must be a positive number");
    if (LOG2E / d.temperature > FLT_MAX) return fail(EBSP_ERR_ARGUMENT, "temperature is too small: its inverse is no number any more");
    if (d.N == 0) return EBSP_OK;
    if (!launchable(d.N, 1024)) return fail(EBSP_ERR_SHAPE, "too many rows for one call");   // (rows in several parts are few)
    if (!d.logits || !d.tokens) return fail(EBSP_ERR_NULL, "logits and tokens must not be NULL");
    if (!stride_ok(d.ld, d.V)) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (!aligned(d.logits, element_size(dtype)) || !aligned(d.tokens, 8) || !aligned(d.grad, element_size(dtype)) || !aligned(d.outer, 4) ||
        !aligned(d.loss, 4) || !aligned(d.logp, 4) || !aligned(d.stats, 4) || !aligned(d.status, 4) || !aligned(d.old_logp, 4) || !aligned(d.advantage, 4) ||
        !aligned(d.ref_logp, 4) || !aligned(d.starts, 8))
        return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    return EBSP_OK;
}

int check_token_gradient(const Tokens& d)
{
    if (!d.grad || !d.outer) return fail(EBSP_ERR_NULL, "the gradients of the call's result and of the logits must not be NULL");
    if (!stride_ok(d.ldd, d.V)) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (d.grad == d.logits && d.ldd != d.ld) return fail(EBSP_ERR_ARGUMENT, "a gradient in the logits' place must have their row stride");
    return EBSP_OK;
}

int check_policy(const Tokens& d)
{
    if (!(d.low >= 0.f) || !(d.high >= 0.f)) return fail(EBSP_ERR_ARGUMENT, "clip_low and clip_high must not be negative");
    if (!finite(d.kl)) return fail(EBSP_ERR_ARGUMENT, "kl_weight must be a finite number");
    if (d.N > 0 && (!d.old_logp || !d.advantage)) return fail(EBSP_ERR_NULL, "old_logp and advantage must not be NULL");
    return EBSP_OK;
}

int check_token_workspace(size_t need, const void* workspace, size_t bytes)
{
    if (need && !workspace) return fail(EBSP_ERR_NULL, "workspace must not be NULL for this shape");
    if (need && (bytes < need || !aligned(workspace, 256))) return fail(EBSP_ERR_WORKSPACE, "workspace too small or not 256-byte aligned");
    return EBSP_OK;
}

// Workgroups of the losses alone, by the row's words.  us with 64 / 128 / 256 / 512 threads: 4096 x 1000 in bf16 5.9 / 8.5 / 14 / 28, 4096 x 4000 10.7 / 9.9 / 15 / 29, 300 x 8000 6.0 / 5.3 / 4.8 / 6.7,
// 300 x 32000 17 / 11 / 8.5 / 10, 1 x 32000 11.6 / 7.3 / 5.7 / 5.8, 128 x 10007 in fp32 7.0 / 5.7 / 5.2 / 5.8.
template <class T>
int token_values(const Tokens& d, hipStream_t st)
{
    const i64 words = (d.V + PER_WORD4<T> - 1) / PER_WORD4<T>;
    const dim3 rows((unsigned)d.N);
    if (words <= 256) LAUNCH((tr_token_value_kernel<64, T>), rows, dim3(64), d);
    else if (words <= 1024) LAUNCH((tr_token_value_kernel<128, T>), rows, dim3(128), d);
    else LAUNCH((tr_token_value_kernel<256, T>), rows, dim3(256), d);
    return EBSP_OK;
}

// Rows that begin at multiples of 16 bytes: no word of theirs crosses a line.
bool whole_words(const Tokens& d, int size) { return aligned(d.logits, 16) && d.ld * size % 16 == 0; }

// Workgroups of a step by the row's words.  Many rows, bf16, us with 64 threads and 8 words each / 64 and 16 / 128 and 16 / 256 and 16 / 512 and 16 (and 8): 4096 x 1000 6.9 / 7.6 / 10.8 / - / -, 4096 x 4000
// 12.3 / 12.4 / 16 / - / -, 4096 x 8000 28 / 22 / 27 / 33 / 46 (38), 4096 x 16000 - / - / - / 56 / 64 (57), 4096 x 32000 - / - / - / 109 / 104 (103), 4096 x 64000 - / - / - / 213 / 190 (202), and with 22 + 9
// words a thread 188.  Few rows of up to 2048 words want more waves: with 256 threads and 8 words, against 64 and 16: 300 x 8000 5.8 / 7.9, 300 x 16000 7.7 / 14.6, 1 x 8000 4.4 / 6.8.
template <class T, bool STREAM>
int token_steps(const Tokens& d, hipStream_t st)
{
    const i64 words = (d.V + PER_WORD4<T> - 1) / PER_WORD4<T>;
    const dim3 rows((unsigned)d.N);
    const bool many = d.N > 1024;
    if (words <= (many ? 512 : 256)) LAUNCH((tr_token_step_kernel<64, T, 8, 0, STREAM>), rows, dim3(64), d);
    else if (many && words <= 1024) LAUNCH((tr_token_step_kernel<64, T, 16, 0, STREAM>), rows, dim3(64), d);
    else if (!many && words <= 2048) LAUNCH((tr_token_step_kernel<256, T, 8, 0, STREAM>), rows, dim3(256), d);
    else if (words <= 2560) LAUNCH((tr_token_step_kernel<256, T, 16, 0, STREAM>), rows, dim3(256), d);
    else if (words <= 4096) LAUNCH((tr_token_step_kernel<512, T, 8, 0, STREAM>), rows, dim3(512), d);
    else if (words <= 16384) LAUNCH((tr_token_step_kernel<512, T, 22, 9, STREAM>), rows, dim3(512), d);
    else LAUNCH((tr_token_step_kernel<1024, T, 16, 8, STREAM>), rows, dim3(1024), d);
    return EBSP_OK;
}

template <class T>
int token_gradient(Tokens d, hipStream_t st)
{
    d.splits = token_gradient_splits(d.N, d.V, sizeof(T));
    // Logits that the last-level cache does not hold are gone from it in part when their sums are through: the gradient then begins with the rows that were read last.  In
    // order / from the last, us: preference_step_16 (370 MB read) 251 / 244, logp_train_1024 (123 MB) 71 / 73.5.
    d.backwards = d.N * d.V * (i64)sizeof(T) > LAST_CACHE;
    const dim3 parts((unsigned)(d.N * d.splits));
    const i64 words = (d.V + PER_WORD4<T> - 1) / PER_WORD4<T>;
    const bool stream = whole_words(d, sizeof(T));
    // A wave a row where the rows are short.  us with 64 / 128 / 256 threads: 4096 x 1000 in bf16 6.8 / 7.4 / 9.8, 4096 x 2000 8.6 / 8.8 / 10.6, 4096 x 4000 15.4 / 14.6 / 14.2, 300 x 8000 6.5 / 5.3 / 4.3.
    if (words <= 256) {
        if (stream) LAUNCH((tr_token_gradient_kernel<64, T, true>), parts, dim3(64), d);
        else LAUNCH((tr_token_gradient_kernel<64, T, false>), parts, dim3(64), d);
    } else {
        if (stream) LAUNCH((tr_token_gradient_kernel<256, T, true>), parts, dim3(256), d);
        else LAUNCH((tr_token_gradient_kernel<256, T, false>), parts, dim3(256), d);
    }
    return EBSP_OK;
}

// Loss and statistics of every row, with `grad` the gradient too.  What needs statistics and is given no place for them has d.stats in the workspace.
template <class T>
int token_loss(Tokens d, bool grad, hipStream_t st)
{
    d.splits = token_splits(d.N, d.V, sizeof(T));
    if (d.splits == 1) return !grad ? token_values<T>(d, st) : whole_words(d, sizeof(T)) ? token_steps<T, true>(d, st) : token_steps<T, false>(d, st);
    LAUNCH((tr_token_part_kernel<256, T>), dim3((unsigned)(d.N * d.splits)), dim3(256), d);
    LAUNCH((tr_token_join_kernel<T>), dim3((unsigned)d.N), dim3(64), d);
    return grad ? token_gradient<T>(d, st) : EBSP_OK;
}

int run_tokens(const Tokens& d, int dtype, bool grad, hipStream_t st)
{
    return with_type(dtype, [&](auto t) { return token_loss<typename decltype(t)::type>(d, grad, st); });
}

int run_token_gradient(const Tokens& d, int dtype, hipStream_t st)
{
    return with_type(dtype, [&](auto t) { return token_gradient<typename decltype(t)::type>(d, st); });
}

int check_pairs(const Tokens& d)
{
    if (d.pairs < 0 || d.pairs >= 1ll << 30) return fail(EBSP_ERR_SHAPE, "invalid shape: pairs must be 0 to 2^30 - 1");
    if ((d.pairs > 0 || d.N > 0) && !d.starts) return fail(EBSP_ERR_NULL, "starts must not be NULL");
    if (!aligned(d.starts, 8) || !aligned(d.stats, 4)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    return EBSP_OK;
}

}  // namespace

extern "C" {

size_t ebsp_residual_norm_workspace_bytes(int64_t M, int64_t K)
{
    if (M < 1 || M >= SIZE_MAX_DIM || K < 1 || K >= WIDTH_MAX) return 0;
    const int narrow = norm_cut(M, K, true).blocks, wide = norm_cut(M, K, false).blocks;
    return (size_t)(narrow > wide ? narrow : wide) * 3 * (size_t)((K + 7) / 8 * 8) * sizeof(float);
}

int ebsp_residual_norm_forward(const void* x, int64_t ldx, const void* branch, int64_t ldb, int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype,
                               const void* weight, const void* post_weight, const void* gate, int64_t ldgate, float scale, float eps, float p,
                               uint64_t seed, uint64_t offset, const int64_t* rng, void* y, int64_t ldy, void* n, int64_t ldn, float* stats, void* stream)
{
    Norm a = {};
    a.x = x, a.ldx = ldx, a.branch = branch, a.ldb = ldb, a.M = M, a.K = (int)K;
    a.weight = weight, a.post_weight = post_weight, a.gate = gate, a.ldgate = ldgate, a.scale = scale, a.eps = eps;
    a.y = y, a.ldy = ldy, a.n = n, a.ldn = ldn, a.stats = stats;
    if (int rc = check_random(p, seed, offset, rng, a.random)) return rc;
    if (int rc = check_norm(a, K, stream_dtype, dtype)) return rc;
    if (!(eps >= 0.f) || !finite(eps)) return fail(EBSP_ERR_ARGUMENT, "eps must be a finite number, not negative");
    if (M == 0 || K == 0) return EBSP_OK;
    if (!x || !n || (branch && !y)) return fail(EBSP_ERR_NULL, "x, n and, with a branch, y must not be NULL");
    if (!stride_ok(ldx, K) || !stride_ok(ldn, K) || (branch && !stride_ok(ldy, K)))
        return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (branch && y == x && ldy != ldx) return fail(EBSP_ERR_ARGUMENT, "a stream in the place of x must have its row stride");
    if (int rc = check_norm_operands(a, stream_dtype, dtype)) return rc;
    if (!launchable(M + 255, group_threads((a.K + 7) / 8))) return fail(EBSP_ERR_SHAPE, "too many rows for one call");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    return with_types(stream_dtype, dtype, [&](auto s, auto t) { return norm_forward<typename decltype(s)::type, typename decltype(t)::type>(a, st); });
}

}  // extern "C"

namespace {

int norm_backward_call(bool join, const void* dy, int64_t lddy, const void* dn, int64_t lddn, const void* y, int64_t ldy, const void* branch, int64_t ldb,
                       int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype, const void* weight, const void* post_weight, const void* gate,
                       int64_t ldgate, float scale, float p, uint64_t seed, uint64_t offset, const int64_t* rng, const float* stats, void* dx,
                       int64_t lddx, void* dbranch, int64_t lddb, void* dweight, void* dpost_weight, void* dgate, int64_t lddgate,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    Norm a = {};
    a.branch = branch, a.ldb = ldb, a.M = M, a.K = (int)K, a.weight = weight, a.post_weight = post_weight, a.gate = gate, a.ldgate = ldgate;
    a.scale = scale, a.y = const_cast<void*>(y), a.ldy = ldy, a.stats = const_cast<float*>(stats);
    a.dy = dy, a.lddy = lddy, a.dn = dn, a.lddn = lddn, a.dx = dx, a.lddx = lddx, a.dbranch = dbranch, a.lddb = lddb;
    if (int rc = check_random(p, seed, offset, rng, a.random)) return rc;
    if (int rc = check_norm(a, K, stream_dtype, dtype)) return rc;
    if (M > 0 && join && (!branch || stream_dtype == EBSP_F32))
        return fail(EBSP_ERR_ARGUMENT, "y is formed again where a branch was joined to a stream of 16 bits: ebsp_residual_norm_backward takes the others");
    if (M > 0 && ((dbranch && !branch) || (dpost_weight && !post_weight) || (dgate && !gate)))
        return fail(EBSP_ERR_ARGUMENT, "a gradient is wanted of an operand that is not there");
    a.sum_w = a.sum_post = a.sum_gate = -1;
    if (dweight) a.column_out[a.sum_w = a.sums++] = dweight;
    if (dpost_weight) a.column_out[a.sum_post = a.sums++] = dpost_weight;
    if (dgate && ldgate == 0) a.column_out[a.sum_gate = a.sums++] = dgate;
    else a.dgate = dgate, a.lddgate = lddgate;
    if (K == 0 || (!dx && !dbranch && !dgate && a.sums == 0)) return EBSP_OK;
    if (M > 0) {
        if (!y || !stats) return fail(EBSP_ERR_NULL, "y (or x) and stats must not be NULL");
        if (!stride_ok(ldy, K) || (dy && !stride_ok(lddy, K)) || (dn && !stride_ok(lddn, K)) || (dx && !stride_ok(lddx, K)) ||
            (dbranch && !stride_ok(lddb, K)) || (a.dgate && !stride_ok(lddgate, K)))
            return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
        if (dx && dx == dy && lddx != lddy) return fail(EBSP_ERR_ARGUMENT, "a gradient in the place of dy must have its row stride");
        if (int rc = check_norm_operands(a, stream_dtype, dtype)) return rc;
    }
    const int size = element_size(dtype);
    for (int i = 0; i < a.sums; ++i)
        if (!aligned(a.column_out[i], size)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (M > 0 && a.sums > 0) {
        if (!workspace) return fail(EBSP_ERR_NULL, "workspace must not be NULL where columns' gradients are wanted");
        if (workspace_bytes < ebsp_residual_norm_workspace_bytes(M, K) || !aligned(workspace, 256))
            return fail(EBSP_ERR_WORKSPACE, "workspace too small or not 256-byte aligned (ebsp_residual_norm_workspace_bytes)");
    }
    a.partial = (float*)workspace;
    a.blocks = M > 0 ? norm_cut(M, K, stream_dtype != EBSP_F32).blocks : 0;
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    return with_types(stream_dtype, dtype, [&](auto s, auto t) {
        using S = typename decltype(s)::type;
        using T = typename decltype(t)::type;
        if constexpr (sizeof(S) == 2)
            if (join) return norm_backward<S, T, true>(a, st);
        return norm_backward<S, T, false>(a, st);
    });
}

}  // namespace

extern "C" {

int ebsp_residual_norm_backward(const void* dy, int64_t lddy, const void* dn, int64_t lddn, const void* y, int64_t ldy, const void* branch, int64_t ldb,
                                int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype, const void* weight, const void* post_weight, const void* gate,
                                int64_t ldgate, float scale, float p, uint64_t seed, uint64_t offset, const int64_t* rng, const float* stats, void* dx,
                                int64_t lddx, void* dbranch, int64_t lddb, void* dweight, void* dpost_weight, void* dgate, int64_t lddgate,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    return norm_backward_call(false, dy, lddy, dn, lddn, y, ldy, branch, ldb, M, K, stream_dtype, dtype, weight, post_weight, gate, ldgate, scale, p, seed, offset, rng,
                              stats, dx, lddx, dbranch, lddb, dweight, dpost_weight, dgate, lddgate, workspace, workspace_bytes, stream);
}

int ebsp_residual_norm_backward_from_x(const void* dy, int64_t lddy, const void* dn, int64_t lddn, const void* x, int64_t ldx, const void* branch, int64_t ldb,
                                       int64_t M, int64_t K, int32_t stream_dtype, int32_t dtype, const void* weight, const void* post_weight, const void* gate,
                                       int64_t ldgate, float scale, float p, uint64_t seed, uint64_t offset, const int64_t* rng, const float* stats, void* dx,
                                       int64_t lddx, void* dbranch, int64_t lddb, void* dweight, void* dpost_weight, void* dgate, int64_t lddgate,
                                       void* workspace, size_t workspace_bytes, void* stream)
{
    return norm_backward_call(true, dy, lddy, dn, lddn, x, ldx, branch, ldb, M, K, stream_dtype, dtype, weight, post_weight, gate, ldgate, scale, p, seed, offset, rng,
                              stats, dx, lddx, dbranch, lddb, dweight, dpost_weight, dgate, lddgate, workspace, workspace_bytes, stream);
}

int ebsp_dropout(const void* x, int64_t ldx, int64_t M, int64_t K, int32_t dtype, float p, uint64_t seed, uint64_t offset, const int64_t* rng,
                 void* out, int64_t ldout, void* stream)
{
    Dropout a = {x, out, ldx, ldout, M, (int)K, {}};
    const int size = element_size(dtype);
    if (!size) return fail(EBSP_ERR_ARGUMENT, "dtype must be EBSP_BF16, EBSP_F16 or EBSP_F32");
    if (int rc = check_random(p, seed, offset, rng, a.random)) return rc;
    if (M < 0 || M >= SIZE_MAX_DIM || K < 0 || K >= WIDTH_MAX) return fail(EBSP_ERR_SHAPE, "invalid shape: M must be 0 to 2^31 - 1 and K 0 to 2^30 - 1");
    if (M == 0 || K == 0) return EBSP_OK;
    if (!x || !out) return fail(EBSP_ERR_NULL, "x and out must not be NULL");
    if (!stride_ok(ldx, K) || !stride_ok(ldout, K)) return fail(EBSP_ERR_ARGUMENT, "a row stride is shorter than the row, or 2^40 and more");
    if (x == out && ldx != ldout) return fail(EBSP_ERR_ARGUMENT, "a result in the place of x must have its row stride");
    if (!launchable(dropout_blocks(a), 256)) return fail(EBSP_ERR_SHAPE, "too many elements for one call");
    if (!aligned(x, size) || !aligned(out, size)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    return with_type(dtype, [&](auto t) { return dropout<typename decltype(t)::type>(a, st); });
}

size_t ebsp_token_logp_workspace_bytes(int64_t N, int64_t V, int32_t dtype) { return token_workspace(N, V, dtype, 0); }

int ebsp_token_logp(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                    float* logp, float* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = temperature, d.kind = TOKEN_LOGP;
    d.logp = logp, d.stats = stats, d.status = status, d.partial = (float*)workspace;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (N == 0) return EBSP_OK;
    if (!logp) return fail(EBSP_ERR_NULL, "logp must not be NULL");
    if (int rc = check_token_workspace(ebsp_token_logp_workspace_bytes(N, V, dtype), workspace, workspace_bytes)) return rc;
    if (int rc = check_device()) return rc;
    return run_tokens(d, dtype, false, (hipStream_t)stream);
}

int ebsp_token_logp_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                             const float* stats, const float* dlogp, void* dlogits, int64_t ldd, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = temperature, d.kind = TOKEN_LOGP;
    d.stats = const_cast<float*>(stats), d.outer = dlogp, d.grad = dlogits, d.ldd = ldd;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (N == 0) return EBSP_OK;
    if (!stats) return fail(EBSP_ERR_NULL, "stats must not be NULL");
    if (int rc = check_token_gradient(d)) return rc;
    if (int rc = check_device()) return rc;
    return run_token_gradient(d, dtype, (hipStream_t)stream);
}

size_t ebsp_policy_workspace_bytes(int64_t N, int64_t V, int32_t dtype)
{
    const int size = element_size(dtype);
    return token_workspace(N, V, dtype, size && token_splits(N, V, size) > 1 ? N : 0);
}

int ebsp_policy_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                        const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                        float* loss, float* logp, float* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = temperature, d.kind = TOKEN_POLICY;
    d.old_logp = old_logp, d.advantage = advantage, d.ref_logp = ref_logp, d.low = clip_low, d.high = clip_high, d.kl = kl_weight;
    d.loss = loss, d.logp = logp, d.stats = stats, d.status = status, d.partial = (float*)workspace;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (int rc = check_policy(d)) return rc;
    if (N == 0) return EBSP_OK;
    if (!loss) return fail(EBSP_ERR_NULL, "loss must not be NULL");
    if (int rc = check_token_workspace(ebsp_token_logp_workspace_bytes(N, V, dtype), workspace, workspace_bytes)) return rc;
    if (int rc = check_device()) return rc;
    return run_tokens(d, dtype, false, (hipStream_t)stream);
}

int ebsp_policy_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                         const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                         const float* stats, const float* dloss, void* dlogits, int64_t ldd, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = temperature, d.kind = TOKEN_POLICY;
    d.old_logp = old_logp, d.advantage = advantage, d.ref_logp = ref_logp, d.low = clip_low, d.high = clip_high, d.kl = kl_weight;
    d.stats = const_cast<float*>(stats), d.outer = dloss, d.grad = dlogits, d.ldd = ldd;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (int rc = check_policy(d)) return rc;
    if (N == 0) return EBSP_OK;
    if (!stats) return fail(EBSP_ERR_NULL, "stats must not be NULL");
    if (int rc = check_token_gradient(d)) return rc;
    if (int rc = check_device()) return rc;
    return run_token_gradient(d, dtype, (hipStream_t)stream);
}

int ebsp_policy_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, float temperature,
                          const float* old_logp, const float* advantage, const float* ref_logp, float clip_low, float clip_high, float kl_weight,
                          const float* dloss, float* loss, float* logp, void* dlogits, int64_t ldd, int32_t* status,
                          void* workspace, size_t workspace_bytes, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = temperature, d.kind = TOKEN_POLICY;
    d.old_logp = old_logp, d.advantage = advantage, d.ref_logp = ref_logp, d.low = clip_low, d.high = clip_high, d.kl = kl_weight;
    d.outer = dloss, d.loss = loss, d.logp = logp, d.grad = dlogits, d.ldd = ldd, d.status = status, d.partial = (float*)workspace;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (int rc = check_policy(d)) return rc;
    if (N == 0) return EBSP_OK;
    if (!loss) return fail(EBSP_ERR_NULL, "loss must not be NULL");
    if (int rc = check_token_gradient(d)) return rc;
    if (int rc = check_token_workspace(ebsp_policy_workspace_bytes(N, V, dtype), workspace, workspace_bytes)) return rc;
    const int splits = token_splits(N, V, element_size(dtype));
    if (splits > 1) d.stats = (float*)((char*)workspace + token_partial_bytes(N, splits));
    if (int rc = check_device()) return rc;
    return run_tokens(d, dtype, true, (hipStream_t)stream);
}

size_t ebsp_preference_workspace_bytes(int64_t N, int64_t pairs, int64_t V, int32_t dtype)
{
    if (pairs < 0 || pairs >= 1ll << 30) return 0;
    return N == 0 && element_size(dtype) ? padded_bytes((size_t)pairs * 3 * sizeof(float)) : token_workspace(N, V, dtype, N + pairs);
}
}  // extern "C"

namespace {

// The rows' log-probabilities, and the pairs' losses and slopes from them.
int run_pairs(const Tokens& d, const float* ref, float beta, int kind, float smoothing, int mean, float* loss, float* sums, int* status, int dtype,
              hipStream_t st)
{
    if (d.N > 0) {
        if (int rc = run_tokens(d, dtype, false, st)) return rc;
    } else LAUNCH(tr_starts_kernel, dim3((unsigned)(d.pairs < WAVE ? d.pairs : WAVE)), dim3(64), d);
    const Preference a = {d, ref, beta, smoothing, kind, mean, loss, sums, status};
    if (d.pairs > 0) LAUNCH((tr_preference_kernel<256>), dim3((unsigned)d.pairs), dim3(256), a);
    return EBSP_OK;
}

int check_preference(const Tokens& d, int dtype, const float* ref, float beta, int kind, float smoothing, const float* loss, const float* sums, const int* status)
{
    if (int rc = check_tokens(d, dtype)) return rc;
    if (int rc = check_pairs(d)) return rc;
    if (kind < EBSP_PREFERENCE_SIGMOID || kind > EBSP_PREFERENCE_SQUARE) return fail(EBSP_ERR_ARGUMENT, "kind must be one of EBSP_PREFERENCE_*");
    if (!(beta > 0.f) || !finite(beta)) return fail(EBSP_ERR_ARGUMENT, "beta must be a positive number");
    if (!(smoothing >= 0.f) || smoothing > 1.f) return fail(EBSP_ERR_ARGUMENT, "smoothing must be 0 to 1");
    if (smoothing != 0.f && kind != EBSP_PREFERENCE_SIGMOID) return fail(EBSP_ERR_ARGUMENT, "smoothing is of the sigmoid loss alone");
    if (d.pairs > 0 && !loss) return fail(EBSP_ERR_NULL, "loss must not be NULL");
    if (!aligned(ref, 4) || !aligned(loss, 4) || !aligned(sums, 4) || !aligned(status, 4)) return fail(EBSP_ERR_ARGUMENT, "a pointer is not aligned to its elements");
    if (!launchable(d.pairs, 256)) return fail(EBSP_ERR_SHAPE, "too many pairs for one call");
    return EBSP_OK;
}

}  // namespace

extern "C" {

int ebsp_preference_forward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                            int64_t pairs, const float* ref, float beta, int32_t kind, float smoothing, int32_t mean, float* loss, float* sums,
                            float* saved, int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = 1.f, d.kind = TOKEN_PREFERENCE;
    d.starts = starts, d.pairs = pairs, d.stats = saved, d.partial = (float*)workspace;
    if (int rc = check_preference(d, dtype, ref, beta, kind, smoothing, loss, sums, status)) return rc;
    if (pairs == 0 && N == 0) return EBSP_OK;
    if (!saved) {
        if (int rc = check_token_workspace(ebsp_preference_workspace_bytes(N, pairs, V, dtype), workspace, workspace_bytes)) return rc;
        d.stats = (float*)((char*)workspace + token_partial_bytes(N, token_splits(N, V, element_size(dtype))));
    } else if (int rc = check_token_workspace(ebsp_token_logp_workspace_bytes(N, V, dtype), workspace, workspace_bytes)) return rc;
    if (int rc = check_device()) return rc;
    return run_pairs(d, ref, beta, kind, smoothing, mean, loss, sums, status, dtype, (hipStream_t)stream);
}

int ebsp_preference_backward(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                             int64_t pairs, const float* saved, const float* dloss, void* dlogits, int64_t ldd, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = 1.f, d.kind = TOKEN_PREFERENCE;
    d.starts = starts, d.pairs = pairs, d.stats = const_cast<float*>(saved), d.outer = dloss, d.grad = dlogits, d.ldd = ldd;
    if (int rc = check_tokens(d, dtype)) return rc;
    if (int rc = check_pairs(d)) return rc;
    if (N == 0) return EBSP_OK;
    if (!saved) return fail(EBSP_ERR_NULL, "saved must not be NULL");
    if (pairs == 0) d.outer = (const float*)starts;                          // (never read: no row is part of an answer)
    if (int rc = check_token_gradient(d)) return rc;
    if (int rc = check_device()) return rc;
    return run_token_gradient(d, dtype, (hipStream_t)stream);
}

int ebsp_preference_loss_grad(const void* logits, int64_t ld, int64_t N, int64_t V, int32_t dtype, const int64_t* tokens, const int64_t* starts,
                              int64_t pairs, const float* ref, float beta, int32_t kind, float smoothing, int32_t mean, const float* dloss, float* loss,
                              float* sums, void* dlogits, int64_t ldd, int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    Tokens d = {};
    d.logits = logits, d.ld = ld, d.N = N, d.V = V, d.tokens = tokens, d.temperature = 1.f, d.kind = TOKEN_PREFERENCE;
    d.starts = starts, d.pairs = pairs, d.outer = dloss, d.grad = dlogits, d.ldd = ldd, d.partial = (float*)workspace;
    if (int rc = check_preference(d, dtype, ref, beta, kind, smoothing, loss, sums, status)) return rc;
    if (pairs == 0 && N == 0) return EBSP_OK;
    if (pairs == 0) d.outer = (const float*)starts;                          // (never read: no row is part of an answer)
    if (N > 0)
        if (int rc = check_token_gradient(d)) return rc;
    if (int rc = check_token_workspace(ebsp_preference_workspace_bytes(N, pairs, V, dtype), workspace, workspace_bytes)) return rc;
    d.stats = (float*)((char*)workspace + token_partial_bytes(N, token_splits(N, V, element_size(dtype))));
    if (int rc = check_device()) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (int rc = run_pairs(d, ref, beta, kind, smoothing, mean, loss, sums, status, dtype, st)) return rc;
    return N > 0 ? run_token_gradient(d, dtype, st) : EBSP_OK;
}

}  // extern "C"
