// Losses of the tokens that were taken: their log-probabilities, the clipped policy loss with a KL term, the preference loss of pairs.
// Part of the ZipLine library (see tuning.hip); device code for gfx950.
//
// Per row, with logits s over a vocabulary, a token t and a temperature T:
//     p = softmax(s / T)     logp = (s_t - m) / T - ln sum_j e^((s_j - m) / T)     d logp / d s_j = ([j = t] - p_j) / T
// and every loss is a function of the rows' logp, so its gradient is a row's slope dL/dlogp times the last.  Policy, with old the log-probability
// under the policy that drew t, A the advantage and ref that of a reference:
//     x = e^(logp - old)     loss = -min(x A, clamp(x, 1 - low, 1 + high) A) + kl (e^(ref - logp) - (ref - logp) - 1)
// Exponentials are taken to base 2, of x_j = s_j c - k with c = log2(e) / T and k = m c, m the row's largest logit: one fused product and sum.  k is rounded, but it
// is the same in the sum, in logp and in the gradient, so what it is off by falls out.  Rows whose k is 2^20 and more, either way (of the type's lowest values, say), where
// that would be too much, take x_j = (s_j - m) c, slower and as good.  Statistics are m and log2 of the sum, apart; m starts from the lowest finite value, so logits of -inf
// weigh nothing.  Rows without a token are not read.
#pragma once
#include "ebsp_training.h"
#include "tr_rows.h"

namespace {

enum TokenLoss { TOKEN_LOGP, TOKEN_POLICY, TOKEN_PREFERENCE };

struct Tokens {
    const void* logits;
    i64 ld, N, V;
    const i64* tokens;
    float temperature;
    int kind;
    const float *old_logp, *advantage, *ref_logp;            // policy
    float low, high, kl;
    const i64* starts;                                       // preference: [2 pairs + 1]
    i64 pairs;
    const float* outer;                                      // dL/dlogp or dL/dloss of every row, dL/dloss of every pair
    float *loss, *logp;
    float* stats;                                            // [N][3]: m, log2 of the sum, logp; behind them, for a preference loss, [pairs][3]
    int* status;
    void* grad;
    i64 ldd;
    float* partial;                                          // [N][splits][2]: m and the sum of a part of a row
    int splits;
    int backwards;                                           // a gradient takes the last row first
};

struct Sum {
    float m, s;
};

constexpr float FAR = 1048576.f;                             // 2^20: k is off by 2^-5 at most, and x by as much where it is largest

// Whether a row whose largest logit is m takes the differences first (also where m is no number), and k of the others.
__device__ __forceinline__ bool is_far(float m, float ct) { return !(fabsf(m) * ct < FAR); }
__device__ __forceinline__ float reference(float m, float ct) { return fmaxf(m * ct, -FAR); }

// What a sum from a's reference is multiplied by, as a power of two, to be one from b's: k, or m c itself where that is far.
__device__ __forceinline__ float apart(float a, float b, float ct)
{
    if (is_far(a, ct)) return is_far(b, ct) ? (a - b) * ct : fmaf(a, ct, -reference(b, ct));
    return is_far(b, ct) ? fmaf(-b, ct, reference(a, ct)) : reference(a, ct) - reference(b, ct);
}

__device__ __forceinline__ Sum joined(Sum a, Sum b, float ct)
{
    Sum r;
    r.m = fmaxf(a.m, b.m);
    r.s = a.s * exp2_fast(apart(a.m, r.m, ct)) + b.s * exp2_fast(apart(b.m, r.m, ct));
    return r;
}

// The sum of a word's exponentials, from k or, of a far row, m.
template <class T, bool FROM_M>
__device__ __forceinline__ void add_exponentials(float& sum, Word4 raw, float from, float ct)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) sum += exp2_fast(FROM_M ? (to_float(w.v[i]) - from) * ct : fmaf(to_float(w.v[i]), ct, -from));
}

// A row's words: those that are whole, and what is left behind them, which the thread whose turn it would be takes by itself.
template <int NT, class T>
struct Words {
    static constexpr u32 N = PER_WORD4<T>;
    u32 first, whole, end;                                   // from `first`, a multiple of N
    __device__ __forceinline__ Words(i64 v0, i64 v1) : first((u32)v0), whole((u32)(v1 / N * N)), end((u32)v1) {}
    __device__ __forceinline__ bool rest() const { return whole >= first && whole < end && (whole - first) / N % NT == threadIdx.x; }

    // AHEAD words, NT apart, from v on; -inf for those that are not there.  Each is loaded from somewhere: no load waits for another, as it would in a branch.
    template <bool STREAM, int AHEAD>
    __device__ __forceinline__ void load(Word4 (&w)[AHEAD], const T* s, u32 v) const
    {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) w[j] = load_last<STREAM>(s + (v + j * NT * N < whole ? v + j * NT * N : first));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (v + j * NT * N >= whole) w[j] = lowest_word<T>();
    }
};

// The sum over a part of a row, in one pass: AHEAD words at a time with the next ones under way, the sum so far times 2^(k - k') where they have a larger one.
template <int NT, class T>
__device__ __forceinline__ Sum part_sum(const T* s, const Words<NT, T> at, float ct)
{
    constexpr u32 N = PER_WORD4<T>, AHEAD = 4, TURN = AHEAD * NT * N;
    Sum sum = {-FLT_MAX, 0.f};
    float k = -FAR;
    Word4 w[AHEAD], next[AHEAD], rest[1];
    const bool has_rest = at.rest();
    if (has_rest) rest[0] = read_logits(s, at.whole, at.end);
    if (at.first < at.whole) {
        at.template load<false>(w, s, at.first + threadIdx.x * N);
        for (u32 base = at.first; base < at.whole; base += TURN) {
            if (base + TURN < at.whole) at.template load<false>(next, s, base + TURN + threadIdx.x * N);
#pragma unroll
            for (u32 j = 0; j < AHEAD; ++j) sum.m = largest<T>(w[j], sum.m);
            const float high = reference(sum.m, ct);
            sum.s *= exp2_fast(k - high);
            k = high;
#pragma unroll
            for (u32 j = 0; j < AHEAD; ++j) add_exponentials<T, false>(sum.s, w[j], k, ct);
#pragma unroll
            for (u32 j = 0; j < AHEAD; ++j) w[j] = next[j];
        }
    }
    if (has_rest) {
        sum.m = largest<T>(rest[0], sum.m);
        const float high = reference(sum.m, ct);
        sum.s *= exp2_fast(k - high);
        add_exponentials<T, false>(sum.s, rest[0], high, ct);
    }
    if (is_far(sum.m, ct)) {                                                 // (sum.m is this thread's own: so is its sum)
        sum.s = 0.f;
        for (u32 v = at.first + threadIdx.x * N; v < at.whole; v += NT * N) add_exponentials<T, true>(sum.s, load_loose(s + v), sum.m, ct);
        if (has_rest) add_exponentials<T, true>(sum.s, rest[0], sum.m, ct);
    }
    return sum;
}

// Starts that are not those of rows one behind the other (one is before 0, beyond N or below the one before) say of no row whose it is: no pair's results stand then.  They are looked
// over beside the rows, in as many slices as rows and pairs allow, up to 64; each slice's finding stands in the third place behind the pair of its number, where the pairs' kernel reads them all.
__device__ __forceinline__ i64 start_slices(const Tokens& d) { return min(d.pairs, d.N > 0 && d.N < WAVE ? d.N : (i64)WAVE); }

__device__ __forceinline__ float* start_finding(const Tokens& d, i64 slice) { return d.stats + (d.N + slice) * 3 + 2; }

template <int NT>
__device__ __forceinline__ void check_starts(const Tokens& d, i64 slice)
{
    const i64 slices = start_slices(d);
    if (slice >= slices) return;                                             // (the same for the workgroup)
    const i64 all = 2 * d.pairs + 1, each = (all + slices - 1) / slices, end = min((slice + 1) * each, all);
    int wrong = 0;
#pragma unroll 4
    for (i64 i = slice * each + threadIdx.x; i < end; i += NT) {
        const i64 at = d.starts[i], before = i > 0 ? d.starts[i - 1] : 0;
        wrong |= (at < before) | (at > d.N);
    }
    wrong = __syncthreads_or(wrong);
    if (threadIdx.x == 0) *start_finding(d, slice) = wrong ? 1.f : 0.f;
}

// The row's token, -1 for none: negative, beyond the vocabulary, or a row outside all answers.
__device__ __forceinline__ int token_of(const Tokens& d, i64 n, bool& bad)
{
    const i64 t = d.tokens[n];
    i64 first = 0, behind = d.N;
    if (d.kind == TOKEN_PREFERENCE) {                                        // (with a return in here the compiler has lost the token)
        first = d.starts[0];
        behind = d.starts[2 * d.pairs];
    }
    bad = t >= d.V;
    return ((t < 0) | bad | (n < first) | (n >= behind)) ? -1 : (int)t;
}

// e^g - g - 1, to its own precision where g is small: there by its series.
__device__ __forceinline__ float exp_above_tangent(float g)
{
    if (fabsf(g) > 0.25f) {
        const float e = expm1f(g);
        return e == INFINITY ? e : e - g;
    }
    float t = 1.f / 40320.f;
    t = fmaf(t, g, 1.f / 5040.f);
    t = fmaf(t, g, 1.f / 720.f);
    t = fmaf(t, g, 1.f / 120.f);
    t = fmaf(t, g, 1.f / 24.f);
    t = fmaf(t, g, 1.f / 6.f);
    return fmaf(t, g, 0.5f) * g * g;
}

// The policy loss of a row, and its slope over logp.  (NaN comes through: comparisons are made so that it takes the slope with the ratio in it.)
__device__ __forceinline__ float policy_of(const Tokens& d, i64 n, float logp, float& loss)
{
    const float a = d.advantage[n], x = expf(logp - d.old_logp[n]);
    const float border = a < 0.f ? 1.f - d.low : 1.f + d.high;
    const bool held = a < 0.f ? x < border : x > border;
    loss = -a * (held ? border : x);
    float slope = held ? a - a : -a * x;
    if (d.ref_logp && d.kl != 0.f) {
        const float g = d.ref_logp[n] - logp;
        loss = fmaf(d.kl, exp_above_tangent(g), loss);
        slope = fmaf(-d.kl, expm1f(g), slope);
    }
    return slope;
}

__device__ __forceinline__ float logp_of(float token_logit, float m, float l, float temperature)
{
    const float ct = LOG2E / temperature;
    if (is_far(m, ct)) return (token_logit - m) / temperature - LN2 * l;
    return LN2 * (fmaf(token_logit, ct, -reference(m, ct)) - l);
}

// What a row with a token leaves behind; one thread writes.
__device__ __forceinline__ void write_row(const Tokens& d, i64 n, float m, float l, float logp, float loss)
{
    if (d.logp) d.logp[n] = logp;
    if (d.loss) d.loss[n] = loss;
    if (d.stats) {
        d.stats[n * 3] = m;
        d.stats[n * 3 + 1] = l;
        d.stats[n * 3 + 2] = logp;
    }
}

// The answer that row n is part of: how many starts are not behind it, less one.  64 starts are looked at together; all lanes of a wave take part.
__device__ __forceinline__ i64 answer_of(const Tokens& d, i64 n)
{
    i64 lo = 0, hi = 2 * d.pairs;                                            // starts[lo] <= n < starts[hi]
    const int lane = threadIdx.x & 63;
    while (hi - lo > 1) {
        const i64 step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step;
        const u32 before = (u32)__popcll(__ballot(at < hi && d.starts[at] <= n));
        lo += before * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// dL/dlogp of row n, whole: times what stands outside the loss.
__device__ __forceinline__ float slope_of(const Tokens& d, i64 n, float logp)
{
    float loss;
    if (d.kind == TOKEN_LOGP) return d.outer[n];
    if (d.kind == TOKEN_POLICY) return policy_of(d, n, logp, loss) * d.outer[n];
    const i64 answer = answer_of(d, n);
    return d.stats[(d.N + answer / 2) * 3 + (answer & 1)] * d.outer[answer / 2];
}

// A row's gradient: c ([j = token] - p_j), with p_j = 2^(x_j) 2^-l.
struct TokenSlope {
    float ct, from, c, scale;                                // from: k, or m of a far row; scale: -c 2^-l
    bool far;
};

__device__ __forceinline__ TokenSlope token_slope(float m, float l, float temperature, float slope)
{
    const float ct = LOG2E / temperature, c = slope / temperature;
    const bool far = is_far(m, ct);
    return TokenSlope{ct, far ? m : reference(m, ct), c, -c * exp2_fast(-l), far};
}

template <class T, bool FROM_M>
__device__ __forceinline__ Word4 gradient_word(const TokenSlope& g, Word4 raw)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) {
        const float s = to_float(w.v[i]);
        w.v[i] = from_float<T>(g.scale * exp2_fast(FROM_M ? (s - g.from) * g.ct : fmaf(s, g.ct, -g.from)));
    }
    return w.raw;
}

template <class T>
__device__ __forceinline__ T token_gradient(const TokenSlope& g, float s)
{
    return from_float<T>(fmaf(g.scale, exp2_fast(g.far ? (s - g.from) * g.ct : fmaf(s, g.ct, -g.from)), g.c));
}

// The body of a loop over a row's words for either kind of row.
template <bool VALUE> struct FromM { static constexpr bool value = VALUE; };
template <class F>
__device__ __forceinline__ void with_far(bool far, F&& f)
{
    if (far) f(FromM<true>());
    else f(FromM<false>());
}

template <int NT, class T>
__device__ __forceinline__ void write_zeros(T* out, i64 v0, i64 v1)
{
    for (i64 v = v0 + (i64)threadIdx.x * PER_WORD4<T>; v < v1; v += NT * PER_WORD4<T>) write_gradient(out, v, v1, Word4{0, 0, 0, 0});
}

// A row without a token: nothing of it is read.
template <int NT, class T>
__device__ __forceinline__ bool leave_row(const Tokens& d, i64 n, int token, bool bad, bool grad)
{
    if (threadIdx.x == 0 && d.status) d.status[n] = bad ? EBSP_STATUS_RANGE : EBSP_STATUS_OK;
    if (token >= 0) return false;
    if (threadIdx.x == 0) write_row(d, n, 0.f, 0.f, 0.f, 0.f);
    if (grad) write_zeros<NT, T>((T*)d.grad + n * d.ldd, 0, d.V);
    return true;
}

// The row's results from its statistics; its slope.
__device__ __forceinline__ float finish_row(const Tokens& d, i64 n, float token_logit, float m, float l)
{
    const float logp = logp_of(token_logit, m, l, d.temperature);
    float loss = 0.f, slope = 0.f;
    if (d.kind == TOKEN_POLICY) slope = policy_of(d, n, logp, loss);
    if (threadIdx.x == 0) write_row(d, n, m, l, logp, loss);
    return slope;
}

// Loss and statistics alone: one workgroup a row, which is read once and kept nowhere.  Memory bounds it: 4096 rows of 128000 in bf16 183 us, 5.7 TB/s, 1024 of 64000 31 (of it
// some 9 to start and to end); with 512 threads 180 and 31, with 1024 183 and 37, two words ahead where there are four 184 and 29, 400 rows of 128000 then 36 where they take 27.
template <int NT, class T>
__global__ void __launch_bounds__(NT) tr_token_value_kernel(Tokens d)
{
    __shared__ Sum shared[16];
    const i64 n = blockIdx.x;
    const T* s = (const T*)d.logits + n * d.ld;
    const float ct = LOG2E / d.temperature;
    bool bad;
    if (d.kind == TOKEN_PREFERENCE) check_starts<NT>(d, n);
    const int token = token_of(d, n, bad);
    if (leave_row<NT, T>(d, n, token, bad, false)) return;
    const float token_logit = to_float(s[token]);
    Sum sum = part_sum(s, Words<NT, T>(0, d.V), ct);
    sum = block_reduce<NT>(sum, shared, [ct](Sum x, Sum y) { return joined(x, y, ct); });
    finish_row(d, n, token_logit, sum.m, log2_sum(sum.s));
}

// Loss, statistics and gradient: one workgroup a row, whose first HELD words a thread stay in registers and the next KEPT in shared memory from the one load on; only what
// lies behind is read twice.
template <int NT, class T, int HELD, int KEPT, bool STREAM>
__global__ void __launch_bounds__(NT) tr_token_step_kernel(Tokens d)
{
    constexpr int N = PER_WORD4<T>;
    constexpr u32 STEP = NT * N, BEHIND = (HELD + KEPT) * STEP;
    __shared__ float scalar[16];
    __shared__ Word4 kept[KEPT > 0 ? KEPT * NT : 1];
    const i64 n = blockIdx.x;
    const T* s = (const T*)d.logits + n * d.ld;
    bool bad;
    const int token = token_of(d, n, bad);
    if (leave_row<NT, T>(d, n, token, bad, true)) return;
    const float token_logit = to_float(s[token]), ct = LOG2E / d.temperature;
    const Words<NT, T> at(0, d.V);
    const u32 v0 = threadIdx.x * N, whole = at.whole, end = min(whole, HELD * STEP);
    Sum rest = {-FLT_MAX, 0.f};
    if (BEHIND < whole) rest = part_sum(s, Words<NT, T>(BEHIND, whole), ct);
    float m = rest.m;
    if constexpr (KEPT > 0) {
        if (HELD * STEP < whole) {
            Word4 w[KEPT];
            at.template load<STREAM>(w, s, v0 + HELD * STEP);
#pragma unroll
            for (int j = 0; j < KEPT; ++j) {
                kept[j * NT + threadIdx.x] = w[j];
                m = largest<T>(w[j], m);
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);                                       // (before the registers fill)
    const bool has_last = at.rest();
    Word4 held[HELD];
#pragma unroll
    for (int j = 0; j < HELD; ++j) held[j] = v0 + j * STEP < end ? load_last<STREAM>(s + j * STEP + v0) : lowest_word<T>();
    Word4 last = lowest_word<T>();
    if (has_last) last = read_logits(s, whole, d.V);
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (j * STEP < end) {
            m = largest<T>(held[j], m);
            __builtin_amdgcn_sched_barrier(0);                               // word by word: the registers are full
        }
    if (has_last) m = largest<T>(last, m);
    forget_floats(held);
    m = block_reduce<NT>(m, scalar, [](float a, float b) { return fmaxf(a, b); });
    float sum = joined(rest, Sum{m, 0.f}, ct).s;                             // (m is the larger)
    const bool far = is_far(m, ct);
    const float from = far ? m : reference(m, ct);
    with_far(far, [&](auto kind) {
        constexpr bool FROM_M = decltype(kind)::value;
#pragma unroll
        for (int j = 0; j < HELD; ++j)
            if (j * STEP < end) {
                add_exponentials<T, FROM_M>(sum, held[j], from, ct);
                __builtin_amdgcn_sched_barrier(0);
            }
        if (has_last) add_exponentials<T, FROM_M>(sum, last, from, ct);
        if constexpr (KEPT > 0)
#pragma unroll 1
            for (int j = 0; j < KEPT && (HELD + j) * STEP < whole; ++j) add_exponentials<T, FROM_M>(sum, kept[j * NT + threadIdx.x], from, ct);
    });
    const float l = log2_sum(block_reduce<NT>(sum, scalar, [](float a, float b) { return a + b; }));
    const float slope = finish_row(d, n, token_logit, m, l);
    const TokenSlope g = token_slope(m, l, d.temperature, slope * d.outer[n]);
    T* out = (T*)d.grad + n * d.ldd;
    __builtin_amdgcn_s_waitcnt(0);                                           // in place: every thread has the token's logit
    __syncthreads();
    if (g.c == 0.f) {
        write_zeros<NT, T>(out, 0, d.V);
        return;
    }
    forget_floats(held);
    with_far(g.far, [&](auto kind) {
        constexpr bool FROM_M = decltype(kind)::value;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            if (v0 + j * STEP < end) store_stream(out + j * STEP + v0, gradient_word<T, FROM_M>(g, held[j]));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (has_last) write_gradient(out, whole, d.V, gradient_word<T, FROM_M>(g, last));
        if constexpr (KEPT > 0)
#pragma unroll 1
            for (int j = 0; j < KEPT; ++j) {
                const u32 v = v0 + (HELD + j) * STEP;
                if (v < whole) store_stream(out + v, gradient_word<T, FROM_M>(g, kept[j * NT + threadIdx.x]));
            }
        for (u32 v = v0 + BEHIND; v < whole; v += STEP) store_stream(out + v, gradient_word<T, FROM_M>(g, load_loose(s + v)));
    });
    __builtin_amdgcn_s_waitcnt(0);                                           // stores to one address arrive in this order
    __syncthreads();
    if (threadIdx.x == 0) out[token] = token_gradient<T>(g, token_logit);
}

__device__ __forceinline__ void part_range(const Tokens& d, int part, int per_word, i64& v0, i64& v1)
{
    const i64 words = (d.V + per_word - 1) / per_word, each = (words + d.splits - 1) / d.splits;
    v0 = min(part * each * per_word, d.V);
    v1 = min(v0 + each * per_word, d.V);
}

// Few rows: the sum of a part of a row by each workgroup ...
template <int NT, class T>
__global__ void __launch_bounds__(NT) tr_token_part_kernel(Tokens d)
{
    __shared__ Sum shared[16];
    const i64 n = blockIdx.x / d.splits;
    const float ct = LOG2E / d.temperature;
    bool bad;
    if (token_of(d, n, bad) < 0) return;
    i64 v0, v1;
    part_range(d, blockIdx.x % d.splits, PER_WORD4<T>, v0, v1);
    Sum sum = part_sum((const T*)d.logits + n * d.ld, Words<NT, T>(v0, v1), ct);
    sum = block_reduce<NT>(sum, shared, [ct](Sum x, Sum y) { return joined(x, y, ct); });
    if (threadIdx.x == 0) {
        float* out = d.partial + (i64)blockIdx.x * 2;
        out[0] = sum.m;
        out[1] = sum.s;
    }
}

// ... joined by one wave a row, in the order of the parts.
template <class T>
__global__ void __launch_bounds__(64) tr_token_join_kernel(Tokens d)
{
    const i64 n = blockIdx.x;
    bool bad;
    if (d.kind == TOKEN_PREFERENCE) check_starts<64>(d, n);
    const int token = token_of(d, n, bad);
    if (leave_row<64, T>(d, n, token, bad, false)) return;
    const float token_logit = to_float(((const T*)d.logits)[n * d.ld + token]), ct = LOG2E / d.temperature;
    Sum sum = {-FLT_MAX, 0.f};
    for (int p = threadIdx.x; p < d.splits; p += 64) {
        const float* in = d.partial + (n * d.splits + p) * 2;
        sum = joined(sum, Sum{in[0], in[1]}, ct);
    }
    sum = block_reduce<64>(sum, (Sum*)nullptr, [ct](Sum x, Sum y) { return joined(x, y, ct); });
    finish_row(d, n, token_logit, sum.m, log2_sum(sum.s));
}

// The gradient from statistics: every row in `splits` parts.  Nothing is read of a row but the workgroup's own part, which it may overwrite.
template <int NT, class T, bool STREAM>
__global__ void __launch_bounds__(NT) tr_token_gradient_kernel(Tokens d)
{
    constexpr int N = PER_WORD4<T>;
    const i64 row = blockIdx.x / d.splits, n = d.backwards ? d.N - 1 - row : row;
    i64 v0, v1;
    part_range(d, blockIdx.x % d.splits, N, v0, v1);
    const T* s = (const T*)d.logits + n * d.ld;
    T* out = (T*)d.grad + n * d.ldd;
    bool bad;
    const int token = token_of(d, n, bad);
    const TokenSlope g = token_slope(d.stats[n * 3], d.stats[n * 3 + 1], d.temperature, token < 0 ? 0.f : slope_of(d, n, d.stats[n * 3 + 2]));
    if (g.c == 0.f) {
        write_zeros<NT, T>(out, v0, v1);
        return;
    }
    const Words<NT, T> at(v0, v1);
    const bool mine = token >= v0 && token < v1 && (token - v0) / N % NT == threadIdx.x, has_rest = at.rest();
    const float token_logit = mine ? to_float(s[token]) : 0.f;
    Word4 rest = lowest_word<T>();
    if (has_rest) rest = read_logits(s, at.whole, at.end);
    constexpr u32 AHEAD = 4;
    with_far(g.far, [&](auto kind) {
        constexpr bool FROM_M = decltype(kind)::value;
        for (u32 base = at.first; base < at.whole; base += AHEAD * NT * N) {
            const u32 v = base + threadIdx.x * N;
            Word4 w[AHEAD];
            at.template load<STREAM>(w, s, v);
#pragma unroll
            for (u32 j = 0; j < AHEAD; ++j)
                if (v + j * NT * N < at.whole) store_stream(out + v + j * NT * N, gradient_word<T, FROM_M>(g, w[j]));
        }
        if (has_rest) write_gradient(out, at.whole, at.end, gradient_word<T, FROM_M>(g, rest));
    });
    if (mine) {
        __builtin_amdgcn_s_waitcnt(0);                                       // behind this thread's own store of that word
        out[token] = token_gradient<T>(g, token_logit);
    }
}

// Pairs without any rows: their starts are looked over here.
__global__ void __launch_bounds__(64) tr_starts_kernel(Tokens d) { check_starts<64>(d, blockIdx.x); }

// The losses of pairs: one workgroup a pair, whose rows' logp stand in the statistics.  Sums over an answer and what follows are in 64 bits.
struct Preference {
    Tokens d;
    const float* ref;                            // [2 pairs], or NULL
    float beta, smoothing;
    int loss_kind, mean;
    float *loss, *sums;
    int* status;
};

template <int NT>
__global__ void __launch_bounds__(NT) tr_preference_kernel(Preference a)
{
    constexpr int HALF = NT / 2, WAVES = HALF / WAVE;
    struct Found { double sum; i64 count; i64 bad; };
    __shared__ Found found[2][WAVES];
    const i64 pair = blockIdx.x;
    const int side = threadIdx.x / HALF;                                     // half of the workgroup for each answer
    const i64* at = a.d.starts + 2 * pair + side;
    const i64 from = at[0] < 0 ? 0 : at[0] < a.d.N ? at[0] : a.d.N, to = at[1] < from ? from : at[1] < a.d.N ? at[1] : a.d.N;
    const i64 slices = start_slices(a.d);
    const float finding = (i64)(threadIdx.x % WAVE) < slices ? *start_finding(a.d, threadIdx.x % WAVE) : 0.f;
    double part = 0.;
    i64 tokens = 0;
    bool bad = false;
    for (i64 n0 = from; n0 < to; n0 += HALF) {                               // (the same turns for a wave)
        const i64 n = n0 + threadIdx.x % HALF;
        bool past = false, has = false;
        if (n < to) {
            has = token_of(a.d, n, past) >= 0;
            if (has) part += a.d.stats[n * 3 + 2];
        }
        tokens += __popcll(__ballot(has));
        bad |= __ballot(past) != 0;
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) part += __shfl_xor(part, x);
    const bool astray = __ballot(finding != 0.f) != 0;                       // (the starts, anyone's)
    if (threadIdx.x % WAVE == 0) found[side][threadIdx.x % HALF / WAVE] = Found{part, tokens, bad};
    __syncthreads();
    if (threadIdx.x) return;
    double sum[2], share[2];
    bad = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        double all = 0.;
        i64 n = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            all += found[s][w].sum;
            n += found[s][w].count;
            bad |= found[s][w].bad != 0;
        }
        share[s] = a.mean && n > 0 ? 1. / (double)n : 1.;
        sum[s] = all * share[s];
    }
    const double beta = a.beta, e = a.smoothing;
    const double h = a.ref ? (sum[0] - a.ref[2 * pair]) - (sum[1] - a.ref[2 * pair + 1]) : sum[0] - sum[1];
    double loss, slope;
    if (a.loss_kind == EBSP_PREFERENCE_HINGE) {
        loss = beta * h < 1. ? 1. - beta * h : beta * h == beta * h ? 0. : h;
        slope = beta * h >= 1. ? 0. : beta * h == beta * h ? -beta : h;
    } else if (a.loss_kind == EBSP_PREFERENCE_SQUARE) {
        const double gap = h - 0.5 / beta;
        loss = gap * gap;
        slope = 2. * gap;
    } else {
        // With low = e^-|z|, -log sigmoid(-|z|) is |z| + log(1 + low) and -log sigmoid(|z|) the second alone: |z| comes with the weight of one side, and not where that is 0 (z may be infinite).
        const double z = beta * h, low = exp(-fabs(z)), wrong = z < 0. ? 1. - e : e;
        loss = (wrong != 0. ? wrong * fabs(z) : z == z ? 0. : z) + log1p(low);
        slope = -beta * (z < 0. ? 1. : low) / (1. + low);                    // (sigmoid(z) is 1 / (1 + low), or low times that)
        if (e != 0.) slope += e * beta;
    }
    if (a.loss) a.loss[pair] = (float)loss;
    if (a.sums) {
        a.sums[2 * pair] = (float)sum[0];
        a.sums[2 * pair + 1] = (float)sum[1];
    }
    if (a.status) a.status[pair] = bad || astray ? EBSP_STATUS_RANGE : EBSP_STATUS_OK;
    float* out = a.d.stats + (a.d.N + pair) * 3;
    out[0] = astray ? 0.f : (float)(slope * share[0]);
    out[1] = astray ? 0.f : (float)(-slope * share[1]);
    if (pair >= slices) out[2] = 0.f;
}

}  // namespace
