// Distillation from a teacher's top logits: the loss of every row, and its gradient.
// Part of the ZipLine library (see training.hip); device code for gfx950.
//
// Per row, with the teacher's entries (i_k, t_k), the student's logits s and a temperature T:
//     q = softmax(t / T) over the entries     p = softmax(s / T)     p1 = softmax(s)
//     loss = kl T^2 sum_k q_k (log q_k - log p_{i_k}) - ce log p1_label
//     d loss / d s_j = kl T (p_j - sum_{k: i_k = j} q_k) + ce (p1_j - [j = label])
// Exponentials are taken to base 2.  A row's statistics are its largest logit m and the sums of 2^((s - m) c) for c = log2(e) / T
// and log2(e), kept apart (not as m + log of the sum), so a row of the type's lowest values is as good as any other.  m starts
// from the lowest finite value: logits of -inf then weigh nothing without a case of their own.
#pragma once
#include "ebsp_training.h"
#include "tr_common.h"

namespace {

constexpr int TOP_MAX = 1024;                    // most entries of a row: they lie in shared memory
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

struct Distill {
    const void* logits;
    i64 ld, N, V;
    const void* top_index;                       // [N][ldt], 32 or 64 bits
    const void* top_logit;                       // [N][ldt]
    i64 ldt;
    const i64* labels;                           // NULL: no second term
    const float* dloss;                          // the rows' weights in the gradient
    float* loss;
    float* stats;                                // [N][3]: m, log2 of the two sums
    int* status;
    void* grad;
    i64 ldd;
    float* partial;                              // [N][splits][3]: m and the two sums of a part of a row
    int top, top_type, index_wide, splits;
    float temperature, kl, ce;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

struct Sums {
    float m, st, s1;
};

__device__ __forceinline__ Sums joined(Sums a, Sums b, float ct)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = a.m - r.m, db = b.m - r.m;
    r.st = a.st * exp2_fast(da * ct) + b.st * exp2_fast(db * ct);
    r.s1 = a.s1 * exp2_fast(da * LOG2E) + b.s1 * exp2_fast(db * LOG2E);
    return r;
}

// Values that every thread of a workgroup has, over all of them, in an order that depends on nothing but NT.
template <int NT, class T, class F>
__device__ __forceinline__ T block_reduce(T v, T* shared, F&& join)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        T o;
        const float* in = reinterpret_cast<const float*>(&v);
        float* out = reinterpret_cast<float*>(&o);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 4); ++i) out[i] = __shfl_xor(in[i], d);
        v = join(v, o);
    }
    if constexpr (NT > WAVE) {
        __syncthreads();                                                     // the last reduction's readers are through
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
        __syncthreads();
        v = shared[0];
#pragma unroll
        for (int w = 1; w < NT / WAVE; ++w) v = join(v, shared[w]);
    }
    return v;
}

constexpr int SEEN_BITS = 15, TWICE_MAX = 32;

// A row's entries in shared memory.
struct alignas(16) Entries {
    u32 seen[1 << (SEEN_BITS - 5)];              // a bit for every value of an index' hash
    int twice[TWICE_MAX];                        // indices that found their bit set
    int twice_count, label_taken;
    int index[TOP_MAX];                          // -1: padding
    float q[TOP_MAX], s[TOP_MAX];                // the teacher's logit, later its weight; the student's logit
    Sums sums[16];
    float scalar[16];
};

struct Row {
    i64 n;
    int label;                                   // -1: none
    bool any;                                    // some entry has weight
    float label_logit;
};

template <class T>
__device__ __forceinline__ float top_logit(const Distill& d, i64 at)
{
    return d.top_type == EBSP_F32 ? ((const float*)d.top_logit)[at]
         : d.top_type == EBSP_F16 ? to_float(((const _Float16*)d.top_logit)[at]) : to_float(((const __bf16*)d.top_logit)[at]);
}

// The larger of two, or the one that is no number: a NaN among a row's entries comes through, its results are not those of the others.
__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }

// Entries and label of row n, checked: what does not lie in the vocabulary is left out and counted as bad.  The student's logits are
// fetched for those from `v0` up to `v1`.  Each thread keeps to its own entries until the next barrier; `top` is the largest of them.
template <int NT, class T>
__device__ __forceinline__ Row read_entries(const Distill& d, i64 n, i64 v0, i64 v1, Entries& e, float& top, bool& bad)
{
    Row row;
    row.n = n;
    bad = false;
    top = -INFINITY;
    const T* s = (const T*)d.logits + n * d.ld;
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const i64 at = n * d.ldt + k;
        const i64 i = d.index_wide ? ((const i64*)d.top_index)[at] : (i64)((const int*)d.top_index)[at];
        const bool in = i >= 0 && i < d.V;
        bad |= i >= d.V;
        const float t = in ? top_logit<T>(d, at) : -INFINITY;
        e.index[k] = in ? (int)i : -1;
        e.q[k] = t;
        e.s[k] = in && i >= v0 && i < v1 ? to_float(s[i]) : 0.f;
        top = larger(t, top);
    }
    row.label = -1;
    if (d.labels) {
        const i64 l = d.labels[n];
        bad |= l >= d.V;
        if (l >= 0 && l < d.V && d.ce != 0.f) row.label = (int)l;
    }
    row.label_logit = row.label >= v0 && row.label < v1 ? to_float(s[row.label]) : 0.f;
    return row;
}

// The entries' weights, not yet divided by their sum, which is returned for the thread's own.
template <int NT>
__device__ __forceinline__ float weigh_entries(const Distill& d, const Row& row, Entries& e, float top)
{
    float sum = 0.f;
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const float w = row.any && e.index[k] >= 0 ? exp2_fast((e.q[k] - top) * (LOG2E / d.temperature)) : 0.f;
        e.q[k] = w;
        sum += w;
    }
    return sum;
}

template <int NT>
__device__ __forceinline__ void share_entries(const Distill& d, const Row& row, Entries& e, float sum)
{
    const float inv = row.any ? 1.f / sum : 0.f;
    for (int k = threadIdx.x; k < d.top; k += NT) e.q[k] *= inv;
}

__device__ __forceinline__ bool has_entries(const Distill& d, float top) { return top != -INFINITY && d.kl != 0.f; }

// All of it for kernels that take a row's sums from elsewhere.
template <int NT, class T>
__device__ __forceinline__ Row read_row(const Distill& d, i64 n, i64 v0, i64 v1, Entries& e, bool flag)
{
    struct Found { float top, bad; };
    bool bad;
    float top;
    Row row = read_entries<NT, T>(d, n, v0, v1, e, top, bad);
    const Found f = block_reduce<NT>(Found{top, bad ? 1.f : 0.f}, reinterpret_cast<Found*>(e.sums),
                                     [](Found a, Found b) { return Found{larger(a.top, b.top), fmaxf(a.bad, b.bad)}; });
    if (flag && threadIdx.x == 0 && d.status) d.status[n] = f.bad > 0.f ? EBSP_STATUS_RANGE : EBSP_STATUS_OK;
    row.any = has_entries(d, f.top);
    const float sum = block_reduce<NT>(weigh_entries<NT>(d, row, e, f.top), e.scalar, [](float a, float b) { return a + b; });
    share_entries<NT>(d, row, e, sum);
    __syncthreads();
    return row;
}

// log2 of a sum, for differences from m; of a row without any finite logit it is taken as 0, so its p are 0.
__device__ __forceinline__ float log2_sum(float s) { return s == 0.f ? 0.f : log2f(s); }

// The row's loss, from its statistics.  A logit's distance from the largest is not multiplied before its weight is: at a place masked with the lowest
// value of bf16 or fp32 the loss is a number of that size, and log2(e) times it, or a sum of several, would be none.
template <int NT, class T>
__device__ __forceinline__ float row_loss(const Distill& d, const Row& row, Entries& e, float m, float lt, float l1)
{
    const float unit = LN2 * d.temperature, weight = d.kl * d.temperature;
    float sum = 0.f;                                                         // weight * T sum_k q_k (log q_k - log p), weighted term by term
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const float q = e.q[k];
        if (q == 0.f) continue;
        const float s = e.s[k];
        sum += s == -INFINITY ? weight * INFINITY : weight * q * fmaf(unit, log2f(q) + lt, -(s - m));
    }
    sum = block_reduce<NT>(sum, e.scalar, [](float a, float b) { return a + b; });
    float loss = row.any ? sum : 0.f;
    const float s = row.label_logit;
    if (row.label >= 0) loss -= d.ce * (s == -INFINITY ? s : (s - m) - LN2 * l1);
    return loss;
}

// p1 beside p: not wanted or of the same temperature, its square (temperature 2: an exponential takes four times as long as a product),
// or by itself, at any other temperature.  Loss and gradient, us, at temperatures 1 / 2 / 4: 4096 rows of 128000 in bf16 472 / 479 / 501, of 32000 122 / 121 / 124,
// 2048 of 128000 in fp32 465 / 478 / 491.
enum Second { ONE, SQUARE, APART };

__host__ __device__ __forceinline__ Second second_of(const Distill& d)
{
    return !d.labels || d.ce == 0.f || d.temperature == 1.f ? ONE : d.temperature == 2.f ? SQUARE : APART;
}

// A row's gradient away from its entries and label: a p + b p1, and what it takes.  A term whose factor is 0 is left out, whatever the logits.
struct Slope {
    float m, ct, lt, l1, a, b;
    float c;                                     // b p1 = c p^T where p1 is p or its square
    int how;                                     // -1: nothing; 0: p alone; 1: p1 alone; 2: both
};

__device__ __forceinline__ Slope slope_of(const Distill& d, const Row& row, float m, float lt, float l1)
{
    const float w = d.dloss[row.n];
    Slope g = {m, LOG2E / d.temperature, lt, l1, row.any ? w * d.kl * d.temperature : 0.f, row.label >= 0 ? w * d.ce : 0.f, 0.f, -1};
    if (g.a != 0.f) g.how = 0;
    if (g.b != 0.f) g.how = g.a != 0.f ? 2 : 1;
    g.c = g.how == 2 ? g.b * exp2_fast(d.temperature * lt - l1) : 0.f;
    return g;
}

template <Second S, int HOW>
__device__ __forceinline__ float slope_at(const Slope& g, float s)
{
    const float x = s - g.m;
    if constexpr (HOW == 0) return g.a * exp2_fast(x * g.ct - g.lt);
    if constexpr (HOW == 1) return g.b * exp2_fast(x * LOG2E - g.l1);
    const float p = exp2_fast(x * g.ct - g.lt);
    if constexpr (S == APART) return g.a * p + g.b * exp2_fast(x * LOG2E - g.l1);
    if constexpr (S == SQUARE) return p * fmaf(g.c, p, g.a);
    return (g.a + g.c) * p;
}

template <class T, Second S>
__device__ __forceinline__ Word4 slope_word(const Slope& g, Word4 raw)
{
    Pack<T> w;
    w.raw = raw;
    auto each = [&](auto&& f) {
#pragma unroll
        for (int i = 0; i < PER_WORD4<T>; ++i) w.v[i] = from_float<T>(f(to_float(w.v[i])));
    };
    if (g.how == 2) each([&](float s) { return slope_at<S, 2>(g, s); });
    else if (g.how == 0) each([&](float s) { return slope_at<S, 0>(g, s); });
    else if (g.how == 1) each([&](float s) { return slope_at<S, 1>(g, s); });
    else each([](float) { return 0.f; });
    return w.raw;
}

// Which indices stand in a row more than once, for write_places: all but the first that sets a hash's bit are listed, and with them
// a few whose hash is another's.  A barrier lies between the two steps, and another before the list is used.
template <int NT>
__device__ __forceinline__ void clear_places(Entries& e)
{
    for (int w = threadIdx.x; w < (1 << (SEEN_BITS - 7)); w += NT) reinterpret_cast<Word4*>(e.seen)[w] = Word4{0, 0, 0, 0};
    if (threadIdx.x == 0) e.twice_count = e.label_taken = 0;
}

template <int NT>
__device__ __forceinline__ void mark_places(const Distill& d, const Row& row, Entries& e)
{
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const int i = e.index[k];
        if (i < 0) continue;
        const u32 h = ((u32)i * 2654435761u) >> (32 - SEEN_BITS), bit = 1u << (h & 31);
        if (atomicOr(&e.seen[h >> 5], bit) & bit) {
            const int at = atomicAdd(&e.twice_count, 1);
            if (at < TWICE_MAX) e.twice[at] = i;
        }
        if (i == row.label) e.label_taken = 1;
    }
}

// The places of the entries and of the label, whose gradients have further terms, written over what stands there.  Entries of
// one index add up, in the order of k, and all write the same value; an entry at the label's place writes for both.  (Looking through all entries
// for those of the same index took 38 of 57 us for 4096 rows of 1000 with 256 entries, 156 of 176 for 512 of 8000 with 1000.)
template <int NT, class T, Second S>
__device__ __forceinline__ void write_places(const Distill& d, const Row& row, const Entries& e, i64 v0, i64 v1, const Slope& g)
{
    if (g.how < 0) return;
    T* grad = (T*)d.grad + row.n * d.ldd;
    const int listed = e.twice_count;
    for (int k = threadIdx.x; k <= d.top; k += NT) {
        const bool own = k == d.top;                                         // the label's turn
        const int i = own ? row.label : e.index[k];
        if (i < v0 || i >= v1) continue;
        if (own && e.label_taken) continue;
        bool others = listed > TWICE_MAX;
        for (int j = 0; j < min(listed, TWICE_MAX); ++j) others |= e.twice[j] == i;
        float q = own ? 0.f : e.q[k];
        if (others && !own) {
            q = 0.f;
            for (int j = 0; j < d.top; ++j) q += e.index[j] == i ? e.q[j] : 0.f;
        }
        const float s = own ? row.label_logit : e.s[k];
        float x = g.how == 2 ? slope_at<S, 2>(g, s) : g.how == 0 ? slope_at<S, 0>(g, s) : slope_at<S, 1>(g, s);
        if (g.a != 0.f) x -= g.a * q;
        if (i == row.label) x -= g.b;
        grad[i] = from_float<T>(x);
    }
}

template <class T>
__device__ __forceinline__ Word4 lowest_word()
{
    Pack<T> w;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) w.v[i] = (T)-INFINITY;
    return w.raw;
}

// 16 bytes of a row from element v on; -inf behind its end.  The word that passes the end is read from where it fits and moved: element
// by element its one lane would hold up the row.
template <class T>
__device__ __forceinline__ Word4 read_logits(const T* s, i64 v, i64 end)
{
    constexpr int N = PER_WORD4<T>;
    if (v + N <= end) return load_loose(s + v);
    Pack<T> w;
    if (end >= N) {
        w.raw = load_loose(s + end - N);
        for (i64 moves = v + N - end; moves > 0; --moves) {
#pragma unroll
            for (int i = 0; i < N - 1; ++i) w.v[i] = w.v[i + 1];
            w.v[N - 1] = (T)-INFINITY;
        }
    } else {
        w.raw = lowest_word<T>();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (v + i < end) w.v[i] = s[v + i];
    }
    return w.raw;
}

// The sums of a word's exponentials, from a maximum that stands.
template <class T, Second S>
__device__ __forceinline__ void add_exponentials(Sums& s, Word4 raw, float m, float ct)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) {
        const float x = to_float(w.v[i]) - m, e = exp2_fast(x * ct);
        s.st += e;
        if constexpr (S == SQUARE) s.s1 = fmaf(e, e, s.s1);
        if constexpr (S == APART) s.s1 += exp2_fast(x * LOG2E);
    }
}

template <class T>
__device__ __forceinline__ float largest(Word4 raw, float m)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) m = fmaxf(m, to_float(w.v[i]));
    return m;
}

// A word more, whose values may pass the maximum so far.
template <class T, Second S>
__device__ __forceinline__ void add_word(Sums& s, Word4 raw, float ct)
{
    const float high = largest<T>(raw, s.m);
    if (high > s.m) {
        s.st *= exp2_fast((s.m - high) * ct);
        s.s1 *= exp2_fast((s.m - high) * LOG2E);
        s.m = high;
    }
    add_exponentials<T, S>(s, raw, s.m, ct);
}

template <class T>
__device__ __forceinline__ void write_gradient(T* g, i64 v, i64 end, Word4 raw)
{
    constexpr int N = PER_WORD4<T>;
    if (v + N <= end) {
        store_loose(g + v, raw);
        return;
    }
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (v + i < end) g[v + i] = w.v[i];
}

template <int NT, class T, Second S>
__device__ __forceinline__ Sums part_sums(const Distill& d, const T* s, i64 v0, i64 v1)
{
    constexpr int N = PER_WORD4<T>, AHEAD = 4;
    const float ct = LOG2E / d.temperature;
    Sums sums = {-FLT_MAX, 0.f, 0.f};
    i64 v = v0 + (i64)threadIdx.x * N;
    for (; v + (AHEAD - 1) * NT * N + N <= v1; v += AHEAD * NT * N) {
        Word4 w[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) w[j] = load_loose(s + v + j * NT * N);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) add_word<T, S>(sums, w[j], ct);
    }
    for (; v < v1; v += NT * N) add_word<T, S>(sums, read_logits(s, v, v1), ct);
    return sums;
}

// The launch's choice of S, as a type for the kernels' bodies.
template <Second S> struct SecondTag { static constexpr Second value = S; };
template <class F>
__device__ __forceinline__ void with_second(const Distill& d, F&& f)
{
    switch (second_of(d)) {
    case ONE: f(SecondTag<ONE>()); break;
    case SQUARE: f(SecondTag<SQUARE>()); break;
    default: f(SecondTag<APART>());
    }
}

__device__ __forceinline__ void write_loss(const Distill& d, i64 n, float loss, float m, float lt, float l1)
{
    if (threadIdx.x) return;
    d.loss[n] = loss;
    if (d.stats) {
        d.stats[n * 3] = m;
        d.stats[n * 3 + 1] = lt;
        d.stats[n * 3 + 2] = l1;
    }
}

// Packed words stay packed: without this the compiler keeps the floats of one use for the next, twice the registers.
template <int N>
__device__ __forceinline__ void forget_floats(Word4 (&w)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(w[j]));
}

// Loss and statistics, and with GRAD the gradient too: one workgroup a row.  The row's first NT x HELD words stay in registers from the one load to
// the gradient, more of a long one in shared memory; only what lies behind is read twice.  A workgroup does one thing at a time, so a CU needs several to keep memory busy while
// one of them computes: rows that fill a CU's registers are cut at half (4096 rows of 128000, bf16: 483 us, 4.3 TB/s, where one workgroup held
// the whole row 597; with nothing in shared memory 487, and 2048 rows of 128000 in fp32 512 where it is 483 now).
template <int NT, class T, bool GRAD, Second S>
__global__ void __launch_bounds__(NT) tr_distill_row_kernel(Distill d)
{
    constexpr int N = PER_WORD4<T>, HELD = 16, KEPT = !GRAD ? 0 : NT == 512 ? 7 : NT == 1024 ? 8 : 0;
    constexpr u32 STEP = NT * N, BEHIND = (HELD + KEPT) * STEP;
    __shared__ Entries e;
    __shared__ Word4 kept[KEPT > 0 ? KEPT * NT : 1];
    const i64 n = blockIdx.x;
    const T* s = (const T*)d.logits + n * d.ld;
    const float ct = LOG2E / d.temperature;
    Sums rest = {-FLT_MAX, 0.f, 0.f};
    if (BEHIND < d.V) rest = part_sums<NT, T, S>(d, s, BEHIND, d.V);
    float kept_m = -FLT_MAX;
    if constexpr (KEPT > 0) {
        if (HELD * STEP < d.V) {
            Word4 w[KEPT];
#pragma unroll
            for (int j = 0; j < KEPT; ++j) {
                const u32 v = threadIdx.x * N + (HELD + j) * STEP;
                w[j] = v < d.V ? read_logits(s, v, d.V) : lowest_word<T>();
            }
#pragma unroll
            for (int j = 0; j < KEPT; ++j) {
                kept[j * NT + threadIdx.x] = w[j];
                kept_m = largest<T>(w[j], kept_m);
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);                                       // (before the registers fill)
    // A word belongs to the row as a whole, or is the part that is left, which one thread has besides.
    const u32 v0 = threadIdx.x * N, whole = (u32)(d.V / N * N), end = min(whole, HELD * STEP);
    const bool has_last = whole < (u32)d.V && whole < HELD * STEP && whole % STEP == v0;
    Word4 held[HELD];
#pragma unroll
    for (int j = 0; j < HELD; ++j) held[j] = v0 + j * STEP < end ? load_loose(s + j * STEP + v0) : lowest_word<T>();
    Word4 last = lowest_word<T>();
    if (has_last) last = read_logits(s, whole, d.V);
    float top;
    bool bad;
    if constexpr (GRAD) clear_places<NT>(e);
    Row row = read_entries<NT, T>(d, n, 0, d.V, e, top, bad);
    struct Found { float top, bad, m; };
    Found f = {top, bad ? 1.f : 0.f, fmaxf(rest.m, kept_m)};
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (j * STEP < end) {
            f.m = largest<T>(held[j], f.m);
            __builtin_amdgcn_sched_barrier(0);                               // word by word: the registers are full
        }
    if (has_last) f.m = largest<T>(last, f.m);
    forget_floats(held);
    f = block_reduce<NT>(f, reinterpret_cast<Found*>(e.sums),
                         [](Found a, Found b) { return Found{larger(a.top, b.top), fmaxf(a.bad, b.bad), fmaxf(a.m, b.m)}; });
    if (threadIdx.x == 0 && d.status) d.status[n] = f.bad > 0.f ? EBSP_STATUS_RANGE : EBSP_STATUS_OK;
    row.any = has_entries(d, f.top);
    if constexpr (GRAD) mark_places<NT>(d, row, e);
    Sums sums = joined(rest, Sums{f.m, 0.f, 0.f}, ct);                       // (f.m is the larger)
#pragma unroll
    for (int j = 0; j < HELD; ++j)
        if (j * STEP < end) {
            add_exponentials<T, S>(sums, held[j], f.m, ct);
            __builtin_amdgcn_sched_barrier(0);
        }
    if (has_last) add_exponentials<T, S>(sums, last, f.m, ct);
    if constexpr (KEPT > 0)
#pragma unroll 1
        for (int j = 0; j < KEPT && (HELD + j) * STEP < d.V; ++j) add_exponentials<T, S>(sums, kept[j * NT + threadIdx.x], f.m, ct);
    struct Totals { float q, st, s1; };
    Totals t = {weigh_entries<NT>(d, row, e, f.top), sums.st, sums.s1};
    t = block_reduce<NT>(t, reinterpret_cast<Totals*>(e.sums), [](Totals a, Totals b) { return Totals{a.q + b.q, a.st + b.st, a.s1 + b.s1}; });
    if constexpr (S == ONE) t.s1 = t.st;                                     // (read where the temperature is 1)
    share_entries<NT>(d, row, e, t.q);
    const float m = f.m, lt = log2_sum(t.st), l1 = log2_sum(t.s1);
    write_loss(d, n, row_loss<NT, T>(d, row, e, m, lt, l1), m, lt, l1);
    if constexpr (GRAD) {
        const Slope g = slope_of(d, row, m, lt, l1);
        T* out = (T*)d.grad + n * d.ldd;
        forget_floats(held);
        __builtin_amdgcn_s_waitcnt(0);                                       // in place: the logits of the places have been read
        __syncthreads();
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            if (v0 + j * STEP < end) store_loose(out + j * STEP + v0, slope_word<T, S>(g, held[j]));
            __builtin_amdgcn_sched_barrier(0);
        }
        if (has_last) write_gradient(out, whole, d.V, slope_word<T, S>(g, last));
        if constexpr (KEPT > 0)
#pragma unroll 1
            for (int j = 0; j < KEPT; ++j) {
                const u32 v = v0 + (HELD + j) * STEP;
                if (v < d.V) write_gradient(out, v, d.V, slope_word<T, S>(g, kept[j * NT + threadIdx.x]));
            }
        for (i64 v = v0 + BEHIND; v < d.V; v += STEP) write_gradient(out, v, d.V, slope_word<T, S>(g, read_logits(s, v, d.V)));
        __builtin_amdgcn_s_waitcnt(0);                                       // stores to one address arrive in this order
        __syncthreads();
        write_places<NT, T, S>(d, row, e, 0, d.V, g);
    }
}

__device__ __forceinline__ void part_range(const Distill& d, int part, int per_word, i64& v0, i64& v1)
{
    const i64 words = (d.V + per_word - 1) / per_word, each = (words + d.splits - 1) / d.splits;
    v0 = min(part * each * per_word, d.V);
    v1 = min(v0 + each * per_word, d.V);
}

// Few rows: the sums of a part of a row by each workgroup ...
template <int NT, class T>
__global__ void __launch_bounds__(NT) tr_distill_part_kernel(Distill d)
{
    __shared__ Sums shared[16];
    const i64 n = blockIdx.x / d.splits;
    const int part = blockIdx.x % d.splits;
    const float ct = LOG2E / d.temperature;
    i64 v0, v1;
    part_range(d, part, PER_WORD4<T>, v0, v1);
    Sums sums;
    with_second(d, [&](auto s) { sums = part_sums<NT, T, decltype(s)::value>(d, (const T*)d.logits + n * d.ld, v0, v1); });
    sums = block_reduce<NT>(sums, shared, [ct](Sums x, Sums y) { return joined(x, y, ct); });
    if (threadIdx.x == 0) {
        float* out = d.partial + (n * d.splits + part) * 3;
        out[0] = sums.m;
        out[1] = sums.st;
        out[2] = sums.s1;
    }
}

// ... joined by one a row, in the order of the parts.
template <int NT, class T>
__global__ void __launch_bounds__(NT) tr_distill_join_kernel(Distill d)
{
    __shared__ Entries e;
    const i64 n = blockIdx.x;
    const Row row = read_row<NT, T>(d, n, 0, d.V, e, true);
    const float ct = LOG2E / d.temperature;
    Sums sums = {-FLT_MAX, 0.f, 0.f};
    for (int p = threadIdx.x; p < d.splits; p += NT) {
        const float* in = d.partial + (n * d.splits + p) * 3;
        sums = joined(sums, Sums{in[0], in[1], in[2]}, ct);
    }
    sums = block_reduce<NT>(sums, e.sums, [ct](Sums x, Sums y) { return joined(x, y, ct); });
    if (second_of(d) == ONE) sums.s1 = sums.st;                 // (read where the temperature is 1)
    const float lt = log2_sum(sums.st), l1 = log2_sum(sums.s1);
    write_loss(d, n, row_loss<NT, T>(d, row, e, sums.m, lt, l1), sums.m, lt, l1);
}

// The gradient from statistics: every row in `splits` parts.
template <int NT, class T>
__global__ void __launch_bounds__(NT) tr_distill_gradient_kernel(Distill d)
{
    __shared__ Entries e;
    constexpr int N = PER_WORD4<T>;
    const i64 n = blockIdx.x / d.splits;
    i64 v0, v1;
    part_range(d, blockIdx.x % d.splits, N, v0, v1);
    const T* s = (const T*)d.logits + n * d.ld;
    clear_places<NT>(e);
    const Row row = read_row<NT, T>(d, n, v0, v1, e, false);
    mark_places<NT>(d, row, e);                                              // (read_row has barriers)
    const Slope g = slope_of(d, row, d.stats[n * 3], d.stats[n * 3 + 1], d.stats[n * 3 + 2]);
    T* out = (T*)d.grad + n * d.ldd;
    __builtin_amdgcn_s_waitcnt(0);                                           // in place: the logits of the places have been read
    __syncthreads();
    with_second(d, [&](auto second) {
        constexpr Second S = decltype(second)::value;
        for (i64 v = v0 + (i64)threadIdx.x * N; v < v1; v += NT * N) write_gradient(out, v, v1, slope_word<T, S>(g, read_logits(s, v, v1)));
        __builtin_amdgcn_s_waitcnt(0);                                       // stores to one address arrive in this order
        __syncthreads();
        write_places<NT, T, S>(d, row, e, v0, v1, g);
    });
}

}  // namespace
