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

// A row's entries in shared memory.
struct Entries {
    int index[TOP_MAX];                          // -1: padding
    float q[TOP_MAX], s[TOP_MAX];                // the teacher's weight, the student's logit
    Sums sums[16];
    float scalar[16];
};

struct Row {
    i64 n;
    int label;                                   // -1: none
    bool any;                                    // some entry has weight
};

template <class T>
__device__ __forceinline__ float top_logit(const Distill& d, i64 at)
{
    return d.top_type == EBSP_F32 ? ((const float*)d.top_logit)[at]
         : d.top_type == EBSP_F16 ? to_float(((const _Float16*)d.top_logit)[at]) : to_float(((const __bf16*)d.top_logit)[at]);
}

// Entries and label of row n, checked: what does not lie in the vocabulary is left out and flagged.  The student's logits are
// fetched for those from `v0` up to `v1`.
template <int NT, class T>
__device__ __forceinline__ Row read_row(const Distill& d, i64 n, i64 v0, i64 v1, Entries& e, bool flag)
{
    Row row;
    row.n = n;
    bool bad = false;
    const float ct = LOG2E / d.temperature;
    const T* s = (const T*)d.logits + n * d.ld;
    float tm = -INFINITY;
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const i64 at = n * d.ldt + k;
        const i64 i = d.index_wide ? ((const i64*)d.top_index)[at] : (i64)((const int*)d.top_index)[at];
        const bool in = i >= 0 && i < d.V;
        bad |= i >= d.V;
        const float t = in ? top_logit<T>(d, at) : -INFINITY;
        e.index[k] = in ? (int)i : -1;
        e.q[k] = t;
        e.s[k] = in && i >= v0 && i < v1 ? to_float(s[i]) : 0.f;
        tm = t > tm || t != t ? t : tm;
    }
    row.label = -1;
    if (d.labels) {
        const i64 l = d.labels[n];
        bad |= l >= d.V;
        if (l >= 0 && l < d.V && d.ce != 0.f) row.label = (int)l;
    }
    if (flag) {
        const float any_bad = block_reduce<NT>(bad ? 1.f : 0.f, e.scalar, [](float a, float b) { return fmaxf(a, b); });
        if (threadIdx.x == 0 && d.status) d.status[n] = any_bad > 0.f ? EBSP_STATUS_RANGE : EBSP_STATUS_OK;
    }
    // a NaN among the entries comes through: the row's results are NaN, not those of the other entries
    tm = block_reduce<NT>(tm, e.scalar, [](float a, float b) { return a > b || a != a ? a : b; });
    row.any = tm != -INFINITY && d.kl != 0.f;
    float sum = 0.f;
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const float w = row.any && e.index[k] >= 0 ? exp2_fast((e.q[k] - tm) * ct) : 0.f;
        e.q[k] = w;
        sum += w;
    }
    sum = block_reduce<NT>(sum, e.scalar, [](float a, float b) { return a + b; });
    const float inv = row.any ? 1.f / sum : 0.f;
    for (int k = threadIdx.x; k < d.top; k += NT) e.q[k] *= inv;
    __syncthreads();
    return row;
}

// log2 of a sum, for differences from m; of a row without any finite logit it is taken as 0, so its p are 0.
__device__ __forceinline__ float log2_sum(float s) { return s == 0.f ? 0.f : log2f(s); }

// The row's loss, from its statistics.
template <int NT, class T>
__device__ __forceinline__ float row_loss(const Distill& d, const Row& row, Entries& e, float m, float lt, float l1, float label_logit)
{
    const float ct = LOG2E / d.temperature;
    float sum = 0.f;
    for (int k = threadIdx.x; k < d.top; k += NT) {
        const float q = e.q[k];
        if (q == 0.f) continue;
        const float s = e.s[k];
        const float logp = s == -INFINITY ? s : (s - m) * ct - lt;
        sum += q * (log2f(q) - logp);
    }
    sum = block_reduce<NT>(sum, e.scalar, [](float a, float b) { return a + b; });
    float loss = row.any ? d.kl * d.temperature * d.temperature * (LN2 * sum) : 0.f;
    if (row.label >= 0) loss -= d.ce * (label_logit == -INFINITY ? label_logit : LN2 * ((label_logit - m) * LOG2E - l1));
    return loss;
}

// The factors of p and p1 in a row's gradient; 0 where the row has no such term.
__device__ __forceinline__ void row_factors(const Distill& d, const Row& row, float& a, float& b)
{
    const float w = d.dloss[row.n];
    a = row.any ? w * d.kl * d.temperature : 0.f;
    b = row.label >= 0 ? w * d.ce : 0.f;
}

__device__ __forceinline__ float gradient(float s, float m, float ct, float lt, float l1, float a, float b)
{
    const float x = s - m;
    float g = 0.f;
    if (a != 0.f) g = a * exp2_fast(x * ct - lt);
    if (b != 0.f) g += b * exp2_fast(x * LOG2E - l1);
    return g;
}

// The places of the entries and of the label, whose gradients have further terms, written over what stands there.  Entries of
// one index add up, in the order of k, and all write the same value.
template <int NT, class T>
__device__ __forceinline__ void write_places(const Distill& d, const Row& row, const Entries& e, i64 v0, i64 v1, float m, float lt, float l1,
                                             float a, float b, float label_logit)
{
    if (a == 0.f && b == 0.f) return;
    const float ct = LOG2E / d.temperature;
    T* grad = (T*)d.grad + row.n * d.ldd;
    for (int k = threadIdx.x; k <= d.top; k += NT) {
        const bool own = k == d.top;                                         // the label's turn
        const int i = own ? row.label : e.index[k];
        if (i < v0 || i >= v1) continue;
        float q = 0.f;
        for (int j = 0; j < d.top; ++j) q += e.index[j] == i ? e.q[j] : 0.f;
        float g = gradient(own ? label_logit : e.s[k], m, ct, lt, l1, a, b) - a * q;
        if (i == row.label) g -= b;
        grad[i] = from_float<T>(g);
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

// 16 bytes of a row from element v on; -inf behind its end.
template <class T>
__device__ __forceinline__ Word4 read_logits(const T* s, i64 v, i64 end)
{
    constexpr int N = PER_WORD4<T>;
    if (v + N <= end) return load_loose(s + v);
    Pack<T> w;
    w.raw = lowest_word<T>();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (v + i < end) w.v[i] = s[v + i];
    return w.raw;
}

template <class T>
__device__ __forceinline__ void add_word(Sums& s, Word4 raw, float ct, bool two)
{
    constexpr int N = PER_WORD4<T>;
    Pack<T> w;
    w.raw = raw;
    float x[N], high = s.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = to_float(w.v[i]);
        high = fmaxf(high, x[i]);
    }
    if (high > s.m) {
        s.st *= exp2_fast((s.m - high) * ct);
        s.s1 *= exp2_fast((s.m - high) * LOG2E);
        s.m = high;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s.st += exp2_fast((x[i] - s.m) * ct);
    if (two)
#pragma unroll
        for (int i = 0; i < N; ++i) s.s1 += exp2_fast((x[i] - s.m) * LOG2E);
}

template <class T>
__device__ __forceinline__ Word4 gradient_word(Word4 raw, float m, float ct, float lt, float l1, float a, float b)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) w.v[i] = from_float<T>(gradient(to_float(w.v[i]), m, ct, lt, l1, a, b));
    return w.raw;
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

// Whether p1 is needed beside p: at T = 1 they are one.
__device__ __forceinline__ bool two_sums(const Distill& d) { return d.labels && d.temperature != 1.f; }

template <int NT, class T>
__device__ __forceinline__ Sums part_sums(const Distill& d, const T* s, i64 v0, i64 v1, Sums* shared)
{
    constexpr int N = PER_WORD4<T>;
    const float ct = LOG2E / d.temperature;
    const bool two = two_sums(d);
    Sums sums = {-FLT_MAX, 0.f, 0.f};
    for (i64 v = v0 + (i64)threadIdx.x * N; v < v1; v += NT * N) add_word<T>(sums, read_logits(s, v, v1), ct, two);
    sums = block_reduce<NT>(sums, shared, [ct](Sums x, Sums y) { return joined(x, y, ct); });
    if (!two) sums.s1 = sums.st;                                             // (only read where T is 1)
    return sums;
}

// Loss and statistics, and with GRAD the gradient too: one workgroup a row.
template <int NT, class T, bool GRAD>
__global__ void __launch_bounds__(NT) tr_distill_row_kernel(Distill d)
{
    __shared__ Entries e;
    constexpr int N = PER_WORD4<T>;
    const i64 n = blockIdx.x;
    const T* s = (const T*)d.logits + n * d.ld;
    const Row row = read_row<NT, T>(d, n, 0, d.V, e, true);
    const float label_logit = row.label >= 0 ? to_float(s[row.label]) : 0.f;
    const Sums sums = part_sums<NT, T>(d, s, 0, d.V, e.sums);
    const float lt = log2_sum(sums.st), l1 = log2_sum(sums.s1), ct = LOG2E / d.temperature;
    const float loss = row_loss<NT, T>(d, row, e, sums.m, lt, l1, label_logit);
    if (threadIdx.x == 0) {
        d.loss[n] = loss;
        if (d.stats) {
            d.stats[n * 3] = sums.m;
            d.stats[n * 3 + 1] = lt;
            d.stats[n * 3 + 2] = l1;
        }
    }
    if constexpr (GRAD) {
        float a, b;
        row_factors(d, row, a, b);
        T* g = (T*)d.grad + n * d.ldd;
        __builtin_amdgcn_s_waitcnt(0);                                       // in place: the logits of the places have been read
        __syncthreads();
        for (i64 v = (i64)threadIdx.x * N; v < d.V; v += NT * N)
            write_gradient(g, v, d.V, gradient_word<T>(read_logits(s, v, d.V), sums.m, ct, lt, l1, a, b));
        __builtin_amdgcn_s_waitcnt(0);                                       // stores to one address arrive in this order
        __syncthreads();
        write_places<NT, T>(d, row, e, 0, d.V, sums.m, lt, l1, a, b, label_logit);
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
    i64 v0, v1;
    part_range(d, part, PER_WORD4<T>, v0, v1);
    const Sums sums = part_sums<NT, T>(d, (const T*)d.logits + n * d.ld, v0, v1, shared);
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
    const T* s = (const T*)d.logits + n * d.ld;
    const Row row = read_row<NT, T>(d, n, 0, d.V, e, true);
    const float label_logit = row.label >= 0 ? to_float(s[row.label]) : 0.f, ct = LOG2E / d.temperature;
    Sums sums = {-FLT_MAX, 0.f, 0.f};
    for (int p = threadIdx.x; p < d.splits; p += NT) {
        const float* in = d.partial + (n * d.splits + p) * 3;
        sums = joined(sums, Sums{in[0], in[1], in[2]}, ct);
    }
    sums = block_reduce<NT>(sums, e.sums, [ct](Sums x, Sums y) { return joined(x, y, ct); });
    const float lt = log2_sum(sums.st), l1 = log2_sum(sums.s1);
    const float loss = row_loss<NT, T>(d, row, e, sums.m, lt, l1, label_logit);
    if (threadIdx.x == 0) {
        d.loss[n] = loss;
        if (d.stats) {
            d.stats[n * 3] = sums.m;
            d.stats[n * 3 + 1] = lt;
            d.stats[n * 3 + 2] = l1;
        }
    }
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
    const Row row = read_row<NT, T>(d, n, v0, v1, e, false);
    const float label_logit = row.label >= v0 && row.label < v1 ? to_float(s[row.label]) : 0.f, ct = LOG2E / d.temperature;
    const float m = d.stats[n * 3], lt = d.stats[n * 3 + 1], l1 = d.stats[n * 3 + 2];
    float a, b;
    row_factors(d, row, a, b);
    T* g = (T*)d.grad + n * d.ldd;
    __builtin_amdgcn_s_waitcnt(0);                                           // in place: the logits of the places have been read
    __syncthreads();
    for (i64 v = v0 + (i64)threadIdx.x * N; v < v1; v += NT * N)
        write_gradient(g, v, v1, gradient_word<T>(read_logits(s, v, v1), m, ct, lt, l1, a, b));
    __builtin_amdgcn_s_waitcnt(0);                                           // stores to one address arrive in this order
    __syncthreads();
    write_places<NT, T>(d, row, e, v0, v1, m, lt, l1, a, b, label_logit);
}

}  // namespace
