// The residual stream around a block, forward and backward, and dropout by itself.
// Part of the ZipLine library (see tuning.hip); device code for gfx950.
//
// A row x of the stream, a block's output b for it, weights w and w', a gate g, a scale a and kept elements z (0, or 1 / (1 - p)):
//     r' = (mean b^2 + eps)^-1/2     h = b r'       d = h w'  (without a norm behind the block: d = b)
//     y = x + a g z d                r = (mean y^2 + eps)^-1/2        n = y r w
// and from dy and dn, with u = y r and f = a z:
//     dy~ = dy + r (dn w - u mean(dn w u))          dx = dy~        dw = sum over rows of dn u
//     dd = f g dy~       dg = f d dy~               dw' = sum over rows of dd h
//     db = r' (dd w' - h mean(dd w' h))             (without that norm: db = dd)
// The second mean is linear in the first: mean(dd w' h) = mean(q h (dy + r dn w)) - r mean(dn w u) mean(q h u) for q = f g w', so a row's three sums
// are one exchange between its threads.  Sums, r and r' are held in 32 bits; y is rounded once, n comes from y before that.
#pragma once
#include "ebsp_training.h"
#include "tr_random.h"

namespace {

struct Norm {
    const void *x, *branch, *weight, *post_weight, *gate;
    i64 ldx, ldb, ldgate;                        // ldgate 0: one gate for every channel
    i64 M;
    int K;
    float scale, eps;
    Random random;
    void *y, *n;                                 // (in the backward pass y is an input, or x in its place)
    i64 ldy, ldn;
    float* stats;                                // [M][2]: r, r'
    const void *dy, *dn;
    i64 lddy, lddn;
    void *dx, *dbranch, *dgate;
    i64 lddx, lddb, lddgate;
    float* partial;                              // [blocks][sums][8 units]
    void* column_out[3];                         // dw, dw', dg of a channel, those that are wanted
    int blocks, sums, sum_w, sum_post, sum_gate; // places among the sums, -1: not wanted
};

// Eight neighbours of a row, as they lie in memory.
template <class T>
struct Raw8 {
    Word4 w[sizeof(T) / 2];
    __device__ __forceinline__ float operator[](int i) const
    {
        return to_float(reinterpret_cast<const Pack<T>*>(&w[i / PER_WORD4<T>])->v[i % PER_WORD4<T>]);
    }
};

template <class T>
__device__ __forceinline__ Raw8<T> zero8()
{
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = Word4{0, 0, 0, 0};
    return r;
}

// Elements moved down by `by`, 1 to 7; zeros come from above.
__device__ __forceinline__ void move_down(Raw8<float>& r, int by)
{
#pragma unroll
    for (int x = 1; x < 8; x *= 2) {
        const Word4 lo = r.w[0], hi = r.w[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.w[0][i] = by & x ? i + x < 4 ? lo[(i + x) & 3] : hi[(i + x) & 3] : lo[i];
            r.w[1][i] = by & x ? i + x < 4 ? hi[(i + x) & 3] : 0 : hi[i];
        }
    }
}
template <class T>
__device__ __forceinline__ void move_down(Raw8<T>& r, int by)
{
    static_assert(sizeof(T) == 2);
    r.w[0] = __builtin_bit_cast(Word4, __builtin_bit_cast(unsigned __int128, r.w[0]) >> 16 * by);
}

// Element k of a row: 32 bits beside the row's address, which is the same for a wave that has one row.
template <class T>
__device__ __forceinline__ T* element(T* row, int k)
{
    return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(row) + (u32)k * (u32)sizeof(T));
}

// The group of G threads that this one is part of, as a number that the whole wave shares where it does.
template <int G>
__device__ __forceinline__ int group_of()
{
    const int group = threadIdx.x / G;
    return G >= WAVE ? __builtin_amdgcn_readfirstlane(group) : group;
}

// Elements k to k + 7 of a row of K; zeros behind its end.  What passes the end is read from where it fits and moved: so no load stands in a
// branch, where it would wait for those before it.
template <bool LAST = false, class T>
__device__ __forceinline__ Raw8<T> load8(const T* row, int k, int K)
{
    Raw8<T> r;
    if (K < 8) {                                                             // (the same for all)
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = load_some(row + k + j * PER_WORD4<T>, (i64)K - k - j * PER_WORD4<T>);
        return r;
    }
    const T* p = element(row, min(k, K - 8));
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = load_last<LAST>(p + j * PER_WORD4<T>);
    if (k >= K) r = zero8<T>();
    else if (k > K - 8) move_down(r, k - (K - 8));
    return r;
}

template <class T>
__device__ __forceinline__ void forget_words(Raw8<T>& r)
{
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) asm volatile("" : "+v"(r.w[j]));
}

template <bool STREAM = false, class T>
__device__ __forceinline__ void store8(T* row, int k, int K, const float (&v)[8])
{
    Pack<T> w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / PER_WORD4<T>].v[i % PER_WORD4<T>] = from_float<T>(v[i]);
    T* p = element(row, k);
    if (k + 8 <= K) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j)
            if (STREAM) store_stream(p + j * PER_WORD4<T>, w[j].raw);
            else store_loose(p + j * PER_WORD4<T>, w[j].raw);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K) p[i] = w[i / PER_WORD4<T>].v[i % PER_WORD4<T>];
}

// v and the same of the lane that CTRL names, within rows of 16 lanes; no trip through shared memory.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float plus_lane(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}

// The sum over each G neighbouring lanes, for all of them; G up to 32.
template <int G>
__device__ __forceinline__ float row_sum(float v)
{
    if constexpr (G > 1) v = plus_lane<0xB1>(v);                             // lanes 1 0 3 2 of each four
    if constexpr (G > 2) v = plus_lane<0x4E>(v);                             // 2 3 0 1
    if constexpr (G > 4) v = plus_lane<0x141>(v);                            // 7 to 0 of each eight
    if constexpr (G > 8) v = plus_lane<0x140>(v);                            // 15 to 0 of each sixteen
    if constexpr (G > 16) v += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401f));   // the sixteen beside
    return v;
}

__device__ __forceinline__ float from_lane(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

// The sum over a wave, as a number that it shares.
__device__ __forceinline__ float wave_sum(float v)
{
    v = row_sum<16>(v);
    v = plus_lane<0x142, 0xa>(v);                                            // lane 15 of the row before, for rows 1 and 3
    v = plus_lane<0x143, 0xc>(v);                                            // lane 31, for rows 2 and 3
    return from_lane(v, 63);
}

// Sums over the G threads of a row, in an order that G fixes.  One barrier: the buffer of one call is written again in the call after the next,
// which no thread reaches before all have read.
template <int G, int NT, int NV>
__device__ __forceinline__ void group_sum(float (&v)[NV], float* shared, int& turn)
{
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = G >= WAVE ? wave_sum(v[i]) : row_sum<G>(v[i]);
    if constexpr (G > WAVE) {
        constexpr int W = G / WAVE;
        float* buffer = shared + turn * (NT / WAVE * NV);
        turn ^= 1;
        const int wave = threadIdx.x / WAVE;
        if (threadIdx.x % WAVE == 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) buffer[wave * NV + i] = v[i];
        __syncthreads();
        const float* mine = buffer + (wave / W * W + threadIdx.x % W) * NV;  // a wave of the row for each lane
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = from_lane(row_sum<W>(mine[i]), 0);
    }
}

// What a block's output is multiplied by at element i of eight, but for the weight of the norm behind it; 0 where it is dropped.
template <class T>
struct Factor {
    Raw8<T> gate;
    u32 keep;
    float scale;
    bool gated;
    __device__ __forceinline__ bool kept(int i) const { return keep >> i & 1; }
    __device__ __forceinline__ float whole(int i) const { return gated ? scale * gate[i] : scale; }
    __device__ __forceinline__ float operator[](int i) const { return kept(i) ? whole(i) : 0.f; }
};

template <class T>
__device__ __forceinline__ Factor<T> factor_of(const Norm& a, const Generator& g, i64 row, int unit)
{
    Factor<T> f;
    f.gated = a.gate != nullptr;
    f.gate = f.gated ? load8((const T*)a.gate + row * a.ldgate, unit * 8, a.K) : zero8<T>();
    f.keep = 0xffu;
    f.scale = a.scale;
    if (a.random.threshold) {
        f.keep = keep_bits(g, a.random.threshold, (u32)unit, (u32)row);
        f.scale = a.scale * a.random.kept;
    }
    return f;
}

__device__ __forceinline__ float inverse_root(float sum, int K, float eps) { return 1.f / sqrtf(sum / (float)K + eps); }

// The stream at eight elements.
template <class S, class T>
__device__ __forceinline__ void stream8(const Norm& a, const Raw8<S>& x, const Raw8<T>& b, const Raw8<T>& wp, const Factor<T>& f, float rb, float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = x[i];
        if (a.branch) {
            const float d = a.post_weight ? b[i] * rb * wp[i] : b[i];
            if (f.kept(i)) y[i] = fmaf(f[i], d, y[i]);
        }
    }
}

// Forward: G threads a row, U units of eight elements each.  Memory bounds it: 8192 x 4096 in bf16 54 us, 5.0 TB/s.  y is stored past the caches, for the next block comes first; n is what that reads.
template <class S, class T, int G, int U, int NT>
__global__ void __launch_bounds__(NT) tr_norm_forward_kernel(Norm a)
{
    __shared__ float shared[2 * NT / WAVE];
    constexpr int R = NT / G;
    const int lane = threadIdx.x % G;
    const i64 mine = (i64)blockIdx.x * R + group_of<G>(), row = min(mine, a.M - 1);
    const bool in = mine < a.M;                                              // (others go along with the last row, for the barriers, and write nothing)
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    Raw8<S> x[U];
    Raw8<T> b[U], w[U], wp[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = lane + u * G;
        x[u] = load8((const S*)a.x + row * a.ldx, unit * 8, a.K);
        b[u] = wp[u] = zero8<T>();
        if (a.branch) b[u] = load8((const T*)a.branch + row * a.ldb, unit * 8, a.K);
        if (a.post_weight) wp[u] = load8((const T*)a.post_weight, unit * 8, a.K);
        w[u] = load8((const T*)a.weight, unit * 8, a.K);
    }
    float rb = 0.f;
    if (a.post_weight) {
        float sum[1] = {0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] = fmaf(b[u][i], b[u][i], sum[0]);
        group_sum<G, NT>(sum, shared, turn);
        rb = inverse_root(sum[0], a.K, a.eps);
    }
    float y[U][8], sum[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = lane + u * G;
        Factor<T> f = {};
        if (a.branch) f = factor_of<T>(a, g, row, unit);
        stream8<S, T>(a, x[u], b[u], wp[u], f, rb, y[u]);
        if (a.branch && in && unit * 8 < a.K) store8<true>((S*)a.y + row * a.ldy, unit * 8, a.K, y[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = fmaf(y[u][i], y[u][i], sum[0]);
    }
    group_sum<G, NT>(sum, shared, turn);
    const float r = inverse_root(sum[0], a.K, a.eps);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!in || (lane + u * G) * 8 >= a.K) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[u][i] = y[u][i] * r * w[u][i];
        store8((T*)a.n + row * a.ldn, (lane + u * G) * 8, a.K, y[u]);
    }
    if (in && lane == 0 && a.stats) {
        a.stats[row * 2] = r;
        a.stats[row * 2 + 1] = rb;
    }
}

// Rows that no workgroup holds: each thread goes over its units once for every sum, and once more for the results.
template <class S, class T, int NT>
__global__ void __launch_bounds__(NT) tr_norm_forward_wide_kernel(Norm a)
{
    __shared__ float shared[2 * NT / WAVE];
    const i64 row = blockIdx.x;
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    const S* xs = (const S*)a.x + row * a.ldx;
    const T* bs = (const T*)a.branch + row * a.ldb;
    float rb = 0.f;
    if (a.post_weight) {
        float sum[1] = {0.f};
        for (int k = threadIdx.x * 8; k < a.K; k += NT * 8) {
            const Raw8<T> b = load8(bs, k, a.K);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] = fmaf(b[i], b[i], sum[0]);
        }
        group_sum<NT, NT>(sum, shared, turn);
        rb = inverse_root(sum[0], a.K, a.eps);
    }
    auto at = [&](int k, float (&y)[8]) {
        Raw8<T> b = zero8<T>(), wp = zero8<T>();
        Factor<T> f = {};
        if (a.branch) {
            b = load8(bs, k, a.K);
            f = factor_of<T>(a, g, row, k / 8);
        }
        if (a.post_weight) wp = load8((const T*)a.post_weight, k, a.K);
        stream8<S, T>(a, load8(xs, k, a.K), b, wp, f, rb, y);
    };
    float sum[1] = {0.f}, y[8];
    for (int k = threadIdx.x * 8; k < a.K; k += NT * 8) {
        at(k, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = fmaf(y[i], y[i], sum[0]);
    }
    group_sum<NT, NT>(sum, shared, turn);
    const float r = inverse_root(sum[0], a.K, a.eps);
    for (int k = threadIdx.x * 8; k < a.K; k += NT * 8) {
        at(k, y);
        if (a.branch) store8((S*)a.y + row * a.ldy, k, a.K, y);         // (after the row's last look at x, which y may replace)
        const Raw8<T> w = load8((const T*)a.weight, k, a.K);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
        store8((T*)a.n + row * a.ldn, k, a.K, y);
    }
    if (threadIdx.x == 0 && a.stats) {
        a.stats[row * 2] = r;
        a.stats[row * 2 + 1] = rb;
    }
}

// Eight elements of a row in the backward pass: as they lie in memory ...  JOIN: with x in the place of y.
template <class S, class T, bool JOIN>
struct Back8 {
    Raw8<S> y, dy;
    Raw8<T> dn, b, gate;

    // (Gates of channels are those of the row before.)
    __device__ __forceinline__ void load(const Norm& a, i64 row, int unit, bool first)
    {
        const int k = unit * 8;
        y = load8((const S*)a.y + row * a.ldy, k, a.K);
        dy = a.dy ? load8((const S*)a.dy + row * a.lddy, k, a.K) : zero8<S>();
        dn = a.dn ? load8((const T*)a.dn + row * a.lddn, k, a.K) : zero8<T>();
        b = a.branch ? load8((const T*)a.branch + row * a.ldb, k, a.K) : zero8<T>();
        if (first) gate = zero8<T>();
        if (a.gate && (first || a.ldgate)) gate = load8((const T*)a.gate + row * a.ldgate, k, a.K);
    }

    // What the branch is multiplied by; computed where it is wanted.
    __device__ __forceinline__ Factor<T> factor(const Norm& a, u32 keep) const
    {
        return Factor<T>{gate, keep, a.random.threshold ? a.scale * a.random.kept : a.scale, a.gate != nullptr};
    }

    // ... and not as the floats of one use kept for the next.
    __device__ __forceinline__ void forget()
    {
        forget_words(y);
        forget_words(dy);
        forget_words(dn);
        forget_words(b);
        forget_words(gate);
    }

    // u of the eight.  With JOIN from x and what the branch adds, in 32 bits and not rounded: from a y of 16 bits every term of dw is off by half a step of y, and dw by as much again as
    // its own rounding (8192 x 4096 in bf16 2.28e-3 of dw, from x 1.67e-3).
    __device__ __forceinline__ void normed(const Norm& a, const Raw8<T>& wp, u32 keep, float r, float rb, float (&u)[8]) const
    {
        const Factor<T> f = factor(a, keep);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = a.post_weight ? b[i] * rb * wp[i] : b[i];
            u[i] = (JOIN && f.kept(i) ? fmaf(f[i], d, y[i]) : y[i]) * r;
        }
    }

    // mean(dn w u), mean(q h (dy + r dn w)) and mean(q h u), not yet divided, and u for the results.  With JOIN q h is what the stream is formed of, so it is computed in any case, and no
    // branch stands in the way (8192 x 4096 in bf16, one set of operands over and over: 89 us for the call with one, 86 without).
    __device__ __forceinline__ void sums(const Norm& a, const Raw8<T>& w, const Raw8<T>& wp, u32 keep, float r, float rb, float (&u)[8], float (&sum)[3]) const
    {
        const Factor<T> f = factor(a, keep);
        if constexpr (!JOIN) normed(a, wp, keep, r, rb, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float dnw = dn[i] * w[i];
            if constexpr (JOIN) {
                const float by = a.post_weight ? wp[i] * rb : 1.f, qh = f.kept(i) ? f.whole(i) * b[i] * by : 0.f;
                u[i] = (y[i] + qh) * r;
                sum[0] = fmaf(dnw, u[i], sum[0]);
                sum[1] = fmaf(qh, fmaf(r, dnw, dy[i]), sum[1]);
                sum[2] = fmaf(qh, u[i], sum[2]);
            } else {
                sum[0] = fmaf(dnw, u[i], sum[0]);
                if (a.post_weight) {
                    const float qh = f[i] * wp[i] * b[i] * rb;
                    sum[1] = fmaf(qh, fmaf(r, dnw, dy[i]), sum[1]);
                    sum[2] = fmaf(qh, u[i], sum[2]);
                }
            }
        }
    }

    // The row's results, and what it adds to the columns' sums.
    __device__ __forceinline__ void results(const Norm& a, const Raw8<T>& w, const Raw8<T>& wp, u32 keep, i64 row, int unit, float r, float rb, const float (&u)[8],
                                            float c1, float c2, float (&dw)[8], float (&dwp)[8], float (&dg)[8]) const
    {
        const Factor<T> f = factor(a, keep);
        const int k = unit * 8;
        float dx[8], db[8], gate[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dx[i] = fmaf(r, fmaf(-u[i], c1, dn[i] * w[i]), dy[i]);
            dw[i] = fmaf(dn[i], u[i], dw[i]);
        }
        if (a.dx) store8<true>((S*)a.dx + row * a.lddx, k, a.K, dx);
        if (!a.branch) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float dd = f[i] * dx[i];
            float h = b[i], d = h;
            db[i] = dd;
            if (a.post_weight) {
                h *= rb;
                d = h * wp[i];
                db[i] = rb * fmaf(-h, c2, dd * wp[i]);
                dwp[i] = fmaf(dd, h, dwp[i]);
            }
            if (a.gate) {
                gate[i] = f.kept(i) ? f.scale * d * dx[i] : 0.f;
                dg[i] += gate[i];
            }
        }
        if (a.dbranch) store8<true>((T*)a.dbranch + row * a.lddb, k, a.K, db);
        if (a.dgate) store8<true>((T*)a.dgate + row * a.lddgate, k, a.K, gate);
    }
};

__device__ __forceinline__ void means(const Norm& a, const float (&sum)[3], float r, float& c1, float& c2)
{
    c1 = sum[0] / (float)a.K;
    c2 = (sum[1] - c1 * r * sum[2]) / (float)a.K;
}

// How a backward pass keeps its row: not at all (what the results need is read again, from the cache), in registers, or with the next row under way besides.  Two units a thread are read again.
enum Keep { REREAD, HOLD, AHEAD };

// Backward: each workgroup takes rows R apart over the whole grid, G threads a row, and keeps its columns' sums in registers until the end.  Memory bounds it, and the sums' way: 8192 x 4096 in bf16
// with both norms, a gate for each channel and dropout 87 us with the columns' kernel, 4.6 TB/s beside 25 MB of columns' sums (fp32 4096 x 4096 104, 3.9; 262144 x 64 52, 3.9; 2048 x 16384 165, 2.4, with
// all three sums in registers, most of them spilled, a ninth more).
// Weights and rows stay as they lie in memory: as floats, which the compiler would keep over the exchange, they took 232 registers a thread, and one workgroup stood where four do.
template <class S, class T, bool JOIN, int G, int U, int NT, Keep KEEP>
__global__ void __launch_bounds__(NT) tr_norm_backward_kernel(Norm a)
{
    static_assert(U == 1 || KEEP == REREAD);
    constexpr int R = NT / G, COLUMNS = G * U * 8;
    __shared__ float shared[2 * NT / WAVE * 3];
    __shared__ float columns[R > 1 ? COLUMNS : 1];
    const int lane = threadIdx.x % G, group = group_of<G>();
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    Raw8<T> w, wp;
    // Two units a thread have no registers for all three sums: two of them stand in shared memory, each thread's own.
    constexpr bool SHARE = U > 1;
    __shared__ float more[SHARE ? 2 * U * 8 : 1][SHARE ? NT : 1];
    float dw[U][8] = {}, dwp[SHARE ? 1 : U][8] = {}, dg[SHARE ? 1 : U][8] = {};
    if constexpr (SHARE)
        for (int i = 0; i < 2 * U * 8; ++i) more[i][threadIdx.x] = 0.f;
    auto fetch = [&](float (&v)[8], int which, int u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = more[SHARE ? (which * U + u) * 8 + i : 0][SHARE ? threadIdx.x : 0];
    };
    auto leave = [&](const float (&v)[8], int which, int u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) more[SHARE ? (which * U + u) * 8 + i : 0][SHARE ? threadIdx.x : 0] = v[i];
    };
    auto load_weights = [&](Raw8<T>& w, Raw8<T>& wp, int unit) {
        w = load8((const T*)a.weight, unit * 8, a.K);
        wp = a.post_weight ? load8((const T*)a.post_weight, unit * 8, a.K) : zero8<T>();
    };
    if constexpr (KEEP != REREAD) load_weights(w, wp, lane);
    struct Row {
        Back8<S, T, JOIN> e;
        float r, rb;
    };
    // Groups behind the last row go along with it, for the barriers, and leave nothing.
    auto load = [&](Row& to, i64 base, bool first) {
        const i64 row = min(base + group, a.M - 1);
        to.r = a.stats[row * 2];
        to.rb = a.stats[row * 2 + 1];
        if constexpr (KEEP != REREAD) to.e.load(a, row, lane, first);
    };
    const i64 step = (i64)gridDim.x * R;
    Row row, next;
    if constexpr (KEEP == AHEAD) load(next, (i64)blockIdx.x * R, true);
    for (i64 base = (i64)blockIdx.x * R; base < a.M; base += step) {         // (the same turns for the whole workgroup: barriers)
        if constexpr (KEEP == AHEAD) {
            row = next;
            if (!JOIN && base + step < a.M) load(next, base + step, false);
        } else load(row, base, base < step);
        const i64 n = base + group, held = min(n, a.M - 1);
        const bool in = n < a.M;
        float sum[3] = {0.f, 0.f, 0.f};
        u32 keep[U];
        constexpr bool STANDS = JOIN && KEEP != REREAD;                      // u, from the sums to the results, in the place of x and of forming it again
        float u8[8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G;
            if constexpr (SHARE) __builtin_amdgcn_sched_barrier(0);          // a unit after the other: no registers for both
            if constexpr (KEEP == REREAD) {
                load_weights(w, wp, unit);
                row.e.load(a, held, unit, true);
            } else {
                forget_words(w);
                forget_words(wp);
            }
            keep[u] = a.random.threshold ? keep_bits(g, a.random.threshold, (u32)unit, (u32)n) : 0xffu;
            row.e.sums(a, w, wp, keep[u], row.r, row.rb, u8, sum);
        }
        if constexpr (KEEP == AHEAD && JOIN)                                 // (before the sums there are no registers for it: 98 us where this takes 86, measured likewise)
            if (base + step < a.M) load(next, base + step, false);
        group_sum<G, NT>(sum, shared, turn);
        float c1, c2;
        means(a, sum, row.r, c1, c2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G;
            if constexpr (SHARE) __builtin_amdgcn_sched_barrier(0);          // a unit after the other: no registers for both
            if constexpr (KEEP == REREAD) {
                load_weights(w, wp, unit);
                row.e.load(a, held, unit, true);
            } else {
                row.e.forget();
                forget_words(w);
                forget_words(wp);
            }
            if (!in || unit * 8 >= a.K) continue;
            const int of = SHARE ? 0 : u;
            if constexpr (SHARE) {
                fetch(dwp[0], 0, u);
                fetch(dg[0], 1, u);
            }
            if constexpr (!STANDS) row.e.normed(a, wp, keep[u], row.r, row.rb, u8);
            row.e.results(a, w, wp, keep[u], n, unit, row.r, row.rb, u8, c1, c2, dw[u], dwp[of], dg[of]);
            if constexpr (SHARE) {
                leave(dwp[0], 0, u);
                leave(dg[0], 1, u);
            }
        }
    }
    const int padded = (a.K + 7) / 8 * 8;
    // The rows' groups joined: those of a wave by exchanges between its lanes, then the waves one after the other.
    constexpr int JOINED = G < WAVE ? WAVE : G, STEPS = NT / JOINED;
    const int turn_of = threadIdx.x / JOINED;
    auto join = [&](float (&v)[U][8], int place) {
        if (place < 0) return;
        float* out = a.partial + ((i64)blockIdx.x * a.sums + place) * padded;
#pragma unroll
        for (int d = G; d < WAVE; d *= 2)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] += __shfl_xor(v[u][i], d);
        if constexpr (STEPS > 1) {
            for (int r = 0; r < STEPS; ++r) {
                __syncthreads();
                if (turn_of != r || (int)(threadIdx.x % JOINED) >= G) continue;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float& c = columns[i * (G * U) + u * G + lane];
                        if (r == STEPS - 1) v[u][i] += c;
                        else c = r == 0 ? v[u][i] : c + v[u][i];
                    }
            }
            if (turn_of != STEPS - 1) return;
        }
        if ((int)(threadIdx.x % JOINED) >= G) return;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G;
            if (unit * 8 < a.K) store8(out, unit * 8, padded, v[u]);
        }
    };
    join(dw, a.sum_w);
    if constexpr (SHARE) {
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int u = 0; u < U; ++u) fetch(dw[u], which, u);
            join(dw, which == 0 ? a.sum_post : a.sum_gate);
        }
    } else {
        join(dwp, a.sum_post);
        join(dg, a.sum_gate);
    }
}

template <class S, class T, bool JOIN, int NT>
__global__ void __launch_bounds__(NT) tr_norm_backward_wide_kernel(Norm a)
{
    __shared__ float shared[2 * NT / WAVE * 3];
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    const int padded = (a.K + 7) / 8 * 8;
    float* mine = a.partial + (i64)blockIdx.x * a.sums * padded;
    for (i64 row = blockIdx.x; row < a.M; row += gridDim.x) {
        const float r = a.stats[row * 2], rb = a.stats[row * 2 + 1];
        float sum[3] = {0.f, 0.f, 0.f}, c1, c2;
        auto each = [&](auto&& f) {
            for (int unit = threadIdx.x; unit * 8 < a.K; unit += NT) {
                Back8<S, T, JOIN> e;
                e.load(a, row, unit, true);
                const Raw8<T> w = load8((const T*)a.weight, unit * 8, a.K);
                const Raw8<T> wp = a.post_weight ? load8((const T*)a.post_weight, unit * 8, a.K) : zero8<T>();
                f(unit, a.random.threshold ? keep_bits(g, a.random.threshold, (u32)unit, (u32)row) : 0xffu, e, w, wp);
            }
        };
        each([&](int, u32 keep, const Back8<S, T, JOIN>& e, const Raw8<T>& w, const Raw8<T>& wp) {
            float u[8];
            e.sums(a, w, wp, keep, r, rb, u, sum);
        });
        group_sum<NT, NT>(sum, shared, turn);
        means(a, sum, r, c1, c2);
        each([&](int unit, u32 keep, const Back8<S, T, JOIN>& e, const Raw8<T>& w, const Raw8<T>& wp) {
            float u[8], v[3][8] = {};
            e.normed(a, wp, keep, r, rb, u);
            const int place[3] = {a.sum_w, a.sum_post, a.sum_gate};
#pragma unroll
            for (int s = 0; s < 3; ++s)                                      // (this thread's alone, from its row before)
                if (place[s] >= 0 && row != blockIdx.x) {
                    const Raw8<float> before = load8(mine + (i64)place[s] * padded, unit * 8, padded);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[s][i] = before[i];
                }
            e.results(a, w, wp, keep, row, unit, r, rb, u, c1, c2, v[0], v[1], v[2]);
#pragma unroll
            for (int s = 0; s < 3; ++s)
                if (place[s] >= 0) store8(mine + (i64)place[s] * padded, unit * 8, padded, v[s]);
        });
    }
}

// The columns' sums over the workgroups' parts, in their order: 64 columns a workgroup at a time, the parts spread over its waves and joined.  Rows above 2^26 have more columns than a launch has
// workgroups for.
constexpr i64 COLUMN_BLOCKS = 1ll << 20;

template <class T>
__global__ void __launch_bounds__(1024) tr_norm_columns_kernel(Norm a)
{
    __shared__ float shared[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, place = blockIdx.y;
    const int padded = (a.K + 7) / 8 * 8;
    const int each = (a.blocks + 15) / 16, from = wave * each, to = min(from + each, a.blocks);
    for (i64 k0 = (i64)blockIdx.x * 64; k0 < a.K; k0 += (i64)gridDim.x * 64) {
        const i64 k = k0 + lane;
        float sum = 0.f;
        if (k < a.K)
#pragma unroll 8
            for (int b = from; b < to; ++b) sum += a.partial[((i64)b * a.sums + place) * padded + k];
        __syncthreads();                                                     // the columns before are read
        shared[wave][lane] = sum;
        __syncthreads();
        if (wave || k >= a.K) continue;
        sum = shared[0][lane];
#pragma unroll
        for (int w = 1; w < 16; ++w) sum += shared[w][lane];
        ((T*)a.column_out[place])[k] = from_float<T>(sum);
    }
}

struct Dropout {
    const void* x;
    void* out;
    i64 ldx, ldout, M;
    int K;
    Random random;
};

// Dropout: every thread takes units of eight elements, 256 apart, of its workgroup's stretch of all the rows' units.  Memory bounds it, 8192 x 12288 in bf16 73 us, 5.5 TB/s; the
// generator's 14 products a unit are 27 us of it, beside.
template <class T, int EACH, bool STREAM>
__global__ void __launch_bounds__(256) tr_dropout_kernel(Dropout a)
{
    const u32 units = ((u32)a.K + 7) / 8;
    const i64 all = a.M * units, first = ((i64)blockIdx.x * EACH) * 256 + threadIdx.x;
    if (first >= all) return;
    i64 row = first / units;
    u32 unit = (u32)(first - row * units);
    const u32 rows = 256 / units, left = 256 % units;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (row < a.M) {
            const Raw8<T> x = load8<STREAM>((const T*)a.x + row * a.ldx, (int)unit * 8, a.K);
            const u32 keep = a.random.threshold ? keep_bits(g, a.random.threshold, unit, (u32)row) : 0xffu;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = keep >> i & 1 ? x[i] * a.random.kept : 0.f;
            store8<STREAM>((T*)a.out + row * a.ldout, (int)unit * 8, a.K, v);
        }
        row += rows;
        unit += left;
        if (unit >= units) {
            unit -= units;
            ++row;
        }
    }
}

}  // namespace
