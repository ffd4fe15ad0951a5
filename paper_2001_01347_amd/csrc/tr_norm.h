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
    void *y, *n;                                 // (in the backward pass y is an input)
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
__device__ __forceinline__ Raw8<T> load8(const T* p, int have)
{
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = load_some(p + j * PER_WORD4<T>, (i64)have - j * PER_WORD4<T>);
    return r;
}

template <class T>
__device__ __forceinline__ Raw8<T> zero8()
{
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = Word4{0, 0, 0, 0};
    return r;
}

template <class T>
__device__ __forceinline__ void store8(T* p, int have, const float (&v)[8])
{
    Pack<T> w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / PER_WORD4<T>].v[i % PER_WORD4<T>] = from_float<T>(v[i]);
    if (have >= 8) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) store_loose(p + j * PER_WORD4<T>, w[j].raw);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < have) p[i] = w[i / PER_WORD4<T>].v[i % PER_WORD4<T>];
}

// Sums over the G threads of a row, in an order that G fixes.  One barrier: the buffer of one call is written again in the call after the next,
// which no thread reaches before all have read.
template <int G, int NT, int NV>
__device__ __forceinline__ void group_sum(float (&v)[NV], float* shared, int& turn)
{
#pragma unroll
    for (int d = (G < WAVE ? G : WAVE) / 2; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += __shfl_xor(v[i], d);
    if constexpr (G > WAVE) {
        float* buffer = shared + turn * (NT / WAVE * NV);
        turn ^= 1;
        const int wave = threadIdx.x / WAVE;
        if (threadIdx.x % WAVE == 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) buffer[wave * NV + i] = v[i];
        __syncthreads();
        const float* mine = buffer + wave / (G / WAVE) * (G / WAVE) * NV;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            v[i] = mine[i];
#pragma unroll
            for (int w = 1; w < G / WAVE; ++w) v[i] += mine[w * NV + i];
        }
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
    __device__ __forceinline__ float plain(int i) const { return kept(i) ? scale : 0.f; }
    __device__ __forceinline__ float operator[](int i) const { return !kept(i) ? 0.f : gated ? scale * gate[i] : scale; }
};

template <class T>
__device__ __forceinline__ Factor<T> factor_of(const Norm& a, const Generator& g, i64 row, int unit, int have)
{
    Factor<T> f;
    f.gated = a.gate != nullptr;
    f.gate = f.gated ? load8((const T*)a.gate + row * a.ldgate + unit * 8, have) : zero8<T>();
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

// Forward: G threads a row, U units of eight elements each.
template <class S, class T, int G, int U, int NT>
__global__ void __launch_bounds__(NT) tr_norm_forward_kernel(Norm a)
{
    __shared__ float shared[2 * NT / WAVE];
    constexpr int R = NT / G;
    const int lane = threadIdx.x % G;
    const i64 row = (i64)blockIdx.x * R + threadIdx.x / G;
    const bool in = row < a.M;
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    Raw8<S> x[U];
    Raw8<T> b[U], w[U], wp[U];
    int have[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = lane + u * G;
        have[u] = in ? a.K - unit * 8 : 0;
        x[u] = load8((const S*)a.x + row * a.ldx + unit * 8, have[u]);
        b[u] = wp[u] = zero8<T>();
        if (a.branch) b[u] = load8((const T*)a.branch + row * a.ldb + unit * 8, have[u]);
        if (a.post_weight) wp[u] = load8((const T*)a.post_weight + unit * 8, have[u]);
        w[u] = load8((const T*)a.weight + unit * 8, have[u]);
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
        if (a.branch && have[u] > 0) f = factor_of<T>(a, g, row, unit, have[u]);
        stream8<S, T>(a, x[u], b[u], wp[u], f, rb, y[u]);
        if (a.branch && have[u] > 0) store8((S*)a.y + row * a.ldy + unit * 8, have[u], y[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = fmaf(y[u][i], y[u][i], sum[0]);
    }
    group_sum<G, NT>(sum, shared, turn);
    const float r = inverse_root(sum[0], a.K, a.eps);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (have[u] <= 0) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[u][i] = y[u][i] * r * w[u][i];
        store8((T*)a.n + row * a.ldn + (lane + u * G) * 8, have[u], y[u]);
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
            const Raw8<T> b = load8(bs + k, a.K - k);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] = fmaf(b[i], b[i], sum[0]);
        }
        group_sum<NT, NT>(sum, shared, turn);
        rb = inverse_root(sum[0], a.K, a.eps);
    }
    auto at = [&](int k, float (&y)[8]) {
        const int have = a.K - k;
        Raw8<T> b = zero8<T>(), wp = zero8<T>();
        Factor<T> f = {};
        if (a.branch) {
            b = load8(bs + k, have);
            f = factor_of<T>(a, g, row, k / 8, have);
        }
        if (a.post_weight) wp = load8((const T*)a.post_weight + k, have);
        stream8<S, T>(a, load8(xs + k, have), b, wp, f, rb, y);
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
        if (a.branch) store8((S*)a.y + row * a.ldy + k, a.K - k, y);         // (after the row's last look at x, which y may replace)
        const Raw8<T> w = load8((const T*)a.weight + k, a.K - k);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = y[i] * r * w[i];
        store8((T*)a.n + row * a.ldn + k, a.K - k, y);
    }
    if (threadIdx.x == 0 && a.stats) {
        a.stats[row * 2] = r;
        a.stats[row * 2 + 1] = rb;
    }
}

// Eight elements of a row in the backward pass.
template <class S, class T>
struct Back8 {
    Raw8<S> y, dy;
    Raw8<T> dn, b;
    Factor<T> f;

    __device__ __forceinline__ void load(const Norm& a, const Generator& g, i64 row, int unit, int have)
    {
        const i64 k = (i64)unit * 8;
        y = load8((const S*)a.y + row * a.ldy + k, have);
        dy = a.dy && have > 0 ? load8((const S*)a.dy + row * a.lddy + k, have) : zero8<S>();
        dn = a.dn && have > 0 ? load8((const T*)a.dn + row * a.lddn + k, have) : zero8<T>();
        b = zero8<T>();
        f = {};
        if (a.branch && have > 0) {
            b = load8((const T*)a.branch + row * a.ldb + k, have);
            f = factor_of<T>(a, g, row, unit, have);
        }
    }

    // mean(dn w u), mean(q h (dy + r dn w)) and mean(q h u), not yet divided.
    __device__ __forceinline__ void sums(const Norm& a, const Raw8<T>& w, const Raw8<T>& wp, float r, float rb, float (&sum)[3]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = y[i] * r, dnw = dn[i] * w[i];
            sum[0] = fmaf(dnw, u, sum[0]);
            if (a.post_weight) {
                const float qh = f[i] * wp[i] * b[i] * rb;
                sum[1] = fmaf(qh, fmaf(r, dnw, dy[i]), sum[1]);
                sum[2] = fmaf(qh, u, sum[2]);
            }
        }
    }

    // The row's results, and what it adds to the columns' sums.
    __device__ __forceinline__ void results(const Norm& a, const Raw8<T>& w, const Raw8<T>& wp, i64 row, int unit, int have, float r, float rb,
                                            float c1, float c2, float (&dw)[8], float (&dwp)[8], float (&dg)[8]) const
    {
        const i64 k = (i64)unit * 8;
        float dx[8], db[8], gate[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = y[i] * r;
            dx[i] = fmaf(r, fmaf(-u, c1, dn[i] * w[i]), dy[i]);
            dw[i] = dn[i] * u;
            db[i] = dwp[i] = dg[i] = gate[i] = 0.f;
            if (a.branch) {
                const float dd = f[i] * dx[i], h = a.post_weight ? b[i] * rb : b[i];
                db[i] = a.post_weight ? rb * fmaf(-h, c2, dd * wp[i]) : dd;
                dwp[i] = dd * h;
                dg[i] = gate[i] = f.kept(i) ? f.scale * (a.post_weight ? h * wp[i] : h) * dx[i] : 0.f;
            }
        }
        if (a.dx) store8((S*)a.dx + row * a.lddx + k, have, dx);
        if (a.dbranch) store8((T*)a.dbranch + row * a.lddb + k, have, db);
        if (a.dgate) store8((T*)a.dgate + row * a.lddgate + k, have, gate);
    }
};

__device__ __forceinline__ void means(const Norm& a, const float (&sum)[3], float r, float& c1, float& c2)
{
    c1 = sum[0] / (float)a.K;
    c2 = (sum[1] - c1 * r * sum[2]) / (float)a.K;
}

// Backward: each workgroup takes rows R apart over the whole grid, G threads a row, and keeps its columns' sums in registers until the end.
template <class S, class T, int G, int U, int NT>
__global__ void __launch_bounds__(NT) tr_norm_backward_kernel(Norm a)
{
    constexpr int R = NT / G, COLUMNS = G * U * 8;
    __shared__ float shared[2 * NT / WAVE * 3];
    __shared__ float columns[R > 1 ? COLUMNS : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    int turn = 0;
    Generator g = {};
    if (a.random.threshold) g = generator(a.random);
    Raw8<T> w[U], wp[U];
    float dw[U][8] = {}, dwp[U][8] = {}, dg[U][8] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = lane + u * G;
        w[u] = load8((const T*)a.weight + unit * 8, a.K - unit * 8);
        wp[u] = zero8<T>();
        if (a.post_weight) wp[u] = load8((const T*)a.post_weight + unit * 8, a.K - unit * 8);
    }
    for (i64 base = (i64)blockIdx.x * R; base < a.M; base += (i64)gridDim.x * R) {       // (the same turns for the whole workgroup: barriers)
        const i64 row = base + group;
        const bool in = row < a.M;
        const float r = in ? a.stats[row * 2] : 0.f, rb = in ? a.stats[row * 2 + 1] : 0.f;
        Back8<S, T> e[U];
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G;
            e[u].load(a, g, row, unit, in ? a.K - unit * 8 : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) e[u].sums(a, w[u], wp[u], r, rb, sum);
        group_sum<G, NT>(sum, shared, turn);
        float c1, c2;
        means(a, sum, r, c1, c2);
        if (!in) continue;                                                   // (its last turn)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G, have = a.K - unit * 8;
            if (have <= 0) continue;
            float w8[8], p8[8], g8[8];
            e[u].results(a, w[u], wp[u], row, unit, have, r, rb, c1, c2, w8, p8, g8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[u][i] += w8[i];
                dwp[u][i] += p8[i];
                dg[u][i] += g8[i];
            }
        }
    }
    const int padded = (a.K + 7) / 8 * 8;
    auto join = [&](float (&v)[U][8], int place) {
        if (place < 0) return;
        float* out = a.partial + ((i64)blockIdx.x * a.sums + place) * padded;
        if constexpr (R > 1) {                                               // the groups one after the other
            for (int r = 0; r < R; ++r) {
                __syncthreads();
                if (group != r) continue;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float& c = columns[i * (G * U) + u * G + lane];
                        if (r == R - 1) v[u][i] += c;
                        else c = r == 0 ? v[u][i] : c + v[u][i];
                    }
            }
            if (group != R - 1) return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int unit = lane + u * G;
            if (unit * 8 < a.K) store8(out + unit * 8, 8, v[u]);
        }
    };
    join(dw, a.sum_w);
    join(dwp, a.sum_post);
    join(dg, a.sum_gate);
}

template <class S, class T, int NT>
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
                const int have = a.K - unit * 8;
                Back8<S, T> e;
                e.load(a, g, row, unit, have);
                const Raw8<T> w = load8((const T*)a.weight + unit * 8, have);
                const Raw8<T> wp = a.post_weight ? load8((const T*)a.post_weight + unit * 8, have) : zero8<T>();
                f(unit, have, e, w, wp);
            }
        };
        each([&](int, int, const Back8<S, T>& e, const Raw8<T>& w, const Raw8<T>& wp) { e.sums(a, w, wp, r, rb, sum); });
        group_sum<NT, NT>(sum, shared, turn);
        means(a, sum, r, c1, c2);
        each([&](int unit, int have, const Back8<S, T>& e, const Raw8<T>& w, const Raw8<T>& wp) {
            float v[3][8];
            e.results(a, w, wp, row, unit, have, r, rb, c1, c2, v[0], v[1], v[2]);
            const int place[3] = {a.sum_w, a.sum_post, a.sum_gate};
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                if (place[s] < 0) continue;
                float* out = mine + (i64)place[s] * padded + unit * 8;       // this thread's alone
                if (row != blockIdx.x) {
                    const Raw8<float> before = load8(out, 8);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[s][i] += before[i];
                }
                store8(out, 8, v[s]);
            }
        });
    }
}

// The columns' sums over the workgroups' parts, in their order: 64 columns a workgroup, the parts spread over its waves and joined.
template <class T>
__global__ void __launch_bounds__(1024) tr_norm_columns_kernel(Norm a)
{
    __shared__ float shared[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, place = blockIdx.y;
    const int padded = (a.K + 7) / 8 * 8;
    const i64 k = (i64)blockIdx.x * 64 + lane;
    const int each = (a.blocks + 15) / 16, from = wave * each, to = min(from + each, a.blocks);
    float sum = 0.f;
    if (k < a.K)
#pragma unroll 8
        for (int b = from; b < to; ++b) sum += a.partial[((i64)b * a.sums + place) * padded + k];
    shared[wave][lane] = sum;
    __syncthreads();
    if (wave || k >= a.K) return;
    sum = shared[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += shared[w][lane];
    ((T*)a.column_out[place])[k] = from_float<T>(sum);
}

struct Dropout {
    const void* x;
    void* out;
    i64 ldx, ldout, M;
    int K;
    Random random;
};

// Dropout: every thread takes units of eight elements, 256 apart, of its workgroup's stretch of all the rows' units.
template <class T, int EACH>
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
            const int have = a.K - (int)unit * 8;
            const Raw8<T> x = load8((const T*)a.x + row * a.ldx + unit * 8, have);
            const u32 keep = a.random.threshold ? keep_bits(g, a.random.threshold, unit, (u32)row) : 0xffu;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = keep >> i & 1 ? x[i] * a.random.kept : 0.f;
            store8((T*)a.out + row * a.ldout + unit * 8, have, v);
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
