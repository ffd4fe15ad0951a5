// The gated feed-forward block: h = act(x Wg^T) * (x Wu^T), and its backward pass.
// Part of the ZipLine library (see training.hip); device code for gfx950.
#pragma once
#include "ebsp_training.h"
#include "tr_product.h"

namespace {

// act(g) and act'(g).  The activation is chosen by a value that is the same for the whole launch.
// (The hardware's exponential and reciprocal are good to an ulp.)
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)); }

// e^(-g^2 / 2).
__device__ __forceinline__ float bell(float g) { return __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g); }

// Phi(g), with `e` = bell(g).  0.5 (1 + erf(g / sqrt 2)) would have no digits left where g is well below 0: it is formed from Phi(-|g|).  Results of 32 bits take the
// error function's complement; for those of 16 bits, Phi(-a) e^(a^2 / 2) = t q(t) with t = 1 / (1 + 0.3 a) and a polynomial fitted to the least largest relative
// error over 0 <= a <= 14.5 (1.7e-7; 6e-7 as evaluated), which is shorter in an epilogue that has it 128 times.  us, with the error function / its complement / this:
// forward 2048 x 2048 x 8192 bf16 122 / 126 / 116; with gradients 1021 x 1000 x 2730 86.8 / 88.1 / 83.8, 8192 x 64 x 12288 773 / 797 / 744.
template <class T>
__device__ __forceinline__ float normal_cdf(float g, float e)
{
    if constexpr (sizeof(T) == 4) return 0.5f * erfcf(g * -0.70710678118654752f);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3f * fabsf(g));
    float q = 0.0354237035f;
    q = fmaf(q, t, -0.156158328f);
    q = fmaf(q, t, 0.204556584f);
    q = fmaf(q, t, -0.0520338379f);
    q = fmaf(q, t, 0.127691686f);
    q = fmaf(q, t, 0.100175969f);
    q = fmaf(q, t, 0.120712131f);
    q = fmaf(q, t, 0.119632006f);
    const float tail = q * t * e;
    return g < 0.f ? tail : 1.f - tail;
}

template <class T>
__device__ __forceinline__ float activation(int act, float g)
{
    switch (act) {
    case EBSP_ACT_SILU: return g * sigmoid(g);
    case EBSP_ACT_SIGMOID: return sigmoid(g);
    case EBSP_ACT_RELU: return g < 0.f ? 0.f : g;                            // (a NaN stays one)
    case EBSP_ACT_GELU: return g * normal_cdf<T>(g, bell(g));
    default: {                                                               // 0.5 g (1 + tanh z) = g sigmoid(2 z)
        const float c = fminf(fmaxf(g, -16.f), 16.f);                        // tanh is 1 long before; the cube stays finite
        const float z = 0.79788456080286536f * (c + 0.044715f * c * c * c);
        return g * sigmoid(2.f * z);
    }
    }
}

template <class T>
__device__ __forceinline__ void activation_both(int act, float g, float& a, float& d)
{
    switch (act) {
    case EBSP_ACT_SILU: {
        const float s = sigmoid(g);
        a = g * s;
        d = s * (1.f + g * (1.f - s));
        break;
    }
    case EBSP_ACT_SIGMOID: {                                                 // a (1 - a) from e^-|g|: 1 - a has no digits left for large g
        const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + e);
        a = g < 0.f ? e * r : r;
        d = e * r * r;
        break;
    }
    case EBSP_ACT_RELU:
        a = g < 0.f ? 0.f : g;
        d = g > 0.f ? 1.f : 0.f;
        break;
    case EBSP_ACT_GELU: {
        const float e = bell(g), cdf = normal_cdf<T>(g, e);
        a = g * cdf;
        d = cdf + g * 0.39894228040143268f * e;
        break;
    }
    default: {
        const float c = fminf(fmaxf(g, -16.f), 16.f);
        const float z = 0.79788456080286536f * (c + 0.044715f * c * c * c);
        const float s = sigmoid(2.f * z);
        a = g * s;
        d = s + g * 2.f * s * (1.f - s) * 0.79788456080286536f * (1.f + 0.134145f * c * c);
    }
    }
}

struct FfForward {
    Operand x, w;                                                            // w: gate and up
    void* h;
    float *g, *u;                                                            // NULL where nothing is kept for a backward pass
    i64 ldh, ldg;
    int act;
    float* partial;                                                          // sums in parts: [parts][gate, up][tokens][units, padded to 4]
    int parts;
};

__host__ __device__ __forceinline__ i64 partial_ld(i64 columns) { return (columns + 3) / 4 * 4; }

// Gate and up of the same units lie in one wave's squares, so h is formed in registers: one read of x for both products, and
// neither product goes to memory unless a backward pass will want it, or the sums are cut into the grid's second axis (few tiles, long sums).
template <class T, class TL, bool DIRECT>
__global__ void __launch_bounds__(TL::NT, 2) tr_ff_forward_kernel(FfForward f)
{
    __shared__ __attribute__((aligned(16))) char lds[TL::LDS];
    constexpr int FM = TL::FM, FN = TL::FN, HALF = FN / 2;
    const u32 tm = (u32)((f.x.index + TL::BM - 1) / TL::BM), tn = (u32)((f.w.index + TL::BN / 2 - 1) / (TL::BN / 2));
    u32 bm, bn;
    tile_of(blockIdx.x, tm, tn, bm, bn);
    const i64 m0 = (i64)bm * TL::BM, n0 = (i64)bn * (TL::BN / 2);
    Float4 acc[FN][FM];
    product_tile<T, TL, ROWS, ROWS, FN, DIRECT>(acc, lds, f.x, f.w, 1, m0, n0, blockIdx.y, f.parts);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const i64 m = m0 + (wm * FM + i) * 16 + (lane & 15);
        if (m >= f.x.index) continue;
#pragma unroll
        for (int j = 0; j < HALF; j += 2) {
            const i64 n = n0 + (wn * HALF + j) * 16;
            const i64 have = f.w.index - n;
            if (have <= 0) continue;
            if (f.parts > 1) {
                const i64 ld = partial_ld(f.w.index), up = f.x.index * ld, at = n + (lane >> 4) * 4;
                float* p = f.partial + (i64)blockIdx.y * 2 * up + m * ld + at;
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (at + 16 * k < ld) {
                        *reinterpret_cast<Float4*>(p + 16 * k) = acc[j + k][i];
                        *reinterpret_cast<Float4*>(p + up + 16 * k) = acc[j + k + HALF][i];
                    }
                continue;
            }
            Float4 h[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) h[k][e] = activation<T>(f.act, acc[j + k][i][e]) * acc[j + k + HALF][i][e];
            store_pair((T*)f.h + m * f.ldh + n, h[0], h[1], have, lane);
            if (f.g) {
                store_pair(f.g + m * f.ldg + n, acc[j][i], acc[j + 1][i], have, lane);
                store_pair(f.u + m * f.ldg + n, acc[j + HALF][i], acc[j + 1 + HALF][i], have, lane);
            }
        }
    }
}

// The parts of gate and up, added up in their order, and what is made of them.
template <class T>
__global__ void __launch_bounds__(256) tr_ff_forward_join_kernel(FfForward f)
{
    const i64 ld = partial_ld(f.w.index), up = f.x.index * ld;
    for (i64 at = (i64)blockIdx.x * 256 + threadIdx.x; at < up / 4; at += (i64)gridDim.x * 256) {
        const i64 m = at / (ld / 4), n = (at - m * (ld / 4)) * 4, have = f.w.index - n;
        const float* p = f.partial + at * 4;
        Float4 g = *reinterpret_cast<const Float4*>(p), u = *reinterpret_cast<const Float4*>(p + up), h;
        for (int part = 1; part < f.parts; ++part) {
            p += 2 * up;
            g += *reinterpret_cast<const Float4*>(p);
            u += *reinterpret_cast<const Float4*>(p + up);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = activation<T>(f.act, g[e]) * u[e];
        store4((T*)f.h + m * f.ldh + n, h, have);
        if (f.g) {
            store4(f.g + m * f.ldg + n, g, have);
            store4(f.u + m * f.ldg + n, u, have);
        }
    }
}

// What the pass that forms dg and du reads and writes.
template <class T>
struct FfUnits {
    const T* dh;
    i64 lddh;
    const float *g, *u;
    i64 ldg;
    T *dg, *du;
    i64 ldd, M, F;
    int act;
    float *largest, *back;                                                   // fp16: see tr_ff_units_kernel
};

constexpr int RANGE_BLOCKS = 2048;                                           // eight workgroups a CU, all resident
constexpr int RANGE_BYTES = RANGE_BLOCKS * 4 + 256;

// dg = dh * u * act'(g) and du = dh * act(g) times `by`, rows padded with zeros to a multiple of 16 bytes; the largest finite size that the
// thread has met, before that product.
template <class T>
__device__ __forceinline__ float form_units(const FfUnits<T>& f, float by)
{
    constexpr int N = PER_WORD4<T>;
    float largest = 0.f;
    const i64 chunks = f.ldd / N, all = f.M * chunks;
    for (i64 at = (i64)blockIdx.x * 256 + threadIdx.x; at < all; at += (i64)gridDim.x * 256) {
        const i64 m = at / chunks, c = (at - m * chunks) * N;
        Pack<T> ph, og, ou;
        Pack<float> pg[N / 4], pu[N / 4];
        ph.raw = load_some(f.dh + m * f.lddh + c, f.F - c);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            pg[i].raw = load_some(f.g + m * f.ldg + c + 4 * i, f.F - c - 4 * i);
            pu[i].raw = load_some(f.u + m * f.ldg + c + 4 * i, f.F - c - 4 * i);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, d;
            activation_both<T>(f.act, pg[i / 4].v[i % 4], a, d);
            const float h = to_float(ph.v[i]);
            const bool in = c + i < f.F;
            const float dg = in ? h * pu[i / 4].v[i % 4] * d : 0.f, du = in ? h * a : 0.f;
            og.v[i] = from_float<T>(dg * by);
            ou.v[i] = from_float<T>(du * by);
            if constexpr (__is_same(T, _Float16)) {
                if (fabsf(dg) <= FLT_MAX) largest = fmaxf(largest, fabsf(dg));
                if (fabsf(du) <= FLT_MAX) largest = fmaxf(largest, fabsf(du));
            }
        }
        *reinterpret_cast<Word4*>(f.dg + m * f.ldd + c) = og.raw;
        *reinterpret_cast<Word4*>(f.du + m * f.ldd + c) = ou.raw;
    }
    return largest;
}

// A value that every thread of 256 has: the largest of theirs.
__device__ __forceinline__ float largest_of_block(float v)
{
    __shared__ float of_wave[4];
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
}

// They are rounded to the inputs' type, which is what the matrix cores multiply; the sums over them stay in 32 bits.  g and u come as
// the forward pass summed them: rounding them too would make the gradients' error 1.8 times that of rounding the results alone, as it is
// 1.4 times.  The range of fp16 does not hold every product of an fp16 and two 32-bit numbers whose sums the results have room for: there the
// pass also leaves every workgroup's largest size for tr_ff_rescale_kernel.
template <class T>
__global__ void __launch_bounds__(256) tr_ff_units_kernel(FfUnits<T> f)
{
    const float largest = form_units(f, 1.f);
    if constexpr (__is_same(T, _Float16)) {
        const float all = largest_of_block(largest);
        if (threadIdx.x == 0) f.largest[blockIdx.x] = all;
    }
}

// fp16: where the largest of dg and du overflows, or lies below 2^-6 (of values a hundredth of it the first are no normal numbers any more), the pass
// runs once more, times the power of two that brings it to 2^14 .. 2^15.  `back` is that power's inverse, for the sums.  Values below 2^-28 of the largest
// lose bits then; no value is off by more than half a step of its own or 2^-39 of the largest.  The look costs a launch and reads some KB (forward and
// gradients, us, without / with it / with the second pass: 512 x 512 x 1024 33 / 38 / -, 1021 x 1000 x 2730 84 / 90 / 95, 8192 x 4096 x 12288 4139 / 4161 / 4411).
__global__ void __launch_bounds__(256) tr_ff_rescale_kernel(FfUnits<_Float16> f, int blocks)
{
    float v = 0.f;
    for (int i = threadIdx.x; i < blocks; i += 256) v = fmaxf(v, f.largest[i]);
    v = largest_of_block(v);
    int up = 0;
    if (v > 65504.f || (v > 0.f && v < 0.015625f)) up = min(14 - ilogbf(v), 100);
    if (blockIdx.x == 0 && threadIdx.x == 0) *f.back = ldexpf(1.f, -up);
    if (up != 0) form_units(f, ldexpf(1.f, up));
}

struct FfGradient {
    Operand a, b;
    void* out[2];                                                            // dWg and dWu, one for each half of the grid; or dx
    i64 ld[2];
    int segments;                                                            // dx: 2, the sum runs over gate and up
    i64 rows;                                                                // of the result (a.index counts the padded ones too)
    float* partial;                                                          // sums in parts: [result][parts][rows][columns, padded to 4]
    int parts, large;                                                        // large: tiles of 256 x 256
    const float* back;                                                       // fp16: what the sums are multiplied by (see tr_ff_rescale_kernel); NULL where they are empty
};

// The sums of dg and du as they are, whatever power of two these came with.
template <class T>
__device__ __forceinline__ Float4 brought_back(Float4 sum, float back)
{
    if constexpr (__is_same(T, _Float16)) sum *= back;
    return sum;
}

// dx = dg Wg + du Wu (A in rows, two segments) and dW = dg^T x, du^T x (A in columns, a half of the grid each).  dx has few tiles and
// long sums where tokens are few, dW where the matrices are small and tokens many; the grid's second axis cuts the sums then, and
// the parts go to memory unrounded.
template <class T, class TL, Layout LA, bool DIRECT>
__device__ __forceinline__ void gradient_tile(const FfGradient& f, u32 tile, int slice, char* lds)
{
    constexpr int FM = TL::FM, FN = TL::FN;
    const u32 tm = (u32)((f.rows + TL::BM - 1) / TL::BM), tn = (u32)((f.b.index + TL::BN - 1) / TL::BN);
    u32 bm, bn;
    tile_of(tile, tm, tn, bm, bn);
    const int parts = f.parts, z = LA == COLS ? slice / parts : 0, part = slice - z * parts;
    const Operand a = {{LA == COLS ? f.a.matrix(z) : f.a.p[0], f.a.p[1]}, {f.a.ld[0], f.a.ld[1]}, f.a.index, f.a.depth};
    const i64 m0 = (i64)bm * TL::BM, n0 = (i64)bn * TL::BN;
    Float4 acc[FN][FM];
    product_tile<T, TL, LA, COLS, 0, DIRECT>(acc, lds, a, f.b, f.segments, m0, n0, part, parts);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
    const float back = __is_same(T, _Float16) && f.back ? *f.back : 1.f;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const i64 m = m0 + (wm * FM + i) * 16 + (lane & 15);
        if (m >= f.rows) continue;
#pragma unroll
        for (int j = 0; j < FN; j += 2) {
            const i64 n = n0 + (wn * FN + j) * 16;
            const i64 have = f.b.index - n;
            if (have <= 0) continue;
            if (parts > 1) {
                const i64 ld = partial_ld(f.b.index);
                float* p = f.partial + (((i64)z * parts + part) * f.rows + m) * ld + n + (lane >> 4) * 4;
                if (n + (lane >> 4) * 4 < ld) *reinterpret_cast<Float4*>(p) = acc[j][i];
                if (n + (lane >> 4) * 4 + 16 < ld) *reinterpret_cast<Float4*>(p + 16) = acc[j + 1][i];
            } else {
                store_pair((T*)f.out[z] + m * f.ld[z] + n, brought_back<T>(acc[j][i], back), brought_back<T>(acc[j + 1][i], back), have, lane);
            }
        }
    }
}

template <class T, class TL, Layout LA, bool DIRECT>
__global__ void __launch_bounds__(TL::NT, 2) tr_ff_gradient_kernel(FfGradient f)
{
    __shared__ __attribute__((aligned(16))) char lds[TL::LDS];
    gradient_tile<T, TL, LA, DIRECT>(f, blockIdx.x, blockIdx.y, lds);
}

// dx and dW side by side, the longer sums first: either alone leaves CUs without work at its end (forward and both gradients, us, one after the
// other / so: bf16 1021 x 1000 x 2730 91 / 85, 2048 x 256 x 1024 50 / 39, 512 x 2048 x 4096 93 / 93; f32 1024 x 1024 x 2816 367 / 337).
template <class T, class TL, bool DIRECT>
__global__ void __launch_bounds__(TL::NT, 2) tr_ff_gradients_kernel(FfGradient x, FfGradient w, u32 x_tiles, u32 x_all, u32 w_tiles, u32 w_first)
{
    __shared__ __attribute__((aligned(16))) char lds[TL::LDS];
    const u32 id = blockIdx.x, id_x = id - w_first, id_w = id - (w_first ? 0 : x_all);   // w_first: how many of dW come before dx's
    if (id_x < x_all) gradient_tile<T, TL, ROWS, DIRECT>(x, id_x % x_tiles, id_x / x_tiles, lds);
    else gradient_tile<T, TL, COLS, DIRECT>(w, id_w % w_tiles, id_w / w_tiles, lds);
}

// The parts of a result, added up in their order and rounded.
template <class T>
__global__ void __launch_bounds__(256) tr_ff_join_kernel(FfGradient f)
{
    const int z = blockIdx.y;
    const i64 columns = f.b.index, ld = partial_ld(columns), all = f.rows * (ld / 4);
    const float* partial = f.partial + (i64)z * f.parts * f.rows * ld;
    const float back = __is_same(T, _Float16) && f.back ? *f.back : 1.f;
    for (i64 at = (i64)blockIdx.x * 256 + threadIdx.x; at < all; at += (i64)gridDim.x * 256) {
        const i64 m = at / (ld / 4), n = (at - m * (ld / 4)) * 4;
        Float4 sum = *reinterpret_cast<const Float4*>(partial + at * 4);
        for (int p = 1; p < f.parts; ++p) sum += *reinterpret_cast<const Float4*>(partial + (p * f.rows * ld + at * 4));
        store4((T*)f.out[z] + m * f.ld[z] + n, brought_back<T>(sum, back), columns - n);
    }
}

// Few tokens: one read of the weights is all there is to it (1 token of 4096 x 12288 in bf16: 201 MB in 37 us, 5.4 TB/s).  They go from memory
// straight to the matrix cores, 128 bytes of a row by each wave in turn; a workgroup has 16 units (gate and up), its waves share the
// contraction and add up through shared memory.  Tokens fill FM squares; those that are not there repeat the last.
template <int FM_>
struct Few {
    static constexpr int FM = FM_, WAVES = 8, NT = WAVES * WAVE, SUMS = 2 * FM;
};

template <class T, class TF, bool GUARD, int HALVES>
__device__ __forceinline__ void few_products(Float4 (&acc)[TF::SUMS], const T* const (&w)[2], const T* const (&x)[TF::FM], i64 k, i64 depth)
{
    constexpr int N = PER_WORD4<T>;
    Word4 rw[HALVES][2], rx[HALVES][TF::FM];
    auto load = [&](const T* p, int h) { return GUARD ? load_some(p + k + h * 4 * N, depth - k - h * 4 * N) : load_loose(p + k + h * 4 * N); };
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        // (k counts from the lane's own position; a wave's steps lie WAVES x 128 bytes apart, the halves of one side by side)
#pragma unroll
        for (int j = 0; j < 2; ++j) rw[h][j] = load(w[j], h % 2 + h / 2 * 2 * TF::WAVES);
#pragma unroll
        for (int i = 0; i < TF::FM; ++i) rx[h][i] = load(x[i], h % 2 + h / 2 * 2 * TF::WAVES);
    }
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < TF::FM; ++i) square_product<T>(acc[j * TF::FM + i], rw[h][j], rx[h][i]);
}

template <class T, class TF>
__global__ void __launch_bounds__(TF::NT, 4) tr_ff_few_kernel(FfForward f)
{
    constexpr int FM = TF::FM, W = TF::WAVES, SUMS = TF::SUMS, N = PER_WORD4<T>;
    constexpr int STEP = 8 * N, HALVES = FM == 1 ? 8 : 4;                    // a step: 128 bytes of a row
    __shared__ Float4 part[W / 2][SUMS][WAVE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const i64 n0 = (i64)blockIdx.x * 16, m0 = (i64)blockIdx.y * (FM * 16);
    const i64 unit = min(n0 + (lane & 15), f.w.index - 1);
    const T *w[2] = {(const T*)f.w.p[0] + unit * f.w.ld[0], (const T*)f.w.p[1] + unit * f.w.ld[1]}, *x[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) x[i] = (const T*)f.x.p[0] + min(m0 + i * 16 + (lane & 15), f.x.index - 1) * f.x.ld[0];
    Float4 acc[SUMS];
#pragma unroll
    for (int i = 0; i < SUMS; ++i) acc[i] = Float4{0, 0, 0, 0};
    const i64 depth = f.x.depth;
    i64 k = (i64)wave * STEP;                                                // the same for the whole wave
    const int mine = (lane >> 4) * N;
    constexpr i64 BATCH = (i64)(HALVES / 2 - 1) * W * STEP + STEP;           // from a wave's first step to behind its last
    for (; k + BATCH <= depth; k += HALVES / 2 * W * STEP) few_products<T, TF, false, HALVES>(acc, w, x, k + mine, depth);
    for (; k + STEP <= depth; k += W * STEP) few_products<T, TF, false, 2>(acc, w, x, k + mine, depth);
    if (k < depth) few_products<T, TF, true, 2>(acc, w, x, k + mine, depth);
    // Half of the waves hand their sums to the others, those put theirs beside each other, and the squares are shared out.
    if (wave >= W / 2)
#pragma unroll
        for (int i = 0; i < SUMS; ++i) part[wave - W / 2][i][lane] = acc[i];
    __syncthreads();
    if (wave < W / 2)
#pragma unroll
        for (int i = 0; i < SUMS; ++i) part[wave][i][lane] += acc[i];
    __syncthreads();
    if (wave < FM) {
        const i64 m = m0 + wave * 16 + (lane & 15), n = n0 + (lane >> 4) * 4, have = f.w.index - n;
        if (m >= f.x.index || have <= 0) return;
        Float4 g = part[0][wave][lane], u = part[0][FM + wave][lane], h;
#pragma unroll
        for (int p = 1; p < W / 2; ++p) {
            g += part[p][wave][lane];
            u += part[p][FM + wave][lane];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = activation<T>(f.act, g[e]) * u[e];
        store4((T*)f.h + m * f.ldh + n, h, have);
        if (f.g) {
            store4(f.g + m * f.ldg + n, g, have);
            store4(f.u + m * f.ldg + n, u, have);
        }
    }
}

}  // namespace
