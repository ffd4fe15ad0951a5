// The gated feed-forward block: h = act(x Wg^T) * (x Wu^T), and its backward pass.
// Part of the ZipLine library (see training.hip); device code for gfx950.
#pragma once
#include "ebsp_training.h"
#include "tr_product.h"

namespace {

// act(g) and act'(g).  The activation is chosen by a value that is the same for the whole launch.
// (The hardware's exponential and reciprocal are good to an ulp.)
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)); }

__device__ __forceinline__ float activation(int act, float g)
{
    switch (act) {
    case EBSP_ACT_SILU: return g * sigmoid(g);
    case EBSP_ACT_SIGMOID: return sigmoid(g);
    case EBSP_ACT_RELU: return g < 0.f ? 0.f : g;                            // (a NaN stays one)
    case EBSP_ACT_GELU: return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
    default: {                                                               // 0.5 g (1 + tanh z) = g sigmoid(2 z)
        const float c = fminf(fmaxf(g, -16.f), 16.f);                        // tanh is 1 long before; the cube stays finite
        const float z = 0.79788456080286536f * (c + 0.044715f * c * c * c);
        return g * sigmoid(2.f * z);
    }
    }
}

__device__ __forceinline__ void activation_both(int act, float g, float& a, float& d)
{
    switch (act) {
    case EBSP_ACT_SILU: {
        const float s = sigmoid(g);
        a = g * s;
        d = s * (1.f + g * (1.f - s));
        break;
    }
    case EBSP_ACT_SIGMOID: {
        a = sigmoid(g);
        d = a * (1.f - a);
        break;
    }
    case EBSP_ACT_RELU:
        a = g < 0.f ? 0.f : g;
        d = g > 0.f ? 1.f : 0.f;
        break;
    case EBSP_ACT_GELU: {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        a = g * cdf;
        d = cdf + g * 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g);
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
    int act, wide_h, wide_g;
};

// Gate and up of the same units lie in one wave's squares, so h is formed in registers: one read of x for both products, and
// neither product goes to memory unless a backward pass will want it.
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
    product_tile<T, TL, ROWS, ROWS, FN, DIRECT>(acc, lds, f.x, f.w, 1, m0, n0);
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
            Float4 h[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) h[k][e] = activation(f.act, acc[j + k][i][e]) * acc[j + k + HALF][i][e];
            store_pair((T*)f.h + m * f.ldh + n, h[0], h[1], have, f.wide_h, lane);
            if (f.g) {
                store_pair(f.g + m * f.ldg + n, acc[j][i], acc[j + 1][i], have, f.wide_g, lane);
                store_pair(f.u + m * f.ldg + n, acc[j + HALF][i], acc[j + 1 + HALF][i], have, f.wide_g, lane);
            }
        }
    }
}

// dg = dh * u * act'(g) and du = dh * act(g), rows padded with zeros to a multiple of 16 bytes.  They are rounded to the inputs' type,
// which is what the matrix cores multiply; the sums over them stay in 32 bits.  g and u come as the forward pass summed them: rounding
// them too would make the gradients' error 1.8 times that of rounding the results alone, as it is 1.4 times.
template <class T>
__global__ void __launch_bounds__(256) tr_ff_units_kernel(const T* dh, i64 lddh, const float* g, const float* u, i64 ldg, T* dg, T* du, i64 ldd,
                                                          i64 M, i64 F, int act)
{
    constexpr int N = PER_WORD4<T>;
    const i64 chunks = ldd / N, all = M * chunks;
    for (i64 at = (i64)blockIdx.x * 256 + threadIdx.x; at < all; at += (i64)gridDim.x * 256) {
        const i64 m = at / chunks, f = (at - m * chunks) * N;
        Pack<T> ph, og, ou;
        Pack<float> pg[N / 4], pu[N / 4];
        ph.raw = load_some(dh + m * lddh + f, F - f);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            pg[i].raw = load_some(g + m * ldg + f + 4 * i, F - f - 4 * i);
            pu[i].raw = load_some(u + m * ldg + f + 4 * i, F - f - 4 * i);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float a, d;
            activation_both(act, pg[i / 4].v[i % 4], a, d);
            const float h = to_float(ph.v[i]);
            const bool in = f + i < F;
            og.v[i] = from_float<T>(in ? h * pu[i / 4].v[i % 4] * d : 0.f);
            ou.v[i] = from_float<T>(in ? h * a : 0.f);
        }
        *reinterpret_cast<Word4*>(dg + m * ldd + f) = og.raw;
        *reinterpret_cast<Word4*>(du + m * ldd + f) = ou.raw;
    }
}

struct FfGradient {
    Operand a, b;
    void* out[2];                                                            // dWg and dWu, one for each half of the grid; or dx
    i64 ld[2];
    int wide[2];
    int segments;                                                            // dx: 2, the sum runs over gate and up
    i64 rows;                                                                // of the result (a.index counts the padded ones too)
};

// dx = dg Wg + du Wu (A in rows, two segments) and dW = dg^T x, du^T x (A in columns, a half of the grid each).
template <class T, class TL, Layout LA, bool DIRECT>
__global__ void __launch_bounds__(TL::NT, 2) tr_ff_gradient_kernel(FfGradient f)
{
    __shared__ __attribute__((aligned(16))) char lds[TL::LDS];
    constexpr int FM = TL::FM, FN = TL::FN;
    const u32 tm = (u32)((f.rows + TL::BM - 1) / TL::BM), tn = (u32)((f.b.index + TL::BN - 1) / TL::BN);
    u32 bm, bn;
    tile_of(blockIdx.x, tm, tn, bm, bn);
    const int z = blockIdx.y;
    const Operand a = {{LA == COLS ? f.a.matrix(z) : f.a.p[0], f.a.p[1]}, {f.a.ld[0], f.a.ld[1]}, f.a.index, f.a.depth};
    const i64 m0 = (i64)bm * TL::BM, n0 = (i64)bn * TL::BN;
    Float4 acc[FN][FM];
    product_tile<T, TL, LA, COLS, 0, DIRECT>(acc, lds, a, f.b, f.segments, m0, n0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const i64 m = m0 + (wm * FM + i) * 16 + (lane & 15);
        if (m >= f.rows) continue;
#pragma unroll
        for (int j = 0; j < FN; j += 2) {
            const i64 n = n0 + (wn * FN + j) * 16;
            const i64 have = f.b.index - n;
            if (have > 0) store_pair((T*)f.out[z] + m * f.ld[z] + n, acc[j][i], acc[j + 1][i], have, f.wide[z], lane);
        }
    }
}

}  // namespace
