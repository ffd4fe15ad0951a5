// Rows of logits: what the losses over a vocabulary share.
// Part of the ZipLine library (see training.hip, tuning.hip); device code for gfx950.
#pragma once
#include "tr_common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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

// The larger of two, or the one that is no number: a NaN among a row's entries comes through, its results are not those of the others.
__device__ __forceinline__ float larger(float a, float b) { return a > b || a != a ? a : b; }

// log2 of a sum, for differences from m; of a row without any finite logit it is taken as 0, so its p are 0.
__device__ __forceinline__ float log2_sum(float s) { return s == 0.f ? 0.f : log2f(s); }

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

template <class T>
__device__ __forceinline__ float largest(Word4 raw, float m)
{
    Pack<T> w;
    w.raw = raw;
#pragma unroll
    for (int i = 0; i < PER_WORD4<T>; ++i) m = fmaxf(m, to_float(w.v[i]));
    return m;
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

// Packed words stay packed: without this the compiler keeps the floats of one use for the next, twice the registers.
template <int N>
__device__ __forceinline__ void forget_floats(Word4 (&w)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(w[j]));
}

}  // namespace
