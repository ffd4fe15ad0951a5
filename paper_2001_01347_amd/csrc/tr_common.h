// Element types, conversions and wave primitives of the training operators.
// Part of the ZipLine library (see training.hip); device code for gfx950.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <float.h>

typedef int64_t i64;
typedef uint32_t u32;

typedef int Word4 __attribute__((ext_vector_type(4), may_alias));            // 16 bytes, the unit of every wide access
typedef Word4 LooseWord4 __attribute__((aligned(2), may_alias));             // the same at any element's address: global memory takes it
typedef int Word2 __attribute__((ext_vector_type(2), may_alias));
typedef Word2 LooseWord2 __attribute__((aligned(2), may_alias));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
typedef short Short4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int WAVE = 64;

// Elements of 16 bytes, as floats.
template <class T> constexpr int PER_WORD4 = 16 / (int)sizeof(T);

template <class T>
union Pack {
    Word4 raw;
    T v[16 / sizeof(T)];
};

// Rounded to nearest, ties to even: the one rounding of a result.
template <class T> __device__ __forceinline__ T from_float(float x) { return (T)x; }
template <class T> __device__ __forceinline__ float to_float(T x) { return (float)x; }

template <class T>
__device__ __forceinline__ Word4 load_loose(const T* p)
{
    return *reinterpret_cast<const LooseWord4*>(p);
}
template <class T>
__device__ __forceinline__ void store_loose(T* p, Word4 v)
{
    *reinterpret_cast<LooseWord4*>(p) = v;
}

// Up to 16 bytes from p: `have` elements exist (any number, also none or more than fit), the others read as zero.
template <class T>
__device__ __forceinline__ Word4 load_some(const T* p, i64 have)
{
    constexpr int N = PER_WORD4<T>;
    if (have >= N) return load_loose(p);
    Pack<T> w;
    w.raw = Word4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have) w.v[i] = p[i];
    return w.raw;
}

}  // namespace
