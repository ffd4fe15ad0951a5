// The merge of the workers' pushes at a barrier, weighted by their iterations.
// Part of the ZipLine library (see training.hip); device code for gfx950.
//
//     c_p = iters_p / sum iters      avg = sum_p c_p push_p
//     v' = momentum v + avg          w' = w + lr (nesterov ? avg + momentum v' : v')
// One pass over the pushes, each read once, in an order that depends on the sizes alone: results do not vary.  Bound by memory: for n
// weights of 16-bit pushes 2 P n bytes and 8 to 18 n around them.
#pragma once
#include "ebsp_training.h"
#include "tr_common.h"

namespace {

struct Merge {
    const void* pushes;
    i64 stride, n;
    const int* iters;
    const float *weights, *velocity;
    float *out, *velocity_out;
    void* pull;
    int P, pull_type, nesterov;
    float lr, momentum;
};

struct Share {                                   // a worker that has a part in the merge
    int worker;
    float c;
};

// The workers with iterations, in order, and their shares; how many there are.
template <int NT>
__device__ __forceinline__ int list_shares(const Merge& g, Share* list, int* shared)
{
    __shared__ double total_part[NT / WAVE];
    double sum = 0;                                                          // whole numbers below 2^53: exact
    for (int p = threadIdx.x; p < g.P; p += NT) sum += g.iters[p] > 0 ? g.iters[p] : 0;
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) total_part[threadIdx.x >> 6] = sum;
    __syncthreads();
    double total = 0;
    for (int w = 0; w < NT / WAVE; ++w) total += total_part[w];
    if (threadIdx.x < WAVE) {
        int at = 0;
        for (int p0 = 0; p0 < g.P; p0 += WAVE) {
            const int p = p0 + threadIdx.x, it = p < g.P ? g.iters[p] : 0;
            const unsigned long long in = __ballot(it > 0);
            if (it > 0) list[at + __popcll(in & ((1ull << threadIdx.x) - 1))] = Share{p, (float)(it / total)};
            at += __popcll(in);
        }
        if (threadIdx.x == 0) *shared = at;
    }
    __syncthreads();
    return *shared;
}

// The sum of worker list[k]'s share times its push for k from k0 up to k1, for the N elements from `at` on (WHOLE; otherwise those behind `have` read as
// zero).  AHEAD rows are under way at a time; where a row is, every lane knows alike.
template <class T, bool WHOLE>
__device__ __forceinline__ void add_pushes(float (&avg)[PER_WORD4<T>], const Merge& g, const Share* list, int k0, int k1, i64 at, i64 have)
{
    constexpr int N = PER_WORD4<T>, AHEAD = 8;
    auto row = [&](int k) {
        const T* p = (const T*)g.pushes + (i64)__builtin_amdgcn_readfirstlane(list[k].worker) * g.stride + at;
        return WHOLE ? load_loose(p) : load_some(p, have);
    };
    auto add = [&](Word4 raw, int k) {
        Pack<T> w;
        w.raw = raw;
        const float c = list[k].c;
#pragma unroll
        for (int i = 0; i < N; ++i) avg[i] = fmaf(c, to_float(w.v[i]), avg[i]);
    };
    int k = k0;
    for (; k + AHEAD <= k1; k += AHEAD) {
        Word4 w[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) w[j] = row(k + j);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) add(w[j], k + j);
    }
    if (k < k1) {                                                            // what is left, once more all together
        Word4 w[AHEAD - 1];
#pragma unroll
        for (int j = 0; j < AHEAD - 1; ++j)
            if (k + j < k1) w[j] = row(k + j);
#pragma unroll
        for (int j = 0; j < AHEAD - 1; ++j)
            if (k + j < k1) add(w[j], k + j);
    }
}

template <class U, int N, bool WHOLE>
__device__ __forceinline__ void store_row(U* p, const float (&v)[N], i64 have)
{
    constexpr int PER = PER_WORD4<U> < N ? PER_WORD4<U> : N;
#pragma unroll
    for (int j = 0; j < N; j += PER) {
        union { U v[PER]; Word2 two; Word4 four; } r;
#pragma unroll
        for (int i = 0; i < PER; ++i) r.v[i] = from_float<U>(v[j + i]);
        if constexpr (WHOLE) {
            if constexpr (sizeof(U) * PER == 16) store_loose(p + j, r.four);
            else *reinterpret_cast<LooseWord2*>(p + j) = r.two;
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (j + i < have) p[j + i] = r.v[i];
        }
    }
}

template <int N, bool WHOLE>
__device__ __forceinline__ void load_row(float (&v)[N], const float* p, i64 have)
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        Pack<float> w;
        w.raw = WHOLE ? load_loose(p + j) : load_some(p + j, have - j);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j + i] = w.v[i];
    }
}

// The step from the merged pushes of N weights at `at`.
template <int N, bool WHOLE>
__device__ __forceinline__ void apply_step(const Merge& g, float (&avg)[N], i64 at, i64 have, bool any)
{
    float w[N], v[N];
    load_row<N, WHOLE>(w, g.weights + at, have);
    if (g.velocity) {
        load_row<N, WHOLE>(v, g.velocity + at, have);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (any) v[i] = fmaf(g.momentum, v[i], avg[i]);                  // a barrier without pushes changes nothing
            avg[i] = g.nesterov ? fmaf(g.momentum, v[i], avg[i]) : v[i];
        }
        store_row<float, N, WHOLE>(g.velocity_out + at, v, have);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (any) w[i] = fmaf(g.lr, avg[i], w[i]);
    store_row<float, N, WHOLE>(g.out + at, w, have);
    if (g.pull) {
        if (g.pull_type == EBSP_BF16) store_row<__bf16, N, WHOLE>((__bf16*)g.pull + at, w, have);
        else if (g.pull_type == EBSP_F16) store_row<_Float16, N, WHOLE>((_Float16*)g.pull + at, w, have);
        else store_row<float, N, WHOLE>((float*)g.pull + at, w, have);
    }
}

// 16 bytes of a row a lane.  SPLIT > 1: each wave of a workgroup takes a part of the workers for the same 64 chunks, and the first adds the parts up in
// their order.  The lane of the last, partial chunk reads the last 16 bytes of the rows and moves its sums afterwards: element by element
// that one lane would take longer than all others together (435 in place of 200 us at 1024 workers x 524309 weights).
template <class T, int SPLIT>
__global__ void __launch_bounds__(SPLIT == 1 ? 256 : SPLIT * 64) tr_merge_kernel(Merge g)
{
    extern __shared__ Share list[];
    __shared__ int shared;
    constexpr int N = PER_WORD4<T>, NT = SPLIT == 1 ? 256 : SPLIT * 64;
    const int count = list_shares<NT>(g, list, &shared);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const i64 at = ((i64)blockIdx.x * (SPLIT == 1 ? NT : 64) + (SPLIT == 1 ? (int)threadIdx.x : lane)) * N, have = g.n - at;
    float avg[N];
#pragma unroll
    for (int i = 0; i < N; ++i) avg[i] = 0.f;
    const int k0 = SPLIT == 1 ? 0 : wave * count / SPLIT, k1 = SPLIT == 1 ? count : (wave + 1) * count / SPLIT;
    if (g.n >= N) {
        if (have > 0) add_pushes<T, true>(avg, g, list, k0, k1, have < N ? g.n - N : at, N);
    } else if (have > 0) {
        add_pushes<T, false>(avg, g, list, k0, k1, at, have);
    }
    if constexpr (SPLIT > 1) {
        __shared__ float part[SPLIT - 1][N][64];
        if (wave > 0)
#pragma unroll
            for (int i = 0; i < N; ++i) part[wave - 1][i][lane] = avg[i];
        __syncthreads();
        if (wave > 0) return;
        for (int p = 0; p < SPLIT - 1; ++p)
#pragma unroll
            for (int i = 0; i < N; ++i) avg[i] += part[p][i][lane];
    }
    if (have >= N) {
        apply_step<N, true>(g, avg, at, have, count > 0);
    } else if (have > 0) {
        if (g.n >= N)
            for (int moves = N - (int)have; moves > 0; --moves)
#pragma unroll
                for (int i = 0; i < N - 1; ++i) avg[i] = avg[i + 1];
        apply_step<N, false>(g, avg, at, have, count > 0);
    }
}

}  // namespace
