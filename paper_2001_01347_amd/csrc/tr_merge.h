// The merge of the workers' pushes at a barrier, weighted by their iterations.
// Part of the ZipLine library (see training.hip); device code for gfx950.
//
//     c_p = iters_p / sum iters      avg = sum_p c_p push_p
//     v' = momentum v + avg          w' = w + lr (nesterov ? avg + momentum v' : v')
// One pass over the pushes, read once and in the order of the workers, whatever the launch: results do not vary.
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

template <class U, int N>
__device__ __forceinline__ void store_pull(U* p, const float (&w)[N], i64 have)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have) p[i] = from_float<U>(w[i]);
}

template <class T>
__global__ void __launch_bounds__(256) tr_merge_kernel(Merge g)
{
    extern __shared__ Share list[];
    __shared__ int shared;
    constexpr int N = PER_WORD4<T>, AHEAD = 8;
    const int count = list_shares<256>(g, list, &shared);
    const i64 at = ((i64)blockIdx.x * 256 + threadIdx.x) * N;
    if (at >= g.n) return;
    const i64 have = g.n - at;
    float avg[N];
#pragma unroll
    for (int i = 0; i < N; ++i) avg[i] = 0.f;
    const T* base = (const T*)g.pushes + at;
    for (int k0 = 0; k0 < count; k0 += AHEAD) {
        Pack<T> w[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k0 + k < count) w[k].raw = load_some(base + list[k0 + k].worker * g.stride, have);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k0 + k < count) {
                const float c = list[k0 + k].c;
#pragma unroll
                for (int i = 0; i < N; ++i) avg[i] = fmaf(c, to_float(w[k].v[i]), avg[i]);
            }
    }
    float out[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i >= have) continue;
        float step = avg[i];
        if (g.velocity) {
            const float old = g.velocity[at + i];
            const float v = count > 0 ? fmaf(g.momentum, old, avg[i]) : old;  // a barrier without pushes changes nothing
            g.velocity_out[at + i] = v;
            step = g.nesterov ? fmaf(g.momentum, v, avg[i]) : v;
        }
        const float w = g.weights[at + i];
        out[i] = count > 0 ? fmaf(g.lr, step, w) : w;
        g.out[at + i] = out[i];
    }
    if (g.pull) {
        if (g.pull_type == EBSP_BF16) store_pull((__bf16*)g.pull + at, out, have);
        else if (g.pull_type == EBSP_F16) store_pull((_Float16*)g.pull + at, out, have);
        else store_pull((float*)g.pull + at, out, have);
    }
}

}  // namespace
