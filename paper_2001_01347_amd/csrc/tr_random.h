// Random bits from a counter: which elements a dropout keeps, computed wherever they are needed and stored nowhere.
// Part of the ZipLine library (see tuning.hip); device code for gfx950.
//
// Philox4x32 of seven rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): a round multiplies
// two of the counter's four words by constants to 64 bits and mixes the halves with the others and the key.  Element k of row r takes 16 of the 128 bits of the
// counter (k / 8, r, offset) under the key (seed), the halves of the four words from low to high: eight neighbours of a row, which a thread holds anyway, share one.
#pragma once
#include "tr_common.h"

namespace {

struct Random {
    uint64_t seed, offset;
    const i64* place;                            // the two on the device, or NULL: the numbers above
    u32 threshold;                               // elements whose 16 bits are below are dropped
    float kept;                                  // what the others are multiplied by
};

struct Generator {
    u32 k0, k1, o0, o1;
};

__device__ __forceinline__ Generator generator(const Random& r)
{
    const uint64_t seed = r.place ? (uint64_t)r.place[0] : r.seed, offset = r.place ? (uint64_t)r.place[1] : r.offset;
    return Generator{(u32)seed, (u32)(seed >> 32), (u32)offset, (u32)(offset >> 32)};
}

// A bit for each of the eight elements from 8 unit on: set where it is kept.
__device__ __forceinline__ u32 keep_bits(const Generator& g, u32 threshold, u32 unit, u32 row)
{
    u32 c0 = unit, c1 = row, c2 = g.o0, c3 = g.o1, k0 = g.k0, k1 = g.k1;
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (u32)(b >> 32) ^ c1 ^ k0;
        c1 = (u32)b;
        c2 = (u32)(a >> 32) ^ c3 ^ k1;
        c3 = (u32)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const u32 c[4] = {c0, c1, c2, c3};
    u32 bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= (c[i] & 0xffffu) >= threshold ? 1u << (2 * i) : 0u;
        bits |= c[i] >> 16 >= threshold ? 2u << (2 * i) : 0u;
    }
    return bits;
}

}  // namespace
