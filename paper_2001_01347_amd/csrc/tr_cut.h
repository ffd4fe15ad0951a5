// How the gated feed-forward block is cut up: which kernel, tiles of what size, sums in how many parts.  Rules on sizes alone.
// Part of the ZipLine library (see training.hip); host code that needs no GPU.
#pragma once
#include <stdint.h>

typedef int64_t i64;

namespace {

inline i64 tiles_of(i64 m, i64 n, int bm, int bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); }

// Tiles of 256 x 256 and not of 128 x 128, of which there would be so many: a large one takes 3.2 times as long as a small one (4 times in 32 bits; 2.8
// times where the sum is long and the last round leaves CUs idle), and either fills the CUs in whole rounds.  us, large / small (M x K x F), bf16: forward 8192 x 2048 x 12288 642 / 795, 8192 x 1024 x 2048 67 / 77, 2126 x 768 x 4160
// 48 / 39, 1169 x 2624 x 8936 117 / 128, 1877 x 1759 x 4592 168 / 136, 2812 x 64 x 3200 25 / 20; dx 8192 x 4096 x 512 78 / 98; dW 1024 x 4096 x 12288 228 / 262; fp32 forward
// 3000 x 512 x 4096 246 / 191.
inline bool large_tiles(i64 large, i64 small, i64 steps, int size)
{
    const i64 large_rounds = (large + 255) / 256, small_rounds = (small + 255) / 256;
    return large >= 192 && large_rounds * (size == 4 ? 20 : steps >= 32 ? 14 : 16) <= small_rounds * 5;
}

// How the forward pass is cut up.
struct ForwardCut {
    int few;                                                                 // squares of 16 tokens of the kernel for few of them, or 0: tiles
    bool large;                                                              // tiles of 256 x 128, not 128 x 64
    int parts;                                                               // of every sum
};

// Tiles want a CU each and long sums.  Where they would be few, either the kernel that shares a sum out among its waves runs, or the sums are cut into
// parts (`room`: there is a workspace for them).  us, that kernel / tiles in parts / whole ones (M x K x F), bf16: 16 x 4096 x 2048 13 / 14 / 33,
// 64 x 1024 x 4096 10 / 14 / 14, 341 x 3984 x 286 15 / 18 / 42, 341 x 3981 x 286 (rows at any alignment) 43 / 25 / 68, 64 x 4096 x 4096 28 / 21 / 43,
// 192 x 4096 x 1024 24 / 17 / 35, 100 x 4096 x 3000 43 / 20 / 42, 657 x 3392 x 936 55 / 23 / 31, 300 x 1024 x 2000 19 / 16 / 14; fp32: 64 x 4096 x 4096
// 61 / 72 / 248, 300 x 512 x 512 10 / 18 / 36, 256 x 1024 x 2816 48 / 44 / 67, 600 x 2048 x 1024 88 / 63 / 127, 384 x 4096 x 4096 354 / 198 / 252.  The kernel's
// squares hold 64 tokens, or 32 where that makes too few workgroups (64 x 4096 x 1024 18, so 24).  The rule knows sizes alone, as the workspace is asked for by
// them: rows of whole 16-byte chunks that a view puts at other addresses or distances are taken for aligned, and can run as the 43 of the pair above where tiles in parts
// would take 25.
inline ForwardCut forward_cut(i64 M, i64 K, i64 F, int size, bool room)
{
    const i64 groups = tiles_of(M, F, 64, 16), tiles = tiles_of(M, F, 128, 64), steps = (K * size + 127) / 128;
    const bool wide = size == 4;
    int parts = 1;
    if (room && steps >= (wide ? 16 : 32) && tiles <= (wide ? 208 : 128)) {
        const i64 wanted = (wide ? 768 : 256) / tiles;
        parts = (int)(wanted < steps / 8 ? wanted : steps / 8);
    }
    const bool aligned_rows = K * size % 16 == 0;
    const i64 most = wide ? (parts > 1 ? 192 : 768) : parts == 1 ? 352 : aligned_rows ? 128 : 32;
    if (M <= 16) return {1, false, 1};
    if (groups <= most || (wide && M <= 64)) return {M <= 32 || groups <= 128 ? 2 : 4, false, 1};
    return {0, large_tiles(tiles_of(M, F, 256, 128), tiles, steps, size), parts};
}

// How a gradient of `rows` x `columns` is cut up, `z` of them in one launch, each a sum of `steps` steps of 128 bytes.
struct Cut {
    bool large;                                                              // tiles of 256 x 256, not 128 x 128
    int parts;                                                               // of every sum
};

// A CU for every tile, or for every part of one.  us, large tiles in parts / small ones in parts / small ones whole: dx 2048 x 2048 x 8192 bf16 (64
// large tiles, 256 steps) 164 / 180 / 192, 512 x 4096 x 12288 (32, 384) 115 / 141 / 247, 1024 x 4096 x 2048 (64, 64) 58 / 58 / 52, 1 x 4096 x 12288 (32
// small, 384) 66 / 45 / 224, f32 1024 x 1024 x 2816 (64 small, 176) 189 / 112 / 361; dW 8192 x 1024 x 2048 (64, 128) 112 / 127 / 123.
// Twice as many parts in 32 bits where sums are long: both gradients end together (1024 x 1024 x 2816 355 -> 337; with sums of 64 steps, 1024 x 1024 x 1024, 133 -> 144).
inline Cut gradient_cut(i64 rows, i64 columns, int z, i64 steps, int size)
{
    const i64 large = tiles_of(rows, columns, 256, 256) * z, small = tiles_of(rows, columns, 128, 128) * z;
    if (large_tiles(large, small, steps, size) || small == 0) return {true, 1};
    if (large >= 32 && large < 192 && steps * large >= 32 * 256) return {true, (int)(256 / large)};
    if (small >= 192 || steps < (size == 4 ? 8 : 24)) return {false, 1};
    const i64 parts = (size == 4 && small >= 64 && steps >= 128 ? 512 : 256) / small, most = size == 4 ? steps / 4 : steps / 8;
    return {false, (int)(parts < most ? parts : most)};
}

inline Cut dx_cut(i64 M, i64 K, i64 F, int size) { return gradient_cut(M, K, 1, 2 * ((F * size + 127) / 128), size); }
inline Cut dw_cut(i64 M, i64 K, i64 F, int size) { return gradient_cut(F, K, 2, (M * size + 127) / 128, size); }

}  // namespace
