// Tiles of matrix products in registers, shared memory and the matrix cores: D[m][n] = sum_k A(m, k) B(n, k).
// Part of the ZipLine library (see training.hip); device code for gfx950.
//
// A workgroup computes a BM x BN tile of D; its WM x WN waves hold FM x FN squares of 16 x 16 each.  A step takes 128 bytes
// of the contraction (64 16-bit or 32 32-bit elements) of every row of both operands through shared memory, two steps'
// worth of which lie there: one is multiplied while the next arrives.
//
// An operand lies in memory in one of two ways, whichever way the caller's matrices give it: ROWS (the contraction is
// contiguous: x and W in x W^T) or COLS (the index is contiguous: W in dg W, both in dg^T x).  ROWS tiles are read from
// shared memory 16 bytes a lane; COLS tiles through the transposing read, four rows of the contraction at a time (32-bit
// elements one by one: their products take sixteen times as long anyway).  Both are laid out so that the lanes of a read
// fall into different banks: position s of row r holds what belongs to position s ^ f(r).
//
// B's rows are the first operand of the matrix instruction, so a lane ends up with four neighbouring n of one m.
// Sums are held in 32 bits from the first product to the epilogue.
#pragma once
#include "tr_common.h"

namespace {

enum Layout { ROWS, COLS };

template <class T, int WM_, int WN_, int FM_, int FN_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 16, BN = WN * FN * 16, NT = WM * WN * WAVE;
    static constexpr int BK = 128 / (int)sizeof(T);
    static constexpr int LDS = 2 * (BM + BN) * 128;
};

// One operand: `index` rows of D's axis, `depth` of the contraction, `ld` elements from a row in memory to the next.
// Two matrices where the contraction runs through both (dx), or where their rows alternate in a tile (gate and up).
struct Operand {
    const void* p[2];
    i64 ld[2];
    i64 index, depth;
};

// Where 16-byte position `pos` of an operand's tile comes from: `row` of the tile in memory, `chunk` of 16 bytes in it.
template <class T, Layout L, int BI>
__device__ __forceinline__ void tile_source(int pos, int& row, int& chunk)
{
    if constexpr (L == ROWS) {
        row = pos >> 3;
        chunk = (pos & 7) ^ (row & 7);
    } else {
        constexpr int SLOTS = BI * (int)sizeof(T) / 16;
        row = pos / SLOTS;
        const int slot = pos % SLOTS;
        if constexpr (sizeof(T) == 2) {
            const int f = ((row & 3) | (((row >> 3) & 3) << 2)) & (SLOTS / 2 - 1);
            chunk = slot ^ (f << 1);
        } else {
            chunk = slot ^ (((row >> 2) & 3) << 2);
        }
    }
}

// The row of memory and the matrix that row `row` of a tile of alternating matrices takes: every wave's share is half the one, half
// the other.
template <int FN>
__device__ __forceinline__ int paired_row(int row, int& which)
{
    const int q = row % (FN * 16);
    which = q >= FN * 8;
    return row / (FN * 16) * (FN * 8) + (which ? q - FN * 8 : q);
}

// The 16 bytes of position `pos`, through registers; what lies outside the operand reads as zero.  WHOLE: chunks lie inside or
// outside as a whole, at multiples of 16 bytes; otherwise whatever the alignment.
template <class T, Layout L, int BI, int PAIRED, bool WHOLE>
__device__ __forceinline__ Word4 fetch_chunk(const Operand& o, int which, i64 i0, i64 k0, int pos)
{
    int row, chunk;
    tile_source<T, L, BI>(pos, row, chunk);
    constexpr int N = PER_WORD4<T>;
    if constexpr (L == ROWS) {
        if constexpr (PAIRED > 0) row = paired_row<PAIRED>(row, which);
        const i64 i = i0 + row, k = k0 + chunk * N;
        const T* p = (const T*)o.p[which] + i * o.ld[which] + k;
        if constexpr (WHOLE) return i < o.index && k < o.depth ? *reinterpret_cast<const Word4*>(p) : Word4{0, 0, 0, 0};
        return i < o.index ? load_some(p, o.depth - k) : Word4{0, 0, 0, 0};
    } else {
        const i64 k = k0 + row, i = i0 + chunk * N;
        const T* p = (const T*)o.p[which] + k * o.ld[which] + i;
        if constexpr (WHOLE) return i < o.index && k < o.depth ? *reinterpret_cast<const Word4*>(p) : Word4{0, 0, 0, 0};
        return k < o.depth ? load_some(p, o.index - i) : Word4{0, 0, 0, 0};
    }
}

// The same tile straight from memory to shared memory, no registers between: the shared side of such a load is 16 bytes a lane in
// lane order, so the lanes' order is permuted on the memory side.  Rows (columns) beyond the operand repeat its last ones; what comes
// of them is not stored.  Needs whole 16-byte chunks: operand_direct() on the host.
template <class T, Layout L, int BI, int NT, int PAIRED>
struct DirectTile {
    static constexpr int P = BI * 8 / NT, N = PER_WORD4<T>;
    const char* base[2];
    i64 step;                                                                // bytes to the next step's part
    u32 off[P];

    __device__ __forceinline__ void init(const Operand& o, i64 i0)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            int row, chunk, which = 0;
            tile_source<T, L, BI>(i * NT + (int)threadIdx.x, row, chunk);
            if constexpr (L == ROWS) {
                if constexpr (PAIRED > 0) row = paired_row<PAIRED>(row, which);
                const i64 last = o.index - 1 - i0;
                off[i] = (u32)((i64)(row < last ? row : last) * o.ld[which] * (i64)sizeof(T)) + chunk * 16;
            } else {
                const i64 last = o.index - N - i0, col = (i64)chunk * N;
                off[i] = (u32)((i64)row * o.ld[0] * (i64)sizeof(T) + (col < last ? col : last) * (i64)sizeof(T));
            }
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) base[w] = (const char*)o.p[w] + (L == ROWS ? i0 * o.ld[w] : i0) * (i64)sizeof(T);
        step = L == ROWS ? 128 : (i64)(128 / sizeof(T)) * o.ld[0] * (i64)sizeof(T);
    }

    // The part at contraction step `s` of segment `seg` into the tile at `lds`.
    __device__ __forceinline__ void bring(char* lds, int seg, int s, int wave) const
    {
        typedef __attribute__((address_space(1))) const void GlobalAny;
        typedef __attribute__((address_space(3))) void LdsAny;
        const i64 at = s * step;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const char* b = base[0];
            if constexpr (PAIRED > 0) {
                if ((i * (NT / 8) + wave * 8) % (PAIRED * 16) >= PAIRED * 8) b = base[1];
            } else {
                if (seg) b = base[1];
            }
            __builtin_amdgcn_global_load_lds((GlobalAny*)(b + at + off[i]), (LdsAny*)(lds + (i * NT + wave * 64) * 16), 16, 0, 0);
        }
    }
};

// A lane's 16 bytes of the square at `base` (a multiple of 16) for half `ks` of a step: index base + lane % 16, contraction
// (lane / 16) * 16 bytes and on.
template <class T, Layout L, int BI>
__device__ __forceinline__ Word4 read_square(const char* tile, int base, int ks, int lane)
{
    if constexpr (L == ROWS) {
        const int row = base + (lane & 15);
        const int chunk = (ks * 4 + (lane >> 4)) ^ (lane & 7);
        return *reinterpret_cast<const Word4*>(tile + row * 128 + chunk * 16);
    } else if constexpr (sizeof(T) == 2) {
        constexpr int RB = BI * 2;
        const int r = (lane >> 2) & 3, g = lane >> 4;
        const int block = (base >> 4) ^ ((r | (g << 2)) & (RB / 32 - 1));
        const char* at = tile + (ks * 32 + g * 8 + r) * RB + block * 32 + (lane & 3) * 8;
        typedef __attribute__((address_space(3))) Short4 LdsShort4;
        union { Word4 w; Short4 s[2]; } u;
        u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)at);
        u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)(at + 4 * RB));
        return u.w;
    } else {
        constexpr int RB = BI * 4;
        const int g = lane >> 4;
        const char* at = tile + (ks * 16 + g * 4) * RB + ((base >> 4) ^ g) * 64 + (lane & 15) * 4;
        Word4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const int*>(at + j * RB);
        return w;
    }
}

template <class T>
__device__ __forceinline__ void square_product(Float4& acc, Word4 n, Word4 m)
{
    if constexpr (sizeof(T) == 4) {
        const Float4 a = __builtin_bit_cast(Float4, n), b = __builtin_bit_cast(Float4, m);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], acc, 0, 0, 0);
    } else if constexpr (__is_same(T, __bf16)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, n), __builtin_bit_cast(Bf16x8, m), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Half8, n), __builtin_bit_cast(Half8, m), acc, 0, 0, 0);
    }
}

// Tiles in an order that keeps what runs at once close together: workgroups go round the eight dies, so every die gets a
// stretch of its own, and in a stretch eight rows of tiles are walked column by column.
__device__ __forceinline__ void tile_of(u32 id, u32 tm, u32 tn, u32& m, u32& n)
{
    const u32 total = tm * tn, die = id & 7, q = total >> 3, r = total & 7;
    const u32 at = die * q + min(die, r) + (id >> 3);
    const u32 group = at / (8 * tn), first = group * 8, rows = min(8u, tm - first), in = at - group * 8 * tn;
    m = first + in % rows;
    n = in / rows;
}

// One step's products out of shared memory.
template <class T, class TL, Layout LA, Layout LB>
__device__ __forceinline__ void step_products(Float4 (&acc)[TL::FN][TL::FM], const char* ta, const char* tb, int wm, int wn, int lane)
{
    constexpr int FM = TL::FM, FN = TL::FN;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        Word4 fm[FM], fn[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) fn[j] = read_square<T, LB, TL::BN>(tb, (wn * FN + j) * 16, ks, lane);
#pragma unroll
        for (int i = 0; i < FM; ++i) fm[i] = read_square<T, LA, TL::BM>(ta, (wm * FM + i) * 16, ks, lane);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) square_product<T>(acc[j][i], fn[j], fm[i]);
    }
}

// The sums of the tile at (m0, n0) over `segments` matrices of each operand one after the other (PAIRED > 0: over one, B's
// two alternating in the tile).
template <class T, class TL, Layout LA, Layout LB, int PAIRED, bool DIRECT>
__device__ __forceinline__ void product_tile(Float4 (&acc)[TL::FN][TL::FM], char* lds, const Operand& a, const Operand& b, int segments, i64 m0, i64 n0)
{
    constexpr int FM = TL::FM, FN = TL::FN, NT = TL::NT, BM = TL::BM, BN = TL::BN, BK = TL::BK;
    constexpr int PA = BM * 8 / NT, PB = BN * 8 / NT;                        // 16-byte positions a thread brings of each operand
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = Float4{0, 0, 0, 0};

    const i64 depth = a.depth > b.depth ? a.depth : b.depth;
    const int steps = (int)((depth + BK - 1) / BK), total = steps * segments;
    if (total == 0) return;
    Word4 ra[PA], rb[PB];
    auto fetch = [&](int s) {
        const int seg = s >= steps;
        const i64 k0 = (i64)(s - seg * steps) * BK;
#pragma unroll
        for (int i = 0; i < PA; ++i) ra[i] = fetch_chunk<T, LA, BM, 0, DIRECT>(a, seg, m0, k0, i * NT + tid);
#pragma unroll
        for (int i = 0; i < PB; ++i) rb[i] = fetch_chunk<T, LB, BN, PAIRED, DIRECT>(b, seg, n0, k0, i * NT + tid);
    };
    auto put = [&](int s) {
        char* at = lds + (s & 1) * (BM + BN) * 128;
#pragma unroll
        for (int i = 0; i < PA; ++i) *reinterpret_cast<Word4*>(at + (i * NT + tid) * 16) = ra[i];
#pragma unroll
        for (int i = 0; i < PB; ++i) *reinterpret_cast<Word4*>(at + BM * 128 + (i * NT + tid) * 16) = rb[i];
    };
    if constexpr (DIRECT) {
        DirectTile<T, LA, BM, NT, 0> da;
        DirectTile<T, LB, BN, NT, PAIRED> db;
        da.init(a, m0);
        db.init(b, n0);
        const int whole = (int)((a.depth < b.depth ? a.depth : b.depth) / BK);   // steps of which nothing lies outside; the last may be another
        auto bring = [&](int s) {
            const int seg = s >= steps, k = s - seg * steps;
            if (k < whole) {
                char* at = lds + (s & 1) * (BM + BN) * 128;
                da.bring(at, seg, k, wave);
                db.bring(at + BM * 128, seg, k, wave);
            } else {
                fetch(s);
                put(s);
            }
        };
        bring(0);
        if (total > 1) bring(1);
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        // A step is 2 FM groups, one square row of A times all of B's squares each.  A's squares are read AHEAD groups before their
        // products, B's of the other half of the step as early; when the last read of a step is through, its half of the shared memory is
        // given to the step after the next, and the last groups read the next step's first squares.  So products never wait for a
        // read that was just issued, and a load has almost a whole step to arrive.
        constexpr int GROUPS = 2 * FM, AHEAD = 4;
        static_assert(FM % AHEAD == 0 && FN <= AHEAD, "the squares of a step are read before its last groups");
        Word4 fm[GROUPS], fn[2][FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) fn[0][j] = read_square<T, LB, BN>(lds + BM * 128, (wn * FN + j) * 16, 0, lane);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fm[i] = read_square<T, LA, BM>(lds, (wm * FM + i) * 16, 0, lane);
        for (int s = 0; s < total; ++s) {
            const char* ta = lds + (s & 1) * (BM + BN) * 128;
            const char* next = lds + (~s & 1) * (BM + BN) * 128;
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) {
                if (q == GROUPS - AHEAD) {
                    __builtin_amdgcn_s_waitcnt(0);
                    __syncthreads();
                    if (s + 2 < total) bring(s + 2);
                }
                if (q < GROUPS - AHEAD) {
                    const int r = q + AHEAD;
                    fm[r] = read_square<T, LA, BM>(ta, (wm * FM + r % FM) * 16, r / FM, lane);
                    if (q < FN) fn[1][q] = read_square<T, LB, BN>(ta + BM * 128, (wn * FN + q) * 16, 1, lane);
                } else {                                                     // (behind the last step: read, and not used)
                    const int r = q - (GROUPS - AHEAD);
                    fm[r] = read_square<T, LA, BM>(next, (wm * FM + r) * 16, 0, lane);
                    if (r < FN) fn[0][r] = read_square<T, LB, BN>(next + BM * 128, (wn * FN + r) * 16, 0, lane);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) square_product<T>(acc[j][q % FM], fn[q / FM][j], fm[q]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    } else {
        fetch(0);
        put(0);
        __syncthreads();
        for (int s = 0; s < total; ++s) {
            const char* ta = lds + (s & 1) * (BM + BN) * 128;
            if (s + 1 < total) fetch(s + 1);
            step_products<T, TL, LA, LB>(acc, ta, ta + BM * 128, wm, wn, lane);
            if (s + 1 < total) put(s + 1);                                   // the half that nothing reads any more
            __syncthreads();
        }
    }
}

// Four neighbouring results of one row, rounded once; `have` of them exist.  `wide`: the row's stride and address let four
// be stored at once.
template <class T>
__device__ __forceinline__ void store4(T* p, Float4 v, i64 have, bool wide)
{
    alignas(16) T r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = from_float<T>(v[i]);
    if (wide && have >= 4) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<Word2*>(p) = *reinterpret_cast<Word2*>(r);
        } else {
            *reinterpret_cast<Word4*>(p) = *reinterpret_cast<Word4*>(r);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) p[i] = r[i];
}

}  // namespace
