// Tiles of matrix products in registers, shared memory and the matrix cores: D[m][n] = sum_k A(m, k) B(n, k).
// Part of the ZipLine library (see training.hip); device code for gfx950.
//
// A workgroup computes a BM x BN tile of D; its WM x WN waves hold FM x FN squares of 16 x 16 each.  A step takes 128 bytes
// of the contraction (64 16-bit or 32 32-bit elements) of every row of both operands through shared memory, where there is room
// for three steps of A and two of B: a wave reads all of its B early in a step, so the step after the next can be sent for as soon as that
// is done, and a load has a step and a half to arrive.  Products of 8192 x 4096 x 12288 in bf16, against two and two: three and two 1.07 (forward),
// 1.13 (dx) and 1.14 (dW) times as fast, with the loads spread over the step 1.19, 1.33 and 1.35 times.  Traced one after the other in a pass with gradients,
// at the clock that such a pass leaves them, they run at 1270, 1270 and 1220 TFLOP/s.
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

template <int N> struct Int { static constexpr int value = N; };

template <class T, int WM_, int WN_, int FM_, int FN_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 16, BN = WN * FN * 16, NT = WM * WN * WAVE;
    static constexpr int BK = 128 / (int)sizeof(T);
    static constexpr int SLOT_A = BM * 128, SLOT_B = BN * 128;
    static constexpr int LDS = 3 * SLOT_A + 2 * SLOT_B;
};

// One operand: `index` rows of D's axis, `depth` of the contraction, `ld` elements from a row in memory to the next.
// Two matrices where the contraction runs through both (dx), or where their rows alternate in a tile (gate and up).
struct Operand {
    const void* p[2];
    i64 ld[2];
    i64 index, depth;
    __device__ __forceinline__ const void* matrix(int which) const { return which ? p[1] : p[0]; }
    __device__ __forceinline__ i64 stride(int which) const { return which ? ld[1] : ld[0]; }
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

// The 16 bytes of position `pos` of the tile that begins at contraction k0, through registers; what lies outside the operand reads as zero.  WHOLE: chunks lie inside or
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
        const T* p = (const T*)o.matrix(which) + i * o.stride(which) + k;
        if constexpr (WHOLE) return i < o.index && k < o.depth ? *reinterpret_cast<const Word4*>(p) : Word4{0, 0, 0, 0};
        return i < o.index ? load_some(p, o.depth - k) : Word4{0, 0, 0, 0};
    } else {
        const i64 k = k0 + row, i = i0 + chunk * N;
        const T* p = (const T*)o.matrix(which) + k * o.stride(which) + i;
        if constexpr (WHOLE) return i < o.index && k < o.depth ? *reinterpret_cast<const Word4*>(p) : Word4{0, 0, 0, 0};
        return k < o.depth ? load_some(p, o.index - i) : Word4{0, 0, 0, 0};
    }
}

// The same tile straight from memory to shared memory, no registers between: the shared side of such a load is 16 bytes a lane in
// lane order, so the lanes' order is permuted on the memory side.  Rows (columns) beyond the operand repeat its last ones; what comes
// of them is not stored.  Needs whole 16-byte chunks: operand_direct() on the host.
//
// LOOSE: the same through registers, whatever the alignment and the length; a chunk of a COLS tile that passes the end of its row takes what
// comes behind it (nothing that comes of that is stored either).  That stays inside the operand for all rows but the last:
// loose_steps() says how far.
template <class T, Layout L, int BI, int NT, int PAIRED, bool LOOSE>
struct DirectTile {
    static constexpr int P = BI * 8 / NT, N = PER_WORD4<T>;
    const char* base;
    i64 other;                                                               // bytes from there to the second matrix
    i64 step;                                                                // bytes from a step to the next
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
                off[i] = (u32)((i64)(row < last ? row : last) * o.stride(which) * (i64)sizeof(T)) + chunk * 16;
            } else {
                const i64 left = o.index - i0, col = (i64)chunk * N, at = LOOSE ? (col < left ? col : 0) : (col < left - N ? col : left - N);
                off[i] = (u32)((i64)row * o.ld[0] * (i64)sizeof(T) + at * (i64)sizeof(T));
            }
        }
        base = (const char*)o.p[0] + (L == ROWS ? i0 * o.ld[0] : i0) * (i64)sizeof(T);
        other = (i64)((uintptr_t)o.p[1] - (uintptr_t)o.p[0]) + (L == ROWS ? i0 * (o.ld[1] - o.ld[0]) : 0) * (i64)sizeof(T);
        step = L == ROWS ? 128 : (i64)(128 / sizeof(T)) * o.ld[0] * (i64)sizeof(T);
    }

    __device__ __forceinline__ bool second(int seg, int wave, int i) const
    {
        return PAIRED > 0 ? (i * (NT / 8) + wave * 8) % (PAIRED > 0 ? PAIRED * 16 : 1) >= PAIRED * 8 : seg != 0;
    }

    __device__ __forceinline__ Word4 load(int seg, int s, int wave, int i) const
    {
        return load_loose((const T*)(base + s * step + (second(seg, wave, i) ? other : 0) + off[i]));
    }

    // The i-th of a thread's loads of step `s` of segment `seg`, into the slot at `lds`.  (Buffer loads, not global ones: those count as
    // accesses that may go to either memory, and the compiler then waits for all reads of shared memory where it needs one.)
    __device__ __forceinline__ void bring(char* lds, int seg, int s, int wave, int i) const
    {
        typedef __attribute__((address_space(3))) void LdsAny;
        const auto resource = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + s * step + (second(seg, wave, i) ? other : 0)), 0, -1, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(resource, (LdsAny*)(lds + (i * NT + wave * 64) * 16), 16, (int)off[i], 0, 0, 0);
    }
};

// Steps at a segment's beginning that a LOOSE tile may take: whole ones that do not come to the last row of COLS, whose rows hold a chunk at
// least and whose two matrices have the same stride, and offsets that fit 31 bits.
template <class T, Layout L>
__device__ __forceinline__ int loose_steps(const Operand& o)
{
    constexpr int BK = 128 / (int)sizeof(T);
    const i64 far = o.ld[0] > o.ld[1] ? o.ld[0] : o.ld[1];
    if (far * (i64)sizeof(T) * 256 > 0x7fffffffll || (L == COLS && (o.index < PER_WORD4<T> || o.ld[0] != o.ld[1]))) return 0;
    return (int)((L == COLS ? o.depth - 1 : o.depth) / BK);
}

// Four rows of 16 16-bit elements each that 16 lanes read, 8 bytes a lane, come back as columns.  (Through a restrict pointer: without any
// aliasing facts the compiler waits for every load to shared memory under way before such a read.  Which loads have to be
// through is product_tile's business.)
typedef __attribute__((address_space(3))) Short4 LdsShort4;
__device__ __forceinline__ Short4 read_transposed(LdsShort4* __restrict p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }

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
        union { Word4 w; Short4 s[2]; } u;
        u.s[0] = read_transposed((LdsShort4*)at);
        u.s[1] = read_transposed((LdsShort4*)(at + 4 * RB));
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

// Waits until no more than VM loads to shared memory and LGKM reads of it are under way, then for the other waves.  Nothing moves across.
template <int VM, int LGKM>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((VM & 15) | (7 << 4) | (LGKM << 8) | ((VM >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// The sums of the tile at (m0, n0) over `segments` matrices of each operand one after the other (PAIRED > 0: over one, B's
// two alternating in the tile), or over the `part`-th of `parts` stretches of their steps.
template <class T, class TL, Layout LA, Layout LB, int PAIRED, bool DIRECT>
__device__ __forceinline__ void product_tile(Float4 (&acc)[TL::FN][TL::FM], char* lds, const Operand& a, const Operand& b, int segments, i64 m0, i64 n0,
                                             int part = 0, int parts = 1)
{
    constexpr int FM = TL::FM, FN = TL::FN, NT = TL::NT, BM = TL::BM, BN = TL::BN, BK = TL::BK;
    constexpr int PA = BM * 8 / NT, PB = BN * 8 / NT;                        // 16-byte positions a thread brings
    static_assert(PA > 0 && PB > 0, "every thread brings something of both operands");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / TL::WN, wn = wave % TL::WN;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = Float4{0, 0, 0, 0};

    const i64 depth = a.depth > b.depth ? a.depth : b.depth;
    const int steps = (int)((depth + BK - 1) / BK);
    struct Step { Word4 a[PA], b[PB]; };                                     // what a thread brings in a step, on its way through registers
    auto fetch = [&](Step& r, int seg, int s) {
#pragma unroll
        for (int i = 0; i < PA; ++i) r.a[i] = fetch_chunk<T, LA, BM, 0, DIRECT>(a, seg, m0, (i64)s * BK, i * NT + tid);
#pragma unroll
        for (int i = 0; i < PB; ++i) r.b[i] = fetch_chunk<T, LB, BN, PAIRED, DIRECT>(b, seg, n0, (i64)s * BK, i * NT + tid);
    };
    auto place_a = [&](int slot) { return lds + slot * TL::SLOT_A; };
    auto place_b = [&](int slot) { return lds + 3 * TL::SLOT_A + slot * TL::SLOT_B; };
    auto put = [&](const Step& r, int slot) {
#pragma unroll
        for (int i = 0; i < PA; ++i) *reinterpret_cast<Word4*>(place_a(slot) + (i * NT + tid) * 16) = r.a[i];
#pragma unroll
        for (int i = 0; i < PB; ++i) *reinterpret_cast<Word4*>(place_b(slot) + (i * NT + tid) * 16) = r.b[i];
    };
    auto square_a = [&](int slot, int i, int ks) { return read_square<T, LA, BM>(place_a(slot), (wm * FM + i) * 16, ks, lane); };
    auto square_b = [&](int slot, int j, int ks) { return read_square<T, LB, BN>(place_b(slot), (wn * FN + j) * 16, ks, lane); };
    auto products = [&](int slot) {
#pragma unroll 1
        for (int ks = 0; ks < 2; ++ks) {
            Word4 fn[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) fn[j] = square_b(slot, j, ks);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const Word4 fm = square_a(slot, i, ks);
#pragma unroll
                for (int j = 0; j < FN; ++j) square_product<T>(acc[j][i], fn[j], fm);
            }
        }
    };
    if constexpr (!DIRECT) {
        const int all = steps * segments, from = (int)((i64)all * part / parts), total = (int)((i64)all * (part + 1) / parts) - from;
        if (total == 0) return;
        DirectTile<T, LA, BM, NT, 0, true> da;
        DirectTile<T, LB, BN, NT, PAIRED, true> db;
        da.init(a, m0);
        db.init(b, n0);
        const int la = loose_steps<T, LA>(a), lb = loose_steps<T, LB>(b), loose = la < lb ? la : lb;
        Step set[2];                                                         // two steps under way: one alone does not cover memory's latency
        auto bring_loose = [&](Step& r, int s) {
            const int seg = s >= steps, k = seg ? s - steps : s;
#pragma unroll
            for (int i = 0; i < PA; ++i) r.a[i] = da.load(seg, k, wave, i);
#pragma unroll
            for (int i = 0; i < PB; ++i) r.b[i] = db.load(seg, k, wave, i);
        };
        auto bring_step = [&](Step& r, int s) {
            const int seg = s >= steps, k = seg ? s - steps : s;
            if (k < loose) bring_loose(r, s);
            else fetch(r, seg, k);
        };
        // Step s of the stretch (its data is in shared memory): the one after the next is sent for, the next put in place.
        auto step = [&](auto odd, int s, auto&& bring) {
            constexpr int O = decltype(odd)::value;
            bring(set[O], s + 2);
            products(O);
            if (s + 1 < total) put(set[O ^ 1], O ^ 1);                       // what nothing reads any more
            __syncthreads();
        };
        bring_step(set[0], from);
        if (total > 1) bring_step(set[1], from + 1);
        put(set[0], 0);
        __syncthreads();
        int s = 0;
        const int plain = (from < steps ? min(from + total, loose) : min(from + total, steps + loose)) - from;   // steps that need no checks
        for (; s + 4 <= plain; s += 2) {
            step(Int<0>(), s, [&](Step& r, int t) { bring_loose(r, from + t); });
            step(Int<1>(), s + 1, [&](Step& r, int t) { bring_loose(r, from + t); });
        }
        for (; s < total; s += 2) {
            auto checked = [&](Step& r, int t) { if (t < total) bring_step(r, from + t); };
            step(Int<0>(), s, checked);
            if (s + 1 < total) step(Int<1>(), s + 1, checked);
        }
        return;
    }
    // Whole steps of all segments first, then (in the last stretch) the parts of a step that are left.
    const int whole = (int)((a.depth < b.depth ? a.depth : b.depth) / BK), all = whole * segments;
    const int from = (int)((i64)all * part / parts), total = (int)((i64)all * (part + 1) / parts) - from;
    if (total > 0) {
        DirectTile<T, LA, BM, NT, 0, false> da;
        DirectTile<T, LB, BN, NT, PAIRED, false> db;
        da.init(a, m0);
        db.init(b, n0);
        constexpr int LOADS = PA + PB;
        auto bring = [&](int s, int slot_a, int slot_b, int i) {             // load i of the LOADS of step s of the stretch
            const int at = from + s, seg = at >= whole, k = at - seg * whole;
            if (i < PA) da.bring(place_a(slot_a), seg, k, wave, i);
            else db.bring(place_b(slot_b), seg, k, wave, i - PA);
        };
#pragma unroll
        for (int i = 0; i < LOADS; ++i) bring(0, 0, 0, i);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) bring(total > 1 ? 1 : 0, 1, 1, i);
        wait_and_meet<LOADS, 15>();
        // A step is 2 FM groups, one square row of A times all of B's squares each.  A's squares are read AHEAD groups before their
        // products; B's of the second half at once, and the last groups read the next step's first squares: products never wait for a
        // read that was just issued.
        constexpr int GROUPS = 2 * FM, AHEAD = 4, SEND = FN / 2 + 1;
        static_assert(FM % AHEAD == 0 && FN == AHEAD && SEND < GROUPS - AHEAD, "the squares of a step are read before its last groups");
        Word4 fm[GROUPS], fn[2][FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) fn[0][j] = square_b(0, j, 0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fm[i] = square_a(0, i, 0);
        int sa = 0;                                                          // s % 3
        for (int s = 0; s < total; ++s) {
            const int sa1 = sa == 2 ? 0 : sa + 1, sa2 = sa == 0 ? 2 : sa - 1, sb = s & 1;
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) {
                if (q == SEND) wait_and_meet<63, 1>();                       // B has been read by all: a group and its read of A later
                if (q == GROUPS - AHEAD) wait_and_meet<LOADS, 15>();         // the next step has arrived; the one behind it is on its way
                // One load a group: all at once they hold each other up (dx of 8192 x 4096 x 12288 takes 12 % longer).  Behind the end the last
                // step is sent for again, into places that nothing reads.
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (q == SEND + i * (GROUPS - AHEAD - SEND) / LOADS) bring(s + 2 < total ? s + 2 : total - 1, sa2, sb, i);
                if (q < GROUPS - AHEAD) {
                    if (q < FN / 2) {
                        fn[1][2 * q] = square_b(sb, 2 * q, 1);
                        fn[1][2 * q + 1] = square_b(sb, 2 * q + 1, 1);
                    }
                    const int r = q + AHEAD;
                    fm[r] = square_a(sa, r % FM, r / FM);
                } else {                                                     // all of B's before the first of A's: the first products need them
#pragma unroll
                    for (int e = 0; e < 2; ++e) {                            // (behind the last step: read, and not used)
                        const int r = 2 * (q - (GROUPS - AHEAD)) + e;
                        if (r < FN) fn[0][r] = square_b(sb ^ 1, r, 0);
                        else fm[r - FN] = square_a(sa1, r - FN, 0);
                    }
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) square_product<T>(acc[j][q % FM], fn[q / FM][j], fm[q]);
                __builtin_amdgcn_sched_barrier(0);
            }
            sa = sa1;
        }
    }
    if (whole < steps && part == parts - 1)
#pragma unroll 1
        for (int seg = 0; seg < segments; ++seg) {
            Step r;
            fetch(r, seg, whole);
            wait_and_meet<0, 0>();                                           // everything before has arrived and been read
            put(r, 0);
            __syncthreads();
            products(0);
        }
}

// Four neighbouring results of one row, rounded once; `have` of them exist.  At any alignment: memory takes wide stores there too.
template <class T>
__device__ __forceinline__ void store4(T* p, Float4 v, i64 have)
{
    union { T r[4]; Word2 two; Word4 four; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.r[i] = from_float<T>(v[i]);
    if (have >= 4) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<LooseWord2*>(p) = u.two;
        else store_loose(p, u.four);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < have) p[i] = u.r[i];
}

// Two squares side by side of 16 rows: a lane has row lane % 16, columns (lane / 16) * 4 and on of either.  `p` is the lane's
// row at the first square's first column, of which `have` columns exist.  For 16-bit results lanes 16 apart exchange
// halves, so that each has eight neighbouring columns of one square and a row's 64 bytes go out at once.
template <class T>
__device__ __forceinline__ void store_pair(T* p, Float4 first, Float4 second, i64 have, int lane)
{
    const int g = lane >> 4;
    if constexpr (sizeof(T) == 2) {
        if (have >= 32) {
            union { T v[4]; int w[2]; } a, b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a.v[i] = from_float<T>(first[i]);
                b.v[i] = from_float<T>(second[i]);
            }
            Word4 out;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto r = __builtin_amdgcn_permlane16_swap((unsigned)a.w[i], (unsigned)b.w[i], false, false);
                out[i] = (int)r[0];
                out[2 + i] = (int)r[1];
            }
            store_loose(p + (g & 1) * 16 + (g >> 1) * 8, out);
            return;
        }
    }
    store4(p + g * 4, first, have - g * 4);
    store4(p + 16 + g * 4, second, have - 16 - g * 4);
}

}  // namespace
