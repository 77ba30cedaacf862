// The matrix core that the 8-bit products and the orthogonalisation share
// (gfx950): C = A B^T for two operands whose rows run along the contraction.
//
// Both operands are rows of bytes to the loader: 16 bytes a lane and operand
// are 16 8-bit integers (v_mfma_i32_16x16x64_i8) or 8 halves
// (v_mfma_f32_16x16x32_f16), and the two instructions hold them in the same
// lanes: lane l has row l % 16, bytes 16 * (l / 16) on. A slice of the
// contraction is 128 bytes of every row: two instructions deep for one 8-bit
// or half operand; or, where a number is the sum of two halves, 64 bytes of 32
// high halves and 64 bytes of their 32 low halves.
#pragma once

#include "rtopk_common.h"

namespace rtopk {

constexpr int kSlice = 128;          // bytes of a row in one slice of the contraction

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// What the bytes are. kPairs: each number is a high and a low half, and the
// product takes high * high, high * low and low * high (what is left out is
// 2^-22 of the product).
enum Operands { kBytes, kHalves, kPairs };

template <Operands kOf> struct Sums { typedef f32x4 type; };
template <> struct Sums<kBytes> { typedef i32x4 type; };

// One operand of a tile: the row that the tile starts with, the rows that are
// there from it on (rows past them repeat the last one: what they give is not
// stored), the bytes from row to row and the bytes of a row that count (the
// same for both operands).
struct TileRows {
    const unsigned char *first;
    u32 rows;
    u32 stride;
    u32 bytes;
};

// 16 bytes from byte `at` of a row of `bytes` bytes, zeros beyond its end; what is not there is not read. In two parts, so that
// several loads are under way together: the load takes the row's last 16 bytes where it would go beyond them, and
// cut_piece moves them down. (A branch around each load, which waits for it, made the last slice of an odd contraction
// cost as much as forty others: 16 us of 55 at 1499 x 5001 x 2003.)
__device__ __forceinline__ i32x4 load_piece(const unsigned char *row, u32 at, u32 bytes)
{
    i32x4 v{0, 0, 0, 0};
    if (bytes >= 16u) {
        __builtin_memcpy(&v, row + min(at, bytes - 16u), 16);
    } else {
        u64 half[2] = {0, 0};
        for (u32 c = 0; c < bytes; ++c) half[c >> 3] |= (u64)row[c] << (8u * (c & 7u));
        v = i32x4{(int)(u32)half[0], (int)(half[0] >> 32), (int)(u32)half[1], (int)(half[1] >> 32)};
    }
    return v;
}
__device__ __forceinline__ i32x4 cut_piece(const i32x4 &v, u32 at, u32 bytes)
{
    const u32 start = bytes >= 16u ? bytes - 16u : 0u, down = at > start ? at - start : 0u;     // bytes to move by
    const u64 lo = (u64)(u32)v[0] | (u64)(u32)v[1] << 32, hi = (u64)(u32)v[2] | (u64)(u32)v[3] << 32;
    const u32 bits = 8u * (down & 7u);
    const u64 a = down >= 8u ? hi : lo, b = down >= 8u ? 0ull : hi;
    u64 x = bits ? a >> bits | b << (64u - bits) : a, y = b >> bits;
    if (down >= 16u) x = y = 0ull;
    return i32x4{(int)(u32)x, (int)(x >> 32), (int)(u32)y, (int)(y >> 32)};
}

// A tile of kM x kN sums on kWavesM x kWavesN wavefronts, by instructions of 16 x 16. kStages slices in LDS, and kAhead: the
// first half of the next slice is read into registers before the second half of this one is multiplied. What each choice
// gave at 8192 x 8192 (8192 bytes of contraction, 10^12 operations a second; a product of pairs counted once):
//                                                              bytes  halves  pairs
//   256 x 256, 2 x 4 wavefronts, 2 stages, kAhead               2554    1240      -    (pairs: 100 registers spilt)
//   256 x 256, the same without kAhead                          2116    1090    479
//   256 x 256, 2 x 4, by instructions of 32 x 32                2359    1161    436
//   256 x 256, 2 x 2                                            2175    1112      -    (one wavefront a SIMD: nobody fills its waits)
//   128 x 128, 2 x 2                                            1953     949    464    (two workgroups a unit; alone on its unit 388)
// What bounds 256 x 256 with bytes is power: the matrix units are busy in 65% of the cycles, and the clock falls from 2.4 to 1.7
// GHz; the library's product reaches 2116 under the same limit. Pairs (1437 as the halves that are multiplied) are within 4% of the
// library's 1491 for halves. Halves alone are not (1240), so power is not all that bounds them; what else does was not found.
// 64 and 128 go to small results, on 2 x 4 wavefronts too: a slice of 64 x 64 takes 0.3 us alone on its unit, of which its
// products are 0.08: the rest is one barrier and two trips to LDS one after the other (six stages in the place of three
// change nothing, so it is not the loads). 192 is for pairs and for results where 256 leaves units without a tile; 160 was
// slower than the best of these on ten of eleven shapes (four squares of 1500: 1% of the call faster).
//
// How the rows of a wavefront's operands are dealt to its instructions, so that what a lane ends up with is stored in wide pieces:
// kInOrder: fragment i has rows 16 i ..; kRuns: of A, a lane's rows are neighbours (eight, or four, or two of them: they
// lie side by side in a result that is turned over); kWide: those, and of B the rows of two fragments alternate by
// four, so that a lane has eight neighbouring columns (16 bytes of a 16-bit result; 64 bytes of a row from four lanes).
enum Deal { kInOrder, kRuns, kWide };

template <Operands kOf, int kM, int kN, int kWavesM, int kWavesN, int kStages, bool kAhead, Deal kDeal = kInOrder>
struct Tile {
    static constexpr int kRowsM = kM, kRowsN = kN;
    static constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * kWave;
    static constexpr int kStage = (kM + kN) * kSlice, kLds = kStages * kStage;
    static constexpr int kFragsM = kM / kWavesM / 16, kFragsN = kN / kWavesN / 16;
    static constexpr int kLoadsM = kM / 8 / kWaves, kLoadsN = kN / 8 / kWaves, kLoads = kLoadsM + kLoadsN;
    static_assert(kLoadsM * kWaves * 8 == kM && kLoadsN * kWaves * 8 == kN, "every wavefront loads whole groups of eight rows");
    static_assert(kFragsM * kWavesM * 16 == kM && kFragsN * kWavesN * 16 == kN, "whole instructions");
    static_assert(kStages >= 2, "one slice under way at least");
    typedef typename Sums<kOf>::type Sum;
    // sum[i][j]: row row_at(i) of A, rows col_at(j) .. + 3 of B
    Sum sum[kFragsM][kFragsN];
    // half a slice: 64 bytes of the wavefront's rows
    struct Half {
        i32x4 a[kFragsM], b[kFragsN];
    };

    static __device__ __forceinline__ u32 wave() { return (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)); }
    static __device__ __forceinline__ u32 row0() { return wave() / kWavesN * (kM / kWavesM); }
    static __device__ __forceinline__ u32 col0() { return wave() % kWavesN * (kN / kWavesN); }

    // row r of fragment i of the wavefront's rows of A, and of fragment j of its rows of B
    static __device__ __forceinline__ u32 of_a(int i, u32 r)
    {
        constexpr int kEight = kFragsM / 8 * 8, kFour = kFragsM / 4 * 4, kRest = kFragsM - kFour;
        if (kDeal == kInOrder) return 16u * i + r;
        if (i < kEight) return 128u * (i / 8) + 8u * r + i % 8;
        if (i < kFour) return 16u * kEight + 64u * ((i - kEight) / 4) + 4u * r + (i - kEight) % 4;
        return 16u * kFour + kRest * r + (i - kFour);
    }
    static __device__ __forceinline__ u32 of_b(int j, u32 r)
    {
        if (kDeal == kWide && (j | 1) < kFragsN) return 32u * (j >> 1) + 8u * (r >> 2) + 4u * (j & 1) + (r & 3u);
        return 16u * j + r;
    }
    static __device__ __forceinline__ u32 row_at(int i) { return row0() + of_a(i, lane_id() & 15u); }
    static __device__ __forceinline__ u32 col_at(int j) { return col0() + of_b(j, 4u * (lane_id() >> 4)); }
    // whether fragments j and j + 1 have eight neighbouring columns
    static constexpr bool wide_at(int j) { return kDeal == kWide && j % 2 == 0 && j + 1 < kFragsN; }
    static constexpr int step_at(int j) { return wide_at(j) ? 2 : 1; }
    static constexpr int next_to(int j) { return j + 1 < kFragsN ? j + 1 : j; }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) sum[i][j] = Sum{0, 0, 0, 0};
    }

    // LDS holds a slice as rows of eight 16-byte pieces; piece c of row r lies in place c ^ turn(r). Two rows fill the 64
    // banks, and a 16-byte read takes sixteen lanes at a time, not in their order: 0-3, 12-15, 20-23, 24-27 (eight rows of
    // one piece, eight others of the next) and so on. The turn puts what they read into sixteen different places: the
    // counter of bank conflicts reads zero; with r / 2 % 8 every read took twice its cycles.
    static __device__ __forceinline__ u32 turn(u32 row) { return (row & 2u) | ((row >> 1) & 4u); }
    static __device__ __forceinline__ u32 place(u32 row, u32 piece) { return row * kSlice + ((piece ^ turn(row)) << 4); }

    // row of its operand that load q of this lane takes (the lane's piece of it: lane % 8, as placed)
    static __device__ __forceinline__ u32 row_of(int q)
    {
        return ((q < kLoadsM ? q : q - kLoadsM) * kWaves + wave()) * 8u + (lane_id() >> 3);
    }
    // the row of the operand that lies in row r of a stage
    static __device__ __forceinline__ u32 dealt(int q, u32 r)
    {
        constexpr u32 kRowsA = kM / kWavesM, kRowsB = kN / kWavesN;
        if (kDeal == kInOrder) return r;
        if (q < kLoadsM) return r / kRowsA * kRowsA + of_a((int)(r % kRowsA / 16u), r & 15u);
        return r / kRowsB * kRowsB + of_b((int)(r % kRowsB / 16u), r & 15u);
    }
    // where the wavefront's load q begins in a stage; lane l's 16 bytes follow at 16 l
    static __device__ __forceinline__ u32 stage_at(int q)
    {
        return (q < kLoadsM ? 0 : kM * kSlice) + ((q < kLoadsM ? q : q - kLoadsM) * kWaves + wave()) * 8 * kSlice;
    }

    // Until at most kMore of this wavefront's loads to LDS are under way and all its reads from there are done, and until
    // every wavefront of the workgroup has come as far. (A fence would wait for every load to LDS.)
    template <int kMore>
    static __device__ __forceinline__ void wait_and_meet()
    {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((kMore & 15) | (kMore >> 4) << 14 | 0x70);       // vmcnt(kMore) lgkmcnt(0), as the compiler can see
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }

    // Adds the slices [from, to) of both operands. kWhole: rows start on 16 bytes (base and stride), and every slice
    // but a last one that goes beyond `bytes` goes to LDS by loads that pass the registers by, the next one under way
    // while this one is multiplied. The slice that goes beyond, and every slice of rows that start anywhere, comes through
    // registers, where what lies beyond `bytes` is not read and counts as zero.
    // prepare(): what else the sums wait for (the sums' first values from memory), called once the first slices are on their way.
    template <bool kWhole>
    __device__ __forceinline__ void multiply(const TileRows &a, const TileRows &b, u32 from, u32 to, unsigned char *lds)
    {
        multiply<kWhole>(a, b, from, to, lds, [] {});
    }
    template <bool kWhole, class Prepare>
    __device__ __forceinline__ void multiply(const TileRows &a, const TileRows &b, u32 from, u32 to, unsigned char *lds, Prepare prepare)
    {
#if defined(__HIP_DEVICE_COMPILE__)      // (the host pass does not know the buffer instructions)
        if (from >= to) {
            prepare();
            return;
        }
        const u32 whole = kWhole ? (a.bytes / kSlice < to ? a.bytes / kSlice : to) : from;
        u32 s = from;
        if (kWhole && s < whole) {
            const u32 lane = lane_id();
            u32 offset[kLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows &t = q < kLoadsM ? a : b;
                const u32 r = row_of(q), row = min(dealt(q, r), t.rows - 1u);
                offset[q] = row * t.stride + (((lane & 7u) ^ turn(r)) << 4);
            }
            const auto ra = __builtin_amdgcn_make_buffer_rsrc((void *)a.first, 0, 0xFFFFFFFFu, 0x00020000);
            const auto rb = __builtin_amdgcn_make_buffer_rsrc((void *)b.first, 0, 0xFFFFFFFFu, 0x00020000);
            auto load = [&](u32 slice) {
                unsigned char *stage = lds + (slice - from) % kStages * kStage;
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(q < kLoadsM ? ra : rb,
                                                             (__attribute__((address_space(3))) void *)(stage + stage_at(q)), 16,
                                                             offset[q], slice * kSlice, 0, 0);
            };
            load(s);
            if constexpr (kAhead) {
#pragma unroll
                for (int q = 1; q < kStages; ++q)
                    if (s + q < whole) load(s + q);
                prepare();
                if (s + kStages <= whole) wait_and_meet<(kStages - 1) * kLoads>();
                else wait_and_meet<0>();
                Half first, second;
                read(first, lds, 0);
                // (three copies of a slice's work, so that none of them branches: a branch stops the reads from going between the products)
                for (; s + kStages < whole; ++s) {
                    read(second, lds + (s - from) % kStages * kStage, 1);
                    add(first, first);
                    mix<0>();
                    // this wavefront has read all of slice s, and its part of slice s + 1 has come; after the barrier
                    // that holds for everybody: the stage of slice s may be overwritten, that of s + 1 read
                    wait_and_meet<(kStages - 2) * kLoads>();
                    load(s + kStages);
                    ahead<kLoads>(first, second, lds + (s + 1 - from) % kStages * kStage);
                }
                for (; s + 1 < whole; ++s) {
                    read(second, lds + (s - from) % kStages * kStage, 1);
                    add(first, first);
                    mix<0>();
                    wait_and_meet<0>();
                    ahead<0>(first, second, lds + (s + 1 - from) % kStages * kStage);
                }
                read(second, lds + (s - from) % kStages * kStage, 1);
                add(first, first);
                mix<0>();
                rest(first, second);
                ++s;
            } else {
#pragma unroll
                for (int q = 1; q < kStages - 1; ++q)
                    if (s + q < whole) load(s + q);
                prepare();
                for (; s < whole; ++s) {
                    // this wavefront's part of slice s has come (those of the kStages - 2 after it may be on their way); after
                    // the barrier everybody's has, and nobody reads the stage of slice s - 1
                    if (s + kStages - 2 < whole) wait_and_meet<(kStages - 2) * kLoads>();
                    else wait_and_meet<0>();
                    if (s + kStages - 1 < whole) load(s + kStages - 1);
                    one_slice(lds + (s - from) % kStages * kStage);
                }
            }
        }
        if (s == from) prepare();
        for (; s < to; ++s) {
            unsigned char *stage = lds + (s - from) % kStages * kStage;
            i32x4 piece[kLoads];
            u32 at[kLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows &t = q < kLoadsM ? a : b;
                const u32 r = row_of(q), row = min(dealt(q, r), t.rows - 1u);
                at[q] = s * kSlice + (((lane_id() & 7u) ^ turn(r)) << 4);
                piece[q] = load_piece(t.first + (u64)row * t.stride, at[q], t.bytes);
            }
#pragma unroll
            for (int q = 0; q < kLoads; ++q) piece[q] = cut_piece(piece[q], at[q], a.bytes);
            // (everybody has read the slice that lay in this stage, two or more slices ago, before the barrier of the last one)
#pragma unroll
            for (int q = 0; q < kLoads; ++q) *(i32x4 *)(stage + stage_at(q) + lane_id() * 16u) = piece[q];
            lds_barrier();
            one_slice(stage);
        }
#endif
    }

    // half h of a slice in LDS
    __device__ __forceinline__ void read(Half &f, const unsigned char *stage, u32 h) const { read(f, stage, stage + kM * kSlice, h); }
    __device__ __forceinline__ void read(Half &f, const unsigned char *stage_a, const unsigned char *stage_b, u32 h) const
    {
        const u32 ra = row0() + (lane_id() & 15u), rb = col0() + (lane_id() & 15u), piece = 4 * h + (lane_id() >> 4);
#pragma unroll
        for (int j = 0; j < kFragsN; ++j) f.b[j] = *(const i32x4 *)(stage_b + place(rb + 16 * j, piece));
#pragma unroll
        for (int i = 0; i < kFragsM; ++i) f.a[i] = *(const i32x4 *)(stage_a + place(ra + 16 * i, piece));
    }

    // one slice that lies in LDS, into the sums
    __device__ __forceinline__ void one_slice(const unsigned char *stage) { one_slice(stage, stage + kM * kSlice); }
    __device__ __forceinline__ void one_slice(const unsigned char *stage_a, const unsigned char *stage_b)
    {
        Half first, second;
        read(first, stage_a, stage_b, 0);
        read(second, stage_a, stage_b, 1);
        add(first, first);
        rest(first, second);
    }

    __device__ __forceinline__ void add(const Half &a, const Half &b)
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) {
                if constexpr (kOf == kBytes)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b.b[j], a.a[i], sum[i][j], 0, 0, 0);
                else
                    sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b.b[j]),
                                                                       __builtin_bit_cast(f16x8, a.a[i]), sum[i][j], 0, 0, 0);
            }
    }

    // what is left to do with a slice once its first half's own products are done
    __device__ __forceinline__ void rest(const Half &first, const Half &second)
    {
        if (kOf == kPairs) {
            add(second, first);
            add(first, second);
        } else {
            add(second, second);
        }
    }
    // that, while the next slice's first half is read
    template <int kOfLoads>
    __device__ __forceinline__ void ahead(Half &first, const Half &second, const unsigned char *next)
    {
        if constexpr (kOf == kPairs) {
            Half after;
            read(after, next, 0);
            rest(first, second);
            mix<kOfLoads>();
            first = after;
        } else {
            read(first, next, 0);
            rest(first, second);
            mix<kOfLoads>();
        }
    }

    // the reads of one half, and loads to LDS, between the products of the other
    template <int kOfLoads>
    __device__ __forceinline__ void mix() const
    {
        constexpr int kReads = kFragsM + kFragsN, kPer = kFragsM * kFragsN / (kReads + kOfLoads), kProducts = kPer ? kPer : 1;
#pragma unroll
        for (int q = 0; q < kReads; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // a read from LDS
            __builtin_amdgcn_sched_group_barrier(0x8, kProducts, 0);
            if (q < kOfLoads) {
                __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);   // a load
                __builtin_amdgcn_sched_group_barrier(0x8, kProducts, 0);
            }
        }
    }

    // act(row, col, sums): this lane's sums of row `row` of A and rows col .. col + 3 of B, counted from the tile's first.
    // Every lane of the wavefront makes the same calls.
    template <class Act>
    __device__ __forceinline__ void each(Act act) const
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) act(row_at(i), col_at(j), sum[i][j]);
    }
};

// Workgroups are dealt to the 8 XCDs in turn, and each XCD has an L2 of its own: workgroup `id` of `of` takes the place
// that gives an XCD neighbouring places.
__device__ __forceinline__ u32 xcd_place(u32 id, u32 of)
{
    const u32 xcd = id & 7u, each = of >> 3, more = of & 7u;
    return xcd * each + (xcd < more ? xcd : more) + (id >> 3);
}

// Tile (i, j) at a place of a grid of rows x cols tiles: bands of four rows of tiles, column by column.
__device__ __forceinline__ void tile_at(u32 place, u32 rows, u32 cols, u32 &i, u32 &j)
{
    constexpr u32 kBand = 4;
    const u32 band = place / (kBand * cols), in = place - band * kBand * cols;
    const u32 high = rows - band * kBand < kBand ? rows - band * kBand : kBand;
    j = in / high;
    i = band * kBand + (in - j * high);
}

// A float in the types that the entry points take (RTOPK_F32, RTOPK_BF16, RTOPK_F16).
__device__ __forceinline__ float read_as(const void *p, u64 at, int type)
{
    return type == 0   ? ((const float *)p)[at]
           : type == 1 ? __uint_as_float((u32)((const u16 *)p)[at] << 16)
                       : (float)((const _Float16 *)p)[at];
}

// Eight neighbours of a row as they are in memory, and as numbers. The load has no branch around it (several are under
// way together): a lane whose eight are not all there takes the row's last eight, and `numbers` moves them down; where the row
// has no eight it takes zeros of the library's, and `numbers` reads what there is one by one.
static __device__ const u32 kNothing[8] = {0, 0, 0, 0, 0, 0, 0, 0};
// (said to be global memory: of a pointer that may be either of the two the compiler does not know it, and its flat loads
// are waited for all together)
typedef const __attribute__((address_space(1))) unsigned char *GlobalBytes;

template <int kType> struct Eight {
    i32x4 w[kType == 0 ? 2 : 1];
    static constexpr u32 kSize = kType == 0 ? 4u : 2u;
    __device__ __forceinline__ void load(const unsigned char *row, u32 c, u32 cols)
    {
        const GlobalBytes p = cols < 8u ? (GlobalBytes)kNothing : (GlobalBytes)(row + min(c, cols - 8u) * kSize);
        __builtin_memcpy(w, (const void *)p, sizeof w);
    }
    __device__ __forceinline__ void numbers(float (&v)[8], const unsigned char *row, u32 c, u32 cols) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x;
            if (kType == 0) {
                x = __uint_as_float((u32)w[kType == 0 ? i >> 2 : 0][i & 3]);
            } else {
                const u16 h = (u16)((u32)w[0][i >> 1] >> (16 * (i & 1)));
                x = kType == 1 ? __uint_as_float((u32)h << 16) : (float)__builtin_bit_cast(_Float16, h);
            }
            v[i] = c < cols ? x : 0.0f;
        }
        if (c + 8u <= cols) return;
        if (cols >= 8u) {                   // a row's last piece was read from the row's last eight on: down it moves
            const u32 down = c - (cols - 8u);
#pragma unroll
            for (int by = 4; by; by >>= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = down & by ? (i + by < 8 ? v[i + by] : 0.0f) : v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < cols) v[i] = read_as(row, c + i, kType);
        }
    }
};

__device__ __forceinline__ u16 half_bits(float v, int type)
{
    return type == 1 ? __builtin_bit_cast(u16, (__bf16)v) : __builtin_bit_cast(u16, (_Float16)v);
}

__device__ __forceinline__ void write_as(void *p, u64 at, int type, float v)
{
    if (type == 0) ((float *)p)[at] = v;
    else ((u16 *)p)[at] = half_bits(v, type);
}

// Four and eight neighbours from `at` on, of which `have` are there. Wide stores at any alignment (rows of an odd
// length start anywhere: a product of 729 x 185 x 16179 into halves 20 us, number by number 35).
__device__ __forceinline__ void write_four(void *p, u64 at, int type, const f32x4 &v, u32 have)
{
    if (have >= 4u) {
        if (type == 0) {
            __builtin_memcpy((float *)p + at, &v, 16);
        } else {
            const u16 w[4] = {half_bits(v[0], type), half_bits(v[1], type), half_bits(v[2], type), half_bits(v[3], type)};
            __builtin_memcpy((u16 *)p + at, w, 8);
        }
    } else {
#pragma unroll
        for (u32 c = 0; c < 4; ++c)
            if (c < have) write_as(p, at + c, type, v[c]);
    }
}
__device__ __forceinline__ void write_eight(void *p, u64 at, int type, const f32x4 &a, const f32x4 &b, u32 have)
{
    if (type != 0 && have >= 8u) {
        u16 w[8];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            w[c] = half_bits(a[c], type);
            w[4 + c] = half_bits(b[c], type);
        }
        __builtin_memcpy((u16 *)p + at, w, 16);
    } else {
        write_four(p, at, type, a, have);
        if (have > 4u) write_four(p, at + 4, type, b, have - 4u);
    }
}

inline bool type_ok(int type) { return type >= 0 && type <= 2; }

// How a call's workspace is laid out, part after part.
struct Cut {
    unsigned char *base;
    u64 at = 0;
    template <class P> P *take(u64 bytes)
    {
        P *p = base ? (P *)(base + at) : nullptr;     // (without a base only the size is asked for)
        at += align_up(bytes, 256);
        return p;
    }
};

// What a launch of tiles costs, in microseconds: a launch, the tiles that one compute unit gets one after the other, their
// slices, and what comes before and after them. 64 x 64: up to three tiles share a unit; 128 x 128: two. From launches of
// 256, 512, .. tiles at 8 and 64 slices, with the slices of smaller tiles as they are where the whole chip reads (a
// slice of 128 x 128 takes 0.62 with 32 tiles, 0.82 with 192). Over thirteen shapes of 100 to 8000 rows and columns and
// contractions of 300 to 16384 the tile and runs that this picks take at most 1.15 times the best ones' time.
struct TileCost {
    double slice64[3], slice128[2], slice192, slice256;      // one slice of one tile alone, of two (three) sharing a unit
};
constexpr TileCost kCostBytes{{0.29, 0.45, 0.75}, {0.75, 0.95}, 0.93, 1.50};
constexpr TileCost kCostHalves{{0.29, 0.45, 0.75}, {0.75, 0.97}, 0.93, 1.46};
constexpr TileCost kCostPairs{{0.30, 0.48, 0.80}, {0.85, 1.20}, 1.18, 1.97};
constexpr u32 kUnits = 256;

inline double tiles_cost(const TileCost &c, u32 edge, u64 tiles, double slices)
{
    const double each = (double)((tiles + kUnits - 1) / kUnits);
    if (edge == 256) return 4.5 + each * (7.0 + slices * c.slice256);
    if (edge == 192) return 4.5 + each * (4.6 + slices * c.slice192);
    if (edge == 128) {
        const double twos = (double)((u64)each / 2), one = each - 2 * twos;
        return 4.5 + twos * (3.1 + slices * c.slice128[1]) + one * (1.5 + slices * c.slice128[0]);
    }
    const double threes = (double)((u64)each / 3), rest = each - 3 * threes;
    return 4.5 + threes * (1.5 + slices * c.slice64[2]) + (rest > 0 ? 0.5 * rest + slices * c.slice64[(int)rest - 1] : 0.0);
}

}  // namespace rtopk
