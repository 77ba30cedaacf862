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
// stored), the bytes from row to row and the bytes of a row that count.
struct TileRows {
    const unsigned char *first;
    u32 rows;
    u32 stride;
    u32 bytes;
};

template <Operands kOf, int kM, int kN, int kWavesM, int kWavesN>
struct Tile {
    static constexpr int kRowsM = kM, kRowsN = kN;
    static constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * kWave;
    static constexpr int kStage = (kM + kN) * kSlice, kLds = 2 * kStage;
    static constexpr int kFragsM = kM / kWavesM / 16, kFragsN = kN / kWavesN / 16;
    static constexpr int kLoadsM = kM / 8 / kWaves, kLoadsN = kN / 8 / kWaves, kLoads = kLoadsM + kLoadsN;
    static_assert(kLoadsM * kWaves * 8 == kM && kLoadsN * kWaves * 8 == kN, "every wavefront loads whole groups of eight rows");
    typedef typename Sums<kOf>::type Sum;
    // sum[i][j]: row 16 i + l % 16 of the wavefront's rows of A, rows 16 j + 4 (l / 16) .. + 3 of its rows of B
    Sum sum[kFragsM][kFragsN];

    static __device__ __forceinline__ u32 wave() { return (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)); }
    static __device__ __forceinline__ u32 row0() { return wave() / kWavesN * (kM / kWavesM); }
    static __device__ __forceinline__ u32 col0() { return wave() % kWavesN * (kN / kWavesN); }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) sum[i][j] = Sum{0, 0, 0, 0};
    }

    // LDS holds a slice as rows of eight 16-byte pieces; piece c of row r lies in place c ^ (r / 2 % 8), so
    // that sixteen rows' pieces of one c are in sixteen different groups of banks (two rows fill the 64 banks).
    static __device__ __forceinline__ u32 place(u32 row, u32 piece) { return row * kSlice + ((piece ^ ((row >> 1) & 7u)) << 4); }

    // row of its operand that load q of this lane takes (the lane's piece of it: lane % 8, as placed)
    static __device__ __forceinline__ u32 row_of(int q)
    {
        return ((q < kLoadsM ? q : q - kLoadsM) * kWaves + wave()) * 8u + (lane_id() >> 3);
    }
    // where the wavefront's load q begins in a stage; lane l's 16 bytes follow at 16 l
    static __device__ __forceinline__ u32 stage_at(int q)
    {
        return (q < kLoadsM ? 0 : kM * kSlice) + ((q < kLoadsM ? q : q - kLoadsM) * kWaves + wave()) * 8 * kSlice;
    }

    // Adds the slices [from, to) of both operands. kWhole: rows start on 16 bytes (base and stride), and every slice
    // but a last one that goes beyond `bytes` goes to LDS by loads that pass the registers by, the next one under way
    // while this one is multiplied. The slice that goes beyond, and every slice of rows that start anywhere, comes through
    // registers, where what lies beyond `bytes` is not read and counts as zero.
    template <bool kWhole>
    __device__ __forceinline__ void multiply(const TileRows &a, const TileRows &b, u32 from, u32 to, unsigned char *lds)
    {
#if defined(__HIP_DEVICE_COMPILE__)      // (the host pass does not know the buffer instructions)
        if (from >= to) return;
        const u32 whole = kWhole ? (a.bytes / kSlice < to ? a.bytes / kSlice : to) : from;
        u32 s = from;
        if (kWhole && s < whole) {
            const u32 lane = lane_id();
            u32 offset[kLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows &t = q < kLoadsM ? a : b;
                const u32 r = row_of(q), row = r < t.rows ? r : t.rows - 1u;
                offset[q] = row * t.stride + (((lane & 7u) ^ ((r >> 1) & 7u)) << 4);
            }
            const auto ra = __builtin_amdgcn_make_buffer_rsrc((void *)a.first, 0, 0xFFFFFFFFu, 0x00020000);
            const auto rb = __builtin_amdgcn_make_buffer_rsrc((void *)b.first, 0, 0xFFFFFFFFu, 0x00020000);
            auto load = [&](u32 slice, unsigned char *stage) {
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(q < kLoadsM ? ra : rb,
                                                             (__attribute__((address_space(3))) void *)(stage + stage_at(q)), 16,
                                                             offset[q], slice * kSlice, 0, 0);
            };
            load(s, lds);
            for (; s < whole; ++s) {
                // this wavefront's part of slice s has come; after the barrier everybody's has, and nobody reads the other stage
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                lds_barrier();
                if (s + 1 < whole) load(s + 1, lds + ((s + 1 - from) & 1u) * kStage);
                one_slice(lds + ((s - from) & 1u) * kStage);
            }
        }
        for (; s < to; ++s) {
            unsigned char *stage = lds + ((s - from) & 1u) * kStage;
            i32x4 piece[kLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows &t = q < kLoadsM ? a : b;
                const u32 r = row_of(q), row = r < t.rows ? r : t.rows - 1u;
                const u32 at = s * kSlice + (((lane_id() & 7u) ^ ((r >> 1) & 7u)) << 4);
                const unsigned char *p = t.first + (u64)row * t.stride + at;
                if (at + 16u <= t.bytes) {
                    __builtin_memcpy(&piece[q], p, 16);
                } else {
                    u32 word[4] = {0u, 0u, 0u, 0u};
                    for (u32 c = 0; at + c < t.bytes; ++c) word[c >> 2] |= (u32)p[c] << (8u * (c & 3u));
                    piece[q] = i32x4{(int)word[0], (int)word[1], (int)word[2], (int)word[3]};
                }
            }
#pragma unroll
            for (int q = 0; q < kLoads; ++q) *(i32x4 *)(stage + stage_at(q) + lane_id() * 16u) = piece[q];
            lds_barrier();      // (a stage is written again two slices later: the barrier between keeps its readers apart)
            one_slice(stage);
        }
#endif
    }

    // one slice that lies in LDS, into the sums
    __device__ __forceinline__ void one_slice(const unsigned char *stage)
    {
        const u32 lane = lane_id();
        const u32 ra = row0() + (lane & 15u), rb = col0() + (lane & 15u);
        i32x4 fa[2][kFragsM], fb[2][kFragsN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < kFragsN; ++j)
                fb[h][j] = *(const i32x4 *)(stage + kM * kSlice + place(rb + 16 * j, 4 * h + (lane >> 4)));
#pragma unroll
            for (int i = 0; i < kFragsM; ++i) fa[h][i] = *(const i32x4 *)(stage + place(ra + 16 * i, 4 * h + (lane >> 4)));
        }
        if (kOf == kPairs) {
            add(fa[0], fb[0]);
            add(fa[1], fb[0]);
            add(fa[0], fb[1]);
        } else {
            add(fa[0], fb[0]);
            add(fa[1], fb[1]);
        }
    }

    __device__ __forceinline__ void add(const i32x4 (&fa)[kFragsM], const i32x4 (&fb)[kFragsN])
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) {
                if constexpr (kOf == kBytes)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], sum[i][j], 0, 0, 0);
                else
                    sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, fb[j]),
                                                                       __builtin_bit_cast(f16x8, fa[i]), sum[i][j], 0, 0, 0);
            }
    }

    // act(row, col, sums): this lane's sums of rows row of A and col .. col + 3 of B, counted from the tile's first
    template <class Act>
    __device__ __forceinline__ void each(Act act) const
    {
        const u32 r = row0() + (lane_id() & 15u), c = col0() + 4u * (lane_id() >> 4);
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) act(r + 16u * i, c + 16u * j, sum[i][j]);
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

__device__ __forceinline__ u16 half_bits(float v, int type)
{
    return type == 1 ? __builtin_bit_cast(u16, (__bf16)v) : __builtin_bit_cast(u16, (_Float16)v);
}

__device__ __forceinline__ void write_as(void *p, u64 at, int type, float v)
{
    if (type == 0) ((float *)p)[at] = v;
    else ((u16 *)p)[at] = half_bits(v, type);
}

// Four neighbours, of which `have` are there; `wide`: all four places start on 4 elements' bytes.
__device__ __forceinline__ void write_four(void *p, u64 at, int type, const f32x4 &v, u32 have, bool wide)
{
    typedef u16 u16x4 __attribute__((ext_vector_type(4)));
    if (wide && have >= 4u) {
        if (type == 0) *(f32x4 *)((float *)p + at) = v;
        else *(u16x4 *)((u16 *)p + at) = u16x4{half_bits(v[0], type), half_bits(v[1], type), half_bits(v[2], type), half_bits(v[3], type)};
    } else {
#pragma unroll
        for (u32 c = 0; c < 4; ++c)
            if (c < have) write_as(p, at + c, type, v[c]);
    }
}

inline u32 type_bytes(int type) { return type == 0 ? 4u : 2u; }

}  // namespace rtopk
