// The matrix core of the 4-bit products (gfx950): C = A B^T for two operands whose rows run along the contraction, two
// numbers a byte, with a byte of scale for each block of 32 numbers (16 bytes) of a row.
//
// One instruction, v_mfma_scale_f32_16x16x128_f8f6f4, takes 64 bytes of 16 rows of each operand: lane l has row l % 16
// and block l / 16 of them, 16 bytes, and that block's scale as a byte of a word. The scales lie turned over
// ([blocks][rows]), and a lane's rows are neighbours by fours: so its scales for four fragments are one word, and each
// instruction takes its byte of it. It also means that a lane ends up with sixteen neighbouring columns of a result's row.
#pragma once

#include <utility>

#include "rtopk_matrix.h"

namespace rtopk {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr u32 kBlock = 32, kBlockBytes = 16;        // numbers that share a scale, and their bytes
constexpr u32 kStepBytes = 64, kStepBlocks = 4;     // of a row, in one instruction

// One operand of a tile: the row that the tile starts with, the rows that are there from it on (rows past them repeat the
// last one: what they give is not stored), the bytes from row to row; the scales of the first block from that row on and
// the bytes from block to block.
struct TileRows4 {
    const unsigned char *first;
    u32 rows, stride;
    const unsigned char *scale;
    u32 scale_stride;
};

// The fragments of 16 rows that a wavefront has of one operand, by groups: fours, then a two, then a one. Row r of fragment i
// is row size * r + (i - first) of its group.
template <int kFrags> struct Groups {
    static constexpr int kFours = kFrags / 4 * 4, kCount = kFrags / 4 + kFrags % 4 / 2 + kFrags % 2;
    // first fragment, number of fragments and place of the group that fragment i is in
    static constexpr int first(int i) { return i < kFours ? i / 4 * 4 : kFrags % 4 >= 2 && i < kFours + 2 ? kFours : kFrags - 1; }
    static constexpr int size(int i) { return i < kFours ? 4 : kFrags % 4 >= 2 && i < kFours + 2 ? 2 : 1; }
    static constexpr int place(int i) { return i < kFours ? i / 4 : kFours / 4 + (kFrags % 4 >= 2 && i >= kFours + 2 ? 1 : 0); }
    // first fragment of group g
    static constexpr int start(int g) { return 4 * g < kFours ? 4 * g : g == kFours / 4 ? kFours : kFrags - 1; }
    static __device__ __forceinline__ u32 row(int i, u32 r) { return 16u * first(i) + size(i) * r + (i - first(i)); }
};

// A tile of kM x kN sums on kWavesM x kWavesN wavefronts. The contraction goes in units of two instructions, a slice of 128 bytes of
// every row; kStages units lie in LDS, and the fragments of the next step are read into registers while this one's are multiplied.
// (Units of one instruction, four in LDS: 2048 x 16384 x 4096 82 us, these 76.)
template <int kM, int kN, int kWavesM, int kWavesN, int kStages>
struct Tile4 {
    static constexpr int kRowsM = kM, kRowsN = kN, kSteps = 2;
    static constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * kWave;
    static constexpr int kRow = kSteps * kStepBytes, kPieces = kRow / 16;        // bytes of a row in a unit, in pieces of 16
    static constexpr int kBlocks = kSteps * kStepBlocks;
    static constexpr int kTogether = kWave / kPieces;                       // rows of one load of a wavefront
    static constexpr int kLoads = (kM + kN) / kTogether / kWaves;
    // scales of a unit: [kBlocks][kM] of A, [kBlocks][kN] of B, in whole loads of 256 bytes for every wavefront
    static constexpr int kScales = kBlocks * (kM + kN), kScaleLoads = (kScales + kWaves * 256 - 1) / (kWaves * 256);
    static constexpr int kData = (kM + kN) * kRow, kStage = kData + kScaleLoads * kWaves * 256, kLds = kStages * kStage;
    static constexpr int kAllLoads = kLoads + kScaleLoads;
    static constexpr int kFragsM = kM / kWavesM / 16, kFragsN = kN / kWavesN / 16;
    typedef Groups<kFragsM> GroupsM;
    typedef Groups<kFragsN> GroupsN;
    static_assert(kLoads * kWaves * kTogether == kM + kN && kM % kTogether == 0, "every wavefront loads whole groups of rows of one operand");
    static_assert(kFragsM * kWavesM * 16 == kM && kFragsN * kWavesN * 16 == kN, "whole instructions");
    static_assert(kBlocks * kM % 256 == 0, "a load of scales is of one operand");
    static_assert(kRow == kSlice, "a unit is a slice");
    static_assert(kStages >= 2 && kStages % 2 == 0 && kLds <= 160 * 1024, "stages");

    // sum[i][j]: row row_at(i) of A, rows of B by result_column()
    f32x4 sum[kFragsM][kFragsN];
    struct Step {
        i32x4 a[kFragsM], b[kFragsN];
        u32 a_scale[GroupsM::kCount], b_scale[GroupsN::kCount];
    };

    static __device__ __forceinline__ u32 wave() { return (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)); }
    static __device__ __forceinline__ u32 row0() { return wave() / kWavesN * (kM / kWavesM); }
    static __device__ __forceinline__ u32 col0() { return wave() % kWavesN * (kN / kWavesN); }
    static __device__ __forceinline__ u32 row_at(int i) { return row0() + GroupsM::row(i, lane_id() & 15u); }
    // the first of the 4 * size neighbouring columns that this lane has of a group of fragments of B; number e of them is
    // sum[i][start + e % size][e / size]
    static __device__ __forceinline__ u32 result_column(int g)
    {
        const int i = GroupsN::start(g);
        return col0() + 16u * i + 4u * GroupsN::size(i) * (lane_id() >> 4);
    }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kFragsN; ++j) sum[i][j] = f32x4{0, 0, 0, 0};
    }

    // LDS holds a unit as rows of pieces of 16 bytes; piece c of row r lies in place c ^ turn(r). A 16-byte read takes sixteen
    // lanes at a time, not in their order: 0-3, 12-15, 20-23, 24-27 (eight rows of one piece, eight others of the next) and so
    // on. The turn puts what they read into sixteen different places of the 64 banks, which two rows of eight pieces fill.
    static __device__ __forceinline__ u32 turn(u32 row) { return (row & 2u) | ((row >> 1) & 4u); }
    static __device__ __forceinline__ u32 place(u32 row, u32 piece) { return row * kRow + ((piece ^ turn(row)) << 4); }

    // A unit's rows lie in LDS as the fragments take them: of A, then of B. Load q of this lane: its row there, and of its operand.
    static __device__ __forceinline__ u32 load_row(int q) { return (u32)(q * kWaves + wave()) * kTogether + lane_id() / kPieces; }
    static __device__ __forceinline__ bool load_of_a(int q) { return (u32)(q * kWaves + wave()) * kTogether < kM; }
    static __device__ __forceinline__ u32 dealt(int q)
    {
        constexpr u32 kRowsA = kM / kWavesM, kRowsB = kN / kWavesN;
        const u32 r = load_row(q);
        if (load_of_a(q)) return r / kRowsA * kRowsA + GroupsM::row((int)(r % kRowsA / 16u), r & 15u);
        return (r - kM) / kRowsB * kRowsB + GroupsN::row((int)((r - kM) % kRowsB / 16u), r & 15u);
    }
    // the lane's piece of it, as placed
    static __device__ __forceinline__ u32 load_piece_at(int q) { return ((lane_id() % kPieces) ^ turn(load_row(q))) << 4; }
    // where the wavefront's load q begins in a stage; lane l's 16 bytes follow at 16 l
    static __device__ __forceinline__ u32 stage_at(int q) { return (u32)(q * kWaves + wave()) * 1024u; }

    // A block's scales of kRows rows lie in LDS turned by so many: the four blocks that a step reads at the same rows, 64 bytes of each,
    // fill the 64 banks (as they come, the reads of a 256-row tile meet four in a bank: a tenth of the cycles in which LDS works).
    template <int kRows> static __device__ __forceinline__ u32 turned_by(u32 block)
    {
        return kRows == 256 ? 64u * (block & 3u) : kRows == 128 ? 64u * (block >> 1 & 1u) : 0u;
    }
    template <int kRows> static __device__ __forceinline__ u32 turned(u32 block, u32 row)
    {
        const u32 at = row + turned_by<kRows>(block);
        return at < kRows ? at : at - kRows;
    }
    // Where the wavefront's load q of scales begins among a stage's scales (lane l's four follow at 4 l), and what they are.
    static __device__ __forceinline__ u32 scales_at(int q) { return (u32)(q * kWaves + wave()) * 256u; }
    static __device__ __forceinline__ bool scales_of_a(int q) { return scales_at(q) < kBlocks * kM; }
    struct ScalePlace {
        u32 block, row;
    };
    template <int kRows> static __device__ __forceinline__ ScalePlace unturned(u32 at)
    {
        const u32 block = at / kRows, row = at % kRows, by = turned_by<kRows>(block);
        return {block, row >= by ? row - by : row + kRows - by};
    }
    static __device__ __forceinline__ ScalePlace scale_place(int q)
    {
        const u32 at = scales_at(q) + 4u * lane_id();
        if (at < kBlocks * kM) return unturned<kM>(at);
        if (at < kScales) return unturned<kN>(at - kBlocks * kM);
        return {0u, 0u};                                // (what fills the last loads)
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
    // the same where the kinds of what may be under way are `units` units, fewer than kStages - 1 of them
    static __device__ __forceinline__ void wait_and_meet_for(u32 units)
    {
        if (kStages > 3 && units == 2) wait_and_meet<(kStages > 3 ? 2 : 0) * kAllLoads>();
        else if (kStages > 2 && units == 1) wait_and_meet<(kStages > 2 ? 1 : 0) * kAllLoads>();
        else wait_and_meet<0>();
    }

    // Adds the units [from, to) of both operands, of rows of `bytes` bytes. kWhole: rows start on 16 bytes and scales on 4
    // (base and stride), and every unit but one that goes beyond `bytes` goes to LDS by loads that pass the registers by. The
    // unit that goes beyond, and every unit of rows that start anywhere, comes through registers, where what lies
    // beyond is not read and counts as zero.
    template <bool kWhole>
    __device__ __forceinline__ void multiply(const TileRows4 &a, const TileRows4 &b, u32 bytes, u32 from, u32 to, unsigned char *lds)
    {
#if defined(__HIP_DEVICE_COMPILE__)      // (the host pass does not know the buffer instructions)
        if (from >= to) return;
        u32 full = bytes / kRow;
        // scales are loaded by fours, beyond a last row that is not there; behind the last block nothing may be read
        if (full * kRow == bytes && ((a.rows | b.rows) & 3u)) --full;
        const u32 whole = kWhole ? (full < to ? full : to) : from;
        u32 u = from;
        auto stage = [&](u32 unit) { return lds + (unit - from) % kStages * kStage; };
        if (kWhole && u < whole) {
            u32 offset[kLoads], scale_offset[kScaleLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows4 &t = load_of_a(q) ? a : b;
                offset[q] = min(dealt(q), t.rows - 1u) * t.stride + load_piece_at(q);
            }
#pragma unroll
            for (int q = 0; q < kScaleLoads; ++q) {
                const TileRows4 &t = scales_of_a(q) ? a : b;
                const ScalePlace at = scale_place(q);
                scale_offset[q] = at.block * t.scale_stride + min(at.row, (t.rows - 1u) & ~3u);
            }
            const auto ra = __builtin_amdgcn_make_buffer_rsrc((void *)a.first, 0, 0xFFFFFFFFu, 0x00020000);
            const auto rb = __builtin_amdgcn_make_buffer_rsrc((void *)b.first, 0, 0xFFFFFFFFu, 0x00020000);
            auto load = [&](u32 unit) {
                unsigned char *to_lds = stage(unit);
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(load_of_a(q) ? ra : rb,
                                                             (__attribute__((address_space(3))) void *)(to_lds + stage_at(q)), 16, offset[q],
                                                             unit * kRow, 0, 0);
#pragma unroll
                for (int q = 0; q < kScaleLoads; ++q) {
                    const TileRows4 &t = scales_of_a(q) ? a : b;
                    const auto r = __builtin_amdgcn_make_buffer_rsrc((void *)(t.scale + (u64)(unit * kBlocks) * t.scale_stride), 0, 0xFFFFFFFFu,
                                                                     0x00020000);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(to_lds + kData + scales_at(q)), 4,
                                                             scale_offset[q], 0, 0, 0);
                }
            };
#pragma unroll
            for (int q = 0; q < kStages; ++q)
                if (u + q < whole) load(u + q);
            if (u + kStages <= whole) wait_and_meet<(kStages - 1) * kAllLoads>();
            else wait_and_meet<0>();
            Step even, odd;
            read(even, stage(u), 0);
            // From a unit whose first step's fragments are in `even` to the next one's. A barrier says that everybody has read all of
            // this unit, and that the next one has come; then this one's stage is loaded again. (Copies of a unit's work, so that
            // none of them branches: a branch stops the reads from going between the products.)
            auto pass = [&](bool more, u32 under_way) __attribute__((always_inline)) {
                read(odd, stage(u), 1);
                add(even);
                mix<0>();
                if (more) wait_and_meet<(kStages - 2) * kAllLoads>();
                else wait_and_meet_for(under_way);
                if (more) load(u + kStages);
                read(even, stage(u + 1), 0);
                add(odd);
                if (more) mix<kAllLoads>();
                else mix<0>();
                ++u;
            };
            while (u + kStages < whole) pass(true, 0);
            while (u + 1 < whole) pass(false, whole - u - 2);
            read(odd, stage(u), 1);
            add(even);
            mix<0>();
            add(odd);
            ++u;
        }
        const u32 blocks = (bytes + kBlockBytes - 1) / kBlockBytes;
        for (; u < to; ++u) {
            unsigned char *to_lds = stage(u);
            i32x4 piece[kLoads];
            u32 scales[kScaleLoads];
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const TileRows4 &t = load_of_a(q) ? a : b;
                piece[q] = load_piece(t.first + (u64)min(dealt(q), t.rows - 1u) * t.stride, u * kRow + load_piece_at(q), bytes);
            }
#pragma unroll
            for (int q = 0; q < kScaleLoads; ++q) {
                const TileRows4 &t = scales_of_a(q) ? a : b;
                const ScalePlace at = scale_place(q);
                const u32 block = u * kBlocks + at.block;
                scales[q] = 0;
#pragma unroll
                for (u32 c = 0; c < 4; ++c)
                    if (block < blocks && at.row + c < t.rows) scales[q] |= (u32)t.scale[(u64)block * t.scale_stride + at.row + c] << (8 * c);
            }
#pragma unroll
            for (int q = 0; q < kLoads; ++q) piece[q] = cut_piece(piece[q], u * kRow + load_piece_at(q), bytes);
            // (everybody has read the unit that lay in this stage, kStages units ago, before the barrier of the one after it)
#pragma unroll
            for (int q = 0; q < kLoads; ++q) *(i32x4 *)(to_lds + stage_at(q) + lane_id() * 16u) = piece[q];
#pragma unroll
            for (int q = 0; q < kScaleLoads; ++q) *(u32 *)(to_lds + kData + scales_at(q) + lane_id() * 4u) = scales[q];
            lds_barrier();
#pragma unroll
            for (int h = 0; h < kSteps; ++h) {
                Step s;
                read(s, to_lds, h);
                add(s);
            }
        }
#endif
    }

    // step h of a unit in LDS
    __device__ __forceinline__ void read(Step &f, const unsigned char *stage, u32 h) const
    {
        const u32 ra = row0() + (lane_id() & 15u), rb = kM + col0() + (lane_id() & 15u), piece = 4 * h + (lane_id() >> 4);
        const unsigned char *scales = stage + kData;
#pragma unroll
        for (int g = 0; g < GroupsN::kCount; ++g) f.b_scale[g] = read_scales<GroupsN, kN>(scales + kBlocks * kM, piece, col0(), g);
#pragma unroll
        for (int g = 0; g < GroupsM::kCount; ++g) f.a_scale[g] = read_scales<GroupsM, kM>(scales, piece, row0(), g);
#pragma unroll
        for (int j = 0; j < kFragsN; ++j) f.b[j] = *(const i32x4 *)(stage + place(rb + 16 * j, piece));
#pragma unroll
        for (int i = 0; i < kFragsM; ++i) f.a[i] = *(const i32x4 *)(stage + place(ra + 16 * i, piece));
    }
    // this lane's scales of a group of fragments, the wavefront's rows being `first` on (sizes divide what rows are turned by)
    template <class G, int kRows>
    static __device__ __forceinline__ u32 read_scales(const unsigned char *p, u32 block, u32 first, int g)
    {
        const int i = G::start(g);
        p += block * kRows + turned<kRows>(block, first + 16 * i + G::size(i) * (lane_id() & 15u));
        return G::size(i) == 4 ? *(const u32 *)p : G::size(i) == 2 ? *(const u16 *)p : *p;
    }

    // (the instruction takes which byte of the scales' words it is as a constant)
    template <int kI, int kJ>
    __device__ __forceinline__ void add_one(const Step &f)
    {
#if defined(__HIP_DEVICE_COMPILE__)
        const i32x4 x = f.b[kJ], y = f.a[kI];
        sum[kI][kJ] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0}, i32x8{y[0], y[1], y[2], y[3], 0, 0, 0, 0}, sum[kI][kJ], 4, 4, kJ - GroupsN::first(kJ),
            (int)f.b_scale[GroupsN::place(kJ)], kI - GroupsM::first(kI), (int)f.a_scale[GroupsM::place(kI)]);
#endif
    }
    template <int... kAt>
    __device__ __forceinline__ void add_all(const Step &f, std::integer_sequence<int, kAt...>)
    {
        (add_one<kAt / kFragsN, kAt % kFragsN>(f), ...);
    }
    __device__ __forceinline__ void add(const Step &f) { add_all(f, std::make_integer_sequence<int, kFragsM * kFragsN>()); }

    // the reads of the next step, and loads to LDS, between the products of this one
    template <int kOfLoads>
    __device__ __forceinline__ void mix() const
    {
        constexpr int kReads = kFragsM + kFragsN + GroupsM::kCount + GroupsN::kCount;
        constexpr int kPer = kFragsM * kFragsN / (kReads + kOfLoads), kProducts = kPer ? kPer : 1;
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
};

}  // namespace rtopk
