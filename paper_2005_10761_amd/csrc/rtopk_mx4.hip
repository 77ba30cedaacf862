// A layer's products in 4-bit floating point with a scale for each block of 32 numbers of the contraction.
//
//   numbers    0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives (E2M1: sign, two exponent bits, one mantissa bit), two
//              a byte, the even one in the lower half; a block's scale is the byte b for 2^(b - 127), 255 for NaN
//   quantise   the least scale with max |x| < 7 scale (7 would round to 8, which there is not), x / scale to the
//              nearest number, ties to even: no number is off by more than half a step. Drawn: the least scale with
//              max |x| <= 6 scale, and up or down by chance, so that the mean is x / scale
//   product    out[i][j] = sum over blocks of a_scale[i] b_scale[j] sum_32 a[i] b[j], + bias[j]
//
// A scale is a power of two, so all of the quantisation is exact but its one rounding; the matrix instruction takes
// 128 numbers of a row with four scales, lane l has row l % 16 and block l / 16 of them, and its sums are binary32.
// The scales lie turned over, [blocks][rows]: what neighbouring lanes need together is together in memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/rtopk.h"
#include "../../include/rtopk_diag.h"
#include "rtopk_tile4.h"

namespace rtopk {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// Quantisation.
// ---------------------------------------------------------------------------

// The scale's byte of a block whose largest |x| has these bits. One added to the exponent where the mantissa is 7/4 (3/2: more
// than it) or more, by a carry; the least byte, 2^-127, for all that is smaller.
__device__ __forceinline__ u32 scale_byte(u32 largest, bool drawn)
{
    if (largest >= 0x7F800000u) return 255u;
    const u32 exponent = (largest + (drawn ? 0x3FFFFFu : 0x200000u)) >> 23;
    return exponent > 2u ? exponent - 2u : 0u;
}
__device__ __forceinline__ float scale_value(u32 byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// Eight numbers by one scale, the first in the lowest bits; zeros where the scale is NaN.
__device__ __forceinline__ u32 nearest_four_bits(const float (&x)[8], u32 byte)
{
    u32 word = 0;
#if defined(__HIP_DEVICE_COMPILE__)
    const float scale = scale_value(byte);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], scale, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], scale, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], scale, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], scale, 3);
#endif
    return byte == 255u ? 0u : word;
}

// t = |x| / scale lies between two numbers, a step apart, a fraction f above the lower: up where a 16-bit draw u has
// u + 1/2 < 65536 f, which is (whole numbers) u < W, W = 65536 f - 1/2 rounded up; so the place among steps is (W + 65535 - u) >> 16, with the
// lower number's place in W's upper bits. Exact: t / step has 24 bits, and 1/2 is subtracted in one rounding that
// loses none of them that count. (Where t is far below a step, t may have lost bits of an f under 2^-17, which is never up.)
__device__ __forceinline__ u32 drawn_four_bits(float x, float inverse, u32 draw)
{
    const float t = fabsf(x) * inverse;
    const bool two = t >= 2.0f, four = t >= 4.0f;
    const float steps = four ? 32768.0f : two ? 65536.0f : 131072.0f;          // 65536 / step
    const u32 from = four ? 0x4FFFFu : two ? 0x2FFFFu : 0xFFFFu;               // 65535, and the place of 0, of 2 below 2, of 4 below 4
    const u32 w = (u32)ceilf(fmaf(t, steps, -0.5f));
    return (w + from - draw) >> 16 | (__float_as_uint(x) >> 28 & 8u);
}
// The conversion instruction goes up where 2^32 f + seed >= 2^32, for the first number of a pair with the seed as it is, for the second with the
// seed turned left by one. The rule above is 2^32 f >= 65536 u + 32769 where 2^32 f is a whole number: seed = (65535 - u) 65536 +
// 32767. Numbers of up to 11 bits, as halves and bfloat16 have, make f a whole number of 2^-32 wherever up is possible;
// of binary32 the rule is computed (8192 x 4096 bfloat16 by 64 rows a workgroup 27 us so, 33 computed).
template <int kType>
__device__ __forceinline__ u32 drawn_four_bits(const float (&x)[8], u32 byte, const EightDraws &u)
{
    u32 word = 0;
    if constexpr (kType == RTOPK_F32) {
        const float inverse = __uint_as_float((254u - byte) << 23);     // (of NaN's byte: not used)
#pragma unroll
        for (int i = 0; i < 8; ++i) word |= drawn_four_bits(x[i], inverse, u[i]) << (4 * i);
    } else {
#if defined(__HIP_DEVICE_COMPILE__)
        const float scale = scale_value(byte);
        u32 pair[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 two{x[2 * i], x[2 * i + 1]};
            const u32 seed = ~u.word[i] << 16 | 0x7FFFu, other_seed = (~u.word[i] >> 1 & 0x7FFF8000u) | 0x80003FFFu;
            // (the lowest byte alone is asked for: the instruction leaves the others of its result as they were)
            const u32 first = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, two, seed, scale, 0);
            const u32 second = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, two, other_seed, scale, 0);
            pair[i] = (first & 0x0Fu) | (second & ~0x0Fu);
        }
        // the pairs' lowest bytes
        word = __builtin_amdgcn_perm(__builtin_amdgcn_perm(pair[3], pair[2], 0x0C0C0400u), __builtin_amdgcn_perm(pair[1], pair[0], 0x0C0C0400u),
                                     0x05040100u);
#endif
    }
    return byte == 255u ? 0u : word;
}

struct Packed {
    unsigned char *q, *scale;
    u64 ldq, lds;               // bytes from row to row of q, from block to block of scale
};

struct ToPack {
    const void *x;
    u64 ldx;                    // elements
    u32 rows, cols;
    u32 fill;                   // numbers of a row of q: zeros from cols on
    Packed to;
    Drawing drawing;
};

__device__ __forceinline__ u32 magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// largest over the four lanes of a quad
__device__ __forceinline__ u32 quad_max(u32 v)
{
    v = max(v, (u32)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
    return max(v, (u32)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

// Bytes of four-bit numbers from `at` on of a row that has `bytes`
__device__ __forceinline__ void write_bytes(unsigned char *row, u32 at, u32 word, u32 bytes)
{
    if (at + 4u <= bytes) {
        __builtin_memcpy(row + at, &word, 4);
    } else {
#pragma unroll
        for (u32 i = 0; i < 4; ++i)
            if (at + i < bytes) row[at + i] = (unsigned char)(word >> (8 * i));
    }
}

// groups of eight draws of a row of a contraction of so many numbers
__device__ __forceinline__ u32 groups_of(u32 k) { return (k + kBlock - 1) / kBlock * (kBlock / 8); }

// Along rows: a workgroup has kTileRows rows and 512 columns, a lane eight neighbours of a row, four lanes a block. The scales
// lie the other way: they are put together in LDS, kTileRows bytes of each block, and workgroups of neighbouring rows are on
// one XCD, so that its L2 has whole lines of them. Bound by its one read and one write: 16384 x 4096 binary32 53 us, 5.7 TB/s; 8192 x 4096
// bfloat16 16 us, 5.2 TB/s.
constexpr int kPackThreads = 256;
constexpr u32 kTileColumns = 8 * kWave, kTileBlocks = kTileColumns / kBlock;

// tiles of a matrix
template <u32 kTileRows> __host__ __device__ inline u32 row_tiles(const ToPack &g)
{
    return (g.rows + kTileRows - 1) / kTileRows * ((g.fill + kTileColumns - 1) / kTileColumns);
}

template <int kType, bool kDrawn, u32 kTileRows, u32 kThreads>
__device__ __forceinline__ void pack_rows(const ToPack &g, u32 id)
{
    constexpr u32 kWaves = kThreads / kWave, kEach = kTileRows / kWaves, kAtOnce = kEach < 4 ? kEach : 4;
    __shared__ __align__(16) unsigned char scales[kTileBlocks][kTileRows + 4];      // (blocks start in different banks)
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, tiles = (g.rows + kTileRows - 1) / kTileRows;
    const u32 place = xcd_place(id, row_tiles<kTileRows>(g)), tile = place % tiles, strip = place / tiles;
    const u32 r0 = tile * kTileRows + wave * kEach, c = strip * kTileColumns + lane * 8u;
    PhiloxSeed seed{};
    if (kDrawn) seed = g.drawing.get();
    const u32 blocks = (g.fill + kBlock - 1) / kBlock, have = (g.fill + 1u) / 2u;
    const u64 row_bytes = g.ldx * Eight<kType>::kSize;
    Eight<kType> next[kAtOnce];
    auto fetch = [&](u32 r) {
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) next[q].load((const unsigned char *)g.x + min(r + q, g.rows - 1u) * row_bytes, c, g.cols);
    };
    fetch(r0);
    for (u32 done = 0; done < kEach && r0 + done < g.rows; done += kAtOnce) {
        Eight<kType> e[kAtOnce];
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) e[q] = next[q];
        if (done + kAtOnce < kEach) fetch(r0 + done + kAtOnce);
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            const u32 r = r0 + done + q;
            float v[8];
            e[q].numbers(v, (const unsigned char *)g.x + min(r, g.rows - 1u) * row_bytes, c, g.cols);
            u32 largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
            const u32 byte = scale_byte(quad_max(largest), kDrawn);
            u32 word;
            if (kDrawn) word = drawn_four_bits<kType>(v, byte, draw_eight((u64)r * groups_of(g.cols) + c / 8u, kDrawsForRows, seed));
            else word = nearest_four_bits(v, byte);
            if (r < g.rows) write_bytes(g.to.q + r * g.to.ldq, c / 2u, word, have);
            if ((lane & 3u) == 0) scales[lane >> 2][wave * kEach + done + q] = (unsigned char)byte;
        }
    }
    __syncthreads();
    constexpr u32 kPerThread = kTileBlocks * kTileRows / kThreads;          // 1, 2 or 4 neighbours
    const u32 row = threadIdx.x * kPerThread % kTileRows, block = threadIdx.x * kPerThread / kTileRows;
    const u32 r = tile * kTileRows + row, b = strip * kTileBlocks + block;
    if (b >= blocks || r >= g.rows) return;
    unsigned char *to = g.to.scale + b * g.to.lds + r;
    if (r + kPerThread <= g.rows) {
        __builtin_memcpy(to, &scales[block][row], kPerThread);
    } else {
        for (u32 i = 0; r + i < g.rows; ++i) to[i] = scales[block][row + i];
    }
}

template <int kType, bool kDrawn, u32 kTileRows>
__global__ void __launch_bounds__(kPackThreads) k_pack_rows(ToPack g)
{
    const u32 id = blockIdx.y * gridDim.x + blockIdx.x;
    if (id < row_tiles<kTileRows>(g)) pack_rows<kType, kDrawn, kTileRows, kPackThreads>(g, id);
}

// Along columns, and turned over: a wavefront has 32 rows and 64 columns, a lane eight neighbouring rows of four columns; a
// workgroup has eight blocks of 32 rows, which it writes as 128 bytes of each column. Bound by memory (4096 x 4096 binary32 14.2 us, 5.4
// TB/s), drawn by vector instructions, the generator's products a third of their cycles (8192 x 4096 bfloat16 24 us; to the nearest 17). Four rows of eight columns a lane, with shuffles, took 35.
constexpr u32 kTurnWaves = 8, kTurnThreads = kTurnWaves * kWave, kTurnRows = kTurnWaves * kBlock;

struct ToTurn {
    ToPack of;
    float *sums;                // [groups of kTurnRows rows][cols], or null: the sums of the columns
};
struct Turns {
    ToTurn of[2];
    u32 drawn;                  // bit i: of[i] by chance
};

// Four neighbours of a row, as Eight does it.
template <int kType> struct Quad {
    u32 w[kType == 0 ? 4 : 2];
    static constexpr u32 kSize = kType == 0 ? 4u : 2u;
    __device__ __forceinline__ void load(const unsigned char *row, u32 c, u32 cols)
    {
        const GlobalBytes p = cols < 4u ? (GlobalBytes)kNothing : (GlobalBytes)(row + min(c, cols - 4u) * kSize);
        __builtin_memcpy(w, (const void *)p, sizeof w);
    }
    __device__ __forceinline__ void numbers(float (&v)[4], const unsigned char *row, u32 c, u32 cols) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x;
            if (kType == 0) {
                x = __uint_as_float(w[kType == 0 ? i : 0]);
            } else {
                const u16 h = (u16)(w[i >> 1] >> (16 * (i & 1)));
                x = kType == 1 ? __uint_as_float((u32)h << 16) : (float)__builtin_bit_cast(_Float16, h);
            }
            v[i] = c < cols ? x : 0.0f;
        }
        if (c + 4u <= cols) return;
        if (cols >= 4u) {
            const u32 down = c - (cols - 4u);
#pragma unroll
            for (int by = 2; by; by >>= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = down & by ? (i + by < 4 ? v[i + by] : 0.0f) : v[i];
            if (down > 3u) v[0] = v[1] = v[2] = v[3] = 0.0f;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < cols) v[i] = read_as(row, c + i, kType);
        }
    }
};

// largest over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ u32 max_of_four_rows(u32 v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max((u32)a[0], (u32)a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((u32)b[0], (u32)b[1]);
#endif
    return v;
}

template <int kType, bool kDrawn>
__device__ __forceinline__ void pack_columns(const ToTurn &t)
{
    const ToPack &g = t.of;
    constexpr u32 kRow = kTurnRows / 2 + 4;                 // bytes of a column in LDS
    __shared__ __align__(16) unsigned char turned[kWave * kRow];
    __shared__ __align__(16) float sums[4 * kTurnWaves][kWave];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave;
    const u32 c0 = blockIdx.x * kWave, first = blockIdx.y * kTurnRows;
    const u32 blocks = (g.fill + kBlock - 1) / kBlock, block = first / kBlock + wave;     // of a column
    const u32 c_in = 4u * (lane & 15u), part = lane >> 4, c = c0 + c_in, r0 = first + wave * kBlock + 8u * part;
    PhiloxSeed seed{};
    if (kDrawn) seed = g.drawing.get();
    const u64 row_bytes = g.ldx * Quad<kType>::kSize;
    Quad<kType> e[8];
    float v[8][4];
#pragma unroll
    for (u32 b = 0; b < 8; ++b) e[b].load((const unsigned char *)g.x + min(r0 + b, g.rows - 1u) * row_bytes, c, g.cols);
#pragma unroll
    for (u32 b = 0; b < 8; ++b)
        e[b].numbers(v[b], (const unsigned char *)g.x + min(r0 + b, g.rows - 1u) * row_bytes, c, r0 + b < g.rows ? g.cols : 0u);
    u32 bytes = 0;
    f32x4 sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32 largest = 0;
        sum[i] = 0;
#pragma unroll
        for (u32 b = 0; b < 8; ++b) {
            largest = max(largest, magnitude(v[b][i]));
            sum[i] += v[b][i];
        }
        const u32 byte = scale_byte(max_of_four_rows(largest), kDrawn);
        bytes |= byte << (8 * i);
        const float eight[8] = {v[0][i], v[1][i], v[2][i], v[3][i], v[4][i], v[5][i], v[6][i], v[7][i]};
        u32 word;
        if (kDrawn) word = drawn_four_bits<kType>(eight, byte, draw_eight((u64)(c + i) * groups_of(g.rows) + r0 / 8u, kDrawsForColumns, seed));
        else word = nearest_four_bits(eight, byte);
        *(u32 *)(turned + (c_in + i) * kRow + wave * 16u + 4u * part) = word;
    }
    if (part == 0 && c < g.cols && block < blocks) write_bytes(g.to.scale + block * g.to.lds + c, 0, bytes, g.cols - c);
    if (t.sums) *(f32x4 *)&sums[4 * wave + part][c_in] = sum;
    __syncthreads();
    if (t.sums && wave == 0 && c0 + lane < g.cols && first < g.rows) {
        float all = sums[0][lane];
        for (u32 w = 1; w < 4 * kTurnWaves; ++w) all += sums[w][lane];
        t.sums[(u64)blockIdx.y * g.cols + c0 + lane] = all;
    }
    const u32 col = threadIdx.x >> 3, at = 16u * (threadIdx.x & 7u);
    if (c0 + col >= g.cols) return;
    unsigned char *q = g.to.q + (u64)(c0 + col) * g.to.ldq;
    const u32 have = (g.fill + 1u) / 2u, from = first / 2u + at;
    u32 word[4];
#pragma unroll
    for (u32 w = 0; w < 4; ++w) word[w] = *(const u32 *)(turned + col * kRow + at + 4 * w);
    if (from + 16u <= have) {
        __builtin_memcpy(q + from, word, 16);
    } else {
#pragma unroll
        for (u32 w = 0; w < 4; ++w)
            if (from + 4 * w < have) write_bytes(q, from + 4 * w, word[w], have);
    }
}

// One matrix along columns, or two, and (blockIdx.z = 2) one along rows: all that a layer's backward quantises, in one launch (8192 x
// 4096, dy drawn both ways and x: 66 us; in two launches 73, dy both ways from one read, eight by eight numbers a lane, 74).
constexpr u32 kBesideRows = 64;

template <int kType>
__global__ void __launch_bounds__(kTurnThreads) k_pack_columns(Turns both, ToPack rows)
{
    if (blockIdx.z == 2) {
        const u32 id = blockIdx.y * gridDim.x + blockIdx.x;
        if (id >= row_tiles<kBesideRows>(rows)) return;
        if (both.drawn & 1u) pack_rows<kType, true, kBesideRows, kTurnThreads>(rows, id);
        else pack_rows<kType, false, kBesideRows, kTurnThreads>(rows, id);
        return;
    }
    const ToTurn &t = both.of[blockIdx.z];
    if (blockIdx.x * kWave >= t.of.cols || blockIdx.y * kTurnRows >= t.of.fill) return;        // (another matrix is larger)
    if (both.drawn >> blockIdx.z & 1u) pack_columns<kType, true>(t);
    else pack_columns<kType, false>(t);
}

// The sums of the groups of rows together, in binary64, 16 columns a workgroup: two dependent trips to memory, 2.6 us at 32 groups of 4096.
constexpr u32 kJoinColumns = 16, kJoinThreads = 512;

__global__ void __launch_bounds__(kJoinThreads) k_sum_groups(const float *part, u32 groups, u32 cols, float *out)
{
    constexpr u32 kWaves = kJoinThreads / kWave, kAtOnce = kJoinThreads / kJoinColumns;
    __shared__ double sums[kWaves][kJoinColumns];
    const u32 c = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    double sum = 0;
#pragma unroll 4
    for (u32 s = threadIdx.x / kJoinColumns; s < groups; s += kAtOnce) sum += (double)part[(u64)s * cols + min(c, cols - 1u)];
#pragma unroll
    for (int o = kJoinColumns; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
    if (lane_id() < kJoinColumns) sums[threadIdx.x / kWave][lane_id()] = sum;
    __syncthreads();
    if (threadIdx.x >= kJoinColumns || c >= cols) return;
    sum = 0;
#pragma unroll
    for (u32 w = 0; w < kWaves; ++w) sum += sums[w][threadIdx.x];
    out[c] = (float)sum;
}

// Back to numbers: a thread has the neighbours that make 16 bytes of the result, four or eight. Bound by the write: 10,000 x 1500
// binary32 13.3 us, 5.1 TB/s.
struct ToUnpack {
    const unsigned char *q, *scale;
    u64 ldq, lds;
    u32 rows, cols;
    void *out;
    int type;
    u64 ldo;
};

__device__ __forceinline__ float four_bit_value(u32 n)
{
    // the exponent's and the mantissa's bits in binary32's place, its exponent moved up by 126: 1/2 is a subnormal there too
    return __uint_as_float((n & 7u) << 22 | (n & 8u) << 28) * 8.50705917302346158658e37f;      // 2^126
}

// kShort: places fit 32 bits (a division of 64 bits is as long as all else)
template <u32 kEach, bool kShort>
__global__ void __launch_bounds__(256) k_unpack(ToUnpack g)
{
    typedef typename std::conditional<kShort, u32, u64>::type Place;
    const u32 each = (g.cols + kEach - 1) / kEach;
    const u64 all = (u64)g.rows * each;
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < all; at += (u64)gridDim.x * 256) {
        const u32 row = (u32)((Place)at / each), c = (u32)(at - (u64)row * each) * kEach, have = g.cols - c;
        const unsigned char *q = g.q + row * g.ldq + c / 2u;
        u32 word = 0;
        if (have + 1u >= kEach) __builtin_memcpy(&word, q, kEach / 2);
        else
            for (u32 i = 0; 2 * i < have; ++i) word |= (u32)q[i] << (8 * i);
        const u32 byte = g.scale[c / kBlock * g.lds + row];
        const float scale = byte == 255u ? __uint_as_float(0x7FC00000u) : scale_value(byte);
        f32x4 v[2];
#pragma unroll
        for (int i = 0; i < (int)kEach; ++i) v[i >> 2][i & 3] = four_bit_value(word >> (4 * i)) * scale;
        if (kEach == 4) write_four(g.out, row * g.ldo + c, g.type, v[0], have);
        else write_eight(g.out, row * g.ldo + c, g.type, v[0], v[1], have);
    }
}

// ---------------------------------------------------------------------------
// The product.
// ---------------------------------------------------------------------------
struct Product4 {
    const unsigned char *a, *b, *a_scale, *b_scale;
    u64 lda, ldb, lda_scale, ldb_scale;
    u32 m, n, k;                // k: numbers
    const float *bias;
    void *out;
    u64 ldo;
    int type;
    u32 slices_each, splits;    // the contraction in runs of so many slices
    float *part;                // [splits][m][n rounded up to 4], splits > 1 only
};

// The biases of neighbouring columns, zeros where there are none.
__device__ __forceinline__ f32x4 four_biases(const Product4 &g, u32 col)
{
    f32x4 v{0, 0, 0, 0};
    if (g.bias) {
#pragma unroll
        for (u32 c = 0; c < 4; ++c) v[c] = g.bias[min(col + c, g.n - 1u)];
    }
    return v;
}

// Lanes l of the upper half of the wavefront give x and take y of the lanes l - 32; of the odd rows of 16 lanes, and the even ones.
__device__ __forceinline__ void exchange_halves(u32 &x, u32 &y)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = r[0];
    y = r[1];
#endif
}
__device__ __forceinline__ void exchange_rows(u32 &x, u32 &y)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = r[0];
    y = r[1];
#endif
}
__device__ __forceinline__ void exchange_halves(f32x4 &x, f32x4 &y)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32 a = __float_as_uint(x[c]), b = __float_as_uint(y[c]);
        exchange_halves(a, b);
        x[c] = __uint_as_float(a);
        y[c] = __uint_as_float(b);
    }
}
__device__ __forceinline__ void exchange_rows(f32x4 &x, f32x4 &y)
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        u32 a = __float_as_uint(x[c]), b = __float_as_uint(y[c]);
        exchange_rows(a, b);
        x[c] = __uint_as_float(a);
        y[c] = __uint_as_float(b);
    }
}

// The results of a row that lanes l % 16 have together (l / 16 = quarter q: columns 4 size q .. of the 16 size from `col` on), at
// out + at. They change hands among the four lanes, so that each store is of 64 neighbouring bytes of the row; cols: of the
// result, 0 where the row is not there.
__device__ __forceinline__ void write_group(void *out, u64 at, int type, f32x4 (&v)[4], int size, u32 col, u32 cols)
{
    const u32 q = lane_id() >> 4, crossed = 2u * (q & 1u) + (q >> 1);
    auto four = [&](u32 c, const f32x4 &x) {
        if (c < cols) write_four(out, at + c, type, x, cols - c);
    };
    auto eight = [&](u32 c, const f32x4 &x, const f32x4 &y) {
        if (c < cols) write_eight(out, at + c, type, x, y, cols - c);
    };
    if (size == 1) {
        four(col + 4u * q, v[0]);
    } else if (type == RTOPK_F32) {
        exchange_halves(v[0], v[size / 2]);
        if (size == 2) {
            four(col + 4u * crossed, v[0]);
            four(col + 16u + 4u * crossed, v[1]);
        } else {
            exchange_halves(v[1], v[3]);
            exchange_rows(v[0], v[1]);
            exchange_rows(v[2], v[3]);
#pragma unroll
            for (u32 w = 0; w < 4; ++w) four(col + 16u * w + 4u * q, v[w]);
        }
    } else if (size == 2) {
        eight(col + 8u * q, v[0], v[1]);
    } else {
        exchange_halves(v[0], v[2]);
        exchange_halves(v[1], v[3]);
        eight(col + 8u * crossed, v[0], v[1]);
        eight(col + 32u + 8u * crossed, v[2], v[3]);
    }
}

// A tile, or a run of its contraction; the bias is added to the sums in registers, and the result written once. 8192 x 8192 x 8192 266 us,
// 4140 10^12 operations a second; 2048 x 16384 x 4096 78 us, 3520. What bounds it: the matrix units are busy in 49% and 38% of the cycles at 1.8 and 2.2
// GHz; fed from registers, with the barriers and stores but without loads and reads from LDS, these take 194 and 57, and where all numbers are equal
// 203 and 61 (power).
template <class T, bool kWhole>
__global__ void __launch_bounds__(T::kThreads) k_product4(Product4 g)
{
    __shared__ __align__(16) unsigned char lds[T::kLds];
    const u32 rows = (g.m + T::kRowsM - 1) / T::kRowsM, cols = (g.n + T::kRowsN - 1) / T::kRowsN;
    const u32 place = xcd_place(blockIdx.x, gridDim.x), split = place / (rows * cols);
    u32 ti, tj;
    tile_at(place - split * rows * cols, rows, cols, ti, tj);
    const u32 i0 = ti * T::kRowsM, j0 = tj * T::kRowsN, bytes = (g.k + 1u) / 2u;
    const TileRows4 a{g.a + i0 * g.lda, g.m - i0, (u32)g.lda, g.a_scale + i0, (u32)g.lda_scale};
    const TileRows4 b{g.b + j0 * g.ldb, g.n - j0, (u32)g.ldb, g.b_scale + j0, (u32)g.ldb_scale};
    const u32 slices = (bytes + kSlice - 1) / kSlice, from = split * g.slices_each;
    T t;
    t.clear();
    t.template multiply<kWhole>(a, b, bytes, from, min(from + g.slices_each, slices), lds);
    const bool last = g.splits == 1;
    const u64 ld = last ? g.ldo : align_up(g.n, 4);
    void *out = last ? g.out : (void *)(g.part + (u64)split * g.m * ld);
    const int type = last ? g.type : RTOPK_F32;
#pragma unroll
    for (int group = 0; group < T::GroupsN::kCount; ++group) {
        const int first = T::GroupsN::start(group), size = T::GroupsN::size(first);
        const u32 col = j0 + T::result_column(group), group_col = j0 + T::col0() + 16u * first;
        f32x4 bias[4];          // `size` of them
#pragma unroll
        for (int w = 0; w < size; ++w) bias[w] = last ? four_biases(g, col + 4 * w) : f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i) {
            const u32 row = i0 + T::row_at(i);
            f32x4 v[4];         // 4 x size neighbours
#pragma unroll
            for (int e = 0; e < 4 * size; ++e) v[e / 4][e % 4] = t.sum[i][first + e % size][e / size] + bias[e / 4][e % 4];
            write_group(out, row * ld, type, v, size, group_col, row < g.m ? g.n : 0u);
        }
    }
}

// The sums of the runs together, in order, and the bias. Bound by its reads, mostly from the caches: two runs of 1499 x 2003 6.5 us.
__global__ void __launch_bounds__(256) k_product4_join(Product4 g)
{
    const u32 fours = (g.n + 3) / 4;
    const u64 all = (u64)g.m * fours, ld = 4ull * fours;
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < all; at += (u64)gridDim.x * 256) {
        const u32 row = (u32)(at / fours), col = (u32)(at - (u64)row * fours) * 4u;
        f32x4 sum = four_biases(g, col);
        for (u32 s = 0; s < g.splits; ++s) sum += *(const f32x4 *)(g.part + ((u64)s * g.m + row) * ld + col);
        write_four(g.out, row * g.ldo + col, g.type, sum, g.n - col);
    }
}

// ---------------------------------------------------------------------------
// Few tokens: one read of the weights. A workgroup has 16 channels; its wavefronts share the contraction and add up in LDS,
// in order. A lane's 16 bytes of a row of weights are a block, as the instruction takes them, at any alignment; the tokens are
// the other operand, up to 16 of them. Neighbouring workgroups are on one XCD: they share the lines that the scales lie in. Bound by the read of the
// weights and a launch: 16384 x 4096 with one token 10 us, 3.5 TB/s, with sixteen (quantised by a launch before) 16; 10000 x 1500 with one 4.7.
// ---------------------------------------------------------------------------
constexpr u32 kFewTokens = 16;              // at most: what one instruction takes
constexpr u32 kInOne = 8192;                // numbers of x that a workgroup can quantise for itself (one launch less)

struct Few4 {
    Product4 p;                             // a: quantised tokens, or null
    const void *x;
    u64 ldx;
};

__device__ __forceinline__ f32x4 multiply_step(const i32x4 &a, const i32x4 &b, const f32x4 &sum, u32 a_scale, u32 b_scale)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0}, i32x8{b[0], b[1], b[2], b[3], 0, 0, 0, 0},
                                                            sum, 4, 4, 0, (int)a_scale, 0, (int)b_scale);
#else
    return sum;
#endif
}

// bytes of a token in LDS: its numbers, its scales, and 16 more (tokens start in different banks)
__host__ __device__ constexpr u32 token_bytes(u32 steps) { return (u32)align_up(steps * (kStepBytes + kStepBlocks), 16) + 16u; }

// kType: of x, or -1 where it is quantised already
template <int kWaves, int kType>
__global__ void __launch_bounds__(kWaves * kWave) k_few4(Few4 f)
{
    constexpr bool kQuantize = kType >= 0;
    constexpr u32 kBatch = 4, kThreads = kWaves * kWave;
    const Product4 &g = f.p;
    const u32 lane = lane_id(), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 group = xcd_place(blockIdx.x, gridDim.x), quarter = lane >> 4, channel = min(group * 16u + (lane & 15u), g.n - 1u);
    extern __shared__ __align__(16) unsigned char lds[];
    const u32 bytes = (g.k + 1u) / 2u, blocks = (g.k + kBlock - 1) / kBlock, steps = (blocks + kStepBlocks - 1) / kStepBlocks;
    const u32 each = (steps + kWaves - 1) / kWaves, from = min(wave * each, steps), to = min(from + each, steps);
    const unsigned char *w = g.b + channel * g.ldb, *w_scale = g.b_scale + channel;
    f32x4 sum{0, 0, 0, 0};
    i32x4 held[kBatch];
    u32 held_scale[kBatch];
    const u32 whole = min(to, bytes / kStepBytes);
    auto fetch = [&](u32 s) {
        if (s + kBatch <= whole) {
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q) __builtin_memcpy(&held[q], w + (s + q) * kStepBytes + quarter * 16u, 16);
        } else {
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q)
                if (s + q < to) held[q] = load_piece(w, (s + q) * kStepBytes + quarter * 16u, bytes);
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q)
                if (s + q < to) held[q] = cut_piece(held[q], (s + q) * kStepBytes + quarter * 16u, bytes);
        }
        // (behind the last block: its scale again, with numbers 0)
#pragma unroll
        for (u32 q = 0; q < kBatch; ++q)
            if (s + q < to) held_scale[q] = w_scale[min((s + q) * kStepBlocks + quarter, blocks - 1u) * g.ldb_scale];
    };
    const u32 row = token_bytes(steps), scales = steps * kStepBytes;
    if constexpr (kQuantize) {
        // every thread holds up to kHeld pieces of eight, whatever token they are of: one trip to memory. Four threads have a block
        constexpr u32 kHeld = (kInOne / 8 + kFewTokens * 4 * kStepBlocks + kThreads - 1) / kThreads;
        typedef Eight<kQuantize ? kType : 0> E;
        const u64 row_bytes = f.ldx * E::kSize;
        const unsigned char *x = (const unsigned char *)f.x;
        const u32 pieces = steps * kStepBlocks * 4u, all = g.m * pieces;
        E held_x[kHeld];
        u32 token[kHeld], c[kHeld];
#pragma unroll
        for (u32 h = 0; h < kHeld; ++h) {
            if (h * kThreads >= all) break;                 // (uniform)
            const u32 at = threadIdx.x + h * kThreads;
            token[h] = g.m == 1 || at >= all ? 0u : at / pieces;
            c[h] = at >= all ? pieces * 8u : (at - token[h] * pieces) * 8u;     // (beyond: zeros)
            held_x[h].load(x + token[h] * row_bytes, c[h], g.k);
        }
        fetch(from);        // (the first weights are on their way while x is quantised; behind x, for loads come back in order)
#pragma unroll
        for (u32 h = 0; h < kHeld; ++h) {
            if (h * kThreads >= all) break;
            float v[8];
            held_x[h].numbers(v, x + token[h] * row_bytes, c[h], g.k);
            u32 largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
            const u32 byte = scale_byte(quad_max(largest), false), word = nearest_four_bits(v, byte);
            if (threadIdx.x + h * kThreads >= all) continue;
            *(u32 *)(lds + token[h] * row + c[h] / 2u) = word;
            if ((lane & 3u) == 0) lds[token[h] * row + scales + c[h] / kBlock] = (unsigned char)byte;
        }
        lds_barrier();
    } else {
        fetch(from);
    }
    const u32 token = min(lane & 15u, g.m - 1u);
    for (u32 s = from; s < to; s += kBatch) {
        i32x4 now[kBatch];
        u32 now_scale[kBatch];
#pragma unroll
        for (u32 q = 0; q < kBatch; ++q) {
            now[q] = held[q];
            now_scale[q] = held_scale[q];
        }
        if (s + kBatch < to) fetch(s + kBatch);
#pragma unroll
        for (u32 q = 0; q < kBatch; ++q) {
            if (s + q >= to) break;
            const u32 block = (s + q) * kStepBlocks + quarter;
            i32x4 x;
            u32 x_scale;
            if constexpr (kQuantize) {
                x = *(const i32x4 *)(lds + token * row + block * 16u);
                x_scale = lds[token * row + scales + block];
            } else {
                x = *(const i32x4 *)(g.a + token * g.lda + block * 16u);
                x_scale = g.a_scale[block * g.lda_scale + token];
            }
            sum = multiply_step(now[q], x, sum, now_scale[q], x_scale);
        }
    }
    // lane l: token l % 16, channels 4 (l / 16) .. + 3
    __syncthreads();
    f32x4 *part = (f32x4 *)lds;
    if (wave) part[(wave - 1) * kWave + lane] = sum;
    __syncthreads();
    if (wave) return;
    const u32 col = group * 16u + 4u * quarter;
    if (col >= g.n || (lane & 15u) >= g.m) return;
    for (int o = 0; o < kWaves - 1; ++o) sum += part[o * kWave + lane];
    write_four(g.out, token * g.ldo + col, g.type, sum + four_biases(g, col), g.n - col);
}

__global__ void __launch_bounds__(256) k_zero4(float *p, u32 rows, u32 cols, u64 ld)
{
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < (u64)rows * cols; at += (u64)gridDim.x * 256)
        p[at / cols * ld + at % cols] = 0.0f;
}

}  // namespace rtopk

using namespace rtopk;

namespace {

// Offsets inside a tile of 256 rows fit 32 bits.
constexpr u64 kMostSize = 1u << 22;

bool size_ok(u64 v) { return v >= 1 && v <= kMostSize; }
int launched() { return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP; }
bool workspace_ok(const void *p, u64 bytes, u64 need) { return need == 0 || (p && ((uintptr_t)p & 255u) == 0 && bytes >= need); }
u64 bytes_of(u64 k) { return (k + 1) / 2; }
u64 blocks_of(u64 k) { return (k + kBlock - 1) / kBlock; }
// a quantised operand [rows][k]: the distances of its rows and of its scales' blocks
bool packed_ok(u64 rows, u64 k, u64 ldq, u64 lds) { return ldq >= bytes_of(k) && ldq <= kMostSize && lds >= rows && lds <= kMostSize; }

// (a launch has less than 2^32 threads along x)
dim3 row_grid(u32 tiles) { return dim3(std::min(tiles, 1u << 20), (tiles + (1u << 20) - 1) >> 20); }

// 64 rows a workgroup where binary32 is rounded to the nearest, a row is longer than there are rows, and two workgroups a unit are
// left; 16 elsewhere. us with 16 and with 64, of matrices that come from memory: binary32 4096 x 16384 66.0 / 61.4, 2048 x 16384 33.1 / 30.6,
// 4096 x 8192 32.2 / 30.6; but 4096 x 4096 14.8 / 15.9, 16384 x 4096 53.2 / 57.7, drawn 4096 x 16384 66.5 / 68.6, 4096 x 8192 34.5 / 37.5;
// bfloat16 4096 x 16384 35.0 / 36.0, 2048 x 16384 18.6 / 17.7, 8192 x 4096 16.2 / 16.7, drawn 21.9 / 23.7.
template <int kType>
int run_pack_rows(const ToPack &g, bool drawn, hipStream_t stream)
{
    if constexpr (kType == RTOPK_F32) {
        if (!drawn && g.cols > g.rows && row_tiles<64>(g) >= 2 * kUnits) {
            k_pack_rows<kType, false, 64><<<row_grid(row_tiles<64>(g)), kPackThreads, 0, stream>>>(g);
            return launched();
        }
    }
    if (drawn) k_pack_rows<kType, true, 16><<<row_grid(row_tiles<16>(g)), kPackThreads, 0, stream>>>(g);
    else k_pack_rows<kType, false, 16><<<row_grid(row_tiles<16>(g)), kPackThreads, 0, stream>>>(g);
    return launched();
}
int run_pack_rows(const ToPack &g, int type, bool drawn, hipStream_t stream)
{
    return type == RTOPK_F32 ? run_pack_rows<RTOPK_F32>(g, drawn, stream)
           : type == RTOPK_BF16 ? run_pack_rows<RTOPK_BF16>(g, drawn, stream) : run_pack_rows<RTOPK_F16>(g, drawn, stream);
}

u32 turn_groups(u32 rows) { return (rows + kTurnRows - 1) / kTurnRows; }

constexpr u32 kMostAlongY = (1u << 16) - 1;

// `count` matrices along columns, and `rows`, if not null, along rows.
int run_pack_columns(const Turns &t, u32 count, const ToPack *rows, int type, hipStream_t stream)
{
    dim3 grid(1, 1, rows ? 3 : count);
    for (u32 i = 0; i < count; ++i) {
        grid.x = std::max(grid.x, (t.of[i].of.cols + kWave - 1) / kWave);
        grid.y = std::max(grid.y, turn_groups(t.of[i].of.fill));
    }
    if (rows) {
        // (a launch has less than 2^16 workgroups along y: 2^22 rows of few numbers take two along x)
        const u32 tiles = row_tiles<kBesideRows>(*rows);
        grid.x = std::max(grid.x, (tiles + kMostAlongY - 1) / kMostAlongY);
        grid.y = std::max(grid.y, (tiles + grid.x - 1) / grid.x);
    }
    const ToPack other = rows ? *rows : ToPack{};
    if (type == RTOPK_F32) k_pack_columns<RTOPK_F32><<<grid, kTurnThreads, 0, stream>>>(t, other);
    else if (type == RTOPK_BF16) k_pack_columns<RTOPK_BF16><<<grid, kTurnThreads, 0, stream>>>(t, other);
    else k_pack_columns<RTOPK_F16><<<grid, kTurnThreads, 0, stream>>>(t, other);
    return launched();
}

// Tiles have 512 threads, and a launch less than 2^32.
constexpr u64 kMostTiles = 1u << 23;

struct Plan {
    u32 edge, tiles, slices_each, splits;
    u64 part_bytes;
};

// What a launch of tiles costs, in microseconds: a launch, and for the tiles that one compute unit gets one after the other what
// comes before and after their slices, and the slices (128 bytes of every row). Two tiles of 64 or 128 share a unit. From 300
// launches over eighteen shapes of 64 to 16384 rows and columns and contractions of 256 to 20000: the tile and runs that this picks took at
// most 1.02 times the best ones' time there, on the shapes that the figures were fitted to.
double launch_cost(u32 edge, u64 tiles, double slices)
{
    const double each = (double)((tiles + kUnits - 1) / kUnits);
    if (edge == 256) return 3.8 + each * (6.9 + slices * 1.63);
    if (edge == 192) return 3.8 + each * (5.3 + slices * 0.97);
    const double twos = (double)((u64)each / 2), one = each - 2 * twos;
    if (edge == 128) return 3.8 + twos * (3.85 + slices * 0.94) + one * (1.93 + slices * 0.63);
    return 3.8 + twos * (1.47 + slices * 0.48) + one * (0.74 + slices * 0.31);
}

// The tile and the number of runs of the contraction that cost least. Runs cost a launch, and four bytes of every sum written and read. Rows
// that do not start on 128 bytes take two lines for every slice.
Plan plan_product(u32 m, u32 n, u32 k, bool on_lines)
{
    Plan best{};
    double least = 0.0;
    const u32 slices = ((k + 1) / 2 + kSlice - 1) / kSlice;
    for (const u32 edge : {64u, 128u, 192u, 256u}) {
        const u64 tiles = (u64)((m + edge - 1) / edge) * ((n + edge - 1) / edge);
        for (u32 splits = 1; splits <= std::max(1u, std::min(16u, slices / 4)); ++splits) {
            const u32 each = std::max(1u, (slices + splits - 1) / splits);
            if (splits > 1 && (slices + each - 1) / each != splits) continue;
            if (tiles * splits >= kMostTiles && edge < 256) continue;
            double cost = launch_cost(edge, tiles * splits, each * (on_lines ? 1.0 : 1.11));
            if (splits > 1) cost += 2.2 + (double)m * n * splits * 8.0 / 5.5e6;
            if (best.edge && cost >= least) continue;
            least = cost;
            best = Plan{edge, (u32)tiles, each, std::max(1u, (slices + each - 1) / each), 0};
        }
    }
    best.part_bytes = best.splits > 1 ? align_up((u64)best.splits * m * align_up(n, 4) * 4, 256) : 0;
    return best;
}
// what a product of these sizes may need for the runs' sums, however its rows lie
u64 part_bytes(u32 m, u32 n, u32 k) { return std::max(plan_product(m, n, k, false).part_bytes, plan_product(m, n, k, true).part_bytes); }

template <int kEdge, int kStages>
void launch_product4(const Product4 &g, const Plan &p, bool whole, hipStream_t stream)
{
    typedef Tile4<kEdge, kEdge, 2, 4, kStages> T;
    if (whole) k_product4<T, true><<<p.tiles * p.splits, T::kThreads, 0, stream>>>(g);
    else k_product4<T, false><<<p.tiles * p.splits, T::kThreads, 0, stream>>>(g);
}

int run_product4(Product4 g, void *part, hipStream_t stream)
{
    const Plan p = plan_product(g.m, g.n, g.k, ((g.lda | g.ldb) & 127u) == 0);
    g.slices_each = p.slices_each;
    g.splits = p.splits;
    g.part = (float *)part;
    const bool whole = (((uintptr_t)g.a | (uintptr_t)g.b | g.lda | g.ldb) & 15u) == 0 &&
                       (((uintptr_t)g.a_scale | (uintptr_t)g.b_scale | g.lda_scale | g.ldb_scale) & 3u) == 0;
    if (p.edge == 256) launch_product4<256, 2>(g, p, whole, stream);
    else if (p.edge == 192) launch_product4<192, 2>(g, p, whole, stream);
    else if (p.edge == 128) launch_product4<128, 2>(g, p, whole, stream);
    else launch_product4<64, 4>(g, p, whole, stream);
    if (const int rc = launched()) return rc;
    if (p.splits > 1) {
        const u64 blocks = ((u64)g.m * ((g.n + 3) / 4) + 255) / 256;
        k_product4_join<<<(unsigned)std::min<u64>(blocks, 16 * kUnits), 256, 0, stream>>>(g);
        return launched();
    }
    return RTOPK_OK;
}

template <int kWaves>
int launch_few4(const Few4 &f, int type, hipStream_t stream)
{
    const u32 blocks = (f.p.n + 15) / 16, sums = (kWaves - 1) * kWave * 16;
    const u32 tokens = f.p.a ? 0 : f.p.m * token_bytes((f.p.k + 4 * kBlock - 1) / (4 * kBlock));
    const u32 lds = std::max(sums, tokens);
    if (f.p.a) k_few4<kWaves, -1><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else if (type == RTOPK_F32) k_few4<kWaves, RTOPK_F32><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else if (type == RTOPK_BF16) k_few4<kWaves, RTOPK_BF16><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else k_few4<kWaves, RTOPK_F16><<<blocks, kWaves * kWave, lds, stream>>>(f);
    return launched();
}

bool few_tokens(u32 m) { return m <= kFewTokens; }
// Every workgroup of a unit quantises the tokens again: 1 x 4096 by 16384 channels (four a unit) 10.4 us so, with a launch for it 13.
bool in_one(u32 m, u32 k, u32 n) { return few_tokens(m) && (u64)m * k <= kInOne && (u64)m * k * ((n + 16 * kUnits - 1) / (16 * kUnits)) <= 20000; }

// us with 4, 8 and 16 wavefronts: 1 x 1500 by 10000 channels 5.2 / 7 / -, 1 x 4096 by 4096 - / 4.7 / 5.5, 1 x 8192 by 1024 - / 5.6 / 5.0.
int run_few4(const Few4 &f, int type, hipStream_t stream)
{
    return f.p.n > kUnits * 16 ? launch_few4<4>(f, type, stream) : f.p.n > kUnits * 8 ? launch_few4<8>(f, type, stream) : launch_few4<16>(f, type, stream);
}

// rows of quantised numbers in a workspace: whole slices of the contraction, zeros behind the row's end
u64 filled(u32 k) { return align_up(k, 2 * kSlice); }
u64 scale_ld(u32 rows) { return align_up(rows, 16); }

struct Operand {
    unsigned char *q, *scale;
    u64 ldq, lds;
};
Operand take_operand(Cut &cut, u32 rows, u32 k)
{
    Operand o;
    o.ldq = filled(k) / 2;
    o.lds = scale_ld(rows);
    o.q = cut.take<unsigned char>(rows * o.ldq);
    o.scale = cut.take<unsigned char>(filled(k) / kBlock * o.lds);
    return o;
}
ToPack to_pack(const void *x, u64 ldx, u32 rows, u32 cols, u32 fill, const Operand &o, const Drawing &drawing)
{
    return ToPack{x, ldx, rows, cols, fill, Packed{o.q, o.scale, o.ldq, o.lds}, drawing};
}

struct LinearParts {
    Operand x;
    void *part;
};
u64 cut_linear(void *base, u32 m, u32 k, u32 n, LinearParts &p)
{
    Cut cut{(unsigned char *)base};
    if (in_one(m, k, n)) return 0;
    p.x = take_operand(cut, m, k);
    p.part = cut.take<void>(few_tokens(m) ? 0 : part_bytes(m, n, k));
    return cut.at;
}

struct BackwardParts {
    Operand dy, dy_turned, x_turned;
    float *sums;
    void *part;
};
u64 cut_backward(void *base, u32 m, u32 k, u32 n, BackwardParts &p)
{
    Cut cut{(unsigned char *)base};
    p.dy = take_operand(cut, m, n);
    p.dy_turned = take_operand(cut, n, m);
    p.x_turned = take_operand(cut, k, m);
    p.sums = cut.take<float>(4ull * turn_groups(m) * n);
    p.part = cut.take<void>(std::max(part_bytes(m, k, n), part_bytes(n, k, m)));
    return cut.at;
}

}  // namespace

extern "C" int rtopk_quantize_mx4(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx, int along, int rounding,
                                  uint64_t seed, uint64_t step, const uint64_t *step_device, uint8_t *q, uint64_t ldq, uint8_t *scale,
                                  uint64_t lds, void *stream_v)
{
    if (!type_ok(type) || rows > kMostSize || !size_ok(cols) || ldx < cols || ldx > kMostSize) return RTOPK_EINVAL;
    if ((along != RTOPK_ROWS && along != RTOPK_COLUMNS) || (rounding != RTOPK_NEAREST && rounding != RTOPK_DRAWN)) return RTOPK_EINVAL;
    if (along == RTOPK_ROWS ? !packed_ok(rows, cols, ldq, lds) : !packed_ok(cols, rows, ldq, lds)) return RTOPK_EINVAL;
    if (rows == 0) return RTOPK_OK;
    if (!x || !q || !scale) return RTOPK_EINVAL;
    hipStream_t stream = (hipStream_t)stream_v;
    const bool drawn = rounding == RTOPK_DRAWN;
    const ToPack g{x, ldx, (u32)rows, (u32)cols, (u32)(along == RTOPK_ROWS ? cols : rows), Packed{q, scale, ldq, lds},
                   Drawing{seed, step, drawn ? step_device : nullptr}};
    if (along == RTOPK_ROWS) return run_pack_rows(g, type, drawn, stream);
    return run_pack_columns(Turns{{ToTurn{g, nullptr}, {}}, drawn ? 1u : 0u}, 1, nullptr, type, stream);
}

extern "C" int rtopk_dequantize_mx4(const uint8_t *q, uint64_t rows, uint64_t cols, uint64_t ldq, const uint8_t *scale, uint64_t lds,
                                    void *out, int type, uint64_t ldo, void *stream_v)
{
    if (!type_ok(type) || rows > kMostSize || cols > kMostSize || !packed_ok(rows, cols, ldq, lds) || ldo < cols || ldo > kMostSize)
        return RTOPK_EINVAL;
    if (rows == 0 || cols == 0) return RTOPK_OK;
    if (!q || !scale || !out) return RTOPK_EINVAL;
    const ToUnpack g{q, scale, ldq, lds, (u32)rows, (u32)cols, out, type, ldo};
    hipStream_t stream = (hipStream_t)stream_v;
    const bool fours = type == RTOPK_F32;
    const u64 all = rows * (fours ? (cols + 3) / 4 : (cols + 7) / 8);
    const u32 grid = (u32)std::min<u64>((all + 255) / 256, 32 * kUnits);
    const bool fits = all + 256ull * grid < 1ull << 32;
    if (fours) fits ? k_unpack<4, true><<<grid, 256, 0, stream>>>(g) : k_unpack<4, false><<<grid, 256, 0, stream>>>(g);
    else fits ? k_unpack<8, true><<<grid, 256, 0, stream>>>(g) : k_unpack<8, false><<<grid, 256, 0, stream>>>(g);
    return launched();
}

extern "C" int rtopk_matmul_mx4_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || n > kMostSize || k > kMostSize) return RTOPK_EINVAL;
    *bytes = m && n ? part_bytes((u32)m, (u32)n, (u32)k) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_matmul_mx4(const uint8_t *a, const uint8_t *a_scale, const uint8_t *b, const uint8_t *b_scale, const float *bias,
                                uint64_t m, uint64_t n, uint64_t k, uint64_t lda, uint64_t lda_scale, uint64_t ldb, uint64_t ldb_scale,
                                void *out, int out_type, uint64_t ldo, void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(out_type) || rtopk_matmul_mx4_workspace_bytes(m, n, k, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (!packed_ok(m, k, lda, lda_scale) || !packed_ok(n, k, ldb, ldb_scale) || ldo < n) return RTOPK_EINVAL;
    if (m == 0 || n == 0) return RTOPK_OK;
    if (((!a || !b || !a_scale || !b_scale) && k) || !out) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    return run_product4(Product4{a, b, a_scale, b_scale, lda, ldb, lda_scale, ldb_scale, (u32)m, (u32)n, (u32)k, bias, out, ldo, out_type,
                                 0, 0, nullptr},
                        workspace, (hipStream_t)stream_v);
}

extern "C" int rtopk_product_mx4_plan(uint64_t m, uint64_t n, uint64_t k, int on_lines, rtopk_product_plan_t *plan)
{
    if (!plan || !size_ok(m) || !size_ok(n) || k > kMostSize) return RTOPK_EINVAL;
    const Plan p = plan_product((u32)m, (u32)n, (u32)k, on_lines != 0);
    *plan = rtopk_product_plan_t{p.edge, p.tiles, p.splits};
    return RTOPK_OK;
}

extern "C" int rtopk_linear_mx4_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || !size_ok(k) || !size_ok(n)) return RTOPK_EINVAL;
    LinearParts p;
    *bytes = m ? cut_linear(nullptr, (u32)m, (u32)k, (u32)n, p) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_linear_mx4(const void *x, int type, uint64_t m, uint64_t k, uint64_t ldx, const uint8_t *w, const uint8_t *w_scale,
                                uint64_t n, uint64_t ldw, uint64_t ldw_scale, const float *bias, void *out, int out_type, uint64_t ldo,
                                void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || !type_ok(out_type) || rtopk_linear_mx4_workspace_bytes(m, k, n, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (ldx < k || ldx > kMostSize || !packed_ok(n, k, ldw, ldw_scale) || ldo < n) return RTOPK_EINVAL;
    if (m == 0) return RTOPK_OK;
    if (!x || !w || !w_scale || !out) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    LinearParts p{};
    cut_linear(workspace, (u32)m, (u32)k, (u32)n, p);
    const Product4 g{p.x.q, w, p.x.scale, w_scale, p.x.ldq, ldw, p.x.lds, ldw_scale, (u32)m, (u32)n, (u32)k, bias, out, ldo, out_type, 0, 0, nullptr};
    if (in_one((u32)m, (u32)k, (u32)n)) return run_few4(Few4{g, x, ldx}, type, stream);
    if (const int rc = run_pack_rows(to_pack(x, ldx, (u32)m, (u32)k, (u32)filled((u32)k), p.x, Drawing{}), type, false, stream)) return rc;
    return few_tokens((u32)m) ? run_few4(Few4{g, nullptr, 0}, type, stream) : run_product4(g, p.part, stream);
}

extern "C" int rtopk_linear_mx4_backward_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || !size_ok(k) || !size_ok(n)) return RTOPK_EINVAL;
    BackwardParts p;
    *bytes = m ? cut_backward(nullptr, (u32)m, (u32)k, (u32)n, p) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_linear_mx4_backward(const void *dy, const void *x, int type, uint64_t m, uint64_t k, uint64_t n, uint64_t lddy,
                                         uint64_t ldx, const uint8_t *w_turned, const uint8_t *w_turned_scale, uint64_t ldw,
                                         uint64_t ldw_scale, int rounding, uint64_t seed, uint64_t step, const uint64_t *step_device,
                                         void *dx, uint64_t lddx, float *dw, uint64_t lddw, float *db, void *workspace,
                                         uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || rtopk_linear_mx4_backward_workspace_bytes(m, k, n, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if ((rounding != RTOPK_NEAREST && rounding != RTOPK_DRAWN) || lddy < n || lddy > kMostSize) return RTOPK_EINVAL;
    if (dx && (!packed_ok(k, n, ldw, ldw_scale) || lddx < k)) return RTOPK_EINVAL;
    if (dw && (ldx < k || ldx > kMostSize || lddw < k)) return RTOPK_EINVAL;
    if ((!dx && !dw) || (db && !dw)) return RTOPK_EINVAL;
    if (m && (!dy || (dx && (!w_turned || !w_turned_scale)) || (dw && !x))) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    if (m == 0) {
        if (!dw) return RTOPK_OK;
        k_zero4<<<kUnits, 256, 0, stream>>>(dw, (u32)n, (u32)k, lddw);
        if (db) k_zero4<<<1, 256, 0, stream>>>(db, 1, (u32)n, n);
        return launched();
    }
    BackwardParts p;
    cut_backward(workspace, (u32)m, (u32)k, (u32)n, p);
    const bool drawn = rounding == RTOPK_DRAWN;
    const Drawing drawing{seed, step, drawn ? step_device : nullptr};
    const ToPack rows = to_pack(dy, lddy, (u32)m, (u32)n, (u32)filled((u32)n), p.dy, drawing);
    if (dw) {
        const u32 fill = (u32)filled((u32)m);
        const Turns t{{ToTurn{to_pack(dy, lddy, (u32)m, (u32)n, fill, p.dy_turned, drawing), db ? p.sums : nullptr},
                       ToTurn{to_pack(x, ldx, (u32)m, (u32)k, fill, p.x_turned, Drawing{}), nullptr}},
                      drawn ? 1u : 0u};
        if (const int rc = run_pack_columns(t, 2, dx ? &rows : nullptr, type, stream)) return rc;
        if (db) {
            k_sum_groups<<<(unsigned)((n + kJoinColumns - 1) / kJoinColumns), kJoinThreads, 0, stream>>>(p.sums, turn_groups((u32)m), (u32)n, db);
            if (const int rc = launched()) return rc;
        }
    } else if (const int rc = run_pack_rows(rows, type, drawn, stream)) {
        return rc;
    }
    if (dx) {
        if (const int rc = run_product4(Product4{p.dy.q, w_turned, p.dy.scale, w_turned_scale, p.dy.ldq, ldw, p.dy.lds, ldw_scale, (u32)m,
                                                 (u32)k, (u32)n, nullptr, dx, lddx, type, 0, 0, nullptr},
                                        p.part, stream))
            return rc;
    }
    if (!dw) return RTOPK_OK;
    return run_product4(Product4{p.dy_turned.q, p.x_turned.q, p.dy_turned.scale, p.x_turned.scale, p.dy_turned.ldq, p.x_turned.ldq,
                                 p.dy_turned.lds, p.x_turned.lds, (u32)n, (u32)k, (u32)m, nullptr, dw, lddw, RTOPK_F32, 0, 0,
                                 nullptr},
                        p.part, stream);
}
