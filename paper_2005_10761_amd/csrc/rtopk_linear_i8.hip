// A layer's products in 8-bit integers with a scale for each token and each
// channel: what makes the binary32 gradient that the encoder sparsifies.
//
//   quantise   s = max |x| / 127 over a row (a token) or a column (a channel of
//              the contraction over tokens), q = round to nearest even (x / s)
//   product    out[i][j] = a_scale[i] b_scale[j] sum_k a[i][k] b[j][k] + bias[j]
//
// Forward: y = x w^T, x quantised by token, w by output channel. Backward, with
// the same numbers passed straight through the rounding: dx = dy w contracts
// over output channels (dy by token, w by input channel), dw = dy^T x contracts
// over tokens (both by column, turned over so that the tokens run along a row).
// The sums are exact in 32-bit integers; everything after them is binary32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/rtopk.h"
#include "../../include/rtopk_diag.h"
#include "rtopk_matrix.h"

namespace rtopk {

// ---------------------------------------------------------------------------
// Quantisation.
// ---------------------------------------------------------------------------

// The scale of a row or column whose largest |x| has these bits. A row of magnitudes under 127 * 2^-126 counts as zeros
// (its scale would have lost its own bits); one with an infinity or a not-a-number makes everything it goes into NaN.
__device__ __forceinline__ float scale_of(u32 largest)
{
    if (largest >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float s = __uint_as_float(largest) / 127.0f;
    return s < 1.17549435e-38f ? 0.0f : s;
}

// Eight of them by one scale: x / s as a binary32 quotient, to the nearest whole number, ties to even; 0 where the scale
// is 0 or NaN. The product by 1 / s is off the quotient by less than 127 * 2^-22, so it rounds the same way unless it is
// as close to a tie: only then the division is made (a wavefront in ten; all divisions would be as long as the reads and writes).
struct Quantizer {
    float s, inv;
    __device__ __forceinline__ explicit Quantizer(float scale) : s(scale), inv(scale > 0.0f ? 1.0f / scale : 0.0f) {}
    template <int kN>
    __device__ __forceinline__ void operator()(int (&q)[kN], const float (&x)[kN]) const
    {
        bool tie = false;
        float t[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const float y = x[i] * inv;
            t[i] = rintf(y);
            tie |= fabsf(y - t[i]) > 0.4999f;
        }
        if (__any(tie)) {
#pragma unroll
            for (int i = 0; i < kN; ++i) t[i] = rintf(x[i] / s);
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) q[i] = s > 0.0f ? (int)t[i] : 0;
    }
};

__device__ __forceinline__ u32 magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ u32 four_bytes(const int *q)
{
    return ((u32)q[0] & 255u) | ((u32)q[1] & 255u) << 8 | ((u32)q[2] & 255u) << 16 | (u32)q[3] << 24;
}

struct RowsToQuantize {
    const void *x;
    u64 ldx;            // elements
    u32 rows, cols, fill;
    signed char *q;
    u64 ldq;
    float *scale;
};

constexpr int kQuantizeThreads = 256;

// kWavesPerRow wavefronts hold a row in registers, kPieces pieces of eight numbers a lane (kPieces = 0: the row is
// longer, and read twice, the second time from the caches). What lies between cols and fill becomes zero. Bound by its one
// read and one write: 8192 x 4096 bfloat16 20 us, 5.0 TB/s; 4096 x 4096 binary32 18 us, 4.7 TB/s.
template <int kType, int kWavesPerRow, int kPieces>
__global__ void __launch_bounds__(kWavesPerRow > 4 ? kWavesPerRow * kWave : kQuantizeThreads) k_quantize_rows(RowsToQuantize g)
{
    constexpr u32 kWaves = kWavesPerRow > 4 ? kWavesPerRow : 4, kRows = kWaves / kWavesPerRow, kStep = 8u * kWave * kWavesPerRow;
    __shared__ u32 most[kWaves];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave;
    const u32 r = (blockIdx.y * gridDim.x + blockIdx.x) * kRows + wave / kWavesPerRow;
    const bool there = r < g.rows;
    const unsigned char *row = (const unsigned char *)g.x + (there ? r : 0u) * g.ldx * Eight<kType>::kSize;
    const u32 c0 = (wave % kWavesPerRow * kWave + lane) * 8u;
    Eight<kType> held[kPieces ? kPieces : 1];
    u32 largest = 0;
    auto look = [&](const Eight<kType> &e, u32 c) {
        float v[8];
        e.numbers(v, row, c, g.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
    };
    if constexpr (kPieces > 0) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) held[p].load(row, c0 + p * kStep, g.cols);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) look(held[p], c0 + p * kStep);
    } else {
        for (u32 c = c0; c < g.cols; c += kStep) {
            held[0].load(row, c, g.cols);
            look(held[0], c);
        }
    }
    largest = wave_max_dpp(largest);
    if (kWavesPerRow > 1) {
        if (lane == 0) most[wave] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWavesPerRow; ++w) largest = max(largest, most[w]);
    }
    if (!there) return;
    const Quantizer quantize(scale_of(largest));
    if (c0 == 0) g.scale[r] = quantize.s;
    signed char *q = g.q + (u64)r * g.ldq;
    auto write = [&](const Eight<kType> &e, u32 c) {
        float v[8];
        int n[8];
        e.numbers(v, row, c, g.cols);
        quantize(n, v);
        const u32 word[2] = {four_bytes(n), four_bytes(n + 4)};
        if (c + 8u <= g.fill) {
            __builtin_memcpy(q + c, word, 8);
        } else {
#pragma unroll
            for (u32 i = 0; i < 8u; ++i)
                if (c + i < g.fill) q[c + i] = (signed char)(word[i >> 2] >> (8 * (i & 3)));
        }
    };
    if constexpr (kPieces > 0) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) write(held[p], c0 + p * kStep);
    } else {
        for (u32 c = c0; c < g.fill; c += kStep) {
            held[0].load(row, c, g.cols);
            write(held[0], c);
        }
    }
}

// Columns: a first kernel leaves the largest magnitude (and, where asked, the sum) of each column of each run of rows, a
// second one takes the runs together, quantises and turns the matrix over: two reads (a column's scale is known only at its
// end) and one write. 4096 x 4096 binary32: 13 and 18 us, 5.2 and 4.8 TB/s.
constexpr u32 kGroup = 8 * kWave;           // columns of one workgroup of the first, eight a lane
constexpr u32 kMostRuns = 128;

inline u32 run_rows(u32 rows, u32 cols)
{
    // two workgroups a compute unit, 16 rows at least (6000 x 1500 binary32, three groups: 128 runs 9.7 us, 64 runs 12.9)
    const u32 groups = (cols + kGroup - 1) / kGroup, runs = std::min(kMostRuns, (2 * kUnits + groups - 1) / groups);
    return std::max((rows + runs - 1) / runs, 16u);
}
inline u32 runs_of(u32 rows, u32 cols) { return (rows + run_rows(rows, cols) - 1) / run_rows(rows, cols); }

struct ColumnsToQuantize {
    const void *x;
    u64 ldx;
    u32 rows, cols, fill;       // fill: the length that a turned row gets, zeros from `rows` on
    u32 run, runs;
    signed char *q;             // [cols][ldq]
    u64 ldq;
    float *scale;
    u32 *most;                  // [runs][cols]
    float *sums;                // [runs][cols], or null
    float *total;               // [cols], or null
    u32 blocks;                 // of kTurnRows rows that a workgroup of the second turns over
};
// one matrix, or two of one type in the same launches (blockIdx.z): a layer's backward quantises dy and x
struct Columns {
    ColumnsToQuantize of[2];
};

template <int kType>
__global__ void __launch_bounds__(kQuantizeThreads) k_column_most(Columns both)
{
    const ColumnsToQuantize &g = both.of[blockIdx.z];
    constexpr u32 kWaves = kQuantizeThreads / kWave, kAtOnce = 8;
    __shared__ u32 most[kWaves - 1][kGroup];
    __shared__ float sums[kWaves - 1][kGroup];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c = blockIdx.x * kGroup + lane * 8u;
    if (blockIdx.x * kGroup >= g.cols || blockIdx.y >= g.runs) return;        // (the other matrix is larger)
    const u32 r0 = blockIdx.y * g.run, r1 = min(r0 + g.run, g.rows);
    const u64 row_bytes = g.ldx * Eight<kType>::kSize;
    u32 largest[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (u32 r = r0 + wave; r < r1; r += kAtOnce * kWaves) {
        Eight<kType> e[kAtOnce];
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) e[q].load((const unsigned char *)g.x + min(r + q * kWaves, r1 - 1u) * row_bytes, c, g.cols);
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            if (r + q * kWaves >= r1) break;
            float v[8];
            e[q].numbers(v, (const unsigned char *)g.x + (r + q * kWaves) * row_bytes, c, g.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                largest[i] = max(largest[i], magnitude(v[i]));
                sum[i] += v[i];
            }
        }
    }
    if (wave) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            most[wave - 1][i * kWave + lane] = largest[i];
            sums[wave - 1][i * kWave + lane] = sum[i];
        }
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (u32 w = 0; w < kWaves - 1; ++w) {
            largest[i] = max(largest[i], most[w][i * kWave + lane]);
            sum[i] += sums[w][i * kWave + lane];
        }
        if (c + i < g.cols) {
            g.most[(u64)blockIdx.y * g.cols + c + i] = largest[i];
            if (g.sums) g.sums[(u64)blockIdx.y * g.cols + c + i] = sum[i];
        }
    }
}

// A workgroup turns some blocks of 64 columns and 128 rows over: a lane reads eight columns of four rows, and puts
// the four numbers of each column side by side into LDS. The next block is on its way while this one is turned.
constexpr u32 kTurnRows = 128, kMostBlocks = 4;

template <int kType>
__global__ void __launch_bounds__(kQuantizeThreads) k_quantize_columns(Columns both)
{
    const ColumnsToQuantize &g = both.of[blockIdx.z];
    constexpr u32 kParts = kQuantizeThreads / kWave;
    __shared__ float scale[kWave];
    __shared__ u32 most[kParts][kWave];
    __shared__ double sums[kParts][kWave];
    __shared__ u32 turned[kWave][kTurnRows / 4 + 1];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c0 = blockIdx.x * kWave, blocks = g.blocks, first = blockIdx.y * blocks * kTurnRows;
    if (c0 >= g.cols || first >= g.fill) return;
    const bool totals = g.total && first == 0;
    const u64 row_bytes = g.ldx * Eight<kType>::kSize;
    const u32 piece = threadIdx.x & 7u, quad = threadIdx.x >> 3, c = c0 + 8u * piece;       // columns c .. c + 7 of rows 4 quad .. + 3
    Eight<kType> e[4];
    auto load = [&](u32 r0) {
#pragma unroll
        for (u32 b = 0; b < 4; ++b) e[b].load((const unsigned char *)g.x + min(r0 + 4 * quad + b, g.rows - 1u) * row_bytes, c, g.cols);
    };
    load(first);
    {
        const u32 at = min(c0 + lane, g.cols - 1u);
        u32 largest = 0;
        double sum = 0.0;
#pragma unroll 8
        for (u32 s = wave; s < g.runs; s += kParts) largest = max(largest, g.most[(u64)s * g.cols + at]);
        if (totals)
            for (u32 s = wave; s < g.runs; s += kParts) sum += (double)g.sums[(u64)s * g.cols + at];
        most[wave][lane] = largest;
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (u32 w = 1; w < kParts; ++w) {
                largest = max(largest, most[w][lane]);
                sum += sums[w][lane];
            }
            scale[lane] = scale_of(largest);
            if (first == 0 && c0 + lane < g.cols) {
                g.scale[c0 + lane] = scale[lane];
                if (totals) g.total[c0 + lane] = (float)sum;
            }
        }
        __syncthreads();
    }
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = scale[8 * piece + i];
    for (u32 block = 0; block < blocks; ++block) {
        const u32 r0 = first + block * kTurnRows;
        if (r0 >= g.fill) break;
        float v[4][8];
#pragma unroll
        for (u32 b = 0; b < 4; ++b) {
            const u32 r = r0 + 4 * quad + b;
            e[b].numbers(v[b], (const unsigned char *)g.x + min(r, g.rows - 1u) * row_bytes, c, r < g.rows ? g.cols : 0u);
        }
        if (block + 1 < blocks) load(r0 + kTurnRows);
        if (block) __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Quantizer quantize(s[i]);
            int n[4];
            quantize(n, {v[0][i], v[1][i], v[2][i], v[3][i]});
            turned[8 * piece + i][quad] = four_bytes(n);
        }
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < 2; ++h) {
            const u32 col = (threadIdx.x >> 3) + 32 * h, at = 16u * (threadIdx.x & 7u);
            if (c0 + col >= g.cols || r0 + at >= g.fill) continue;
            u32 word[4];
#pragma unroll
            for (u32 b = 0; b < 4; ++b) word[b] = turned[col][at / 4 + b];
            signed char *q = g.q + (u64)(c0 + col) * g.ldq + r0 + at;
            if (r0 + at + 16u <= g.fill) {
                __builtin_memcpy(q, word, 16);
            } else {
#pragma unroll
                for (u32 b = 0; b < 16u; ++b)
                    if (r0 + at + b < g.fill) q[b] = (signed char)(word[b >> 2] >> (8 * (b & 3)));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// The product.
// ---------------------------------------------------------------------------
struct Scaled {
    const signed char *a, *b;
    u64 lda, ldb;
    u32 m, n, k;
    const float *a_scale, *b_scale, *bias;
    void *out;
    u64 ldo;
    int type;
    u32 slices_each, splits;    // the contraction in runs of so many slices
    int *part;                  // [splits][m][n rounded up to 4], splits > 1 only
};

// four neighbours of a row of the result, and their channels' scales and biases
struct Four {
    f32x4 scale, bias;
};
__device__ __forceinline__ Four channels(const Scaled &g, u32 col)
{
    Four f;
    const float *bias = g.bias ? g.bias : (const float *)kNothing;
#pragma unroll
    for (u32 c = 0; c < 4; ++c) {
        const u32 at = min(col + c, g.n - 1u);
        f.scale[c] = g.b_scale[at];
        f.bias[c] = bias[g.bias ? at : 0u];
    }
    return f;
}
__device__ __forceinline__ f32x4 scaled(const f32x4 &sum, float a_scale, const Four &f)
{
    f32x4 v;
#pragma unroll
    for (u32 c = 0; c < 4; ++c) v[c] = fmaf(sum[c] * a_scale, f.scale[c], f.bias[c]);
    return v;
}
__device__ __forceinline__ void write_scaled(const Scaled &g, u32 row, u32 col, const f32x4 &sum, float a_scale, const Four &f)
{
    write_four(g.out, (u64)row * g.ldo + col, g.type, scaled(sum, a_scale, f), g.n - col);
}

// A tile, or a run of its contraction. The scales and the bias are applied to the sums in registers: the result is written
// once, in its type. Bound by the matrix units, at 8192 x 8192 x 8192 by power (2561 10^12 operations a second; 4096: 2365,
// 2048: 1323, a launch of 256 tiles of 128 x 128).
template <class T, bool kWhole>
__global__ void __launch_bounds__(T::kThreads) k_product(Scaled g)
{
    __shared__ __align__(16) unsigned char lds[T::kLds];
    const u32 rows = (g.m + T::kRowsM - 1) / T::kRowsM, cols = (g.n + T::kRowsN - 1) / T::kRowsN;
    const u32 place = xcd_place(blockIdx.x, gridDim.x), split = place / (rows * cols);
    u32 ti, tj;
    tile_at(place - split * rows * cols, rows, cols, ti, tj);
    const u32 i0 = ti * T::kRowsM, j0 = tj * T::kRowsN;
    const TileRows a{(const unsigned char *)g.a + (u64)i0 * g.lda, g.m - i0, (u32)g.lda, g.k};
    const TileRows b{(const unsigned char *)g.b + (u64)j0 * g.ldb, g.n - j0, (u32)g.ldb, g.k};
    const u32 slices = (g.k + kSlice - 1) / kSlice, from = split * g.slices_each;
    T t;
    t.clear();
    t.template multiply<kWhole>(a, b, from, min(from + g.slices_each, slices), lds);
    if (g.splits == 1) {
        float a_scale[T::kFragsM];
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i) a_scale[i] = g.a_scale[min(i0 + T::row_at(i), g.m - 1u)];
#pragma unroll
        for (int j = 0; j < T::kFragsN; ++j) {
            const u32 col = j0 + T::col_at(j);
            if (col >= g.n) continue;
            const Four f = channels(g, col);
#pragma unroll
            for (int i = 0; i < T::kFragsM; ++i) {
                const i32x4 sum = t.sum[i][j];
                const f32x4 v = scaled(f32x4{(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]}, a_scale[i], f);
                t.sum[i][j] = __builtin_bit_cast(i32x4, v);
            }
        }
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i) {
            const u32 row = i0 + T::row_at(i);
            if (row >= g.m) continue;
#pragma unroll
            for (int j = 0; j < T::kFragsN; j += T::step_at(j)) {
                const u32 col = j0 + T::col_at(j);
                const f32x4 v = __builtin_bit_cast(f32x4, t.sum[i][j]), u = __builtin_bit_cast(f32x4, t.sum[i][T::next_to(j)]);
                if (col >= g.n) continue;
                if (T::wide_at(j)) write_eight(g.out, (u64)row * g.ldo + col, g.type, v, u, g.n - col);
                else write_four(g.out, (u64)row * g.ldo + col, g.type, v, g.n - col);
            }
        }
    } else {
        const u64 ld = align_up(g.n, 4);
        int *part = g.part + (u64)split * g.m * ld;
        t.each([&](u32 r, u32 c, const i32x4 &sum) {
            if (i0 + r < g.m && j0 + c < g.n) *(i32x4 *)(part + (u64)(i0 + r) * ld + j0 + c) = sum;
        });
    }
}

// The sums of the runs together (in binary64: whole numbers up to 2^53), and the scales. Bound by their reads, mostly from
// the caches: two runs of 1499 x 2003, 36 MB moved, 12 us.
__global__ void __launch_bounds__(256) k_product_join(Scaled g)
{
    const u32 fours = (g.n + 3) / 4;
    const u64 all = (u64)g.m * fours, ld = 4ull * fours;
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < all; at += (u64)gridDim.x * 256) {
        const u32 row = (u32)(at / fours), col = (u32)(at - (u64)row * fours) * 4u;
        double sum[4] = {0, 0, 0, 0};
        for (u32 s = 0; s < g.splits; ++s) {
            const i32x4 v = *(const i32x4 *)(g.part + ((u64)s * g.m + row) * ld + col);
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += (double)v[c];
        }
        write_scaled(g, row, col, f32x4{(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]}, g.a_scale[row], channels(g, col));
    }
}

// ---------------------------------------------------------------------------
// Few tokens: one read of the weights. A workgroup has 16 channels; its wavefronts share the contraction and add up in
// LDS. A lane's 16 bytes of a row of weights are its part of the instruction's operand as they come, at any alignment; the
// tokens are the other operand, up to 16 of them. Bound by the read of the weights: 16384 x 4096 with 13 tokens 17.6 us,
// 3.8 TB/s; 10000 x 1500 with one token, quantised in the same launch, 6.2 us, of which a launch of nothing is 2.
// ---------------------------------------------------------------------------
constexpr u32 kFewTokens = 16;          // at most: what one instruction takes
constexpr u32 kInOne = 8192;            // numbers of x that a workgroup can quantise for itself (one launch less)

struct Few {
    Scaled s;                           // a: quantised tokens, or null
    const void *x;
    u64 ldx;
};

// kType: of x, or -1 where it is quantised already
template <int kWaves, int kType>
__global__ void __launch_bounds__(kWaves * kWave) k_few(Few f)
{
    constexpr bool kQuantize = kType >= 0;
    constexpr u32 kBatch = 8;
    const Scaled &g = f.s;
    const u32 lane = lane_id(), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const u32 channel = blockIdx.x * 16u + (lane & 15u), piece = (lane >> 4) * 16u;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float token_scale[kFewTokens];
    __shared__ u32 most[kFewTokens];
    const u32 steps = (g.k + 63u) / 64u;
    const u32 each = (steps + kWaves - 1) / kWaves, from = min(wave * each, steps), to = min(from + each, steps);
    const unsigned char *w = (const unsigned char *)g.b + (u64)min(channel, g.n - 1u) * g.ldb;
    i32x4 sum{0, 0, 0, 0}, held[kBatch];
    const u32 whole = min(to, g.k / 64u);
    auto fetch = [&](u32 s) {
        if (s + kBatch <= whole) {
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q) __builtin_memcpy(&held[q], w + (s + q) * 64u + piece, 16);
        } else {
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q)            // (no more loads than steps: rows at odd places are slow to read, 16 x 123 x 1359
                // took 13 us with eight loads for each wavefront, 7 so)
                if (s + q < to) held[q] = load_piece(w, (s + q) * 64u + piece, g.k);
#pragma unroll
            for (u32 q = 0; q < kBatch; ++q)
                if (s + q < to) held[q] = cut_piece(held[q], (s + q) * 64u + piece, g.k);
        }
    };
    fetch(from);                            // the first weights are on their way while x is quantised
    const u32 row = steps * 64u + 16u;      // bytes of a token in LDS (16 more: tokens start in different banks)
    if constexpr (kQuantize) {
        // every thread holds up to kHeld pieces of eight, whatever token they are of: one trip to memory
        constexpr u32 kHeld = (kInOne / 8 + kFewTokens + kWaves * kWave - 1) / (kWaves * kWave);
        typedef Eight<kQuantize ? kType : 0> E;
        const u64 row_bytes = f.ldx * E::kSize;
        const unsigned char *x = (const unsigned char *)f.x;
        const u32 pieces = (g.k + 7u) / 8u, all = g.m * pieces;
        E held_x[kHeld];
        float v[kHeld][8];
        u32 token[kHeld], c[kHeld];
#pragma unroll
        for (u32 h = 0; h < kHeld; ++h) {
            if (h * kWaves * kWave >= all) break;               // (uniform: a short token is one round of 1500 instructions less)
            const u32 at = threadIdx.x + h * kWaves * kWave;
            token[h] = g.m == 1 || at >= all ? 0u : at / pieces;
            c[h] = (at - token[h] * pieces) * 8u;
            if (at >= all) c[h] = pieces * 8u;              // nothing: zeros
            held_x[h].load(x + token[h] * row_bytes, c[h], g.k);
        }
        if (threadIdx.x < kFewTokens) most[threadIdx.x] = 0u;
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < kHeld; ++h) {
            if (h * kWaves * kWave >= all) break;
            held_x[h].numbers(v[h], x + token[h] * row_bytes, c[h], g.k);
            u32 largest = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[h][i]));
            if (g.m == 1) {
                largest = wave_max_dpp(largest);
                if (lane == 0) atomicMax(&most[0], largest);
            } else {
                atomicMax(&most[token[h]], largest);
            }
        }
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < kHeld; ++h) {
            if (h * kWaves * kWave >= all) break;
            const Quantizer quantize(scale_of(most[token[h]]));
            int n[8];
            quantize(n, v[h]);
            if (threadIdx.x + h * kWaves * kWave >= all) continue;
            if (c[h] == 0) token_scale[token[h]] = quantize.s;
            *(uint2 *)(lds + token[h] * row + c[h]) = make_uint2(four_bytes(n), four_bytes(n + 4));
        }
        // what fills a token's last step (the weights there are zeros, but the numbers have to be some)
        for (u32 at = threadIdx.x; at < g.m * 8u; at += kWaves * kWave) {
            const u32 c = (pieces + (at & 7u)) * 8u;
            if (c < steps * 64u) *(uint2 *)(lds + (at >> 3) * row + c) = make_uint2(0u, 0u);
        }
        __syncthreads();
    } else {
        if (threadIdx.x < g.m) token_scale[threadIdx.x] = g.a_scale[threadIdx.x];
    }
    for (u32 s = from; s < to; s += kBatch) {
        i32x4 now[kBatch];
#pragma unroll
        for (u32 q = 0; q < kBatch; ++q) now[q] = held[q];
        if (s + kBatch < to) fetch(s + kBatch);
#pragma unroll
        for (u32 q = 0; q < kBatch; ++q) {
            if (s + q >= to) break;
            const u32 token = min(lane & 15u, g.m - 1u), at = (s + q) * 64u + piece;
            const i32x4 x = kQuantize ? *(const i32x4 *)(lds + token * row + at) : *(const i32x4 *)(g.a + (u64)token * g.lda + at);
            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[q], x, sum, 0, 0, 0);
        }
    }
    // lane l: token l % 16, channels 4 (l / 16) .. + 3
    __syncthreads();
    i32x4 *part = (i32x4 *)lds;
    if (wave) part[(wave - 1) * kWave + lane] = sum;
    __syncthreads();
    if (wave) return;
    const u32 col = blockIdx.x * 16u + 4u * (lane >> 4), token = lane & 15u;
    if (col >= g.n || token >= g.m) return;
    const Four four = channels(g, col);
    // (a sum of kMostSlices slices stays below 2^31: longer contractions do not come here)
    for (int o = 0; o < kWaves - 1; ++o) sum += part[o * kWave + lane];
    write_scaled(g, token, col, f32x4{(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]}, token_scale[token], four);
}

// no tokens: the weights' gradient is zero
__global__ void __launch_bounds__(256) k_zero(float *p, u32 rows, u32 cols, u64 ld)
{
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < (u64)rows * cols; at += (u64)gridDim.x * 256)
        p[at / cols * ld + at % cols] = 0.0f;
}

}  // namespace rtopk

using namespace rtopk;

namespace {

// A sum of so many slices of products of -128 .. 127 stays below 2^31.
constexpr u32 kMostSlices = 1016;

// Tiles have 512 threads, and a launch less than 2^32 (2^22 x 2^15 of few terms would take so many tiles of 128).
constexpr u64 kMostTiles = 1u << 23;

struct Plan {
    u32 edge, tiles, slices, slices_each, splits;
    u64 part_bytes;
};

// The tile and the number of runs of the contraction that cost least. Runs cost a launch, and four bytes of every sum
// written and read. Rows that do not start on 128 bytes take two lines for every slice: a slice is 1.3 times as long
// (1499 x 5001 x 2003, rows 5248 or 5008 bytes apart: 38 / 46 us; 2048 x 4096 x 4096, 4096 or 4160: 37 / 45).
Plan plan_product(u32 m, u32 n, u32 k, bool on_lines)
{
    Plan best{};
    double least = 0.0;
    const u32 slices = (k + kSlice - 1) / kSlice, must = std::max(1u, (slices + kMostSlices - 1) / kMostSlices);
    for (const u32 edge : {64u, 128u, 192u, 256u}) {
        const u64 tiles = (u64)((m + edge - 1) / edge) * ((n + edge - 1) / edge);
        for (u32 splits = must; splits <= std::max(must, std::min(16u, slices / 4)); ++splits) {
            const u32 each = std::max(1u, (slices + splits - 1) / splits);
            if (splits > must && (slices + each - 1) / each != splits) continue;
            if (tiles * splits >= kMostTiles && edge < 256) continue;
            double cost = tiles_cost(kCostBytes, edge, tiles * splits, each * (on_lines ? 1.0 : 1.3));
            if (splits > 1) cost += 3.0 + (double)m * n * splits * 8.0 / 6e6;
            if (best.edge && cost >= least) continue;
            least = cost;
            best = Plan{edge, (u32)tiles, slices, each, std::max(1u, (slices + each - 1) / each), 0};
        }
    }
    best.part_bytes = best.splits > 1 ? align_up((u64)best.splits * m * align_up(n, 4) * 4, 256) : 0;
    return best;
}
// what a product of these sizes may need for the runs' sums, however its rows lie
u64 part_bytes(u32 m, u32 n, u32 k) { return std::max(plan_product(m, n, k, false).part_bytes, plan_product(m, n, k, true).part_bytes); }

// eight columns a lane where the result has 16 bits, four where it (or a run's sums) has 32
template <int kEdge, int kWavesM, int kWavesN, int kStages, bool kAhead>
void launch_product(const Scaled &g, const Plan &p, bool whole, hipStream_t stream)
{
    typedef Tile<kBytes, kEdge, kEdge, kWavesM, kWavesN, kStages, kAhead, kWide> Eights;
    typedef Tile<kBytes, kEdge, kEdge, kWavesM, kWavesN, kStages, kAhead, kRuns> Fours;
    const u32 grid = p.tiles * p.splits;
    if (!whole) k_product<Fours, false><<<grid, Fours::kThreads, 0, stream>>>(g);
    else if (g.type != 0 && p.splits == 1) k_product<Eights, true><<<grid, Eights::kThreads, 0, stream>>>(g);
    else k_product<Fours, true><<<grid, Fours::kThreads, 0, stream>>>(g);
}

template <int kWaves>
void launch_few(const Few &f, int type, hipStream_t stream)
{
    const u32 blocks = (f.s.n + 15) / 16, sums = (kWaves - 1) * kWave * 16;
    const u32 tokens = f.s.a ? 0 : f.s.m * ((f.s.k + 63) / 64 * 64 + 16);
    const u32 lds = std::max(sums, tokens);
    if (f.s.a) k_few<kWaves, -1><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else if (type == RTOPK_F32) k_few<kWaves, RTOPK_F32><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else if (type == RTOPK_BF16) k_few<kWaves, RTOPK_BF16><<<blocks, kWaves * kWave, lds, stream>>>(f);
    else k_few<kWaves, RTOPK_F16><<<blocks, kWaves * kWave, lds, stream>>>(f);
}

// us with the weights in memory, k x n = 4096 x 16384 / 1504 x 10000 / 4096 x 4096 / 8192 x 1024: one token 15 / 7 / 8 / 8, by
// tiles 20 / 11 / 13 / 14; sixteen 23 / 10 / 11 / 13, by tiles 20 / 10 / 13 / 16. (Two and four instructions' worth of
// tokens were slower than tiles: 32 tokens 30 / 12 / 13 / 17, by tiles 21 / 11 / 14 / 16.)
bool few_tokens(u32 m, u32 k) { return m <= kFewTokens && k <= kMostSlices * kSlice; }
// Every workgroup of a unit quantises the tokens again: 16 x 500 by 30000 channels (eight workgroups a unit) 19 us, in a
// launch of its own 10; but 1 x 4096 by 16384 (four) 15, and with that launch 20.
bool in_one(u32 m, u32 k, u32 n)
{
    return few_tokens(m, k) && (u64)m * k <= kInOne && (u64)m * k * ((n + 16 * kUnits - 1) / (16 * kUnits)) <= 20000;
}

// Up to a workgroup a unit each has sixteen wavefronts (4 x 8192 by 1024 channels 12 us, with four wavefronts 15), then four (1 x
// 4096 by 8000 channels 9 us, with sixteen 14).
int run_few(const Few &f, int type, hipStream_t stream)
{
    f.s.n > kUnits * 16 ? launch_few<4>(f, type, stream) : launch_few<16>(f, type, stream);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

int run_product(Scaled g, void *part, hipStream_t stream)
{
    const Plan p = plan_product(g.m, g.n, g.k, ((g.lda | g.ldb) & 127u) == 0);
    g.slices_each = p.slices_each;
    g.splits = p.splits;
    g.part = (int *)part;
    const bool whole = (((uintptr_t)g.a | (uintptr_t)g.b | g.lda | g.ldb) & 15u) == 0;
    if (p.edge == 256) launch_product<256, 2, 4, 2, true>(g, p, whole, stream);
    else if (p.edge == 192) launch_product<192, 2, 4, 3, true>(g, p, whole, stream);
    else if (p.edge == 128) launch_product<128, 2, 4, 2, true>(g, p, whole, stream);
    else launch_product<64, 2, 4, 3, true>(g, p, whole, stream);
    if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    if (p.splits > 1) {
        const u64 blocks = ((u64)g.m * ((g.n + 3) / 4) + 255) / 256;
        k_product_join<<<(unsigned)std::min<u64>(blocks, 16 * kUnits), 256, 0, stream>>>(g);
        if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    }
    return RTOPK_OK;
}

// What every length is limited to: offsets inside a tile of 256 rows fit 32 bits.
constexpr u64 kMostSize = 1u << 22;

bool size_ok(u64 v) { return v >= 1 && v <= kMostSize; }

template <int kType>
void launch_rows(const RowsToQuantize &g, hipStream_t stream)
{
    // what a wavefront's lanes hold in one piece each is 512 numbers: one wavefront for a short row where there are many
    const u32 rows = g.rows, fill = g.fill;
    // (a launch has less than 2^32 threads along x: 2^22 rows of 1024 threads go along y too)
    const auto grid = [](u32 blocks) { return dim3(std::min(blocks, 1u << 20), (blocks + (1u << 20) - 1) >> 20); };
    if (fill <= 512 && rows >= 4 * kUnits) k_quantize_rows<kType, 1, 1><<<grid((rows + 3) / 4), kQuantizeThreads, 0, stream>>>(g);
    else if (fill <= 1024 && rows >= 4 * kUnits) k_quantize_rows<kType, 1, 2><<<grid((rows + 3) / 4), kQuantizeThreads, 0, stream>>>(g);
    else if (fill <= 2048) k_quantize_rows<kType, 4, 1><<<grid(rows), kQuantizeThreads, 0, stream>>>(g);
    else if (fill <= 4096) k_quantize_rows<kType, 4, 2><<<grid(rows), kQuantizeThreads, 0, stream>>>(g);
    else if (fill <= 8192) k_quantize_rows<kType, 4, 4><<<grid(rows), kQuantizeThreads, 0, stream>>>(g);
    else if (fill <= 16384) k_quantize_rows<kType, 16, 2><<<grid(rows), 16 * kWave, 0, stream>>>(g);
    else k_quantize_rows<kType, 16, 0><<<grid(rows), 16 * kWave, 0, stream>>>(g);
}

int quantize_rows(const void *x, int type, u32 rows, u32 cols, u64 ldx, signed char *q, u64 ldq, u32 fill, float *scale,
                  hipStream_t stream)
{
    const RowsToQuantize g{x, ldx, rows, cols, fill, q, ldq, scale};
    if (type == RTOPK_F32) launch_rows<RTOPK_F32>(g, stream);
    else if (type == RTOPK_BF16) launch_rows<RTOPK_BF16>(g, stream);
    else launch_rows<RTOPK_F16>(g, stream);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

u64 column_scratch(u32 rows, u32 cols, bool sums) { return align_up((u64)runs_of(rows, cols) * cols * (sums ? 8 : 4), 256); }

template <int kType>
int launch_columns(const Columns &c, u32 count, hipStream_t stream)
{
    dim3 most(1, 1, count), turn(1, 1, count);
    for (u32 i = 0; i < count; ++i) {
        const ColumnsToQuantize &g = c.of[i];
        most.x = std::max(most.x, (g.cols + kGroup - 1) / kGroup);
        most.y = std::max(most.y, g.runs);
        turn.x = std::max(turn.x, (g.cols + kWave - 1) / kWave);
        turn.y = std::max(turn.y, ((g.fill + kTurnRows - 1) / kTurnRows + g.blocks - 1) / g.blocks);
    }
    k_column_most<kType><<<most, kQuantizeThreads, 0, stream>>>(c);
    if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    k_quantize_columns<kType><<<turn, kQuantizeThreads, 0, stream>>>(c);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

ColumnsToQuantize columns_of(const void *x, u32 rows, u32 cols, u64 ldx, signed char *q, u64 ldq, u32 fill, float *scale,
                             float *total, void *scratch)
{
    const u32 runs = runs_of(rows, cols);
    u32 *most = (u32 *)scratch;
    // as many blocks for a workgroup (each of which takes the runs together) as leave four workgroups a unit
    const u32 groups = (cols + kWave - 1) / kWave, all = (fill + kTurnRows - 1) / kTurnRows;
    const u32 blocks = std::max(1u, std::min(kMostBlocks, (u32)((u64)groups * all / (4 * kUnits))));
    return ColumnsToQuantize{x, ldx, rows, cols, fill, run_rows(rows, cols), runs, q, ldq, scale, most,
                             total ? (float *)(most + (u64)runs * cols) : nullptr, total, blocks};
}

int quantize_columns(const Columns &c, u32 count, int type, hipStream_t stream)
{
    return type == RTOPK_F32 ? launch_columns<RTOPK_F32>(c, count, stream)
           : type == RTOPK_BF16 ? launch_columns<RTOPK_BF16>(c, count, stream) : launch_columns<RTOPK_F16>(c, count, stream);
}

bool workspace_ok(const void *p, u64 bytes, u64 need) { return need == 0 || (p && ((uintptr_t)p & 255u) == 0 && bytes >= need); }

u64 filled(u32 k) { return align_up(k, kSlice); }

struct LinearParts {
    signed char *x;
    float *x_scale;
    void *part;
};
u64 cut_linear(void *base, u32 m, u32 k, u32 n, LinearParts &p)
{
    Cut cut{(unsigned char *)base};
    if (in_one(m, k, n)) return 0;
    p.x = cut.take<signed char>(m * filled(k));
    p.x_scale = cut.take<float>(4ull * m);
    p.part = cut.take<void>(few_tokens(m, k) ? 0 : part_bytes(m, n, k));
    return cut.at;
}

struct BackwardParts {
    signed char *dy, *dy_turned, *x_turned;
    float *dy_scale, *dy_turned_scale, *x_turned_scale;
    void *dy_scratch, *x_scratch, *part;
};
u64 cut_backward(void *base, u32 m, u32 k, u32 n, BackwardParts &p)
{
    Cut cut{(unsigned char *)base};
    p.dy = cut.take<signed char>(m * filled(n));
    p.dy_turned = cut.take<signed char>(n * filled(m));
    p.x_turned = cut.take<signed char>(k * filled(m));
    p.dy_scale = cut.take<float>(4ull * m);
    p.dy_turned_scale = cut.take<float>(4ull * n);
    p.x_turned_scale = cut.take<float>(4ull * k);
    p.dy_scratch = cut.take<void>(column_scratch(m, n, true));
    p.x_scratch = cut.take<void>(column_scratch(m, k, false));
    p.part = cut.take<void>(std::max(part_bytes(m, k, n), part_bytes(n, k, m)));
    return cut.at;
}

}  // namespace

extern "C" int rtopk_quantize_i8_workspace_bytes(uint64_t rows, uint64_t cols, int along, uint64_t *bytes)
{
    if (!bytes || rows > kMostSize || !size_ok(cols) || (along != RTOPK_ROWS && along != RTOPK_COLUMNS)) return RTOPK_EINVAL;
    *bytes = along == RTOPK_ROWS ? 0 : column_scratch((u32)rows, (u32)cols, false);
    return RTOPK_OK;
}

extern "C" int rtopk_quantize_i8(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx, int along, int8_t *q,
                                 uint64_t ldq, float *scale, void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || rtopk_quantize_i8_workspace_bytes(rows, cols, along, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (ldx < cols || ldx > kMostSize || ldq > kMostSize || ldq < (along == RTOPK_ROWS ? cols : rows)) return RTOPK_EINVAL;
    if ((!scale && (rows || along == RTOPK_COLUMNS)) || ((!x || !q) && rows)) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    if (along == RTOPK_ROWS)
        return rows ? quantize_rows(x, type, (u32)rows, (u32)cols, ldx, q, ldq, (u32)cols, scale, stream) : RTOPK_OK;
    if (!rows) {
        k_zero<<<1, 256, 0, stream>>>(scale, 1, (u32)cols, cols);
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
    }
    const Columns c{{columns_of(x, (u32)rows, (u32)cols, ldx, q, ldq, (u32)rows, scale, nullptr, workspace), {}}};
    return quantize_columns(c, 1, type, stream);
}

extern "C" int rtopk_matmul_i8_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || n > kMostSize || k > kMostSize) return RTOPK_EINVAL;
    *bytes = m && n ? part_bytes((u32)m, (u32)n, (u32)k) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_matmul_i8(const int8_t *a, const float *a_scale, const int8_t *b, const float *b_scale, const float *bias,
                               uint64_t m, uint64_t n, uint64_t k, uint64_t lda, uint64_t ldb, void *out, int out_type,
                               uint64_t ldo, void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(out_type) || rtopk_matmul_i8_workspace_bytes(m, n, k, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (lda < k || ldb < k || ldo < n || lda > kMostSize || ldb > kMostSize) return RTOPK_EINVAL;
    if (m == 0 || n == 0) return RTOPK_OK;
    if (((!a || !b) && k) || !a_scale || !b_scale || !out) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    return run_product(Scaled{a, b, lda, ldb, (u32)m, (u32)n, (u32)k, a_scale, b_scale, bias, out, ldo, out_type, 0, 0, nullptr},
                       workspace, (hipStream_t)stream_v);
}

extern "C" int rtopk_product_plan(uint64_t m, uint64_t n, uint64_t k, int on_lines, rtopk_product_plan_t *plan)
{
    if (!plan || !size_ok(m) || !size_ok(n) || k > kMostSize) return RTOPK_EINVAL;
    const Plan p = plan_product((u32)m, (u32)n, (u32)k, on_lines != 0);
    *plan = rtopk_product_plan_t{p.edge, p.tiles, p.splits};
    return RTOPK_OK;
}

extern "C" int rtopk_linear_i8_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || !size_ok(k) || !size_ok(n)) return RTOPK_EINVAL;
    LinearParts p;
    *bytes = m ? cut_linear(nullptr, (u32)m, (u32)k, (u32)n, p) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_linear_i8(const void *x, int type, uint64_t m, uint64_t k, uint64_t ldx, const int8_t *w,
                               const float *w_scale, uint64_t n, uint64_t ldw, const float *bias, void *out, int out_type,
                               uint64_t ldo, void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || !type_ok(out_type) || rtopk_linear_i8_workspace_bytes(m, k, n, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (ldx < k || ldx > kMostSize || ldw < k || ldw > kMostSize || ldo < n) return RTOPK_EINVAL;
    if (m == 0) return RTOPK_OK;
    if (!x || !w || !w_scale || !out) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    LinearParts p{};
    cut_linear(workspace, (u32)m, (u32)k, (u32)n, p);
    const u64 ld = filled((u32)k);
    const Scaled g{p.x, w, ld, ldw, (u32)m, (u32)n, (u32)k, p.x_scale, w_scale, bias, out, ldo, out_type, 0, 0, nullptr};
    if (in_one((u32)m, (u32)k, (u32)n)) return run_few(Few{g, x, ldx}, type, stream);
    if (const int rc = quantize_rows(x, type, (u32)m, (u32)k, ldx, p.x, ld, (u32)ld, p.x_scale, stream)) return rc;
    return few_tokens((u32)m, (u32)k) ? run_few(Few{g, nullptr, 0}, type, stream) : run_product(g, p.part, stream);
}

extern "C" int rtopk_linear_i8_backward_workspace_bytes(uint64_t m, uint64_t k, uint64_t n, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || !size_ok(k) || !size_ok(n)) return RTOPK_EINVAL;
    BackwardParts p;
    *bytes = m ? cut_backward(nullptr, (u32)m, (u32)k, (u32)n, p) : 0;
    return RTOPK_OK;
}

extern "C" int rtopk_linear_i8_backward(const void *dy, const void *x, int type, uint64_t m, uint64_t k, uint64_t n, uint64_t lddy,
                                        uint64_t ldx, const int8_t *w_turned, const float *w_turned_scale, uint64_t ldw, void *dx,
                                        uint64_t lddx, float *dw, uint64_t lddw, float *db, void *workspace,
                                        uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || rtopk_linear_i8_backward_workspace_bytes(m, k, n, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (lddy < n || lddy > kMostSize) return RTOPK_EINVAL;
    if (dx && (ldw < n || ldw > kMostSize || lddx < k)) return RTOPK_EINVAL;
    if (dw && (ldx < k || ldx > kMostSize || lddw < k)) return RTOPK_EINVAL;
    if ((!dx && !dw) || (db && !dw)) return RTOPK_EINVAL;
    if (m && (!dy || (dx && (!w_turned || !w_turned_scale)) || (dw && !x))) return RTOPK_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    if (m == 0) {
        if (!dw) return RTOPK_OK;
        k_zero<<<kUnits, 256, 0, stream>>>(dw, (u32)n, (u32)k, lddw);
        if (db) k_zero<<<1, 256, 0, stream>>>(db, 1, (u32)n, n);
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
    }
    BackwardParts p;
    cut_backward(workspace, (u32)m, (u32)k, (u32)n, p);
    if (dx) {
        const u64 ld = filled((u32)n);
        if (const int rc = quantize_rows(dy, type, (u32)m, (u32)n, lddy, p.dy, ld, (u32)ld, p.dy_scale, stream)) return rc;
        if (const int rc = run_product(Scaled{p.dy, w_turned, ld, ldw, (u32)m, (u32)k, (u32)n, p.dy_scale, w_turned_scale, nullptr,
                                              dx, lddx, type, 0, 0, nullptr},
                                       p.part, stream))
            return rc;
    }
    if (!dw) return RTOPK_OK;
    const u64 ld = filled((u32)m);
    const Columns c{{columns_of(dy, (u32)m, (u32)n, lddy, p.dy_turned, ld, (u32)ld, p.dy_turned_scale, db, p.dy_scratch),
                     columns_of(x, (u32)m, (u32)k, ldx, p.x_turned, ld, (u32)ld, p.x_turned_scale, nullptr, p.x_scratch)}};
    if (const int rc = quantize_columns(c, 2, type, stream)) return rc;
    return run_product(Scaled{p.dy_turned, p.x_turned, ld, ld, (u32)n, (u32)k, (u32)m, p.dy_turned_scale, p.x_turned_scale, nullptr,
                              dw, lddw, RTOPK_F32, 0, 0, nullptr},
                       p.part, stream);
}
