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

// x / s as a binary32 quotient, to the nearest whole number, ties to even; 0 where the scale is 0 or NaN
__device__ __forceinline__ int quantized(float x, float s) { return s > 0.0f ? (int)rintf(x / s) : 0; }

__device__ __forceinline__ u32 magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

struct RowsToQuantize {
    const void *x;
    u64 ldx;            // elements
    u32 rows, cols, fill;
    int type;
    signed char *q;
    u64 ldq;
    float *scale;
};

constexpr int kQuantizeThreads = 256;

// kWavesPerRow wavefronts read a row twice (the second time from the caches) and write it once; what lies between cols
// and fill becomes zero.
template <int kWavesPerRow>
__global__ void __launch_bounds__(kQuantizeThreads) k_quantize_rows(RowsToQuantize g)
{
    constexpr u32 kRows = kQuantizeThreads / kWave / kWavesPerRow, kStep = 8u * kWave * kWavesPerRow;
    __shared__ u32 most[kQuantizeThreads / kWave];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave;
    const u32 r = blockIdx.x * kRows + wave / kWavesPerRow;
    const bool there = r < g.rows;
    const unsigned char *row = (const unsigned char *)g.x + (u64)(there ? r : 0u) * g.ldx * (g.type == 0 ? 4u : 2u);
    const bool wide = (((uintptr_t)g.x | (g.ldx * (g.type == 0 ? 4u : 2u))) & 15u) == 0;
    const u32 c0 = (wave % kWavesPerRow * kWave + lane) * 8u;
    u32 largest = 0;
    if (there)
        for (u32 c = c0; c < g.cols; c += kStep) {
            float v[8];
            read_eight(v, row, c, g.cols, g.type, wide);
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(v[i]));
        }
    largest = wave_max_dpp(largest);
    if (kWavesPerRow > 1) {
        if (lane == 0) most[wave] = largest;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWavesPerRow; ++w) largest = max(largest, most[w]);
    }
    if (!there) return;
    const float s = scale_of(largest);
    if (c0 == 0) g.scale[r] = s;
    signed char *q = g.q + (u64)r * g.ldq;
    const bool wide_q = (((uintptr_t)g.q | g.ldq) & 7u) == 0;
    for (u32 c = c0; c < g.fill; c += kStep) {
        float v[8];
        read_eight(v, row, c, g.cols, g.type, wide);
        u32 word[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) word[i >> 2] |= ((u32)quantized(v[i], s) & 255u) << (8 * (i & 3));
        if (wide_q && c + 8u <= g.fill) {
            *(uint2 *)(q + c) = make_uint2(word[0], word[1]);
        } else {
            for (u32 i = 0; i < 8u && c + i < g.fill; ++i) q[c + i] = (signed char)(word[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// Columns: a first kernel leaves the largest magnitude (and, where asked, the sum) of each column of each run of rows, a
// second one takes the runs together, quantises and turns the matrix over.
constexpr u32 kRunRows = 256, kMostRuns = 64;

inline u32 run_rows(u32 rows)
{
    u32 each = kRunRows;
    while ((rows + each - 1) / each > kMostRuns) each *= 2;
    return each;
}
inline u32 runs_of(u32 rows) { return rows ? (rows + run_rows(rows) - 1) / run_rows(rows) : 0u; }

struct ColumnsToQuantize {
    const void *x;
    u64 ldx;
    u32 rows, cols, fill;       // fill: the length that a turned row gets, zeros from `rows` on
    u32 run, runs;
    int type;
    signed char *q;             // [cols][ldq]
    u64 ldq;
    float *scale;
    u32 *most;                  // [runs][cols]
    float *sums;                // [runs][cols], or null
    float *total;               // [cols], or null
};

__global__ void __launch_bounds__(kQuantizeThreads) k_column_most(ColumnsToQuantize g)
{
    __shared__ u32 most[kQuantizeThreads / kWave][kWave];
    __shared__ float sums[kQuantizeThreads / kWave][kWave];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    const u32 r0 = blockIdx.y * g.run, r1 = min(r0 + g.run, g.rows);
    u32 largest = 0;
    float sum = 0.0f;
    if (c < g.cols)
        for (u32 r = r0 + wave; r < r1; r += kQuantizeThreads / kWave) {
            const float v = read_as(g.x, (u64)r * g.ldx + c, g.type);
            largest = max(largest, magnitude(v));
            sum += v;
        }
    most[wave][lane] = largest;
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= g.cols) return;
#pragma unroll
    for (int w = 1; w < kQuantizeThreads / kWave; ++w) {
        largest = max(largest, most[w][lane]);
        sum += sums[w][lane];
    }
    g.most[(u64)blockIdx.y * g.cols + c] = largest;
    if (g.sums) g.sums[(u64)blockIdx.y * g.cols + c] = sum;
}

constexpr u32 kTurnRows = 128;

__global__ void __launch_bounds__(kQuantizeThreads) k_quantize_columns(ColumnsToQuantize g)
{
    __shared__ float scale[kWave];
    __shared__ u32 turned[kWave][kTurnRows / 4 + 1];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c0 = blockIdx.x * kWave, c = c0 + lane, r0 = blockIdx.y * kTurnRows;
    if (wave == 0 && c < g.cols) {
        u32 largest = 0;
        double sum = 0.0;
        for (u32 s = 0; s < g.runs; ++s) {
            largest = max(largest, g.most[(u64)s * g.cols + c]);
            if (g.total && r0 == 0) sum += (double)g.sums[(u64)s * g.cols + c];
        }
        scale[lane] = scale_of(largest);
        if (r0 == 0) {
            g.scale[c] = scale[lane];
            if (g.total) g.total[c] = (float)sum;
        }
    }
    __syncthreads();
    const float s = c < g.cols ? scale[lane] : 0.0f;
    for (u32 i = wave; i < kTurnRows / 4; i += kQuantizeThreads / kWave) {
        u32 word = 0;
#pragma unroll
        for (u32 b = 0; b < 4; ++b) {
            const u32 r = r0 + 4 * i + b;
            if (c < g.cols && r < g.rows) word |= ((u32)quantized(read_as(g.x, (u64)r * g.ldx + c, g.type), s) & 255u) << (8 * b);
        }
        turned[lane][i] = word;
    }
    __syncthreads();
    const bool wide = (((uintptr_t)g.q | g.ldq) & 3u) == 0;
    for (u32 i = threadIdx.x; i < kWave * (kTurnRows / 4); i += kQuantizeThreads) {
        const u32 row = c0 + i / (kTurnRows / 4), at = r0 + 4 * (i % (kTurnRows / 4));
        if (row >= g.cols || at >= g.fill) continue;
        const u32 word = turned[i / (kTurnRows / 4)][i % (kTurnRows / 4)];
        signed char *q = g.q + (u64)row * g.ldq + at;
        if (wide && at + 4u <= g.fill) *(u32 *)q = word;
        else
            for (u32 b = 0; b < 4u && at + b < g.fill; ++b) q[b] = (signed char)(word >> (8 * b));
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

__device__ __forceinline__ void write_scaled(const Scaled &g, u32 row, u32 col, const f32x4 &sum)
{
    const float s = g.a_scale[row];
    const u32 have = g.n - col;
    f32x4 v;
#pragma unroll
    for (u32 c = 0; c < 4; ++c) {
        const u32 at = c < have ? col + c : col;
        v[c] = sum[c] * s * g.b_scale[at] + (g.bias ? g.bias[at] : 0.0f);
    }
    const u32 size = g.type == 0 ? 4u : 2u;
    const bool wide = (((uintptr_t)g.out | (g.ldo * size)) & (4u * size - 1u)) == 0;
    write_four(g.out, (u64)row * g.ldo + col, g.type, v, have, wide);
}

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
        t.each([&](u32 r, u32 c, const i32x4 &sum) {
            if (i0 + r < g.m && j0 + c < g.n)
                write_scaled(g, i0 + r, j0 + c, f32x4{(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]});
        });
    } else {
        const u64 ld = align_up(g.n, 4);
        int *part = g.part + (u64)split * g.m * ld;
        t.each([&](u32 r, u32 c, const i32x4 &sum) {
            if (i0 + r < g.m && j0 + c < g.n) *(i32x4 *)(part + (u64)(i0 + r) * ld + j0 + c) = sum;
        });
    }
}

// the sums of the runs together (in binary64: whole numbers up to 2^53), and the scales
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
        write_scaled(g, row, col, f32x4{(float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]});
    }
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

typedef Tile<kBytes, 256, 256, 2, 4, 2, true> Large;
typedef Tile<kBytes, 128, 128, 2, 2, 2, false> Middle;
typedef Tile<kBytes, 64, 64, 2, 2, 2, false> Small;

// A sum of so many slices of products of -128 .. 127 stays below 2^31.
constexpr u32 kMostSlices = 1016;
enum Shape { kLarge, kMiddle, kSmall };
struct Plan {
    Shape shape;
    u32 tiles, slices, slices_each, splits;
    u64 part_bytes;
};

Plan plan_product(u32 m, u32 n, u32 k)
{
    Plan p{};
    auto tiles = [&](u32 t) { return (u64)((m + t - 1) / t) * ((n + t - 1) / t); };
    p.shape = tiles(256) >= 200 ? kLarge : tiles(128) >= 64 ? kMiddle : kSmall;
    const u32 edge = p.shape == kLarge ? 256 : p.shape == kMiddle ? 128 : 64;
    p.tiles = (u32)tiles(edge);
    p.slices = (k + kSlice - 1) / kSlice;
    u32 splits = p.tiles ? 2 * kUnits / p.tiles : 1;
    splits = std::min(splits, p.slices / 4);
    splits = std::max(splits, (p.slices + kMostSlices - 1) / kMostSlices);
    splits = std::max(splits, 1u);
    p.slices_each = std::max(1u, (p.slices + splits - 1) / splits);
    p.splits = std::max(1u, (p.slices + p.slices_each - 1) / p.slices_each);
    p.part_bytes = p.splits > 1 ? align_up((u64)p.splits * m * align_up(n, 4) * 4, 256) : 0;
    return p;
}

template <class T>
void launch_product(const Scaled &g, const Plan &p, bool whole, hipStream_t stream)
{
    if (whole) k_product<T, true><<<p.tiles * p.splits, T::kThreads, 0, stream>>>(g);
    else k_product<T, false><<<p.tiles * p.splits, T::kThreads, 0, stream>>>(g);
}

int run_product(Scaled g, void *part, hipStream_t stream)
{
    const Plan p = plan_product(g.m, g.n, g.k);
    g.slices_each = p.slices_each;
    g.splits = p.splits;
    g.part = (int *)part;
    const bool whole = (((uintptr_t)g.a | (uintptr_t)g.b | g.lda | g.ldb) & 15u) == 0;
    if (p.shape == kLarge) launch_product<Large>(g, p, whole, stream);
    else if (p.shape == kMiddle) launch_product<Middle>(g, p, whole, stream);
    else launch_product<Small>(g, p, whole, stream);
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
bool type_ok(int type) { return type == RTOPK_F32 || type == RTOPK_BF16 || type == RTOPK_F16; }

int quantize_rows(const void *x, int type, u32 rows, u32 cols, u64 ldx, signed char *q, u64 ldq, u32 fill, float *scale,
                  hipStream_t stream)
{
    const RowsToQuantize g{x, ldx, rows, cols, fill, type, q, ldq, scale};
    if (rows >= 4 * kUnits) k_quantize_rows<1><<<(rows + 3) / 4, kQuantizeThreads, 0, stream>>>(g);
    else k_quantize_rows<4><<<rows, kQuantizeThreads, 0, stream>>>(g);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

u64 column_scratch(u32 rows, u32 cols, bool sums) { return align_up((u64)runs_of(rows) * cols * (sums ? 8 : 4), 256); }

int quantize_columns(const void *x, int type, u32 rows, u32 cols, u64 ldx, signed char *q, u64 ldq, u32 fill, float *scale,
                     float *total, void *scratch, hipStream_t stream)
{
    const u32 runs = runs_of(rows);
    u32 *most = (u32 *)scratch;
    const ColumnsToQuantize g{x, ldx, rows, cols, fill, run_rows(rows), runs, type, q, ldq, scale, most,
                              total ? (float *)(most + (u64)runs * cols) : nullptr, total};
    const u32 groups = (cols + kWave - 1) / kWave;
    k_column_most<<<dim3(groups, runs), kQuantizeThreads, 0, stream>>>(g);
    if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    k_quantize_columns<<<dim3(groups, (fill + kTurnRows - 1) / kTurnRows), kQuantizeThreads, 0, stream>>>(g);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

bool workspace_ok(const void *p, u64 bytes, u64 need) { return need == 0 || (p && ((uintptr_t)p & 255u) == 0 && bytes >= need); }

u64 filled(u32 k) { return align_up(k, kSlice); }

// How the workspaces of the two layer calls are laid out, part after part.
struct Cut {
    unsigned char *base;
    u64 at = 0;
    template <class P> P *take(u64 bytes)
    {
        P *p = (P *)(base + at);
        at += align_up(bytes, 256);
        return p;
    }
};

struct LinearParts {
    signed char *x;
    float *x_scale;
    void *part;
};
u64 cut_linear(void *base, u32 m, u32 k, u32 n, LinearParts &p)
{
    Cut cut{(unsigned char *)base};
    p.x = cut.take<signed char>(m * filled(k));
    p.x_scale = cut.take<float>(4ull * m);
    p.part = cut.take<void>(plan_product(m, n, k).part_bytes);
    return cut.at;
}

struct BackwardParts {
    signed char *dy, *dy_turned, *x_turned;
    float *dy_scale, *dy_turned_scale, *x_turned_scale;
    void *scratch, *part;
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
    p.scratch = cut.take<void>(std::max(column_scratch(m, n, true), column_scratch(m, k, false)));
    p.part = cut.take<void>(std::max(plan_product(m, k, n).part_bytes, plan_product(n, k, m).part_bytes));
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
    return quantize_columns(x, type, (u32)rows, (u32)cols, ldx, q, ldq, (u32)rows, scale, nullptr, workspace, stream);
}

extern "C" int rtopk_matmul_i8_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, uint64_t *bytes)
{
    if (!bytes || m > kMostSize || n > kMostSize || k > kMostSize) return RTOPK_EINVAL;
    *bytes = m && n ? plan_product((u32)m, (u32)n, (u32)k).part_bytes : 0;
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
    LinearParts p;
    cut_linear(workspace, (u32)m, (u32)k, (u32)n, p);
    const u64 ld = filled((u32)k);
    if (const int rc = quantize_rows(x, type, (u32)m, (u32)k, ldx, p.x, ld, (u32)ld, p.x_scale, stream)) return rc;
    return run_product(Scaled{p.x, w, ld, ldw, (u32)m, (u32)n, (u32)k, p.x_scale, w_scale, bias, out, ldo, out_type, 0, 0, nullptr},
                       p.part, stream);
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
    if (const int rc = quantize_columns(dy, type, (u32)m, (u32)n, lddy, p.dy_turned, ld, (u32)ld, p.dy_turned_scale, db, p.scratch,
                                        stream))
        return rc;
    if (const int rc = quantize_columns(x, type, (u32)m, (u32)k, ldx, p.x_turned, ld, (u32)ld, p.x_turned_scale, nullptr, p.scratch,
                                        stream))
        return rc;
    return run_product(Scaled{p.dy_turned, p.x_turned, ld, ld, (u32)n, (u32)k, (u32)m, p.dy_turned_scale, p.x_turned_scale, nullptr,
                              dw, lddw, RTOPK_F32, 0, 0, nullptr},
                       p.part, stream);
}
