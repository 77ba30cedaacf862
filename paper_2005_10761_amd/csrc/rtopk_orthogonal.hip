// Orthogonalised updates (gfx950): the polar factor of a matrix, approached by
// Newton-Schulz products, and the master's weight step that uses it.
//
//   X = G / (|G|_F + eps), turned over where G has more rows than columns
//   each step, with coefficients (a, b, c):
//     A = X X^T,  X <- (a I + b A + c A A) X
//
// as three products around a multiple of the identity that is near A's diagonal
// (h; k is what the polynomial a + b h + c h^2 is there):
//     D = X X^T - h I,  Q = (b + 2 c h) D + c D D,  X <- k X + Q X.
// What is stored rounded, D and Q, is small where A and the polynomial are
// mostly their diagonals: in the first steps, where A is nothing but small
// (h = 0 would do), and in the last ones, where a, b A and c A A cancel (3.4, -4.8
// and 2.0 leave 0.7; h = 1 would do). h is what the diagonal of A becomes if all
// singular values are alike: 1 / m, and from step to step h (a + b h + c h^2)^2. It only
// decides what the roundings are: halves, 256 x 2304, relative error of the result 13 10^-4 with
// h = 0 and the polynomial itself in Q's place, 16 with h = 1, 7.5 so. With pairs, k goes into Q (k X is not read then).
//
// All three products have both operands' rows along the contraction: D's rows
// and Q's are its columns too, and X is kept twice, as it is and turned over
// (the product that makes a new X writes both). D and Q are symmetric: only
// tiles on and above the diagonal are computed, and written on both sides.
//
// Numbers between the products are halves (11 bits; bfloat16, in common use
// here, has 8) or pairs of halves (22 bits), times a power of two that puts
// what the iteration can hold into a half's range: its singular values are
// bounded by the coefficients, which the host checks before it launches. Where they
// are small (the norm is below eps, or the coefficients shrink them), each
// step's X has a power of two of its own, from a bound that follows them.
// Products are summed in binary32. |G|_F is summed in binary64. Of the division by it
// only the power of two is applied to G (that is exact); the rest, between 1 and
// 2 (or less, by eps), goes into the first step's coefficients, so that a
// bfloat16 G enters the products unrounded.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/rtopk.h"
#include "../../include/rtopk_diag.h"
#include "rtopk_direction.h"
#include "rtopk_matrix.h"

namespace rtopk {

// powers of two that X, D and Q are stored with: singular values of X up to kMostX, entries of D up to its square,
// entries of Q up to kMostP (or, less k, its double) stay finite
constexpr int kLogX = 12, kLogD = 10;
constexpr double kMostX = 7.5, kMostP = 30.0;
constexpr int kMostDown = 100;          // X is scaled by no less than 2^-100: quotients of two scales are binary32
struct Members { void *p[kMembers]; };

constexpr u32 kMostSteps = 64;
struct Steps {
    u32 count;
    float abc[kMostSteps][3];
};

// Four lanes with four halves each: lane i gets the i-th of all four.
__device__ __forceinline__ uint2 turned_quad(uint2 d)
{
    const bool upper = (lane_id() & 2u) != 0, odd = (lane_id() & 1u) != 0;
    // two lanes on: the lower two keep halves 0 and 1 of lanes q and q + 2, the upper two 2 and 3
    const u32 got = (u32)__builtin_amdgcn_mov_dpp((int)(upper ? d.x : d.y), 0x4E /* quad_perm 2 3 0 1 */, 0xF, 0xF, true);
    const u32 a = upper ? got : d.x, b = upper ? d.y : got;
    // the neighbour: even lanes keep the low halves
    const u32 give = odd ? (a & 0xFFFFu) | (b << 16) : (a >> 16) | (b & 0xFFFF0000u);
    const u32 r = (u32)__builtin_amdgcn_mov_dpp((int)give, 0xB1 /* quad_perm 1 0 3 2 */, 0xF, 0xF, true);
    return odd ? make_uint2((r & 0xFFFFu) | (a & 0xFFFF0000u), (r >> 16) | (b & 0xFFFF0000u))
               : make_uint2((a & 0xFFFFu) | (r << 16), (b & 0xFFFFu) | (r & 0xFFFF0000u));
}

// ---- stored numbers -------------------------------------------------------
// A row of halves, or of blocks of 128 bytes: 32 high halves, their 32 low halves.
template <Operands kOf> struct Stored {
    static constexpr u32 kBlock = kOf == kPairs ? 32u : 64u;      // numbers in a slice
    static __host__ __device__ u32 row_bytes(u32 cols) { return (cols + kBlock - 1) / kBlock * kSlice; }
    static __host__ __device__ u32 padded(u32 cols) { return (cols + kBlock - 1) / kBlock * kBlock; }
    static __device__ __forceinline__ u32 at(u32 col) { return kOf == kPairs ? (col >> 5) * kSlice + (col & 31u) * 2u : col * 2u; }
    // four neighbours from a multiple of four on
    static __device__ __forceinline__ void put(unsigned char *row, u32 col, const f32x4 &v)
    {
        f16x4 hi;
#pragma unroll
        for (int c = 0; c < 4; ++c) hi[c] = (_Float16)v[c];
        *(f16x4 *)(row + at(col)) = hi;
        if (kOf == kPairs) {
            f16x4 lo;
#pragma unroll
            for (int c = 0; c < 4; ++c) lo[c] = (_Float16)(v[c] - (float)hi[c]);
            *(f16x4 *)(row + at(col) + 64) = lo;
        }
    }
    // kN neighbours (2, 4 or 8) from a multiple of kN on
    template <int kN>
    static __device__ __forceinline__ void put_run(unsigned char *row, u32 col, const float (&v)[kN])
    {
        typedef _Float16 Run __attribute__((ext_vector_type(kN)));
        Run hi;
#pragma unroll
        for (int c = 0; c < kN; ++c) hi[c] = (_Float16)v[c];
        *(Run *)(row + at(col)) = hi;
        if (kOf == kPairs) {
            Run lo;
#pragma unroll
            for (int c = 0; c < kN; ++c) lo[c] = (_Float16)(v[c] - (float)hi[c]);
            *(Run *)(row + at(col) + 64) = lo;
        }
    }
    // Every four lanes 4 q .. 4 q + 3 have a row each (neighbours, from a multiple of four on) and the same four columns:
    // lane 4 q + i stores column i, the four rows side by side, to `column` of the matrix turned over.
    static __device__ __forceinline__ void put_turned(unsigned char *column, u32 row, const f32x4 &v, bool there)
    {
        f16x4 hi, lo;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            hi[c] = (_Float16)v[c];
            lo[c] = (_Float16)(v[c] - (float)hi[c]);
        }
        const uint2 h = turned_quad(__builtin_bit_cast(uint2, hi));
        if (there) *(uint2 *)(column + at(row & ~3u)) = h;
        if (kOf == kPairs) {
            const uint2 l = turned_quad(__builtin_bit_cast(uint2, lo));
            if (there) *(uint2 *)(column + at(row & ~3u) + 64) = l;
        }
    }
    static __device__ __forceinline__ f32x4 get(const unsigned char *row, u32 col)
    {
        const f16x4 hi = *(const f16x4 *)(row + at(col));
        f32x4 v;
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = (float)hi[c];
        if (kOf == kPairs) {
            const f16x4 lo = *(const f16x4 *)(row + at(col) + 64);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] += (float)lo[c];
        }
        return v;
    }
    // eight neighbours from a multiple of eight on
    static __device__ __forceinline__ void get_eight(f32x4 &a, f32x4 &b, const unsigned char *row, u32 col)
    {
        const f16x8 hi = *(const f16x8 *)(row + at(col));
        f16x8 lo{0, 0, 0, 0, 0, 0, 0, 0};
        if (kOf == kPairs) lo = *(const f16x8 *)(row + at(col) + 64);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            a[c] = (float)hi[c] + (float)lo[c];
            b[c] = (float)hi[4 + c] + (float)lo[4 + c];
        }
    }
};

// ---- the norm ---------------------------------------------------------------
constexpr u32 kNormThreads = 256, kNormBlocks = 256;     // workgroups (and parts of the sum) for one matrix, at most

// the sum of the workgroup's values, in every thread
template <int kThreads>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double part[kThreads / kWave];
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if (lane_id() == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) v += part[w];
    return v;
}

// Pieces of eight neighbours of a matrix (from a multiple of eight columns on), four of a thread under way. Bound by the one
// read: four matrices of 6000 x 1500 binary32 37 us, 3.9 TB/s. By itself, since the scale of the first stored numbers needs
// all of it; the weight step makes its sums where it makes the direction.
template <int kType>
__global__ void __launch_bounds__(kNormThreads)
k_norm(Members x, u32 rows, u32 cols, u64 ld, double *__restrict__ part)
{
    constexpr u32 kAtOnce = 4;
    const unsigned char *g = (const unsigned char *)x.p[blockIdx.y];
    const u32 pieces = (cols + 7) / 8;
    const u64 all = (u64)rows * pieces, step = (u64)gridDim.x * kNormThreads;
    const u64 row_bytes = ld * Eight<kType>::kSize;
    double sum = 0.0;
    for (u64 at = (u64)blockIdx.x * kNormThreads + threadIdx.x; at < all; at += kAtOnce * step) {
        Eight<kType> e[kAtOnce];
        const unsigned char *row[kAtOnce];
        u32 c[kAtOnce];
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            const u64 here = min(at + q * step, all - 1u);
            const u32 r = (u32)(here / pieces);
            row[q] = g + r * row_bytes;
            c[q] = (u32)(here - (u64)r * pieces) * 8u;
            e[q].load(row[q], c[q], cols);
        }
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            if (at + q * step >= all) break;
            float v[8];
            e[q].numbers(v, row[q], c[q], cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)v[i] * (double)v[i];
        }
    }
    sum = block_sum<kNormThreads>(sum);
    if (threadIdx.x == 0) part[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
}

// ---- G into stored numbers, as it is and turned over --------------------------
struct Start {
    Members x;
    u32 rows, cols;
    u64 ld;
    unsigned char *as_is, *turned;      // [rows] rows of cols, [cols] rows of rows
    u64 as_is_stride, turned_stride;    // from matrix to matrix
    const double *part;
    u32 parts;
    float eps;
    Steps steps;
    float *scale;                       // of X before each step and after the last, see exponent_of
};

constexpr u32 kSide = 64;               // k_start's and k_join's blocks, and what a narrow matrix is at most

__device__ __forceinline__ float read_lane(float v, u32 lane)
{
    return __uint_as_float((u32)__builtin_amdgcn_readlane((int)__float_as_uint(v), (int)lane));
}

// From the parts of a matrix's norm: the exponent that its elements are moved by, and (where there is a `scale`) what X is its
// stored numbers times, but for 2^-kLogX, before step i: scale[i * kMembers]. Before the first that is what is left of the division; then
// it is 1 unless a bound on the singular values is below a half, which then lie in a half's range as they do elsewhere
// (without it a norm of 10^-4 eps lost 5 of the 22 bits of pairs, one of 10^-8 eps all of them).
// By all kThreads threads of a workgroup.
template <int kThreads>
__device__ __forceinline__ int exponent_of(const double *part, u32 parts, float eps, const Steps &steps, float *scale)
{
    static_assert(kNormBlocks <= kThreads, "a part of the norm for each thread");
    const double norm = sqrt(block_sum<kThreads>(threadIdx.x < parts ? part[threadIdx.x] : 0.0));
    int exponent = 0;
    if (norm > 0.0 && norm < __builtin_huge_val()) (void)frexp(norm, &exponent);
    if (threadIdx.x < kWave && scale) {
        // zeros stay zeros; an infinity or a not-a-number makes all of it NaN
        const bool some = norm > 0.0 && norm < __builtin_huge_val();
        const u32 lane = threadIdx.x;
        if (lane == 0)
            scale[0] = norm == 0.0 ? 0.0f : some ? (float)(ldexp(1.0, exponent) / (norm + (double)eps)) : __uint_as_float(0x7FC00000u);
        // the singular values' bound; lane i has step i's coefficients, and its bound after it
        float a = 0.0f, b = 0.0f, c = 0.0f, most = some ? (float)(norm / (norm + (double)eps)) : 1.0f, mine = most;
        if (lane < steps.count) {
            a = fabsf(steps.abc[lane][0]);
            b = fabsf(steps.abc[lane][1]);
            c = fabsf(steps.abc[lane][2]);
        }
        for (u32 i = 0; i < steps.count; ++i) {
            const float square = most * most;
            most = fminf(most * (read_lane(a, i) + square * (read_lane(b, i) + square * read_lane(c, i))), (float)kMostX);
            if (lane == i) mine = most;
        }
        int e = 0;
        if (mine < 0.5f) (void)frexpf(mine, &e);
        if (lane < steps.count) scale[(lane + 1) * kMembers] = ldexpf(1.0f, max(e, -kMostDown));
    }
    return kLogX - exponent;
}

// Blocks of 64 x 64, turned over in LDS, so that both forms are written in rows. Bound by one read and two writes: four
// matrices of 6000 x 1500 binary32 into pairs, 432 MB, 81 us, 5.3 TB/s (the turned reads from LDS conflict in a third of
// its cycles, which the stores cover).
template <Operands kOf, int kType>
__global__ void __launch_bounds__(kNormThreads) k_start(Start g)
{
    typedef Stored<kOf> S;
    __shared__ float tile[kSide][kSide + 1];
    const u32 r0 = blockIdx.y * kSide, c0 = blockIdx.x * kSide, member = blockIdx.z;
    const int e = exponent_of<kNormThreads>(g.part + member * kNormBlocks, g.parts, g.eps, g.steps,
                                            blockIdx.x == 0 && blockIdx.y == 0 ? g.scale + member : nullptr);
    const u64 row_bytes = g.ld * Eight<kType>::kSize;
    const unsigned char *x = (const unsigned char *)g.x.p[member];
    const u32 row_a = S::row_bytes(g.cols), row_t = S::row_bytes(g.rows);
    unsigned char *as_is = g.as_is + member * g.as_is_stride, *turned = g.turned + member * g.turned_stride;
    // a piece of eight neighbours, the two pieces of a thread 32 rows apart
    const u32 r = threadIdx.x >> 3, c = (threadIdx.x & 7u) * 8u;
    float v[2][8];
    Eight<kType> held[2];
#pragma unroll
    for (u32 h = 0; h < 2; ++h) held[h].load(x + min(r0 + r + 32 * h, g.rows - 1u) * row_bytes, c0 + c, g.cols);
#pragma unroll
    for (u32 h = 0; h < 2; ++h) {
        const u32 row = r0 + r + 32 * h;
        held[h].numbers(v[h], x + min(row, g.rows - 1u) * row_bytes, c0 + c, row < g.rows ? g.cols : 0u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[h][i] = ldexpf(v[h][i], e);
            tile[r + 32 * h][c + i] = v[h][i];
        }
        if (row < g.rows) {
            if (c0 + c < S::padded(g.cols)) S::template put_run<8>(as_is + (u64)row * row_a, c0 + c, v[h]);
        }
    }
    __syncthreads();
#pragma unroll
    for (u32 h = 0; h < 2; ++h) {
        const u32 col = c0 + r + 32 * h, row = r0 + c;
        float u[8];
#pragma unroll
        for (u32 q = 0; q < 8; ++q) u[q] = tile[c + q][r + 32 * h];
        if (col < g.cols && row < S::padded(g.rows)) S::template put_run<8>(turned + (u64)col * row_t, row, u);
    }
}

// ---- the products -------------------------------------------------------------
// kSymmetric: a product of two matrices that commute and are symmetric, or X X^T; kPart: a run of X X^T's contraction, its
// sums in binary32 for k_join; kNext: the new X and its turned form; kLast: the result, with G's orientation.
enum Step { kSymmetric, kPart, kNext, kLast };

struct Product {
    const unsigned char *left, *right;      // rows of the result, columns of the result
    u64 left_stride, right_stride;          // from matrix to matrix
    u32 rows, cols, inner;                  // of the result, and numbers of the contraction
    u32 tiles_m, tiles_n, tiles;            // tiles: of one matrix
    unsigned char *out, *turned;            // the result, and turned over
    u64 out_stride, turned_stride;
    // kSymmetric: result = c_sum scale^2 product + c_old old + c_one I; kNext, kLast: (c_sum product + c_old old) scale / next
    float c_sum, c_old, c_one;
    const unsigned char *old;               // laid out as the result, or null
    const float *scale, *next;              // of the matrices' X before and after, or null for 1
    // kPart
    float *part;                            // [splits][matrices][rows][rows rounded up to 4]
    u32 members, splits, slices_each;
    // kLast
    Members to;
    int type;
    u64 ldo;
    float gain, keep;                       // to <- keep * to + gain * result, where `update`
    int update;
};

// tile `at` of the triangle on and above the diagonal of n x n tiles: row i of them has n - i
__device__ __forceinline__ void triangle_at(u32 at, u32 n, u32 &i, u32 &j)
{
    i = 0;
    while (at >= n - i) at -= n - i++;
    j = i + at;
}

// One tile of one product, its polynomial's terms and both forms of the result from the registers. Bound by the matrix
// units where matrices are large: P X of 4096 x 4096 with pairs 286 us, 481 10^12 operations a second counted once and 1443 as the
// halves that are multiplied (the library's product of halves reaches 1491), with halves 123 us, 1117; of four 1500 x 6000 with
// pairs 282 us, 384 and 1151; D of 512 x 512, three of them, 8.5 us, which
// are a launch, sixteen slices' barriers and a store.
template <Operands kOf, class T, Step kStep>
__global__ void __launch_bounds__(T::kThreads) k_step(Product g)
{
    typedef Stored<kOf> S;
    __shared__ __align__(16) unsigned char lds[T::kLds];
    constexpr bool kTriangle = kStep == kSymmetric || kStep == kPart;
    const u32 place = xcd_place(blockIdx.x, gridDim.x), split = kStep == kPart ? place / (g.tiles * g.members) : 0u;
    const u32 left_over = place - split * g.tiles * g.members, member = left_over / g.tiles, at = left_over - member * g.tiles;
    u32 ti, tj;
    if (kTriangle) triangle_at(at, g.tiles_n, ti, tj);
    else tile_at(at, g.tiles_m, g.tiles_n, ti, tj);
    const u32 i0 = ti * T::kRowsM, j0 = tj * T::kRowsN;
    const u32 bytes = S::row_bytes(g.inner), slices = bytes / kSlice;
    const TileRows a{g.left + member * g.left_stride + (u64)i0 * bytes, g.rows - i0, bytes, bytes};
    const TileRows b{g.right + member * g.right_stride + (u64)j0 * bytes, g.cols - j0, bytes, bytes};
    const u32 row_out = S::row_bytes(g.cols), row_turned = S::row_bytes(g.rows);
    float scale = 1.0f, next = 1.0f;
    T t;
    t.clear();
    const u32 from = kStep == kPart ? split * g.slices_each : 0u;
    t.template multiply<true>(a, b, from, kStep == kPart ? min(from + g.slices_each, slices) : slices, lds, [&] {
        if (kStep == kPart) return;
        if (g.scale) scale = g.scale[member];           // (on its way with the first slices too)
        if (kStep == kNext) next = g.next[member];
        if (!g.old) return;
        // the old matrix's part goes into the sums first: its loads are under way together, and with the first slices (after the
        // products, between the stores, each would be waited for: 95 us for 4096 x 4096, 72 without it; and so they are where a
        // branch stands around each: what lies beyond the matrix is read from its edge, and not stored)
        const unsigned char *old = g.old + member * g.out_stride;
        const float ratio = g.c_old / g.c_sum;
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i) {
            const unsigned char *row = old + (u64)min(i0 + T::row_at(i), g.rows - 1u) * row_out;
            constexpr int kPaired = T::wide_at(0) ? T::kFragsN / 2 * 2 : 0;
#pragma unroll
            for (int j = 0; j < kPaired; j += 2)
                S::get_eight(t.sum[i][j], t.sum[i][T::next_to(j)], row, min(j0 + T::col_at(j), S::padded(g.cols) - 8u));
#pragma unroll
            for (int j = kPaired; j < T::kFragsN; ++j) t.sum[i][j] = S::get(row, min(j0 + T::col_at(j), S::padded(g.cols) - 4u));
        }
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < T::kFragsN; ++j) t.sum[i][j] *= ratio;
    });

    if constexpr (kStep == kPart) {
        const u64 ld = align_up(g.rows, 4);
        float *part = g.part + ((u64)split * g.members + member) * g.rows * ld;
        t.each([&](u32 r, u32 c, const f32x4 &sum) {
            if (i0 + r < g.rows && j0 + c < g.cols) *(f32x4 *)(part + (i0 + r) * ld + j0 + c) = sum;
        });
        return;
    }
    const float c_sum = kTriangle ? g.c_sum * scale * scale : g.c_sum * (scale / next);
    if constexpr (kStep == kLast) {
        void *to = g.to.p[member];
        // the old weights of a row of fragments, on their way while the row before is stored; without a branch, as above
        f32x4 w[2][T::kFragsN];
        auto weights = [&](f32x4 (&to_w)[T::kFragsN], int i) {
            const float *row = (const float *)to + (u64)min(i0 + T::row_at(i), g.rows - 1u) * g.ldo;
            if (g.cols >= 4u) {
#pragma unroll
                for (int j = 0; j < T::kFragsN; ++j) __builtin_memcpy(&to_w[j], row + min(j0 + T::col_at(j), g.cols - 4u), 16);
            }
#pragma unroll
            for (int j = 0; j < T::kFragsN; ++j) {
                const u32 col = j0 + T::col_at(j);
                if (col < g.cols && col + 4u > g.cols)
#pragma unroll
                    for (u32 q = 0; q < 4; ++q) to_w[j][q] = col + q < g.cols ? row[col + q] : 0.0f;
            }
        };
        if (g.update) weights(w[0], 0);
#pragma unroll
        for (int i = 0; i < T::kFragsM; ++i) {
            const u32 row = i0 + T::row_at(i);
            if (g.update && i + 1 < T::kFragsM) weights(w[(i + 1) & 1], i + 1 < T::kFragsM ? i + 1 : i);
            if (row >= g.rows) continue;
            const u64 first = (u64)row * g.ldo;
#pragma unroll
            for (int j = 0; j < T::kFragsN; ++j) {
                t.sum[i][j] *= c_sum;
                if (g.update)
#pragma unroll
                    for (u32 q = 0; q < 4; ++q) t.sum[i][j][q] = fmaf(g.gain, t.sum[i][j][q], g.keep * w[i & 1][j][q]);
            }
#pragma unroll
            for (int j = 0; j < T::kFragsN; j += T::step_at(j)) {
                const u32 col = j0 + T::col_at(j);
                if (col >= g.cols) continue;
                if (T::wide_at(j)) write_eight(to, first + col, g.type, t.sum[i][j], t.sum[i][T::next_to(j)], g.cols - col);
                else write_four(to, first + col, g.type, t.sum[i][j], g.cols - col);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < T::kFragsM; ++i)
#pragma unroll
        for (int j = 0; j < T::kFragsN; ++j) {
            const u32 row = i0 + T::row_at(i), col = j0 + T::col_at(j);
            t.sum[i][j] *= c_sum;
#pragma unroll
            for (u32 q = 0; q < 4; ++q) {
                if (kTriangle && col + q == row) t.sum[i][j][q] += g.c_one;
                if (row >= g.rows || col + q >= g.cols) t.sum[i][j][q] = 0.0f;          // what pads the rows is zero
            }
        }
    unsigned char *out = g.out + member * g.out_stride, *turned = g.turned + member * g.turned_stride;
#pragma unroll
    for (int i = 0; i < T::kFragsM; ++i) {
        const u32 row = i0 + T::row_at(i);
        if (row >= g.rows) continue;
        unsigned char *to = out + (u64)row * row_out;
#pragma unroll
        for (int j = 0; j < T::kFragsN; j += T::step_at(j)) {
            const u32 col = j0 + T::col_at(j);
            if (col >= S::padded(g.cols)) continue;
            const f32x4 &v = t.sum[i][j], &u = t.sum[i][T::next_to(j)];
            if (T::wide_at(j)) S::template put_run<8>(to, col, {v[0], v[1], v[2], v[3], u[0], u[1], u[2], u[3]});
            else S::put(to, col, v);
        }
    }
    if (kTriangle && ti == tj) return;
#pragma unroll
    for (int j = 0; j < T::kFragsN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const u32 col = j0 + T::col_at(j) + e;
            if (col >= g.cols) continue;
            unsigned char *to = turned + (u64)col * row_turned;
            constexpr int kEight = T::kFragsM / 8 * 8, kFour = T::kFragsM / 4 * 4;
            static_assert(T::kFragsM % 4 == 0 || T::kFragsM % 4 == 2, "a rest of two");
#pragma unroll
            for (int i = 0; i + 8 <= kEight; i += 8) {
                const u32 row = i0 + T::row_at(i);
                if (row < S::padded(g.rows))
                    S::template put_run<8>(to, row, {t.sum[i][j][e], t.sum[i + 1][j][e], t.sum[i + 2][j][e], t.sum[i + 3][j][e],
                                                     t.sum[i + 4][j][e], t.sum[i + 5][j][e], t.sum[i + 6][j][e], t.sum[i + 7][j][e]});
            }
#pragma unroll
            for (int i = kEight; i + 4 <= kFour; i += 4) {
                const u32 row = i0 + T::row_at(i);
                if (row < S::padded(g.rows))
                    S::template put_run<4>(to, row, {t.sum[i][j][e], t.sum[i + 1][j][e], t.sum[i + 2][j][e], t.sum[i + 3][j][e]});
            }
            if constexpr (T::kFragsM % 4 == 2) {
                const u32 row = i0 + T::row_at(kFour);
                if (row < S::padded(g.rows)) S::template put_run<2>(to, row, {t.sum[kFour][j][e], t.sum[kFour + 1][j][e]});
            }
        }
}

// The runs of X X^T together, in their order, scaled, less the multiple of the identity: D, both sides of the diagonal, by
// blocks of 64 x 64. Bound by the reads of the parts: four of 1500 x 1500 in three runs (the half of 108 MB) 20 us.
constexpr u32 kJoinThreads = kSide * kSide / 4;

template <Operands kOf>
__global__ void __launch_bounds__(kJoinThreads) k_join(Product g)
{
    typedef Stored<kOf> S;
    __shared__ float tile[kSide][kSide + 1];
    const u32 member = blockIdx.y, n = (g.rows + kSide - 1) / kSide;
    u32 ti, tj;
    triangle_at(blockIdx.x, n, ti, tj);
    const u32 r = threadIdx.x >> 4, c = (threadIdx.x & 15u) * 4u;
    const u64 ld = align_up(g.rows, 4), one = (u64)g.rows * ld;
    const float scale = g.scale[member], c_sum = g.c_sum * scale * scale;
    const u32 row_out = S::row_bytes(g.rows);
    unsigned char *out = g.out + member * g.out_stride;
    {
        const u32 row = ti * kSide + r, col = tj * kSide + c;
        f32x4 v{0, 0, 0, 0};
        if (row < g.rows && col < g.rows) {
            const float *p = g.part + member * one + row * ld + col;
#pragma unroll 8
            for (u32 s = 0; s < g.splits; ++s) v += *(const f32x4 *)(p + s * g.members * one);
        }
        v *= c_sum;
#pragma unroll
        for (u32 q = 0; q < 4; ++q) {
            if (col + q == row) v[q] += g.c_one;
            if (row >= g.rows || col + q >= g.rows) v[q] = 0.0f;
            tile[r][c + q] = v[q];
        }
        if (row < g.rows && col < S::padded(g.rows)) S::put(out + (u64)row * row_out, col, v);
    }
    if (ti == tj) return;
    __syncthreads();
    const u32 row = tj * kSide + r, col = ti * kSide + c;
    if (row < g.rows) S::put(out + (u64)row * row_out, col, f32x4{tile[c][r], tile[c + 1][r], tile[c + 2][r], tile[c + 3][r]});
}

// ---- matrices with a side of up to 64: one launch for a step ---------------------
// X's long side is cut into runs of blocks of 64. A workgroup has a run: it takes the runs' parts of X X^T together (every
// workgroup for itself, in one order: they all have the same D), makes D and P in LDS, the new X of its run block by
// block, and that block's part of the next X X^T while it is in LDS. Only X turned over and the parts go through memory.
// 64 x 576, four of them, five steps: 16 launches of the kernels above take 95 us (each as long as a launch), seven of these
// 44: 7.5 a step, of which three follow one another through LDS with a barrier between.
typedef unsigned char u8;
constexpr int kNarrowThreads = 512;

struct Narrow {
    Members x;                  // k_narrow_start: G
    u32 rows, cols;             // of G
    u64 ld;
    const double *norm;
    u32 norm_parts;
    float eps;
    float *scale;               // k_narrow_start: of all steps, written; k_narrow: of its step and the next
    const u8 *xt;               // [members][n] rows of m, k_narrow: read
    u8 *xt_next;                // written
    u64 xt_stride;
    const float *part;          // [members][runs][64][64], read; or, joined, [members][64][64]
    float *part_next;           // [members][runs][64][64], written
    float *joined;              // [members][64][64], or null
    u32 runs, blocks_each;
    float c_gram, shift, c_sum, c_old, c_one, c_x;      // D = c_gram X X^T - shift; Q = c_sum D D + c_old D + c_one; X <- Q X + c_x X
    bool last;
    Members to;                 // the result
    int to_type;
    u64 ldo;
    float gain, keep, c_last;
    int update;
};

template <Operands kOf> struct Block {      // 64 rows of 64 numbers in LDS, slices as Tile reads them
    typedef Tile<kOf, 64, 64, 2, 4, 2, false> T;
    static constexpr u32 kSlices = kSide / Stored<kOf>::kBlock, kBytes = kSlices * kSide * kSlice;
    static __device__ __forceinline__ u8 *at(u8 *block, u32 row, u32 byte)
    {
        return block + (byte / kSlice) * (kSide * kSlice) + T::place(row, (byte % kSlice) >> 4) + (byte & 15u);
    }
    static __device__ __forceinline__ void put(u8 *block, u32 row, u32 col, const f32x4 &v)
    {
        f16x4 hi, lo;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            hi[c] = (_Float16)v[c];
            lo[c] = (_Float16)(v[c] - (float)hi[c]);
        }
        const u32 byte = Stored<kOf>::at(col);
        *(f16x4 *)at(block, row, byte) = hi;
        if (kOf == kPairs) *(f16x4 *)at(block, row, byte + 64) = lo;
    }
    static __device__ __forceinline__ f32x4 get(u8 *block, u32 row, u32 col)
    {
        const u32 byte = Stored<kOf>::at(col);
        const f16x4 hi = *(const f16x4 *)at(block, row, byte);
        f32x4 v;
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = (float)hi[c];
        if (kOf == kPairs) {
            const f16x4 lo = *(const f16x4 *)at(block, row, byte + 64);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] += (float)lo[c];
        }
        return v;
    }
    static __device__ __forceinline__ void multiply(T &t, const u8 *a, const u8 *b)
    {
#pragma unroll
        for (u32 s = 0; s < kSlices; ++s) t.one_slice(a + s * kSide * kSlice, b + s * kSide * kSlice);
    }
};

// a block's part of X X^T, all of them of one workgroup: in binary32 to memory
template <class T>
__device__ __forceinline__ void write_part(const T &gram, float *to)
{
    gram.each([&](u32 r, u32 c, const f32x4 &sum) { *(f32x4 *)(to + r * kSide + c) = sum; });
}

template <Operands kOf, int kType>
__global__ void __launch_bounds__(kNarrowThreads) k_narrow_start(Narrow g, Steps steps)
{
    typedef Stored<kOf> S;
    typedef Block<kOf> B;
    __shared__ float tile[kSide][kSide + 1];            // [m][n]
    __shared__ __align__(16) u8 rows[B::kBytes];
    const u32 member = blockIdx.y, run = blockIdx.x;
    const bool over = g.rows > g.cols;
    const u32 m = over ? g.cols : g.rows, n = over ? g.rows : g.cols;
    const int e = exponent_of<kNarrowThreads>(g.norm + member * kNormBlocks, g.norm_parts, g.eps, steps,
                                               run == 0 ? g.scale + member : nullptr);
    const u64 row_bytes = g.ld * Eight<kType>::kSize;
    const u8 *x = (const u8 *)g.x.p[member];
    u8 *xt = g.xt_next + member * g.xt_stride;
    typename B::T gram;
    gram.clear();
    for (u32 b = 0; b < g.blocks_each; ++b) {
        const u32 n0 = (run * g.blocks_each + b) * kSide;
        if (n0 >= n) break;
        {   // pieces of eight along G's rows
            const u32 r = threadIdx.x >> 3, c = (threadIdx.x & 7u) * 8u;
            const u32 row = over ? n0 + r : r, col = over ? c : n0 + c;
            float v[8];
            Eight<kType> held;
            held.load(x + min(row, g.rows - 1u) * row_bytes, col, g.cols);
            held.numbers(v, x + min(row, g.rows - 1u) * row_bytes, col, row < g.rows ? g.cols : 0u);
#pragma unroll
            for (int i = 0; i < 8; ++i) (over ? tile[c + i][r] : tile[r][c + i]) = ldexpf(v[i], e);
        }
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < 2; ++h) {
            const u32 r = (threadIdx.x >> 4) + 32 * h, c = (threadIdx.x & 15u) * 4u;
            B::put(rows, r, c, f32x4{tile[r][c], tile[r][c + 1], tile[r][c + 2], tile[r][c + 3]});
            if (n0 + r < n && c < S::padded(m))
                S::put(xt + (u64)(n0 + r) * S::row_bytes(m), c, f32x4{tile[c][r], tile[c + 1][r], tile[c + 2][r], tile[c + 3][r]});
        }
        __syncthreads();
        B::multiply(gram, rows, rows);
    }
    write_part(gram, g.part_next + ((u64)member * g.runs + run) * kSide * kSide);
}

// Many runs' parts together, by themselves (every workgroup of a step reading 27 of them took 10 us of its 25): sixteen
// groups of sixteen threads each add up every sixteenth part of 64 sums, then the groups in order.
__global__ void __launch_bounds__(256) k_narrow_join(Narrow g)
{
    __shared__ f32x4 part[16][16];
    const u32 group = threadIdx.x >> 4, at = blockIdx.x * 16u + (threadIdx.x & 15u), member = blockIdx.y;
    const f32x4 *p = (const f32x4 *)(g.part + (u64)member * g.runs * kSide * kSide) + at;
    f32x4 sum{0, 0, 0, 0};
#pragma unroll 8
    for (u32 s = group; s < g.runs; s += 16) sum += p[s * (kSide * kSide / 4)];
    part[group][threadIdx.x & 15u] = sum;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (u32 s = 1; s < 16; ++s) sum += part[s][threadIdx.x];
    ((f32x4 *)(g.joined + (u64)member * kSide * kSide))[at] = sum;
}

template <Operands kOf>
__global__ void __launch_bounds__(kNarrowThreads) k_narrow(Narrow g)
{
    typedef Stored<kOf> S;
    typedef Block<kOf> B;
    typedef typename B::T T;
    __shared__ __align__(16) u8 lds[3][B::kBytes];      // D, then rows of the new X; P; X turned over
    const u32 member = blockIdx.y, run = blockIdx.x;
    const bool over = g.rows > g.cols;
    const u32 m = over ? g.cols : g.rows, n = over ? g.rows : g.cols;
    const u32 row_xt = S::row_bytes(m), pieces = row_xt / 16;       // 16-byte pieces of a row of X turned over
    const u8 *xt = g.xt + member * g.xt_stride;
    u8 *xt_next = g.xt_next + member * g.xt_stride;
    // a block of X turned over: rows of the long side, 16 bytes a thread and time
    constexpr u32 kPieces = B::kBytes / 16 / kNarrowThreads;
    auto load = [&](i32x4 (&v)[kPieces], u32 n0) {
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 at = threadIdx.x + q * kNarrowThreads, r = at / (B::kSlices * 8u), piece = at % (B::kSlices * 8u);
            v[q] = i32x4{0, 0, 0, 0};
            if (n0 + r < n && piece < pieces) v[q] = *(const i32x4 *)(xt + (u64)(n0 + r) * row_xt + piece * 16u);
        }
    };
    const u32 first_block = run * g.blocks_each;
    i32x4 held[kPieces];
    load(held, first_block * kSide);
    // (vector loads, on their way with the parts: scalar ones are waited for with the next kernel argument, 0.5 us a launch)
    u32 at_scale = member;
    asm("" : "+v"(at_scale));
    const float x_scale = g.scale[at_scale], x_next = g.scale[kMembers + at_scale];
    {
        // D
        const u32 r = threadIdx.x >> 3, c = (threadIdx.x & 7u) * 8u;
        const u32 runs = g.joined ? 1u : g.runs;
        const float *part = (g.joined ? g.joined : g.part) + (u64)member * runs * kSide * kSide + r * kSide + c;
        f32x4 sum[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll 8
        for (u32 s = 0; s < runs; ++s)
#pragma unroll
            for (int q = 0; q < 2; ++q) sum[q] += *(const f32x4 *)(part + s * kSide * kSide + 4 * q);
        const float scale = g.c_gram * x_scale * x_scale;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            f32x4 v = sum[q] * scale;
#pragma unroll
            for (u32 i = 0; i < 4; ++i)
                if (c + 4 * q + i == r && r < m) v[i] -= g.shift;
            B::put(lds[0], r, c + 4 * q, v);
        }
    }
    __syncthreads();
    {
        // P
        T t;
        t.clear();
        B::multiply(t, lds[0], lds[0]);
        t.each([&](u32 r, u32 c, const f32x4 &sum) {
            f32x4 v = g.c_sum * sum + g.c_old * B::get(lds[0], r, c);
#pragma unroll
            for (u32 i = 0; i < 4; ++i)
                if (c + i == r && r < m) v[i] += g.c_one;
            B::put(lds[1], r, c, v);
        });
    }
    T gram;
    gram.clear();
    for (u32 b = 0; b < g.blocks_each; ++b) {
        const u32 n0 = (first_block + b) * kSide;
        if (n0 >= n) break;
#pragma unroll
        for (u32 q = 0; q < kPieces; ++q) {
            const u32 at = threadIdx.x + q * kNarrowThreads, r = at / (B::kSlices * 8u), piece = at % (B::kSlices * 8u);
            *(i32x4 *)B::at(lds[2], r, piece * 16u) = held[q];
        }
        __syncthreads();                // (and P, and everybody has read D and the last block's rows)
        if (b + 1 < g.blocks_each) load(held, n0 + kSide);
        T t;
        t.clear();
        if (kOf == kHalves) {           // (the part of X itself: X turned over holds it)
#pragma unroll
            for (int i = 0; i < T::kFragsM; ++i)
#pragma unroll
                for (int j = 0; j < T::kFragsN; ++j)
#pragma unroll
                    for (u32 q = 0; q < 4; ++q)
                        t.sum[i][j][q] = g.c_x * (float)*(const _Float16 *)B::at(lds[2], T::col_at(j) + q, S::at(T::row_at(i)));
        }
        B::multiply(t, lds[1], lds[2]);
        if (g.last) {
            void *to = g.to.p[member];
            t.each([&](u32 r, u32 c, const f32x4 &sum) {
                if (r >= m || n0 + c >= n) return;
                f32x4 v = sum * (g.c_last * x_scale);
                const u32 have = n - n0 - c;
                const u64 at = over ? (u64)(n0 + c) * g.ldo + r : (u64)r * g.ldo + n0 + c, next = over ? g.ldo : 1u;
                if (g.update) {
                    const float *w = (const float *)to;
#pragma unroll
                    for (u32 q = 0; q < 4; ++q)
                        if (q < have) v[q] = fmaf(g.gain, v[q], g.keep * w[at + q * next]);
                }
                if (!over) write_four(to, at, g.to_type, v, have);
                else
#pragma unroll
                    for (u32 q = 0; q < 4; ++q)
                        if (q < have) write_as(to, at + q * next, g.to_type, v[q]);
            });
        } else {
            const float c = ldexpf(x_scale / x_next, -kLogD);
            t.each([&](u32 r, u32 col, const f32x4 &sum) {
                f32x4 v = sum * c;
#pragma unroll
                for (u32 q = 0; q < 4; ++q)
                    if (r >= m || n0 + col + q >= n) v[q] = 0.0f;
                B::put(lds[0], r, col, v);
                const u32 column = n0 + col + (lane_id() & 3u);
                S::put_turned(xt_next + (u64)column * row_xt, r, v, column < n && (r & ~3u) < S::padded(m));
            });
            __syncthreads();
            B::multiply(gram, lds[0], lds[0]);
        }
        __syncthreads();
    }
    if (!g.last) write_part(gram, g.part_next + ((u64)member * g.runs + run) * kSide * kSide);
}

}  // namespace rtopk

using namespace rtopk;

namespace {

constexpr u64 kMostSide = 1u << 21;      // offsets inside a tile of 256 rows fit 32 bits
struct Shape {
    u32 rows, cols;
    u32 m() const { return std::min(rows, cols); }
    u32 n() const { return std::max(rows, cols); }
    bool over() const { return rows > cols; }       // X is G turned over
};

// How X X^T is made: tiles of `edge`, the contraction in so many runs.
struct GramPlan {
    u32 edge, splits, slices_each;
};

template <Operands kOf>
u32 best_edge(bool triangle, u32 rows, u32 cols, u32 members, double slices, double *cost)
{
    u32 best = 0;
    for (const u32 edge : {64u, 128u, 192u, 256u}) {
        const u64 i = (rows + edge - 1) / edge, j = (cols + edge - 1) / edge;
        const double c = tiles_cost(kOf == kPairs ? kCostPairs : kCostHalves, edge, (triangle ? j * (j + 1) / 2 : i * j) * members, slices);
        if (best && c >= *cost) continue;
        best = edge;
        *cost = c;
    }
    return best;
}

// Runs cost a launch, and their sums, four bytes each, written and read.
template <Operands kOf>
GramPlan plan_gram(u32 members, const Shape &s, double *cost)
{
    const u32 m = s.m(), slices = Stored<kOf>::row_bytes(s.n()) / kSlice;
    GramPlan best{0, 1, slices};
    best.edge = best_edge<kOf>(true, m, m, members, slices, cost);
    for (u32 splits = 2; splits <= std::min(16u, slices / 4); ++splits) {
        const u32 each = (slices + splits - 1) / splits;
        if ((slices + each - 1) / each != splits) continue;
        double c = 0.0;
        const u32 edge = best_edge<kOf>(true, m, m, members * splits, each, &c);
        c += 5.0 + 4.0 * m * m * members * (splits + 1) / 4e6;
        if (c >= *cost) continue;
        *cost = c;
        best = GramPlan{edge, splits, each};
    }
    return best;
}

// What a step of matrices with both sides beyond 64 is made of.
struct StepPlan {
    GramPlan gram;
    u32 square_edge, next_edge;
    // Two steps at a time: from D and P of the first, X X^T of the second is P (D + h I) P without X, and both polynomials
    // go to X as one. Three more products of m x m, X X^T and P X once less: where X is long. With pairs only, and not with
    // coefficients that make P large: the second D takes up the first one's roundings, up to P^2 times larger (1500 x 6000:
    // relative error 2.2 10^-6, one step at a time 1.2, a plain binary32 iteration 2.1; with h = 1 it would be 24).
    bool twos;
};
template <Operands kOf>
StepPlan plan_step(u32 members, const Shape &s, double largest_p)
{
    StepPlan p{};
    double gram_cost, square_cost, next_cost;
    const double square_slices = Stored<kOf>::row_bytes(s.m()) / kSlice;
    p.gram = plan_gram<kOf>(members, s, &gram_cost);
    p.square_edge = best_edge<kOf>(true, s.m(), s.m(), members, square_slices, &square_cost);
    p.next_edge = best_edge<kOf>(false, s.m(), s.n(), members, square_slices, &next_cost);
    p.twos = kOf == kPairs && largest_p <= 4.0 && gram_cost + next_cost > 1.05 * 3.0 * square_cost;
    return p;
}

// A side of up to 64: the long side's blocks of 64 in so many runs. Up to kFewRuns of them are added up by every workgroup of
// the next step; beyond, a launch does it, and there are as many runs as fill the chip. us a call of five steps, one matrix of
// 64 x 320 / 1024 / 2048 / 5056 / 10048: every workgroup for itself 39 / 47 / 58 / 100 / 153, a launch 48 / 49 / 49 / 54 / 57.
constexpr u32 kFewRuns = 16;
struct NarrowPlan {
    u32 runs, blocks_each;
    bool join;
};
NarrowPlan plan_narrow(const Shape &s, u32 members)
{
    const u32 blocks = (s.n() + kSide - 1) / kSide;
    const u32 most = std::max(kFewRuns, 2 * kUnits / members);
    const u32 each = (blocks + most - 1) / most;
    const u32 runs = (blocks + each - 1) / each;
    return NarrowPlan{runs, each, runs > kFewRuns};
}
bool is_narrow(const Shape &s) { return s.m() <= kSide; }

struct Parts {
    double *norm;
    float *scale, *direction, *part, *joined;
    unsigned char *x[2], *xt[2], *square[4];
    u64 x_stride, xt_stride, square_stride;
};

template <Operands kOf>
u64 cut(void *base, u32 count, const Shape &s, bool direction, Parts &p)
{
    typedef Stored<kOf> S;
    const u32 members = std::min(count, kMembers);
    Cut cut{(unsigned char *)base};
    p.x_stride = align_up((u64)s.m() * S::row_bytes(s.n()), 256);
    p.xt_stride = align_up((u64)s.n() * S::row_bytes(s.m()), 256);
    p.square_stride = align_up((u64)s.m() * S::row_bytes(s.m()), 256);
    p.norm = cut.take<double>(kMembers * kNormBlocks * sizeof(double));
    p.scale = cut.take<float>((kMostSteps + 1) * kMembers * sizeof(float));
    if (is_narrow(s)) {
        for (int i = 0; i < 2; ++i) p.xt[i] = cut.take<unsigned char>(members * p.xt_stride);
        // (fewer matrices have more runs each, but not more in all than 2 * kUnits and what rounding up adds)
        const u64 runs = std::max((u64)members * plan_narrow(s, members).runs,
                                  count > kMembers && count % kMembers ? (u64)(count % kMembers) * plan_narrow(s, count % kMembers).runs : 0);
        p.part = cut.take<float>(2 * runs * kSide * kSide * sizeof(float));
        p.joined = cut.take<float>((u64)members * kSide * kSide * sizeof(float));
        p.direction = direction ? cut.take<float>(members * align_up((u64)s.rows * s.cols, 64) * sizeof(float)) : nullptr;
        return cut.at;
    }
    for (int i = 0; i < 2; ++i) {
        p.x[i] = cut.take<unsigned char>(members * p.x_stride);
        p.xt[i] = cut.take<unsigned char>(members * p.xt_stride);
    }
    for (int i = 0; i < 4; ++i) p.square[i] = cut.take<unsigned char>(members * p.square_stride);
    auto sums = [&](u32 matrices) {
        double cost;
        const u32 splits = matrices ? plan_gram<kOf>(matrices, s, &cost).splits : 1;
        return splits > 1 ? (u64)splits * matrices * s.m() * align_up(s.m(), 4) : 0;
    };
    // (the last launches may have fewer matrices, and more runs)
    const u64 part = std::max(sums(members), sums(count > kMembers ? count % kMembers : 0));
    p.part = cut.take<float>(part * sizeof(float));
    p.direction = direction ? cut.take<float>(members * align_up((u64)s.rows * s.cols, 64) * sizeof(float)) : nullptr;
    return cut.at;
}

u64 cut(int products, void *base, u32 count, const Shape &s, bool direction, Parts &p)
{
    return products == RTOPK_PRODUCTS_PAIRS ? cut<kPairs>(base, count, s, direction, p) : cut<kHalves>(base, count, s, direction, p);
}

// Whether iterates that start with singular values in [0, 1] stay where their stored forms are finite. largest: of
// |a + b s^2 + c s^4| in any step.
bool coefficients_ok(const float *abc, u32 steps, double *largest)
{
    *largest = 0.0;
    double hi = 1.0;
    for (u32 s = 0; s < steps; ++s) {
        const double a = abc[3 * s], b = abc[3 * s + 1], c = abc[3 * s + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        // largest |a t + b t^3 + c t^5| and |a + b u + c u^2|, u = t^2, for t up to hi: at the ends or where the derivatives vanish
        double x = 0.0, p = std::fabs(a);
        auto look = [&](double u) {
            if (!(u > 0.0) || u > hi * hi) return;
            x = std::max(x, std::fabs(std::sqrt(u) * (a + u * (b + u * c))));
            p = std::max(p, std::fabs(a + u * (b + u * c)));
        };
        look(hi * hi);
        if (c != 0.0) {
            look(-b / (2.0 * c));
            const double root = 9.0 * b * b - 20.0 * a * c;
            if (root >= 0.0) {
                look((-3.0 * b + std::sqrt(root)) / (10.0 * c));
                look((-3.0 * b - std::sqrt(root)) / (10.0 * c));
            }
        } else if (b != 0.0) {
            look(-a / (3.0 * b));
        }
        if (!(x <= kMostX) || !(p <= kMostP)) return false;
        *largest = std::max(*largest, p);
        hi = x;
    }
    return true;
}

template <Operands kOf, class T, Step kStep>
int launch(Product g, u32 members, hipStream_t stream)
{
    constexpr bool kTriangle = kStep == kSymmetric || kStep == kPart;
    g.tiles_m = (g.rows + T::kRowsM - 1) / T::kRowsM;
    g.tiles_n = (g.cols + T::kRowsN - 1) / T::kRowsN;
    g.tiles = kTriangle ? g.tiles_n * (g.tiles_n + 1) / 2 : g.tiles_m * g.tiles_n;
    g.members = members;
    k_step<kOf, T, kStep><<<g.tiles * members * (kStep == kPart ? g.splits : 1u), T::kThreads, 0, stream>>>(g);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

template <Operands kOf, Step kStep>
int launch(const Product &g, u32 members, u32 edge, hipStream_t stream)
{
    // eight columns a lane where halves are stored; four where binary32 is (a fragment's 64 bytes of a row)
    constexpr Deal kDeal = kStep == kPart || (kStep == kLast && kOf == kPairs) ? kRuns : kWide;
    if (edge == 256) return launch<kOf, Tile<kOf, 256, 256, 2, 4, 2, kOf != kPairs, kDeal>, kStep>(g, members, stream);
    if (edge == 192) return launch<kOf, Tile<kOf, 192, 192, 2, 4, 3, true, kDeal>, kStep>(g, members, stream);
    if (edge == 128) return launch<kOf, Tile<kOf, 128, 128, 2, 4, 2, true, kDeal>, kStep>(g, members, stream);
    return launch<kOf, Tile<kOf, 64, 64, 2, 4, 3, true, kDeal>, kStep>(g, members, stream);
}

struct Target {
    Members to;
    int type;
    u64 ld;
    float gain, keep;
    int update;
};

// A step's polynomial a + b x + c x^2 around h, and h for the next step.
struct Around {
    double c, slope, value, next;
    Around(const float *k, double h) : c(k[2]), slope(k[1] + 2.0 * k[2] * h), value(k[0] + h * (k[1] + h * k[2])), next(h * value * value) {}
};

template <Operands kOf>
int iterate_narrow(const Members &x, int type, u64 ldx, const Shape &s, u32 members, u32 norm_parts, const Steps &steps, float eps,
                   const Parts &p, const Target &target, hipStream_t stream)
{
    const NarrowPlan plan = plan_narrow(s, members);
    const dim3 grid(plan.runs, members);
    float *part[2] = {p.part, p.part + (u64)members * plan.runs * kSide * kSide};
    Narrow g{};
    g.x = x;
    g.rows = s.rows;
    g.cols = s.cols;
    g.ld = ldx;
    g.norm = p.norm;
    g.norm_parts = norm_parts;
    g.eps = eps;
    g.scale = p.scale;
    g.xt_stride = p.xt_stride;
    g.runs = plan.runs;
    g.blocks_each = plan.blocks_each;
    g.xt_next = p.xt[0];
    g.part_next = part[0];
    g.joined = plan.join ? p.joined : nullptr;
    g.c_gram = ldexpf(1.0f, kLogD - 2 * kLogX);
    g.c_last = ldexpf(1.0f, -kLogD - kLogX);
    g.to = target.to;
    g.to_type = target.type;
    g.ldo = target.ld;
    g.gain = target.gain;
    g.keep = target.keep;
    g.update = target.update;
    if (type == RTOPK_F32) k_narrow_start<kOf, RTOPK_F32><<<grid, kNarrowThreads, 0, stream>>>(g, steps);
    else if (type == RTOPK_BF16) k_narrow_start<kOf, RTOPK_BF16><<<grid, kNarrowThreads, 0, stream>>>(g, steps);
    else k_narrow_start<kOf, RTOPK_F16><<<grid, kNarrowThreads, 0, stream>>>(g, steps);
    if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    double h = 1.0 / s.m();
    for (u32 i = 0; i < steps.count; ++i) {
        const Around at(steps.abc[i], h);
        g.scale = p.scale + i * kMembers;
        g.xt = p.xt[i & 1];
        g.xt_next = p.xt[1 - (i & 1)];
        g.part = part[i & 1];
        g.part_next = part[1 - (i & 1)];
        g.shift = (float)(h * ldexp(1.0, kLogD));
        g.c_sum = (float)(at.c * ldexp(1.0, -kLogD));
        g.c_old = (float)at.slope;
        g.c_one = kOf == kPairs ? (float)(at.value * ldexp(1.0, kLogD)) : 0.0f;
        g.c_x = kOf == kPairs ? 0.0f : (float)(at.value * ldexp(1.0, kLogD));
        h = at.next;
        g.last = i + 1 == steps.count;
        if (plan.join) {
            k_narrow_join<<<dim3(kSide * kSide / 64, members), 256, 0, stream>>>(g);
            if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
        }
        k_narrow<kOf><<<grid, kNarrowThreads, 0, stream>>>(g);
        if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    }
    return RTOPK_OK;
}

// From G and the parts of its norm to the end.
template <Operands kOf>
int iterate(const Members &x, int type, u64 ldx, const Shape &s, u32 members, u32 norm_parts, const Steps &steps,
            double largest_p, float eps, const Parts &p, const Target &target, hipStream_t stream)
{
    typedef Stored<kOf> S;
    if (is_narrow(s)) return iterate_narrow<kOf>(x, type, ldx, s, members, norm_parts, steps, eps, p, target, stream);
    const u32 m = s.m(), n = s.n();
    const Start start{x, s.rows, s.cols, ldx, s.over() ? p.xt[0] : p.x[0], s.over() ? p.x[0] : p.xt[0],
                      s.over() ? p.xt_stride : p.x_stride, s.over() ? p.x_stride : p.xt_stride, p.norm, norm_parts, eps, steps, p.scale};
    const dim3 grid((S::padded(s.cols) + kSide - 1) / kSide, (S::padded(s.rows) + kSide - 1) / kSide, members);
    if (type == RTOPK_F32) k_start<kOf, RTOPK_F32><<<grid, kNormThreads, 0, stream>>>(start);
    else if (type == RTOPK_BF16) k_start<kOf, RTOPK_BF16><<<grid, kNormThreads, 0, stream>>>(start);
    else k_start<kOf, RTOPK_F16><<<grid, kNormThreads, 0, stream>>>(start);
    if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
    const StepPlan plan = plan_step<kOf>(members, s, largest_p);
    const GramPlan &gram = plan.gram;

    // X X^T - h I
    auto make_gram = [&](const unsigned char *x_now, unsigned char *to, double h, const float *scale) -> int {
        Product g{};
        g.left = g.right = x_now;
        g.left_stride = g.right_stride = p.x_stride;
        g.rows = g.cols = m;
        g.inner = n;
        g.out = g.turned = to;
        g.out_stride = g.turned_stride = p.square_stride;
        g.c_sum = ldexpf(1.0f, kLogD - 2 * kLogX);
        g.c_one = (float)(-h * ldexp(1.0, kLogD));
        g.scale = scale;
        if (gram.splits == 1) return launch<kOf, kSymmetric>(g, members, gram.edge, stream);
        g.part = p.part;
        g.splits = gram.splits;
        g.slices_each = gram.slices_each;
        if (const int rc = launch<kOf, kPart>(g, members, gram.edge, stream)) return rc;
        g.members = members;
        const u32 side = (m + kSide - 1) / kSide;
        k_join<kOf><<<dim3(side * (side + 1) / 2, members), kJoinThreads, 0, stream>>>(g);
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
    };
    // to = c left right + d old + e I, of matrices that commute and are symmetric
    auto make_square = [&](const unsigned char *left, const unsigned char *right, const unsigned char *old, unsigned char *to, double c,
                           double d, double e) -> int {
        Product g{};
        g.left = left;
        g.right = right;
        g.left_stride = g.right_stride = p.square_stride;
        g.rows = g.cols = g.inner = m;
        g.out = g.turned = to;
        g.out_stride = g.turned_stride = p.square_stride;
        // (d old is divided by c to go into the sums: a c of zero is made so small that it adds nothing)
        if (std::fabs(c) < ldexp(std::fabs(d), -40)) c = ldexp(std::fabs(d), -40);
        g.c_sum = (float)(c * ldexp(1.0, -kLogD));
        g.c_old = (float)d;
        g.c_one = (float)(e * ldexp(1.0, kLogD));
        g.old = d != 0.0 ? old : nullptr;
        return launch<kOf, kSymmetric>(g, members, plan.square_edge, stream);
    };
    unsigned char *const *q = p.square;
    // Q from D; with pairs the whole polynomial
    auto make_poly = [&](const unsigned char *d, unsigned char *to, const Around &at) -> int {
        return make_square(d, d, d, to, at.c, at.slope, kOf == kPairs ? at.value : 0.0);
    };
    u32 now = 0;
    double h = 1.0 / m;
    for (u32 i = 0; i < steps.count;) {
        const unsigned char *x_now = p.x[now], *xt_now = p.xt[now];
        const float *scale = p.scale + i * kMembers;
        const Around at(steps.abc[i], h);
        if (const int rc = make_gram(x_now, q[0], h, scale)) return rc;
        if (const int rc = make_poly(q[0], q[1], at)) return rc;
        unsigned char *poly = q[1];
        u32 did = 1;
        if (plan.twos && i + 1 < steps.count) {
            const Around second(steps.abc[i + 1], at.next);
            if (const int rc = make_square(q[1], q[1], nullptr, q[2], 1.0, 0.0, 0.0)) return rc;            // E = P P
            if (const int rc = make_square(q[0], q[2], q[2], q[3], 1.0, h, -at.next)) return rc;            // D E + h E - h' I
            if (const int rc = make_poly(q[3], q[0], second)) return rc;
            if (const int rc = make_square(q[0], q[1], nullptr, q[2], 1.0, 0.0, 0.0)) return rc;            // both polynomials
            poly = q[2];
            did = 2;
            h = second.next;
        } else {
            h = at.next;
        }
        i += did;
        Product g{};
        g.scale = scale;
        if (i < steps.count) {
            g.next = p.scale + i * kMembers;
            g.left = poly;
            g.left_stride = p.square_stride;
            g.right = xt_now;
            g.right_stride = p.xt_stride;
            g.rows = g.inner = m;
            g.cols = n;
            now = 1 - now;
            g.out = p.x[now];
            g.turned = p.xt[now];
            g.out_stride = p.x_stride;
            g.turned_stride = p.xt_stride;
            g.c_sum = ldexpf(1.0f, -kLogD);
            if (kOf == kHalves) {
                g.old = x_now;
                g.c_old = (float)at.value;
            }
            if (const int rc = launch<kOf, kNext>(g, members, plan.next_edge, stream)) return rc;
            continue;
        }
        // the last product writes with G's orientation
        g.left = s.over() ? xt_now : poly;
        g.right = s.over() ? poly : xt_now;
        g.left_stride = s.over() ? p.xt_stride : p.square_stride;
        g.right_stride = s.over() ? p.square_stride : p.xt_stride;
        g.rows = s.rows;
        g.cols = s.cols;
        g.inner = m;
        g.c_sum = ldexpf(1.0f, -kLogD - kLogX);
        if (kOf == kHalves) {
            g.old = s.over() ? xt_now : x_now;
            g.out_stride = s.over() ? p.xt_stride : p.x_stride;
            g.c_old = (float)(at.value * ldexp(1.0, -kLogX));
        }
        g.to = target.to;
        g.type = target.type;
        g.ldo = target.ld;
        g.gain = target.gain;
        g.keep = target.keep;
        g.update = target.update;
        if (const int rc = launch<kOf, kLast>(g, members, plan.next_edge, stream)) return rc;
    }
    return RTOPK_OK;
}

int iterate(int products, const Members &x, int type, u64 ldx, const Shape &s, u32 members, u32 norm_parts, const Steps &steps,
            double largest_p, float eps, const Parts &p, const Target &target, hipStream_t stream)
{
    return products == RTOPK_PRODUCTS_PAIRS
               ? iterate<kPairs>(x, type, ldx, s, members, norm_parts, steps, largest_p, eps, p, target, stream)
               : iterate<kHalves>(x, type, ldx, s, members, norm_parts, steps, largest_p, eps, p, target, stream);
}

// workgroups for the norm of one of so many matrices: a few elements for every thread, and not many more than fill the chip
u32 norm_blocks(u64 d, u32 members)
{
    const u64 most = std::max<u64>(1, 8 * kUnits / members), enough = (d + 8 * kNormThreads - 1) / (8 * kNormThreads);
    return (u32)std::min<u64>(std::min(most, enough), kNormBlocks);
}

bool sizes_ok(uint32_t count, uint64_t rows, uint64_t cols, int products)
{
    return count >= 1 && rows >= 1 && cols >= 1 && rows <= kMostSide && cols <= kMostSide && rows * cols <= 0xFFFFFFFFull &&
           (products == RTOPK_PRODUCTS_PAIRS || products == RTOPK_PRODUCTS_HALVES);
}
Steps steps_of(uint32_t count, const float *abc)
{
    Steps s{count, {}};
    std::memcpy(s.abc, abc, count * sizeof s.abc[0]);
    return s;
}
bool iteration_ok(uint32_t steps, const float *abc, float eps, double *largest_p)
{
    return steps >= 1 && steps <= kMostSteps && abc && eps >= 0.0f && std::isfinite(eps) && coefficients_ok(abc, steps, largest_p);
}

}  // namespace

extern "C" int rtopk_orthogonalize_workspace_bytes(uint32_t count, uint64_t rows, uint64_t cols, int products, uint64_t *bytes)
{
    if (!bytes || !sizes_ok(count, rows, cols, products)) return RTOPK_EINVAL;
    Parts p;
    *bytes = cut(products, nullptr, count, Shape{(u32)rows, (u32)cols}, false, p);
    return RTOPK_OK;
}

extern "C" int rtopk_orthogonalize_plan(uint32_t count, uint64_t rows, uint64_t cols, int products, uint32_t steps,
                                        const float *coefficients, rtopk_orthogonalize_plan_t *plan)
{
    double largest_p = 0.0;
    if (!plan || count > kMembers || !sizes_ok(count, rows, cols, products) || !iteration_ok(steps, coefficients, 0.0f, &largest_p))
        return RTOPK_EINVAL;
    const Shape s{(u32)rows, (u32)cols};
    *plan = rtopk_orthogonalize_plan_t{};
    if (is_narrow(s)) {
        const NarrowPlan p = plan_narrow(s, count);
        plan->narrow = 1;
        plan->gram_runs = p.runs;
        plan->joined = p.join;
        return RTOPK_OK;
    }
    const StepPlan p = products == RTOPK_PRODUCTS_PAIRS ? plan_step<kPairs>(count, s, largest_p) : plan_step<kHalves>(count, s, largest_p);
    plan->gram_edge = p.gram.edge;
    plan->gram_runs = p.gram.splits;
    plan->joined = p.gram.splits > 1;
    plan->square_edge = p.square_edge;
    plan->next_edge = p.next_edge;
    plan->two_at_a_time = p.twos;
    return RTOPK_OK;
}

extern "C" int rtopk_orthogonalize(uint32_t count, const void *const *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx,
                                   uint32_t steps, const float *coefficients, float eps, int products, void *const *out, int out_type,
                                   uint64_t ldo, void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    double largest_p = 0.0;
    if (!x || !out || !type_ok(type) || !type_ok(out_type) ||
        rtopk_orthogonalize_workspace_bytes(count, rows, cols, products, &need) != RTOPK_OK)
        return RTOPK_EINVAL;
    if (ldx < cols || ldo < cols || !iteration_ok(steps, coefficients, eps, &largest_p)) return RTOPK_EINVAL;
    for (uint32_t i = 0; i < count; ++i)
        if (!x[i] || !out[i]) return RTOPK_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    const Shape s{(u32)rows, (u32)cols};
    const Steps all = steps_of(steps, coefficients);
    Parts p;
    cut(products, workspace, count, s, false, p);
    for (uint32_t first = 0; first < count; first += kMembers) {
        const u32 members = std::min(count - first, kMembers);
        Members from{};
        Target to{Members{}, out_type, ldo, 0.0f, 0.0f, 0};
        for (u32 i = 0; i < members; ++i) {
            from.p[i] = const_cast<void *>(x[first + i]);
            to.to.p[i] = out[first + i];
        }
        const u32 parts = norm_blocks((u64)s.rows * s.cols, members);
        const dim3 grid(parts, members);
        if (type == RTOPK_F32) k_norm<RTOPK_F32><<<grid, kNormThreads, 0, stream>>>(from, s.rows, s.cols, ldx, p.norm);
        else if (type == RTOPK_BF16) k_norm<RTOPK_BF16><<<grid, kNormThreads, 0, stream>>>(from, s.rows, s.cols, ldx, p.norm);
        else k_norm<RTOPK_F16><<<grid, kNormThreads, 0, stream>>>(from, s.rows, s.cols, ldx, p.norm);
        if (hipGetLastError() != hipSuccess) return RTOPK_EHIP;
        if (const int rc = iterate(products, from, type, ldx, s, members, parts, all, largest_p, eps, p, to, stream)) return rc;
    }
    return RTOPK_OK;
}

extern "C" int rtopk_aggregate_update_orthogonal_workspace_bytes(uint32_t count, uint64_t rows, uint64_t cols, int products,
                                                                 uint64_t *bytes)
{
    if (!bytes || !sizes_ok(count, rows, cols, products)) return RTOPK_EINVAL;
    Parts p;
    *bytes = cut(products, nullptr, count, Shape{(u32)rows, (u32)cols}, true, p);
    return RTOPK_OK;
}

extern "C" int rtopk_aggregate_update_orthogonal(uint32_t count, const uint32_t *const *idx, const float *const *val, uint32_t n,
                                                 uint64_t k, uint64_t rows, uint64_t cols, float eta, float scale, float mu,
                                                 int nesterov, float decay, float gain, uint32_t steps, const float *coefficients,
                                                 float eps, int products, float *const *omega, float *const *velocity,
                                                 void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    double largest_p = 0.0;
    if (!idx || !val || !omega || !velocity || n < 1 || k < 1 ||
        rtopk_aggregate_update_orthogonal_workspace_bytes(count, rows, cols, products, &need) != RTOPK_OK)
        return RTOPK_EINVAL;
    if (!iteration_ok(steps, coefficients, eps, &largest_p)) return RTOPK_EINVAL;
    const u64 d = rows * cols;
    for (uint32_t i = 0; i < count; ++i) {
        if (!idx[i] || !val[i] || !omega[i] || !velocity[i]) return RTOPK_EINVAL;
        const uintptr_t w0 = (uintptr_t)omega[i], v0 = (uintptr_t)velocity[i];
        if (w0 < v0 + d * 4 && v0 < w0 + d * 4) return RTOPK_EINVAL;
    }
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    const Shape s{(u32)rows, (u32)cols};
    const Steps all = steps_of(steps, coefficients);
    Parts p;
    cut(products, workspace, count, s, true, p);
    for (uint32_t first = 0; first < count; first += kMembers) {
        const u32 members = std::min(count - first, kMembers);
        Members directions{};
        DirectionMembers from{};
        Target to{Members{}, RTOPK_F32, cols, -(eta * gain), 1.0f - eta * decay, 1};
        for (u32 i = 0; i < members; ++i) {
            from.idx[i] = idx[first + i];
            from.val[i] = val[first + i];
            from.velocity[i] = velocity[first + i];
            directions.p[i] = p.direction + i * align_up(d, 64);
            to.to.p[i] = omega[first + i];
        }
        u32 parts = 0;
        if (const int rc = launch_direction(members, from, n, k, d, scale, mu, nesterov != 0, p.direction, align_up(d, 64), p.norm, kNormBlocks,
                                            &parts, stream))
            return rc;
        if (const int rc = iterate(products, directions, RTOPK_F32, cols, s, members, parts, all, largest_p, eps, p, to, stream)) return rc;
    }
    return RTOPK_OK;
}
