// Layer norm, forward and backward, over the rows of a matrix.
//
//   forward    mean = sum x / c, rstd = (sum (x - mean)^2 / c + eps)^-1/2,
//              y = (x - mean) rstd gamma + beta
//              A sum's roundings are off by parts of x, not of what varies around the mean. Where the mean is larger than that:
//              with m the mean that the sum gives and d = x - m, what is left is e = sum d / c, and mean = m + e,
//              x - mean = d - e, off by parts of d. (Where all numbers are equal, d is e, and y beta. Where the mean is smaller,
//              e would only add the roundings of d, which lean one way.)
//   backward   h = (x - mean) rstd, g = dy gamma:
//              dx = rstd (g - mean(g) - h mean(g h)) (+ add)
//              dgamma = sum over rows of dy h, dbeta = sum over rows of dy
//
// Everything between the loads and the stores is binary32 or more. The sums over rows are taken run by run, and the runs
// in order: no atomics, the same bits every time. What bounds all of it is memory: x, dy, add once, dx once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/rtopk.h"
#include "rtopk_matrix.h"

namespace rtopk {

struct Norm {
    const void *x;
    u64 ldx;
    u32 rows, cols;
    const float *gamma, *beta;      // or null: 1 and 0
    float eps;
    void *out;
    int out_type;
    u64 ldo;
    float *mean, *rstd;             // or null
};

constexpr int kNormThreads = 256;

// Eight numbers of a vector of binary32 that may be missing.
__device__ __forceinline__ void eight_or(float (&v)[8], const float *p, u32 c, u32 cols, float otherwise)
{
    if (p) {
        Eight<0> e;
        e.load((const unsigned char *)p, c, cols);
        e.numbers(v, (const unsigned char *)p, c, cols);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
    }
}

// The sum of one number of each lane of the kWavesPerRow wavefronts that share a row; `part` has a place for each wavefront.
template <int kWavesPerRow, class T>
__device__ __forceinline__ T sum_of_row(T v, T *part)
{
    T sum;
    if constexpr (sizeof(T) == 4) {
        sum = wave_sum_f32(v);
    } else {
        sum = v;
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    }
    if constexpr (kWavesPerRow > 1) {
        const u32 wave = threadIdx.x / kWave, first = wave / kWavesPerRow * kWavesPerRow;
        if (lane_id() == 0) part[wave] = sum;
        lds_barrier();
        sum = 0;
#pragma unroll
        for (u32 w = 0; w < kWavesPerRow; ++w) sum += part[first + w];
    }
    return sum;
}

// Rows by workgroups that keep going: kWavesPerRow wavefronts hold a row in registers, kPieces pieces of eight numbers a
// lane, and gamma and beta for all of their rows; the next row is on its way while this one's mean and variance are taken. Bound by its read
// and write: 16384 x 4096 bfloat16 48 to 53 us, 5.1 to 5.6 TB/s (a workgroup a row, which reads gamma and beta with each, 65); one row of 1500 2.9. Rows whose mean is larger than their
// standard deviation take two sums more: 53, 3.1.
template <int kType, int kWavesPerRow, int kPieces>
__global__ void __launch_bounds__(kWavesPerRow > 4 ? kWavesPerRow * kWave : kNormThreads) k_norm(Norm g)
{
    constexpr u32 kWaves = kWavesPerRow > 4 ? kWavesPerRow : 4, kRows = kWaves / kWavesPerRow, kStep = 8u * kWave * kWavesPerRow;
    __shared__ float part[8][kWaves];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c0 = (wave % kWavesPerRow * kWave + lane) * 8u, step = gridDim.x * kRows;
    const float cols = (float)g.cols;
    Eight<kType> next[kPieces];
    auto fetch = [&](u32 r) {
        const unsigned char *row = (const unsigned char *)g.x + min(r, g.rows - 1u) * g.ldx * Eight<kType>::kSize;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) next[p].load(row, c0 + p * kStep, g.cols);
    };
    u32 r = blockIdx.x * kRows + wave / kWavesPerRow, turn = 0;
    fetch(r);
    float gamma[kPieces][8], beta[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        eight_or(gamma[p], g.gamma, c0 + p * kStep, g.cols, 1.0f);
        eight_or(beta[p], g.beta, c0 + p * kStep, g.cols, 0.0f);
    }
    for (; r < g.rows; r += step, turn ^= 4u) {
        const unsigned char *row = (const unsigned char *)g.x + r * g.ldx * Eight<kType>::kSize;
        float x[kPieces][8], sum = 0, squares = 0;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            next[p].numbers(x[p], row, c0 + p * kStep, g.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[p][i];
        }
        if (r + step < g.rows) fetch(r + step);
        // around `by`, and the squares of that
        auto around = [&](float by) {
            squares = 0;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[p][i] = c0 + p * kStep + i < g.cols ? x[p][i] - by : 0.0f;
                    squares = fmaf(x[p][i], x[p][i], squares);
                }
        };
        // (places in turn: a wavefront that is a row ahead has passed all of this row's barriers)
        float mean = sum_of_row<kWavesPerRow>(sum, part[turn]) / cols;
        around(mean);
        squares = sum_of_row<kWavesPerRow>(squares, part[turn + 1]);
        // (the same in all of a row's wavefronts; what is beyond binary32's range counts as a larger mean)
        if (__builtin_amdgcn_readfirstlane(!(mean * mean * cols < squares))) {
            sum = 0;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[p][i];
            const float e = sum_of_row<kWavesPerRow>(sum, part[turn + 2]) / cols;
            around(e);
            squares = sum_of_row<kWavesPerRow>(squares, part[turn + 3]);
            mean += e;
        }
        const float rstd = 1.0f / sqrtf(squares / cols + g.eps);
        if (c0 == 0) {
            if (g.mean) g.mean[r] = mean;
            if (g.rstd) g.rstd[r] = rstd;
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const u32 c = c0 + p * kStep;
            if (c >= g.cols) continue;
            f32x4 y[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i >> 2][i & 3] = fmaf(x[p][i] * rstd, gamma[p][i], beta[p][i]);
            write_eight(g.out, r * g.ldo + c, g.out_type, y[0], y[1], g.cols - c);
        }
    }
}

// A longer row by one workgroup: it is read three times (the second and third time from the caches), with sums in binary64; e is what
// m loses of the mean as binary32. 2000 x 20,000 binary32 95 us, 3.4 TB/s, 256 x 262,144 bfloat16 105, 2.6.
template <int kType>
__global__ void __launch_bounds__(1024) k_norm_row(Norm g)
{
    constexpr int kWaves = 16;
    __shared__ double part[2][kWaves];
    const u64 r = (u64)blockIdx.y * gridDim.x + blockIdx.x;
    if (r >= g.rows) return;
    const unsigned char *row = (const unsigned char *)g.x + r * g.ldx * Eight<kType>::kSize;
    auto each = [&](auto act) {
        for (u32 c = threadIdx.x * 8u; c < g.cols; c += 8u * kWaves * kWave) {
            Eight<kType> e;
            float x[8];
            e.load(row, c, g.cols);
            e.numbers(x, row, c, g.cols);
            act(x, c);
        }
    };
    double sum = 0, squares = 0;
    each([&](const float (&x)[8], u32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)x[i];
    });
    const double mean = sum_of_row<kWaves>(sum, part[0]) / g.cols;
    const float m = (float)mean, e = (float)(mean - m);
    each([&](const float (&x)[8], u32 c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double d = c + i < g.cols ? x[i] - m : 0.0f;
            squares += d * d;
        }
    });
    const double var = sum_of_row<kWaves>(squares, part[1]) / g.cols - (mean - m) * (mean - m);
    const float rstd = 1.0f / sqrtf((float)(var < 0 ? 0.0 : var) + g.eps);
    if (threadIdx.x == 0) {
        if (g.mean) g.mean[r] = m;
        if (g.rstd) g.rstd[r] = rstd;
    }
    each([&](const float (&x)[8], u32 c) {
        float gamma[8], beta[8];
        eight_or(gamma, g.gamma, c, g.cols, 1.0f);
        eight_or(beta, g.beta, c, g.cols, 0.0f);
        f32x4 y[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i >> 2][i & 3] = fmaf((x[i] - m - e) * rstd, gamma[i], beta[i]);
        write_eight(g.out, r * g.ldo + c, g.out_type, y[0], y[1], g.cols - c);
    });
}

// ---------------------------------------------------------------------------
// Backward.
// ---------------------------------------------------------------------------

// Eight neighbours of a type that is known when the kernel runs only (the same for all lanes).
struct EightOf {
    i32x4 w[2];
    __device__ __forceinline__ void load(const unsigned char *row, u32 c, u32 cols, int type)
    {
        if (type == RTOPK_F32) {
            Eight<RTOPK_F32> e;
            e.load(row, c, cols);
            w[0] = e.w[0];
            w[1] = e.w[1];
        } else {
            Eight<RTOPK_BF16> e;
            e.load(row, c, cols);
            w[0] = e.w[0];
        }
    }
    __device__ __forceinline__ void numbers(float (&v)[8], const unsigned char *row, u32 c, u32 cols, int type) const
    {
        if (type == RTOPK_F32) {
            Eight<RTOPK_F32> e;
            e.w[0] = w[0];
            e.w[1] = w[1];
            e.numbers(v, row, c, cols);
        } else if (type == RTOPK_BF16) {
            Eight<RTOPK_BF16> e;
            e.w[0] = w[0];
            e.numbers(v, row, c, cols);
        } else {
            Eight<RTOPK_F16> e;
            e.w[0] = w[0];
            e.numbers(v, row, c, cols);
        }
    }
};
__device__ __forceinline__ u32 size_of(int type) { return type == RTOPK_F32 ? 4u : 2u; }

struct NormBack {
    const void *dy, *x, *add;       // add: of x's type, or null
    int dy_type;
    u64 lddy, ldx, ldadd;
    u32 rows, cols;
    const float *mean, *rstd, *gamma;
    void *dx;                       // of x's type, or null
    u64 lddx;
    u32 groups;                     // workgroups that share the rows
    u32 runs, run;                  // the sums over rows: runs of so many rows
    float *dgamma, *dbeta;          // or null
    float *part;                    // [2][runs][cols], or null
};

// All of the sums of 32 columns by one workgroup of kThreads: four lanes have eight columns each, and every kThreads / 4th row. For
// small matrices: neither runs of rows to be joined nor a launch for them.
constexpr u32 kDirectColumns = 32, kDirectLanes = kDirectColumns / 8;

template <int kType, u32 kThreads>
__device__ __forceinline__ void sum_columns(const NormBack &g, u32 strip)
{
    constexpr u32 kWaves = kThreads / kWave, kLanes = kThreads / kDirectLanes, kAtOnce = 4;
    __shared__ __align__(16) float part[2][kWaves][kDirectColumns];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c = strip * kDirectColumns + 8u * (threadIdx.x % kDirectLanes);
    float dgamma[8] = {0, 0, 0, 0, 0, 0, 0, 0}, dbeta[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (u32 r = threadIdx.x / kDirectLanes; r < g.rows; r += kAtOnce * kLanes) {
        Eight<kType> ex[kAtOnce];
        EightOf ey[kAtOnce];
        float mean[kAtOnce], rstd[kAtOnce];
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            const u64 row = min(r + q * kLanes, g.rows - 1u);
            ex[q].load((const unsigned char *)g.x + row * g.ldx * Eight<kType>::kSize, c, g.cols);
            ey[q].load((const unsigned char *)g.dy + row * g.lddy * size_of(g.dy_type), c, g.cols, g.dy_type);
            mean[q] = g.mean[row];
            rstd[q] = g.rstd[row];
        }
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            const u64 row = r + q * kLanes;
            if (row >= g.rows) break;
            float x[8], d[8];
            ex[q].numbers(x, (const unsigned char *)g.x + row * g.ldx * Eight<kType>::kSize, c, g.cols);
            ey[q].numbers(d, (const unsigned char *)g.dy + row * g.lddy * size_of(g.dy_type), c, g.cols, g.dy_type);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dgamma[i] = fmaf(d[i], (x[i] - mean[q]) * rstd[q], dgamma[i]);
                dbeta[i] += d[i];
            }
        }
    }
#pragma unroll
    for (int o = kDirectLanes; o < kWave; o <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dgamma[i] += __shfl_xor(dgamma[i], o, kWave);
            dbeta[i] += __shfl_xor(dbeta[i], o, kWave);
        }
    if (lane < kDirectLanes) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[0][wave][8 * lane + i] = dgamma[i];
            part[1][wave][8 * lane + i] = dbeta[i];
        }
    }
    __syncthreads();
    const u32 which = threadIdx.x / kDirectColumns, col = threadIdx.x % kDirectColumns, at = strip * kDirectColumns + col;
    float *out = which ? g.dbeta : g.dgamma;
    if (which > 1 || at >= g.cols || !out) return;
    float sum = 0;
#pragma unroll
    for (u32 w = 0; w < kWaves; ++w) sum += part[which][w][col];
    out[at] = sum;
}

template <int kType>
__global__ void __launch_bounds__(kNormThreads) k_norm_back_sums(NormBack g)
{
    sum_columns<kType, kNormThreads>(g, blockIdx.x);
}

// Rows by workgroups that keep going: kWavesPerRow wavefronts hold a row in registers, kPieces pieces of eight numbers a
// lane, the next row's x and dy on their way while this one's means are taken and its dx is written. One read of everything,
// one write: a lane's share of dgamma and dbeta stays in registers over all of its rows, and goes to g.part, if that is there, to be
// joined with the other workgroups'. Workgroups of the launch from g.groups on, if there are any, take the sums by themselves. Bound by
// memory to 8192 columns: 16384 x 4096 bfloat16 with `add` 104 us, 5.2 TB/s (dx and the sums by a kernel each 240), 8192 x 8192 109, 4.9; 700 x 1500
// 9.6 us, sums beside. Sixteen wavefronts a row (8193 to 16384 columns) have 128 registers a lane and spill: 264 bytes a lane of binary32, 184 of the
// other types, read back with each row; 4096 x 12,000 bfloat16 201 us, 2.0 TB/s, 4096 x 16,384 228, 2.4.
template <int kType, int kWavesPerRow, int kPieces>
__global__ void __launch_bounds__(kWavesPerRow > 4 ? kWavesPerRow * kWave : kNormThreads) k_norm_back(NormBack g)
{
    if (blockIdx.x >= g.groups) {
        sum_columns<kType, (kWavesPerRow > 4 ? kWavesPerRow * kWave : kNormThreads)>(g, blockIdx.x - g.groups);
        return;
    }
    constexpr u32 kWaves = kWavesPerRow > 4 ? kWavesPerRow : 4, kRows = kWaves / kWavesPerRow, kStep = 8u * kWave * kWavesPerRow;
    __shared__ float means[2][2][kWaves];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c0 = (wave % kWavesPerRow * kWave + lane) * 8u;
    const u32 step = g.groups * kRows;
    const float per_row = 1.0f / (float)g.cols;
    float gamma[kPieces][8], dgamma[kPieces][8], dbeta[kPieces][8];
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        eight_or(gamma[p], g.gamma, c0 + p * kStep, g.cols, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) dgamma[p][i] = dbeta[p][i] = 0.0f;
    }
    Eight<kType> next_x[kPieces];
    EightOf next_dy[kPieces];
    float next_mean, next_rstd;
    auto fetch = [&](u32 r) {
        const u64 row = min(r, g.rows - 1u);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            next_x[p].load((const unsigned char *)g.x + row * g.ldx * Eight<kType>::kSize, c0 + p * kStep, g.cols);
            next_dy[p].load((const unsigned char *)g.dy + row * g.lddy * size_of(g.dy_type), c0 + p * kStep, g.cols, g.dy_type);
        }
        next_mean = g.mean[row];
        next_rstd = g.rstd[row];
    };
    u32 r = blockIdx.x * kRows + wave / kWavesPerRow, turn = 0;
    fetch(r);
    for (; r < g.rows; r += step, turn ^= 1u) {
        const unsigned char *x_row = (const unsigned char *)g.x + r * g.ldx * Eight<kType>::kSize;
        const unsigned char *dy_row = (const unsigned char *)g.dy + r * g.lddy * size_of(g.dy_type);
        const unsigned char *add_row = (const unsigned char *)g.add + r * g.ldadd * Eight<kType>::kSize;
        const float mean = next_mean, rstd = next_rstd;
        Eight<kType> held_add[kPieces];
        float h[kPieces][8], d[kPieces][8], sum = 0, inner = 0;
        if (g.add) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p) held_add[p].load(add_row, c0 + p * kStep, g.cols);
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const u32 c = c0 + p * kStep;
            next_x[p].numbers(h[p], x_row, c, g.cols);
            next_dy[p].numbers(d[p], dy_row, c, g.cols, g.dy_type);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[p][i] = c + i < g.cols ? (h[p][i] - mean) * rstd : 0.0f;      // (d is zero there)
                dgamma[p][i] = fmaf(d[p][i], h[p][i], dgamma[p][i]);
                dbeta[p][i] += d[p][i];
                d[p][i] *= gamma[p][i];
                sum += d[p][i];
                inner = fmaf(d[p][i], h[p][i], inner);
            }
        }
        if (r + step < g.rows) fetch(r + step);
        sum = wave_sum_f32(sum);
        inner = wave_sum_f32(inner);
        if constexpr (kWavesPerRow > 1) {
            // (two places in turn: a wavefront that is a row ahead has passed this row's barrier)
            if (lane == 0) {
                means[turn][0][wave] = sum;
                means[turn][1][wave] = inner;
            }
            lds_barrier();
            sum = inner = 0;
#pragma unroll
            for (u32 w = 0; w < kWavesPerRow; ++w) {
                sum += means[turn][0][w];
                inner += means[turn][1][w];
            }
        }
        const float m0 = sum * per_row, m1 = inner * per_row;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const u32 c = c0 + p * kStep;
            if (c >= g.cols) continue;
            float more[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (g.add) held_add[p].numbers(more, add_row, c, g.cols);
            f32x4 v[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = fmaf(rstd, fmaf(-h[p][i], m1, d[p][i] - m0), more[i]);
            write_eight(g.dx, r * g.lddx + c, kType, v[0], v[1], g.cols - c);
        }
    }
    if (g.part) {
        float *out = g.part + (u64)blockIdx.x * g.cols;
        const u64 beta = (u64)g.runs * g.cols;
        if constexpr (kRows > 1) {
            // the rows' wavefronts together
            __shared__ float joined[2][kRows - 1][kPieces * 8 * kWave];
            if (wave) {
#pragma unroll
                for (int p = 0; p < kPieces; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        joined[0][wave - 1][(8 * p + i) * kWave + lane] = dgamma[p][i];
                        joined[1][wave - 1][(8 * p + i) * kWave + lane] = dbeta[p][i];
                    }
            }
            __syncthreads();
            if (wave) return;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (u32 w = 0; w < kRows - 1; ++w) {
                        dgamma[p][i] += joined[0][w][(8 * p + i) * kWave + lane];
                        dbeta[p][i] += joined[1][w][(8 * p + i) * kWave + lane];
                    }
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const u32 c = c0 + p * kStep;
            if (c >= g.cols) continue;
            write_eight(out, c, RTOPK_F32, f32x4{dgamma[p][0], dgamma[p][1], dgamma[p][2], dgamma[p][3]},
                        f32x4{dgamma[p][4], dgamma[p][5], dgamma[p][6], dgamma[p][7]}, g.cols - c);
            write_eight(out + beta, c, RTOPK_F32, f32x4{dbeta[p][0], dbeta[p][1], dbeta[p][2], dbeta[p][3]},
                        f32x4{dbeta[p][4], dbeta[p][5], dbeta[p][6], dbeta[p][7]}, g.cols - c);
        }
    }
}

// A longer row by one workgroup: its two means, then dx; dy and x are read twice, the second time from the caches. With the sums over rows by
// runs before it, 2000 x 20,000 bfloat16 with `add` 113 us (76 without the sums), 2.8 TB/s.
template <int kType>
__global__ void __launch_bounds__(1024) k_norm_back_row(NormBack g)
{
    constexpr int kWaves = 16;
    __shared__ double part[2][kWaves];
    const u64 r = (u64)blockIdx.y * gridDim.x + blockIdx.x;
    if (r >= g.rows) return;
    const unsigned char *x_row = (const unsigned char *)g.x + r * g.ldx * Eight<kType>::kSize;
    const unsigned char *dy_row = (const unsigned char *)g.dy + r * g.lddy * size_of(g.dy_type);
    const unsigned char *add_row = g.add ? (const unsigned char *)g.add + r * g.ldadd * Eight<kType>::kSize : nullptr;
    const float mean = g.mean[r], rstd = g.rstd[r];
    float h[8], d[8], gamma[8];
    auto read = [&](u32 c) {
        Eight<kType> ex;
        EightOf ey;
        ex.load(x_row, c, g.cols);
        ey.load(dy_row, c, g.cols, g.dy_type);
        eight_or(gamma, g.gamma, c, g.cols, 1.0f);
        ex.numbers(h, x_row, c, g.cols);
        ey.numbers(d, dy_row, c, g.cols, g.dy_type);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = (h[i] - mean) * rstd;
            d[i] = c + i < g.cols ? d[i] * gamma[i] : 0.0f;
        }
    };
    double sum = 0, inner = 0;
    for (u32 c = threadIdx.x * 8u; c < g.cols; c += 8u * kWaves * kWave) {
        read(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum += (double)d[i];
            inner += c + i < g.cols ? (double)d[i] * (double)h[i] : 0.0;
        }
    }
    const float m0 = (float)(sum_of_row<kWaves>(sum, part[0]) / g.cols), m1 = (float)(sum_of_row<kWaves>(inner, part[1]) / g.cols);
    for (u32 c = threadIdx.x * 8u; c < g.cols; c += 8u * kWaves * kWave) {
        read(c);
        float more[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (add_row) {
            Eight<kType> ea;
            ea.load(add_row, c, g.cols);
            ea.numbers(more, add_row, c, g.cols);
        }
        f32x4 v[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = fmaf(rstd, fmaf(-h[i], m1, d[i] - m0), more[i]);
        write_eight(g.dx, r * g.lddx + c, kType, v[0], v[1], g.cols - c);
    }
}

// The sums of a run of rows, 512 columns a workgroup: a wavefront takes every fourth row.
constexpr u32 kSumColumns = 8 * kWave;

template <int kType>
__global__ void __launch_bounds__(kNormThreads) k_norm_back_columns(NormBack g)
{
    constexpr u32 kWaves = kNormThreads / kWave, kAtOnce = 4;
    __shared__ float part[2][kWaves - 1][kSumColumns];
    const u32 lane = lane_id(), wave = threadIdx.x / kWave, c = blockIdx.x * kSumColumns + lane * 8u;
    const u32 r0 = blockIdx.y * g.run, r1 = min(r0 + g.run, g.rows);
    float dgamma[8] = {0, 0, 0, 0, 0, 0, 0, 0}, dbeta[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (u32 r = r0 + wave; r < r1; r += kAtOnce * kWaves) {
        Eight<kType> ex[kAtOnce];
        EightOf ey[kAtOnce];
        float mean[kAtOnce], rstd[kAtOnce];
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            const u64 row = min(r + q * kWaves, r1 - 1u);
            ex[q].load((const unsigned char *)g.x + row * g.ldx * Eight<kType>::kSize, c, g.cols);
            ey[q].load((const unsigned char *)g.dy + row * g.lddy * size_of(g.dy_type), c, g.cols, g.dy_type);
            mean[q] = g.mean[row];
            rstd[q] = g.rstd[row];
        }
#pragma unroll
        for (u32 q = 0; q < kAtOnce; ++q) {
            if (r + q * kWaves >= r1) break;
            const u64 row = r + q * kWaves;
            float x[8], d[8];
            ex[q].numbers(x, (const unsigned char *)g.x + row * g.ldx * Eight<kType>::kSize, c, g.cols);
            ey[q].numbers(d, (const unsigned char *)g.dy + row * g.lddy * size_of(g.dy_type), c, g.cols, g.dy_type);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dgamma[i] = fmaf(d[i], (x[i] - mean[q]) * rstd[q], dgamma[i]);
                dbeta[i] += d[i];
            }
        }
    }
    if (wave) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[0][wave - 1][i * kWave + lane] = dgamma[i];
            part[1][wave - 1][i * kWave + lane] = dbeta[i];
        }
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (u32 w = 0; w < kWaves - 1; ++w) {
            dgamma[i] += part[0][w][i * kWave + lane];
            dbeta[i] += part[1][w][i * kWave + lane];
        }
        if (c + i < g.cols) {
            g.part[(u64)blockIdx.y * g.cols + c + i] = dgamma[i];
            g.part[((u64)g.runs + blockIdx.y) * g.cols + c + i] = dbeta[i];
        }
    }
}

// The runs together, in binary64, 16 columns a workgroup; blockIdx.y: dgamma, dbeta. 512 runs of 4096 columns 7 us, mostly from the caches.
constexpr u32 kJoinColumns = 16, kJoinThreads = 1024;

__global__ void __launch_bounds__(kJoinThreads) k_norm_back_join(NormBack g)
{
    constexpr u32 kWaves = kJoinThreads / kWave, kAtOnce = kJoinThreads / kJoinColumns;
    __shared__ double part[kWaves][kJoinColumns];
    const u32 c = blockIdx.x * kJoinColumns + threadIdx.x % kJoinColumns;
    float *out = blockIdx.y ? g.dbeta : g.dgamma;
    if (!out) return;
    const float *from = g.part + (u64)blockIdx.y * g.runs * g.cols + min(c, g.cols - 1u);
    double sum = 0;
#pragma unroll 8
    for (u32 s = threadIdx.x / kJoinColumns; s < g.runs; s += kAtOnce) sum += (double)from[(u64)s * g.cols];
#pragma unroll
    for (int o = kJoinColumns; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
    if (lane_id() < kJoinColumns) part[threadIdx.x / kWave][lane_id()] = sum;
    __syncthreads();
    if (threadIdx.x >= kJoinColumns || c >= g.cols) return;
    sum = 0;
#pragma unroll
    for (u32 w = 0; w < kWaves; ++w) sum += part[w][threadIdx.x];
    out[c] = (float)sum;
}

__global__ void __launch_bounds__(256) k_norm_zero(float *p, u32 count)
{
    for (u64 at = (u64)blockIdx.x * 256 + threadIdx.x; at < count; at += (u64)gridDim.x * 256) p[at] = 0.0f;
}

}  // namespace rtopk

using namespace rtopk;

namespace {

constexpr u64 kMostSize = 1u << 22;

bool size_ok(u64 v) { return v >= 1 && v <= kMostSize; }
int launched() { return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP; }

// (a launch has less than 2^32 threads along x)
dim3 row_grid(u32 blocks) { return dim3(std::min(blocks, 1u << 20), (blocks + (1u << 20) - 1) >> 20); }

// Rows that registers hold: workgroups that keep going, two a compute unit (one of sixteen wavefronts).
constexpr u32 kHeldColumns = 16384;
u32 rows_at_once(u32 cols) { return cols <= 1024 ? 4 : 1; }
u32 held_groups(u32 rows, u32 cols, u32 each)
{
    return std::min((rows + rows_at_once(cols) - 1) / rows_at_once(cols), (cols <= 4096 ? each : cols <= 8192 ? (each + 1) / 2 : 1) * kUnits);
}

template <int kType>
int launch_norm(const Norm &g, hipStream_t stream)
{
    const u32 cols = g.cols, grid = held_groups(g.rows, g.cols, 4);
    if (cols <= 1024) k_norm<kType, 1, 2><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 2048) k_norm<kType, 4, 1><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 4096) k_norm<kType, 4, 2><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 8192) k_norm<kType, 8, 2><<<grid, 8 * kWave, 0, stream>>>(g);
    else if (cols <= kHeldColumns) k_norm<kType, 16, 2><<<grid, 16 * kWave, 0, stream>>>(g);
    else k_norm_row<kType><<<row_grid(g.rows), 1024, 0, stream>>>(g);
    return launched();
}

// Sums alone, or of longer rows: runs of rows, two workgroups a compute unit, 16 rows at least.
constexpr u32 kMostRuns = 128;
u32 run_rows(u32 rows, u32 cols)
{
    const u32 groups = (cols + kSumColumns - 1) / kSumColumns, runs = std::min(kMostRuns, (2 * kUnits + groups - 1) / groups);
    return std::max((rows + runs - 1) / runs, 16u);
}
u32 run_count(u32 rows, u32 cols) { return (rows + run_rows(rows, cols) - 1) / run_rows(rows, cols); }

// Small matrices: their sums cost less than a launch that joins them (the second read comes from the caches).
bool small(u64 rows, u64 cols) { return rows <= 2048 && rows * cols <= 1u << 21; }

template <int kType>
int launch_held(const NormBack &g, u32 beside, hipStream_t stream)
{
    const u32 cols = g.cols, grid = g.groups + beside;
    if (cols <= 1024) k_norm_back<kType, 1, 2><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 2048) k_norm_back<kType, 4, 1><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 4096) k_norm_back<kType, 4, 2><<<grid, kNormThreads, 0, stream>>>(g);
    else if (cols <= 8192) k_norm_back<kType, 8, 2><<<grid, 8 * kWave, 0, stream>>>(g);
    else k_norm_back<kType, 16, 2><<<grid, 16 * kWave, 0, stream>>>(g);
    return launched();
}

int join_sums(const NormBack &g, hipStream_t stream)
{
    k_norm_back_join<<<dim3((g.cols + kJoinColumns - 1) / kJoinColumns, 2), kJoinThreads, 0, stream>>>(g);
    return launched();
}

template <int kType>
int launch_back(NormBack g, hipStream_t stream)
{
    const bool held = g.dx && g.cols <= kHeldColumns, direct = small(g.rows, g.cols);
    const bool sums = g.dgamma || g.dbeta;
    const u32 strips = (g.cols + kDirectColumns - 1) / kDirectColumns;
    g.groups = held_groups(g.rows, g.cols, 2);
    float *const room = g.part;
    g.part = nullptr;
    if (held && sums && direct && g.dx != g.x && g.dx != g.dy) return launch_held<kType>(g, strips, stream);
    if (held && sums && !direct) {
        g.runs = g.groups;
        g.part = room;
        if (const int rc = launch_held<kType>(g, 0, stream)) return rc;
        return join_sums(g, stream);
    }
    // the sums first: dx may be x or dy
    if (sums && direct) {
        k_norm_back_sums<kType><<<strips, kNormThreads, 0, stream>>>(g);
        if (const int rc = launched()) return rc;
    } else if (sums) {
        g.run = run_rows(g.rows, g.cols);
        g.runs = run_count(g.rows, g.cols);
        g.part = room;
        k_norm_back_columns<kType><<<dim3((g.cols + kSumColumns - 1) / kSumColumns, g.runs), kNormThreads, 0, stream>>>(g);
        if (const int rc = launched()) return rc;
        if (const int rc = join_sums(g, stream)) return rc;
    }
    g.part = nullptr;
    if (held) return launch_held<kType>(g, 0, stream);
    if (g.dx) k_norm_back_row<kType><<<row_grid(g.rows), 1024, 0, stream>>>(g);
    return launched();
}

}  // namespace

extern "C" int rtopk_layer_norm(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx, const float *gamma,
                                const float *beta, float eps, void *out, int out_type, uint64_t ldo, float *mean, float *rstd,
                                void *stream_v)
{
    if (!type_ok(type) || !type_ok(out_type) || rows > kMostSize || !size_ok(cols)) return RTOPK_EINVAL;
    if (ldx < cols || ldx > kMostSize || ldo < cols || ldo > kMostSize || !(eps >= 0.0f) || std::isinf(eps)) return RTOPK_EINVAL;
    if (rows == 0) return RTOPK_OK;
    if (!x || !out || (x == out && (ldx != ldo || (type == RTOPK_F32) != (out_type == RTOPK_F32)))) return RTOPK_EINVAL;
    const Norm g{x, ldx, (u32)rows, (u32)cols, gamma, beta, eps, out, out_type, ldo, mean, rstd};
    hipStream_t stream = (hipStream_t)stream_v;
    return type == RTOPK_F32 ? launch_norm<RTOPK_F32>(g, stream)
           : type == RTOPK_BF16 ? launch_norm<RTOPK_BF16>(g, stream) : launch_norm<RTOPK_F16>(g, stream);
}

extern "C" int rtopk_layer_norm_backward_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t *bytes)
{
    if (!bytes || rows > kMostSize || !size_ok(cols)) return RTOPK_EINVAL;
    *bytes = 0;
    if (!small(rows, cols)) {
        const u32 runs = run_count((u32)rows, (u32)cols), held = cols <= kHeldColumns ? held_groups((u32)rows, (u32)cols, 2) : 0;
        *bytes = align_up(8ull * std::max(runs, held) * cols, 256);
    }
    return RTOPK_OK;
}

extern "C" int rtopk_layer_norm_backward(const void *dy, int dy_type, const void *x, int type, uint64_t rows, uint64_t cols,
                                         uint64_t lddy, uint64_t ldx, const float *mean, const float *rstd, const float *gamma,
                                         const void *add, uint64_t ldadd, void *dx, uint64_t lddx, float *dgamma, float *dbeta,
                                         void *workspace, uint64_t workspace_bytes, void *stream_v)
{
    uint64_t need = 0;
    if (!type_ok(type) || !type_ok(dy_type) || rtopk_layer_norm_backward_workspace_bytes(rows, cols, &need) != RTOPK_OK) return RTOPK_EINVAL;
    if (lddy < cols || lddy > kMostSize || ldx < cols || ldx > kMostSize) return RTOPK_EINVAL;
    if ((!dx && !dgamma && !dbeta) || (add && !dx) || (dx && (lddx < cols || lddx > kMostSize))) return RTOPK_EINVAL;
    if (add && (ldadd < cols || ldadd > kMostSize)) return RTOPK_EINVAL;
    if (rows && (!dy || !x || !mean || !rstd)) return RTOPK_EINVAL;
    // dx may be dy, x or add itself, element for element
    if (dx && rows && ((dx == dy && (lddx != lddy || (type == RTOPK_F32) != (dy_type == RTOPK_F32))) || (dx == x && lddx != ldx) ||
                       (dx == add && lddx != ldadd)))
        return RTOPK_EINVAL;
    const bool sums = dgamma || dbeta;
    if (sums && need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return RTOPK_EWORKSPACE;
    hipStream_t stream = (hipStream_t)stream_v;
    if (rows == 0) {
        for (float *p : {dgamma, dbeta}) {
            if (!p) continue;
            k_norm_zero<<<(unsigned)((cols + 255) / 256), 256, 0, stream>>>(p, (u32)cols);
            if (const int rc = launched()) return rc;
        }
        return RTOPK_OK;
    }
    const NormBack g{dy, x, add, dy_type, lddy, ldx, ldadd, (u32)rows, (u32)cols, mean, rstd, gamma, dx, lddx, 0, 0, 0,
                     dgamma, dbeta, (float *)workspace};
    return type == RTOPK_F32 ? launch_back<RTOPK_F32>(g, stream)
           : type == RTOPK_BF16 ? launch_back<RTOPK_BF16>(g, stream) : launch_back<RTOPK_F16>(g, stream);
}
