// Dropout, the mask drawn and never stored.
//
//   out = (u >= T ? x * 65536 / (65536 - T) : 0) + residual,   T = p * 65536 rounded to a whole number
//
// u is a 16-bit draw of its own for each element: number e % 8 of the generator's group e / 8, e = row * cols + col. So the
// mask depends on the element's place alone, not on strides or launches, the gradient is the same call on dy, and
// what is kept is scaled by its true chance. One call of the generator for eight elements, 20 products of 16 cycles, stays under what 16-bit
// elements take to be read and written: bound by memory, 16384 x 4096 bfloat16 with a residual 79 us, 5.1 TB/s, without 48, 5.6 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/rtopk.h"
#include "rtopk_matrix.h"

namespace rtopk {

struct Dropout {
    const void *x, *residual;       // residual: of out's type, or null
    void *out;
    u64 ldx, ldr, ldo, rows, cols;
    int out_type;
    u32 below;                      // T
    float scale;
    Drawing drawing;
};

constexpr int kDropoutThreads = 256;

// kWhole: a group of eight lies in one row, as neighbours (the matrices are one piece, then rows = 1; or cols % 8 = 0). Otherwise
// element by element: 16384 x 4095 bfloat16 with rows 4100 apart 288 us with a residual, 189 without, of one piece 76 and 44.
template <int kType, bool kWhole>
__global__ void __launch_bounds__(kDropoutThreads) k_dropout(Dropout g)
{
    const PhiloxSeed seed = g.drawing.get();
    const u64 count = g.rows * g.cols, groups = (count + 7) / 8, each = (g.cols + 7) / 8;
    for (u64 at = (u64)blockIdx.x * kDropoutThreads + threadIdx.x; at < groups; at += (u64)gridDim.x * kDropoutThreads) {
        if constexpr (kWhole) {
            const u64 row = g.rows == 1 ? 0 : at / each, col = (at - row * each) * 8;
            const u64 left = g.cols - col;
            const u32 have = left < 8 ? (u32)left : 8u;
            const unsigned char *x = (const unsigned char *)g.x + (row * g.ldx + col) * Eight<kType>::kSize;
            Eight<kType> e;
            float v[8], more[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (have == 8) e.load(x, 0, 8);
            if (g.residual) {
                if (have == 8) {
                    if (g.out_type == RTOPK_F32) {
                        Eight<0> r;
                        r.load((const unsigned char *)g.residual + (row * g.ldr + col) * 4, 0, 8);
                        r.numbers(more, nullptr, 0, 8);
                    } else {
                        i32x4 w;
                        __builtin_memcpy(&w, (const u16 *)g.residual + row * g.ldr + col, 16);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const u16 h = (u16)((u32)w[i >> 1] >> (16 * (i & 1)));
                            more[i] = g.out_type == RTOPK_BF16 ? __uint_as_float((u32)h << 16) : (float)__builtin_bit_cast(_Float16, h);
                        }
                    }
                } else {
                    for (u32 i = 0; i < have; ++i) more[i] = read_as(g.residual, row * g.ldr + col + i, g.out_type);
                }
            }
            if (have == 8) e.numbers(v, x, 0, 8);
            else
                for (u32 i = 0; i < 8; ++i) v[i] = i < have ? read_as(x, i, kType) : 0.0f;
            const EightDraws u = draw_eight(at, kDrawsForDropout, seed);
            f32x4 y[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i >> 2][i & 3] = u[i] >= g.below ? fmaf(v[i], g.scale, more[i]) : more[i];
            write_eight(g.out, row * g.ldo + col, g.out_type, y[0], y[1], have);
        } else {
            const EightDraws u = draw_eight(at, kDrawsForDropout, seed);
            u64 row = at * 8 / g.cols, col = at * 8 - row * g.cols;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (at * 8 + i < count) {
                    const float more = g.residual ? read_as(g.residual, row * g.ldr + col, g.out_type) : 0.0f;
                    const float v = read_as(g.x, row * g.ldx + col, kType);
                    write_as(g.out, row * g.ldo + col, g.out_type, u[i] >= g.below ? fmaf(v, g.scale, more) : more);
                }
                if (++col == g.cols) {
                    col = 0;
                    ++row;
                }
            }
        }
    }
}

}  // namespace rtopk

using namespace rtopk;

namespace {

constexpr u64 kMostElements = 1ull << 40, kMostLength = 1ull << 32;

template <int kType>
int launch_dropout(Dropout g, hipStream_t stream)
{
    const bool one_piece = g.rows == 1 || (g.ldx == g.cols && g.ldo == g.cols && (!g.residual || g.ldr == g.cols));
    const bool whole = one_piece || g.cols % 8 == 0;
    if (one_piece) {
        g.cols *= g.rows;
        g.rows = 1;
    }
    const u64 groups = (g.rows * g.cols + 7) / 8, blocks = (groups + kDropoutThreads - 1) / kDropoutThreads;
    const u32 grid = (u32)std::min<u64>(blocks, 16 * kUnits);
    if (whole) k_dropout<kType, true><<<grid, kDropoutThreads, 0, stream>>>(g);
    else k_dropout<kType, false><<<grid, kDropoutThreads, 0, stream>>>(g);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_EHIP;
}

}  // namespace

extern "C" int rtopk_dropout(const void *x, int type, uint64_t rows, uint64_t cols, uint64_t ldx, const void *residual, uint64_t ldr,
                             void *out, int out_type, uint64_t ldo, double p, uint64_t seed, uint64_t step, const uint64_t *step_device,
                             void *stream_v)
{
    if (!type_ok(type) || !type_ok(out_type) || rows >= kMostLength || cols >= kMostLength || rows * cols > kMostElements) return RTOPK_EINVAL;
    if (!(p >= 0.0 && p <= 1.0) || ldx < cols || ldx >= kMostLength || ldo < cols || ldo >= kMostLength) return RTOPK_EINVAL;
    if (residual && (ldr < cols || ldr >= kMostLength)) return RTOPK_EINVAL;
    if (rows == 0 || cols == 0) return RTOPK_OK;
    if (!x || !out) return RTOPK_EINVAL;
    // out may be x or residual itself, element for element
    if ((out == x && (ldo != ldx || (type == RTOPK_F32) != (out_type == RTOPK_F32))) || (out == residual && ldo != ldr)) return RTOPK_EINVAL;
    const u32 below = (u32)std::rint(p * 65536.0);
    const Dropout g{x, residual, out, ldx, ldr, ldo, rows, cols, out_type, below, below < 65536u ? 65536.0f / (float)(65536u - below) : 0.0f,
                    Drawing{seed, step, step_device}};
    hipStream_t stream = (hipStream_t)stream_v;
    return type == RTOPK_F32 ? launch_dropout<RTOPK_F32>(g, stream)
           : type == RTOPK_BF16 ? launch_dropout<RTOPK_BF16>(g, stream) : launch_dropout<RTOPK_F16>(g, stream);
}
