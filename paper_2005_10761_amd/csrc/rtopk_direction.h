// The direction of the master's step for matrices, from the messages: made beside the other master kernels, used by
// the orthogonalised update.
#pragma once

#include "rtopk_common.h"

namespace rtopk {

constexpr u32 kMembers = 16;            // matrices in one launch

struct DirectionMembers {
    const u32 *idx[kMembers];
    const float *val[kMembers];
    float *velocity[kMembers];
};

// velocity <- mu velocity + scale average; direction[i * direction_stride ..] = mu velocity + scale average, or the new
// velocity; part[i * part_stride ..]: *parts (at most part_stride) parts of matrix i's squared norm.
int launch_direction(u32 members, const DirectionMembers &g, u32 n, u64 k, u64 d, float scale, float mu, bool nesterov, float *direction,
                     u64 direction_stride, double *part, u32 part_stride, u32 *parts, hipStream_t stream);

}  // namespace rtopk
