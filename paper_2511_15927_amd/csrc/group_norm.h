// The norm of groups of channels with an activation or a gate: what its kernels take, and their launcher (group_norm_inst.hip, one object
// per activation).
#pragma once
#include "model_ops.h"

namespace bm {

struct GroupNormArgs {
    RowView x, z, y, dy, dx, dz;
    const float *weight, *bias;   // null: 1, 0
    float *mean, *rstd;           // [rows][G]; forward: null, not wanted
    float *dw, *db;               // sums of a row group, null: not wanted
    long long slot;               // from one row group's to the next one's
    unsigned L, rows, per_wave;   // steps that a wave takes, or the waves that share a group together
    int at_once;                  // rows of a step: several where a row's groups leave lanes free
    int G, n, d, lanes;           // groups, channels of one; lanes of a wave that hold one
    int centred;
    float eps;
};
// Which waves hold a group, in how many pieces a lane, how many waves a workgroup has, and the launch.
struct GroupPlan {
    int waves, pieces, lanes, at_once, team;
    unsigned tiles, row_groups, per_wave;
};
template <int kAct>
void launch_group_norm(const GroupPlan& p, const GroupNormArgs& a, bool bf16, bool past, bool bwd, hipStream_t st);

}  // namespace bm
