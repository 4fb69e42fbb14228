// Launches of the kernels that hold a picture's groups in registers.
#pragma once
#include "group_norm.h"
#include "norm_plan.h"

namespace ax {

int launch_gn_slab_forward(GnArgs a, const SlabPlan& p, int type, int keep, hipStream_t st);
// a.part_c: [n][2][c], untouched for one picture
int launch_gn_slab_backward(GnArgs a, const SlabPlan& p, int type, int src, hipStream_t st);

}  // namespace ax
