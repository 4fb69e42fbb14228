// Launches of the kernels that hold a picture's groups in registers.
#pragma once
#include "group_norm.h"
#include "norm_plan.h"

namespace ax {

// Pixels of a thread at most: 1024 threads have 128 registers each.  Backward a thread keeps four channels of any type: with
// eight 16-bit ones what it knows per channel would take half its registers.
constexpr int kForwardRegs = 16, kBackwardRegs = 8, kBackwardRegs1024 = 6, kBackwardVec = 4;
int launch_gn_slab_forward(GnArgs a, const SlabPlan& p, int type, int keep, hipStream_t st);
// a.part_c: [n][2][c], untouched for one picture
int launch_gn_slab_backward(GnArgs a, const SlabPlan& p, int type, int src, hipStream_t st);

}  // namespace ax
