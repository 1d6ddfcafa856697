// Launcher of the planning kernels.
#include "kv_launch.hpp"
#include "kv_plan_kernels.hpp"

namespace ts {

void launch_kv_plan(const KvPlanParams& p, hipStream_t s) {
  hipLaunchKernelGGL(kv_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
  if (p.slot) {
    const int blocks = (p.cap + kSlotThreads - 1) / kSlotThreads;
    hipLaunchKernelGGL(kv_slot_kernel, dim3(p.R, blocks < 64 ? blocks : 64), dim3(kSlotThreads), 0, s, p);
  }
}

}  // namespace ts
