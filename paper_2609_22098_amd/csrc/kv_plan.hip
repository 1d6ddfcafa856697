// Launcher of the planning kernels.
#include "kv_launch.hpp"
#include "kv_plan_kernels.hpp"

namespace ts {

void launch_kv_plan(const KvPlanParams& p, hipStream_t s) {
  // A slot map of a few entries a thread goes with the plan; a larger one is
  // spread over the device by a launch of its own.
  const bool slots = p.slot && (int64_t)p.R * p.cap <= 8192, few = p.R <= 16 && (!slots || p.R * p.cap <= 1024);
  if (few && slots)
    hipLaunchKernelGGL((kv_plan_kernel<256, true>), dim3(1), dim3(256), 0, s, p);
  else if (few)
    hipLaunchKernelGGL((kv_plan_kernel<256, false>), dim3(1), dim3(256), 0, s, p);
  else if (slots)
    hipLaunchKernelGGL((kv_plan_kernel<1024, true>), dim3(1), dim3(1024), 0, s, p);
  else
    hipLaunchKernelGGL((kv_plan_kernel<1024, false>), dim3(1), dim3(1024), 0, s, p);
  if (p.slot && !slots) {
    const int blocks = (p.cap + kSlotThreads - 1) / kSlotThreads;
    hipLaunchKernelGGL(kv_slot_kernel, dim3(p.R, blocks < 64 ? blocks : 64), dim3(kSlotThreads), 0, s, p);
  }
}

}  // namespace ts
