// Launchers of the cache's row kernels.
#include <type_traits>

#include "kv_launch.hpp"
#include "kv_rows_kernels.hpp"

namespace ts {
namespace {

// Calls f with the head dimension as a constant.
template <typename F>
void with_dim(int head_dim, F f) {
  if (head_dim == 64) f(std::integral_constant<int, 64>{});
  if (head_dim == 128) f(std::integral_constant<int, 128>{});
  if (head_dim == 256) f(std::integral_constant<int, 256>{});
}

}  // namespace

void launch_kv_append(const KvAppendParams& p, int head_dim, bool bf16, hipStream_t s) {
  with_dim(head_dim, [&](auto d) {
    constexpr int D = decltype(d)::value;
    const int64_t per = kRowThreads / (D / 8), items = (int64_t)p.rows * p.c.heads;
    const dim3 grid((uint32_t)((items + per - 1) / per)), block(kRowThreads);
    if (bf16)
      hipLaunchKernelGGL((kv_append_kernel<__bf16, D>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((kv_append_kernel<float, D>), grid, block, 0, s, p);
  });
}

void launch_kv_read(const KvReadParams& p, int head_dim, bool bf16, hipStream_t s) {
  with_dim(head_dim, [&](auto d) {
    constexpr int D = decltype(d)::value;
    const int64_t per = kRowThreads / (D / 8), items = (int64_t)p.rows * p.c.heads;
    const dim3 grid((uint32_t)((items + per - 1) / per), p.layers), block(kRowThreads);
    if (bf16)
      hipLaunchKernelGGL((kv_read_kernel<__bf16, D>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((kv_read_kernel<float, D>), grid, block, 0, s, p);
  });
}

void launch_kv_accept(const KvAcceptParams& p, int head_dim, hipStream_t s) {
  with_dim(head_dim, [&](auto d) {
    constexpr int D = decltype(d)::value;
    hipLaunchKernelGGL((kv_accept_kernel<D>), dim3(p.R, p.layers), dim3(kAcceptThreads), 0, s, p);
  });
}

}  // namespace ts
