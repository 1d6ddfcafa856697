// Launcher of the cache attention.
#include "kv_attention_kernels.hpp"
#include "kv_launch.hpp"

namespace ts {

template <typename TE>
static void launch_t(const KvAttnParams& p, int head_dim, hipStream_t s) {
  const int64_t items = (int64_t)p.R * p.cap * p.q_heads;
  const dim3 grid((uint32_t)((items + kAttnWaves - 1) / kAttnWaves)), block(64 * kAttnWaves);
  if (head_dim == 64) hipLaunchKernelGGL((kv_attention_kernel<TE, 64>), grid, block, 0, s, p);
  if (head_dim == 128) hipLaunchKernelGGL((kv_attention_kernel<TE, 128>), grid, block, 0, s, p);
  if (head_dim == 256) hipLaunchKernelGGL((kv_attention_kernel<TE, 256>), grid, block, 0, s, p);
}

void launch_kv_attention(const KvAttnParams& p, int head_dim, bool bf16, hipStream_t s) {
  if (bf16)
    launch_t<__bf16>(p, head_dim, s);
  else
    launch_t<float>(p, head_dim, s);
}

}  // namespace ts
