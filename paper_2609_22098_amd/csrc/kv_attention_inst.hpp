// Launcher of the cache attention for one head dimension; each has its own
// translation unit so that they compile in parallel.
#pragma once

#include "kv_attention_kernels.hpp"
#include "kv_launch.hpp"

namespace ts {

template <typename S>
static void launch_attention_shape(const KvAttnParams& p, int groups, hipStream_t s) {
  hipLaunchKernelGGL((kv_attention_kernel<S>), dim3(groups), dim3(S::kThreads), 0, s, p);
  if (p.whole_tiles) return;
  constexpr int kThreads = S::kRows > 32 ? 256 : 512, kUnit = S::kRows > 32 ? 1024 / S::D : 4, kMost = S::kRows > 32 ? 2048 : 1024;
  const int units = groups * (S::kRows / kUnit);
  hipLaunchKernelGGL((kv_join_kernel<typename S::TE, S::D, kThreads, kUnit>), dim3(units < kMost ? units : kMost), dim3(kThreads), 0, s, p,
                     __builtin_ctz(S::kRows), groups);
}

template <int D, bool WHOLE>
static void launch_attention_pages(const KvAttnParams& p, AttnTile tile, bool bf16, int groups, hipStream_t s) {
  if (bf16) {
    if (tile == AttnTile::k16) launch_attention_shape<AttnShape<D, 1, 1, 4, __bf16, WHOLE>>(p, groups, s);
    if (tile == AttnTile::k32) launch_attention_shape<AttnShape<D, 2, 1, 4, __bf16, WHOLE>>(p, groups, s);
    if (tile == AttnTile::k128) launch_attention_shape<AttnShape<D, 2, 4, 1, __bf16, WHOLE>>(p, groups, s);
  } else {
    if (tile == AttnTile::k16) launch_attention_shape<AttnShape<D, 1, 1, 4, float, WHOLE>>(p, groups, s);
    if (tile == AttnTile::k64) launch_attention_shape<AttnShape<D, 1, 4, 1, float, WHOLE>>(p, groups, s);
  }
}

template <int D>
void launch_kv_attention_t(const KvAttnParams& p, AttnTile tile, bool bf16, int groups, hipStream_t s) {
  if (p.c.page_shift >= 6)
    launch_attention_pages<D, true>(p, tile, bf16, groups, s);
  else
    launch_attention_pages<D, false>(p, tile, bf16, groups, s);
}

}  // namespace ts
