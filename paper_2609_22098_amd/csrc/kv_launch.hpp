// Launchers of the cache kernels.
#pragma once

#include "kv_format.hpp"

namespace ts {

void launch_kv_plan(const KvPlanParams& p, hipStream_t s);
void launch_kv_append(const KvAppendParams& p, int head_dim, bool bf16, hipStream_t s);
void launch_kv_read(const KvReadParams& p, int head_dim, bool bf16, hipStream_t s);
void launch_kv_accept(const KvAcceptParams& p, int head_dim, hipStream_t s);
// Attention with `groups` workgroups, and the joining of their parts.
template <int D>
void launch_kv_attention_t(const KvAttnParams& p, AttnTile tile, bool bf16, int groups, hipStream_t s);

}  // namespace ts
