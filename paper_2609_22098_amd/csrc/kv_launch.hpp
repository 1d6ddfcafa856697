// Launchers of the cache kernels.
#pragma once

#include "kv_format.hpp"

namespace ts {

void launch_kv_plan(const KvPlanParams& p, hipStream_t s);
void launch_kv_append(const KvAppendParams& p, int head_dim, bool bf16, hipStream_t s);
void launch_kv_read(const KvReadParams& p, int head_dim, bool bf16, hipStream_t s);
void launch_kv_accept(const KvAcceptParams& p, int head_dim, hipStream_t s);
void launch_kv_attention(const KvAttnParams& p, int head_dim, bool bf16, hipStream_t s);

}  // namespace ts
