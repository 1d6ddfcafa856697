// Cache attention for head_dim 128.
#include "kv_attention_inst.hpp"

namespace ts {
template void launch_kv_attention_t<128>(const KvAttnParams&, AttnTile, bool, int, hipStream_t);
}  // namespace ts
