// Cache attention for head_dim 256.
#include "kv_attention_inst.hpp"

namespace ts {
template void launch_kv_attention_t<256>(const KvAttnParams&, AttnTile, bool, int, hipStream_t);
}  // namespace ts
