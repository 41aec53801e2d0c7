// Attention of many queries over small pages of 8 bits.
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_small8(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return attn::launch_tile<attn::kSmall8>(a, p, dtype, s);
}

}  // namespace spc
