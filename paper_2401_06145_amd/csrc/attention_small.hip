// Attention of many queries over small pages of the rows' type.
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_small(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return attn::launch_tile<attn::kSmall>(a, p, dtype, s);
}

}  // namespace spc
