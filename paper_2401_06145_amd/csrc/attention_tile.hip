// Attention with many queries per document over packed keys.
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_tile(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return attn::launch_tile<attn::kPacked>(a, p, dtype, s);
}

}  // namespace spc
