// Attention with few queries per document over packed keys.
#include "attention_rows.h"

namespace spc {

hipError_t launch_attention_rows(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return attn::launch_rows<attn::kPacked>(a, p, dtype, s);
}

}  // namespace spc
