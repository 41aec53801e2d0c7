// Attention over pages of 8 bits: both forms.
#include "attention_rows.h"
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_pages8(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return p.rows ? attn::launch_rows<attn::kPages8>(a, p, dtype, s) : attn::launch_tile<attn::kPages8>(a, p, dtype, s);
}

}  // namespace spc
