// Attention over pages of the rows' type: both forms.
#include "attention_rows.h"
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_pages(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  return p.rows ? attn::launch_rows<attn::kPages>(a, p, dtype, s) : attn::launch_tile<attn::kPages>(a, p, dtype, s);
}

}  // namespace spc
