// Attention over pages of the rows' type: both forms.
#include "attention_rows.h"
#include "attention_tile.h"

namespace spc {

hipError_t launch_attention_pages(const AttnArgs& a, const AttnPlan& p, int dtype, hipStream_t s) {
  if (p.rows) return attn::launch_rows<attn::kPages>(a, p, dtype, s);
  const int d = a.d <= 32 ? 32 : a.d <= 64 ? 64 : a.d <= 96 ? 96 : a.d <= 128 ? 128 : 256;
  if (1 << a.shift < attn::rows_of_load(d, dtype == 0 ? 4 : 2, false)) return launch_attention_small(a, p, dtype, s);
  return attn::launch_tile<attn::kPages>(a, p, dtype, s);
}

}  // namespace spc
