// Attention over a paged KV cache, as tree_dev.h has it, with plain scores.
#include "tree_dev.h"

namespace vla {

size_t tree_attn_scratch(const TreeAttnDesc& d) {
  const size_t w = tree_wgs(d), rows = tile_rows(d), hdp = pad_hd(d.c.dtype, d.c.hd);
  return w * 32 + 2 * w * rows * (hdp + 2) * 4;
}

hipError_t launch_tree_attn(const TreeAttnDesc& d, hipStream_t st) { return launch<false>(d, st); }

}  // namespace vla
