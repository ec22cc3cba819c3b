// Attention over a paged KV cache, as tree_dev.h has it, whose scores are shaped
// (capped, biased by distance) and seen in spans or windows.
#include "tree_dev.h"

namespace vla {

hipError_t launch_score_attn(const TreeAttnDesc& d, hipStream_t st) { return launch<true>(d, st); }

}  // namespace vla
