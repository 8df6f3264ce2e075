// The attention of drafted tokens, of which each sees its ancestors: as stem_prefix.hip has it but for the new tokens' masks.
#include "stem_prefix_kernels.h"
#include "stem_tree_common.h"

namespace stem {

int launch_tree_attn(const PrefixCall& c, const int64_t* masks, hipStream_t stream) { return launch_attn<true>(c, masks, stream); }

}  // namespace stem
