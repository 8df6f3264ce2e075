// Attention of many short rows to one long prefix that they share, and of each request's rows to its own pages behind it, causal among
// a request's new tokens.
#include "stem_prefix_kernels.h"

namespace stem {

int launch_prefix_attn(const PrefixCall& c, hipStream_t stream) { return launch_attn<false>(c, nullptr, stream); }

}  // namespace stem
