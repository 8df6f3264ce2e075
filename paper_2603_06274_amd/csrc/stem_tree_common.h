// Internal declarations shared by the host API (stem_tree_api.cpp) and the kernels of include/stem_tree.h.
#pragma once

#include "stem_decode_common.h"
#include "stem_tree.h"

namespace stem {

struct TreeMasksCall {
    stem_tree_shape shape;
    const int32_t *parents, *lens, *cu_new;
    int32_t* positions;
    uint64_t* masks;
    int32_t* status;
};
int launch_tree_masks(const TreeMasksCall& call, hipStream_t stream);

struct AcceptCall {
    stem_accept_shape shape;
    const int32_t* parents;
    const void *draft_ids, *target_ids;
    const int32_t *cu_new, *lens, *ring_state, *table;
    int32_t *ring, *lens_out, *ring_state_out, *accepted, *path, *status;
    void* next_ids;
};
int launch_tree_accept(const AcceptCall& call, hipStream_t stream);

struct CommitCall {
    stem_accept_shape shape;
    stem_pages pages;
    int32_t heads, row_bytes;            // of a token's K: heads of row_bytes bytes
    int32_t value_bytes;
    const int32_t *path, *slots, *cu_new;
    void *k_pages, *v_pages;
};
int launch_tree_commit(const CommitCall& call, hipStream_t stream);

int launch_tree_attn(const PrefixCall& call, const int64_t* masks, hipStream_t stream);

#if defined(__HIPCC__)
// First of request r's new tokens, and their number: those that are rows of the call.
__device__ __forceinline__ void tree_tokens(const int32_t* cu_new, int tokens, int r, int& first, int& n) {
    first = min(max(cu_new[r], 0), tokens);
    n = max(min(cu_new[r + 1], tokens) - first, 0);
}
#endif

}  // namespace stem
