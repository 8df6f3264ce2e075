// Host side of include/stem_tree.h: argument checks and workspace sizes.  No allocation, no synchronisation.
#include "stem_decode_checks.h"
#include "stem_tree_common.h"

namespace stem {

static int check_tree_sizes(int32_t requests, int32_t tokens, int32_t max_new) {
    if (requests < 1 || tokens < 0 || max_new < 1) return STEM_ERR_INVALID_ARG;
    return requests > STEM_MAX_REQUESTS || max_new > STEM_MAX_TREE ? STEM_ERR_UNSUPPORTED : STEM_OK;
}

static int check_accept(const stem_accept_shape* s) {
    if (!s) return STEM_ERR_INVALID_ARG;
    if (const int st = check_tree_sizes(s->requests, s->tokens, s->max_new)) return st;
    if (s->num_pages < 1 || s->pages_per_request < 1 || (s->id_bits != 32 && s->id_bits != 64)) return STEM_ERR_INVALID_ARG;
    if (const int st = check_page_size(s->page_size)) return st;
    if ((int64_t)s->requests * s->pages_per_request > kInt32Max || (int64_t)s->num_pages * s->page_size > kInt32Max)
        return STEM_ERR_UNSUPPORTED;
    return STEM_OK;
}

static int check_tree_attn(const stem_prefix_shape* s) {
    if (const int st = check_prefix(s)) return st;
    return s->max_new > STEM_MAX_TREE ? STEM_ERR_UNSUPPORTED : STEM_OK;
}

}  // namespace stem

using namespace stem;

extern "C" {

int stem_tree_masks(const stem_tree_shape* shape, const int32_t* parents, const int32_t* lens, const int32_t* cu_new,
                    int32_t* positions, int64_t* masks, int32_t* status, void* hip_stream) {
    if (!shape) return STEM_ERR_INVALID_ARG;
    if (const int st = check_tree_sizes(shape->requests, shape->tokens, shape->max_new)) return st;
    if (shape->position_offset < 0) return STEM_ERR_INVALID_ARG;
    if (shape->tokens == 0) return STEM_OK;
    const void* needed[] = {parents, lens, cu_new, status};
    for (const void* p : needed)
        if (!p || !aligned(p, 4)) return STEM_ERR_INVALID_ARG;
    if (!aligned(positions, 4) || !masks || !aligned(masks, 8)) return STEM_ERR_INVALID_ARG;
    const TreeMasksCall call = {*shape, parents, lens, cu_new, positions, reinterpret_cast<uint64_t*>(masks), status};
    return launch_tree_masks(call, static_cast<hipStream_t>(hip_stream));
}

int stem_tree_attn_workspace_bytes(const stem_prefix_shape* shape, size_t* host_bytes) {
    if (const int st = check_tree_attn(shape)) return st;
    if (!host_bytes) return STEM_ERR_INVALID_ARG;
    PrefixPlan plan;
    if (const int st = prefix_plan(*shape, &plan, compute_units, true)) return st;
    *host_bytes = plan.bytes;
    return STEM_OK;
}

int stem_tree_attn(const stem_prefix_shape* shape, const void* q, const void* prefix_k, const void* prefix_v, const void* k_pages,
                   const void* v_pages, const int32_t* table, const int32_t* lens, const int32_t* cu_new, const int64_t* masks,
                   float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int st = check_tree_attn(shape)) return st;
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.f)) return STEM_ERR_INVALID_ARG;
    if (!cu_new || !aligned(cu_new, 4)) return STEM_ERR_INVALID_ARG;
    if (shape->tokens == 0) return STEM_OK;
    if (!masks || !aligned(masks, 8)) return STEM_ERR_INVALID_ARG;
    PrefixCall call = {*shape, {}, q, prefix_k, prefix_v, k_pages, v_pages, table, lens, cu_new, softmax_scale, out, lse, workspace};
    if (const int st = prepare_prefix(call, workspace_bytes, true)) return st;
    return launch_tree_attn(call, masks, static_cast<hipStream_t>(hip_stream));
}

int stem_tree_accept_workspace_bytes(const stem_accept_shape* shape, size_t* host_bytes) {
    if (const int st = check_accept(shape)) return st;
    if (!host_bytes) return STEM_ERR_INVALID_ARG;
    *host_bytes = 256;
    return STEM_OK;
}

int stem_tree_accept(const stem_accept_shape* shape, const int32_t* parents, const void* draft_ids, const void* target_ids,
                     const int32_t* cu_new, const int32_t* lens, const int32_t* ring_state, int32_t* ring, const int32_t* table,
                     int32_t* lens_out, int32_t* ring_state_out, int32_t* accepted, int32_t* path, void* next_ids, int32_t* status,
                     void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int st = check_accept(shape)) return st;
    const void* needed[] = {cu_new, lens, ring_state, ring, table, lens_out, ring_state_out, accepted, status};
    for (const void* p : needed)
        if (!p || !aligned(p, 4)) return STEM_ERR_INVALID_ARG;
    const uintptr_t id_bytes = shape->id_bits / 8;
    if (!next_ids || !aligned(next_ids, id_bytes)) return STEM_ERR_INVALID_ARG;
    if (shape->tokens > 0) {
        if (!parents || !path || !draft_ids || !target_ids) return STEM_ERR_INVALID_ARG;
        if (!aligned(parents, 4) || !aligned(path, 4) || !aligned(draft_ids, id_bytes) || !aligned(target_ids, id_bytes))
            return STEM_ERR_INVALID_ARG;
    }
    if (!workspace || !aligned(workspace, 16)) return STEM_ERR_INVALID_ARG;
    if (workspace_bytes < 256) return STEM_ERR_WORKSPACE;
    const AcceptCall call = {*shape, parents, draft_ids, target_ids, cu_new, lens, ring_state, table, ring, lens_out, ring_state_out,
                             accepted, path, status, next_ids};
    return launch_tree_accept(call, static_cast<hipStream_t>(hip_stream));
}

int stem_tree_commit(const stem_accept_shape* shape, const stem_pages* pages, int32_t dtype, int32_t num_kv_heads, int32_t head_dim,
                     const int32_t* path, const int32_t* slots, const int32_t* cu_new, void* k_pages, void* v_pages, void* hip_stream) {
    if (!shape || !pages) return STEM_ERR_INVALID_ARG;
    if (const int st = check_tree_sizes(shape->requests, shape->tokens, shape->max_new)) return st;
    if (dtype != STEM_BF16 && dtype != STEM_FP16 && dtype != STEM_FP32) return STEM_ERR_INVALID_ARG;
    if (num_kv_heads < 1 || head_dim < 1 || head_dim % 8) return STEM_ERR_INVALID_ARG;
    const int32_t bytes = dtype == STEM_FP32 ? 4 : 2;
    // (a token's rows of K and V are one line of a grid, in workgroups of 4 KiB)
    if (head_dim > STEM_MAX_HEAD_DIM || (int64_t)num_kv_heads * head_dim * bytes > 1 << 26) return STEM_ERR_UNSUPPORTED;
    if (const int st = check_pages(*pages, head_dim)) return st;
    if (!cu_new || !aligned(cu_new, 4)) return STEM_ERR_INVALID_ARG;
    if (shape->tokens == 0) return STEM_OK;
    if (!path || !aligned(path, 4) || !slots || !aligned(slots, 4)) return STEM_ERR_INVALID_ARG;
    if (pages->num_pages == 0) return STEM_OK;
    if (!k_pages || !aligned(k_pages, 16) || !v_pages || !aligned(v_pages, 16)) return STEM_ERR_INVALID_ARG;
    const CommitCall call = {*shape, *pages, num_kv_heads, head_dim * bytes, bytes, path, slots, cu_new, k_pages, v_pages};
    return launch_tree_commit(call, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
