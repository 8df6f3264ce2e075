/*
 * stem_tree.h - C ABI of decoding steps whose new tokens are drafts that form a tree, on the MI355X (gfx950):
 *
 *   stem_tree_masks     which of its request's new tokens each of them sees (its ancestors and itself), and its position;
 *   stem_tree_attn      attention of the new tokens to a shared prefix, to their requests' pages, and to the new tokens that they see;
 *   stem_tree_accept    which drafts the model's own choices confirm, the requests' lengths without the others, and the pages that go back;
 *   stem_tree_commit    the confirmed tokens' keys and values, one behind the other in the pages.
 *
 * A step of them: stem_block_table, stem_tree_masks, stem_rotary_append (or stem_norm_rotary_append), stem_tree_attn, the model's choice
 * behind every token, stem_tree_accept, stem_tree_commit.  The conventions of stem.h and stem_decode.h hold: status codes, device
 * pointers unless a name starts with host_, buffers owned by the caller, no allocation, no state, no synchronisation, all work on the
 * caller's stream, arguments checked before anything is enqueued.  Every call may be captured into a HIP graph; lengths are read on the
 * device.
 *
 *   - Request r's new tokens are the rows cu_new[r] .. cu_new[r + 1] - 1, as far as there are such rows (of `tokens`), and stand at the
 *     end of its lens[r] tokens; n is their number.  cu_new int32 [requests + 1] ascends.
 *   - parents int32 [tokens]: the number among its request's new tokens of the one that a token was drafted behind, less than its own
 *     number; -1 (or what is no such number): it stands behind the request's tokens of earlier steps.
 *   - masks int64 [tokens, words], words = ceil(max_new / 64): bit j % 64 of word j / 64 says that a token sees the new token number j of
 *     its request.  max_new is at most STEM_MAX_TREE.
 */
#ifndef STEM_TREE_H
#define STEM_TREE_H

#include "stem_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STEM_MAX_TREE  1024

typedef struct stem_tree_shape {
    int32_t requests;                /* 1 .. STEM_MAX_REQUESTS                                           */
    int32_t tokens;                  /* rows of the step's tensors, >= 0                                 */
    int32_t max_new;                 /* most new tokens of a request, 1 .. STEM_MAX_TREE                 */
    int32_t position_offset;         /* position of a request's first own token, >= 0                    */
} stem_tree_shape;

/*
 * masks: every new token sees itself and its ancestors.  positions[t] = position_offset + lens[r] - n + number of t's ancestors; positions may
 * be NULL.  Rows of no request, and a request's rows from max_new on, are left as they were.
 * status int32 [1] grows by the number of tokens whose parent is neither -1 nor a number less than their own (they are taken to have none),
 * and of those from max_new on; the caller clears it.
 */
int stem_tree_masks(const stem_tree_shape* shape, const int32_t* parents, const int32_t* lens, const int32_t* cu_new,
                    int32_t* positions, int64_t* masks, int32_t* status, void* hip_stream);

int stem_tree_attn_workspace_bytes(const stem_prefix_shape* shape, size_t* host_bytes);

/*
 * stem_prefix_attn, but that new token i of a request sees, of its n new tokens, those whose bits are set in its row of masks (any
 * bits: a tree's, or none at all), not those up to itself.  Besides:
 *   - max_new is at most STEM_MAX_TREE (STEM_ERR_UNSUPPORTED).  cu_new may not be NULL.  A request's rows from max_new on are left as they were;
 *     new tokens from number 64 * words on are seen by nobody.
 *   - An inf or NaN in a new token's value is in the results of the rows that see it, an infinite one as itself, however small its weight, and in
 *     no others'; one in its key counts in the scores of the rows that see it, and in no others'.  (In prefix and earlier tokens: in those of all
 *     rows that see them.)
 */
int stem_tree_attn(const stem_prefix_shape* shape, const void* q, const void* prefix_k, const void* prefix_v, const void* k_pages,
                   const void* v_pages, const int32_t* table, const int32_t* lens, const int32_t* cu_new, const int64_t* masks,
                   float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

typedef struct stem_accept_shape {
    int32_t requests;                /* 1 .. STEM_MAX_REQUESTS                                           */
    int32_t tokens;                  /* rows of the step's tensors, >= 0                                 */
    int32_t max_new;                 /* most new tokens of a request, 1 .. STEM_MAX_TREE                 */
    int32_t page_size;
    int32_t num_pages;               /* pages of the cache and entries of the ring, >= 1                 */
    int32_t pages_per_request;       /* entries of a table row, >= 1                                     */
    int32_t id_bits;                 /* 32 or 64: draft_ids, target_ids and next_ids are int32 or int64  */
} stem_accept_shape;

int stem_tree_accept_workspace_bytes(const stem_accept_shape* shape, size_t* host_bytes);

/*
 * What a step keeps.  draft_ids[t] is the token at row t, target_ids[t] what the model chooses behind it.  Of each request with new tokens,
 * number 0 is kept (it was chosen before the step); behind a kept token c the lowest-numbered child of c whose draft is target_ids[c], if
 * there is one, and so on.
 *   - accepted[r] = number of kept tokens (0 without new ones); path int32 [tokens]: path[cu_new[r] + k] the number of the k-th kept
 *     one, -1 from accepted[r] on; next_ids[r] = target_ids of the last kept one (-1 without): the token to begin the next step with.
 *   - lens_out[r] = lens[r] - n + accepted[r].  The pages of table row r behind its last kept token, entries ceil(lens_out / page_size)
 *     to ceil(lens / page_size) - 1, go behind the ring's last entry (the ring as stem_block_table has it), in the order of requests and
 *     entries; the table keeps them.
 *   - lens_out may be lens and ring_state_out may be ring_state; nothing else may overlap.
 *   - status int32 [2]: requests with more than max_new new tokens, fewer tokens than new ones or more than a table row holds; pages given
 *     back that the ring has no room for (1 at least if ring_state is no state).  Unless both are 0 the step is refused: the ring is left
 *     as it is, lens_out and ring_state_out say what was, accepted is 0, path and next_ids -1.
 *   - Entries of path that are no request's are left as they were.
 * workspace: 16-byte aligned, of stem_tree_accept_workspace_bytes.  Nothing is written there now, so calls may share one, and any other's.
 * STEM_ERR_UNSUPPORTED if requests * pages_per_request or num_pages * page_size exceeds 2^31 - 1.
 */
int stem_tree_accept(const stem_accept_shape* shape, const int32_t* parents, const void* draft_ids, const void* target_ids,
                     const int32_t* cu_new, const int32_t* lens, const int32_t* ring_state, int32_t* ring, const int32_t* table,
                     int32_t* lens_out, int32_t* ring_state_out, int32_t* accepted, int32_t* path, void* next_ids, int32_t* status,
                     void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Rows of K and V of kept tokens move up: for k = 0, 1, .. the row at slots[cu_new[r] + path[cu_new[r] + k]] goes to slots[cu_new[r] + k],
 * for each request until its path's first entry that is no number of a new token.  path ascends strictly.  slots are those of the step's
 * new tokens as stem_block_table left them (before lens_out took lens' place); tokens without a place (-1) stay out.  Of the shape,
 * requests, tokens and max_new count.  The pages have num_kv_heads heads of head_dim values (a multiple of 8, at most STEM_MAX_HEAD_DIM) of dtype,
 * 64 MiB per token at most (STEM_ERR_UNSUPPORTED).
 */
int stem_tree_commit(const stem_accept_shape* shape, const stem_pages* pages, int32_t dtype, int32_t num_kv_heads, int32_t head_dim,
                     const int32_t* path, const int32_t* slots, const int32_t* cu_new, void* k_pages, void* v_pages, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* STEM_TREE_H */
