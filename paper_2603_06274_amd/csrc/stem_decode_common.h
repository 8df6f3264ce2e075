// Internal declarations shared by the host API (stem_decode_api.cpp) and the kernels of include/stem_decode.h.
#pragma once

#include "stem_common.h"
#include "stem_decode.h"

namespace stem {

// --- rotary positions ---------------------------------------------------------------------------------------

struct RotaryCall {
    stem_rotary_shape shape;
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out;         // k_out and v_out: the pages, if `pages` says so
    const int32_t* positions;
    const int32_t* slots;                // nullptr: no pages
    const double* turns;
    float factor;
    int32_t backward;
    stem_pages pages;
};
int launch_rotary(const RotaryCall& call, hipStream_t stream);

// --- block tables -------------------------------------------------------------------------------------------

// What the first of two launches leaves for the second: sums over the requests before each, and the ring's state.
struct TableWorkspace {
    size_t pages_before, back_before, ring, total;
};
TableWorkspace table_workspace(int32_t requests);

struct TableCall {
    stem_table_shape shape;
    const int32_t *past_lens, *new_lens, *ring_state;
    int32_t *ring, *table, *lens, *ring_state_out, *cu_new, *positions, *slots, *status;
    int32_t *pages_before, *back_before, *ring_then;   // workspace
};
int launch_block_table(const TableCall& call, hipStream_t stream);

// --- attention to a shared prefix ---------------------------------------------------------------------------

// How a call is split over workgroups.  Rows are (token, query head of the group) per KV head.
struct PrefixPlan {
    int32_t row_tile;          // rows of a workgroup in the prefix, and per request in its pages
    int32_t row_tiles;         // of the prefix: ceil(tokens * G / row_tile)
    int32_t prefix_splits;     // 0 if there is no prefix
    int32_t split_keys;        // keys per split (a multiple of 32), the last may be shorter
    int32_t suffix_row_tile;
    int32_t suffix_row_tiles;  // per request: ceil(max_new * G / suffix_row_tile)
    int32_t suffix_splits;     // 0 if there are no pages
    // Pairs (request, row tile) per KV head and part of the own keys: suffix_row_tiles for every request or, where that is more,
    // rows / tile for all together and one for each (own_by_rows: slot_before says whose a slot is).
    int64_t own_slots;
    bool own_by_rows;
    // Rows (token, head) that are joined: max_new tokens of every request or, where that is more, the call's tokens (join_by_rows).
    int64_t join_rows;
    bool join_by_rows;
    int64_t prefix_groups, groups;   // workgroups of the prefix, and with those of the own keys
    bool small;                // all of a request's keys by one workgroup per KV head, no parts
    size_t partial_ml;         // byte offset in the workspace: (maximum, sum) of every partial result
    size_t bytes;
};
// units: where the number of compute units comes from
int prefix_plan(const stem_prefix_shape& s, PrefixPlan* plan, int (*units)() = compute_units);

struct PrefixCall {
    stem_prefix_shape shape;
    PrefixPlan plan;
    const void *q, *prefix_k, *prefix_v, *k_pages, *v_pages;
    const int32_t *table, *lens, *cu_new;
    float softmax_scale;
    void* out;
    float* lse;
    void* workspace;
};
int launch_prefix_attn(const PrefixCall& call, hipStream_t stream);

// Most own tokens of a request.  The kernel counts keys in 32 bits: parts are rounded up to 128 keys and there are 64 at most, and a
// walk looks three tiles of at most 256 keys past its last one, so that nothing that it forms passes 2^31.
constexpr int32_t kMaxSuffix = 0x7fffffff - 0x3fff;

// Row tiles' slots before those of request r, whose first row is `row`: whole tiles before the row and one for each request
// before, which is at least as many as these have tiles.  (floor(b / t) + 1 - floor(a / t) is whole and more than (b - a) / t.)
__host__ __device__ inline int64_t slot_before(int r, int64_t row, int tile) { return row / tile + r; }

// Keys of a part of a request's own `len`, of which there are at most `splits`: whole 128s, so that short ones use few parts.  The
// kernel that computes partial results and the one that joins them both ask here.
__host__ __device__ inline int suffix_split_keys(int len, int splits) {
    const uint32_t each = ((uint32_t)len + (uint32_t)splits - 1) / (uint32_t)splits;
    return (int)((each + 127) & ~127u);
}
// and the number of parts that are not empty
__host__ __device__ inline int suffix_parts(int len, int splits) {
    return len > 0 ? (int)((uint32_t)(len - 1) / (uint32_t)suffix_split_keys(len, splits)) + 1 : 0;
}

}  // namespace stem
