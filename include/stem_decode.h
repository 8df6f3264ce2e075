/*
 * stem_decode.h - C ABI of what stands before and behind Stem's pre-filling of a prompt, on the MI355X (gfx950):
 *
 *   stem_rotary          rotary positions of queries and keys, and the transposed map of their gradients;
 *   stem_block_table     the bookkeeping of a paged KV cache for one step of a batch of requests: pages handed out and taken
 *                        back, block tables, slots and positions of the new tokens, from the requests' lengths on the GPU;
 *   stem_rotary_append   the new tokens' queries and keys rotated, their keys and values written into the pages;
 *   stem_prefix_attn     attention of the new tokens to one long prefix that all requests share (read once for all of
 *                        them: K and V of the pre-filled prompt) and to each request's own pages behind it.
 *
 * The conventions of stem.h hold: status codes, device pointers unless a name starts with host_, buffers owned by the caller, no
 * allocation, no state, no synchronisation, all work on the caller's stream, arguments checked before anything is enqueued.
 * Every call may be captured into a HIP graph.  What the host has to know is a bound; lengths are read on the device, so
 * that a captured step can be replayed while they change.
 *
 *   - dtype is STEM_BF16 or STEM_FP16 (stem_rotary and stem_rotary_append also take STEM_FP32); all of a call's tensors of
 *     values share it.
 *   - With 0 tokens stem_rotary, stem_rotary_append and stem_prefix_attn do nothing, and their tensors' addresses are not looked at.
 *   - The last dimension is contiguous.  Strides are in elements and multiples of 8, base pointers of values 16-byte aligned,
 *     those of whole numbers aligned to their size.
 *   - Pages: k_pages and v_pages hold num_pages pages of page_size tokens of num_kv_heads rows of head_dim values, with
 *     strides between pages, tokens of a page and heads (the same for both).  page_size is 16, 32, 64, 128 or 256.  A slot is
 *     page * page_size + place in the page; num_pages * page_size <= 2^31 - 1.  A block table is int32
 *     [requests, pages_per_request]: entry j of a request's row is the page of its tokens j * page_size and on.
 */
#ifndef STEM_DECODE_H
#define STEM_DECODE_H

#include "stem.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STEM_BF16 0
#define STEM_FP16 1
#define STEM_FP32 2

#define STEM_ROTARY_HALF         0   /* pair i is (x[i], x[i + rotary_dim / 2])                          */
#define STEM_ROTARY_INTERLEAVED  1   /* pair i is (x[2 i], x[2 i + 1])                                   */

#define STEM_MAX_REQUESTS    65536
#define STEM_MAX_HEAD_DIM    1024    /* of stem_rotary and stem_rotary_append                            */

/* How frequencies are changed for contexts beyond the trained length.  With f(i) = theta^(-2 i / rotary_dim):
 *   NONE    f(i)
 *   LINEAR  f(i) / factor
 *   NTK     f(i) with theta * factor^(rotary_dim / (rotary_dim - 2)) for theta       (rotary_dim > 2)
 *   YARN    f(i) (1 - x) + f(i) / factor * x, x = clamp((i - lo) / max(hi - lo, 0.001), 0, 1), where
 *           dim(n) = rotary_dim ln(trained_length / (2 pi n)) / (2 ln theta) is the pair that turns n times within the trained
 *           length, lo = max(floor(dim(high)), 0) and hi = min(ceil(dim(low)), rotary_dim - 1)   (arXiv 2309.00071)
 *   BANDS   f(i) y + f(i) / factor (1 - y), y = clamp((trained_length f(i) / (2 pi) - low) / (high - low), 0, 1)
 * low < high are numbers of turns within the trained length (1 and 32 with YARN, 1 and 4 with BANDS, where a model says nothing else). */
#define STEM_ROTARY_NONE    0
#define STEM_ROTARY_LINEAR  1
#define STEM_ROTARY_NTK     2
#define STEM_ROTARY_YARN    3
#define STEM_ROTARY_BANDS   4

typedef struct stem_rotary_scaling {
    int32_t kind;                    /* STEM_ROTARY_NONE .. STEM_ROTARY_BANDS                            */
    double factor;                   /* >= 1: how many times the trained length (not used by NONE)       */
    double trained_length;           /* > 0, tokens (YARN, BANDS)                                        */
    double low, high;                /* 0 < low < high (YARN, BANDS)                                     */
} stem_rotary_scaling;

/* Host: turns per position, f(i) / (2 pi), of the rotary_dim / 2 pairs, and the factor that the method puts on rotated
 * values (YARN: 0.1 ln(factor) + 1, else 1).  host_scaling NULL means NONE.  theta > 1.  Copy host_turns to the device for
 * the calls below. */
int stem_rotary_frequencies(int32_t rotary_dim, double theta, const stem_rotary_scaling* host_scaling,
                            double* host_turns, double* host_attention_factor);

typedef struct stem_rotary_shape {
    int32_t dtype;                   /* STEM_BF16, STEM_FP16 or STEM_FP32                                */
    int32_t tokens;                  /* rows of Q and K; >= 0                                            */
    int32_t num_q_heads;             /* >= 0; 0: no Q                                                    */
    int32_t num_kv_heads;            /* >= 0; 0: no K (not both 0)                                       */
    int32_t head_dim;                /* multiple of 8, <= STEM_MAX_HEAD_DIM                              */
    int32_t rotary_dim;              /* even, 2 .. head_dim: the first rotary_dim values of a head turn  */
    int32_t layout;                  /* STEM_ROTARY_HALF or STEM_ROTARY_INTERLEAVED                      */
    int64_t q_stride_token, q_stride_head;
    int64_t k_stride_token, k_stride_head;          /* of K, and of V in stem_rotary_append              */
    int64_t q_out_stride_token, q_out_stride_head;
    int64_t k_out_stride_token, k_out_stride_head;  /* not read by stem_rotary_append                    */
} stem_rotary_shape;

/*
 * Rotary positions.  For every token t, head and pair i with values (x1, x2), in fp32 and rounded once:
 *   a = 2 pi * positions[t] * turns[i]          (the product in 64 bits, its whole turns dropped)
 *   y1 = c x1 - s x2,  y2 = c x2 + s x1,  c = attention_factor cos a,  s = attention_factor sin a
 * and y = x for the values from rotary_dim on.  With backward = 1, s is negated: the transposed map, which takes the gradients
 * of y to those of x (and, if attention_factor is 1, the inverse).
 * positions is int32 [tokens] (any sign), turns fp64 [rotary_dim / 2].  q_out may be q and k_out may be k, with the same
 * strides; otherwise an output shares no value with an input or the other output.  STEM_ERR_UNSUPPORTED from 2^24 tokens or
 * beyond 65535 heads in all.
 */
int stem_rotary(const stem_rotary_shape* shape, const void* q, const void* k, const int32_t* positions,
                const double* turns, float attention_factor, int32_t backward, void* q_out, void* k_out,
                void* hip_stream);

typedef struct stem_table_shape {
    int32_t requests;                /* 1 .. STEM_MAX_REQUESTS                                           */
    int32_t page_size;
    int32_t num_pages;               /* pages of the cache and entries of the ring, >= 1                 */
    int32_t pages_per_request;       /* entries of a table row, >= 1                                     */
    int32_t token_capacity;          /* entries of positions and slots, >= 0                             */
    int32_t position_offset;         /* position of a request's first own token (a shared prefix's length), >= 0 */
    int32_t max_new;                 /* most new tokens of a request that the step's attention takes; 0: any number */
} stem_table_shape;

int stem_block_table_workspace_bytes(const stem_table_shape* shape, size_t* host_bytes);

/*
 * One step's bookkeeping.  Request r has past_lens[r] tokens in its pages; new_lens[r] >= 0 more come (new_lens NULL: one for
 * every request), and new_lens[r] < 0 says that the request has finished.
 *   - The free pages are a ring: int32 ring[num_pages], of which the ring_state[1] entries from ring_state[0] on (modulo
 *     num_pages) are free pages.  Requests in order get the pages that they lack, the ring's first entries first, into their
 *     rows' entries ceil(past / page_size) and on.  The ceil(past / page_size) pages of a finished request go behind the ring's
 *     last entry, in the order of requests and rows; they are handed out from the next call on, and the row keeps its
 *     entries (which mean nothing any more).
 *   - lens[r] = past + new tokens (0 for a finished request); cu_new int32 [requests + 1] the sums of the new tokens before
 *     each request; for the new token t, number i of request r: positions[t] = position_offset + past_lens[r] + i and slots[t] its
 *     slot (-1 if the table's or ring's page is not one of the cache's).  From cu_new[requests] on (a padded batch)
 *     positions are 0 and slots -1.  ring_state_out is the ring's new state.
 *   - lens may be past_lens and ring_state_out may be ring_state; nothing else may overlap.
 *   - status int32 [4]: pages that are lacking; requests whose past length is negative, whose tokens a row cannot hold or that have more
 *     than max_new new ones; tokens beyond token_capacity; pages given back that the ring has no room for (1 at least if ring_state is no state).  (Each
 *     at most 2^31 - 1.)  Unless all are 0 the step is refused: table and ring are left as they are, lens and ring_state_out say what
 *     was, cu_new and positions are 0, slots -1.
 * workspace: 16-byte aligned, of stem_block_table_workspace_bytes, this call's alone until its work has finished.
 * STEM_ERR_UNSUPPORTED if requests * pages_per_request, num_pages * page_size or position_offset + pages_per_request * page_size
 * exceeds 2^31 - 1.
 */
int stem_block_table(const stem_table_shape* shape, const int32_t* past_lens, const int32_t* new_lens,
                     const int32_t* ring_state, int32_t* ring, int32_t* table, int32_t* lens, int32_t* ring_state_out,
                     int32_t* cu_new, int32_t* positions, int32_t* slots, int32_t* status, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

typedef struct stem_pages {
    int32_t page_size;
    int32_t num_pages;               /* >= 0                                                             */
    int64_t stride_page, stride_token, stride_head;
} stem_pages;

/*
 * stem_rotary of Q and K (forward), with K's rotated rows and V's rows written to k_pages and v_pages at the tokens' slots
 * (int32 [tokens]).  A token whose slot is not one of the cache's (-1) is skipped: none of its rows is written, of Q neither.  No
 * slot may occur twice.  Q may be absent (num_q_heads 0), K and V may not.  V has K's strides.
 */
int stem_rotary_append(const stem_rotary_shape* shape, const stem_pages* pages, const void* q, const void* k,
                       const void* v, const int32_t* positions, const int32_t* slots, const double* turns,
                       float attention_factor, void* q_out, void* k_pages, void* v_pages, void* hip_stream);

typedef struct stem_prefix_shape {
    int32_t dtype;                   /* STEM_BF16 or STEM_FP16                                           */
    int32_t num_q_heads;             /* Hq                                                               */
    int32_t num_kv_heads;            /* Hkv, divides Hq                                                  */
    int32_t head_dim;                /* 64, 128 or 256                                                   */
    int32_t requests;                /* 1 .. STEM_MAX_REQUESTS                                           */
    int32_t tokens;                  /* rows of Q, O; >= 0                                               */
    int32_t max_new;                 /* most new tokens of a request, >= 1                               */
    int32_t prefix_len;              /* >= 0                                                             */
    int32_t max_suffix;              /* most tokens that a request has in its pages, 0 .. pages_per_request * page_size,
                                        and at most 2^31 - 2^14 (beyond: STEM_ERR_UNSUPPORTED)           */
    int32_t pages_per_request;       /* entries of a table row                                           */
    int64_t q_stride_token, q_stride_head;          /* of Q and O                                        */
    int64_t prefix_stride_token, prefix_stride_head;/* of prefix_k and prefix_v                          */
    stem_pages pages;
} stem_prefix_shape;

int stem_prefix_attn_workspace_bytes(const stem_prefix_shape* shape, size_t* host_bytes);

/*
 * Exact softmax attention of every request's new tokens to the shared prefix and to the request's own tokens:
 *   out[t, h, :] = sum_u softmax_u( softmax_scale * <Q[t, h], K[u, g]> ) V[u, g],   g = h / (Hq / Hkv)
 * over the prefix_len rows of prefix_k, prefix_v [prefix_len, Hkv, d] and the request's rows j in the pages with
 * j <= lens[r] - n + i, where t is number i of the n new tokens of request r (which stand at the end of its lens[r] tokens; n
 * counts the rows that there are).
 *   - lens is int32 [requests], table int32 [requests, pages_per_request], cu_new int32 [requests + 1]: request r's new tokens are
 *     the rows cu_new[r] .. cu_new[r + 1] - 1 of Q and O, as far as there are such rows.  cu_new ascends (where it does not, rows of
 *     O and lse hold nothing defined); NULL: one token each, then tokens = requests.  Rows of no request are left as they were, in O
 *     and in lse, and so are a request's rows from max_new on.  max_new may be as large as a request's tokens can get: the work goes
 *     by the rows that there are.
 *   - lens outside 0 .. max_suffix count as the nearer of the two.  Rows in pages that are not the cache's (a table entry outside
 *     0 .. num_pages - 1) contribute nothing, and nothing is read there; nor is anything behind a request's last token.
 *   - A row that sees no key at all gives zeros, lse -inf.
 *   - 16-bit inputs, matrix products with fp32 accumulation (probabilities rounded to the inputs' type), fp32 softmax, row sums of
 *     the unrounded probabilities.  lse, fp32 [Hq, tokens], may be NULL: log sum_u exp(softmax_scale * <Q, K>).
 *   - Q, K and V are expected to hold finite values.  An inf or NaN in them spreads as in stem_sparse_attn: to the rows that see it,
 *     and a value of a new token also to its own request's earlier new tokens.  Requests do not reach each other.
 *   - The same inputs give the same bits; what the rest of the batch holds has no influence on a row beyond rounding.
 * workspace: 16-byte aligned, of stem_prefix_attn_workspace_bytes (which depends on the current device), this call's alone until its work has
 * finished.  prefix_k and prefix_v may be NULL if prefix_len is 0; k_pages, v_pages, table and lens if max_suffix is 0.
 * STEM_ERR_UNSUPPORTED, from both functions, if 16 rows of a page or 128 of the prefix span 2 GiB or more, if tokens * num_q_heads or
 * max_new * num_q_heads exceeds 2^31 - 1, or if a launch would have about 2^31 workgroups (tokens * num_q_heads beyond
 * 2^31 - 2^20, or requests * num_kv_heads that are as many).
 */
int stem_prefix_attn(const stem_prefix_shape* shape, const void* q, const void* prefix_k, const void* prefix_v,
                     const void* k_pages, const void* v_pages, const int32_t* table, const int32_t* lens,
                     const int32_t* cu_new, float softmax_scale, void* out, float* lse, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* STEM_DECODE_H */
