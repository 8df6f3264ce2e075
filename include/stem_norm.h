/*
 * stem_norm.h - C ABI of queries and keys that are normalised head by head before their rotary positions, on the MI355X (gfx950):
 *
 *   stem_norm_rotary            norm, weights and rotation in one pass;
 *   stem_norm_rotary_append     the same for new tokens whose keys and values go to their pages;
 *   stem_norm_rotary_backward   the gradients of the values and of the weights.
 *
 * The conventions of stem.h and stem_decode.h hold: status codes, device pointers unless a name starts with host_, buffers owned by the
 * caller, no allocation, no state, no synchronisation, all work on the caller's stream, arguments checked before anything is enqueued.
 * Every call may be captured into a HIP graph.  Shapes, layouts, positions and turns are those of stem_rotary.
 */
#ifndef STEM_NORM_H
#define STEM_NORM_H

#include "stem_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct stem_head_norm {
    const void* q_weight;            /* [head_dim], of weight_dtype, one for all heads of Q; NULL: none  */
    const void* k_weight;            /* the same for K                                                   */
    int32_t weight_dtype;            /* STEM_BF16, STEM_FP16 or STEM_FP32, whatever the values' type     */
    float weight_offset;             /* added to the weights (1 where they are kept as what they differ from 1 by) */
    float eps;                       /* a normal number > 0                                              */
} stem_head_norm;

/*
 * For every token, head and value i of the head, in fp32 and rounded once, at the end:
 *   n[i] = x[i] r (weight[i] + weight_offset),  r = 1 / sqrt(mean_j x[j]^2 + eps)     (n = x r where there is no weight)
 *   y = n, its first rotary_dim values turned as stem_rotary turns them.
 * q_out may be q and k_out may be k, with the same strides; otherwise an output shares no value with an input or the other output.
 * The mean of a head's squares has to be within fp32 (values of about 10^19 and beyond give what inf gives).  An inf or NaN
 * in a head makes values of that head NaN or 0, and no other's.  With 0 tokens nothing is done.  Limits as for stem_rotary.
 */
int stem_norm_rotary(const stem_rotary_shape* shape, const stem_head_norm* norm, const void* q, const void* k, const int32_t* positions,
                     const double* turns, float attention_factor, void* q_out, void* k_out, void* hip_stream);

/*
 * stem_rotary_append with heads of Q and K normalised first.  V's rows go to their pages as they are.
 */
int stem_norm_rotary_append(const stem_rotary_shape* shape, const stem_head_norm* norm, const stem_pages* pages, const void* q,
                            const void* k, const void* v, const int32_t* positions, const int32_t* slots, const double* turns,
                            float attention_factor, void* q_out, void* k_pages, void* v_pages, void* hip_stream);

int stem_norm_rotary_backward_workspace_bytes(const stem_rotary_shape* shape, size_t* host_bytes);

/*
 * The gradients of stem_norm_rotary's inputs from grad_q, grad_k, those of its outputs (of the outputs' strides, the values' type).  With g
 * the gradient turned back and u = x r:
 *   dweight[i] = sum over tokens and heads of g[i] u[i]          fp32 [head_dim], the same bits for the same inputs
 *   dx[i] = r (h[i] - u[i] mean_j(h[j] u[j])),  h[i] = g[i] (weight[i] + weight_offset)
 * q_grad and k_grad have q's and k's strides and may be q and k, or grad_q and grad_k if those have the same strides; otherwise an output
 * shares no value with an input or another output.  q_weight_grad and k_weight_grad may be NULL (not wanted); they have to be where there
 * is no such weight.  With 0 tokens they become 0 and nothing else is done.
 * workspace: 16-byte aligned, of stem_norm_rotary_backward_workspace_bytes, this call's alone until its work has finished; may be NULL if
 * neither weight's gradient is wanted.
 */
int stem_norm_rotary_backward(const stem_rotary_shape* shape, const stem_head_norm* norm, const void* q, const void* k,
                              const int32_t* positions, const double* turns, float attention_factor, const void* grad_q,
                              const void* grad_k, void* q_grad, void* k_grad, float* q_weight_grad, float* k_weight_grad,
                              void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* STEM_NORM_H */
