// Internal declarations shared by the host API (stem_norm_api.cpp) and the kernels of include/stem_norm.h.
#pragma once

#include "stem_decode_common.h"
#include "stem_norm.h"

namespace stem {

struct NormCall {
    RotaryCall rotary;                   // backward: q, k, the gradients' places q_out, k_out (of q's and k's strides)
    stem_head_norm norm;
    const void *grad_q, *grad_k;         // of the shape's output strides
    float *q_weight_grad, *k_weight_grad;
    float* partial;                      // workspace: [norm_parts(shape)][2][head_dim], nullptr if no weight's gradient is wanted
};
int launch_norm_rotary(const NormCall& call, hipStream_t stream);
int launch_norm_rotary_backward(const NormCall& call, hipStream_t stream);

// Most workgroups of the backward pass, each with a sum of the weights' gradients over its tokens.  By the shape alone, so that a sum's order
// does not depend on the device: one for 10240 values of Q and K, but 256 if there are as many tokens, and four of four waves on each of
// 256 compute units at most.  Adding up costs 5 us with up to 256 of them, 7 with 512 and 9 with 1024; 256 / 512 / 1024, us in a graph: 40 heads
// of 128, 1024 tokens 18.5 / 16.8 / 18.8, 2048 30.7 / 23.2 / 23.4, 4096 52.9 / 35.0 / 31.5; 9 heads of 64, 4096 tokens 13.0 / 12.9 / 15.5.
constexpr int kNormMostParts = 1024;
inline int norm_parts(const stem_rotary_shape& s) {
    const int64_t values = (int64_t)s.tokens * (s.num_q_heads + s.num_kv_heads) * s.head_dim;
    int64_t parts = values / 10240;
    parts = parts < 256 ? 256 : parts > kNormMostParts ? kNormMostParts : parts;
    return parts < s.tokens ? (int)parts : s.tokens;
}

}  // namespace stem
