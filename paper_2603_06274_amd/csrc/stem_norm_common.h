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
    float* partial;                      // workspace: [norm_parts][2][head_dim], nullptr if no weight's gradient is wanted
};
int launch_norm_rotary(const NormCall& call, hipStream_t stream);
int launch_norm_rotary_backward(const NormCall& call, hipStream_t stream);

// Workgroups of the backward pass, each with tokens of its own and a sum of the weights' gradients over them.  By the tokens alone, so that a
// sum's order does not depend on the device: four workgroups of four waves on each of 256 compute units, of four tokens and more.
constexpr int kNormMostParts = 1024;
inline int norm_parts(int tokens) {
    const int parts = (tokens + 3) / 4;
    return parts < kNormMostParts ? parts : kNormMostParts;
}

}  // namespace stem
