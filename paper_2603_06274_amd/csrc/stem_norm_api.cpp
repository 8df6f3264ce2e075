// Host side of include/stem_norm.h: argument checks and workspace sizes.  No allocation, no synchronisation.
#include "stem_decode_checks.h"
#include "stem_norm_common.h"

namespace stem {

static int check_norm(const stem_head_norm* n) {
    if (!n) return STEM_ERR_INVALID_ARG;
    if (n->weight_dtype != STEM_BF16 && n->weight_dtype != STEM_FP16 && n->weight_dtype != STEM_FP32) return STEM_ERR_INVALID_ARG;
    if (!aligned(n->q_weight, 16) || !aligned(n->k_weight, 16)) return STEM_ERR_INVALID_ARG;
    if (!std::isfinite(n->weight_offset) || !std::isnormal(n->eps) || !(n->eps > 0.f)) return STEM_ERR_INVALID_ARG;
    return STEM_OK;
}

static size_t partial_bytes(const stem_rotary_shape& s) { return align256(2 * sizeof(float) * (size_t)norm_parts(s) * s.head_dim); }

}  // namespace stem

using namespace stem;

extern "C" {

int stem_norm_rotary(const stem_rotary_shape* shape, const stem_head_norm* norm, const void* q, const void* k, const int32_t* positions,
                     const double* turns, float attention_factor, void* q_out, void* k_out, void* hip_stream) {
    if (const int st = check_rotary(shape, attention_factor)) return st;
    if (const int st = check_norm(norm)) return st;
    const stem_rotary_shape& s = *shape;
    if (s.num_kv_heads > 0 && !good_strides(s.k_out_stride_token, s.k_out_stride_head, s.head_dim)) return STEM_ERR_INVALID_ARG;
    if (s.tokens == 0) return STEM_OK;
    if (const int st = check_rotary_addresses(s, q, k, positions, turns, q_out)) return st;
    if (s.num_kv_heads > 0) {
        if (!k_out || !aligned(k_out, 16)) return STEM_ERR_INVALID_ARG;
        if (k == k_out && (s.k_stride_token != s.k_out_stride_token || s.k_stride_head != s.k_out_stride_head))
            return STEM_ERR_INVALID_ARG;
    }
    NormCall call = {};
    call.rotary = {s, q, k, nullptr, q_out, k_out, nullptr, positions, nullptr, turns, attention_factor, 0, {}};
    call.norm = *norm;
    return launch_norm_rotary(call, static_cast<hipStream_t>(hip_stream));
}

int stem_norm_rotary_append(const stem_rotary_shape* shape, const stem_head_norm* norm, const stem_pages* pages, const void* q,
                            const void* k, const void* v, const int32_t* positions, const int32_t* slots, const double* turns,
                            float attention_factor, void* q_out, void* k_pages, void* v_pages, void* hip_stream) {
    if (const int st = check_rotary(shape, attention_factor)) return st;
    if (const int st = check_norm(norm)) return st;
    const stem_rotary_shape& s = *shape;
    if (!pages || s.num_kv_heads == 0) return STEM_ERR_INVALID_ARG;
    if (const int st = check_pages(*pages, s.head_dim)) return st;
    if (s.tokens == 0) return STEM_OK;
    if (const int st = check_rotary_addresses(s, q, k, positions, turns, q_out)) return st;
    if (!slots || !aligned(slots, 4) || !v || !aligned(v, 16)) return STEM_ERR_INVALID_ARG;
    if (pages->num_pages == 0) return STEM_OK;
    if (!k_pages || !aligned(k_pages, 16) || !v_pages || !aligned(v_pages, 16)) return STEM_ERR_INVALID_ARG;
    NormCall call = {};
    call.rotary = {s, q, k, v, q_out, k_pages, v_pages, positions, slots, turns, attention_factor, 0, *pages};
    call.norm = *norm;
    return launch_norm_rotary(call, static_cast<hipStream_t>(hip_stream));
}

int stem_norm_rotary_backward_workspace_bytes(const stem_rotary_shape* shape, size_t* host_bytes) {
    if (const int st = check_rotary(shape, 1.f)) return st;
    if (!host_bytes) return STEM_ERR_INVALID_ARG;
    *host_bytes = partial_bytes(*shape);
    return STEM_OK;
}

int stem_norm_rotary_backward(const stem_rotary_shape* shape, const stem_head_norm* norm, const void* q, const void* k,
                              const int32_t* positions, const double* turns, float attention_factor, const void* grad_q,
                              const void* grad_k, void* q_grad, void* k_grad, float* q_weight_grad, float* k_weight_grad,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int st = check_rotary(shape, attention_factor)) return st;
    if (const int st = check_norm(norm)) return st;
    const stem_rotary_shape& s = *shape;
    if (s.num_kv_heads > 0 && !good_strides(s.k_out_stride_token, s.k_out_stride_head, s.head_dim)) return STEM_ERR_INVALID_ARG;
    if (!aligned(q_weight_grad, 4) || !aligned(k_weight_grad, 4)) return STEM_ERR_INVALID_ARG;
    if ((q_weight_grad && !norm->q_weight) || (k_weight_grad && !norm->k_weight)) return STEM_ERR_INVALID_ARG;
    if (s.tokens > 0) {
        if (!positions || !aligned(positions, 4) || !turns || !aligned(turns, 8)) return STEM_ERR_INVALID_ARG;
        auto good_rows = [](const void* x, const void* grad, const void* x_grad, bool same_strides) {
            return x && aligned(x, 16) && grad && aligned(grad, 16) && x_grad && aligned(x_grad, 16) && (grad != x_grad || same_strides);
        };
        if (s.num_q_heads > 0 && !good_rows(q, grad_q, q_grad, s.q_stride_token == s.q_out_stride_token && s.q_stride_head == s.q_out_stride_head))
            return STEM_ERR_INVALID_ARG;
        if (s.num_kv_heads > 0 && !good_rows(k, grad_k, k_grad, s.k_stride_token == s.k_out_stride_token && s.k_stride_head == s.k_out_stride_head))
            return STEM_ERR_INVALID_ARG;
    }
    const bool sums = q_weight_grad || k_weight_grad;
    if (sums && s.tokens > 0) {
        if (!workspace || !aligned(workspace, 16)) return STEM_ERR_INVALID_ARG;
        if (workspace_bytes < partial_bytes(s)) return STEM_ERR_WORKSPACE;
    }
    if (s.tokens == 0 && !sums) return STEM_OK;
    NormCall call = {};
    call.rotary = {s, q, k, nullptr, q_grad, k_grad, nullptr, positions, nullptr, turns, attention_factor, 1, {}};
    call.norm = *norm;
    call.grad_q = grad_q, call.grad_k = grad_k;
    call.q_weight_grad = q_weight_grad, call.k_weight_grad = k_weight_grad;
    call.partial = sums ? static_cast<float*>(workspace) : nullptr;
    return launch_norm_rotary_backward(call, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
