// Checks of arguments that the host APIs of include/stem_decode.h, include/stem_norm.h and include/stem_tree.h share.
#pragma once

#include <cmath>

#include "stem_decode_common.h"

namespace stem {

constexpr int64_t kInt32Max = 0x7fffffff;
constexpr int64_t kMostGroups = kInt32Max - (1 << 20);   // of a launch, whose grid is rounded up to lines of 2^20

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Strides of [tokens, heads, head_dim] rows.
inline bool good_strides(int64_t token, int64_t head, int32_t head_dim) {
    return token >= head_dim && head >= head_dim && !((token | head) & 7);
}

inline int check_page_size(int32_t n) {
    if (n <= 0) return STEM_ERR_INVALID_ARG;
    return n == 16 || n == 32 || n == 64 || n == 128 || n == 256 ? STEM_OK : STEM_ERR_UNSUPPORTED;
}

inline int check_pages(const stem_pages& p, int32_t head_dim) {
    if (const int st = check_page_size(p.page_size)) return st;
    if (p.num_pages < 0) return STEM_ERR_INVALID_ARG;
    if ((int64_t)p.num_pages * p.page_size > kInt32Max) return STEM_ERR_UNSUPPORTED;
    if (!good_strides(p.stride_token, p.stride_head, head_dim) || p.stride_page < head_dim || (p.stride_page & 7))
        return STEM_ERR_INVALID_ARG;
    return STEM_OK;
}

inline int check_rotary(const stem_rotary_shape* s, float factor) {
    if (!s) return STEM_ERR_INVALID_ARG;
    if (s->dtype != STEM_BF16 && s->dtype != STEM_FP16 && s->dtype != STEM_FP32) return STEM_ERR_INVALID_ARG;
    if (s->tokens < 0 || s->num_q_heads < 0 || s->num_kv_heads < 0) return STEM_ERR_INVALID_ARG;
    if (s->tokens >= 1 << 24 || (int64_t)s->num_q_heads + 2 * (int64_t)s->num_kv_heads > 65535) return STEM_ERR_UNSUPPORTED;
    if (s->num_q_heads + s->num_kv_heads == 0 || s->head_dim <= 0 || s->head_dim % 8) return STEM_ERR_INVALID_ARG;
    if (s->head_dim > STEM_MAX_HEAD_DIM) return STEM_ERR_UNSUPPORTED;
    if (s->rotary_dim < 2 || s->rotary_dim % 2 || s->rotary_dim > s->head_dim) return STEM_ERR_INVALID_ARG;
    if (s->layout != STEM_ROTARY_HALF && s->layout != STEM_ROTARY_INTERLEAVED) return STEM_ERR_INVALID_ARG;
    if (!std::isfinite(factor)) return STEM_ERR_INVALID_ARG;
    if (s->num_q_heads > 0) {
        if (!good_strides(s->q_stride_token, s->q_stride_head, s->head_dim)) return STEM_ERR_INVALID_ARG;
        if (!good_strides(s->q_out_stride_token, s->q_out_stride_head, s->head_dim)) return STEM_ERR_INVALID_ARG;
    }
    if (s->num_kv_heads > 0 && !good_strides(s->k_stride_token, s->k_stride_head, s->head_dim)) return STEM_ERR_INVALID_ARG;
    return STEM_OK;
}

// Of a call that has tokens (an empty tensor has no address).
inline int check_rotary_addresses(const stem_rotary_shape& s, const void* q, const void* k, const int32_t* positions,
                                  const double* turns, const void* q_out) {
    if (!positions || !aligned(positions, 4) || !turns || !aligned(turns, 8)) return STEM_ERR_INVALID_ARG;
    if (s.num_q_heads > 0) {
        if (!q || !aligned(q, 16) || !q_out || !aligned(q_out, 16)) return STEM_ERR_INVALID_ARG;
        if (q == q_out && (s.q_stride_token != s.q_out_stride_token || s.q_stride_head != s.q_out_stride_head))
            return STEM_ERR_INVALID_ARG;
    }
    if (s.num_kv_heads > 0 && (!k || !aligned(k, 16))) return STEM_ERR_INVALID_ARG;
    return STEM_OK;
}

}  // namespace stem
