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

// How pairs lie in a lane's values: neighbours; the two chunks; or one of them in another lane.
enum Pairs { kNeighbours, kHalves, kAcross };

// Where a head's values are: the registers of 2^lane_bits lanes, of which `items` have two chunks of 16 bytes each, if it is not too long.
struct HeadLayout {
    Pairs pairs;
    bool in_registers;
    int32_t items, turning, lane_bits;                 // turning: of kHalves, items that turn
    int32_t padded;                                    // places of a token's (cos, sin) in LDS
};
inline HeadLayout head_layout(const stem_rotary_shape& s) {
    const int W = s.dtype == STEM_FP32 ? 4 : 8, half = s.rotary_dim / 2;
    HeadLayout l;
    l.pairs = s.layout != STEM_ROTARY_HALF ? kNeighbours : half % W == 0 ? kHalves : kAcross;
    l.turning = half / W;                              // (whole chunks of either half)
    l.items = (s.head_dim + 2 * W - 1) / (2 * W);
    l.in_registers = l.items <= 64;
    l.padded = !l.in_registers ? half : l.pairs == kAcross ? 2 * l.items * (W + 1) : (half + W / 2 - 1) / (W / 2) * (W / 2);   // (of whole chunks)
    l.lane_bits = 2;
    while (1 << l.lane_bits < l.items && l.lane_bits < 6) ++l.lane_bits;
    if (!l.in_registers) l.lane_bits = 6;
    return l;
}

// What a lane has of a head: the chunks at `first` and `second`, W values each.  Neighbouring lanes have neighbouring chunks, so that a load or a
// store of a wave is of whole lines (40961 tokens of 28 + 4 heads of 128, fp16, 64 values of each turning in neighbouring pairs: 118 us;
// with 32 bytes in a row for a lane 157).
struct Item {
    int first, second, pair, second_pair;              // the chunks' first pairs, -1 if a chunk does not turn (kHalves: one for both)
    bool has_first, has_second;
};
template <int W, Pairs PAIRS>
__host__ __device__ inline Item item_of(int items, int turning, int half, int head_dim, int i) {
    Item it;
    if (PAIRS == kHalves) {                            // chunk i of the one half and of the other; behind them the others' two halves
        const int rest = items - turning, x = i - turning;
        it.first = i < turning ? i * W : 2 * half + x * W;
        it.second = i < turning ? half + i * W : 2 * half + (rest + x) * W;
        it.pair = it.second_pair = i < turning ? i * W : -1;
    } else {
        it.first = i * W, it.second = (items + i) * W;
        // (a lane behind the head's has nothing to turn: the places of its chunks are another lane's)
        it.pair = i < items && it.first < 2 * half ? it.first / 2 : -1;
        it.second_pair = i < items && it.second < 2 * half ? it.second / 2 : -1;
    }
    it.has_first = i < items && it.first < head_dim;
    it.has_second = i < items && it.second < head_dim;
    return it;
}

// kAcross: chunks lie W + 1 places apart in LDS.  Where value y of a chunk has the other of its pair, `half` values further on or back, in places from the
// chunk's begin: the same for all lanes.
template <int W>
__host__ __device__ inline int place_on(int half, int y) {
    return half / W * (W + 1) + y + half % W + (y + half % W >= W);
}
template <int W>
__host__ __device__ inline int place_back(int half, int y) {
    return y - half / W * (W + 1) - half % W - (y < half % W);
}

}  // namespace stem
