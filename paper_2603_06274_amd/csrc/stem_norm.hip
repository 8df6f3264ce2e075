// Queries and keys normalised head by head, scaled by weights and turned by their positions in one pass; the same with the keys
// and values of new tokens going to their pages; and the gradients of both values and weights.
//
//     r = 1 / sqrt(mean x^2 + eps),  n = x r w,  y = R(position) n
//     g = R^T dy,  u = x r,  dw = sum g u,  h = g w,  dx = r (h - u mean(h u))
//
// Every value is read once and written once (two reads in the backward pass): HBM bounds a large call, latency a small one.  A
// head's values lie in the registers of `lanes` lanes (4 to 64), 32 bytes each: the two chunks of 16 bytes that turn with each other.  So
// sums over a head are a few exchanges between neighbouring lanes, and the row is read once.  A wave takes 64 / lanes heads at a
// time, a workgroup a few tokens, whose (cos, sin) it computes once, beside the weights, into LDS.
//
// Halves that do not both begin at 16 bytes lie in the lanes as they lie in memory, and are exchanged through LDS: 16-bit values are bound by
// that and its places (16384 tokens of 32 + 8 heads of 128, 50 values of each turning, bf16: 72 us, backwards 173; 48 values: 74 and 124;
// fp32 values: 110 and 178, as fast as memory; one pair of values per lane at a time, as below: 312 and 674 in bf16).  Heads that are longer
// than 64 lanes hold (fp32 beyond 512 values) go one wave each, a pair of values per lane at a time, read twice (the second time from the caches).
#include "stem_rotary_common.h"
#include "stem_norm_common.h"

namespace stem {

struct NormArgs {
    const void *q, *k, *v, *gq, *gk;
    void *q_out, *k_out, *v_out;
    const void *q_weight, *k_weight;
    const int32_t *positions, *slots;
    const double* turns;
    float* partial;
    float factor, sine_factor, eps, weight_offset, by_dim; // sine_factor is negated for the transposed map; by_dim: 1 / head_dim
    int32_t weight_dtype;
    int32_t tokens, Hq, Hkv, half, padded, head_dim;   // half: pairs of a head; padded: with those that turn by nothing in LDS
    int32_t per_step, per_block;                       // tokens at a time, tokens of a workgroup
    int32_t lane_bits, turning, items;                 // lanes of a head; items of kHalves that turn; all items (of two chunks)
    FastDiv by_heads, by_q, by_k;
    int64_t q_st, q_sh, k_st, k_sh, qo_st, qo_sh, ko_st, ko_sh;
    int64_t page_st;                                   // k_out and v_out are pages: ko_st and ko_sh within one
    int32_t page_shift, page_mask;
    uint32_t slots_end;
};

constexpr int kNormThreads = 256;
constexpr int kNormPairs = 2048;                       // (cos, sin) that a workgroup holds at most

// v_rsq_f32 is within 1 ulp; its argument is a normal number, as eps is one
__device__ __forceinline__ float inverse_root(float x) { return __builtin_amdgcn_rsqf(x); }

// Sum over the 2^bits lanes of a head (2 <= bits <= 6), the same in each of them and in any order of adding: within a row of 16 lanes by data
// parallel moves, which are as fast as any vector instruction, beyond it by exchanges through LDS hardware.
template <int CONTROL>
__device__ __forceinline__ float add_moved(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ float head_sum(float x, int bits) {
    x = add_moved<0xB1>(x);                            // lanes 1 0 3 2
    x = add_moved<0x4E>(x);                            // 2 3 0 1
    if (bits > 2) x = add_moved<0x141>(x);             // the other four of eight
    if (bits > 3) x = add_moved<0x140>(x);             // the other eight of sixteen
    if (bits > 4) x += __shfl_xor(x, 16);
    if (bits > 5) x += __shfl_xor(x, 32);
    return x;
}

// weight[i] + offset, 1 where there is none
__device__ __forceinline__ float weight_at(const void* w, int dtype, float offset, int i) {
    if (!w) return 1.f;
    return offset + (dtype == STEM_FP32 ? static_cast<const float*>(w)[i]
                     : dtype == STEM_BF16 ? (float)static_cast<const __bf16*>(w)[i] : (float)static_cast<const _Float16*>(w)[i]);
}
// Both tensors' weights -> [2][head_dim]
__device__ __forceinline__ void weights_to(float* w, const NormArgs& a) {
    for (int i = threadIdx.x; i < a.head_dim; i += kNormThreads) {
        w[i] = weight_at(a.q_weight, a.weight_dtype, a.weight_offset, i);
        w[a.head_dim + i] = weight_at(a.k_weight, a.weight_dtype, a.weight_offset, i);
    }
}
// (cos, sin) of `here` tokens from t0 on -> [here][padded]; pairs behind the rotary part turn by nothing.  SPREAD > 0: with one place free
// behind every SPREAD pairs.
template <int SPREAD>
__device__ __forceinline__ void turns_to(float2* turn_of, const NormArgs& a, int t0, int here) {
    const int pairs = SPREAD ? a.half : a.padded;
    for (int x = threadIdx.x; x < here * pairs; x += kNormThreads) {
        const int t = x / pairs, i = x - t * pairs;
        float2 cs = make_float2(1.f, 0.f);
        if (i < a.half) {
            cs = cos_sin((double)a.positions[t0 + t] * a.turns[i]);
            cs = make_float2(cs.x * a.factor, cs.y * a.sine_factor);
        }
        turn_of[t * a.padded + i + (SPREAD ? i / (SPREAD ? SPREAD : 1) : 0)] = cs;
    }
}

// A lane's values turned, if any of them turn.  PAIRS says where the other of a pair is: in x[W + e], next to it, or in the lane that has the value
// `half` further on or back.  cs: a token's (cos, sin).
// exchange: the head's values for its other lanes, W + 1 places to a chunk (as in cs), so that one value of all lanes lies in different
// banks.  Values that do not turn ask for what lies there, and do not use it.
template <int W, Pairs PAIRS>
__device__ __forceinline__ void turn(float (&x)[2 * W], const float2* cs, const Item& it, const NormArgs& a, float* exchange) {
    if (it.pair < 0) return;
    if constexpr (PAIRS == kHalves) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float2 c = cs[it.pair + e];
            const float y = x[e] * c.x - x[W + e] * c.y;
            x[W + e] = x[W + e] * c.x + x[e] * c.y;
            x[e] = y;
        }
    } else if constexpr (PAIRS == kNeighbours) {
        auto chunk = [&](float* v, const float2* c) {
#pragma unroll
            for (int e = 0; e < W / 2; ++e) {
                const float y = v[2 * e] * c[e].x - v[2 * e + 1] * c[e].y;
                v[2 * e + 1] = v[2 * e + 1] * c[e].x + v[2 * e] * c[e].y;
                v[2 * e] = y;
            }
        };
        chunk(x, cs + it.pair);
        if (it.second_pair >= 0) chunk(x + W, cs + it.second_pair);
    } else {
        constexpr int S = W + 1;
        const int half = a.half;
        float* const mine[2] = {exchange + it.first / W * S, exchange + it.second / W * S};
        const float2* const turn_at[2] = {cs + it.first / W * S, cs + it.second / W * S};
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) mine[e / W][e % W] = x[e];
        // (all lanes of a head are in one wave, whose reads and writes of LDS stay in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float2 c[2 * W];
        float other[2 * W];
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) {              // (all asked for before any is used)
            const int y = e % W, on = place_on<W>(half, y), back = place_back<W>(half, y);
            const bool in_first = (e < W ? it.first : it.second) + y < half;
            other[e] = mine[e / W][in_first ? on : back];
            c[e] = turn_at[e / W][in_first ? y : back];
        }
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) {
            const int i = (e < W ? it.first : it.second) + e % W;
            const float y = x[e] * c[e].x + (i < half ? -other[e] : other[e]) * c[e].y;
            x[e] = i < 2 * half ? y : x[e];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int W, bool STREAM>
__device__ __forceinline__ void load_item(float (&x)[2 * W], const T* row, const Item& it) {
    using C = Chunk<T, W>;
    C lo = {}, hi = {};
    if (it.has_first) lo = load<C, STREAM>(row + it.first);
    if (it.has_second) hi = load<C, STREAM>(row + it.second);
#pragma unroll
    for (int e = 0; e < W; ++e) x[e] = Narrow<T>::up(lo.x[e]), x[W + e] = Narrow<T>::up(hi.x[e]);
}
template <typename T, int W, bool STREAM>
__device__ __forceinline__ void store_item(T* row, const float (&x)[2 * W], const Item& it) {
    using C = Chunk<T, W>;
    C lo, hi;
#pragma unroll
    for (int e = 0; e < W; ++e) lo.x[e] = (T)x[e], hi.x[e] = (T)x[W + e];
    if (it.has_first) store<C, STREAM>(row + it.first, lo);
    if (it.has_second) store<C, STREAM>(row + it.second, hi);
}
template <int W>
__device__ __forceinline__ void scale_item(float (&x)[2 * W], const float* w, const Item& it, float r) {
#pragma unroll
    for (int e = 0; e < W; ++e) {
        x[e] = x[e] * r * (it.has_first ? w[it.first + e] : 0.f);
        x[W + e] = x[W + e] * r * (it.has_second ? w[it.second + e] : 0.f);
    }
}

// Where row `row` of a workgroup's tokens comes from and goes to.  false: a token without a place.
template <typename T, bool PAGES>
__device__ __forceinline__ bool place_row(const NormArgs& a, int t0, uint32_t row, const T*& src, T*& dst, int& t, int& kind) {
    const int heads = a.Hq + (PAGES ? 2 : 1) * a.Hkv;
    t = (int)div_by(row, a.by_heads);
    const int head = (int)row - t * heads;
    kind = head < a.Hq ? 0 : PAGES && head >= a.Hq + a.Hkv ? 2 : 1;
    const int h = head - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv);
    const int64_t token = t0 + t;
    src = static_cast<const T*>(kind == 0 ? a.q : kind == 2 ? a.v : a.k) + token * (kind == 0 ? a.q_st : a.k_st) +
          h * (kind == 0 ? a.q_sh : a.k_sh);
    if (PAGES) {
        const uint32_t slot = (uint32_t)a.slots[token];
        if (slot >= a.slots_end) return false;         // -1 among them
        dst = kind == 0 ? static_cast<T*>(a.q_out) + token * a.qo_st + h * a.qo_sh
                        : static_cast<T*>(kind == 2 ? a.v_out : a.k_out) + (int64_t)(slot >> a.page_shift) * a.page_st +
                              (int64_t)(slot & a.page_mask) * a.ko_st + h * a.ko_sh;
    } else {
        dst = kind == 0 ? static_cast<T*>(a.q_out) + token * a.qo_st + h * a.qo_sh
                        : static_cast<T*>(a.k_out) + token * a.ko_st + h * a.ko_sh;
    }
    return true;
}

template <typename T, Pairs PAIRS, bool PAGES, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void norm_rotary_kernel(NormArgs a) {
    constexpr int W = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char norm_lds[];
    float* const weights = reinterpret_cast<float*>(norm_lds);
    float* const exchange = weights + 2 * a.head_dim + (threadIdx.x >> a.lane_bits << a.lane_bits) * 2 * (W + 1);
    float2* const turn_of = reinterpret_cast<float2*>(weights + 2 * a.head_dim + (PAIRS == kAcross ? kNormThreads * 2 * (W + 1) : 0));
    const int t0 = blockIdx.x * a.per_block, here = min(a.per_block, a.tokens - t0);
    weights_to(weights, a);
    turns_to<PAIRS == kAcross ? W : 0>(turn_of, a, t0, here);
    __syncthreads();
    const int lane = threadIdx.x & ((1 << a.lane_bits) - 1);
    const Item it = item_of<W, PAIRS>(a.items, a.turning, a.half, a.head_dim, lane);
    const uint32_t rows = (uint32_t)here * (a.Hq + (PAGES ? 2 : 1) * a.Hkv);
    for (uint32_t row = threadIdx.x >> a.lane_bits; row < rows; row += kNormThreads >> a.lane_bits) {
        const T* src;
        T* dst;
        int t, kind;
        if (!place_row<T, PAGES>(a, t0, row, src, dst, t, kind)) continue;
        float x[2 * W];
        load_item<T, W, STREAM>(x, src, it);
        if (!PAGES || kind != 2) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
            const float r = inverse_root(__builtin_fmaf(head_sum(sum, a.lane_bits), a.by_dim, a.eps));
            scale_item<W>(x, weights + (kind == 0 ? 0 : a.head_dim), it, r);
            turn<W, PAIRS>(x, turn_of + t * a.padded, it, a, exchange);
        }
        store_item<T, W, STREAM>(dst, x, it);
    }
}

// One wave per head.
template <typename T, bool PAGES>
__global__ __launch_bounds__(kNormThreads) void norm_rotary_any_kernel(NormArgs a, bool half_layout) {
    extern __shared__ __align__(16) unsigned char norm_lds[];
    float* const weights = reinterpret_cast<float*>(norm_lds);
    float2* const turn_of = reinterpret_cast<float2*>(weights + 2 * a.head_dim);
    const int t0 = blockIdx.x * a.per_block, here = min(a.per_block, a.tokens - t0);
    weights_to(weights, a);
    turns_to<0>(turn_of, a, t0, here);
    __syncthreads();
    const int lane = threadIdx.x & 63;
    const uint32_t rows = (uint32_t)here * (a.Hq + (PAGES ? 2 : 1) * a.Hkv);
    for (uint32_t row = threadIdx.x >> 6; row < rows; row += kNormThreads / 64) {
        const T* src;
        T* dst;
        int t, kind;
        if (!place_row<T, PAGES>(a, t0, row, src, dst, t, kind)) continue;
        const float* w = weights + (kind == 0 ? 0 : a.head_dim);
        if (PAGES && kind == 2) {
            for (int i = lane; i < a.head_dim; i += 64) dst[i] = src[i];
            continue;
        }
        float sum = 0.f;
        for (int i = lane; i < a.head_dim; i += 64) {
            const float x = Narrow<T>::up(src[i]);
            sum = __builtin_fmaf(x, x, sum);
        }
        const float r = inverse_root(__builtin_fmaf(head_sum(sum, 6), a.by_dim, a.eps));
        // (in place: all of the row has been read for the sum, and each value is read again by the lane that writes it)
        for (int i = lane; i < a.half; i += 64) {
            const int p = half_layout ? i : 2 * i, s = half_layout ? i + a.half : 2 * i + 1;
            const float x = Narrow<T>::up(src[p]) * r * w[p], y = Narrow<T>::up(src[s]) * r * w[s];
            const float2 cs = turn_of[t * a.padded + i];
            dst[p] = (T)(x * cs.x - y * cs.y);
            dst[s] = (T)(y * cs.x + x * cs.y);
        }
        for (int i = 2 * a.half + lane; i < a.head_dim; i += 64) dst[i] = (T)(Narrow<T>::up(src[i]) * r * w[i]);
    }
}

// One tensor's heads of `here` tokens: its gradients, and the lane's share of its weights' into acc.
template <typename T, Pairs PAIRS, bool STREAM>
__device__ __forceinline__ void backward_rows(const NormArgs& a, const void* x_base, const void* g_base, void* out, int64_t st, int64_t sh,
                                              int64_t go_st, int64_t go_sh, int heads, FastDiv by, const float* w, const float2* turn_of,
                                              float* exchange, int t0, int here, const Item& it, float (&acc)[2 * (16 / sizeof(T))]) {
    constexpr int W = 16 / sizeof(T);
    const uint32_t rows = (uint32_t)here * heads;
    for (uint32_t row = threadIdx.x >> a.lane_bits; row < rows; row += kNormThreads >> a.lane_bits) {
        const int t = (int)div_by(row, by), h = (int)row - t * heads;
        const int64_t token = t0 + t;
        float x[2 * W], g[2 * W];
        load_item<T, W, STREAM>(x, static_cast<const T*>(x_base) + token * st + h * sh, it);
        load_item<T, W, STREAM>(g, static_cast<const T*>(g_base) + token * go_st + h * go_sh, it);
        turn<W, PAIRS>(g, turn_of + t * a.padded, it, a, exchange);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
        const float r = inverse_root(__builtin_fmaf(head_sum(sum, a.lane_bits), a.by_dim, a.eps));
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) {
            x[e] *= r;                                 // u
            acc[e] = __builtin_fmaf(g[e], x[e], acc[e]);
        }
        scale_item<W>(g, w, it, 1.f);                  // h
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) dot = __builtin_fmaf(g[e], x[e], dot);
        const float mean = head_sum(dot, a.lane_bits) * a.by_dim;
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) g[e] = r * (g[e] - x[e] * mean);
        store_item<T, W, STREAM>(static_cast<T*>(out) + token * st + h * sh, g, it);
    }
}

// A workgroup takes per_step tokens at a time, one step of all workgroups behind the other: what is read at a time lies
// together (32768 tokens of 32 + 8 heads of 128: 181 us, 805 MB; each workgroup's tokens one behind the other 196).
template <typename T, Pairs PAIRS, bool STREAM>
__global__ __launch_bounds__(kNormThreads) void norm_backward_kernel(NormArgs a) {
    constexpr int W = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char norm_lds[];
    float* const weights = reinterpret_cast<float*>(norm_lds);
    float* const exchange = weights + 2 * a.head_dim + (threadIdx.x >> a.lane_bits << a.lane_bits) * 2 * (W + 1);
    float2* const turn_of = reinterpret_cast<float2*>(weights + 2 * a.head_dim + (PAIRS == kAcross ? kNormThreads * 2 * (W + 1) : 0));
    const int lane = threadIdx.x & ((1 << a.lane_bits) - 1);
    const Item it = item_of<W, PAIRS>(a.items, a.turning, a.half, a.head_dim, lane);
    float acc_q[2 * W] = {}, acc_k[2 * W] = {};
    weights_to(weights, a);
    for (int t0 = blockIdx.x * a.per_step; t0 < a.tokens; t0 += gridDim.x * a.per_step) {
        const int here = min(a.per_step, a.tokens - t0);
        turns_to<PAIRS == kAcross ? W : 0>(turn_of, a, t0, here);
        __syncthreads();
        if (a.Hq > 0)
            backward_rows<T, PAIRS, STREAM>(a, a.q, a.gq, a.q_out, a.q_st, a.q_sh, a.qo_st, a.qo_sh, a.Hq, a.by_q, weights, turn_of, exchange,
                                            t0, here, it, acc_q);
        if (a.Hkv > 0)
            backward_rows<T, PAIRS, STREAM>(a, a.k, a.gk, a.k_out, a.k_st, a.k_sh, a.ko_st, a.ko_sh, a.Hkv, a.by_k, weights + a.head_dim,
                                            turn_of, exchange, t0, here, it, acc_k);
        __syncthreads();
    }
    if (!a.partial) return;
    // the heads' lanes of a workgroup together: [groups][head_dim], which the launch has room for
    float* const sums = reinterpret_cast<float*>(norm_lds);
    const int groups = kNormThreads >> a.lane_bits, group = threadIdx.x >> a.lane_bits;
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        float(&acc)[2 * W] = tensor ? acc_k : acc_q;
        if (tensor) __syncthreads();
#pragma unroll
        for (int e = 0; e < W; ++e) {
            if (it.has_first) sums[group * a.head_dim + it.first + e] = acc[e];
            if (it.has_second) sums[group * a.head_dim + it.second + e] = acc[W + e];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.head_dim; i += kNormThreads) {
            float sum = 0.f;
            for (int x = 0; x < groups; ++x) sum += sums[x * a.head_dim + i];
            a.partial[((int64_t)blockIdx.x * 2 + tensor) * a.head_dim + i] = sum;
        }
    }
}

// One wave per head; its share of the weights' gradients in LDS, [waves][2][head_dim], where a lane always has the same values.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_backward_any_kernel(NormArgs a, bool half_layout) {
    extern __shared__ __align__(16) unsigned char norm_lds[];
    constexpr int kWaves = kNormThreads / 64;
    float* const weights = reinterpret_cast<float*>(norm_lds);
    float* const sums = weights + 2 * a.head_dim;
    float2* const turn_of = reinterpret_cast<float2*>(sums + kWaves * 2 * a.head_dim);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    weights_to(weights, a);
    for (int i = threadIdx.x; i < kWaves * 2 * a.head_dim; i += kNormThreads) sums[i] = 0.f;
    for (int t0 = blockIdx.x * a.per_step; t0 < a.tokens; t0 += gridDim.x * a.per_step) {
        const int here = min(a.per_step, a.tokens - t0);
        turns_to<0>(turn_of, a, t0, here);
        __syncthreads();
        const uint32_t rows = (uint32_t)here * (a.Hq + a.Hkv);
        for (uint32_t row = wave; row < rows; row += kWaves) {
            const int t = (int)div_by(row, a.by_heads), head = (int)row - t * (a.Hq + a.Hkv);
            const bool is_q = head < a.Hq;
            const int h = is_q ? head : head - a.Hq;
            const int64_t token = t0 + t, at = token * (is_q ? a.q_st : a.k_st) + h * (is_q ? a.q_sh : a.k_sh);
            const T* x = static_cast<const T*>(is_q ? a.q : a.k) + at;
            const T* gy = static_cast<const T*>(is_q ? a.gq : a.gk) + token * (is_q ? a.qo_st : a.ko_st) + h * (is_q ? a.qo_sh : a.ko_sh);
            T* out = static_cast<T*>(is_q ? a.q_out : a.k_out) + at;
            const float* w = weights + (is_q ? 0 : a.head_dim);
            float* mine = sums + (wave * 2 + (is_q ? 0 : 1)) * a.head_dim;
            auto turned = [&](int i, int& p, int& s, float& gp, float& gs) {       // pair i's places, and its gradients turned back
                p = half_layout ? i : 2 * i, s = half_layout ? i + a.half : 2 * i + 1;
                const float2 cs = turn_of[t * a.padded + i];
                const float yp = Narrow<T>::up(gy[p]), ys = Narrow<T>::up(gy[s]);
                gp = yp * cs.x - ys * cs.y;
                gs = ys * cs.x + yp * cs.y;
            };
            float squares = 0.f, dot = 0.f;
            for (int i = lane; i < a.head_dim; i += 64) {
                const float v = Narrow<T>::up(x[i]);
                squares = __builtin_fmaf(v, v, squares);
            }
            const float r = inverse_root(__builtin_fmaf(head_sum(squares, 6), a.by_dim, a.eps));
            for (int i = lane; i < a.half; i += 64) {
                int p, s;
                float gp, gs;
                turned(i, p, s, gp, gs);
                const float up = Narrow<T>::up(x[p]) * r, us = Narrow<T>::up(x[s]) * r;
                mine[p] += gp * up;
                mine[s] += gs * us;
                dot = __builtin_fmaf(gp * w[p], up, __builtin_fmaf(gs * w[s], us, dot));
            }
            for (int i = 2 * a.half + lane; i < a.head_dim; i += 64) {
                const float g = Narrow<T>::up(gy[i]), u = Narrow<T>::up(x[i]) * r;
                mine[i] += g * u;
                dot = __builtin_fmaf(g * w[i], u, dot);
            }
            const float mean = head_sum(dot, 6) * a.by_dim;
            for (int i = lane; i < a.half; i += 64) {
                int p, s;
                float gp, gs;
                turned(i, p, s, gp, gs);
                const float up = Narrow<T>::up(x[p]) * r, us = Narrow<T>::up(x[s]) * r;
                out[p] = (T)(r * (gp * w[p] - up * mean));
                out[s] = (T)(r * (gs * w[s] - us * mean));
            }
            for (int i = 2 * a.half + lane; i < a.head_dim; i += 64)
                out[i] = (T)(r * (Narrow<T>::up(gy[i]) * w[i] - Narrow<T>::up(x[i]) * r * mean));
        }
        __syncthreads();
    }
    if (!a.partial) return;
    for (int i = threadIdx.x; i < 2 * a.head_dim; i += kNormThreads) {
        float sum = 0.f;
        for (int x = 0; x < kWaves; ++x) sum += sums[x * 2 * a.head_dim + i];
        a.partial[(int64_t)blockIdx.x * 2 * a.head_dim + i] = sum;
    }
}

// The workgroups' sums together, in 64 bits: four values per workgroup, every 256th part per lane, all asked for at once (6 us with 1024 parts
// of 2 x 128 values; with 16 values per workgroup, so that whole lines are read, 9: 16 workgroups wait for 64 KiB each).
constexpr int kSumThreads = 256;
__global__ __launch_bounds__(kSumThreads) void norm_weights_kernel(const float* partial, int parts, int head_dim, float* q_grad, float* k_grad) {
    constexpr int kWaves = kSumThreads / 64, kEach = kNormMostParts / kSumThreads;
    __shared__ double sums[kWaves][4];
    const int i = blockIdx.x * 4;                      // (2 head_dim is a multiple of 4)
    float4 next[kEach];
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int p = threadIdx.x + x * kSumThreads;
        next[x] = p < parts ? *reinterpret_cast<const float4*>(partial + (int64_t)p * 2 * head_dim + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    double sum[4] = {};
#pragma unroll
    for (int x = 0; x < kEach; ++x) sum[0] += next[x].x, sum[1] += next[x].y, sum[2] += next[x].z, sum[3] += next[x].w;
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += __shfl_xor(sum[c], d);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int c = 0; c < 4; ++c) sums[threadIdx.x >> 6][c] = sum[c];
    __syncthreads();
    if (threadIdx.x >= 4) return;
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += sums[w][threadIdx.x];
    const int at = i + threadIdx.x;
    float* const out = at < head_dim ? q_grad : k_grad;
    if (out) out[at < head_dim ? at : at - head_dim] = (float)all;
}

// A launch's arguments but for its split into workgroups; whether heads lie in registers, and how.
static bool arguments_of(const NormCall& c, NormArgs& a, Pairs& pairs) {
    const RotaryCall& r = c.rotary;
    const stem_rotary_shape& s = r.shape;
    const bool pages = r.slots != nullptr;
    a = {};
    a.q = r.q, a.k = r.k, a.v = r.v, a.gq = c.grad_q, a.gk = c.grad_k;
    a.q_out = r.q_out, a.k_out = r.k_out, a.v_out = r.v_out;
    a.q_weight = c.norm.q_weight, a.k_weight = c.norm.k_weight;
    a.positions = r.positions, a.slots = r.slots, a.turns = r.turns;
    a.partial = c.partial;
    a.factor = r.factor, a.sine_factor = r.backward ? -r.factor : r.factor;
    a.eps = c.norm.eps, a.weight_offset = c.norm.weight_offset, a.by_dim = 1.f / s.head_dim, a.weight_dtype = c.norm.weight_dtype;
    a.tokens = s.tokens, a.Hq = s.num_q_heads, a.Hkv = s.num_kv_heads, a.half = s.rotary_dim / 2, a.head_dim = s.head_dim;
    const HeadLayout l = head_layout(s);
    pairs = l.pairs, a.items = l.items, a.turning = l.turning, a.lane_bits = l.lane_bits, a.padded = l.padded;
    const int heads = a.Hq + (pages ? 2 : 1) * a.Hkv;
    a.by_heads = fast_div(heads);
    a.by_q = fast_div(a.Hq > 0 ? a.Hq : 1), a.by_k = fast_div(a.Hkv > 0 ? a.Hkv : 1);
    a.q_st = s.q_stride_token, a.q_sh = s.q_stride_head, a.k_st = s.k_stride_token, a.k_sh = s.k_stride_head;
    a.qo_st = s.q_out_stride_token, a.qo_sh = s.q_out_stride_head;
    a.ko_st = s.k_out_stride_token, a.ko_sh = s.k_out_stride_head;
    if (pages) {
        a.ko_st = r.pages.stride_token, a.ko_sh = r.pages.stride_head, a.page_st = r.pages.stride_page;
        a.page_shift = __builtin_ctz(r.pages.page_size);
        a.page_mask = r.pages.page_size - 1;
        a.slots_end = (uint32_t)r.pages.num_pages * r.pages.page_size;
    }
    return l.in_registers;
}

// Tokens of which a workgroup's lanes have a head each, of `heads` per token; at most what its LDS has room for.
static int tokens_for(const NormArgs& a, int heads) {
    const int groups = kNormThreads >> a.lane_bits;
    int n = groups / heads;
    if (n > kNormPairs / a.padded) n = kNormPairs / a.padded;
    return n < 1 ? 1 : n;
}

// LDS of the weights, of what lanes exchange, and of the (cos, sin) of per_step tokens
template <typename T>
static size_t lds_of(const NormArgs& a, bool exchanges) {
    return sizeof(float) * (2 * a.head_dim + (exchanges ? kNormThreads * 2 * (16 / sizeof(T) + 1) : 0)) + sizeof(float2) * (size_t)a.per_step * a.padded;
}

template <typename T>
static void launch_forward(const NormArgs& a, bool wide, Pairs pairs, bool pages, bool through, hipStream_t stream) {
    const dim3 grid((a.tokens + a.per_block - 1) / a.per_block), block(kNormThreads);
    const size_t lds = lds_of<T>(a, wide && pairs == kAcross);
    if (!wide) {
        const bool half_layout = pairs != kNeighbours;
        if (pages) hipLaunchKernelGGL((norm_rotary_any_kernel<T, true>), grid, block, lds, stream, a, half_layout);
        else hipLaunchKernelGGL((norm_rotary_any_kernel<T, false>), grid, block, lds, stream, a, half_layout);
        return;
    }
#define STEM_NORM_LAUNCH(PAIRS)                                                                                          \
    do {                                                                                                                 \
        if (pages && through) hipLaunchKernelGGL((norm_rotary_kernel<T, PAIRS, true, true>), grid, block, lds, stream, a);   \
        else if (pages) hipLaunchKernelGGL((norm_rotary_kernel<T, PAIRS, true, false>), grid, block, lds, stream, a);    \
        else if (through) hipLaunchKernelGGL((norm_rotary_kernel<T, PAIRS, false, true>), grid, block, lds, stream, a);  \
        else hipLaunchKernelGGL((norm_rotary_kernel<T, PAIRS, false, false>), grid, block, lds, stream, a);              \
    } while (0)
    if (pairs == kHalves) STEM_NORM_LAUNCH(kHalves);
    else if (pairs == kNeighbours) STEM_NORM_LAUNCH(kNeighbours);
    else STEM_NORM_LAUNCH(kAcross);
#undef STEM_NORM_LAUNCH
}

static size_t value_bytes(int32_t dtype) { return dtype == STEM_FP32 ? 4 : 2; }

int launch_norm_rotary(const NormCall& c, hipStream_t stream) {
    const stem_rotary_shape& s = c.rotary.shape;
    NormArgs a;
    Pairs pairs;
    const bool wide = arguments_of(c, a, pairs), pages = c.rotary.slots != nullptr;
    const int heads = a.Hq + (pages ? 2 : 1) * a.Hkv;
    // A long call's workgroups take two tokens where they would take one, four if lanes exchange halves: the vector instructions of 16-bit
    // values fill 75 % of the time of one (weights, (cos, sin) and partly idle waves for 40 heads).  1 / 2 / 4 tokens: 131072 of 32 + 8 heads of 128
    // 468 / 451 / 466 us (four read from further apart), 16384 with 50 values turning 96 / 78 / 72, in fp32 109 / 113 / 123.
    a.per_block = tokens_for(a, heads);
    const int most = s.dtype == STEM_FP32 ? 1 : pairs == kAcross ? 4 : 2;
    while (2 * a.per_block <= most && s.tokens / (2 * a.per_block) >= 4096 && 2 * a.per_block * a.padded <= kNormPairs) a.per_block *= 2;
    a.per_step = a.per_block;
    const bool through = (int64_t)s.tokens * heads * s.head_dim * value_bytes(s.dtype) > 64 << 20;
    if (s.dtype == STEM_BF16) launch_forward<__bf16>(a, wide, pairs, pages, through, stream);
    else if (s.dtype == STEM_FP16) launch_forward<_Float16>(a, wide, pairs, pages, through, stream);
    else launch_forward<float>(a, wide, pairs, pages, through, stream);
    return check_launch();
}

template <typename T>
static void launch_backward(const NormArgs& a, int groups, bool wide, Pairs pairs, bool through, hipStream_t stream) {
    const dim3 grid(groups), block(kNormThreads);
    if (!wide) {
        const size_t lds = lds_of<T>(a, false) + 2 * sizeof(float) * a.head_dim * (kNormThreads / 64);
        hipLaunchKernelGGL((norm_backward_any_kernel<T>), grid, block, lds, stream, a, pairs != kNeighbours);
        return;
    }
    const size_t sums = sizeof(float) * (size_t)(kNormThreads >> a.lane_bits) * a.head_dim, others = lds_of<T>(a, pairs == kAcross);
    const size_t lds = others > sums ? others : sums;
#define STEM_NORM_LAUNCH(PAIRS)                                                                                          \
    do {                                                                                                                 \
        if (through) hipLaunchKernelGGL((norm_backward_kernel<T, PAIRS, true>), grid, block, lds, stream, a);            \
        else hipLaunchKernelGGL((norm_backward_kernel<T, PAIRS, false>), grid, block, lds, stream, a);                   \
    } while (0)
    if (pairs == kHalves) STEM_NORM_LAUNCH(kHalves);
    else if (pairs == kNeighbours) STEM_NORM_LAUNCH(kNeighbours);
    else STEM_NORM_LAUNCH(kAcross);
#undef STEM_NORM_LAUNCH
}

int launch_norm_rotary_backward(const NormCall& c, hipStream_t stream) {
    const stem_rotary_shape& s = c.rotary.shape;
    NormArgs a;
    Pairs pairs;
    const bool wide = arguments_of(c, a, pairs);
    const int parts = norm_parts(s);
    int groups = 0;                                    // workgroups, of the `parts` that there may be
    if (parts > 0) {
        const int fewest = a.Hq > 0 && (a.Hkv == 0 || a.Hq < a.Hkv) ? a.Hq : a.Hkv, each = (s.tokens + parts - 1) / parts;
        a.per_step = tokens_for(a, fewest);
        if (a.per_step > each) a.per_step = each;
        groups = (s.tokens + a.per_step - 1) / a.per_step;
        if (groups > parts) groups = parts;
        const bool through = (int64_t)s.tokens * (a.Hq + a.Hkv) * s.head_dim * value_bytes(s.dtype) > 64 << 20;
        if (s.dtype == STEM_BF16) launch_backward<__bf16>(a, groups, wide, pairs, through, stream);
        else if (s.dtype == STEM_FP16) launch_backward<_Float16>(a, groups, wide, pairs, through, stream);
        else launch_backward<float>(a, groups, wide, pairs, through, stream);
        if (const int st = check_launch()) return st;
        if (!a.partial) return STEM_OK;
    }
    hipLaunchKernelGGL(norm_weights_kernel, dim3(2 * s.head_dim / 4), dim3(kSumThreads), 0, stream, c.partial, groups, s.head_dim,
                        c.q_weight_grad, c.k_weight_grad);
    return check_launch();
}

}  // namespace stem
