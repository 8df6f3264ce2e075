// Rotary positions of queries and keys (forward and transposed), and the same with the keys and values of new tokens going to
// their pages.
//
// A pair (x1, x2) of head values turns by the angle 2 pi * position * turns: (c x1 - s x2, c x2 + s x1).  Every value is read
// and written once, so a large call is bound by HBM and a small one by the latency of its launch.  All heads of a token share
// its angles: a workgroup takes a few tokens, computes their (cos, sin) once into LDS, one pair per thread, and then streams
// the tokens' rows, 16 bytes per access.
//
// Angles: position * turns is formed in 64 bits and its whole turns are dropped there (a position of 10^6 times a turn of 0.16
// has 2^18 whole turns; in 32 bits the angle would keep 5 bits behind them), then the rest is reduced to an eighth
// of a turn around the nearest quarter and goes through the Taylor polynomials of sine and cosine in 32 bits: at |x| <= pi / 4
// the first left out terms, x^11 / 11! and x^12 / 12!, are below 2e-9.
#include "stem_decode_common.h"

namespace stem {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// n / d for 0 <= n < 2^31 by a multiplication: (n * mul) >> (32 + shift)
struct FastDiv {
    uint32_t d, mul, shift;
};
static FastDiv fast_div(uint32_t d) {
    uint32_t shift = 0;
    while ((1u << shift) < d && shift < 31) ++shift;
    // ceil(2^(31 + shift) / d): exact for n < 2^31 as 2^shift >= d
    const uint64_t mul = ((1ull << (31 + shift)) + d - 1) / d;
    return {d, (uint32_t)mul, shift};
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, FastDiv f) {
    return (uint32_t)(((uint64_t)n * f.mul) >> (31 + f.shift));
}

struct RotaryArgs {
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out;
    const int32_t *positions, *slots;
    const double* turns;
    float factor, sine_factor;                         // the latter negated for the transposed map
    int32_t tokens, Hq, Hkv, half, head_dim;           // half: pairs of a head
    int32_t per_block;                                 // tokens of a workgroup
    int32_t turning, items;                            // items of a head that turn, and all that are written
    bool copies_q, copies_k;                           // whether the values that do not turn are written (not in place)
    FastDiv by_items, by_heads;
    int64_t q_st, q_sh, k_st, k_sh, qo_st, qo_sh, ko_st, ko_sh;
    int64_t page_st;                                   // k_out and v_out are pages: ko_st and ko_sh within one
    int32_t page_shift, page_mask;
    uint32_t slots_end;
};

constexpr int kRotaryThreads = 256;
constexpr int kPairsAtOnce = 2048;                     // (cos, sin) that a workgroup holds

template <typename T> struct Narrow;
template <> struct Narrow<__bf16> {
    static __device__ __forceinline__ float up(__bf16 x) { return (float)x; }
};
template <> struct Narrow<_Float16> {
    static __device__ __forceinline__ float up(_Float16 x) { return (float)x; }
};
template <> struct Narrow<float> {
    static __device__ __forceinline__ float up(float x) { return x; }
};

template <typename T, int V>
struct alignas(sizeof(T) * V) Chunk {
    T x[V];
};

// cos and sin of 2 pi * turn, turn in 64 bits
__device__ __forceinline__ float2 cos_sin(double turn) {
    turn -= __builtin_rint(turn);                      // -1/2 .. 1/2
    const double quarter = __builtin_rint(4.0 * turn);
    const float x = (float)(turn - 0.25 * quarter) * 6.28318530717958648f;
    const int n = (int)quarter;                        // -2 .. 2 (0 for a turn that is not finite)
    const float y = x * x;
    const float s = x * (1.f + y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880)))));
    const float c = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 - y * (1.f / 3628800)))));
    const float a = n & 1 ? s : c, b = n & 1 ? c : s;
    // n quarters further: cos (c, -s, -c, s), sin (s, c, -s, -c)
    return make_float2((n + 1) & 2 ? -a : a, n & 2 ? -b : b);
}

// V: values per access.  The half layout turns chunk c of the first half with chunk c of the second, the interleaved one the
// pairs within a chunk.
template <typename T, int V, bool HALF, bool PAGES>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
    __shared__ float2 turn_of[kPairsAtOnce];
    const int t0 = blockIdx.x * a.per_block, tid = threadIdx.x;
    const int here = min(a.per_block, a.tokens - t0);
    for (int x = tid; x < here * a.half; x += kRotaryThreads) {
        const int t = x / a.half, i = x - t * a.half;
        const float2 cs = cos_sin((double)a.positions[t0 + t] * a.turns[i]);
        turn_of[x] = make_float2(cs.x * a.factor, cs.y * a.sine_factor);
    }
    __syncthreads();
    const int heads = a.Hq + (PAGES ? 2 : 1) * a.Hkv;
    const uint32_t all = (uint32_t)here * heads * a.items;
    for (uint32_t x = tid; x < all; x += kRotaryThreads) {
        const uint32_t row = div_by(x, a.by_items), c = x - row * a.items;
        const int t = div_by(row, a.by_heads), head = row - t * heads;
        const bool is_q = head < a.Hq, is_v = PAGES && head >= a.Hq + a.Hkv;
        const int h = is_q ? head : is_v ? head - a.Hq - a.Hkv : head - a.Hq;
        const int64_t token = t0 + t;
        const T* src = static_cast<const T*>(is_q ? a.q : is_v ? a.v : a.k) + token * (is_q ? a.q_st : a.k_st) +
                       h * (is_q ? a.q_sh : a.k_sh);
        T* dst;
        if (PAGES) {
            const uint32_t slot = (uint32_t)a.slots[token];
            if (slot >= a.slots_end) continue;         // -1 among them
            dst = is_q ? static_cast<T*>(a.q_out) + token * a.qo_st + h * a.qo_sh
                       : static_cast<T*>(is_v ? a.v_out : a.k_out) + (int64_t)(slot >> a.page_shift) * a.page_st +
                             (int64_t)(slot & a.page_mask) * a.ko_st + h * a.ko_sh;
        } else {
            dst = is_q ? static_cast<T*>(a.q_out) + token * a.qo_st + h * a.qo_sh
                       : static_cast<T*>(a.k_out) + token * a.ko_st + h * a.ko_sh;
        }
        using C = Chunk<T, V>;
        if ((int)c >= a.turning) {                     // behind the rotary part
            if (is_q ? !a.copies_q : !a.copies_k) continue;
            const int at = 2 * a.half + ((int)c - a.turning) * V;
            *reinterpret_cast<C*>(dst + at) = *reinterpret_cast<const C*>(src + at);
            continue;
        }
        if constexpr (HALF) {
            const int at = c * V;
            C lo = *reinterpret_cast<const C*>(src + at), hi = *reinterpret_cast<const C*>(src + at + a.half);
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 cs = turn_of[t * a.half + at + e];
                    const float p = Narrow<T>::up(lo.x[e]), r = Narrow<T>::up(hi.x[e]);
                    lo.x[e] = (T)(p * cs.x - r * cs.y);
                    hi.x[e] = (T)(r * cs.x + p * cs.y);
                }
            }
            *reinterpret_cast<C*>(dst + at) = lo;
            *reinterpret_cast<C*>(dst + at + a.half) = hi;
        } else {
            const int at = c * V;
            C w = *reinterpret_cast<const C*>(src + at);
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 cs = turn_of[t * a.half + (at + e) / 2];
                    const float p = Narrow<T>::up(w.x[e]), r = Narrow<T>::up(w.x[e + 1]);
                    w.x[e] = (T)(p * cs.x - r * cs.y);
                    w.x[e + 1] = (T)(r * cs.x + p * cs.y);
                }
            }
            *reinterpret_cast<C*>(dst + at) = w;
        }
    }
}

template <typename T>
static void launch(const RotaryArgs& args, bool half_layout, bool wide, bool pages, hipStream_t stream) {
    constexpr int W = 16 / sizeof(T);
    const dim3 grid((args.tokens + args.per_block - 1) / args.per_block), block(kRotaryThreads);
#define STEM_ROTARY_LAUNCH(V, HALF)                                                                          \
    do {                                                                                                     \
        if (pages) hipLaunchKernelGGL((rotary_kernel<T, V, HALF, true>), grid, block, 0, stream, args);      \
        else hipLaunchKernelGGL((rotary_kernel<T, V, HALF, false>), grid, block, 0, stream, args);           \
    } while (0)
    if (half_layout) {
        if (wide) STEM_ROTARY_LAUNCH(W, true);
        else STEM_ROTARY_LAUNCH(1, true);
    } else {
        if (wide) STEM_ROTARY_LAUNCH(W, false);
        else STEM_ROTARY_LAUNCH(2, false);
    }
#undef STEM_ROTARY_LAUNCH
}

int launch_rotary(const RotaryCall& call, hipStream_t stream) {
    const stem_rotary_shape& s = call.shape;
    const bool pages = call.slots != nullptr, half_layout = s.layout == STEM_ROTARY_HALF;
    const int W = s.dtype == STEM_FP32 ? 4 : 8;
    RotaryArgs a = {};
    a.q = call.q, a.k = call.k, a.v = call.v;
    a.q_out = call.q_out, a.k_out = call.k_out, a.v_out = call.v_out;
    a.positions = call.positions, a.slots = call.slots, a.turns = call.turns;
    a.factor = call.factor;
    a.sine_factor = call.backward ? -call.factor : call.factor;
    a.tokens = s.tokens, a.Hq = s.num_q_heads, a.Hkv = s.num_kv_heads, a.half = s.rotary_dim / 2, a.head_dim = s.head_dim;
    // 16-byte accesses where the parts that turn together begin and end at them, single values (or pairs) otherwise: strides,
    // head size and addresses are multiples of them already.
    const bool wide = (half_layout ? a.half : s.rotary_dim) % W == 0;
    const int V = wide ? W : half_layout ? 1 : 2;
    a.turning = (half_layout ? a.half : s.rotary_dim) / V;
    a.copies_q = call.q_out != call.q, a.copies_k = pages || call.k_out != call.k;
    a.items = a.turning + (s.head_dim - s.rotary_dim) / V;
    const int heads = s.num_q_heads + (pages ? 2 : 1) * s.num_kv_heads;
    a.per_block = 4;
    while (a.per_block > 1 && (a.per_block * a.half > kPairsAtOnce || s.tokens < a.per_block * 1024)) a.per_block /= 2;
    a.by_items = fast_div(a.items);
    a.by_heads = fast_div(heads);
    a.q_st = s.q_stride_token, a.q_sh = s.q_stride_head, a.k_st = s.k_stride_token, a.k_sh = s.k_stride_head;
    a.qo_st = s.q_out_stride_token, a.qo_sh = s.q_out_stride_head;
    a.ko_st = s.k_out_stride_token, a.ko_sh = s.k_out_stride_head;
    if (pages) {
        a.ko_st = call.pages.stride_token, a.ko_sh = call.pages.stride_head, a.page_st = call.pages.stride_page;
        a.page_shift = __builtin_ctz(call.pages.page_size);
        a.page_mask = call.pages.page_size - 1;
        a.slots_end = (uint32_t)call.pages.num_pages * call.pages.page_size;
    }
    if (s.dtype == STEM_BF16) launch<__bf16>(a, half_layout, wide, pages, stream);
    else if (s.dtype == STEM_FP16) launch<_Float16>(a, half_layout, wide, pages, stream);
    else launch<float>(a, half_layout, wide, pages, stream);
    return check_launch();
}

}  // namespace stem
