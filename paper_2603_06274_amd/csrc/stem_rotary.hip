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
    int32_t turning, single, items;                    // items of a head that turn, with those behind them of V values, and all
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
struct Chunk {
    T x[V];
};
template <int BYTES> struct Raw;
template <> struct Raw<16> { using type = u32x4_t; };
template <> struct Raw<8> { using type = uint64_t; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };
// One access each.  STREAM: what is read and written is more than the caches hold on to, and claims no place in them (128K tokens of 32 / 8
// heads 454 us without, 456 for the reads alone, 451 for the writes alone, 441 for both: 5.9 and 6.1 TB/s).
template <typename C, bool STREAM>
__device__ __forceinline__ C load(const void* p) {
    using R = typename Raw<sizeof(C)>::type;
    if constexpr (STREAM) return __builtin_bit_cast(C, __builtin_nontemporal_load(static_cast<const R*>(p)));
    else return __builtin_bit_cast(C, *static_cast<const R*>(p));
}
template <typename C, bool STREAM>
__device__ __forceinline__ void store(void* p, const C& c) {
    using R = typename Raw<sizeof(C)>::type;
    if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(R, c), static_cast<R*>(p));
    else *static_cast<R*>(p) = __builtin_bit_cast(R, c);
}

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
template <typename T, int V, bool HALF, bool PAGES, bool STREAM>
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
        if ((int)c >= a.turning) {                     // behind the rotary part, from the next 16 bytes on in whole ones
            if (is_q ? !a.copies_q : !a.copies_k) continue;
            constexpr int kWide = 16 / sizeof(T);
            if (V < kWide && (int)c >= a.single) {
                const int at = a.head_dim - (a.items - (int)c) * kWide;
                using W = Chunk<T, kWide>;
                store<W, STREAM>(dst + at, load<W, STREAM>(src + at));
                continue;
            }
            const int at = 2 * a.half + ((int)c - a.turning) * V;
            store<C, STREAM>(dst + at, load<C, STREAM>(src + at));
            continue;
        }
        if constexpr (HALF) {
            const int at = c * V;
            C lo = load<C, STREAM>(src + at), hi = load<C, STREAM>(src + at + a.half);
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 cs = turn_of[t * a.half + at + e];
                    const float p = Narrow<T>::up(lo.x[e]), r = Narrow<T>::up(hi.x[e]);
                    lo.x[e] = (T)(p * cs.x - r * cs.y);
                    hi.x[e] = (T)(r * cs.x + p * cs.y);
                }
            }
            store<C, STREAM>(dst + at, lo);
            store<C, STREAM>(dst + at + a.half, hi);
        } else {
            const int at = c * V;
            C w = load<C, STREAM>(src + at);
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 cs = turn_of[t * a.half + (at + e) / 2];
                    const float p = Narrow<T>::up(w.x[e]), r = Narrow<T>::up(w.x[e + 1]);
                    w.x[e] = (T)(p * cs.x - r * cs.y);
                    w.x[e + 1] = (T)(r * cs.x + p * cs.y);
                }
            }
            store<C, STREAM>(dst + at, w);
        }
    }
}

template <typename T>
static void launch(const RotaryArgs& args, bool half_layout, int V, bool pages, bool stream_through, hipStream_t stream) {
    constexpr int W = 16 / sizeof(T);
    const dim3 grid((args.tokens + args.per_block - 1) / args.per_block), block(kRotaryThreads);
#define STEM_ROTARY_LAUNCH(VV, HALF, STREAM)                                                                     \
    do {                                                                                                         \
        if (pages) hipLaunchKernelGGL((rotary_kernel<T, VV, HALF, true, STREAM>), grid, block, 0, stream, args);  \
        else hipLaunchKernelGGL((rotary_kernel<T, VV, HALF, false, STREAM>), grid, block, 0, stream, args);       \
    } while (0)
#define STEM_ROTARY_LAUNCH_WIDE(HALF)                         \
    do {                                                      \
        if (stream_through) STEM_ROTARY_LAUNCH(W, HALF, true); \
        else STEM_ROTARY_LAUNCH(W, HALF, false);              \
    } while (0)
    if (half_layout) {
        if (V == W) STEM_ROTARY_LAUNCH_WIDE(true);
        else if (V == 2) STEM_ROTARY_LAUNCH(2, true, false);
        else STEM_ROTARY_LAUNCH(1, true, false);
    } else {
        if (V == W) STEM_ROTARY_LAUNCH_WIDE(false);
        else STEM_ROTARY_LAUNCH(2, false, false);
    }
#undef STEM_ROTARY_LAUNCH
#undef STEM_ROTARY_LAUNCH_WIDE
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
    // 16-byte accesses where the parts that turn together begin and end at them, pairs or single values otherwise: strides, head
    // size and addresses are multiples of them already.
    const int part = half_layout ? a.half : s.rotary_dim;
    const int V = part % W == 0 ? W : part % 2 == 0 ? 2 : 1;
    a.turning = part / V;
    a.copies_q = call.q_out != call.q, a.copies_k = pages || call.k_out != call.k;
    const int behind = V == W ? s.head_dim : (s.rotary_dim + W - 1) / W * W;   // where 16-byte accesses begin
    a.single = a.turning + (behind - s.rotary_dim) / V;
    a.items = a.single + (s.head_dim - behind) / W;
    const int heads = s.num_q_heads + (pages ? 2 : 1) * s.num_kv_heads;
    // One token per workgroup unless its lanes would find less to do than one access each.  (32 / 8 heads of 128, 128K tokens, 1 / 2 / 4 tokens
    // 417 / 449 / 465 us.)
    a.per_block = kRotaryThreads / (heads * a.items);
    if (a.per_block > kPairsAtOnce / a.half) a.per_block = kPairsAtOnce / a.half;
    if (a.per_block < 1) a.per_block = 1;
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
    // What a smaller call leaves in the caches is read from there by the next one.
    const bool through = (int64_t)s.tokens * heads * s.head_dim * (s.dtype == STEM_FP32 ? 4 : 2) > 64 << 20;
    if (s.dtype == STEM_BF16) launch<__bf16>(a, half_layout, V, pages, through, stream);
    else if (s.dtype == STEM_FP16) launch<_Float16>(a, half_layout, V, pages, through, stream);
    else launch<float>(a, half_layout, V, pages, through, stream);
    return check_launch();
}

}  // namespace stem
