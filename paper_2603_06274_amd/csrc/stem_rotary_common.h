// What the kernels share that turn heads by their positions: 16-byte and narrower accesses, divisions by constants of a launch,
// sines and cosines.
//
// Angles: position * turns is formed in 64 bits and its whole turns are dropped there (a position of 10^6 times a turn of 0.16
// has 2^18 whole turns; in 32 bits the angle would keep 5 bits behind them), then the rest is reduced to an eighth
// of a turn around the nearest quarter and goes through the Taylor polynomials of sine and cosine in 32 bits: at |x| <= pi / 4
// the first left out terms, x^11 / 11! and x^12 / 12!, are below 2e-9.
#pragma once

#include "stem_decode_common.h"

namespace stem {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// n / d for 0 <= n < 2^31 by a multiplication: (n * mul) >> (32 + shift)
struct FastDiv {
    uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
    uint32_t shift = 0;
    while ((1u << shift) < d && shift < 31) ++shift;
    // ceil(2^(31 + shift) / d): exact for n < 2^31 as 2^shift >= d
    const uint64_t mul = ((1ull << (31 + shift)) + d - 1) / d;
    return {d, (uint32_t)mul, shift};
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, FastDiv f) {
    return (uint32_t)(((uint64_t)n * f.mul) >> (31 + f.shift));
}

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

}  // namespace stem
