// Attention of many short rows to one long prefix that they share, and of each request's rows to its own pages behind it.
//
// With Q the rows (token, query head of the group) of one KV head,
//     o = softmax(scale Q [Kp; Ks]^T) [Vp; Vs]
// is computed in parts over the keys: a part leaves its largest score m, its sum l = sum e^(s - m) and its o = sum e^(s - m) v, and
//     o = sum_p e^(m_p - m) o_p / sum_p e^(m_p - m) l_p,  m = max_p m_p
// joins them (join_kernel).  The prefix is one dense product of all requests' rows together, so K and V of the prefix are read once
// for all of them; the keys are split so that every CU has a part.
//
// Products and softmax are those of stage 3: S^T = K Q^T, so that one query is one lane's column and its softmax needs no exchange
// but when its reference moves and at the end; P^T lies in the registers as the second product O^T += V^T P^T takes it, V^T comes from
// row-major V by transposing LDS reads.  Every wave has a softmax and an o of its own; those over other keys of the same rows are
// joined at a workgroup's end through LDS.
//
// K and V are on their way to registers for one tile while the tile before is used from LDS.  Rows are asked for by up to 16, through a
// buffer resource whose size ends with the last valid one: rows behind it, and all of a page that is none, arrive as zeros and
// are masked.  A tile begins at a multiple of 16 keys, so 16 rows lie in one page.
#include <type_traits>
#include <utility>

#include "stem_decode_common.h"

namespace stem {

// f(0), f(1), .. f(N - 1) with compile-time arguments
#define STEM_INLINE __attribute__((always_inline))
template <typename F, int... I>
__device__ __forceinline__ void for_each_constant(std::integer_sequence<int, I...>, F&& f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
    for_each_constant(std::make_integer_sequence<int, N>{}, f);
}
// Nothing is scheduled across this point.
#define STEM_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8_t;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

template <typename T>
__device__ __forceinline__ f32x4_t product(u32x4_t a, u32x4_t b, f32x4_t c) {
    if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
template <typename T>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const f32x2_t f = {lo, hi};
    if constexpr (std::is_same_v<T, __bf16>) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2_t));
}
__device__ __forceinline__ float max3(float a, float b, float c) {   // ignores NaN
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

struct PrefixArgs {
    const uint16_t *q, *prefix_k, *prefix_v, *k_pages, *v_pages;
    const int32_t *table, *lens, *cu_new;
    void* out;
    float *lse, *part_o;
    float2* part_ml;
    float scale_log2;                                  // softmax_scale * log2(e)
    int32_t Hq, Hkv, G, tokens, requests, max_new, rows;   // rows: tokens * G
    int32_t prefix_len, split_keys, prefix_splits, row_tiles;
    int32_t max_suffix, suffix_splits, suffix_row_tiles;
    int32_t table_row, page_shift, num_pages;
    int32_t prefix_groups, groups;                     // workgroups of the prefix, and with those of the own keys
    bool own_by_rows;                                  // how the latter are counted: PrefixPlan
    int64_t q_st, q_sh, p_st, p_sh, page_st, tok_st, head_st;
};

// First row of request r's new tokens, within the call's tokens.
__device__ __forceinline__ int first_token(const PrefixArgs& a, int r) { return a.cu_new ? min(max(a.cu_new[r], 0), a.tokens) : r; }
// New tokens of request r: the first and their number, within the call's tokens.
__device__ __forceinline__ void new_tokens(const PrefixArgs& a, int r, int& first, int& n) {
    if (a.cu_new) {
        const int lo = a.cu_new[r], hi = a.cu_new[r + 1];
        first = min(max(lo, 0), a.tokens);
        n = max(min(hi, a.tokens) - first, 0);
    } else {
        first = r;
        n = 1;
    }
}
// The last of 0 .. count - 1 whose key is at most x, -1 if there is none; keys ascend.  The whole wave looks for one x, 64 keys at a time:
// one load for 64 requests, three for 65536, instead of one after the other.
template <typename Key>
__device__ __forceinline__ int last_at_most(int count, int64_t x, Key key) {
    const int lane = threadIdx.x & 63;
    int from = 0;
    while (count > 64) {
        const int step = (count + 63) / 64, i = lane * step;
        const uint64_t below = __builtin_amdgcn_ballot_w64(i < count && key(from + i) <= x);
        if (!below) return -1;
        const int at = (63 - __builtin_clzll(below)) * step;
        from += at;
        count = min(step, count - at);
    }
    const uint64_t below = __builtin_amdgcn_ballot_w64(lane < count && key(from + lane) <= x);
    return below ? from + 63 - __builtin_clzll(below) : -1;
}
// A launch's workgroups are numbered along lines of 2^20, of which a grid has more than one if there are very many.  (A constant: the grid's
// size would be one more load that every workgroup waits for.)  There are at most 2^31 - 2^20, which whole lines do not bring beyond 2^31.
constexpr int kLineBits = 20;
__device__ __forceinline__ uint32_t group_number() { return (blockIdx.y << kLineBits) + blockIdx.x; }
__device__ __forceinline__ int suffix_len(const PrefixArgs& a, int r) {
    return a.max_suffix > 0 ? min(max(a.lens[r], 0), a.max_suffix) : 0;
}

constexpr float kNone = -3e38f;                        // reference of a row that has met no key: below any score, and finite
// A reference moves to where the largest weight is 2^lift, when one passes 2^(lift + 8).  In fp16 weights begin to lose bits below 2^-14: a
// lift of 7 keeps those down to 2^-21 of the largest whole, and 2^15 is within the type.
template <typename T> constexpr float kLift = std::is_same_v<T, _Float16> ? 7.f : 0.f;
template <typename T> constexpr float kMost = kLift<T> + 8.f;

typedef __attribute__((address_space(4))) const int32_t const_i32_t;

// Cache policy of a load that nothing else on the chip will repeat: 128K keys of 8 KV heads for 16 / 32 / 64 rows 104.9 / 102.5 / 108.8 us
// without, 91.1 / 92.9 / 99.4 with it (5.1 and 5.9 TB/s); with 128 rows and more, whose row tiles share K and V in an L2, 161 and 162.
constexpr int kStreaming = 2;

// Every wave's reads and writes of LDS are done, and then all waves go on.  (Not __syncthreads, whose fence would wait for the loads
// that are on their way to registers.)
#define STEM_LDS_BARRIER() asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory")

// Four values of a row's output from their sums, and (with the first four) its lse.
template <typename T>
__device__ __forceinline__ void write_row(const PrefixArgs& a, int token, int head, int at, f32x4_t o, float l, float m) {
    const bool empty = l == 0.f;
    const float inv = empty ? 0.f : 1.f / l;
    uint2 packed;
    packed.x = pack<T>(o[0] * inv, o[1] * inv);
    packed.y = pack<T>(o[2] * inv, o[3] * inv);
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + (int64_t)token * a.q_st + (int64_t)head * a.q_sh)[at] = packed;
    if (a.lse && at == 0)
        a.lse[(int64_t)head * a.tokens + token] = empty ? -__builtin_huge_valf() : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// How the waves of a workgroup share its rows and keys: RW groups of 16 NQ rows times KW groups of 32 keys.  With RW = 1 every wave has
// keys of its own and waits for no other; with RW > 1 the tile of 32 KW keys in LDS is read by RW waves each, and there are two
// of them in turn, with a barrier per tile.
template <int NQ_, int RW_, int KW_>
struct Split {
    static constexpr int NQ = NQ_, RW = RW_, KW = KW_, kWaves = RW * KW, kRows = 16 * NQ * RW, kKeys = 32 * KW;
};

template <typename T, int D, typename S>
struct Part {
    static constexpr int NQ = S::NQ, RW = S::RW, KW = S::KW, kWaves = S::kWaves;
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kKS = D / 32;                 // 32-wide steps of S^T along d
    static constexpr int kDT = D / 16;                 // 16-column tiles of O^T
    static constexpr int kTileBytes = S::kKeys * kRowBytes;   // of K, or of V
    // tiles of K, and of V, in LDS
    static constexpr int kBuffers = RW > 1 ? 2 : 1;
    static constexpr int kLdsTiles = 2 * kBuffers * kTileBytes, kLdsJoin = KW > 1 ? KW * S::kRows * D * 4 : 0;
    static constexpr int kLds = kLdsTiles > kLdsJoin ? kLdsTiles : kLdsJoin;
    // rows of K and V that a wave fetches of a tile, in pieces of at most 16 (which lie in one page), 1 KiB per load
    static constexpr int kMyRows = 32 / RW, kPieces = kMyRows > 16 ? 2 : 1, kPieceRows = kMyRows / kPieces;
    static constexpr int kRowsPerLoad = 1024 / kRowBytes, kLoads = kPieceRows / kRowsPerLoad;
    static_assert(kLoads >= 1, "a whole load per piece");

    using Rows = u32x4_t[kPieces][kLoads];             // a wave's rows of K or V, on their way

    bool idle;                                         // no row of the wave's is one
    u32x4_t q[NQ][kKS];
    f32x4_t o[kDT][NQ];
    float off[NQ], l[NQ];                              // minus the reference, in powers of two; sum of the lane's keys

    static __device__ __forceinline__ int k_swz(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int v_swz(int row) { return D == 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ int row_group() { return RW == 1 ? 0 : wave() % RW; }
    static __device__ __forceinline__ int key_group() { return RW == 1 ? wave() : wave() / RW; }
    // first row of the tile that this wave fetches
    static __device__ __forceinline__ int my_row() { return wave() * kMyRows; }

    // Row m of a KV head is token first + m / G, head m % G of the group; m0 is the workgroup's first.
    __device__ __forceinline__ void load_q(const uint16_t* base, int64_t st, int64_t sh, int first, int G, int m0, int m_end) {
        const int lane = threadIdx.x & 63;
        idle = m0 + 16 * NQ * row_group() >= m_end;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int m = min(m0 + 16 * (NQ * row_group() + n) + (lane & 15), m_end - 1), t = m / G;   // rows past the end repeat the last
            const uint16_t* row = base + (int64_t)(first + t) * st + (int64_t)(m - t * G) * sh + 8 * (lane >> 4);
#pragma unroll
            for (int ks = 0; ks < kKS; ++ks) q[n][ks] = *reinterpret_cast<const u32x4_t*>(row + 32 * ks);
            off[n] = -kNone;
            l[n] = 0.f;
#pragma unroll
            for (int x = 0; x < kDT; ++x) o[x][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // Asks for a piece of this wave's rows, from `first` bytes behind the resource's begin on; what lies behind its end becomes zeros.
    static __device__ __forceinline__ void fetch(u32x4_t (&in)[kLoads], __amdgpu_buffer_rsrc_t rsrc, uint32_t row_bytes, uint32_t first) {
        const int lane = threadIdx.x & 63;
        constexpr int kChunks = D / 8;
        const uint32_t at = lane / kChunks * row_bytes + lane % kChunks * 16;
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
            in[u] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, first + u * kRowsPerLoad * row_bytes, kKept ? 0 : kStreaming);
    }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_resource(const uint16_t* base, uint32_t row_bytes, int rows) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, rows > 0 ? (int)((rows - 1) * row_bytes) + kRowBytes : 0,
                                                 0x00020000);
    }

    // With 128 rows, where instructions count, the byte offsets in LDS that a lane uses in every tile are kept in registers (82 -> 51 vector
    // instructions of a step beside products and exponentials), and so are the operands of the next S^T, read a step ahead.  With
    // fewer rows memory is what counts, and a wave, which has more rows of K and V on their way, has no registers left for them.
    static constexpr bool kKept = RW == 4;
    int k_read[kKS], v_read[kDT], k_write[kPieces * kLoads], v_write[kPieces * kLoads];
    __device__ __forceinline__ void place() {
        const int lane = threadIdx.x & 63, c16 = lane & 15, grp = lane >> 4, row = 4 * grp + (c16 >> 2);
        constexpr int kChunks = D / 8;
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) {
            k_read[ks] = (key_group() * 32 + c16) * kRowBytes + (((4 * ks + grp) ^ k_swz(c16)) << 4);
            if constexpr (kKept) asm("" : "+v"(k_read[ks]));
        }
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
            v_read[dt] = (key_group() * 32 + row) * kRowBytes + (((2 * dt + ((c16 >> 1) & 1)) ^ v_swz(row)) << 4) + (c16 & 1) * 8;
            if constexpr (kKept) asm("" : "+v"(v_read[dt]));
        }
#pragma unroll
        for (int u = 0; u < kPieces * kLoads; ++u) {
            const int w_row = my_row() + u * kRowsPerLoad + lane / kChunks, c = lane % kChunks;
            k_write[u] = w_row * kRowBytes + ((c ^ k_swz(w_row)) << 4);
            v_write[u] = w_row * kRowBytes + ((c ^ v_swz(w_row)) << 4);
            if constexpr (kKept) asm("" : "+v"(k_write[u]), "+v"(v_write[u]));
        }
    }

    // What has been asked for -> LDS.  The 16-byte chunks of a row are exchanged within it (swz), which spreads the rows that are read
    // together over the banks.
    template <bool V>
    __device__ __forceinline__ void store(unsigned char* lds, const Rows& in, int u) const {
        *reinterpret_cast<u32x4_t*>(lds + (V ? v_write[u] : k_write[u])) = in[u / kLoads][u % kLoads];
    }
    template <bool V>
    __device__ __forceinline__ void store_all(unsigned char* lds, const Rows& in) const {
#pragma unroll
        for (int u = 0; u < kPieces * kLoads; ++u) store<V>(lds, in, u);
    }

    // Operand m of S^T of this wave's 32 keys: 16 keys m % 2 of them (in turn, as a product waits for the one before it in the same
    // registers), 32-wide step m / 2 along d.
    __device__ __forceinline__ u32x4_t load_k(const unsigned char* k_lds, int m) const {
        return *reinterpret_cast<const u32x4_t*>(k_lds + k_read[m >> 1] + (m & 1) * 16 * kRowBytes);
    }
    // Operand dt of O^T: 16 columns of the wave's 32 rows of V, in two transposing reads.
    __device__ __forceinline__ u32x4_t load_v(const unsigned char* v_lds, int dt) const {
        const unsigned char* p = v_lds + v_read[dt];
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)p);
        const s16x4_t up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(p + 16 * kRowBytes));
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, up);
        return u32x4_t{a.x, a.y, b.x, b.y};
    }

    using Scores = f32x4_t[2][NQ];                     // [16 keys][query tile], or exponents

    __device__ __forceinline__ void exponents_of(Scores& f, const Scores& s, int n, float scale_log2) const {
#pragma unroll
        for (int x = 0; x < 8; ++x) f[x >> 2][n][x & 3] = __builtin_fmaf(s[x >> 2][n][x & 3], scale_log2, off[n]);
    }
    static __device__ __forceinline__ float largest(const Scores& s, int n) {
        return max3(max3(s[0][n][0], s[0][n][1], s[0][n][2]), max3(s[0][n][3], s[1][n][0], s[1][n][1]),
                    max3(s[1][n][2], s[1][n][3], s[1][n][2]));
    }

    // The exponents f of scores s (powers of two over the reference) are to be at most kMost: where one passes it the reference moves,
    // and what has been summed up is scaled.  edge: key x of query n's column counts only if seen(n, x).
    template <typename Seen>
    __device__ __forceinline__ void keep_in_range(Scores& f, Scores& s, float scale_log2, bool edge, Seen seen) {
        float high = largest(f, 0);
#pragma unroll
        for (int n = 1; n < NQ; ++n) high = max3(high, largest(f, n), high);
        if (__builtin_expect(!edge & (__builtin_amdgcn_ballot_w64(high > kMost<T>) == 0), 1)) return;
        const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            if (edge) {
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (!seen(n, (x >> 2) * 16 + 4 * grp + (x & 3))) s[x >> 2][n][x & 3] = -__builtin_huge_valf();
            }
            // the largest of the raw scores: beside the first reference an exponent says nothing
            float raw = largest(s, n);
            raw = fmaxf(raw, __shfl_xor(raw, 16));
            raw = fmaxf(raw, __shfl_xor(raw, 32));      // the same in the column's four lanes
            if (__builtin_fmaf(raw, scale_log2, off[n]) > kMost<T>) {
                const float then = off[n];
                off[n] = __builtin_fmaf(-raw, scale_log2, kLift<T>);
                const float corr = __builtin_amdgcn_exp2f(off[n] - then);
                l[n] *= corr;
#pragma unroll
                for (int dt = 0; dt < kDT; ++dt) o[dt][n] *= corr;
            }
            exponents_of(f, s, n, scale_log2);
        }
    }

    // Weight x of a lane's 8 NQ (key x % 8 of query tile x / 8): 2^exponent, into its sum and its place in P^T.
    // The sum takes it as it is; P^T has it in the inputs' type (off by half a step at most), which is what a matrix instruction reads: more
    // bits would take a second product for what the first leaves.  Beside a key that has most of a row the roundings do not show, among many
    // alike they are as large as the output's own: relative error of bf16 rows of 32K keys 2.06e-3 against 1.67e-3 with weights in 32 bits,
    // fp16 2.54e-4 against 2.05e-4.
    __device__ __forceinline__ void weight(Scores& f, u32x4_t (&p)[NQ], int x) {
        const int n = x >> 3, y = x & 7;
        f[y >> 2][n][y & 3] = __builtin_amdgcn_exp2f(f[y >> 2][n][y & 3]);
        if (y & 1) {
            const float a = f[y >> 2][n][(y & 3) - 1], b = f[y >> 2][n][y & 3];
            l[n] += a + b;
            p[n][y >> 1] = pack<T>(a, b);
        }
    }

    // All tiles of S::kKeys keys.  ask_k(rows, t) and ask_v ask for a tile (one that does not exist gives zeros); edge(t) says whether
    // seen(t, n, x) has to be asked for this wave's keys.
    // Step t forms the weights of tile t and uses them, and the scores of tile t + 1, whose operands it begins with.  Under the products of
    // S^T go the operands of O^T and the weights (the last four of the second query tile under the first tile's products of O^T); under
    // those of O^T the next tile's rows -> LDS, the loads of the one after, a barrier, the operands of the next S^T and the next exponents.
    // So matrix and vector instructions, LDS and waits lie beside each other all along.
    template <typename AskK, typename AskV, typename Edge, typename Seen>
    __device__ __forceinline__ void walk(int tiles, unsigned char* lds, float scale_log2, AskK ask_k, AskV ask_v, Edge edge, Seen seen) {
        constexpr int kS = 2 * kKS;                        // operands of S^T; those of O^T are kDT, as many
        constexpr int kRows = kPieces * kLoads;            // writes of K, and of V
        const f32x4_t zero4 = {0.f, 0.f, 0.f, 0.f};
        auto k_at = [&](int t) STEM_INLINE { return lds + t % kBuffers * kTileBytes; };
        auto v_at = [&](int t) STEM_INLINE { return lds + (kBuffers + t % kBuffers) * kTileBytes; };
        auto barrier = []() STEM_INLINE {
            if constexpr (RW > 1) STEM_LDS_BARRIER();
        };
        place();
        Rows a, b;
        if (RW > 1 && idle) {                              // all of the wave's rows lie behind the last: its share of the loads is all it does
            ask_k(a, 0);
            ask_k(b, 1);
            store_all<false>(k_at(0), a);
            ask_v(a, 0);
            barrier();
            store_all<false>(k_at(1), b);
            store_all<true>(v_at(0), a);
            ask_k(a, 2);
            ask_v(b, 1);
            barrier();
            for (int t = 0; t + 1 < tiles; ++t) {
                store_all<false>(k_at(t + 2), a);
                store_all<true>(v_at(t + 1), b);
                ask_k(a, t + 3);
                ask_v(b, t + 2);
                barrier();
            }
            return;
        }
        Scores f, s;
        u32x4_t k[kS];
        ask_k(a, 0);
        ask_k(b, 1);
        store_all<false>(k_at(0), a);
        ask_v(a, 0);
        barrier();
        unrolled<kS>([&](auto m) STEM_INLINE { k[m] = load_k(k_at(0), m); });
        unrolled<kS>([&](auto m) STEM_INLINE {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[m & 1][n] = product<T>(k[m], q[n][m >> 1], m < 2 ? zero4 : s[m & 1][n]);
        });
#pragma unroll
        for (int n = 0; n < NQ; ++n) exponents_of(f, s, n, scale_log2);
        keep_in_range(f, s, scale_log2, edge(0), [&](int n, int x) { return seen(0, n, x); });
        store_all<false>(k_at(1), b);
        store_all<true>(v_at(0), a);
        ask_k(a, 2);
        ask_v(b, 1);
        barrier();
        if constexpr (kKept) unrolled<kS>([&](auto m) STEM_INLINE { k[m] = load_k(k_at(1), m); });
        auto step = [&](int t, auto j) STEM_INLINE {       // j: t modulo 2
            constexpr int kEarly = 8 * NQ - 4 * (NQ - 1);  // weights under S^T
            u32x4_t v[kDT], p[NQ];
            if constexpr (!kKept) unrolled<kS>([&](auto m) STEM_INLINE { k[m] = load_k(k_at(j + 1), m); });
            __builtin_amdgcn_s_setprio(1);
            STEM_SCHED_FENCE();
            unrolled<kS>([&](auto m_tag) STEM_INLINE {
                constexpr int m = decltype(m_tag)::value;
                v[m] = load_v(v_at(j), m);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[m & 1][n] = product<T>(k[m], q[n][m >> 1], m < 2 ? zero4 : s[m & 1][n]);
#pragma unroll
                for (int x = m * kEarly / kS; x < (m + 1) * kEarly / kS; ++x) weight(f, p, x);
                STEM_SCHED_FENCE();
            });
            constexpr int kProducts = kDT * NQ, kHalf = kProducts / 2;
            unrolled<kProducts>([&](auto y_tag) STEM_INLINE {
                constexpr int y = decltype(y_tag)::value, n = y / kDT, dt = y % kDT;
                o[dt][n] = product<T>(v[dt], p[n], o[dt][n]);
                if constexpr (n + 1 < NQ) {
#pragma unroll
                    for (int x = dt * 4 / kDT; x < (dt + 1) * 4 / kDT; ++x) weight(f, p, kEarly + x);
                }
#pragma unroll
                for (int x = dt * 8 / kDT; x < (dt + 1) * 8 / kDT; ++x)
                    f[x >> 2][n][x & 3] = __builtin_fmaf(s[x >> 2][n][x & 3], scale_log2, off[n]);
                if constexpr (y < kHalf) {
#pragma unroll
                    for (int u = y * 2 * kRows / kHalf; u < (y + 1) * 2 * kRows / kHalf; ++u) {
                        if (u < kRows) store<false>(k_at(j + 2), a, u);
                        else store<true>(v_at(j + 1), b, u - kRows);
                    }
                    if constexpr (y == kHalf - 1) {
                        ask_k(a, t + 3);
                        ask_v(b, t + 2);
                        barrier();
                    }
                } else if constexpr (kKept) {
#pragma unroll
                    for (int m = (y - kHalf) * kS / (kProducts - kHalf); m < (y + 1 - kHalf) * kS / (kProducts - kHalf); ++m)
                        k[m] = load_k(k_at(j + 2), m);
                }
                STEM_SCHED_FENCE();
            });
            __builtin_amdgcn_s_setprio(0);
            keep_in_range(f, s, scale_log2, edge(t + 1), [&](int n, int x) { return seen(t + 1, n, x); });
        };
        constexpr int kUnroll = RW > 1 ? 2 : 1;
        int t = 0;
        for (; t + kUnroll < tiles; t += kUnroll) unrolled<kUnroll>([&](auto j) STEM_INLINE { step(t + j, j); });
        if constexpr (kUnroll == 2)
            if (t + 1 < tiles) {
                step(t, std::integral_constant<int, 0>{});
                ++t;
            }
        u32x4_t p[NQ];
        unrolled<8 * NQ>([&](auto x) STEM_INLINE { weight(f, p, x); });
        unrolled<kDT>([&](auto dt) STEM_INLINE {
            const u32x4_t v = load_v(v_at(t), dt);
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[dt][n] = product<T>(v, p[n], o[dt][n]);
        });
    }

    // The waves' results together -> the rows' outputs, where there are no other parts.  Row m0 of m_end is row m0 of token `first`.
    __device__ __forceinline__ void finish_rows(unsigned char* lds, float2* wave_ml, const PrefixArgs& a, int first, int g, int m0, int m_end) {
        const int lane = threadIdx.x & 63, c16 = lane & 15, grp = lane >> 4, kw = key_group(), row0 = 16 * NQ * row_group();
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (grp == 0) wave_ml[kw * S::kRows + row0 + 16 * n + c16] = make_float2(-off[n], l[n]);
        }
        __syncthreads();                               // every wave is done with its tiles
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = row0 + 16 * n + c16;
            float m = wave_ml[row].x;
#pragma unroll
            for (int v = 1; v < KW; ++v) m = fmaxf(m, wave_ml[v * S::kRows + row].x);
            const float mine = __builtin_amdgcn_exp2f(-off[n] - m);
            float* dst = reinterpret_cast<float*>(lds) + (kw * S::kRows + row) * D + 4 * grp;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(dst + 16 * dt) = o[dt][n] * mine;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < S::kRows * D / 4; x += 64 * kWaves) {
            const int row = x / (D / 4), at = x % (D / 4);
            if (m0 + row >= m_end) break;
            float m = wave_ml[row].x, sum = 0.f;
#pragma unroll
            for (int v = 1; v < KW; ++v) m = fmaxf(m, wave_ml[v * S::kRows + row].x);
            f32x4_t all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < KW; ++v) {
                const float2 ml = wave_ml[v * S::kRows + row];
                sum += ml.y * __builtin_amdgcn_exp2f(ml.x - m);
                all += reinterpret_cast<const f32x4_t*>(lds)[v * S::kRows * D / 4 + x];
            }
            const int t = (m0 + row) / a.G;
            write_row<T>(a, first + t, g * a.G + m0 + row - t * a.G, at, all, sum, m);
        }
    }

    // The waves' results together -> the part's: rows m0 .. of at most m_end, at `part` (rows of D floats) and ml.
    __device__ __forceinline__ void finish(unsigned char* lds, float2* wave_ml, float* part, float2* ml, int m0, int m_end) {
        const int lane = threadIdx.x & 63, c16 = lane & 15, grp = lane >> 4, kw = key_group(), row0 = 16 * NQ * row_group();
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
        }
        if constexpr (KW == 1) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int m = m0 + row0 + 16 * n + c16;
                if (m >= m_end) continue;
                if (grp == 0) ml[m] = make_float2(-off[n], l[n]);
#pragma unroll
                for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(part + (int64_t)m * D + 16 * dt + 4 * grp) = o[dt][n];
            }
            return;
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (grp == 0) wave_ml[kw * S::kRows + row0 + 16 * n + c16] = make_float2(-off[n], l[n]);
        __syncthreads();                               // every wave is done with its tiles
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = row0 + 16 * n + c16;
            float m = wave_ml[row].x;
#pragma unroll
            for (int v = 1; v < KW; ++v) m = fmaxf(m, wave_ml[v * S::kRows + row].x);
            const float mine = __builtin_amdgcn_exp2f(-off[n] - m);   // 1 if nothing has been met by any wave
            if (kw == 0 && grp == 0 && m0 + row < m_end) {
                float sum = 0.f;
#pragma unroll
                for (int v = 0; v < KW; ++v) {
                    const float2 x = wave_ml[v * S::kRows + row];
                    sum += x.y * __builtin_amdgcn_exp2f(x.x - m);
                }
                ml[m0 + row] = make_float2(m, sum);
            }
            float* dst = reinterpret_cast<float*>(lds) + (kw * S::kRows + row) * D + 4 * grp;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(dst + 16 * dt) = o[dt][n] * mine;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < S::kRows * D / 4; x += 64 * kWaves) {
            if (m0 + x / (D / 4) >= m_end) break;
            f32x4_t sum = reinterpret_cast<const f32x4_t*>(lds)[x];
#pragma unroll
            for (int v = 1; v < KW; ++v) sum += reinterpret_cast<const f32x4_t*>(lds)[v * S::kRows * D / 4 + x];
            reinterpret_cast<f32x4_t*>(part)[(int64_t)m0 * (D / 4) + x] = sum;
        }
    }
};

// The prefix's keys key0 .. key0 + keys - 1 of KV head g.
template <typename S, typename P>
__device__ __forceinline__ void walk_prefix(P& t, const PrefixArgs& a, int g, int key0, int keys, unsigned char* lds) {
    const uint16_t* k = a.prefix_k + (int64_t)key0 * a.p_st + g * a.p_sh;
    const uint16_t* v = a.prefix_v + (int64_t)key0 * a.p_st + g * a.p_sh;
    const uint32_t row_bytes = (uint32_t)a.p_st * 2;
    const auto rk = P::rows_resource(k, row_bytes, keys), rv = P::rows_resource(v, row_bytes, keys);
    const int tiles = (keys + S::kKeys - 1) / S::kKeys;
    auto ask = [&](typename P::Rows& rows, __amdgpu_buffer_rsrc_t rsrc, int tile) STEM_INLINE {
        // behind the last tile there is nothing (and its offset is within 32 bits, which those further on need not be)
        const uint32_t first = (uint32_t)(min(tile, tiles) * S::kKeys + t.my_row()) * row_bytes;
#pragma unroll
        for (int x = 0; x < P::kPieces; ++x) t.fetch(rows[x], rsrc, row_bytes, first + x * P::kPieceRows * row_bytes);
    };
    const int left = keys - t.key_group() * 32;        // of this wave's keys in tile 0
    t.walk(
        tiles, lds, a.scale_log2, [&](auto& rows, int tile) STEM_INLINE { ask(rows, rk, tile); },
        [&](auto& rows, int tile) STEM_INLINE { ask(rows, rv, tile); }, [&](int tile) { return left - tile * S::kKeys < 32; },
        [&](int tile, int, int x) { return x < left - tile * S::kKeys; });
}

// Keys key0 .. key0 + keys - 1 of request r's `len` own, for rows m0 .. of its m_end (new tokens times heads of the group); n new tokens.
template <typename S, typename P>
__device__ __forceinline__ void walk_own(P& t, const PrefixArgs& a, int r, int g, int n, int len, int key0, int keys, int m0, int m_end,
                                         unsigned char* lds) {
    const int lane = threadIdx.x & 63;
    // keys of this part that the lane's columns see: those up to the token itself
    int sees[S::NQ];
#pragma unroll
    for (int x = 0; x < S::NQ; ++x)
        sees[x] = len - key0 - n + min(m0 + 16 * (S::NQ * t.row_group() + x) + (lane & 15), m_end - 1) / a.G + 1;
    const int least = min(len - key0 - n + m0 / a.G + 1, keys);   // of the workgroup's rows
    const_i32_t* row = (const_i32_t*)(a.table + (int64_t)r * a.table_row);
    const int mask = (1 << a.page_shift) - 1;
    auto page_of = [&](int key) {                      // -1: no key of this part, or no page of the cache's
        const int page = key < keys ? __builtin_amdgcn_readfirstlane(row[(key0 + key) >> a.page_shift]) : -1;
        return (uint32_t)page < (uint32_t)a.num_pages ? page : -1;
    };
    const uint32_t row_bytes = (uint32_t)a.tok_st * 2;
    auto ask = [&](typename P::Rows& rows, const uint16_t* pages, int tile) STEM_INLINE {
#pragma unroll
        for (int x = 0; x < P::kPieces; ++x) {
            const int key = tile * S::kKeys + t.my_row() + x * P::kPieceRows, page = page_of(key);
            const int64_t at_key = page < 0 ? 0 : (int64_t)page * a.page_st + (int64_t)((key0 + key) & mask) * a.tok_st + g * a.head_st;
            t.fetch(rows[x], P::rows_resource(pages + at_key, row_bytes, page < 0 ? 0 : min(keys - key, P::kPieceRows)), row_bytes, 0);
        }
    };
    bool lo = false, hi = false;                       // whether the halves of the wave's 32 keys are in a page
    t.walk(
        (keys + S::kKeys - 1) / S::kKeys, lds, a.scale_log2, [&](auto& rows, int tile) STEM_INLINE { ask(rows, a.k_pages, tile); },
        [&](auto& rows, int tile) STEM_INLINE { ask(rows, a.v_pages, tile); },
        [&](int tile) {
            const int key = tile * S::kKeys + t.key_group() * 32;
            lo = page_of(key) >= 0, hi = page_of(key + 16) >= 0;
            return !lo || !hi || key + 32 > least;
        },
        [&](int tile, int nq, int x) { return tile * S::kKeys + t.key_group() * 32 + x < sees[nq] && (x < 16 ? lo : hi); });
}

// SP: how the rows of the prefix are shared, SO: those of a request and its own keys.
template <typename T, int D, typename SP, typename SO>
__global__ __launch_bounds__(64 * SP::kWaves, D == 256 ? 1 : 2) void prefix_attn_kernel(PrefixArgs a) {
    static_assert(SP::kWaves == SO::kWaves, "one size of workgroup");
    using PartP = Part<T, D, SP>;
    using PartO = Part<T, D, SO>;
    __shared__ __align__(1024) unsigned char lds[PartP::kLds > PartO::kLds ? PartP::kLds : PartO::kLds];
    __shared__ float2 wave_ml[SP::kRows * SP::KW > SO::kRows * SO::KW ? SP::kRows * SP::KW : SO::kRows * SO::KW];
    const int id = (int)group_number();
    if (id >= a.groups) return;
    if (id < a.prefix_groups) {
        // row tiles of the same keys on one XCD (workgroup id modulo 8), one after the other: they share its L2
        const int x = id & 7, y = id >> 3, row_tile = y % a.row_tiles, combo = y / a.row_tiles * 8 + x;
        if (combo >= a.Hkv * a.prefix_splits) return;
        const int g = combo % a.Hkv, split = combo / a.Hkv, m0 = row_tile * SP::kRows;
        PartP t;
        t.load_q(a.q + (int64_t)g * a.G * a.q_sh, a.q_st, a.q_sh, 0, a.G, m0, a.rows);
        const int key0 = split * a.split_keys;
        walk_prefix<SP>(t, a, g, key0, min(a.split_keys, a.prefix_len - key0), lds);
        const int64_t place = ((int64_t)split * a.Hkv + g) * a.rows;
        t.finish(lds, wave_ml, a.part_o + place * D, a.part_ml + place, m0, a.rows);
        return;
    }
    // a request's own keys
    int at = id - a.prefix_groups;
    const int g = at % a.Hkv;
    at /= a.Hkv;
    const int split = at % a.suffix_splits, slot = at / a.suffix_splits;
    int r, row_tile;
    if (__builtin_expect(a.own_by_rows, 0)) {
        auto before = [&](int x) { return slot_before(x, (int64_t)first_token(a, x) * a.G, SO::kRows); };
        r = last_at_most(a.requests, slot, before);
        if (r < 0) return;
        row_tile = slot - (int)before(r);
    } else {
        r = slot / a.suffix_row_tiles;
        row_tile = slot - r * a.suffix_row_tiles;
    }
    int first, n;
    new_tokens(a, r, first, n);
    const int mine = min(n, a.max_new) * a.G;
    if ((int64_t)row_tile * SO::kRows >= mine) return;
    const int m0 = row_tile * SO::kRows;
    const int len = suffix_len(a, r);
    const int split_keys = suffix_split_keys(len, a.suffix_splits), key0 = split * split_keys, keys = min(len - key0, split_keys);
    if (keys <= 0) return;
    PartO t;
    t.load_q(a.q + (int64_t)g * a.G * a.q_sh, a.q_st, a.q_sh, first, a.G, m0, mine);
    walk_own<SO>(t, a, r, g, n, len, key0, keys, m0, mine, lds);
    const int64_t place = ((int64_t)(a.prefix_splits + split) * a.Hkv + g) * a.rows + (int64_t)first * a.G;
    t.finish(lds, wave_ml, a.part_o + place * D, a.part_ml + place, m0, mine);
}

// Small calls in one launch: a workgroup has all keys of its request's rows, the prefix's (which are read once per request then) and its own.
template <typename T, int D, typename S>
__global__ __launch_bounds__(64 * S::kWaves) void small_attn_kernel(PrefixArgs a) {
    using P = Part<T, D, S>;
    __shared__ __align__(1024) unsigned char lds[P::kLds];
    __shared__ float2 wave_ml[S::kRows * S::KW];
    const int g = blockIdx.x % a.Hkv, r = blockIdx.x / a.Hkv;
    int first, n;
    new_tokens(a, r, first, n);
    const int mine = min(n, a.max_new) * a.G;
    if (mine <= 0) return;
    P t;
    t.load_q(a.q + (int64_t)g * a.G * a.q_sh, a.q_st, a.q_sh, first, a.G, 0, mine);
    if (a.prefix_len > 0) walk_prefix<S>(t, a, g, 0, a.prefix_len, lds);
    const int len = suffix_len(a, r);
    if (len > 0) walk_own<S>(t, a, r, g, n, len, 0, len, 0, mine, lds);
    t.finish_rows(lds, wave_ml, a, first, g, 0, mine);
}

// Joins the parts of a row.  D / 4 lanes take four values each, GROUPS such groups of lanes every GROUPS-th part; all that a group reads
// at a time is asked for before any of it is used, as a row waits for memory and does next to nothing else.
constexpr int kJoinThreads = 256;
template <typename T, int D, int GROUPS, bool BY_ROWS>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(PrefixArgs a) {
    constexpr int kLanes = D / 4, kRows = kJoinThreads / (kLanes * GROUPS), kAtOnce = 4;
    __shared__ f32x4_t group_o[GROUPS > 1 ? kJoinThreads : 1];
    __shared__ float2 group_ml[GROUPS > 1 ? kRows * GROUPS : 1];
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes % GROUPS, my_row = threadIdx.x / (kLanes * GROUPS);
    const uint32_t item0 = group_number() * kRows, item = item0 + my_row;   // (2^31 and less than a line's more)
    int r = 0, i = 0, h = 0, first = 0, n = 0, parts = 0;
    bool mine = false;                                 // whether the row is one of a request's
    if constexpr (BY_ROWS) {                           // token, head
        constexpr int kWaveRows = GROUPS > 1 ? 1 : 64 / kLanes;   // different rows of a wave
        const uint32_t wave0 = GROUPS > 1 ? item0 : item0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kWaveRows;
        int known = -1, owner = -1;
#pragma unroll
        for (int x = 0; x < kWaveRows; ++x) {
            const uint32_t token = (wave0 + x) / (uint32_t)a.Hq;
            if (token >= (uint32_t)a.tokens) break;
            if ((int)token != known) owner = last_at_most(a.requests, token, [&](int y) { return (int64_t)first_token(a, y); });
            known = (int)token;
            if (item == wave0 + x) r = owner, i = known, h = (int)(item - token * (uint32_t)a.Hq), mine = owner >= 0;
        }
        if (mine) {
            new_tokens(a, r, first, n);
            i -= first;
            mine = i < min(n, a.max_new);
        }
    } else {                                           // request, new token, head
        const uint32_t per_request = (uint32_t)a.max_new * a.Hq, request = item / per_request;
        const int rest = (int)(item - request * per_request);
        i = rest / a.Hq, h = rest - i * a.Hq;
        if (request < (uint32_t)a.requests) {
            r = (int)request;
            new_tokens(a, r, first, n);
            mine = i < n;
        }
    }
    const int g = h / a.G;
    if (mine) parts = a.prefix_splits + suffix_parts(suffix_len(a, r), a.suffix_splits);
    const int64_t step = (int64_t)a.Hkv * a.rows, row = (int64_t)g * a.rows + (int64_t)(first + i) * a.G + (h - g * a.G);
    float m = kNone, l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = group; p0 < parts; p0 += kAtOnce * GROUPS) {
        float2 ml[kAtOnce];
        f32x4_t part[kAtOnce];
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            const int p = p0 + x * GROUPS;
            const int64_t at = (p < parts ? p : p0) * step + row;
            ml[x] = a.part_ml[at];
            part[x] = reinterpret_cast<const f32x4_t*>(a.part_o + at * D)[lane];
            if (p >= parts) ml[x] = make_float2(kNone, 0.f);
        }
        float top = m;
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) top = fmaxf(top, ml[x].x);
        const float then = __builtin_amdgcn_exp2f(m - top);
        l *= then;
        o *= then;
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            const float c = p0 + x * GROUPS < parts ? __builtin_amdgcn_exp2f(ml[x].x - top) : 0.f;
            l += c * ml[x].y;
            if (c != 0.f) o += c * part[x];            // (0 times a part that is not finite is nothing of this row's)
        }
        m = top;
    }
    if constexpr (GROUPS > 1) {
        group_o[threadIdx.x] = o;
        if (lane == 0) group_ml[my_row * GROUPS + group] = make_float2(m, l);
        __syncthreads();
        if (group > 0) return;
        float top = m;
#pragma unroll
        for (int x = 1; x < GROUPS; ++x) top = fmaxf(top, group_ml[my_row * GROUPS + x].x);
        const float mine = __builtin_amdgcn_exp2f(m - top);
        l *= mine;
        o *= mine;
#pragma unroll
        for (int x = 1; x < GROUPS; ++x) {
            const float2 other = group_ml[my_row * GROUPS + x];
            const float c = __builtin_amdgcn_exp2f(other.x - top);
            l += c * other.y;
            o += c * group_o[threadIdx.x + x * kLanes];
        }
        m = top;
    }
    if (!mine) return;
    write_row<T>(a, first + i, h, lane, o, l, m);
}

template <typename T, int D>
static int launch(const PrefixArgs& a, const PrefixPlan& p, hipStream_t stream) {
    constexpr int W = 4;
    using Rows16 = Split<1, 1, W>;
    using Rows32 = Split<1, 2, W / 2>;
    using Rows64 = Split<2, 2, W / 2>;
    using Rows128 = Split<2, 4, W / 4>;
    if constexpr (D != 256)
        if (p.small) {
            using Small = Split<1, 1, D == 64 ? 8 : 4>;
            hipLaunchKernelGGL((small_attn_kernel<T, D, Small>), dim3((unsigned)(a.requests * a.Hkv)), dim3(64 * Small::kWaves), 0, stream, a);
            return check_launch();
        }
    // several groups of lanes per row where there are parts for them
    constexpr int kGroups = 4 * kJoinThreads / D;
    const bool many = p.prefix_splits + p.suffix_splits > 4;
    // (a line of a grid has less than 2^32 threads, and where there are lines each begins with a workgroup of XCD 0)
    constexpr int64_t kLine = 1 << kLineBits;
    auto grid_of = [](int64_t n) { return n <= kLine ? dim3((unsigned)n) : dim3((unsigned)kLine, (unsigned)((n + kLine - 1) >> kLineBits)); };
    const dim3 grid = grid_of(p.groups), joins = grid_of(many ? p.join_rows : (p.join_rows + kGroups - 1) / kGroups);
    if (p.groups > 0) {
#define STEM_PREFIX_LAUNCH(SP, SO) \
    hipLaunchKernelGGL((prefix_attn_kernel<T, D, SP, SO>), grid, dim3(64 * SP::kWaves), 0, stream, a)
        const bool few = p.suffix_row_tile == 16;
        if (p.row_tile == 16) STEM_PREFIX_LAUNCH(Rows16, Rows16);
        else if (p.row_tile == 32 && few) STEM_PREFIX_LAUNCH(Rows32, Rows16);
        else if (p.row_tile == 32) STEM_PREFIX_LAUNCH(Rows32, Rows64);
        else if (p.row_tile == 64 && few) STEM_PREFIX_LAUNCH(Rows64, Rows16);
        else if (p.row_tile == 64) STEM_PREFIX_LAUNCH(Rows64, Rows64);
        else if (few) STEM_PREFIX_LAUNCH(Rows128, Rows16);
        else STEM_PREFIX_LAUNCH(Rows128, Rows64);
#undef STEM_PREFIX_LAUNCH
        if (const int st = check_launch()) return st;
    }
#define STEM_JOIN_LAUNCH(GROUPS, BY_ROWS) hipLaunchKernelGGL((join_kernel<T, D, GROUPS, BY_ROWS>), joins, dim3(kJoinThreads), 0, stream, a)
    if (many && p.join_by_rows) STEM_JOIN_LAUNCH(kGroups, true);
    else if (many) STEM_JOIN_LAUNCH(kGroups, false);
    else if (p.join_by_rows) STEM_JOIN_LAUNCH(1, true);
    else STEM_JOIN_LAUNCH(1, false);
#undef STEM_JOIN_LAUNCH
    return check_launch();
}

int launch_prefix_attn(const PrefixCall& c, hipStream_t stream) {
    const stem_prefix_shape& s = c.shape;
    const PrefixPlan& p = c.plan;
    PrefixArgs a = {};
    a.q = static_cast<const uint16_t*>(c.q);
    a.prefix_k = static_cast<const uint16_t*>(c.prefix_k);
    a.prefix_v = static_cast<const uint16_t*>(c.prefix_v);
    a.k_pages = static_cast<const uint16_t*>(c.k_pages);
    a.v_pages = static_cast<const uint16_t*>(c.v_pages);
    a.table = c.table, a.lens = c.lens, a.cu_new = c.cu_new;
    a.out = c.out, a.lse = c.lse;
    a.part_o = static_cast<float*>(c.workspace);
    a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(c.workspace) + p.partial_ml);
    a.scale_log2 = c.softmax_scale * 1.4426950408889634f;
    a.Hq = s.num_q_heads, a.Hkv = s.num_kv_heads, a.G = a.Hq / a.Hkv;
    a.tokens = s.tokens, a.requests = s.requests, a.max_new = s.max_new, a.rows = a.tokens * a.G;
    a.prefix_len = s.prefix_len, a.split_keys = p.split_keys, a.prefix_splits = p.prefix_splits, a.row_tiles = p.row_tiles;
    a.max_suffix = s.max_suffix, a.suffix_splits = p.suffix_splits, a.suffix_row_tiles = p.suffix_row_tiles;
    a.table_row = s.pages_per_request;
    a.page_shift = s.max_suffix > 0 ? __builtin_ctz(s.pages.page_size) : 0;
    a.num_pages = s.pages.num_pages;
    a.prefix_groups = (int32_t)p.prefix_groups, a.groups = (int32_t)p.groups;
    a.own_by_rows = p.own_by_rows;
    a.q_st = s.q_stride_token, a.q_sh = s.q_stride_head, a.p_st = s.prefix_stride_token, a.p_sh = s.prefix_stride_head;
    a.page_st = s.pages.stride_page, a.tok_st = s.pages.stride_token, a.head_st = s.pages.stride_head;
    if (s.dtype == STEM_BF16) {
        if (s.head_dim == 64) return launch<__bf16, 64>(a, p, stream);
        if (s.head_dim == 128) return launch<__bf16, 128>(a, p, stream);
        return launch<__bf16, 256>(a, p, stream);
    }
    if (s.head_dim == 64) return launch<_Float16, 64>(a, p, stream);
    if (s.head_dim == 128) return launch<_Float16, 128>(a, p, stream);
    return launch<_Float16, 256>(a, p, stream);
}

}  // namespace stem
