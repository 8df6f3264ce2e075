// Attention of many short rows to one long prefix that they share, and of each request's rows to its own pages behind it.
//
// With Q the rows (token, query head of the group) of one KV head,
//     o = softmax(scale Q [Kp; Ks]^T) [Vp; Vs]
// is computed in parts over the keys: a part leaves its largest score m, its sum l = sum e^(s - m) and its o = sum e^(s - m) v, and
//     o = sum_p e^(m_p - m) o_p / sum_p e^(m_p - m) l_p,  m = max_p m_p
// joins them (join_kernel).  The prefix is one dense product of all requests' rows together, so K and V of the prefix are read once
// for all of them; the keys are split so that every CU has a part.
//
// A workgroup's waves share the rows and take turns over tiles of 32 keys, each wave with tiles, softmax and o of its own, joined at its
// end through LDS: no barrier while keys go by.  Products and softmax are those of stage 3: S^T = K Q^T, so that one query is one lane's
// column and its softmax needs no exchange but at its start and when its reference moves; P^T lies in the registers as the second
// product O^T += V^T P^T takes it, V^T comes from row-major V by transposing LDS reads.
//
// K and V go from global memory straight into LDS (one tile ahead), 16 keys per buffer resource: its size ends with the last valid
// row, so that rows behind it, and all of a page that is none, arrive as zeros and are masked.  A tile of 32 keys begins at a multiple
// of 32, so each of its halves lies in one page.
#include <type_traits>

#include "stem_decode_common.h"

namespace stem {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8_t;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// s_waitcnt with only vmcnt set (bits [3:0] and [15:14])
#define STEM_WAIT_VMCNT(N) __builtin_amdgcn_s_waitcnt(0x0F70 | ((N) & 15) | (((N) >> 4) << 14))

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
    int32_t prefix_groups;                             // workgroups of the prefix
    int64_t q_st, q_sh, p_st, p_sh, page_st, tok_st, head_st;
};

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
__device__ __forceinline__ int suffix_len(const PrefixArgs& a, int r) {
    return a.max_suffix > 0 ? min(max(a.lens[r], 0), a.max_suffix) : 0;
}

constexpr float kNone = -3e38f;                        // reference of a row that has met no key: below any score, and finite
constexpr float kSlack = 8.f;                          // how far (in powers of two) scores may pass the reference before it moves

// Rows of a row tile: row m of the KV head is token first + m / G, head m % G of the group.
template <typename T, int D, int NQ, int WAVES>
struct RowTile {
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kKS = D / 32;                 // 32-wide steps of S^T along d
    static constexpr int kDT = D / 16;                 // 16-column tiles of O^T
    static constexpr int kHalfBytes = 16 * kRowBytes;  // 16 rows of K or V
    static constexpr int kStageBytes = 4 * kHalfBytes; // 32 keys of K, then of V
    static constexpr int kWaveBytes = 2 * kStageBytes;
    static constexpr int kRows = 16 * NQ;
    static constexpr int kRequests = kStageBytes / 1024;   // loads of 1 KiB per tile
    static constexpr int kPerHalf = kHalfBytes / 1024;

    u32x4_t q[NQ][kKS];
    f32x4_t o[kDT][NQ];
    float off[NQ], l[NQ];                              // minus the reference, in powers of two; sum of the lane's keys

    static __device__ __forceinline__ int k_swz(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int v_swz(int row) { return D == 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }

    __device__ __forceinline__ void load_q(const uint16_t* base, int64_t st, int64_t sh, int first, int G, int m0, int m_end) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int m = min(m0 + 16 * n + (lane & 15), m_end - 1), t = m / G;   // rows past the end repeat the last
            const uint16_t* row = base + (int64_t)(first + t) * st + (int64_t)(m - t * G) * sh + 8 * (lane >> 4);
#pragma unroll
            for (int ks = 0; ks < kKS; ++ks) q[n][ks] = *reinterpret_cast<const u32x4_t*>(row + 32 * ks);
            off[n] = -kNone;
            l[n] = 0.f;
#pragma unroll
            for (int x = 0; x < kDT; ++x) o[x][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // 16 rows of K or V -> LDS.  The 16-byte chunks of a row are exchanged within it (swz), which spreads the rows that are read together
    // over the banks; a lane fetches the chunk that belongs at its place.
    template <bool V>
    static __device__ __forceinline__ void fetch(const uint16_t* base, int64_t row_stride, int valid, unsigned char* lds) {
        const int lane = threadIdx.x & 63;
        constexpr int kChunks = D / 8, kRowsPerLoad = 64 / kChunks;
        const int bytes = valid > 0 ? (int)((valid - 1) * row_stride * 2) + kRowBytes : 0;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, bytes, 0x00020000);
#pragma unroll
        for (int u = 0; u < kPerHalf; ++u) {
            const int row = u * kRowsPerLoad + lane / kChunks, c = (lane % kChunks) ^ (V ? v_swz(row) : k_swz(row));
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_t*)(lds + u * 1024), 16,
                                                     (int)(row * row_stride * 2) + c * 16, 0, 0, 0);
        }
    }

    // One tile of 32 keys that is in LDS.  EDGE: key x of the lane's column counts if x < seen(n) and its half is there.
    template <bool EDGE, typename Seen>
    __device__ __forceinline__ void tile(const unsigned char* lds, float scale_log2, Seen seen) {
        const int lane = threadIdx.x & 63, c16 = lane & 15, grp = lane >> 4;
        f32x4_t s[2][NQ];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const unsigned char* row = lds + kt * kHalfBytes + c16 * kRowBytes;
#pragma unroll
            for (int ks = 0; ks < kKS; ++ks) {
                const u32x4_t k = *reinterpret_cast<const u32x4_t*>(row + (((ks * 4 + grp) ^ k_swz(c16)) << 4));
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    s[kt][n] = product<T>(k, q[n][ks], ks == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : s[kt][n]);
            }
        }
        u32x4_t p[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            if constexpr (EDGE) {
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (!seen(n, (x >> 2) * 16 + 4 * grp + (x & 3))) s[x >> 2][n][x & 3] = -__builtin_huge_valf();
            }
            float f[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] = __builtin_fmaf(s[x >> 2][n][x & 3], scale_log2, off[n]);
            const float high = max3(max3(f[0], f[1], f[2]), max3(f[3], f[4], f[5]), fmaxf(f[6], f[7]));
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(high > kSlack) != 0, 0)) {
                float top = fmaxf(high, __shfl_xor(high, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (top > kSlack) {                    // the same in the column's four lanes
                    const float then = off[n];
                    // the largest of the raw scores: from `high` it would be lost beside the first reference
                    float raw = max3(max3(s[0][n][0], s[0][n][1], s[0][n][2]), max3(s[0][n][3], s[1][n][0], s[1][n][1]),
                                     fmaxf(s[1][n][2], s[1][n][3]));
                    raw = fmaxf(raw, __shfl_xor(raw, 16));
                    raw = fmaxf(raw, __shfl_xor(raw, 32));
                    off[n] = -raw * scale_log2;
                    const float corr = __builtin_amdgcn_exp2f(off[n] - then);
                    l[n] *= corr;
#pragma unroll
                    for (int dt = 0; dt < kDT; ++dt) o[dt][n] *= corr;
#pragma unroll
                    for (int x = 0; x < 8; ++x) f[x] = __builtin_fmaf(s[x >> 2][n][x & 3], scale_log2, off[n]);
                }
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] = __builtin_amdgcn_exp2f(f[x]);
            l[n] += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
#pragma unroll
            for (int x = 0; x < 4; ++x) p[n][x] = pack<T>(f[2 * x], f[2 * x + 1]);
        }
        const unsigned char* v = lds + 2 * kHalfBytes;
        const int v_row = 4 * grp + (c16 >> 2);
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
            const unsigned char* at = v + v_row * kRowBytes + (((2 * dt + ((c16 >> 1) & 1)) ^ v_swz(v_row)) << 4) + (c16 & 1) * 8;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)at);
            const s16x4_t up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + kHalfBytes));
            const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, up);
            const u32x4_t vt = {a.x, a.y, b.x, b.y};
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[dt][n] = product<T>(vt, p[n], o[dt][n]);
        }
    }

    // The waves' results together -> the part's: rows m0 .. of at most m_end, at `part` (rows of D floats) and ml.
    __device__ __forceinline__ void finish(unsigned char* lds, float2* wave_ml, float* part, float2* ml, int m0, int m_end) {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c16 = lane & 15, grp = lane >> 4;
        __syncthreads();                               // every wave is done with its tiles
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (grp == 0) wave_ml[w * kRows + 16 * n + c16] = make_float2(-off[n], l[n]);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = 16 * n + c16;
            float m = wave_ml[row].x;
#pragma unroll
            for (int v = 1; v < WAVES; ++v) m = fmaxf(m, wave_ml[v * kRows + row].x);
            const float mine = __builtin_amdgcn_exp2f(-off[n] - m);   // 1 if nothing has been met by any wave
            if (w == 0 && grp == 0 && m0 + row < m_end) {
                float sum = 0.f;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    const float2 x = wave_ml[v * kRows + row];
                    sum += x.y * __builtin_amdgcn_exp2f(x.x - m);
                }
                ml[m0 + row] = make_float2(m, sum);
            }
            float* dst = reinterpret_cast<float*>(lds) + (w * kRows + row) * D + 4 * grp;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) *reinterpret_cast<f32x4_t*>(dst + 16 * dt) = o[dt][n] * mine;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < kRows * D / 4; x += 64 * WAVES) {
            const int row = x / (D / 4);
            if (m0 + row >= m_end) break;
            f32x4_t sum = reinterpret_cast<const f32x4_t*>(lds)[x];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) sum += reinterpret_cast<const f32x4_t*>(lds)[v * kRows * D / 4 + x];
            reinterpret_cast<f32x4_t*>(part)[(int64_t)m0 * (D / 4) + x] = sum;
        }
    }
};

// Tiles first, first + WAVES, .. before `end` (wave-uniform), one ahead.  fetch(tile, lds) asks for a tile, use(tile, lds) takes it.
template <int REQUESTS, int STAGE, int WAVES, typename Fetch, typename Use>
__device__ __forceinline__ void walk_tiles(int first, int end, unsigned char* lds, Fetch fetch, Use use) {
    if (first >= end) return;
    fetch(first, lds);
    int at = 0;
    for (int t = first; t < end; t += WAVES) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what was read from the other buffer is there
        if (t + WAVES < end) {
            fetch(t + WAVES, lds + (at ^ STAGE));
            STEM_WAIT_VMCNT(REQUESTS);
        } else {
            STEM_WAIT_VMCNT(0);
        }
        asm volatile("" ::: "memory");
        use(t, lds + at);
        at ^= STAGE;
    }
}

template <typename T, int D, int NQ, int NS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void prefix_attn_kernel(PrefixArgs a) {
    constexpr int kMost = NQ > NS ? NQ : NS;
    __shared__ __align__(1024) unsigned char lds[WAVES * RowTile<T, D, kMost, WAVES>::kWaveBytes];
    __shared__ float2 wave_ml[WAVES * 16 * kMost];
    static_assert(sizeof(lds) >= WAVES * 16 * kMost * D * sizeof(float), "the waves' results");
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = blockIdx.x;
    if (id < a.prefix_groups) {
        // row tiles of the same keys on one XCD (workgroup id modulo 8), one after the other: they share its L2
        const int x = id & 7, y = id >> 3, row_tile = y % a.row_tiles, combo = y / a.row_tiles * 8 + x;
        if (combo >= a.Hkv * a.prefix_splits) return;
        const int g = combo % a.Hkv, split = combo / a.Hkv;
        using Tile = RowTile<T, D, NQ, WAVES>;
        Tile t;
        const int m0 = row_tile * Tile::kRows;
        t.load_q(a.q + (int64_t)g * a.G * a.q_sh, a.q_st, a.q_sh, 0, a.G, m0, a.rows);
        const int key0 = split * a.split_keys, keys = min(a.split_keys, a.prefix_len - key0);
        const uint16_t* k = a.prefix_k + (int64_t)key0 * a.p_st + g * a.p_sh;
        const uint16_t* v = a.prefix_v + (int64_t)key0 * a.p_st + g * a.p_sh;
        walk_tiles<Tile::kRequests, Tile::kStageBytes, WAVES>(
            w, (keys + 31) / 32, lds + w * Tile::kWaveBytes,
            [&](int tile, unsigned char* to) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int key = tile * 32 + 16 * h, valid = min(max(keys - key, 0), 16);
                    t.template fetch<false>(k + key * a.p_st, a.p_st, valid, to + h * Tile::kHalfBytes);
                    t.template fetch<true>(v + key * a.p_st, a.p_st, valid, to + (2 + h) * Tile::kHalfBytes);
                }
            },
            [&](int tile, const unsigned char* from) {
                const int left = keys - tile * 32;
                if (left >= 32) t.template tile<false>(from, a.scale_log2, [](int, int) { return true; });
                else t.template tile<true>(from, a.scale_log2, [&](int, int x) { return x < left; });
            });
        const int64_t place = ((int64_t)split * a.Hkv + g) * a.rows;
        t.finish(lds, wave_ml, a.part_o + place * D, a.part_ml + place, m0, a.rows);
        return;
    }
    // a request's own keys
    using Tile = RowTile<T, D, NS, WAVES>;
    int at = id - a.prefix_groups;
    const int g = at % a.Hkv;
    at /= a.Hkv;
    const int row_tile = at % a.suffix_row_tiles;
    at /= a.suffix_row_tiles;
    const int split = at % a.suffix_splits, r = at / a.suffix_splits;
    int first, n;
    new_tokens(a, r, first, n);
    const int mine = min(n, a.max_new) * a.G, m0 = row_tile * Tile::kRows;
    if (m0 >= mine) return;
    const int len = suffix_len(a, r), tiles = (len + 31) / 32;
    const int each = suffix_split_tiles(tiles, a.suffix_splits, WAVES), tile0 = split * each;
    if (tile0 >= tiles) return;
    Tile t;
    t.load_q(a.q + (int64_t)g * a.G * a.q_sh, a.q_st, a.q_sh, first, a.G, m0, mine);
    const int lane = threadIdx.x & 63;
    // keys that the lane's columns see: those up to the token itself
    int sees[NS];
#pragma unroll
    for (int x = 0; x < NS; ++x) sees[x] = len - n + min(m0 + 16 * x + (lane & 15), mine - 1) / a.G + 1;
    const int least = len - n + m0 / a.G + 1;          // of the tile's rows
    const int32_t* row = a.table + (int64_t)r * a.table_row;
    uint32_t there = 0, there_next = 0;                // halves of the tile in use and of the one asked for that are in a page
    auto fetch = [&](int tile, unsigned char* to) {
        there = there_next;
        there_next = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = tile * 32 + 16 * h;
            int valid = min(max(len - key, 0), 16);
            const int page = valid > 0 ? __builtin_amdgcn_readfirstlane(row[key >> a.page_shift]) : -1;
            if ((uint32_t)page >= (uint32_t)a.num_pages) valid = 0;
            if (valid > 0) there_next |= 1u << h;
            const int64_t at_key = valid > 0 ? (int64_t)page * a.page_st + (int64_t)(key & ((1 << a.page_shift) - 1)) * a.tok_st + g * a.head_st : 0;
            t.template fetch<false>(a.k_pages + at_key, a.tok_st, valid, to + h * Tile::kHalfBytes);
            t.template fetch<true>(a.v_pages + at_key, a.tok_st, valid, to + (2 + h) * Tile::kHalfBytes);
        }
    };
    walk_tiles<Tile::kRequests, Tile::kStageBytes, WAVES>(
        tile0 + w, min(tile0 + each, tiles), lds + w * Tile::kWaveBytes, fetch,
        [&](int tile, const unsigned char* from) {
            const bool last = tile + WAVES >= min(tile0 + each, tiles);   // then nothing has been asked for behind it
            const uint32_t have = last ? there_next : there;
            if (have == 3u && tile * 32 + 32 <= least) t.template tile<false>(from, a.scale_log2, [](int, int) { return true; });
            else t.template tile<true>(from, a.scale_log2, [&](int nq, int x) { return tile * 32 + x < sees[nq] && (have >> (x >> 4) & 1u); });
        });
    const int64_t place = ((int64_t)(a.prefix_splits + split) * a.Hkv + g) * a.rows + (int64_t)first * a.G;
    t.finish(lds, wave_ml, a.part_o + place * D, a.part_ml + place, m0, mine);
}

// Joins the parts of a row: D / 4 lanes per row, four values each.
constexpr int kJoinThreads = 256;
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(PrefixArgs a) {
    constexpr int kLanes = D / 4, kRows = kJoinThreads / kLanes;
    const int64_t item = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;   // request, new token, head
    const int per_request = a.max_new * a.Hq;
    const int64_t r = item / per_request;
    if (r >= a.requests) return;
    const int rest = (int)(item - r * per_request), i = rest / a.Hq, h = rest - i * a.Hq, g = h / a.G;
    int first, n;
    new_tokens(a, (int)r, first, n);
    if (i >= n) return;
    const int tiles = (suffix_len(a, (int)r) + 31) / 32;
    int parts = a.prefix_splits;
    if (tiles > 0) {
        const int each = suffix_split_tiles(tiles, a.suffix_splits, WAVES);
        parts += (tiles + each - 1) / each;
    }
    const int lane = threadIdx.x % kLanes;
    const int64_t step = (int64_t)a.Hkv * a.rows, row = (int64_t)g * a.rows + (int64_t)(first + i) * a.G + (h - g * a.G);
    float m = kNone;
    for (int p = 0; p < parts; ++p) m = fmaxf(m, a.part_ml[p * step + row].x);
    float l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
        const float2 ml = a.part_ml[p * step + row];
        const float c = __builtin_amdgcn_exp2f(ml.x - m);
        l += c * ml.y;
        o += c * reinterpret_cast<const f32x4_t*>(a.part_o + (p * step + row) * D)[lane];
    }
    const bool empty = l == 0.f;
    const float inv = empty ? 0.f : 1.f / l;
    uint2 packed;
    packed.x = pack<T>(o[0] * inv, o[1] * inv);
    packed.y = pack<T>(o[2] * inv, o[3] * inv);
    uint16_t* out = static_cast<uint16_t*>(a.out) + (int64_t)(first + i) * a.q_st + (int64_t)h * a.q_sh;
    reinterpret_cast<uint2*>(out)[lane] = packed;
    if (a.lse && lane == 0)
        a.lse[(int64_t)h * a.tokens + first + i] = empty ? -__builtin_huge_valf() : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D>
static int launch(const PrefixArgs& a, const PrefixPlan& p, hipStream_t stream) {
    constexpr int WAVES = D == 256 ? 2 : 4;
    constexpr int kMost = D == 256 ? 2 : 4;
    const int64_t own_groups = p.suffix_splits > 0 ? (int64_t)a.requests * a.Hkv * p.suffix_row_tiles * p.suffix_splits : 0;
    const int64_t joins = ((int64_t)a.requests * a.max_new * a.Hq + kJoinThreads / (D / 4) - 1) / (kJoinThreads / (D / 4));
    if (a.prefix_groups + own_groups > 1 << 23 || joins > 1 << 23) return STEM_ERR_UNSUPPORTED;   // threads of a launch: 32 bits
    const dim3 grid((unsigned)(a.prefix_groups + own_groups)), block(64 * WAVES);
    if (grid.x > 0) {
        const bool short_own = p.suffix_row_tile == 16;
        if (p.row_tile == 16) hipLaunchKernelGGL((prefix_attn_kernel<T, D, 1, 1, WAVES>), grid, block, 0, stream, a);
        else if (p.row_tile == 32 && short_own) hipLaunchKernelGGL((prefix_attn_kernel<T, D, 2, 1, WAVES>), grid, block, 0, stream, a);
        else if (p.row_tile == 32) hipLaunchKernelGGL((prefix_attn_kernel<T, D, 2, 2, WAVES>), grid, block, 0, stream, a);
        else if constexpr (kMost == 4) {
            if (short_own) hipLaunchKernelGGL((prefix_attn_kernel<T, D, 4, 1, WAVES>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((prefix_attn_kernel<T, D, 4, 4, WAVES>), grid, block, 0, stream, a);
        }
        if (const int st = check_launch()) return st;
    }
    hipLaunchKernelGGL((join_kernel<T, D, WAVES>), dim3((unsigned)joins), dim3(kJoinThreads), 0, stream, a);
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
    const int64_t combos = ((int64_t)a.Hkv * p.prefix_splits + 7) / 8 * 8;
    if (combos * p.row_tiles > 1 << 23) return STEM_ERR_UNSUPPORTED;
    a.prefix_groups = (int32_t)(combos * p.row_tiles);
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
