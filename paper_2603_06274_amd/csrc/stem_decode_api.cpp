// Host side of include/stem_decode.h: argument checks, rotary frequencies, workspace layouts and the split of the attention
// to a shared prefix.  No allocation, no synchronisation.
#include <cmath>
#include <limits>

#include "stem_decode_common.h"

namespace stem {

constexpr int64_t kInt32Max = 0x7fffffff;
constexpr int64_t kMostGroups = kInt32Max - (1 << 20);   // of a launch, whose grid is rounded up to lines of 2^20

static bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Strides of [tokens, heads, head_dim] rows.
static bool good_strides(int64_t token, int64_t head, int32_t head_dim) {
    return token >= head_dim && head >= head_dim && !((token | head) & 7);
}

static int check_page_size(int32_t n) {
    if (n <= 0) return STEM_ERR_INVALID_ARG;
    return n == 16 || n == 32 || n == 64 || n == 128 || n == 256 ? STEM_OK : STEM_ERR_UNSUPPORTED;
}

static int check_pages(const stem_pages& p, int32_t head_dim) {
    if (const int st = check_page_size(p.page_size)) return st;
    if (p.num_pages < 0) return STEM_ERR_INVALID_ARG;
    if ((int64_t)p.num_pages * p.page_size > kInt32Max) return STEM_ERR_UNSUPPORTED;
    if (!good_strides(p.stride_token, p.stride_head, head_dim) || p.stride_page < head_dim || (p.stride_page & 7))
        return STEM_ERR_INVALID_ARG;
    return STEM_OK;
}

static int check_rotary(const stem_rotary_shape* s, float factor) {
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
static int check_rotary_addresses(const stem_rotary_shape& s, const void* q, const void* k, const int32_t* positions,
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

TableWorkspace table_workspace(int32_t requests) {
    TableWorkspace w;
    w.pages_before = 0;
    w.back_before = align256(sizeof(int32_t) * (size_t)requests);
    w.ring = w.back_before + align256(sizeof(int32_t) * (size_t)requests);
    w.total = w.ring + 256;
    return w;
}

static int check_table(const stem_table_shape* s) {
    if (!s) return STEM_ERR_INVALID_ARG;
    if (s->requests < 1 || s->num_pages < 1 || s->pages_per_request < 1 || s->token_capacity < 0 || s->position_offset < 0 ||
        s->max_new < 0)
        return STEM_ERR_INVALID_ARG;
    if (const int st = check_page_size(s->page_size)) return st;
    if (s->requests > STEM_MAX_REQUESTS) return STEM_ERR_UNSUPPORTED;
    if ((int64_t)s->requests * s->pages_per_request > kInt32Max || (int64_t)s->num_pages * s->page_size > kInt32Max ||
        s->position_offset + (int64_t)s->pages_per_request * s->page_size > kInt32Max)
        return STEM_ERR_UNSUPPORTED;
    return STEM_OK;
}

static int check_prefix(const stem_prefix_shape* s) {
    if (!s) return STEM_ERR_INVALID_ARG;
    if (s->dtype != STEM_BF16 && s->dtype != STEM_FP16) return STEM_ERR_INVALID_ARG;
    if (s->num_q_heads <= 0 || s->num_kv_heads <= 0 || s->num_q_heads % s->num_kv_heads) return STEM_ERR_INVALID_ARG;
    if (s->head_dim <= 0 || s->requests < 1 || s->tokens < 0 || s->max_new < 1 || s->prefix_len < 0 || s->max_suffix < 0)
        return STEM_ERR_INVALID_ARG;
    if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return STEM_ERR_UNSUPPORTED;
    if (s->requests > STEM_MAX_REQUESTS || s->num_q_heads > 65535) return STEM_ERR_UNSUPPORTED;
    // rows are counted in 32 bits
    if ((int64_t)s->tokens * s->num_q_heads > kInt32Max || (int64_t)s->max_new * s->num_q_heads > kInt32Max)
        return STEM_ERR_UNSUPPORTED;
    if (!good_strides(s->q_stride_token, s->q_stride_head, s->head_dim)) return STEM_ERR_INVALID_ARG;
    // the kernel addresses a tile of the prefix (128 rows at most), and 16 rows of a page, through a 32-bit byte offset
    const int64_t most = (kInt32Max - 2 * s->head_dim) / (2 * 15), most_prefix = kInt32Max / (2 * 128);
    if (s->prefix_len > 0) {
        if (!good_strides(s->prefix_stride_token, s->prefix_stride_head, s->head_dim)) return STEM_ERR_INVALID_ARG;
        if (s->prefix_stride_token > most_prefix) return STEM_ERR_UNSUPPORTED;
    }
    if (s->max_suffix > 0) {
        if (s->max_suffix > kMaxSuffix) return STEM_ERR_UNSUPPORTED;
        if (const int st = check_pages(s->pages, s->head_dim)) return st;
        if (s->pages.stride_token > most) return STEM_ERR_UNSUPPORTED;
        if (s->pages_per_request < 1) return STEM_ERR_INVALID_ARG;
        if ((int64_t)s->pages_per_request * s->pages.page_size < s->max_suffix) return STEM_ERR_INVALID_ARG;
        if ((int64_t)s->requests * s->pages_per_request > kInt32Max) return STEM_ERR_UNSUPPORTED;
    }
    return STEM_OK;
}

int prefix_plan(const stem_prefix_shape& s, PrefixPlan* plan, int (*units)()) {
    const int units_here = units();
    if (units_here <= 0) return STEM_ERR_HIP;
    const int64_t G = s.num_q_heads / s.num_kv_heads, rows = s.tokens * G;
    PrefixPlan p;
    auto tile_of = [](int64_t n) { return n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : 128; };
    p.row_tile = tile_of(rows);
    const int cus = units_here * (s.head_dim == 256 ? 1 : 2);   // workgroups at a time
    p.row_tiles = (int32_t)((rows + p.row_tile - 1) / p.row_tile);
    p.prefix_splits = p.split_keys = 0;
    if (s.prefix_len > 0 && rows > 0) {
        // Parts of whole tiles, one to four rounds of workgroups (two run on a CU at a time, one with head size 256): whichever ends first,
        // where a part costs its tiles and about two more to begin and end.
        const int64_t others = (int64_t)p.row_tiles * s.num_kv_heads;
        const int32_t waves = 4, row_groups = p.row_tile == 16 ? 1 : p.row_tile == 128 ? 4 : 2;
        const int64_t tile = 32 * waves / row_groups, tiles = (s.prefix_len + tile - 1) / tile;
        const int64_t most_each = kInt32Max / (2 * s.prefix_stride_token * tile);   // a part's rows: 32-bit byte offsets
        int64_t best = -1, best_each = 0;
        for (int rounds = 1; rounds <= 4; ++rounds) {
            int64_t splits = (int64_t)rounds * cus / others;
            splits = splits < 1 ? 1 : splits > tiles ? tiles : splits;
            int64_t each = (tiles + splits - 1) / splits;
            each = each < most_each ? each : most_each;
            splits = (tiles + each - 1) / each;
            const int64_t cost = (splits * others + cus - 1) / cus * (each + 2);
            if (best < 0 || cost < best) best = cost, best_each = each;
        }
        p.split_keys = (int32_t)(best_each * tile);
        p.prefix_splits = (int32_t)((tiles + best_each - 1) / best_each);
    }
    const int64_t own_rows = s.max_new * G < rows ? s.max_new * G : rows;
    p.suffix_row_tile = own_rows <= 16 ? 16 : 64;
    p.suffix_row_tiles = (int32_t)((own_rows + p.suffix_row_tile - 1) / p.suffix_row_tile);
    // By the rows that there are, not by what each request might have: max_new is a bound for the longest (a prompt of 2048 tokens beside 63
    // single ones, four heads per KV head: 8192 row tiles by the one count, 195 by the other; 1490 and 1200 us behind 32K keys).
    const int64_t by_request = (int64_t)s.requests * p.suffix_row_tiles, by_rows = slot_before(s.requests, rows, p.suffix_row_tile);
    p.own_by_rows = by_request > by_rows;
    p.own_slots = p.own_by_rows ? by_rows : by_request;
    p.join_by_rows = (int64_t)s.requests * s.max_new > s.tokens;
    p.join_rows = (p.join_by_rows ? s.tokens : (int64_t)s.requests * s.max_new) * s.num_q_heads;
    p.suffix_splits = 0;
    if (s.max_suffix > 0 && rows > 0) {
        const int64_t others = p.own_slots * s.num_kv_heads;
        const int64_t wanted = (units_here + others - 1) / others;   // (half as many as fit at a time: 52.0, twice as many 53.9 us with 32K keys)
        const int64_t tiles = ((int64_t)s.max_suffix + 255) / 256;
        p.suffix_splits = (int32_t)(wanted < tiles ? wanted : tiles);
        if (p.suffix_splits > 64) p.suffix_splits = 64;
    }
    // A second launch costs about 3 us: that is what a workgroup takes for the tiles that it would have shared with others.  One launch / two, us a
    // call of 8 requests: d = 64, 8 / 2 heads, 300 keys 8.2 / 11.1, 1000 9.3 / 11.1, 1500 10.5 / 11.1, 2000 11.8 / 11.2; d = 128, 32 / 8 heads, 240 keys 9.4 /
    // 11.1, 1040 14.5 / 11.5; d = 256, 140 keys 13.4 / 15.3 and for one request 13.6 / 10.9.  (The prefix within 32-bit byte offsets, too.)
    const int64_t most_small = s.head_dim == 64 ? 1536 : s.head_dim == 128 ? 384 : -1;
    p.small = own_rows <= 16 && (int64_t)s.requests * s.num_kv_heads <= units_here && (int64_t)s.prefix_len + s.max_suffix <= most_small &&
              (s.prefix_len == 0 || ((int64_t)s.prefix_len + 127) / 128 * 128 * s.prefix_stride_token * 2 <= kInt32Max);
    if (p.small) p.prefix_splits = p.suffix_splits = 0;
    p.prefix_groups = ((int64_t)s.num_kv_heads * p.prefix_splits + 7) / 8 * 8 * p.row_tiles;
    p.groups = p.prefix_groups + p.own_slots * s.num_kv_heads * p.suffix_splits;
    if (p.groups > kMostGroups || p.join_rows > kMostGroups) return STEM_ERR_UNSUPPORTED;
    const int64_t parts = (int64_t)(p.prefix_splits + p.suffix_splits) * s.num_kv_heads * rows;
    p.partial_ml = align256(sizeof(float) * (size_t)parts * s.head_dim);
    p.bytes = p.partial_ml + align256(2 * sizeof(float) * (size_t)parts);
    if (p.bytes == 0) p.bytes = 256;
    *plan = p;
    return STEM_OK;
}

}  // namespace stem

using namespace stem;

extern "C" {

int stem_rotary_frequencies(int32_t rotary_dim, double theta, const stem_rotary_scaling* scaling, double* host_turns,
                            double* host_attention_factor) {
    if (rotary_dim < 2 || rotary_dim % 2 || !host_turns || !host_attention_factor) return STEM_ERR_INVALID_ARG;
    if (rotary_dim > STEM_MAX_HEAD_DIM) return STEM_ERR_UNSUPPORTED;
    if (!std::isfinite(theta) || !(theta > 1.0)) return STEM_ERR_INVALID_ARG;
    const int32_t kind = scaling ? scaling->kind : STEM_ROTARY_NONE;
    if (kind < STEM_ROTARY_NONE || kind > STEM_ROTARY_BANDS) return STEM_ERR_INVALID_ARG;
    const double r = rotary_dim, two_pi = 6.283185307179586;
    double factor = 1.0, trained = 0.0, low = 0.0, high = 0.0;
    if (kind != STEM_ROTARY_NONE) {
        factor = scaling->factor;
        if (!std::isfinite(factor) || !(factor >= 1.0)) return STEM_ERR_INVALID_ARG;
    }
    if (kind == STEM_ROTARY_NTK) {
        if (rotary_dim == 2) return STEM_ERR_INVALID_ARG;
        theta *= std::pow(factor, r / (r - 2.0));
        if (!std::isfinite(theta)) return STEM_ERR_INVALID_ARG;
    }
    double ramp_lo = 0.0, ramp_span = 1.0;
    if (kind == STEM_ROTARY_YARN || kind == STEM_ROTARY_BANDS) {
        trained = scaling->trained_length;
        low = scaling->low;
        high = scaling->high;
        if (!std::isfinite(trained) || !(trained > 0.0) || !std::isfinite(low) || !std::isfinite(high) || !(low > 0.0) ||
            !(high > low))
            return STEM_ERR_INVALID_ARG;
        auto dim = [&](double n) { return r * std::log(trained / (n * two_pi)) / (2.0 * std::log(theta)); };
        if (kind == STEM_ROTARY_YARN) {
            ramp_lo = std::fmax(std::floor(dim(high)), 0.0);
            ramp_span = std::fmax(std::fmin(std::ceil(dim(low)), r - 1.0) - ramp_lo, 0.001);
        }
    }
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        const double f = std::pow(theta, -2.0 * i / r);
        double share = 0.0;                            // of f / factor
        if (kind == STEM_ROTARY_LINEAR) share = 1.0;
        else if (kind == STEM_ROTARY_YARN) share = std::fmin(std::fmax((i - ramp_lo) / ramp_span, 0.0), 1.0);
        else if (kind == STEM_ROTARY_BANDS)
            share = 1.0 - std::fmin(std::fmax((trained * f / two_pi - low) / (high - low), 0.0), 1.0);
        host_turns[i] = (f * (1.0 - share) + f / factor * share) / two_pi;
    }
    *host_attention_factor = kind == STEM_ROTARY_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return STEM_OK;
}

int stem_rotary(const stem_rotary_shape* shape, const void* q, const void* k, const int32_t* positions,
                const double* turns, float attention_factor, int32_t backward, void* q_out, void* k_out,
                void* hip_stream) {
    if (const int st = check_rotary(shape, attention_factor)) return st;
    if (backward != 0 && backward != 1) return STEM_ERR_INVALID_ARG;
    const stem_rotary_shape& s = *shape;
    if (s.num_kv_heads > 0 && !good_strides(s.k_out_stride_token, s.k_out_stride_head, s.head_dim)) return STEM_ERR_INVALID_ARG;
    if (s.tokens == 0) return STEM_OK;
    if (const int st = check_rotary_addresses(s, q, k, positions, turns, q_out)) return st;
    if (s.num_kv_heads > 0) {
        if (!k_out || !aligned(k_out, 16)) return STEM_ERR_INVALID_ARG;
        if (k == k_out && (s.k_stride_token != s.k_out_stride_token || s.k_stride_head != s.k_out_stride_head))
            return STEM_ERR_INVALID_ARG;
    }
    const RotaryCall call = {s, q, k, nullptr, q_out, k_out, nullptr, positions, nullptr, turns, attention_factor, backward, {}};
    return launch_rotary(call, static_cast<hipStream_t>(hip_stream));
}

int stem_rotary_append(const stem_rotary_shape* shape, const stem_pages* pages, const void* q, const void* k,
                       const void* v, const int32_t* positions, const int32_t* slots, const double* turns,
                       float attention_factor, void* q_out, void* k_pages, void* v_pages, void* hip_stream) {
    if (const int st = check_rotary(shape, attention_factor)) return st;
    const stem_rotary_shape& s = *shape;
    if (!pages || s.num_kv_heads == 0) return STEM_ERR_INVALID_ARG;
    if (const int st = check_pages(*pages, s.head_dim)) return st;
    if (s.tokens == 0) return STEM_OK;
    if (const int st = check_rotary_addresses(s, q, k, positions, turns, q_out)) return st;
    if (!slots || !aligned(slots, 4) || !v || !aligned(v, 16)) return STEM_ERR_INVALID_ARG;
    if (pages->num_pages == 0) return STEM_OK;
    if (!k_pages || !aligned(k_pages, 16) || !v_pages || !aligned(v_pages, 16)) return STEM_ERR_INVALID_ARG;
    const RotaryCall call = {s, q, k, v, q_out, k_pages, v_pages, positions, slots, turns, attention_factor, 0, *pages};
    return launch_rotary(call, static_cast<hipStream_t>(hip_stream));
}

int stem_block_table_workspace_bytes(const stem_table_shape* shape, size_t* host_bytes) {
    if (const int st = check_table(shape)) return st;
    if (!host_bytes) return STEM_ERR_INVALID_ARG;
    *host_bytes = table_workspace(shape->requests).total;
    return STEM_OK;
}

int stem_block_table(const stem_table_shape* shape, const int32_t* past_lens, const int32_t* new_lens,
                     const int32_t* ring_state, int32_t* ring, int32_t* table, int32_t* lens, int32_t* ring_state_out,
                     int32_t* cu_new, int32_t* positions, int32_t* slots, int32_t* status, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
    if (const int st = check_table(shape)) return st;
    const void* needed[] = {past_lens, ring_state, ring, table, lens, ring_state_out, cu_new, status};
    for (const void* p : needed)
        if (!p || !aligned(p, 4)) return STEM_ERR_INVALID_ARG;
    if (!aligned(new_lens, 4) || !aligned(positions, 4) || !aligned(slots, 4)) return STEM_ERR_INVALID_ARG;
    if (shape->token_capacity > 0 && (!positions || !slots)) return STEM_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 16)) return STEM_ERR_INVALID_ARG;
    const TableWorkspace w = table_workspace(shape->requests);
    if (workspace_bytes < w.total) return STEM_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    auto part = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
    const TableCall call = {*shape, past_lens, new_lens, ring_state, ring, table, lens, ring_state_out, cu_new, positions, slots, status,
                            part(w.pages_before), part(w.back_before), part(w.ring)};
    return launch_block_table(call, static_cast<hipStream_t>(hip_stream));
}

int stem_prefix_attn_workspace_bytes(const stem_prefix_shape* shape, size_t* host_bytes) {
    if (const int st = check_prefix(shape)) return st;
    if (!host_bytes) return STEM_ERR_INVALID_ARG;
    PrefixPlan plan;
    if (const int st = prefix_plan(*shape, &plan)) return st;
    *host_bytes = plan.bytes;
    return STEM_OK;
}

int stem_prefix_attn(const stem_prefix_shape* shape, const void* q, const void* prefix_k, const void* prefix_v,
                     const void* k_pages, const void* v_pages, const int32_t* table, const int32_t* lens,
                     const int32_t* cu_new, float softmax_scale, void* out, float* lse, void* workspace,
                     size_t workspace_bytes, void* hip_stream) {
    if (const int st = check_prefix(shape)) return st;
    const stem_prefix_shape& s = *shape;
    if (!std::isfinite(softmax_scale) || !(softmax_scale > 0.f)) return STEM_ERR_INVALID_ARG;
    if (!aligned(cu_new, 4) || (!cu_new && s.tokens != s.requests)) return STEM_ERR_INVALID_ARG;
    if (s.tokens == 0) return STEM_OK;
    if (!q || !aligned(q, 16) || !out || !aligned(out, 16) || q == out || !aligned(lse, 4)) return STEM_ERR_INVALID_ARG;
    if (s.prefix_len > 0 && (!prefix_k || !aligned(prefix_k, 16) || !prefix_v || !aligned(prefix_v, 16)))
        return STEM_ERR_INVALID_ARG;
    if (s.max_suffix > 0) {
        if (!table || !aligned(table, 4) || !lens || !aligned(lens, 4)) return STEM_ERR_INVALID_ARG;
        if (s.pages.num_pages > 0 && (!k_pages || !aligned(k_pages, 16) || !v_pages || !aligned(v_pages, 16)))
            return STEM_ERR_INVALID_ARG;
    }
    if (!workspace || !aligned(workspace, 16)) return STEM_ERR_INVALID_ARG;
    PrefixCall call = {s, {}, q, prefix_k, prefix_v, k_pages, v_pages, table, lens, cu_new, softmax_scale, out, lse, workspace};
    if (const int st = prefix_plan(s, &call.plan)) return st;
    if (workspace_bytes < call.plan.bytes) return STEM_ERR_WORKSPACE;
    return launch_prefix_attn(call, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
