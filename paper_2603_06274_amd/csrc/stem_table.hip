// Block tables, slots and positions of one step, from the requests' lengths.
//
// Three sums over the requests decide everything: pages that the requests before lack (where in the ring a request's new pages
// begin), pages that those before give back, and their new tokens.  Whole numbers of a few KiB: what a call costs is the
// latency of its launches and of the chain lengths -> sums -> ring -> slots.  One workgroup forms the sums, 1024 requests at a
// time (a wave adds up by lane shifts, the waves' totals go through LDS).  Where the step is small it also moves the pages and
// writes the slots; otherwise a second launch does that, with one row of workgroups per request.
#include "stem_decode_common.h"

namespace stem {

constexpr int kTableThreads = 1024;
constexpr int kTableWaves = kTableThreads / 64;
constexpr int kMapThreads = 256;

struct TableArgs {
    const int32_t *past_lens, *new_lens, *ring_state;
    int32_t *ring, *table, *lens, *ring_state_out, *cu_new, *positions, *slots, *status;
    int32_t *pages_before, *back_before, *ring_then;
    int32_t requests, num_pages, row, capacity, offset, shift;   // page_size = 1 << shift, row: entries of a table row
    int32_t most_new;
};

// What a step does with one request.
struct Step {
    int32_t past, have, need, back, more;              // tokens, pages held, lacking and given back, new tokens
    bool bad;
};
__device__ __forceinline__ Step step_of(const TableArgs& a, int32_t past, int32_t fresh) {
    Step s;
    const int64_t most = (int64_t)a.row << a.shift;
    const bool gone = fresh < 0;
    s.more = gone ? 0 : fresh;
    s.bad = past < 0 || (int64_t)past + s.more > most || s.more > a.most_new;
    if (s.bad) {                                       // counted, and then nothing is done at all
        s.past = s.have = s.need = s.back = s.more = 0;
        return s;
    }
    const int32_t mask = (1 << a.shift) - 1;
    s.past = past;
    s.have = (int32_t)(((int64_t)past + mask) >> a.shift);
    s.need = gone ? 0 : (int32_t)(((int64_t)past + s.more + mask) >> a.shift) - s.have;
    s.back = gone ? s.have : 0;
    return s;
}

// place `at` places from `from` on in the ring
__device__ __forceinline__ int32_t in_ring(int32_t from, int64_t at, int32_t size) {
    const int64_t x = from + at;                       // 0 <= from < size, 0 <= at <= 2 size
    return (int32_t)(x < size ? x : x - size < size ? x - size : x - 2 * (int64_t)size);
}

// Moves a request's pages and maps its tokens: every `stride`-th from `lane` on.  The ring's entries that are read (the first
// `count`) are not those that are written (behind them), and a slot in a new page takes the page from the ring, so
// no order between lanes is needed.
__device__ __forceinline__ void move_and_map(const TableArgs& a, int r, const Step& s, int32_t pages_before, int32_t back_before,
                                             int32_t cu, int32_t head, int32_t count, int lane, int stride) {
    int32_t* row = a.table + (int64_t)r * a.row;
    for (int i = lane; i < s.need; i += stride) row[s.have + i] = a.ring[in_ring(head, (int64_t)pages_before + i, a.num_pages)];
    for (int i = lane; i < s.back; i += stride) a.ring[in_ring(head, (int64_t)count + back_before + i, a.num_pages)] = row[i];
    for (int i = lane; i < s.more; i += stride) {
        const int32_t place = s.past + i, j = place >> a.shift;
        const int32_t page = j < s.have ? row[j] : a.ring[in_ring(head, (int64_t)pages_before + j - s.have, a.num_pages)];
        a.positions[cu + i] = a.offset + place;
        a.slots[cu + i] = (uint32_t)page < (uint32_t)a.num_pages ? (page << a.shift) + (place & ((1 << a.shift) - 1)) : -1;
    }
}

// Sum over the lanes up to and with this one.
template <typename N>
__device__ __forceinline__ N wave_sum_to(N x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const N y = __shfl_up(x, d);
        x += lane >= d ? y : N(0);
    }
    return x;
}

// One workgroup of at most kTableThreads lanes, one request per lane at a time.  ALL: it also moves the pages and maps the tokens, and
// there are no more requests than lanes.
template <bool ALL>
__global__ __launch_bounds__(kTableThreads) void table_sums_kernel(TableArgs a) {
    // per wave: new tokens (which may need 64 bits), pages lacking, pages given back, bad requests
    __shared__ int64_t wave_more[kTableWaves];
    __shared__ int4 wave_pages[kTableWaves];
    const int tid = threadIdx.x, w = tid >> 6, waves = blockDim.x >> 6;
    const int32_t then0 = a.ring_state[0], then1 = a.ring_state[1];
    const bool good_ring = then0 >= 0 && then0 < a.num_pages && then1 >= 0 && then1 <= a.num_pages;
    const int32_t head = good_ring ? then0 : 0, count = good_ring ? then1 : 0;
    int64_t more_all = 0;
    int32_t need_all = 0, back_all = 0, bad_all = 0;   // (32 bits: requests * pages_per_request at most)
    Step s = {};
    int32_t past = 0, fresh = 0, need_before = 0, back_before = 0;
    int64_t more_before = 0;
    for (int r0 = 0; r0 < a.requests; r0 += blockDim.x) {
        const int r = r0 + tid;
        s = Step{};
        if (r < a.requests) {
            past = a.past_lens[r];
            fresh = a.new_lens ? a.new_lens[r] : 1;
            s = step_of(a, past, fresh);
        }
        // sums within the wave, then the waves' totals
        const int32_t need_to = wave_sum_to(s.need), back_to = wave_sum_to(s.back);
        const int64_t more_to = wave_sum_to<int64_t>(s.more);
        const int32_t bad = (int32_t)__popcll(__builtin_amdgcn_ballot_w64(s.bad));
        if (r0 > 0) __syncthreads();                   // the totals before have been read
        if ((tid & 63) == 63) {
            wave_more[w] = more_to;
            wave_pages[w] = make_int4(need_to, back_to, bad, 0);
        }
        __syncthreads();
        need_before = need_all + need_to - s.need;
        back_before = back_all + back_to - s.back;
        more_before = more_all + more_to - s.more;
        for (int v = 0; v < waves; ++v) {
            const int64_t m = wave_more[v];
            const int4 p = wave_pages[v];
            if (v < w) need_before += p.x, back_before += p.y, more_before += m;
            need_all += p.x, back_all += p.y, bad_all += p.z, more_all += m;
        }
        if (!ALL && r < a.requests) {                  // (a sum that 32 bits do not hold refuses the step)
            a.pages_before[r] = need_before;
            a.back_before[r] = back_before;
            a.cu_new[r] = (int32_t)more_before;
        }
    }
    const int64_t lacking = (int64_t)need_all - count, beyond = more_all - a.capacity, no_room = (int64_t)count + back_all - a.num_pages;
    const bool ok = lacking <= 0 && bad_all == 0 && beyond <= 0 && no_room <= 0 && good_ring;
    if constexpr (ALL) {
        if (tid < a.requests) {
            a.lens[tid] = !ok ? past : fresh < 0 ? 0 : past + fresh;
            a.cu_new[tid] = ok ? (int32_t)more_before : 0;
        }
    } else {
        for (int r = tid; r < a.requests; r += blockDim.x) {
            const int32_t was = a.past_lens[r], came = a.new_lens ? a.new_lens[r] : 1;
            a.lens[r] = !ok ? was : came < 0 ? 0 : was + came;
            if (!ok) a.cu_new[r] = 0;
        }
    }
    if (tid == 0) {
        auto number = [](int64_t n) { return (int32_t)(n < 0 ? 0 : n > 0x7fffffff ? 0x7fffffff : n); };
        a.status[0] = number(lacking);
        a.status[1] = bad_all;
        a.status[2] = number(beyond);
        a.status[3] = good_ring ? number(no_room) : 1;
        a.cu_new[a.requests] = ok ? (int32_t)more_all : 0;
        a.ring_state_out[0] = ok ? in_ring(head, need_all, a.num_pages) : then0;
        a.ring_state_out[1] = ok ? count - need_all + back_all : then1;
        if (!ALL) {
            a.ring_then[0] = head;
            a.ring_then[1] = ok ? count : -1;          // -1: the step is refused
            a.ring_then[2] = back_all;
        }
    }
    if constexpr (ALL) {
        if (ok) {
            // requests of a few pages and tokens by their own lane, longer ones by the whole wave, one after the other
            const bool few = s.need <= 4 && s.back <= 4 && s.more <= 4;
            uint64_t left = __builtin_amdgcn_ballot_w64(!few);
            if (!few) s = Step{};                      // the lane does nothing in the first turn
            int r = tid, lane = 0, stride = 1;
            const int32_t mine[] = {past, fresh, need_before, back_before, (int32_t)more_before};
            int32_t need0 = need_before, back0 = back_before, more0 = (int32_t)more_before;
            for (;;) {
                move_and_map(a, r, s, need0, back0, more0, head, count, lane, stride);
                if (!left) break;
                const int l = __builtin_ctzll(left);
                left &= left - 1;
                s = step_of(a, __shfl(mine[0], l), __shfl(mine[1], l));
                need0 = __shfl(mine[2], l), back0 = __shfl(mine[3], l), more0 = __shfl(mine[4], l);
                r = (tid & ~63) + l, lane = tid & 63, stride = 64;
            }
        }
        for (int64_t t = (ok ? more_all : 0) + tid; t < a.capacity; t += blockDim.x) {
            a.positions[t] = 0;
            a.slots[t] = -1;
        }
    }
}

// The second launch: request blockIdx.x (one more: what lies behind the last token), shared by gridDim.y workgroups.
__global__ __launch_bounds__(kMapThreads) void table_map_kernel(TableArgs a) {
    const int r = blockIdx.x, lane = blockIdx.y * kMapThreads + threadIdx.x, stride = gridDim.y * kMapThreads;
    const int32_t head = a.ring_then[0], count = a.ring_then[1];
    if (r == a.requests) {
        for (int64_t t = (int64_t)a.cu_new[r] + lane; t < a.capacity; t += stride) {
            a.positions[t] = 0;
            a.slots[t] = -1;
        }
        return;
    }
    if (count < 0) return;
    // what was, from what is: `lens` may have taken the place of past_lens
    const int32_t cu = a.cu_new[r], more = a.cu_new[r + 1] - cu;
    const bool gone = a.new_lens && a.new_lens[r] < 0;
    Step s;
    if (gone) {
        const int32_t next = r + 1 < a.requests ? a.back_before[r + 1] : a.ring_then[2];
        s = Step{0, 0, 0, next - a.back_before[r], 0, false};
    } else {
        s = step_of(a, a.lens[r] - more, more);
    }
    move_and_map(a, r, s, a.pages_before[r], a.back_before[r], cu, head, count, lane, stride);
}

int launch_block_table(const TableCall& c, hipStream_t stream) {
    const stem_table_shape& s = c.shape;
    const TableArgs a = {c.past_lens, c.new_lens, c.ring_state, c.ring, c.table, c.lens, c.ring_state_out, c.cu_new, c.positions,
                         c.slots, c.status, c.pages_before, c.back_before, c.ring_then, s.requests, s.num_pages,
                         s.pages_per_request, s.token_capacity, s.position_offset, __builtin_ctz(s.page_size),
                         s.max_new > 0 ? s.max_new : 0x7fffffff};
    // One launch where a step is about a token per request, two where requests have many: a wave takes its long requests one after the
    // other.  One launch / two, us a call: 64 requests of one token 7.9 / 11.0, 1000 of one 10.4 / 11.4, 16 of 40 tokens on average 9.7 / 11.6, 64 of 29
    // 32.1 / 11.5, 256 of 7 28.5 / 11.4.  (And not where a finished request can have thousands of pages to give back.)
    const dim3 lanes(s.requests < kTableThreads ? (s.requests + 63) / 64 * 64 : kTableThreads);
    if (s.requests <= kTableThreads && s.token_capacity <= 2 * s.requests + 64 && s.pages_per_request <= 2048) {
        hipLaunchKernelGGL(table_sums_kernel<true>, dim3(1), lanes, 0, stream, a);
        return check_launch();
    }
    hipLaunchKernelGGL(table_sums_kernel<false>, dim3(1), lanes, 0, stream, a);
    if (const int st = check_launch()) return st;
    const int64_t each = ((int64_t)s.token_capacity / s.requests + 4 * kMapThreads - 1) / (4 * kMapThreads);
    const int shared = (int)(each < 1 ? 1 : each > 256 ? 256 : each);
    hipLaunchKernelGGL(table_map_kernel, dim3(s.requests + 1, shared), dim3(kMapThreads), 0, stream, a);
    return check_launch();
}

}  // namespace stem
