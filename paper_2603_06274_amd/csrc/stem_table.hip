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
    s.bad = past < 0 || (int64_t)past + s.more > most;
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

// Sum over the lanes before this one, and over all of the wave.
template <typename N>
__device__ __forceinline__ N wave_before(N x, N& all) {
    const int lane = threadIdx.x & 63;
    N sum = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const N y = __shfl_up(sum, d);
        sum += lane >= d ? y : N(0);
    }
    all = __shfl(sum, 63);
    return sum - x;
}

// ALL: also moves the pages and maps the tokens; at most kTableThreads requests.
template <bool ALL>
__global__ __launch_bounds__(kTableThreads) void table_sums_kernel(TableArgs a) {
    __shared__ int64_t wave_sum[4][kTableWaves];
    const int tid = threadIdx.x, w = tid >> 6;
    int32_t head = a.ring_state[0], count = a.ring_state[1];
    const bool good_ring = head >= 0 && head < a.num_pages && count >= 0 && count <= a.num_pages;
    if (!good_ring) head = count = 0;
    int64_t total[4] = {0, 0, 0, 0};                   // pages lacking, given back, new tokens, bad requests
    Step s = {};
    int64_t before[3] = {0, 0, 0};
    for (int r0 = 0; r0 < a.requests; r0 += kTableThreads) {
        const int r = r0 + tid;
        s = Step{};
        if (r < a.requests) s = step_of(a, a.past_lens[r], a.new_lens ? a.new_lens[r] : 1);
        int64_t wave_all[4];
        before[0] = wave_before<int64_t>(s.need, wave_all[0]);
        before[1] = wave_before<int64_t>(s.back, wave_all[1]);
        before[2] = wave_before<int64_t>(s.more, wave_all[2]);
        wave_all[3] = __popcll(__builtin_amdgcn_ballot_w64(s.bad));
        if (r0 > 0) __syncthreads();                   // the sums before have been read
        if ((tid & 63) == 0)
            for (int x = 0; x < 4; ++x) wave_sum[x][w] = wave_all[x];
        __syncthreads();
        for (int x = 0; x < 4; ++x) {
            int64_t earlier = total[x];
            for (int v = 0; v < kTableWaves; ++v) {
                const int64_t n = wave_sum[x][v];
                if (v < w) earlier += n;
                total[x] += n;
            }
            if (x < 3) before[x] += earlier;
        }
        if (r < a.requests) {
            if (!ALL) {                                // (a sum that 32 bits do not hold refuses the step)
                a.pages_before[r] = (int32_t)before[0];
                a.back_before[r] = (int32_t)before[1];
            }
            a.cu_new[r] = (int32_t)before[2];
        }
    }
    const int64_t lacking = total[0] - count, beyond = total[2] - a.capacity, no_room = count + total[1] - a.num_pages;
    const bool ok = lacking <= 0 && total[3] == 0 && beyond <= 0 && no_room <= 0 && good_ring;
    for (int r = tid; r < a.requests; r += kTableThreads) {
        const int32_t past = a.past_lens[r], fresh = a.new_lens ? a.new_lens[r] : 1;
        a.lens[r] = !ok ? past : fresh < 0 ? 0 : past + fresh;
        if (!ok) a.cu_new[r] = 0;
    }
    if (tid == 0) {
        auto number = [](int64_t n) { return (int32_t)(n < 0 ? 0 : n > 0x7fffffff ? 0x7fffffff : n); };
        a.status[0] = number(lacking);
        a.status[1] = number(total[3]);
        a.status[2] = number(beyond);
        a.status[3] = good_ring ? number(no_room) : 1;
        a.cu_new[a.requests] = ok ? (int32_t)total[2] : 0;
        const int32_t then0 = a.ring_state[0], then1 = a.ring_state[1];
        a.ring_state_out[0] = ok ? in_ring(head, total[0], a.num_pages) : then0;
        a.ring_state_out[1] = ok ? (int32_t)(count - total[0] + total[1]) : then1;
        if (!ALL) {
            a.ring_then[0] = head;
            a.ring_then[1] = ok ? count : -1;          // -1: the step is refused
            a.ring_then[2] = (int32_t)total[1];
        }
    }
    if constexpr (ALL) {
        if (ok) {
            // requests of a few pages and tokens by their own lane, longer ones by the whole wave, one after the other
            const bool small = s.need <= 4 && s.back <= 4 && s.more <= 4;
            if (small) move_and_map(a, tid, s, (int32_t)before[0], (int32_t)before[1], (int32_t)before[2], head, count, 0, 1);
            for (uint64_t left = __builtin_amdgcn_ballot_w64(!small); left; left &= left - 1) {
                const int l = __builtin_ctzll(left);
                Step other;
                other.past = __shfl(s.past, l), other.have = __shfl(s.have, l), other.need = __shfl(s.need, l);
                other.back = __shfl(s.back, l), other.more = __shfl(s.more, l), other.bad = false;
                move_and_map(a, (tid & ~63) + l, other, __shfl((int32_t)before[0], l), __shfl((int32_t)before[1], l),
                             __shfl((int32_t)before[2], l), head, count, tid & 63, 64);
            }
        }
        for (int64_t t = (ok ? total[2] : 0) + tid; t < a.capacity; t += kTableThreads) {
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
                         s.pages_per_request, s.token_capacity, s.position_offset, __builtin_ctz(s.page_size)};
    // One launch for steps that a single workgroup has through about as soon as a second launch begins.
    if (s.requests <= kTableThreads && s.token_capacity <= 4096) {
        hipLaunchKernelGGL(table_sums_kernel<true>, dim3(1), dim3(kTableThreads), 0, stream, a);
        return check_launch();
    }
    hipLaunchKernelGGL(table_sums_kernel<false>, dim3(1), dim3(kTableThreads), 0, stream, a);
    if (const int st = check_launch()) return st;
    const int64_t each = ((int64_t)s.token_capacity / s.requests + 4 * kMapThreads - 1) / (4 * kMapThreads);
    const int shared = (int)(each < 1 ? 1 : each > 256 ? 256 : each);
    hipLaunchKernelGGL(table_map_kernel, dim3(s.requests + 1, shared), dim3(kMapThreads), 0, stream, a);
    return check_launch();
}

}  // namespace stem
