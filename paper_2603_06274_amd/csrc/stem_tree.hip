// Steps whose new tokens are drafts that form a tree: what each of them sees, what the model's choices confirm of them, and the
// confirmed ones' rows moved up in the pages.  Whole numbers of a few KiB and some rows: what a call costs is the latency of its
// launches and of the chain of loads and exchanges in each.
#include "stem_tree_common.h"

namespace stem {

// --- masks --------------------------------------------------------------------------------------------------

// One workgroup per request, one lane per new token.  A token's ancestors by doubling: after step s a lane has the bits of the 2^s nearest
// ones and the number of the next; it takes over that one's.  The steps end when no lane has a next one, so shallow trees take
// few: ceil(log2(depth)) + 1.
template <int WORDS>
__global__ void tree_masks_kernel(TreeMasksCall a, int words) {
    constexpr int kWords = WORDS < 4 ? WORDS : 4;      // exchanged at a time
    extern __shared__ uint64_t tree_lds[];             // [kWords][lanes] bits, then [lanes] numbers
    const int r = blockIdx.x, i = threadIdx.x, lanes = blockDim.x;
    int32_t* const next_of = reinterpret_cast<int32_t*>(tree_lds + kWords * lanes);
    int first, n;
    tree_tokens(a.cu_new, a.shape.tokens, r, first, n);
    if (n == 0) return;
    const int past = a.lens[r] - n, here = min(n, a.shape.max_new);
    const bool mine = i < here;
    int up = mine ? a.parents[first + i] : -1;
    const bool bad = up < -1 || up >= i;
    if (bad) up = -1;
    const int strange = __popcll(__builtin_amdgcn_ballot_w64(mine && bad)) + (i == 0 ? n - here : 0);
    if ((i & 63) == 0 && strange > 0) atomicAdd(a.status, strange);
    uint64_t bits[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bits[w] = i >> 6 == w ? 1ull << (i & 63) : 0;
    while (__syncthreads_or(up >= 0)) {
        next_of[i] = up;
#pragma unroll
        for (int w0 = 0; w0 < WORDS; w0 += kWords) {
            if (w0 > 0) __syncthreads();               // the words before have been read
#pragma unroll
            for (int w = 0; w < kWords; ++w) tree_lds[w * lanes + i] = bits[w0 + w];
            __syncthreads();
            if (up >= 0) {
#pragma unroll
                for (int w = 0; w < kWords; ++w) bits[w0 + w] |= tree_lds[w * lanes + up];
            }
        }
        if (up >= 0) up = next_of[up];
    }
    if (!mine) return;
    int seen = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        seen += __popcll(bits[w]);
        if (w < words) a.masks[(int64_t)(first + i) * words + w] = bits[w];
    }
    if (a.positions) a.positions[first + i] = a.shape.position_offset + past + seen - 1;
}

int launch_tree_masks(const TreeMasksCall& c, hipStream_t stream) {
    const int words = (c.shape.max_new + 63) / 64, lanes = words * 64;
    const dim3 grid(c.shape.requests), block(lanes);
#define STEM_MASKS_LAUNCH(WORDS) \
    hipLaunchKernelGGL(tree_masks_kernel<WORDS>, grid, block, (8 * (WORDS < 4 ? WORDS : 4) + 4) * (size_t)lanes, stream, c, words)
    if (words == 1) STEM_MASKS_LAUNCH(1);
    else if (words == 2) STEM_MASKS_LAUNCH(2);
    else if (words <= 4) STEM_MASKS_LAUNCH(4);
    else if (words <= 8) STEM_MASKS_LAUNCH(8);
    else STEM_MASKS_LAUNCH(16);
#undef STEM_MASKS_LAUNCH
    return check_launch();
}

// --- what a step keeps --------------------------------------------------------------------------------------

// A request whose numbers cannot be (counted, and then the step is refused).
__device__ __forceinline__ bool bad_request(const AcceptCall& a, int len, int n) {
    return n > a.shape.max_new || len < n || len > (int64_t)a.shape.pages_per_request * a.shape.page_size;
}

// One wave's walk of request r.  A token that is its parent's choice offers itself to the parent, of several the lowest-numbered; then the kept
// ones are a walk along these offers.  lds: [max_new] offers, [max_new] path, [max_new] choices.
template <typename Id>
__device__ __forceinline__ void walk_request(const AcceptCall& a, int r, int lane, int32_t* lds) {
    int first, n;
    tree_tokens(a.cu_new, a.shape.tokens, r, first, n);
    Id* const next = static_cast<Id*>(a.next_ids);
    const Id *drafts = static_cast<const Id*>(a.draft_ids) + first, *targets = static_cast<const Id*>(a.target_ids) + first;
    int32_t* const path = a.path + first;
    if (n == 0 || bad_request(a, a.lens[r], n)) {
        for (int i = lane; i < n; i += 64) path[i] = -1;
        if (lane == 0) a.accepted[r] = 0, next[r] = -1;
        return;
    }
    const int most = a.shape.max_new;
    int32_t *const offer = lds, *const kept = lds + most;
    Id* const choice = reinterpret_cast<Id*>(lds + 2 * most);
    constexpr int kNone = 0x7fffffff;
    // (a wave's reads and writes of LDS stay in order: the compiler has to keep them so)
    auto in_order = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    for (int i = lane; i < n; i += 64) {
        offer[i] = kNone;
        choice[i] = targets[i];
    }
    in_order();
    for (int i = lane; i < n; i += 64) {
        const int p = a.parents[first + i];
        if (p >= 0 && p < i && drafts[i] == choice[p]) atomicMin(&offer[p], i);
    }
    in_order();
    int count = 0, here = 0, last = 0;                 // the same in all lanes
    while (here != kNone) {
        if (lane == 0) kept[count] = here;
        ++count;
        last = here;
        here = offer[here];
    }
    in_order();
    for (int i = lane; i < n; i += 64) path[i] = i < count ? kept[i] : -1;
    if (lane == 0) a.accepted[r] = count, next[r] = choice[last];
}
template <typename Id>
__global__ __launch_bounds__(64) void tree_walk_kernel(AcceptCall a) {
    extern __shared__ int32_t walk_lds[];
    walk_request<Id>(a, blockIdx.x, threadIdx.x, walk_lds);
}

// One workgroup: lengths without the tokens that are not kept, and the pages behind them back to the ring, which takes sums over the requests.
// WALKS: of few requests it does the walks as well, a wave each.
constexpr int kBooksThreads = 1024;
template <typename Id, bool WALKS>
__global__ __launch_bounds__(kBooksThreads) void tree_books_kernel(AcceptCall a) {
    extern __shared__ int32_t walks_lds[];             // WALKS: [waves] as a walk has it
    if constexpr (WALKS) {
        const int w = threadIdx.x >> 6;                // as many waves as requests
        int32_t* const mine = walks_lds + w * a.shape.max_new * (2 + (int)sizeof(Id) / 4);
        walk_request<Id>(a, w, threadIdx.x & 63, mine);
        __syncthreads();
    }
    __shared__ int2 wave_sums[kBooksThreads / 64];     // pages back, bad requests
    const int tid = threadIdx.x, w = tid >> 6, waves = blockDim.x >> 6;
    const int shift = __builtin_ctz(a.shape.page_size), mask = a.shape.page_size - 1, pages = a.shape.num_pages;
    const int32_t then0 = a.ring_state[0], then1 = a.ring_state[1];
    const bool good_ring = then0 >= 0 && then0 < pages && then1 >= 0 && then1 <= pages;
    const int32_t head = good_ring ? then0 : 0, count = good_ring ? then1 : 0;
    auto pages_of = [&](int len) { return (int)(((int64_t)len + mask) >> shift); };
    struct Request { int len, left, keep, back; bool bad; };
    auto request = [&](int r) {
        Request q = {0, 0, 0, 0, false};
        int first, n;
        tree_tokens(a.cu_new, a.shape.tokens, r, first, n);
        q.len = a.lens[r];
        q.bad = bad_request(a, q.len, n);
        q.left = q.bad ? q.len : q.len - n + a.accepted[r];
        if (!q.bad) q.keep = pages_of(q.left), q.back = pages_of(q.len) - q.keep;
        return q;
    };
    // The sums; then, if nothing is wrong, the moves, whose order does not matter (what the ring takes is not what it holds).
    int back_all = 0, bad_all = 0;
    for (int turn = 0; turn < 2; ++turn) {
        const int64_t no_room = (int64_t)count + back_all - pages;
        const bool ok = turn == 0 || (bad_all == 0 && good_ring && no_room <= 0);
        if (turn == 1 && tid == 0) {
            a.status[0] = bad_all;
            a.status[1] = good_ring ? (int32_t)(no_room > 0 ? no_room : 0) : 1;
            a.ring_state_out[0] = then0;
            a.ring_state_out[1] = ok ? count + back_all : then1;
        }
        int before_all = 0;
        for (int r0 = 0; r0 < a.shape.requests; r0 += blockDim.x) {
            const int r = r0 + tid;
            Request q = {0, 0, 0, 0, false};
            if (r < a.shape.requests) q = request(r);
            if (turn == 1 && !ok) {
                if (r < a.shape.requests) {
                    int first, n;
                    tree_tokens(a.cu_new, a.shape.tokens, r, first, n);
                    for (int i = 0; i < n; ++i) a.path[first + i] = -1;
                    a.accepted[r] = 0, static_cast<Id*>(a.next_ids)[r] = -1, a.lens_out[r] = q.len;
                }
                continue;
            }
            int to = q.back;                           // sum up to and with this lane
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int y = __shfl_up(to, d);
                to += (tid & 63) >= d ? y : 0;
            }
            const int bad = (int)__popcll(__builtin_amdgcn_ballot_w64(q.bad));
            __syncthreads();                           // the totals before have been read
            if ((tid & 63) == 63) wave_sums[w] = make_int2(to, bad);
            __syncthreads();
            int before = before_all + to - q.back;
            for (int v = 0; v < waves; ++v) {
                const int2 s = wave_sums[v];
                if (v < w) before += s.x;
                before_all += s.x;
                if (turn == 0) back_all += s.x, bad_all += s.y;
            }
            if (turn == 1 && r < a.shape.requests) {
                const int32_t* row = a.table + (int64_t)r * a.shape.pages_per_request + q.keep;
                for (int i = 0; i < q.back; ++i) {
                    const int64_t at = (int64_t)head + count + before + i;          // < 2 pages, as there is room
                    a.ring[at < pages ? at : at - pages] = row[i];
                }
                a.lens_out[r] = q.left;
            }
        }
    }
}

// Up to 16 requests in one launch (16 drafts each, 16 requests: 5.1 us a call and 5.0 in a graph, with two launches 8.0 and 5.5; 256 drafts 6.4 and
// 6.5, 8.3 and 6.8).  Two walks after the other in a wave are slower in a graph: 32 requests 6.1 and 5.6.
constexpr int kWalksAtOnce = kBooksThreads / 64;
constexpr size_t kWalksLds = 64 << 10;

template <typename Id>
static int launch_accept(const AcceptCall& c, hipStream_t stream) {
    const stem_accept_shape& s = c.shape;
    const size_t lds = (size_t)s.max_new * (2 * sizeof(int32_t) + sizeof(Id));
    if (s.requests <= kWalksAtOnce && s.requests * lds <= kWalksLds) {
        hipLaunchKernelGGL((tree_books_kernel<Id, true>), dim3(1), dim3(s.requests * 64), s.requests * lds, stream, c);
        return check_launch();
    }
    const dim3 lanes(s.requests < kBooksThreads ? (s.requests + 63) / 64 * 64 : kBooksThreads);
    hipLaunchKernelGGL(tree_walk_kernel<Id>, dim3(s.requests), dim3(64), lds, stream, c);
    if (const int st = check_launch()) return st;
    hipLaunchKernelGGL((tree_books_kernel<Id, false>), dim3(1), lanes, 0, stream, c);
    return check_launch();
}
int launch_tree_accept(const AcceptCall& c, hipStream_t stream) {
    return c.shape.id_bits == 32 ? launch_accept<int32_t>(c, stream) : launch_accept<int64_t>(c, stream);
}

// --- kept rows move up --------------------------------------------------------------------------------------

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// A lane has 16 bytes of the request's rows and moves them for one kept token after the other.  path[k] >= k, and ascending: a row that is
// written has been read before, by this lane, as long as those of a turn are all read before the first is written.
constexpr int kCommitThreads = 256, kAtOnce = 8;
__global__ __launch_bounds__(kCommitThreads) void tree_commit_kernel(CommitCall a, int page_shift) {
    extern __shared__ int32_t commit_lds[];            // [max_new] from, [max_new] to
    __shared__ int ends;
    const int r = blockIdx.x, most = a.shape.max_new;
    int32_t *const from = commit_lds, *const to = commit_lds + most;
    int first, n;
    tree_tokens(a.cu_new, a.shape.tokens, r, first, n);
    n = min(n, most);
    if (threadIdx.x == 0) ends = n;
    for (int i = threadIdx.x; i < n; i += kCommitThreads) {
        from[i] = a.path[first + i];
        to[i] = a.slots[first + i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kCommitThreads)
        if ((uint32_t)from[i] >= (uint32_t)n) atomicMin(&ends, i);
    __syncthreads();
    n = ends;
    const int chunks = a.row_bytes / 16, all = 2 * a.heads * chunks;
    const uint32_t slots_end = (uint32_t)a.pages.num_pages * a.pages.page_size;
    const int c = blockIdx.y * kCommitThreads + threadIdx.x;
    if (c >= all) return;
    const int row = c / chunks, chunk = c - row * chunks, head = row < a.heads ? row : row - a.heads;
    char* const base = static_cast<char*>(row < a.heads ? a.k_pages : a.v_pages) + head * a.pages.stride_head * a.value_bytes + chunk * 16;
    auto place = [&](uint32_t slot) {
        const int64_t page = slot >> page_shift, in = slot & (a.pages.page_size - 1);
        return reinterpret_cast<u32x4_t*>(base + (page * a.pages.stride_page + in * a.pages.stride_token) * a.value_bytes);
    };
    for (int k0 = 0; k0 < n; k0 += kAtOnce) {
        u32x4_t held[kAtOnce];
        bool moves[kAtOnce];
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) {
            const int k = min(k0 + x, n - 1), i = from[k];
            moves[x] = k == k0 + x && i != k && (uint32_t)to[i] < slots_end && (uint32_t)to[k] < slots_end;
            held[x] = *place(moves[x] ? to[i] : 0);    // (a load from the first row where nothing moves)
        }
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x)
            if (moves[x]) *place(to[k0 + x]) = held[x];
    }
}

int launch_tree_commit(const CommitCall& c, hipStream_t stream) {
    const int all = 2 * c.heads * (c.row_bytes / 16);
    const dim3 grid(c.shape.requests, (all + kCommitThreads - 1) / kCommitThreads);
    hipLaunchKernelGGL(tree_commit_kernel, grid, dim3(kCommitThreads), 2 * sizeof(int32_t) * (size_t)c.shape.max_new, stream, c,
                       __builtin_ctz(c.pages.page_size));
    return check_launch();
}

}  // namespace stem
