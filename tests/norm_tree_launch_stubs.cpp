// Stand-ins for the kernel launchers of include/stem_norm.h and include/stem_tree.h, beside tests/decode_launch_stubs.cpp in a host-only
// build of their host code.  Nothing here touches a GPU: a launch that the host code lets through is recorded as done.
// stem_test_tree_plan gives the split of the attention of drafted tokens for a device of so many compute units.
#include "stem_norm_common.h"
#include "stem_tree_common.h"

namespace stem {

int launch_norm_rotary(const NormCall&, hipStream_t) { return STEM_OK; }
int launch_norm_rotary_backward(const NormCall&, hipStream_t) { return STEM_OK; }
int launch_tree_masks(const TreeMasksCall&, hipStream_t) { return STEM_OK; }
int launch_tree_accept(const AcceptCall&, hipStream_t) { return STEM_OK; }
int launch_tree_commit(const CommitCall&, hipStream_t) { return STEM_OK; }
int launch_tree_attn(const PrefixCall&, const int64_t*, hipStream_t) { return STEM_OK; }

}  // namespace stem

static int units_of_tree;
static int give_tree_units() { return units_of_tree; }
extern "C" int stem_test_tree_plan(const stem_prefix_shape* shape, int32_t units, int64_t* out) {
    units_of_tree = units;
    stem::PrefixPlan p;
    const int st = stem::prefix_plan(*shape, &p, give_tree_units, true);
    if (st != STEM_OK) return st;
    const int64_t all[] = {p.suffix_row_tile, p.suffix_row_tiles, p.suffix_splits, p.suffix_least, p.prefix_splits, p.own_slots,
                           (int64_t)p.partial_ml, (int64_t)p.bytes, p.small, p.groups};
    for (int i = 0; i < 10; ++i) out[i] = all[i];
    return STEM_OK;
}
extern "C" int stem_test_split_keys(int32_t len, int32_t splits, int32_t least) { return stem::suffix_split_keys(len, splits, least); }
extern "C" int stem_test_parts(int32_t len, int32_t splits, int32_t least) { return stem::suffix_parts(len, splits, least); }
