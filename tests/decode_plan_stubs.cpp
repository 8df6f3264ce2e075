// Windows on the split of the attention to a shared prefix, beside tests/decode_launch_stubs.cpp in a host-only build.
#include "stem_decode_common.h"

extern "C" int stem_test_suffix_split_keys(int32_t len, int32_t splits) { return stem::suffix_split_keys(len, splits); }
extern "C" int stem_test_suffix_parts(int32_t len, int32_t splits) { return stem::suffix_parts(len, splits); }

static int units_there;
static int there() { return units_there; }
// prefix_groups, groups, own_slots, own_by_rows, join_rows, join_by_rows
extern "C" int stem_test_prefix_launches(const stem_prefix_shape* shape, int32_t units, int64_t* out) {
    units_there = units;
    stem::PrefixPlan p;
    const int st = stem::prefix_plan(*shape, &p, there);
    if (st != STEM_OK) return st;
    const int64_t all[] = {p.prefix_groups, p.groups, p.own_slots, p.own_by_rows, p.join_rows, p.join_by_rows};
    for (int i = 0; i < 6; ++i) out[i] = all[i];
    return STEM_OK;
}
extern "C" int64_t stem_test_slot_before(int32_t r, int64_t row, int32_t tile) { return stem::slot_before(r, row, tile); }
