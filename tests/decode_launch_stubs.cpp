// Stand-ins for the kernel launchers of include/stem_decode.h, for a host-only build of its host code.  Nothing here touches a
// GPU: a launch that the host code lets through is recorded as done.  stem_test_prefix_plan gives the split of the attention to
// a shared prefix for a device of so many compute units.
#include "stem_decode_common.h"

namespace stem {

int launch_rotary(const RotaryCall&, hipStream_t) { return STEM_OK; }
int launch_block_table(const TableCall&, hipStream_t) { return STEM_OK; }
int launch_prefix_attn(const PrefixCall&, hipStream_t) { return STEM_OK; }

}  // namespace stem

static int units_of_device;
static int give_units() { return units_of_device; }
extern "C" int stem_test_prefix_plan(const stem_prefix_shape* shape, int32_t units, int64_t* out) {
    units_of_device = units;
    stem::PrefixPlan p;
    const int st = stem::prefix_plan(*shape, &p, give_units);
    if (st != STEM_OK) return st;
    const int64_t all[] = {p.row_tile, p.row_tiles, p.prefix_splits, p.split_keys, p.suffix_row_tile, p.suffix_row_tiles,
                           p.suffix_splits, (int64_t)p.partial_ml, (int64_t)p.bytes, p.small};
    for (int i = 0; i < 10; ++i) out[i] = all[i];
    return STEM_OK;
}
