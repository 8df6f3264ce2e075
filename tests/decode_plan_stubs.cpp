// Windows on the split of the attention to a shared prefix, beside tests/decode_launch_stubs.cpp in a host-only build.
#include "stem_decode_common.h"

extern "C" int stem_test_suffix_split_keys(int32_t len, int32_t splits) { return stem::suffix_split_keys(len, splits); }
