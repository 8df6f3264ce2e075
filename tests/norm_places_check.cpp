// The places of LDS that lanes use where a head's halves are exchanged through it (stem_norm.hip), one lane after the other on the CPU, for
// every head size and rotary part: who stores to each, and what is read from each.  Nothing here touches a GPU.
#include <cstdio>
#include <vector>

#include "stem_norm_common.h"

using namespace stem;

static int failed(const char* what, int W, int d, int rot, int lane, int e) {
    std::printf("%s: %d values a chunk, head of %d, %d turning, lane %d, value %d\n", what, W, d, rot, lane, e);
    return 1;
}

template <int W>
static int check(int d, int rot) {
    stem_rotary_shape s = {};
    s.dtype = W == 4 ? STEM_FP32 : STEM_BF16;
    s.head_dim = d, s.rotary_dim = rot, s.layout = STEM_ROTARY_HALF;
    const HeadLayout l = head_layout(s);
    if (!l.in_registers || l.pairs != kAcross) return 0;
    constexpr int S = W + 1;
    const int lanes = 1 << l.lane_bits, half = rot / 2;
    std::vector<int> value(lanes * 2 * S, -1), turn(l.padded, -1);     // which of the head's values, which pair's (cos, sin), is where
    for (int i = 0; i < half; ++i) turn[i + i / W] = i;
    auto of = [&](int lane) { return item_of<W, kAcross>(l.items, l.turning, half, d, lane); };
    for (int lane = 0; lane < lanes; ++lane) {
        const Item it = of(lane);
        if (it.pair < 0) continue;
        for (int e = 0; e < 2 * W; ++e) {
            const int chunk = e < W ? it.first : it.second, at = chunk / W * S + e % W;
            if (at < 0 || at >= (int)value.size()) return failed("stores outside", W, d, rot, lane, e);
            if (value[at] >= 0) return failed("stores to another lane's place", W, d, rot, lane, e);
            value[at] = chunk + e % W;
        }
    }
    for (int lane = 0; lane < lanes; ++lane) {
        const Item it = of(lane);
        if (it.pair < 0) continue;
        for (int e = 0; e < 2 * W; ++e) {
            const int chunk = e < W ? it.first : it.second, y = e % W, i = chunk + y, place = chunk / W * S;
            const int on = place_on<W>(half, y), back = place_back<W>(half, y), other = place + (i < half ? on : back), cs = place + (i < half ? y : back);
            if (other < 0 || other >= (int)value.size()) return failed("reads a value outside", W, d, rot, lane, e);
            if (cs < 0 || cs >= l.padded) return failed("reads (cos, sin) outside", W, d, rot, lane, e);
            if (i >= 2 * half) continue;                               // (not used)
            if (value[other] != (i < half ? i + half : i - half)) return failed("reads another value", W, d, rot, lane, e);
            if (turn[cs] != i % half) return failed("reads another pair's (cos, sin)", W, d, rot, lane, e);
        }
    }
    return 0;
}

int main() {
    int n = 0;
    for (int d = 8; d <= 1024; d += 8)
        for (int rot = 2; rot <= d; rot += 2) n += check<8>(d, rot) + check<4>(d, rot);
    std::printf("%d of the heads are wrong\n", n);
    return n != 0;
}
