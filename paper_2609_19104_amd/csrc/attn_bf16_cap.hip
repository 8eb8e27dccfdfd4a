// bf16 attention kernels for caps above kLowCap (rm_attn.h): kernels of their own, since the choice in the tile loop costs
// calls without a cap up to 6 % (8192 rows on 8192 keys, 16 heads of 64 on 4: 370 us, with it 393).  There is one for
// each width, which full heads take too.
#include "rm_attn_bf16.h"

namespace rm_attn {

hipError_t launch_bf16_high_cap(const Plan &p, const Args &a, hipStream_t st) {
    if (a.D <= 64) return by_waves<false, 64, true>(p, a, st);
    if (a.D <= 96) return by_waves<false, 96, true>(p, a, st);
    if (a.D <= 128) return by_waves<false, 128, true>(p, a, st);
    if (a.D <= 192) return by_waves<false, 192, true>(p, a, st);
    return by_waves<false, 256, true>(p, a, st);
}

}  // namespace rm_attn
