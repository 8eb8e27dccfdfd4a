// bf16 attention kernels (rm_attn.h).
#include "rm_attn_bf16.h"

namespace rm_attn {

hipError_t launch_bf16(const Plan &p, const Args &a, hipStream_t st) {
    if (a.D == 64) return by_waves<true, 64, false>(p, a, st);
    if (a.D == 128) return by_waves<true, 128, false>(p, a, st);
    if (a.D == 256) return by_waves<true, 256, false>(p, a, st);
    if (a.D < 64) return by_waves<true, 64, true>(p, a, st);
    if (a.D <= 96) return by_waves<true, 96, true>(p, a, st);
    if (a.D < 128) return by_waves<true, 128, true>(p, a, st);
    if (a.D <= 192) return by_waves<true, 192, true>(p, a, st);
    return by_waves<true, 256, true>(p, a, st);
}

}  // namespace rm_attn
