// float32 attention kernels (rm_attn.h), on the float32 matrix cores.
#include "rm_attn.h"

namespace rm_attn {

template <int DH, int DC, bool PAD, int RW, int KW, int KT, int NBUF, int WPE>
static hipError_t go(const Args &a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.n_tiles) * a.splits * a.U * a.Hk);
    attn_kernel<false, false, DH, DC, PAD, RW, KW, KT, NBUF, WPE><<<grid, 64 * RW * KW, 0, st>>>(a);
    return hipGetLastError();
}

// The least of 64, 96, 128, 192 and 256 columns that hold the head.
template <int DC, bool PAD>
static hipError_t by_waves(const Plan &p, const Args &a, hipStream_t st) {
    if constexpr (DC == 64)
        return p.kw > 1 ? go<64, DC, PAD, 1, 4, 128, 1, 2>(a, st) : go<64, DC, PAD, 4, 1, 64, 2, 2>(a, st);
    else if constexpr (DC <= 128)
        return p.kw > 1 ? go<128, DC, PAD, 1, 4, 128, 1, 1>(a, st) : go<128, DC, PAD, 4, 1, 64, 1, 2>(a, st);
    else
        return go<256, DC, PAD, 2, 2, 64, 1, 1>(a, st);  // (the plan has p.kw > 1 here)
}

hipError_t launch_f32(const Plan &p, const Args &a, hipStream_t st) {
    if (a.D == 64) return by_waves<64, false>(p, a, st);
    if (a.D == 128) return by_waves<128, false>(p, a, st);
    if (a.D == 256) return by_waves<256, false>(p, a, st);
    if (a.D < 64) return by_waves<64, true>(p, a, st);
    if (a.D <= 96) return by_waves<96, true>(p, a, st);
    if (a.D < 128) return by_waves<128, true>(p, a, st);
    if (a.D <= 192) return by_waves<192, true>(p, a, st);
    return by_waves<256, true>(p, a, st);
}

}  // namespace rm_attn
