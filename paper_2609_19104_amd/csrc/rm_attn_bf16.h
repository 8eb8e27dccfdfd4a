// Launches of the bf16 attention kernels by head width and waves (attn_bf16.hip and attn_bf16_cap.hip).
#pragma once

#include "rm_attn.h"

namespace rm_attn {

template <bool LOW, int DH, int DC, bool PAD, int RW, int KW, int KT, int NBUF, int WPE>
static hipError_t go(const Args &a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.n_tiles) * a.splits * a.U * a.Hk);
    attn_kernel<true, LOW, DH, DC, PAD, RW, KW, KT, NBUF, WPE><<<grid, 64 * RW * KW, 0, st>>>(a);
    return hipGetLastError();
}

// The least of 64, 96, 128, 192 and 256 columns that hold the head.
template <bool LOW, int DC, bool PAD>
static hipError_t by_waves(const Plan &p, const Args &a, hipStream_t st) {
    if constexpr (DC == 64)
        return p.kw > 1 ? go<LOW, 64, DC, PAD, 1, 4, 128, 2, 2>(a, st) : go<LOW, 64, DC, PAD, 4, 1, 64, 2, 2>(a, st);
    else if constexpr (DC <= 128)
        return p.kw > 1 ? go<LOW, 128, DC, PAD, 1, 4, 128, 1, 2>(a, st) : go<LOW, 128, DC, PAD, 4, 1, 64, 2, 2>(a, st);
    else
        return p.kw > 1 ? go<LOW, 256, DC, PAD, 1, 4, 128, 1, 1>(a, st) : go<LOW, 256, DC, PAD, 4, 1, 64, 2, 1>(a, st);
}

}  // namespace rm_attn
