// bf16 attention kernels (rm_attn.h).
#include "rm_attn.h"

namespace rm_attn {

template <int DH, int RW, int KW, int QB, int KT, int NBUF, int WPE>
static hipError_t go(const Plan &p, const Args &a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.n_tiles) * a.splits * a.U * a.Hk);
    if (p.pad) attn_kernel<true, DH, true, RW, KW, QB, KT, NBUF, WPE><<<grid, 64 * RW * KW, 0, st>>>(a);
    else attn_kernel<true, DH, false, RW, KW, QB, KT, NBUF, WPE><<<grid, 64 * RW * KW, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_bf16(const Plan &p, const Args &a, hipStream_t st) {
    if (p.kw > 1) {
        if (p.dh == 64) return go<64, 1, 4, 1, 128, 2, 2>(p, a, st);
        if (p.dh == 128) return go<128, 1, 4, 1, 128, 1, 2>(p, a, st);
        return go<256, 1, 4, 1, 128, 1, 1>(p, a, st);
    }
    if (p.dh == 64) return go<64, 4, 1, 1, 64, 2, 2>(p, a, st);
    if (p.dh == 128) return go<128, 4, 1, 1, 64, 2, 2>(p, a, st);
    return go<256, 4, 1, 1, 64, 2, 1>(p, a, st);
}

}  // namespace rm_attn
