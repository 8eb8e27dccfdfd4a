// Joins the partial results of the workgroups that divided a row block's keys (rm_attn.h).
#include "rm_attn_plan.h"

namespace rm_attn {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// LPR lanes per row, 4 columns a lane (D <= 4 LPR).  Slices are added in order, so the sums are the same on every
// call.  One launch of latency: 4 us for 408 rows of 256 columns in 8 slices, 7 for 128 rows of 128 in 32.  A slice
// without keys for the row has m = -inf and l = 0; its other sums are 0 or were not written, and are not used.
template <bool BF, int LPR>
__global__ __launch_bounds__(256) void combine_kernel(Args a) {
    const int64_t rows = static_cast<int64_t>(a.U) * a.Hk * a.R;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / LPR) + threadIdx.x / LPR;
    const int col = (threadIdx.x % LPR) * 4, c = min(col, a.D - 4);
    if (row >= rows) return;  // all of the row's lanes
    // The slices' maxima and sums, one slice a lane: their common maximum, and each slice's factor.
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + row;
    const float *po = a.part_o + row * a.D + c;
    const int lane = threadIdx.x % LPR;
    float top = -INFINITY;
    for (int s = lane; s < a.splits; s += LPR) top = fmaxf(top, ml[s * rows].x);
    for (int o = LPR / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    rm_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < a.splits; s0 += LPR) {
        const float2 mine = s0 + lane < a.splits ? ml[(s0 + lane) * rows] : make_float2(-INFINITY, 0.0f);
        const float f = __builtin_amdgcn_exp2f(mine.x - ref);  // 0 for a slice without keys
        const int n = min(a.splits - s0, LPR);
        for (int i0 = 0; i0 < n; i0 += 8) {
            rm_f32x4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = *reinterpret_cast<const rm_f32x4 *>(po + min(s0 + i0 + i, a.splits - 1) * rows * a.D);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int from = (i0 + i) % LPR;
                const float fi = __shfl(f, from, LPR), li = __shfl(mine.y, from, LPR);
                if (i0 + i < n && li != 0.0f) {
                    l += li * fi;
                    o += v[i] * fi;
                }
            }
        }
    }
    if (col >= a.D) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int ng = static_cast<int>(row / a.R), r = static_cast<int>(row - static_cast<int64_t>(ng) * a.R);
    const int u = ng / a.Hk, hk = ng - u * a.Hk;
    const int tok = r / a.G, g = r - tok * a.G;
    const int smp = tok / a.T, t = tok - smp * a.T;
    char *dst = a.o + (static_cast<int64_t>(u) * a.per + smp) * a.o_b + t * a.o_t +
                static_cast<int64_t>(hk * a.G + g) * a.o_h;
    if constexpr (BF) {
        bf16x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<__bf16>(o[i] * inv);
        *reinterpret_cast<bf16x4 *>(dst + c * 2) = w;
    } else {
        *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = o * inv;
    }
}

hipError_t launch_combine(bool bf16, const Args &a, hipStream_t st) {
    const int64_t rows = static_cast<int64_t>(a.U) * a.Hk * a.R;
    const int lpr = a.D > 128 ? 64 : a.D > 64 ? 32 : 16;
    const dim3 grid(static_cast<unsigned>((rows * lpr + 255) / 256));
    if (bf16) {
        if (lpr == 64) combine_kernel<true, 64><<<grid, 256, 0, st>>>(a);
        else if (lpr == 32) combine_kernel<true, 32><<<grid, 256, 0, st>>>(a);
        else combine_kernel<true, 16><<<grid, 256, 0, st>>>(a);
    } else {
        if (lpr == 64) combine_kernel<false, 64><<<grid, 256, 0, st>>>(a);
        else if (lpr == 32) combine_kernel<false, 32><<<grid, 256, 0, st>>>(a);
        else combine_kernel<false, 16><<<grid, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace rm_attn
