// Attention of one new token over a paged cache (rm_paged_attention).
#include "rm_attn.h"
#include "rm_serve.h"

namespace rm_serve {

namespace {

template <bool BF>
__device__ __forceinline__ float at(const char *p, int i) {
    if constexpr (BF) return static_cast<float>(reinterpret_cast<const __bf16 *>(p)[i]);
    else return reinterpret_cast<const float *>(p)[i];
}

// One workgroup a token and query head, its waves taking keys by turns; a lane holds up to four of the columns.
template <bool BF>
__global__ __launch_bounds__(256) void paged_kernel(PagedArgs a) {
    __shared__ float so[4][256], sm[4], sl[4];
    const int n = blockIdx.x / a.Hq, h = blockIdx.x - n * a.Hq, hk = h / a.G;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int s = a.seq ? a.seq[n] : n, pos = a.pos[n];
    const int64_t cap = static_cast<int64_t>(a.per) * a.page;
    int end = s < 0 || s >= a.seqs || pos < 0 ? 0 : static_cast<int>(min(static_cast<int64_t>(pos) + 1, cap));
    const int lo = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
    const int32_t *table = a.table + static_cast<int64_t>(end > 0 ? s : 0) * a.per;
    const char *q = a.q + n * a.q_t + h * a.q_h;
    const float slope = a.slopes ? a.slopes[h] * rm_attn::kLog2e : 0.0f;
    float qv[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0.0f;
    for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < a.D ? at<BF>(q, lane + 64 * i) : 0.0f;
    for (int j = lo + wave; j < end; j += 4) {
        const int p = table[j / a.page];
        if (p < 0 || p >= a.n_pages) continue;
        const char *k = a.k + p * a.k_p + (j % a.page) * a.k_t + hk * a.k_h;
        const char *v = a.v + p * a.v_p + (j % a.page) * a.v_t + hk * a.v_h;
        float x = 0.0f;
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.D) x = fmaf(qv[i], at<BF>(k, lane + 64 * i), x);
        for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
        x *= a.scale;
        if (a.cap != 0.0f) x = a.cap * tanhf(x);
        x -= slope * static_cast<float>(pos - j);
        if (x > m) {
            const float f = m == -INFINITY ? 0.0f : exp2f(m - x);
            l *= f;
            for (int i = 0; i < 4; ++i) o[i] *= f;
            m = x;
        }
        const float w = m == -INFINITY ? (x == -INFINITY ? 0.0f : x) : exp2f(x - m);
        l += w;
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < a.D) o[i] = w == 0.0f && x == -INFINITY ? o[i] : fmaf(w, at<BF>(v, lane + 64 * i), o[i]);
    }
    for (int i = 0; i < 4; ++i) so[wave][lane + 64 * i] = o[i];
    if (lane == 0) sm[wave] = m, sl[wave] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    float total = 0.0f, r = 0.0f;
    const int c = threadIdx.x;
    for (int w = 0; w < 4; ++w) {
        if (sl[w] == 0.0f) continue;
        const float f = exp2f(sm[w] - top);
        total += sl[w] * f;
        r += so[w][c] * f;
    }
    r = total == 0.0f ? 0.0f : r / total;
    if (c >= a.D) return;
    char *dst = a.o + n * a.o_t + h * a.o_h;
    if constexpr (BF) reinterpret_cast<__bf16 *>(dst)[c] = static_cast<__bf16>(r);
    else reinterpret_cast<float *>(dst)[c] = r;
}

}  // namespace

hipError_t launch_paged(const PagedArgs &a, bool bf16, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.N) * a.Hq);
    if (bf16) paged_kernel<true><<<grid, 256, 0, st>>>(a);
    else paged_kernel<false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rm_serve
