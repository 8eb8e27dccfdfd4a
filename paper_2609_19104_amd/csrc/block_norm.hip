// Norm of a block's output, gate, residual, and the next block's norm and modulation in one pass (rm_block_norm).
#include "rm_serve.h"

namespace rm_serve {

namespace {

template <bool BF>
__device__ __forceinline__ float load(const char *p, int64_t i) {
    if constexpr (BF) return static_cast<float>(reinterpret_cast<const __bf16 *>(p)[i]);
    else return reinterpret_cast<const float *>(p)[i];
}
template <bool BF>
__device__ __forceinline__ void store(char *p, int64_t i, float v) {
    if constexpr (BF) reinterpret_cast<__bf16 *>(p)[i] = static_cast<__bf16>(v);
    else reinterpret_cast<float *>(p)[i] = v;
}

// One workgroup a row, three passes over it.
template <bool XB, bool FB, bool OB>
__global__ __launch_bounds__(256) void block_norm_kernel(NormArgs a) {
    __shared__ float red[4];
    const int64_t row = blockIdx.x, base = row * a.d;
    const int64_t b = row / a.T;
    const int tid = threadIdx.x;
    auto sum_all = [&](float s) {
        for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
        __syncthreads();
        if ((tid & 63) == 0) red[tid >> 6] = s;
        __syncthreads();
        return (red[0] + red[1]) + (red[2] + red[3]);
    };
    float rf = 1.0f;
    if (a.f && a.norm_post) {
        float s = 0.0f;
        for (int c = tid; c < a.d; c += 256) {
            const float f = load<FB>(a.f, base + c);
            s = fmaf(f, f, s);
        }
        rf = rm_rnorm_from_ssq(sum_all(s), a.d, a.eps);
    }
    auto value = [&](int c) {
        float u = a.x_scale * load<XB>(a.x, base + c);
        if (a.f) {
            float f = load<FB>(a.f, base + c) * rf;
            if (a.gain_post) f *= a.gain_post[c];
            if (a.gate) f *= a.gate[b * a.gate_b + c];
            u = fmaf(a.f_scale, f, u);
        }
        return u;
    };
    float ru = 0.0f;
    if (a.out) {
        float s = 0.0f;
        for (int c = tid; c < a.d; c += 256) {
            const float u = value(c);
            s = fmaf(u, u, s);
        }
        ru = rm_rnorm_from_ssq(sum_all(s), a.d, a.eps);
    }
    for (int c = tid; c < a.d; c += 256) {
        const float u = value(c);
        if (a.out) {
            float o = u * ru;
            if (a.gain_pre) o *= a.gain_pre[c];
            if (a.scale) o *= 1.0f + a.scale[b * a.scale_b + c];
            if (a.shift) o += a.shift[b * a.shift_b + c];
            store<OB>(a.out, base + c, o);
        }
        if (a.y) store<XB>(a.y, base + c, u);
    }
}

template <bool XB, bool FB>
hipError_t by_out(const NormArgs &a, bool ob, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.rows));
    if (ob) block_norm_kernel<XB, FB, true><<<grid, 256, 0, st>>>(a);
    else block_norm_kernel<XB, FB, false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const NormArgs &a, bool xb, bool fb, bool ob, hipStream_t st) {
    if (xb) return fb ? by_out<true, true>(a, ob, st) : by_out<true, false>(a, ob, st);
    return fb ? by_out<false, true>(a, ob, st) : by_out<false, false>(a, ob, st);
}

}  // namespace rm_serve
