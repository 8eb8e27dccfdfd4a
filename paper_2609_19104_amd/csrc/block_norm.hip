// Norm of a block's output, gate, residual, and the next block's norm and modulation in one pass (rm_block_norm).
#include "rm_serve.h"

namespace rm_serve {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));

// Eight elements as they lie in memory.
template <bool BF>
using Raw = typename std::conditional<BF, bf16x8, f32x8>::type;

template <bool BF>
__device__ __forceinline__ Raw<BF> load(const char *p, int64_t i) {
    return *reinterpret_cast<const Raw<BF> *>(p + i * (BF ? 2 : 4));
}
template <bool BF>
__device__ __forceinline__ void store(char *p, int64_t i, f32x8 v) {
    *reinterpret_cast<Raw<BF> *>(p + i * (BF ? 2 : 4)) = __builtin_convertvector(v, Raw<BF>);
}
__device__ __forceinline__ f32x8 load(const float *p, int c) { return *reinterpret_cast<const f32x8 *>(p + c); }

// A row's sum over its TPR threads.
template <int TPR>
__device__ __forceinline__ float sum_row(float s, float *red) {
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.0f;
        for (int w = 0; w < TPR / 64; ++w) s += red[w];
    }
    return s;
}

// TPR threads hold a row in registers, N chunks of 8 columns each, so that x and f are read once, all at the start.
template <bool XB, bool FB, bool OB, int TPR, int N>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void block_norm_kernel(NormArgs a) {
    constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;  // of a workgroup
    __shared__ float red[2][16];
    const int t = threadIdx.x % TPR;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    if (row >= a.rows) return;  // (the whole wave)
    const int b = static_cast<int>(row) / a.T;
    const int64_t base = row * a.d;
    Raw<XB> x[N];
    Raw<FB> f[N];
    f32x8 u[N];
    // Columns past the row's end are its last ones again, and count as zeros.
    int c[N];
    bool has[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        c[i] = (t + i * TPR) * 8;
        has[i] = c[i] < a.d;
        c[i] = min(c[i], a.d - 8);
        x[i] = load<XB>(a.x, base + c[i]);
        if (a.f) f[i] = load<FB>(a.f, base + c[i]);
    }
    if (a.f) {
        float rf = a.f_scale;
        if (a.norm_post) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float p = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) p = fmaf(static_cast<float>(f[i][e]), static_cast<float>(f[i][e]), p);
                s += has[i] ? p : 0.0f;
            }
            rf *= rm_rnorm_from_ssq(sum_row<TPR>(s, red[0]), a.d, a.eps);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f32x8 v = __builtin_convertvector(f[i], f32x8) * rf;
            if (a.gain_post) v *= load(a.gain_post, c[i]);
            if (a.gate) v *= load(a.gate + b * a.gate_b, c[i]);
            u[i] = __builtin_convertvector(x[i], f32x8) * a.x_scale + v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = __builtin_convertvector(x[i], f32x8) * a.x_scale;
    }
    if (a.y) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (has[i]) store<XB>(a.y, base + c[i], u[i]);
    }
    if (!a.out) return;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float p = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) p = fmaf(u[i][e], u[i][e], p);
        s += has[i] ? p : 0.0f;
    }
    const float ru = rm_rnorm_from_ssq(sum_row<TPR>(s, red[1]), a.d, a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f32x8 v = u[i] * ru;
        if (a.gain_pre) v *= load(a.gain_pre, c[i]);
        if (a.scale) v *= 1.0f + load(a.scale + b * a.scale_b, c[i]);
        if (a.shift) v += load(a.shift + b * a.shift_b, c[i]);
        if (has[i]) store<OB>(a.out, base + c[i], v);
    }
}

template <bool XB, bool FB, bool OB>
hipError_t by_row(const NormArgs &a, hipStream_t st) {
    const int chunks = a.d / 8;
    const auto rows = static_cast<unsigned>(a.rows);
    const dim3 fours((rows + 3) / 4), ones(rows);
    if (chunks <= 64) block_norm_kernel<XB, FB, OB, 64, 1><<<fours, 256, 0, st>>>(a);
    else if (a.rows >= a.many && chunks <= 128) block_norm_kernel<XB, FB, OB, 64, 2><<<fours, 256, 0, st>>>(a);
    else if (a.rows >= a.many && chunks <= 256) block_norm_kernel<XB, FB, OB, 64, 4><<<fours, 256, 0, st>>>(a);
    else if (chunks <= 256) block_norm_kernel<XB, FB, OB, 256, 1><<<ones, 256, 0, st>>>(a);
    else if (chunks <= 512) block_norm_kernel<XB, FB, OB, 256, 2><<<ones, 256, 0, st>>>(a);
    else if (chunks <= 1024) block_norm_kernel<XB, FB, OB, 256, 4><<<ones, 256, 0, st>>>(a);
    else if (chunks <= 2048) block_norm_kernel<XB, FB, OB, 1024, 2><<<ones, 1024, 0, st>>>(a);
    else block_norm_kernel<XB, FB, OB, 1024, 4><<<ones, 1024, 0, st>>>(a);
    return hipGetLastError();
}
template <bool XB, bool FB>
hipError_t by_out(const NormArgs &a, bool ob, hipStream_t st) {
    return ob ? by_row<XB, FB, true>(a, st) : by_row<XB, FB, false>(a, st);
}

}  // namespace

hipError_t launch_block_norm(const NormArgs &a, bool xb, bool fb, bool ob, hipStream_t st) {
    if (xb) return fb ? by_out<true, true>(a, ob, st) : by_out<true, false>(a, ob, st);
    return fb ? by_out<false, true>(a, ob, st) : by_out<false, false>(a, ob, st);
}

}  // namespace rm_serve
