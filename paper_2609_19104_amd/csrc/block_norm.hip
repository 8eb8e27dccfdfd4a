// Norm of a block's output, gate, residual, and the next block's norm and modulation in one pass (rm_block_norm).
#include <algorithm>

#include "rm_serve.h"

namespace rm_serve {

namespace {

template <int V>
using Floats = float __attribute__((ext_vector_type(V), aligned(16)));

// V elements as they lie in memory.
template <bool BF, int V>
using Raw = typename std::conditional<BF, __bf16 __attribute__((ext_vector_type(V))), Floats<V>>::type;

// Nontemporal: a row is read once and not written again, and passes by the caches' other lines.
template <bool BF, int V>
__device__ __forceinline__ Raw<BF, V> load(const char *p, int64_t i) {
    return __builtin_nontemporal_load(reinterpret_cast<const Raw<BF, V> *>(p + i * (BF ? 2 : 4)));
}
template <bool BF, int V>
__device__ __forceinline__ void store(char *p, int64_t i, Floats<V> v) {
    __builtin_nontemporal_store(__builtin_convertvector(v, Raw<BF, V>), reinterpret_cast<Raw<BF, V> *>(p + i * (BF ? 2 : 4)));
}
template <int V>
__device__ __forceinline__ Floats<V> load(const float *p, int c) {
    return *reinterpret_cast<const Floats<V> *>(p + c);
}

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

// TPR threads hold a row in registers, N chunks of V columns each, so that x and f are read once, all at the start, and
// both sums of squares and the norms are float32.  A chunk is 16 bytes of the widest of the three types, so that a wave's
// loads of it are consecutive.  out is made of u before u is rounded for y: two roundings fewer than from y.
//
// Bound by memory: 16384 rows of 2048 columns, float32 x and y, bf16 f and out, gains, gate, scale and shift: 77 us, 5.2 TB/s
// (a copy: 4.9).  On the way there: three passes over a row 282; a wave a row in registers, eight columns a chunk, 99.5, as
// its float32 loads leave every other 16 bytes to the next one; 256 threads a row 94; past the caches 90.  850 rows 5.9 us
// and 51 of 1024 columns 3.4, in a graph: a launch and two trips to memory.
template <bool XB, bool FB, bool OB, int TPR, int N>
__global__ __launch_bounds__(TPR < 128 ? 256 : TPR) void block_norm_kernel(NormArgs a) {
    constexpr int V = XB && FB && OB ? 8 : 4, ROWS = TPR < 128 ? 256 / TPR : 1;  // rows of a workgroup
    typedef Floats<V> Vec;
    __shared__ float red[2][16];
    const int t = threadIdx.x % TPR;
    const int64_t row = a.row0 + static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    if (row >= a.rows) return;  // (the whole wave, and with more than one wave to a row the whole workgroup)
    const int b = static_cast<int>(row) / a.T;
    const int64_t base = row * a.d;
    Raw<XB, V> x[N];
    Raw<FB, V> f[N];
    Vec u[N];
    // Columns past the row's end are its last ones again, and count as zeros.
    int c[N];
    bool has[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        c[i] = (t + i * TPR) * V;
        has[i] = c[i] < a.d;
        c[i] = min(c[i], a.d - V);
        x[i] = load<XB, V>(a.x, base + c[i]);
        if (a.f) f[i] = load<FB, V>(a.f, base + c[i]);
    }
    if (a.f) {
        float rf = a.f_scale;
        if (a.norm_post) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float p = 0.0f;
#pragma unroll
                for (int e = 0; e < V; ++e) p = fmaf(static_cast<float>(f[i][e]), static_cast<float>(f[i][e]), p);
                s += has[i] ? p : 0.0f;
            }
            rf *= rm_rnorm_from_ssq(sum_row<TPR>(s, red[0]), a.d, a.eps);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            Vec v = __builtin_convertvector(f[i], Vec) * rf;
            if (a.gain_post) v *= load<V>(a.gain_post, c[i]);
            if (a.gate) v *= load<V>(a.gate + b * a.gate_b, c[i]);
            u[i] = __builtin_convertvector(x[i], Vec) * a.x_scale + v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = __builtin_convertvector(x[i], Vec) * a.x_scale;
    }
    if (a.y) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (has[i]) store<XB, V>(a.y, base + c[i], u[i]);
    }
    if (!a.out) return;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float p = 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) p = fmaf(u[i][e], u[i][e], p);
        s += has[i] ? p : 0.0f;
    }
    const float ru = rm_rnorm_from_ssq(sum_row<TPR>(s, red[1]), a.d, a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        Vec v = u[i] * ru;
        if (a.gain_pre) v *= load<V>(a.gain_pre, c[i]);
        if (a.scale) v *= 1.0f + load<V>(a.scale + b * a.scale_b, c[i]);
        if (a.shift) v += load<V>(a.shift + b * a.shift_b, c[i]);
        if (has[i]) store<OB, V>(a.out, base + c[i], v);
    }
}

template <bool XB, bool FB, bool OB, int TPR, int COLUMNS>
hipError_t go(const NormArgs &a, hipStream_t st) {
    constexpr int V = XB && FB && OB ? 8 : 4, ROWS = TPR < 128 ? 256 / TPR : 1, THREADS = TPR < 128 ? 256 : TPR;
    // A launch holds below 2^32 threads: of rows above 8192 columns 2^22 - 1.
    constexpr int64_t most = INT64_C(0xffffffff) / THREADS * ROWS;
    for (NormArgs part = a; part.row0 < a.rows; part.row0 += most) {
        const int64_t rows = std::min(a.rows - part.row0, most);
        block_norm_kernel<XB, FB, OB, TPR, COLUMNS / V><<<static_cast<unsigned>((rows + ROWS - 1) / ROWS), THREADS, 0, st>>>(part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
// Eight columns a thread while 256 threads hold the row with that, then more.
template <bool XB, bool FB, bool OB>
hipError_t by_row(const NormArgs &a, hipStream_t st) {
    if (a.d <= 512) return go<XB, FB, OB, 64, 8>(a, st);
    if (a.d <= 1024) return go<XB, FB, OB, 128, 8>(a, st);
    if (a.d <= 2048) return go<XB, FB, OB, 256, 8>(a, st);
    if (a.d <= 4096) return go<XB, FB, OB, 256, 16>(a, st);
    if (a.d <= 8192) return go<XB, FB, OB, 256, 32>(a, st);
    if (a.d <= 16384) return go<XB, FB, OB, 1024, 16>(a, st);
    return go<XB, FB, OB, 1024, 32>(a, st);
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
