// Per-head RMSNorm and position rotation of queries and keys, keys and values into cache rows (rm_qk_norm_rope).
#include <algorithm>

#include "rm_rope.h"

namespace rm {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// V elements at p to and from float32.
template <bool BF, int V>
__device__ __forceinline__ void load(const char *p, float (&x)[V]) {
    if constexpr (BF) {
        typedef __bf16 vec __attribute__((ext_vector_type(V)));
        const vec v = *reinterpret_cast<const vec *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = static_cast<float>(v[i]);
    } else {
        constexpr int W = V < 4 ? V : 4;
        typedef float vec __attribute__((ext_vector_type(W)));
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
            const vec v = reinterpret_cast<const vec *>(p)[j];
#pragma unroll
            for (int i = 0; i < W; ++i) x[j * W + i] = v[i];
        }
    }
}
template <bool BF, int V>
__device__ __forceinline__ void store(char *p, const float (&x)[V]) {
    if constexpr (BF) {
        typedef __bf16 vec __attribute__((ext_vector_type(V)));
        vec v;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = static_cast<__bf16>(x[i]);
        *reinterpret_cast<vec *>(p) = v;
    } else {
        constexpr int W = V < 4 ? V : 4;
        typedef float vec __attribute__((ext_vector_type(W)));
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
            vec v;
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = x[j * W + i];
            reinterpret_cast<vec *>(p)[j] = v;
        }
    }
}

// V consecutive float32 values of 4-byte alignment.
template <int V>
__device__ __forceinline__ void load_unaligned(const float *p, float (&x)[V]) {
    constexpr int W = V < 4 ? V : 4;
    typedef float vec __attribute__((ext_vector_type(W), aligned(4)));
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
        const vec v = *reinterpret_cast<const vec *>(p + j * W);
#pragma unroll
        for (int i = 0; i < W; ++i) x[j * W + i] = v[i];
    }
}

// A head's D elements are chunks of V; a lane holds two of them, those whose elements rotate with each other where
// the pairs are halves apart, so that no lane needs another's values but for the sum of squares.  A wave works on one
// token, whose sines and cosines its lanes compute once: its lane groups (a power of two lanes, as a head has chunk
// pairs) take consecutive heads, so that the wave reads and writes consecutive memory, and then the next ones, HB at a
// time with the following HB heads' loads in flight.
//
// Bound by memory: 32768 tokens of 32 + 2 x 8 heads of 128 in bf16 take 157 us, 5.1 TB/s of reads and writes (a copy: 4.7).
// A lane group that took a token's heads one after the other, the angles anew every four, took 304 us, with them once
// for all heads 263 (its 64 lanes then touched 8 tokens far apart).  850 tokens of 8 + 2 x 1 heads of 256 take 5.7 us
// and 51 3.5, which are a launch and two round trips.
template <bool IBF, bool OBF, int V, int HB>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeArgs a) {
    constexpr int IS = IBF ? 2 : 4, OS = OBF ? 2 : 4;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int n = wave / a.groups;
    if (n >= a.N) return;
    const int lane = threadIdx.x & 63, stride = 64 >> a.lane_bits;
    const int h_begin = (wave - n * a.groups) * a.per, h_end = min(h_begin + a.per, a.H);
    const int h0 = h_begin + (lane >> a.lane_bits);
    const int unit = lane & ((1 << a.lane_bits) - 1);
    const int rot_units = a.rot / (2 * V), chunks = a.D / V;
    // Elements of this lane's chunks; those it does not have are read as another's and count as zeros.
    const bool rotated = unit < rot_units;
    const int c0 = rotated ? (a.pairs ? 2 * unit : unit) : 2 * unit;
    const int c1 = rotated ? (a.pairs ? 2 * unit + 1 : unit + rot_units) : 2 * unit + 1;
    const bool has_a = c0 < chunks, has_b = c1 < chunks;
    const int ca = has_a ? c0 * V : 0, cb = has_b ? c1 * V : 0;
    const int n_qk = a.Hq + a.Hk;
    const char *const q = a.q + n * a.q_t, *const k = a.k + n * a.k_t, *const v = a.v ? a.v + n * a.v_t : nullptr;

    float xa[HB][V], xb[HB][V], ya[HB][V], yb[HB][V];
    auto fetch = [&](int h_first, float(&x)[HB][V], float(&y)[HB][V]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int h = min(h_first + i * stride, h_end - 1);  // (past the last: the last again)
            const char *src = h < a.Hq ? q + h * a.q_h : h < n_qk ? k + (h - a.Hq) * a.k_h : v + (h - n_qk) * a.v_h;
            load<IBF, V>(src + ca * IS, x[i]);
            load<IBF, V>(src + cb * IS, y[i]);
        }
    };
    fetch(h0, xa, xb);
    const int row = a.slot ? a.slot[n] : n;
    const bool keep_row = row >= 0 && row < a.rows;
    float fr[V], ga[V], gb[V];
    if (rotated) load_unaligned<V>(a.inv_freq + unit * V, fr);
    // The gain at this lane's elements: of the queries, then of the keys.
    auto load_gain = [&](const float *gain) __attribute__((always_inline)) {
        load_unaligned<V>(gain + ca, ga);
        load_unaligned<V>(gain + cb, gb);
    };
    const float *gain = h0 < a.Hq ? a.gain_q : a.gain_k;
    if (gain) load_gain(gain);
    // Angles in turns, in 64 bits: a far position times a frequency has more whole turns than float32 has digits for.
    float cs[V], sn[V];
    if (rotated && h_begin < n_qk) {
        const double pos = static_cast<double>(a.pos[n]) * 0.15915494309189535;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const double t = pos * static_cast<double>(fr[j]);
            sincospif(2.0f * static_cast<float>(t - rint(t)), &sn[j], &cs[j]);
        }
    }
    bool keys = h0 >= a.Hq;  // whose gain is loaded
    for (int h_first = h0; h_first < h_end; h_first += HB * stride) {
        if (HB > 1) fetch(h_first + HB * stride, ya, yb);
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int h = h_first + i * stride;
            if (h >= h_end) break;
            const bool is_v = h >= n_qk;
            if (!is_v) {
                gain = h < a.Hq ? a.gain_q : a.gain_k;
                if (gain) {
                    if (h >= a.Hq && !keys) {
                        load_gain(gain);
                        keys = true;
                    }
                    float sa = 0.0f, sb = 0.0f;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        sa = fmaf(xa[i][j], xa[i][j], sa);
                        sb = fmaf(xb[i][j], xb[i][j], sb);
                    }
                    float ss = (has_a ? sa : 0.0f) + (has_b ? sb : 0.0f);
                    for (int o = 1 << a.lane_bits >> 1; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
                    const float rn = rm_rnorm_from_ssq(ss, a.D, a.eps);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        xa[i][j] *= rn * ga[j];
                        xb[i][j] *= rn * gb[j];
                    }
                }
                if (rotated) {
                    if (a.pairs) {  // elements 2 j and 2 j + 1 of the lane's 2 V
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            float &e0 = 2 * j < V ? xa[i][(2 * j) % V] : xb[i][(2 * j) % V];
                            float &e1 = 2 * j < V ? xa[i][(2 * j + 1) % V] : xb[i][(2 * j + 1) % V];
                            const float u0 = e0, u1 = e1;
                            e0 = u0 * cs[j] - u1 * sn[j];
                            e1 = u1 * cs[j] + u0 * sn[j];
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float u0 = xa[i][j], u1 = xb[i][j];
                            xa[i][j] = u0 * cs[j] - u1 * sn[j];
                            xb[i][j] = u1 * cs[j] + u0 * sn[j];
                        }
                    }
                }
            }
            char *dst;
            if (h < a.Hq) dst = a.q_out + n * a.qo_t + h * a.qo_h;
            else if (!is_v) dst = a.k_out + row * a.ko_t + (h - a.Hq) * a.ko_h;
            else dst = a.v_out + row * a.vo_t + (h - n_qk) * a.vo_h;
            if (h < a.Hq || keep_row) {
                if (has_a) store<OBF, V>(dst + ca * OS, xa[i]);
                if (has_b) store<OBF, V>(dst + cb * OS, xb[i]);
            }
        }
        if (HB > 1) {
#pragma unroll
            for (int i = 0; i < HB; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) xa[i][j] = ya[i][j], xb[i][j] = yb[i][j];
        }
    }
}

template <bool IBF, bool OBF, int V>
hipError_t go(RopeArgs a, hipStream_t st) {
    const int units = a.rot / (2 * V) + (a.D / V - a.rot / V + 1) / 2;
    a.lane_bits = 0;
    while ((1 << a.lane_bits) < units) ++a.lane_bits;
    // All heads of a token in one wave, sharing its sines and cosines, once that gives every SIMD four waves; fewer tokens
    // divide their heads among waves, down to as many heads as a wave has lane groups (bf16, us, one wave a token / as
    // many as can be: 51 tokens of 48 heads of 128 8.3 / 3.9, 850 9.6 / 8.0, 2000 12.8 / 15.1, 4000 17.8 / 23.5).
    const int at_once = 64 >> a.lane_bits, most = (a.H + at_once - 1) / at_once;
    const int groups = std::min(most, std::max(1, 4096 / a.N));
    a.per = (most + groups - 1) / groups * at_once;
    a.groups = (a.H + a.per - 1) / a.per;
    const int64_t wgs = (static_cast<int64_t>(a.N) * a.groups + 3) / 4;
    if (a.per > at_once) qk_norm_rope_kernel<IBF, OBF, V, 2><<<dim3(static_cast<unsigned>(wgs)), 256, 0, st>>>(a);
    else qk_norm_rope_kernel<IBF, OBF, V, 1><<<dim3(static_cast<unsigned>(wgs)), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int V>
hipError_t by_type(const RopeArgs &a, bool ibf, bool obf, hipStream_t st) {
    if (ibf) return obf ? go<true, true, V>(a, st) : go<true, false, V>(a, st);
    return obf ? go<false, true, V>(a, st) : go<false, false, V>(a, st);
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs &a, bool in_bf16, bool out_bf16, hipStream_t st) {
    // Chunks of 8 elements (16 bytes of bf16) where the rotated half is made of whole ones, else of 4 or 2.
    const int part = a.rot / 2;
    if (part % 8 == 0) return by_type<8>(a, in_bf16, out_bf16, st);
    if (part % 4 == 0) return by_type<4>(a, in_bf16, out_bf16, st);
    return by_type<2>(a, in_bf16, out_bf16, st);
}

}  // namespace rm
