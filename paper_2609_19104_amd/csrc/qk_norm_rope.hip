// Per-head RMSNorm and position rotation of queries and keys, keys and values into cache rows (rm_qk_norm_rope).
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

// A head's D elements are chunks of V; a lane holds two of them, those whose elements rotate with each other where
// the pairs are halves apart, so that no lane needs another's values but for the sum of squares.  `lanes` (a power
// of two) lanes work on one token's heads h0, h0 + 1, ..., HPG of them, with the token's sines and cosines computed
// once and the loads of all HPG heads in flight together.
template <bool IBF, bool OBF, int V, int HPG>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(RopeArgs a) {
    constexpr int IS = IBF ? 2 : 4, OS = OBF ? 2 : 4;
    const int gid = static_cast<int>(blockIdx.x) * (256 >> a.lane_bits) + (threadIdx.x >> a.lane_bits);
    const int n = gid / a.groups, h0 = (gid - n * a.groups) * HPG;
    const int unit = threadIdx.x & ((1 << a.lane_bits) - 1);
    if (n >= a.N) return;  // a whole lane group: the others' shuffles stay within theirs
    const int rot_units = a.rot / (2 * V), chunks = a.D / V;
    // Chunks of this lane (-1: none).
    int ca = -1, cb = -1;
    if (unit < rot_units) {
        ca = a.pairs ? 2 * unit : unit;
        cb = a.pairs ? 2 * unit + 1 : unit + rot_units;
    } else {
        const int c = 2 * unit;
        if (c < chunks) ca = c;
        if (c + 1 < chunks) cb = c + 1;
    }
    float xa[HPG][V], xb[HPG][V];
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
        const int h = h0 + i;
        const char *src;
        if (h < a.Hq) src = a.q + n * a.q_t + h * a.q_h;
        else if (h < a.Hq + a.Hk) src = a.k + n * a.k_t + (h - a.Hq) * a.k_h;
        else src = a.v + n * a.v_t + (min(h, a.H - 1) - a.Hq - a.Hk) * a.v_h;
#pragma unroll
        for (int j = 0; j < V; ++j) xa[i][j] = xb[i][j] = 0.0f;
        if (h < a.H) {
            if (ca >= 0) load<IBF, V>(src + ca * V * IS, xa[i]);
            if (cb >= 0) load<IBF, V>(src + cb * V * IS, xb[i]);
        }
    }
    // Angles in turns, in 64 bits: a far position times a frequency has more whole turns than float32 has digits for.
    float cs[V], sn[V];
    const bool rotate = unit < rot_units && h0 < a.Hq + a.Hk;
    if (rotate) {
        const double pos = static_cast<double>(a.pos[n]) * 0.15915494309189535;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const double t = pos * static_cast<double>(a.inv_freq[unit * V + j]);
            sincospif(2.0f * static_cast<float>(t - rint(t)), &sn[j], &cs[j]);
        }
    }
    const int row = a.slot ? a.slot[n] : n;
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
        const int h = h0 + i;
        if (h >= a.H) break;
        const bool is_v = h >= a.Hq + a.Hk;
        const float *gain = h < a.Hq ? a.gain_q : a.gain_k;
        if (!is_v && gain) {
            float ss = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) ss = fmaf(xa[i][j], xa[i][j], fmaf(xb[i][j], xb[i][j], ss));
            for (int o = 1 << a.lane_bits >> 1; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
            const float rn = rm_rnorm_from_ssq(ss, a.D, a.eps);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (ca >= 0) xa[i][j] *= rn * gain[ca * V + j];
                if (cb >= 0) xb[i][j] *= rn * gain[cb * V + j];
            }
        }
        if (!is_v && rotate) {
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
        char *dst;
        if (h < a.Hq) {
            dst = a.q_out + n * a.qo_t + h * a.qo_h;
        } else {
            if (row < 0 || row >= a.rows) continue;
            dst = is_v ? a.v_out + row * a.vo_t + (h - a.Hq - a.Hk) * a.vo_h : a.k_out + row * a.ko_t + (h - a.Hq) * a.ko_h;
        }
        if (ca >= 0) store<OBF, V>(dst + ca * V * OS, xa[i]);
        if (cb >= 0) store<OBF, V>(dst + cb * V * OS, xb[i]);
    }
}

template <bool IBF, bool OBF, int V>
hipError_t go(RopeArgs a, hipStream_t st) {
    const int units = a.rot / (2 * V) + (a.D / V - a.rot / V + 1) / 2;
    a.lane_bits = 0;
    while ((1 << a.lane_bits) < units) ++a.lane_bits;
    // Four heads a lane group once that still gives every compute unit several workgroups.
    const int per_wg = 256 >> a.lane_bits;
    const bool many = static_cast<int64_t>(a.N) * a.H >= static_cast<int64_t>(4) * 1024 * per_wg;
    a.groups = many ? (a.H + 3) / 4 : a.H;
    const int64_t wgs = (static_cast<int64_t>(a.N) * a.groups + per_wg - 1) / per_wg;
    if (many) qk_norm_rope_kernel<IBF, OBF, V, 4><<<dim3(static_cast<unsigned>(wgs)), 256, 0, st>>>(a);
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
