// The attention kernel shared by rm_span_attention and rm_prefix_attention (bf16 in attn_bf16.hip, float32 in
// attn_f32.hip): one pass over the keys with a running maximum and sum per query row.
//
// A workgroup takes 32 RW QB query rows (the tokens of one group times the query heads of one key head, so that a
// key head's rows are read once for all its query heads) and walks tiles of KT keys that its waves stage in LDS
// together, keys and values each in one buffer: while the scores of a tile are formed its values arrive, and while
// they are summed the next tile's keys.  RW of the waves divide the rows and KW the keys of a tile; the KW partial
// results are joined in LDS at the end.  With `splits` > 1 several workgroups divide a row block's tiles and leave
// partial results in the workspace for the combine kernel.
//
// Matrix-core layout (32x32 tiles): S^T = K Q^T, so a lane holds scores of one query row (column lane % 32) and
// row statistics, spans and slopes are one register per lane; O^T = V^T P^T takes P straight from the score
// registers: the 16 keys of a matrix-core step may come in any order as long as V's rows come in the same, and the
// order the scores have (keys 16 s + 4 h + {0..3} and + 8 for lane half h) is the one V's fragments are read in.
#pragma once

#include "rm_attn_plan.h"
#include "rm_dma.h"

typedef float rm_f32x16 __attribute__((ext_vector_type(16)));
typedef float rm_f32x8 __attribute__((ext_vector_type(8)));
typedef short rm_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 rm_bf16x4 __attribute__((ext_vector_type(4)));

namespace rm_attn {

constexpr float kLog2e = 1.4426950408889634f;
// A row's running maximum is raised only when a tile's scores pass it by more than this (in powers of two): the
// sums then stay below 2^8 times their final size, which float32 and bf16 hold at the same relative precision, and
// most tiles need no rescaling of the output registers.
constexpr float kRaise = 8.0f;

static __device__ uint4 zero16;  // what rows and columns outside a tile are staged from

// rm_dma::dma16 with a 64-bit base in scalar registers and a 32-bit byte offset per lane.
__device__ __forceinline__ void dma16_base(const void *base, uint32_t off, uint32_t lds) {
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(off), "s"(base), "s"(lds)
        : "memory");
}

__device__ __forceinline__ float xor32_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }

__device__ __forceinline__ int wave_min(int v) {
    for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v) {
    for (int o = 32; o >= 1; o >>= 1) v = max(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}

// Whether any of the values packed in v is infinite or NaN (all exponent bits set): the carry out of the exponent
// field reaches the sign bit.
__device__ __forceinline__ uint32_t nonfinite_bf16x2(uint32_t v) { return ((v & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t nonfinite_f32(float v) {
    return ((__float_as_uint(v) & 0x7f800000u) + 0x00800000u) & 0x80000000u;
}

// A fragment of V^T (32 columns x 16 keys) from rows of V in LDS: two transposing reads of 4 keys x 16 columns per 16
// lanes, 8 rows apart.
template <int ROWB>
__device__ __forceinline__ rm_bf16x8 read_v_rows(const uint8_t *p) {
    typedef __attribute__((address_space(3))) rm_s16x4 lds_s16x4;
    struct Pair {
        rm_s16x4 a, b;
    };
    const Pair v = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p)),
                    __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 8 * ROWB))};
    return __builtin_bit_cast(rm_bf16x8, v);
}

// One tile's place: keys [kb, min(kb + KT, end)) of segment seg (-1: the group's shared keys, else a sample).
struct Tile {
    const char *k, *v;
    int64_t kn, vn;  // bytes from key to key
    int kb, end, seg;
};

template <bool BF, int DH, int RW, int KW, int QB, int KT, int WPE>
__global__ __launch_bounds__(64 * RW * KW, WPE) void attn_kernel(Args a) {
    constexpr int W = RW * KW, ES = BF ? 2 : 4, ROWB = DH * ES, CPR = ROWB / 16;
    constexpr int RPI = 64 / CPR;             // tile rows per load instruction of a wave (1 KB)
    constexpr int NI = KT / RPI / W;          // load instructions per wave and matrix
    constexpr int KPW = KT / KW, NS = KPW / 32;
    constexpr int DB = DH / 32;               // output blocks of 32 columns
    constexpr int QF = BF ? DH / 16 : DH / 8; // fragments of a query row block
    static_assert(CPR >= 8 && CPR <= 64 && NI >= 1 && NI * RPI * W == KT && NS >= 1, "tile shape");
    constexpr int TILEB = KT * ROWB;
    // O of every wave passes through LDS when the key waves are joined.
    constexpr int JOINB = KW > 1 ? W * QB * 32 * DH * 4 + W * QB * 32 * 8 : 0;
    constexpr int LDSB = 2 * TILEB > JOINB ? 2 * TILEB : JOINB;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[LDSB];

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kw = wave / RW;

    // This workgroup's key head of a group, row block and slice of the keys.
    int ng, tile_id;
    {
        const int nt = a.n_tiles * a.splits, id = blockIdx.x;
        if (((a.U * a.Hk) & 7) == 0) {  // whole groups to an XCD, whose L2 then holds their keys
            const int i = id >> 3;
            ng = (id & 7) + 8 * (i / nt);
            tile_id = i % nt;
        } else {
            ng = id / nt;
            tile_id = id % nt;
        }
    }
    const int split = tile_id % a.splits;
    // Row blocks from the last to the first: with causal masks the later ones see more keys and start first.
    const int row0 = (a.n_tiles - 1 - tile_id / a.splits) * (32 * RW * QB);
    const int u = ng / a.Hk, hk = ng % a.Hk;
    const int rows_end = min(row0 + 32 * RW * QB, a.R);

    // ---------------------------------------------------------------- rows
    const int n0 = a.n0 == 0 ? 0 : (a.len0 ? min(max(a.len0[u], 0), a.n0) : a.n0);
    int r_sample[QB], r_lo[QB], r_len[QB];
    float r_slope[QB];
    int r_pos[QB];
    int w_maxlo = 0, w_minhi = 0x7fffffff, w_minlo = 0x7fffffff, w_maxhi = 0, w_s0 = 0x7fffffff, w_s1 = -1;
    const char *qrow[QB];
    char *orow[QB];
    bool r_ok[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = row0 + (rw * QB + qb) * 32 + col;
        r_ok[qb] = r < a.R;
        const int rc = min(r, a.R - 1);
        const int tok = rc / a.G, g = rc - tok * a.G;
        const int smp = tok / a.T, t = tok - smp * a.T;
        const int64_t b = static_cast<int64_t>(u) * a.per + smp;
        const int h = hk * a.G + g;
        qrow[qb] = a.q + b * a.q_b + t * a.q_t + h * a.q_h;
        orow[qb] = a.o + b * a.o_b + t * a.o_t + h * a.o_h;
        int lo = 0, end = a.n1;
        if (a.span) {
            const int2 sp = *reinterpret_cast<const int2 *>(a.span + 2 * (b * a.T + t));
            lo = min(max(sp.x, 0), a.n1);
            end = min(max(sp.y, 0), a.n1);
        } else if (a.n1 > 0) {
            if (a.len1) end = min(max(a.len1[b], 0), a.n1);
            if (a.causal) end = min(max(end - a.T + t + 1, 0), end);
        }
        r_sample[qb] = smp;
        r_lo[qb] = lo;
        r_len[qb] = max(end - lo, 0);
        r_slope[qb] = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
        r_pos[qb] = (a.slopes && a.q_start ? a.q_start[b] : 0) + t;
        if (r_ok[qb]) {
            if (r_len[qb] > 0) {
                w_maxlo = max(w_maxlo, lo);
                w_minhi = min(w_minhi, end);
                w_minlo = min(w_minlo, lo);
                w_maxhi = max(w_maxhi, end);
            } else {
                w_maxlo = 0x7fffffff;  // no tile is whole for a row that sees nothing
            }
            w_s0 = min(w_s0, smp);
            w_s1 = max(w_s1, smp);
        }
    }
    w_maxlo = wave_max(w_maxlo);
    w_minhi = wave_min(w_minhi);
    w_minlo = wave_min(w_minlo);
    w_maxhi = wave_max(w_maxhi);
    w_s0 = wave_min(w_s0);
    w_s1 = wave_max(w_s1);

    // ---------------------------------------------------------------- segments of keys
    const int s_first = row0 / a.G / a.T, s_last = (rows_end - 1) / a.G / a.T;
    int b_lo = 0, b_hi = 0;  // with spans: the keys that any of the workgroup's rows sees
    if (a.span) {
        int lo = 0x7fffffff, end = 0;
        const int t0 = row0 / a.G, t1 = (rows_end - 1) / a.G;
        for (int t = t0 + lane; t <= t1; t += 64) {
            const int2 sp = *reinterpret_cast<const int2 *>(a.span + 2 * (static_cast<int64_t>(u) * a.T + t));
            const int x = min(max(sp.x, 0), a.n1), y = min(max(sp.y, 0), a.n1);
            if (x < y) {
                lo = min(lo, x);
                end = max(end, y);
            }
        }
        b_lo = wave_min(lo);
        b_hi = wave_max(end);
        if (b_lo > b_hi) b_lo = b_hi;
    }
    auto seg_keys = [&](int sg, int &lo, int &end) {
        lo = 0;
        if (sg < 0) {
            end = n0;
        } else if (a.span) {
            lo = b_lo;
            end = b_hi;
        } else {
            end = a.n1;
            if (a.n1 > 0 && a.len1)
                end = __builtin_amdgcn_readfirstlane(min(max(a.len1[static_cast<int64_t>(u) * a.per + sg], 0), a.n1));
        }
    };
    auto seg_base = [&](Tile &t) {
        const Src &s = t.seg < 0 ? a.s0 : a.s1;
        const int64_t b = t.seg < 0 ? u : static_cast<int64_t>(u) * a.per + t.seg;
        t.kn = s.k_n;
        t.vn = s.v_n;
        t.k = s.k + b * s.k_b + hk * s.k_h + t.kb * s.k_n;
        t.v = s.v + b * s.v_b + hk * s.v_h + t.kb * s.v_n;
    };
    int64_t total = 0;
    for (int sg = -1; sg <= s_last; sg = sg < 0 ? s_first : sg + 1) {
        int lo, end;
        seg_keys(sg, lo, end);
        total += (end - lo + KT - 1) / KT;
    }
    int64_t n_left;  // tiles of this slice
    Tile cur;
    {
        const int64_t first = total * split / a.splits;
        n_left = total * (split + 1) / a.splits - first;
        int64_t skip = first;
        cur.seg = -1;
        cur.kb = cur.end = 0;
        for (int sg = -1; sg <= s_last; sg = sg < 0 ? s_first : sg + 1) {
            int lo, end;
            seg_keys(sg, lo, end);
            const int n = (end - lo + KT - 1) / KT;
            cur.seg = sg;
            cur.kb = lo + static_cast<int>(min(skip, static_cast<int64_t>(n))) * KT;
            cur.end = end;
            if (skip < n) break;
            skip -= n;
        }
        seg_base(cur);
    }
    auto advance = [&](Tile &t) {  // only called when another tile follows
        t.kb += KT;
        if (t.kb < t.end) {
            t.k += KT * t.kn;
            t.v += KT * t.vn;
            return;
        }
        do {
            t.seg = t.seg < 0 ? s_first : t.seg + 1;
            seg_keys(t.seg, t.kb, t.end);
        } while (t.kb >= t.end);
        seg_base(t);
    };

    // ---------------------------------------------------------------- staging
    const int lrow = lane / CPR, pos = lane % CPR;
    auto swz_k = [](int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; };
    auto swz_v = [](int row) {
        if constexpr (BF)
            return CPR == 8 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
        else
            return 8 * ((row >> 2) & 1);
    };
    const uint32_t lds_k = rm_dma::lds_addr(lds), lds_v = lds_k + TILEB;
    const bool whole_head = a.D == DH;
    auto stage = [&](const Tile &t, bool values) {
        const char *base = values ? t.v : t.k;
        const int64_t sn = values ? t.vn : t.kn;
        const uint32_t to = (values ? lds_v : lds_k) + wave * 1024;
        if (whole_head && t.kb + KT <= t.end) {
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int row = (n * W + wave) * RPI;
                const int chunk = pos ^ (values ? swz_v(row + lrow) : swz_k(row + lrow));
                const uint32_t off = static_cast<uint32_t>(lrow) * static_cast<uint32_t>(sn) + chunk * 16;
                dma16_base(base + row * sn, off, to + n * W * 1024);
            }
        } else {  // rows past the end and columns past the head's are zeros
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int row = (n * W + wave) * RPI + lrow;
                const int chunk = pos ^ (values ? swz_v(row) : swz_k(row));
                const bool in = t.kb + row < t.end && chunk * 16 < a.D * ES;
                const char *src = in ? base + row * sn + chunk * 16 : reinterpret_cast<const char *>(&zero16);
                rm_dma::dma16(src, to + n * W * 1024);
            }
        }
    };

    // ---------------------------------------------------------------- queries
    typedef typename std::conditional<BF, rm_bf16x8, rm_f32x4>::type QFrag;
    QFrag qf[QB][QF];
    if (n_left > 0) stage(cur, false);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int c = 0; c < QF; ++c) {
            const int byte = (2 * c + hi) * 16;
            rm_u32x4 v = {0, 0, 0, 0};
            if (byte < a.D * ES) v = *reinterpret_cast<const rm_u32x4 *>(qrow[qb] + byte);
            qf[qb][c] = __builtin_bit_cast(QFrag, v);
        }

    // ---------------------------------------------------------------- fragment addresses (bytes in LDS)
    const uint8_t *kb_ptr[8];  // keys: chunk 2 c + hi of row kw KPW + 32 ns + col, by c mod 8 (the rest are offsets)
    {
        const int row = kw * KPW + col;
#pragma unroll
        for (int c = 0; c < 8; ++c) kb_ptr[c] = lds + row * ROWB + (((2 * c + hi) ^ swz_k(row)) & (CPR - 1)) * 16;
    }
    constexpr int VP = BF ? (DB < 4 ? DB : 4) : 2;
    const uint8_t *v_ptr[VP];
    if constexpr (BF) {
        const int i = (lane & 15) >> 2, row = kw * KPW + 4 * hi + i;
        const int inner = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
        for (int d = 0; d < VP; ++d) v_ptr[d] = lds + TILEB + row * ROWB + ((d * 64) ^ (swz_v(i) * 16)) + inner;
    } else {
        const int row = kw * KPW + 4 * hi;
#pragma unroll
        for (int d = 0; d < VP; ++d) v_ptr[d] = lds + TILEB + row * ROWB + ((d * 128) ^ (hi * 128)) + col * 4;
    }

    auto read_v = [](const uint8_t *p) { return read_v_rows<ROWB>(p); };
    rm_f32x16 o[QB][DB];
    float m[QB], l[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[qb][d] = rm_f32x16{};
    }

    // ---------------------------------------------------------------- tiles
    for (; n_left > 0; --n_left) {
        Tile nxt = cur;
        if (n_left > 1) advance(nxt);
        rm_dma::wait_barrier<0>();  // the keys are there, and every wave has read the last tile's values
        stage(cur, true);

        const int kbw = cur.kb + kw * KPW;
        bool active = kbw < cur.end, mixed = kbw + KPW > cur.end;
        if (cur.seg >= 0) {
            active = active && cur.seg >= w_s0 && cur.seg <= w_s1 && kbw < w_maxhi && kbw + KPW > w_minlo;
            mixed = mixed || w_s0 != w_s1 || kbw < w_maxlo || kbw + KPW > w_minhi;
        }
        rm_f32x16 s[QB][NS];
        if (active) {
#pragma unroll
            for (int ns = 0; ns < NS; ++ns) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) s[qb][ns] = rm_f32x16{};
#pragma unroll
                for (int c = 0; c < QF; ++c) {
                    const uint8_t *p = kb_ptr[c & 7] + ns * 32 * ROWB + (c >> 3) * 256;
                    const QFrag kf = *reinterpret_cast<const QFrag *>(p);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) {
                        if constexpr (BF) {
                            s[qb][ns] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[qb][c], s[qb][ns], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                s[qb][ns] =
                                    __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], qf[qb][c][i], s[qb][ns], 0, 0, 0);
                        }
                    }
                }
            }
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                int lo = r_lo[qb], len = r_len[qb];
                if (cur.seg < 0) {
                    lo = 0;
                    len = n0;
                } else if (r_sample[qb] != cur.seg) {
                    len = 0;
                }
                float top = -INFINITY;
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) {
                    const int k0 = kbw + 32 * ns + 4 * hi;
                    rm_f32x16 &x = s[qb][ns];
                    if (a.cap != 0.0f) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float z = x[i] * a.scale;  // score / cap
                            float th;
                            if constexpr (BF)
                                th = 1.0f - 2.0f * __builtin_amdgcn_rcpf(
                                                       __builtin_amdgcn_exp2f(z * (2.0f * kLog2e)) + 1.0f);
                            else
                                th = tanhf(z);
                            x[i] = a.cap * th;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] *= a.scale;
                    }
                    if (a.slopes) {
                        const int d0 = r_pos[qb] - k0;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            x[i] -= r_slope[qb] * fabsf(static_cast<float>(d0 - (8 * (i >> 2) + (i & 3))));
                    }
                    if (mixed) {
                        const int d0 = k0 - lo;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            x[i] = static_cast<uint32_t>(d0 + 8 * (i >> 2) + (i & 3)) < static_cast<uint32_t>(len)
                                       ? x[i]
                                       : -INFINITY;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
                }
                top = xor32_max(top);
                if (__any(top > m[qb] + kRaise || (m[qb] == -INFINITY && top > -INFINITY))) {
                    const float mn = fmaxf(m[qb], top);
                    const float f = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[qb] - mn);
                    m[qb] = mn;
                    l[qb] *= f;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[qb][d][i] *= f;
                }
                const float ref = m[qb] == -INFINITY ? 0.0f : m[qb];
                float sum = 0.0f;
#pragma unroll
                for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[qb][ns][i] = __builtin_amdgcn_exp2f(s[qb][ns][i] - ref);
                        sum += s[qb][ns][i];
                    }
                l[qb] += sum;
            }
        }
        rm_dma::wait_barrier<0>();  // the values are there, and every wave has read the keys
        if (n_left > 1) stage(nxt, false);
        if (active) {
            // A key that some rows see and others do not may hold infinities or NaN: 0 times those would spoil the
            // rows that do not see it.  The rare tile that has both goes the long way.
            bool bad = false;
            if (mixed) {
                uint32_t any = 0;
                if constexpr (BF) {
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(v_ptr[d % VP] + (d / VP) * 256 +
                                                                                 (32 * ns + 8 * j) * ROWB);
                                any |= nonfinite_bf16x2(v.x) | nonfinite_bf16x2(v.y);
                            }
                } else {
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
#pragma unroll
                            for (int d = 0; d < DB; ++d)
                                any |= nonfinite_f32(*reinterpret_cast<const float *>(
                                    v_ptr[d % VP] + (d / VP) * 256 + (32 * ns + 8 * (i >> 2) + (i & 3)) * ROWB));
                }
                bad = __any(any != 0);
            }
            // o += V^T P^T; CLEAN leaves out V's infinities and NaN.
            auto add_values = [&](auto clean) {
                constexpr bool CLEAN = decltype(clean)::value;
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) {
                    if constexpr (BF) {
#pragma unroll
                        for (int st = 0; st < 2; ++st) {
                            rm_bf16x8 p[QB];
#pragma unroll
                            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                                for (int i = 0; i < 8; ++i) p[qb][i] = static_cast<__bf16>(s[qb][ns][8 * st + i]);
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                rm_bf16x8 vf = read_v(v_ptr[d % VP] + (d / VP) * 256 + (32 * ns + 16 * st) * ROWB);
                                if constexpr (CLEAN) {
#pragma unroll
                                    for (int i = 0; i < 8; ++i)
                                        vf[i] = fabsf(static_cast<float>(vf[i])) < INFINITY ? vf[i]
                                                                                          : static_cast<__bf16>(0.0f);
                                }
#pragma unroll
                                for (int qb = 0; qb < QB; ++qb)
                                    o[qb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[qb], o[qb][d], 0, 0, 0);
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                float vf = *reinterpret_cast<const float *>(
                                    v_ptr[d % VP] + (d / VP) * 256 + (32 * ns + 8 * (i >> 2) + (i & 3)) * ROWB);
                                if constexpr (CLEAN) vf = fabsf(vf) < INFINITY ? vf : 0.0f;
#pragma unroll
                                for (int qb = 0; qb < QB; ++qb)
                                    o[qb][d] =
                                        __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[qb][ns][i], o[qb][d], 0, 0, 0);
                            }
                    }
                }
            };
            if (!bad) {
                add_values(std::false_type{});
            } else {
                add_values(std::true_type{});
                // For each row and column, whether a key that the row sees holds +inf (or NaN), and -inf (or NaN):
                // products of the 0/1 matrices of both, then the sums that the definition has.
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    const int lo = cur.seg < 0 ? 0 : r_lo[qb];
                    const int len = cur.seg < 0 ? n0 : (r_sample[qb] == cur.seg ? r_len[qb] : 0);
                    auto sees = [&](int ns, int i) {
                        const int k = kbw + 32 * ns + 4 * hi + 8 * (i >> 2) + (i & 3);
                        return static_cast<uint32_t>(k - lo) < static_cast<uint32_t>(len) ? 1.0f : 0.0f;
                    };
                    auto plus = [](float x) { return !(fabsf(x) < INFINITY) && !(x < 0.0f) ? 1.0f : 0.0f; };
                    auto minus = [](float x) { return !(fabsf(x) < INFINITY) && !(x > 0.0f) ? 1.0f : 0.0f; };
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        rm_f32x16 np{}, nn{};
#pragma unroll 1
                        for (int ns = 0; ns < NS; ++ns) {
                            const uint8_t *vp = v_ptr[d % VP] + (d / VP) * 256 + 32 * ns * ROWB;
                            if constexpr (BF) {
#pragma unroll
                                for (int st = 0; st < 2; ++st) {
                                    const rm_bf16x8 vf = read_v(vp + 16 * st * ROWB);
                                    rm_bf16x8 vis, fp, fn;
#pragma unroll
                                    for (int i = 0; i < 8; ++i) {
                                        vis[i] = static_cast<__bf16>(sees(ns, 8 * st + i));
                                        fp[i] = static_cast<__bf16>(plus(static_cast<float>(vf[i])));
                                        fn[i] = static_cast<__bf16>(minus(static_cast<float>(vf[i])));
                                    }
                                    np = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp, vis, np, 0, 0, 0);
                                    nn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fn, vis, nn, 0, 0, 0);
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const float vf =
                                        *reinterpret_cast<const float *>(vp + (8 * (i >> 2) + (i & 3)) * ROWB);
                                    const float vis = sees(ns, i);
                                    np = __builtin_amdgcn_mfma_f32_32x32x2f32(plus(vf), vis, np, 0, 0, 0);
                                    nn = __builtin_amdgcn_mfma_f32_32x32x2f32(minus(vf), vis, nn, 0, 0, 0);
                                }
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            o[qb][d][i] += np[i] > 0.0f ? INFINITY : 0.0f;
                            o[qb][d][i] += nn[i] > 0.0f ? -INFINITY : 0.0f;
                        }
                    }
                }
            }
        }
        cur = nxt;
    }

    // ---------------------------------------------------------------- join and write
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l[qb] += __shfl_xor(l[qb], 32);
    float *join = reinterpret_cast<float *>(lds);
    if constexpr (KW > 1) {
        float *ml = join + W * QB * 32 * DH;  // [wave][qb][2][32]
        rm_dma::wait_barrier<0>();            // every wave has read the last tile
        if (hi == 0) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                ml[((wave * QB + qb) * 2 + 0) * 32 + col] = m[qb];
                ml[((wave * QB + qb) * 2 + 1) * 32 + col] = l[qb];
            }
        }
        __syncthreads();
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int k = 0; k < KW; ++k) top = fmaxf(top, ml[(((k * RW + rw) * QB + qb) * 2 + 0) * 32 + col]);
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < KW; ++k)
                sum += ml[(((k * RW + rw) * QB + qb) * 2 + 1) * 32 + col] *
                       __builtin_amdgcn_exp2f(ml[(((k * RW + rw) * QB + qb) * 2 + 0) * 32 + col] - ref);
            const float f = __builtin_amdgcn_exp2f(m[qb] - ref);
            m[qb] = top;
            l[qb] = sum;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const rm_f32x4 v = {o[qb][d][4 * i] * f, o[qb][d][4 * i + 1] * f, o[qb][d][4 * i + 2] * f,
                                        o[qb][d][4 * i + 3] * f};
                    *reinterpret_cast<rm_f32x4 *>(join + ((((wave * QB + qb) * DB + d) * 4 + i) * 64 + lane) * 4) = v;
                }
        }
        __syncthreads();
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = row0 + (rw * QB + qb) * 32 + col;
        const float inv = a.splits > 1 ? 1.0f : (l[qb] == 0.0f ? 0.0f : 1.0f / l[qb]);
        const int64_t prow = (static_cast<int64_t>(split) * a.U * a.Hk + ng) * a.R + r;
        if (a.splits > 1 && r_ok[qb] && hi == 0 && kw == 0) {
            a.part_ml[2 * prow] = m[qb];
            a.part_ml[2 * prow + 1] = l[qb];
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if (KW > 1 && d % KW != kw) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                rm_f32x4 v;
                if constexpr (KW > 1) {
                    v = rm_f32x4{};
#pragma unroll
                    for (int k = 0; k < KW; ++k)
                        v += *reinterpret_cast<const rm_f32x4 *>(
                            join + (((((k * RW + rw) * QB + qb) * DB + d) * 4 + i) * 64 + lane) * 4);
                } else {
                    v = rm_f32x4{o[qb][d][4 * i], o[qb][d][4 * i + 1], o[qb][d][4 * i + 2], o[qb][d][4 * i + 3]};
                }
                const int c = 32 * d + 8 * i + 4 * hi;
                if (!r_ok[qb] || c >= a.D) continue;
                if (a.splits > 1) {
                    *reinterpret_cast<rm_f32x4 *>(a.part_o + prow * a.D + c) = v;
                } else if constexpr (BF) {
                    rm_bf16x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = static_cast<__bf16>(v[e] * inv);
                    *reinterpret_cast<rm_bf16x4 *>(orow[qb] + c * 2) = w;
                } else {
                    *reinterpret_cast<rm_f32x4 *>(orow[qb] + c * 4) = v * inv;
                }
            }
        }
    }
}

}  // namespace rm_attn
