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

// rm_dma::dma16 for two loads, STEP bytes apart in LDS, each lane at its 32-bit offset from a base in scalar registers.
template <int STEP>
__device__ __forceinline__ void dma16_pair(const void *base, uint32_t off0, uint32_t off1, uint32_t lds) {
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
        "s_add_u32 m0, m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(off0), "v"(off1), "s"(base), "s"(lds), "n"(STEP)
        : "memory", "scc");
}

// A value that is the same in every lane, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32));
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}
__device__ __forceinline__ const char *uniform(const char *p) {
    return reinterpret_cast<const char *>(uniform(reinterpret_cast<int64_t>(p)));
}

__device__ __forceinline__ float xor32_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }

// a * b rounded, not part of a fused multiply-add.
__device__ __forceinline__ float scaled(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

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

// Scheduling of a block of N steps of R LDS reads and M matrix-core instructions each: the reads run AHEAD steps ahead.
template <int N, int AHEAD, int M, int R>
__device__ __forceinline__ void pipeline() {
    constexpr int A = AHEAD < N ? AHEAD : N;
    __builtin_amdgcn_sched_group_barrier(0x100, A * R, 0);
#pragma unroll
    for (int i = 0; i < N - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, A * M, 0);
}

// One tile's place: keys [kb, min(kb + KT, end)) of segment seg (-1: the group's shared keys, else a sample).
struct Tile {
    const char *k, *v;
    int64_t kn, vn;  // bytes from key to key
    int kb, end, seg;
};

template <bool BF, int DH, int RW, int KW, int QB, int KT, int NBUF, int WPE>
__global__ __launch_bounds__(64 * RW * KW, WPE) void attn_kernel(Args a) {
    constexpr int W = RW * KW, ES = BF ? 2 : 4, ROWB = DH * ES, CPR = ROWB / 16;
    constexpr int RPI = 64 / CPR;             // tile rows per load instruction of a wave (1 KB)
    constexpr int KPW = KT / KW, NS = KPW / 32;  // keys of a tile that a wave takes
    constexpr int NI = KPW / RPI / RW;        // load instructions per wave and matrix
    constexpr int DB = DH / 32;               // output blocks of 32 columns
    constexpr int QF = BF ? DH / 16 : DH / 8; // fragments of a query row block
    constexpr int AHEAD = 4;                  // LDS reads run this many matrix-core steps ahead
    static_assert(CPR >= 8 && CPR <= 64 && NI >= 1 && NI * RPI * RW == KPW && NS * 32 == KPW, "tile shape");
    constexpr int TILEB = KPW * ROWB, KWB = 2 * NBUF * TILEB;  // one matrix's keys, and all buffers of a key wave
    // O of every wave passes through LDS when the key waves are joined.
    constexpr int JOINB = KW > 1 ? W * QB * 32 * DH * 4 + W * QB * 32 * 8 : 0;
    constexpr int LDSB = KW * KWB > JOINB ? KW * KWB : JOINB;
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
    auto seg_keys = [&](int sg, int &lo, int &end) __attribute__((always_inline)) {
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
    auto seg_base = [&](Tile &t) __attribute__((always_inline)) {
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
    const int64_t first = total * split / a.splits, n_tiles = total * (split + 1) / a.splits - first;
    auto first_tile = [&](Tile &t) __attribute__((always_inline)) {
        int64_t skip = first;
        t.seg = -1;
        t.kb = t.end = 0;
        for (int sg = -1; sg <= s_last; sg = sg < 0 ? s_first : sg + 1) {
            int lo, end;
            seg_keys(sg, lo, end);
            const int n = (end - lo + KT - 1) / KT;
            t.seg = sg;
            t.kb = lo + static_cast<int>(min(skip, static_cast<int64_t>(n))) * KT;
            t.end = end;
            if (skip < n) break;
            skip -= n;
        }
        seg_base(t);
    };
    Tile cur;
    first_tile(cur);
    auto advance = [&](Tile &t) __attribute__((always_inline)) {  // only called when another tile follows
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
    // A key wave's buffers: NBUF times its keys of a tile, then its values.  The RW waves that share them fill them.
    uint8_t *const lds_w = lds + kw * KWB;
    const uint32_t lds_at = rm_dma::lds_addr(lds_w);
    const bool whole_head = a.D == DH;
    // The swizzle of a wave's load instructions repeats every PER of them.
    constexpr int PERK = RW * RPI >= 16 ? 1 : 16 / (RW * RPI);
    constexpr int PERV = BF ? (RW * RPI >= 4 ? 1 : 4 / (RW * RPI)) : (RW * RPI >= 8 ? 1 : 8 / (RW * RPI));
    static_assert(NI % 2 == 0 && NI % PERK == 0 && NI % PERV == 0, "load instructions");
    auto stage = [&](const Tile &t, int buf, bool values) __attribute__((always_inline)) {
        const int64_t sn = uniform(values ? t.vn : t.kn);
        const char *base = uniform(values ? t.v : t.k) + kw * KPW * sn;
        const uint32_t to = lds_at + (buf * 2 + (values ? 1 : 0)) * TILEB + rw * 1024;
        const int left = t.end - t.kb - kw * KPW;  // keys from the wave's first to the end
        if (whole_head && left >= KPW) {
            // Row (n RW + rw) RPI + lrow: token strides are below 2^24 bytes, so a tile's offsets fit in 32 bits.
            const uint32_t row0 = (rw * RPI + lrow) * static_cast<uint32_t>(sn);
            const uint32_t step = RW * RPI * static_cast<uint32_t>(sn);
            uint32_t chunk[PERK > PERV ? PERK : PERV];
#pragma unroll
            for (int n = 0; n < (values ? PERV : PERK); ++n) {
                const int row = (n * RW + rw) * RPI + lrow;
                chunk[n] = row0 + (pos ^ (values ? swz_v(row) : swz_k(row))) * 16;
            }
#pragma unroll
            for (int n = 0; n < NI; n += 2)
                dma16_pair<RW * 1024>(base, chunk[n % (values ? PERV : PERK)] + n * step,
                                      chunk[(n + 1) % (values ? PERV : PERK)] + (n + 1) * step,
                                      __builtin_amdgcn_readfirstlane(to + n * RW * 1024));
        } else {  // rows past the end and columns past the head's are zeros
            const int64_t zero = reinterpret_cast<int64_t>(&zero16);
            const char *at = base + (rw * RPI + lrow) * sn;
#pragma unroll 2
            for (int n = 0; n < NI; ++n, at += RW * RPI * sn) {
                const int row = (n * RW + rw) * RPI + lrow;
                const int chunk = pos ^ (values ? swz_v(row) : swz_k(row));
                // 0 or -1, without a branch
                const int64_t in = static_cast<int64_t>((row - left) & (chunk * 16 - a.D * ES)) >> 63;
                const int64_t src = zero + ((reinterpret_cast<int64_t>(at) + chunk * 16 - zero) & in);
                rm_dma::dma16(reinterpret_cast<const char *>(src), __builtin_amdgcn_readfirstlane(to + n * RW * 1024));
            }
        }
    };
    // Waits until all but this wave's last `N` loads are there and its LDS reads are done; where several waves share
    // the buffers, until that holds for all of them.
    auto sync = [&](auto n) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        if constexpr (RW > 1) rm_dma::wait_barrier<N>();
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, NI> OneMatrix;
    typedef std::integral_constant<int, 63> Any;  // reads only

    // ---------------------------------------------------------------- queries
    typedef typename std::conditional<BF, rm_bf16x8, rm_f32x4>::type QFrag;
    QFrag qf[QB][QF];
    if (n_tiles > 0) {
        stage(cur, 0, false);
        stage(cur, 0, true);
    }
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
    const uint8_t *kb_ptr[8];  // keys: chunk 2 c + hi of row 32 ns + col, by c mod 8 (the rest are offsets)
    {
        const int row = col;
#pragma unroll
        for (int c = 0; c < 8; ++c) kb_ptr[c] = lds_w + row * ROWB + (((2 * c + hi) ^ swz_k(row)) & (CPR - 1)) * 16;
    }
    constexpr int VP = BF ? (DB < 4 ? DB : 4) : 2;
    const uint8_t *v_ptr[VP];
    if constexpr (BF) {
        const int i = (lane & 15) >> 2, row = 4 * hi + i;
        const int inner = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
        for (int d = 0; d < VP; ++d) v_ptr[d] = lds_w + TILEB + row * ROWB + ((d * 64) ^ (swz_v(i) * 16)) + inner;
    } else {
        const int row = 4 * hi;
#pragma unroll
        for (int d = 0; d < VP; ++d) v_ptr[d] = lds_w + TILEB + row * ROWB + ((d * 128) ^ (hi * 128)) + col * 4;
    }

    auto read_v = [](const uint8_t *p) { return read_v_rows<ROWB>(p); };
    rm_f32x16 o[QB][DB];
    float m[QB], l[QB];
    // Scores with a cap or a bias are formed in powers of two; plain ones are scaled on the way into exp2.
    const float sc = a.cap != 0.0f || a.slopes ? 1.0f : a.scale;

    // ---------------------------------------------------------------- tiles
    // One pass over the slice's tiles, the first one's keys under way.  Returns whether a tile of keys that some rows
    // see and others do not holds infinities or NaN among its values: 0 times those would spoil the rows that do not
    // see them.  Such a workgroup (there is hardly ever one) makes a second pass with `clean`, which sets them to 0 in
    // LDS, the other sums staying as they are bit for bit, and then adds them to the rows that see them.
    auto pass = [&](const bool clean) __attribute__((always_inline)) -> bool {
        uint32_t spoilt = 0;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            m[qb] = -INFINITY;
            l[qb] = 0.0f;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[qb][d] = rm_f32x16{};
        }
        int buf = 0;
        for (int64_t n_left = n_tiles; n_left > 0; --n_left) {
            Tile nxt = cur;
            if (n_left > 1) advance(nxt);
            const int at = NBUF == 2 ? buf * 2 * TILEB : 0;  // this tile's buffers
            if constexpr (NBUF == 2) {  // keys and values a tile ahead
                sync(None{});
                if (n_left > 1) {
                    stage(nxt, buf ^ 1, false);
                    stage(nxt, buf ^ 1, true);
                }
                buf ^= 1;
            } else {  // the tile's keys; its values are under way
                sync(OneMatrix{});
            }

            const int kbw = cur.kb + kw * KPW;
            bool active = kbw < cur.end, mixed = kbw + KPW > cur.end, apart = false;
            if (cur.seg >= 0) {
                active = active && cur.seg >= w_s0 && cur.seg <= w_s1 && kbw < w_maxhi && kbw + KPW > w_minlo;
                apart = w_s0 != w_s1 || kbw < w_maxlo || min(kbw + KPW, cur.end) > w_minhi;
                mixed = mixed || apart;
            }
            auto interval = [&](int qb, int &lo, int &len) {  // the keys of this segment that the lane's row sees
                lo = cur.seg < 0 ? 0 : r_lo[qb];
                len = cur.seg < 0 ? n0 : (r_sample[qb] == cur.seg ? r_len[qb] : 0);
            };
            rm_f32x16 s[QB][NS];
            if (active) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns) s[qb][ns] = rm_f32x16{};
                // Key fragments AHEAD ahead of the products that take them.
                QFrag kf[QF * NS];
                auto read_k = [&](int x) {  // x = c NS + ns
                    const int c = x / NS, ns = x % NS;
                    return *reinterpret_cast<const QFrag *>(kb_ptr[c & 7] + at + ns * 32 * ROWB + (c >> 3) * 256);
                };
#pragma unroll
                for (int x = 0; x < QF * NS; ++x) kf[x] = read_k(x);
#pragma unroll
                for (int x = 0; x < QF * NS; ++x)
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) {
                        if constexpr (BF) {
                            s[qb][x % NS] =
                                __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x], qf[qb][x / NS], s[qb][x % NS], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                s[qb][x % NS] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[x][i], qf[qb][x / NS][i],
                                                                                    s[qb][x % NS], 0, 0, 0);
                        }
                    }
                pipeline<QF * NS, AHEAD, BF ? QB : 4 * QB, 1>();
            }
            if constexpr (NBUF == 1) {  // every wave has read the keys: the next ones'
                sync(Any{});
                if (n_left > 1) stage(nxt, 0, false);
            }
            if (active) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    if (a.cap != 0.0f) {
#pragma unroll
                        for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float z = s[qb][ns][i] * a.scale;  // score / cap
                                float th;
                                if constexpr (BF)
                                    th = 1.0f - 2.0f * __builtin_amdgcn_rcpf(
                                                           __builtin_amdgcn_exp2f(z * (2.0f * kLog2e)) + 1.0f);
                                else
                                    th = tanhf(z);
                                s[qb][ns][i] = a.cap * th;
                            }
                    }
                    if (a.slopes) {
                        const float in = a.cap != 0.0f ? 1.0f : a.scale;
#pragma unroll
                        for (int ns = 0; ns < NS; ++ns) {
                            const int d0 = r_pos[qb] - (kbw + 32 * ns + 4 * hi);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                s[qb][ns][i] = s[qb][ns][i] * in -
                                               r_slope[qb] * fabsf(static_cast<float>(d0 - (8 * (i >> 2) + (i & 3))));
                        }
                    }
                    if (mixed) {
                        int lo, len;
                        interval(qb, lo, len);
#pragma unroll
                        for (int ns = 0; ns < NS; ++ns) {
                            const int d0 = kbw + 32 * ns + 4 * hi - lo;
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                s[qb][ns][i] =
                                    static_cast<uint32_t>(d0 + 8 * (i >> 2) + (i & 3)) < static_cast<uint32_t>(len)
                                        ? s[qb][ns][i]
                                        : -INFINITY;
                        }
                    }
                    float top = s[qb][0][0];
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[qb][ns][i]);
                    top = xor32_max(top) * sc;
                    // Raising the maximum of a row without sums so far (m = -inf) needs no rescaling.
                    const bool raise = top > m[qb] + kRaise;  // (false for top = -inf)
                    if (__any(raise)) {
                        const float mn = raise ? top : m[qb];
                        const bool any = __any(raise && m[qb] != -INFINITY);
                        const float f = raise ? __builtin_amdgcn_exp2f(m[qb] - mn) : 1.0f;
                        m[qb] = mn;
                        if (any) {
                            l[qb] *= f;
#pragma unroll
                            for (int d = 0; d < DB; ++d)
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[qb][d][i] *= f;
                        }
                    }
                    const float ref = m[qb] == -INFINITY ? 0.0f : m[qb];
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            // (float32 rounds the score first, as the maximum was: the largest weight is 1 exactly)
                            const float x = BF ? fmaf(s[qb][ns][i], sc, -ref) : scaled(s[qb][ns][i], sc) - ref;
                            s[qb][ns][i] = __builtin_amdgcn_exp2f(x);
                            sum[i & 3] += s[qb][ns][i];
                        }
                    l[qb] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                }
            }
            if constexpr (NBUF == 1) {  // the values
                if (n_left > 1) sync(OneMatrix{});
                else sync(None{});
            }
            if (clean && cur.seg >= 0) {
                for (int i = rw * 64 + lane; i < TILEB / 16; i += 64 * RW) {
                    rm_u32x4 *p = reinterpret_cast<rm_u32x4 *>(lds_w + TILEB + at) + i;
                    rm_u32x4 v = *p;
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (BF) {
                            const uint32_t bad = nonfinite_bf16x2(v[e]);
                            v[e] &= (bad & 0x8000u ? 0u : 0xffffu) | (bad >> 31 ? 0u : 0xffff0000u);
                        } else {
                            v[e] = nonfinite_f32(__uint_as_float(v[e])) ? 0u : v[e];
                        }
                    }
                    *p = v;
                }
                sync(Any{});
            }
            if (active) {
                if (apart && !clean) {
#pragma unroll 1
                    for (int r = 0; r < KPW; r += BF ? 8 : 1) {  // the wave's values, each lane some of them
                        if (!BF && (r & 4)) continue;            // (float32: rows r and r + 4 in the two halves)
#pragma unroll
                        for (int d = 0; d < DB; ++d) {
                            const uint8_t *vp = v_ptr[d % VP] + at + (d / VP) * 256 + r * ROWB;
                            if constexpr (BF) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(vp);
                                spoilt |= nonfinite_bf16x2(v.x) | nonfinite_bf16x2(v.y);
                            } else {
                                spoilt |= nonfinite_f32(*reinterpret_cast<const float *>(vp));
                            }
                        }
                    }
                }
                if constexpr (BF) {
                    rm_bf16x8 p[QB][2 * NS];
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                        for (int st = 0; st < 2 * NS; ++st)
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                p[qb][st][i] = static_cast<__bf16>(s[qb][st / 2][8 * (st % 2) + i]);
#pragma unroll
                    for (int x = 0; x < 2 * NS * DB; ++x) {
                        const int st = x / DB, d = x % DB;
                        const rm_bf16x8 vf = read_v(v_ptr[d % VP] + at + (d / VP) * 256 + 16 * st * ROWB);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb)
                            o[qb][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[qb][st], o[qb][d], 0, 0, 0);
                    }
                    pipeline<2 * NS * DB, AHEAD, QB, 2>();
                } else {
#pragma unroll
                    for (int x = 0; x < 16 * NS * DB; ++x) {
                        const int ns = x / (16 * DB), i = x / DB % 16, d = x % DB;
                        const float vf = *reinterpret_cast<const float *>(
                            v_ptr[d % VP] + at + (d / VP) * 256 + (32 * ns + 8 * (i >> 2) + (i & 3)) * ROWB);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb)
                            o[qb][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[qb][ns][i], o[qb][d], 0, 0, 0);
                    }
                    pipeline<16 * NS * DB, AHEAD, QB, 1>();
                }
            }
            if constexpr (NBUF == 1) {  // every wave has read the values: the next ones'
                sync(Any{});
                if (n_left > 1) stage(nxt, 0, true);
            }
            cur = nxt;
        }
        return spoilt != 0;
    };
    bool clean = false;
    while (__builtin_amdgcn_readfirstlane(__syncthreads_or(pass(clean)))) {  // a pass with `clean` returns false
        clean = true;
        first_tile(cur);
        stage(cur, 0, false);
        stage(cur, 0, true);
    }
    if (__builtin_expect(clean, false)) {  // the infinities and NaN that the second pass left out
        first_tile(cur);
        for (int64_t n_left = n_tiles; n_left > 0; --n_left) {
            const int k0 = cur.kb + kw * KPW, k1 = min(k0 + KPW, cur.end);
            for (int k = k0; cur.seg >= 0 && k < k1; ++k) {
                const char *row = cur.v + (k - cur.kb) * cur.vn;
                for (int c0 = 0; c0 < a.D; c0 += 64) {
                    float x = 0.0f;
                    if (c0 + lane < a.D) {
                        if constexpr (BF) x = rm_bf16_bits_to_f32(reinterpret_cast<const uint16_t *>(row)[c0 + lane]);
                        else x = reinterpret_cast<const float *>(row)[c0 + lane];
                    }
                    for (uint64_t bad = __ballot(!(fabsf(x) < INFINITY)); bad != 0; bad &= bad - 1) {
                        const int from = __ffsll(static_cast<unsigned long long>(bad)) - 1;
                        const float add = __shfl(x, from);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) {
                            const bool sees = r_sample[qb] == cur.seg &&
                                              static_cast<uint32_t>(k - r_lo[qb]) < static_cast<uint32_t>(r_len[qb]);
                            const int at = sees ? c0 + from - 4 * hi : -1;
#pragma unroll
                            for (int d = 0; d < DB; ++d)
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    o[qb][d][i] += at == 32 * d + 8 * (i >> 2) + (i & 3) ? add : 0.0f;
                        }
                    }
                }
            }
            if (n_left > 1) advance(cur);
        }
    }

    // ---------------------------------------------------------------- join and write
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l[qb] += __shfl_xor(l[qb], 32);
    float *join = reinterpret_cast<float *>(lds);
    if constexpr (KW > 1) {
        float *ml = join + W * QB * 32 * DH;  // [wave][qb][2][32]
        rm_dma::wait_barrier<0>();            // every wave has read the last tile (of a second pass)
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
