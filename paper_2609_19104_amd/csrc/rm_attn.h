// The attention kernel shared by rm_span_attention and rm_prefix_attention (bf16 in attn_bf16.hip and
// attn_bf16_cap.hip, float32 in attn_f32.hip): one pass over the keys with a running maximum and sum per query row.
//
// A workgroup takes 32 RW query rows (the tokens of one group times the query heads of one key head, so that a
// key head's rows are read once for all its query heads) and walks tiles of KT keys.  RW of its waves divide the rows
// and KW the keys of a tile; the waves that take the same keys load them straight into LDS buffers of their own, so
// with RW = 1 no wave waits for another before the KW partial results are joined in LDS at the end.  With
// `splits` > 1 several workgroups divide a row block's tiles and leave partial results for the combine kernel.
//
// Matrix-core layout (32x32 tiles): S^T = K Q^T, so a lane holds scores of one query row (column lane % 32) and
// row statistics, spans and slopes are one register per lane; O^T = V^T P^T takes P straight from the score
// registers: the 16 keys of a matrix-core step may come in any order as long as V's rows come in the same, and the
// order the scores have (keys 16 s + 4 h + {0..3} and + 8 for lane half h) is the one V's fragments are read in.
//
// What bounds it (bf16, MI355X): with RW = 4 the matrix cores and the exponentials, two workgroups to a compute unit,
// one in its softmax while the other multiplies: 8192 x 8192 rows and keys, 16 heads of 128 columns on 4: 572 us, 960
// TFLOP/s; of 64: 375 us, 730 (a score costs as many exponentials for half the products); 8 heads of 256 on 1: 558 us,
// 985 (a library product of 8192^3: 1222).  With KW = 4, where a compute unit has few rows, its load unit and LDS: 64
// bytes a cycle in and 128 out, which a tile of 128 keys and 256 columns keeps for 2048 of its 3800 cycles (1.6 us),
// and one wave to a SIMD, whose softmax (700 cycles) nothing else covers; a launch's own 6 us are its first trips to
// memory and the join.  The load instructions go out between the matrix-core steps, since a wave that issues several in
// a row waits for the load unit, 16 cycles an instruction and wave (a tile 4400 -> 3800 cycles).  Float32: the matrix
// cores' 153 TFLOP/s, of which 16 heads of 128 on 4096 rows reach 122.
#pragma once

#include "rm_attn_plan.h"
#include "rm_dma.h"

typedef float rm_f32x16 __attribute__((ext_vector_type(16)));
typedef short rm_s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 rm_bf16x4 __attribute__((ext_vector_type(4)));

namespace rm_attn {

constexpr float kLog2e = 1.4426950408889634f;
// A row's running maximum is raised only when a tile's scores pass it by more than this (in powers of two): the
// sums then stay below 2^8 times their final size, which float32 and bf16 hold at the same relative precision, and
// most tiles need no rescaling of the output registers.
constexpr float kRaise = 8.0f;

// A value that is the same in every lane, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32));
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}
__device__ __forceinline__ const char *uniform(const char *p) {
    return reinterpret_cast<const char *>(uniform(reinterpret_cast<int64_t>(p)));
}

// Two loads of 16 bytes per lane straight into LDS at lds + 16 lane and lds + STEP + 16 lane, each lane at its 32-bit
// offset from a base in scalar registers; only the lanes of mask take part.  M0 and EXEC are kept and put back.
// No memory clobber: the buffers are read between the waits below only, which have one.
template <int STEP>
__device__ __forceinline__ void dma16_pair(const void *base, uint32_t off0, uint32_t off1, uint32_t lds,
                                           uint64_t mask) {
    uint32_t keep;
    uint64_t exec;
    mask = uniform(static_cast<int64_t>(mask));
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_and_saveexec_b64 %1, %7\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\t"
        "s_mov_b64 exec, %1\n\ts_mov_b32 m0, %0"
        : "=&s"(keep), "=&s"(exec)
        : "v"(off0), "v"(off1), "s"(uniform(static_cast<const char *>(base))), "s"(lds), "n"(STEP), "s"(mask)
        : "scc");
}

// The other lane half's value joined with this one's.
__device__ __forceinline__ float xor32_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor32_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// tanh x to 16 roundings of its value, for every x: -1 / (1 + e^2x) is off by a last place of 1, which 1 + 2 times it
// keeps where tanh x is small, so there x (1 - x^2 / 3 + 2 x^4 / 15 - 17 x^6 / 315 + 62 x^8 / 2835) takes its place (the
// next term is 4 roundings at 0.35; with a correctly rounded power and reciprocal all of it is at most 7 for x from 1e-30
// to 12).
__device__ __forceinline__ float tanh_relative(float x) {
    const float e = __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(x * (2.0f * kLog2e)));
    const float z = x * x;
    const float p = fmaf(fmaf(fmaf(62.0f / 2835.0f, z, -17.0f / 315.0f), z, 2.0f / 15.0f), z, -1.0f / 3.0f);
    return fabsf(x) < 0.35f ? fmaf(x * z, p, x) : fmaf(2.0f, e, 1.0f);
}

// a * b rounded, not part of a fused multiply-add.
__device__ __forceinline__ float scaled(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// Maximum over the wave, in data-parallel steps along the rows of 16 lanes and then across them.
__device__ __forceinline__ int wave_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xa, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_min(int v) { return -wave_max(-v); }  // (no value here is INT_MIN)

// A value's bits in the passes over a block whose results are not finite: in kClean infinities and NaN are 0, in kPlus
// (kMinus) those that add +infinity (-infinity), an infinity of that sign or NaN, are 1 and all others 0.
enum : int { kFirst = 0, kClean = 1, kPlus = 2, kMinus = 3 };
template <bool BF>
__device__ __forceinline__ uint32_t marked(uint32_t v, int mode) {
    constexpr uint32_t EXP = BF ? 0x7f80u : 0x7f800000u, ONE = BF ? 0x3f80u : 0x3f800000u;
    constexpr uint32_t SIGN = BF ? 0x8000u : 0x80000000u;
    const bool bad = (v & EXP) == EXP, nan = (v & ~SIGN) > EXP;
    if (mode == kClean) return bad ? 0u : v;
    return bad && (nan || ((v & SIGN) != 0) == (mode == kMinus)) ? ONE : 0u;
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


__device__ __forceinline__ int divide(int n, Divisor d) {  // n < 2^30
    return d.mul == 0 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), d.mul) >> d.shift);
}

// One tile's place: keys [kb, min(kb + KT, end)) of segment seg (-1: the group's shared keys, else a sample).
struct Tile {
    const char *k, *v;
    int64_t kn, vn;  // bytes from key to key
    int kb, end, seg, before;
};

// Rows have room for DH columns in LDS; the products take DC of them.  PAD: the head has at most DC, more than LEAST.
// LOW: caps up to kLowCap (bf16).
template <bool BF, bool LOW, int DH, int DC, bool PAD, int RW, int KW, int KT, int NBUF, int WPE>
__global__ __launch_bounds__(64 * RW * KW, WPE) void attn_kernel(Args a) {
    constexpr int W = RW * KW, ES = BF ? 2 : 4, ROWB = DH * ES, CPR = ROWB / 16;
    constexpr int RPI = 64 / CPR;                // rows per load instruction of a wave (1 KB)
    constexpr int KPW = KT / KW, NS = KPW / 32;  // keys of a tile that a wave takes
    constexpr int NP = KPW / RPI / RW / 2;       // pairs of load instructions per wave and matrix
    constexpr int STEP = RW * RPI;               // rows from one of a wave's load instructions to the next
    constexpr int DB = DC / 32;                  // output blocks of 32 columns
    constexpr int QF = BF ? DC / 16 : DC / 8;    // fragments of a query row block
    constexpr int LEAST = !PAD ? DC : DC == 256 ? 192 : DC == 192 ? 128 : DC == 128 ? 96 : DC == 96 ? 64 : 0;
    static_assert(DC <= DH && (PAD || DC == DH), "columns");
    constexpr int AHEAD = 4;                     // LDS reads run this many matrix-core steps ahead
    static_assert(CPR >= 8 && CPR <= 64 && NP >= 1 && NP * 2 * STEP == KPW && NS * 32 == KPW, "tile shape");
    constexpr int TILEB = KPW * ROWB, KWB = 2 * NBUF * TILEB;  // one matrix's keys, and all buffers of a key wave
    // O of every wave passes through LDS when the key waves are joined.
    constexpr int JOINB = KW > 1 ? W * 32 * DC * 4 + W * 32 * 8 : 0;
    constexpr int LDSB = KW * KWB > JOINB ? KW * KWB : JOINB;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[LDSB];

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, kw = wave / RW;

    // Every cache line of the arguments requested at once: met one after the other, each would cost a trip to the L2.
    {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&a);
        constexpr int N = sizeof(Args) / 64;
        static_assert(N <= 8, "argument lines");
        asm volatile("" ::"s"(w[0]), "s"(w[16]), "s"(w[32]), "s"(w[48]), "s"(w[64]), "s"(w[16 * (N < 5 ? N : 5)]),
                     "s"(w[16 * (N < 6 ? N : 6)]), "s"(w[16 * (N < 7 ? N : 7)]));
    }
    // This workgroup's key head of a group, row block and slice of the keys.  A group's workgroups go to one XCD where
    // the groups divide among the XCDs, whose L2 then holds their keys; few groups (of an XCD) take turns, so that the
    // row blocks with the most keys of all of them start first, many follow each other.
    int ng, tile_id;
    {
        const int id = blockIdx.x, i = a.by_xcd ? id >> 3 : id;
        const int x = divide(i, a.by_order), y = i - x * a.order;
        const int g = a.turns ? y : x;
        tile_id = a.turns ? x : y;
        ng = a.by_xcd ? (id & 7) + 8 * g : g;
    }
    const int row_tile = divide(tile_id, a.by_splits), split = tile_id - row_tile * a.splits;
    // Row blocks from the last to the first: with causal masks the later ones see more keys and start first.
    const int row0 = (a.n_tiles - 1 - row_tile) * (32 * RW);
    const int u = divide(ng, a.by_hk), hk = ng - u * a.Hk;
    const int rows_end = min(row0 + 32 * RW, a.R);

    // ---------------------------------------------------------------- queries
    typedef typename std::conditional<BF, rm_bf16x8, rm_f32x4>::type QFrag;
    QFrag qf[QF];
    const int row = row0 + rw * 32 + col;  // the lane's (both halves'); rows past the last are the last again
    const int tok = divide(min(row, a.R - 1), a.by_g);
    const int r_head = hk * a.G + min(row, a.R - 1) - tok * a.G;
    const int r_smp = divide(tok, a.by_t), r_tok = tok - r_smp * a.T;  // sample and token
    const char *q = a.q + (static_cast<int64_t>(u) * a.per + r_smp) * a.q_b + r_tok * a.q_t + r_head * a.q_h;
#pragma unroll
    for (int c = 0; c < QF; ++c) {
        const int byte = (2 * c + hi) * 16;
        rm_u32x4 v = {0, 0, 0, 0};
        if (!PAD || byte < a.D * ES) v = *reinterpret_cast<const rm_u32x4 *>(q + byte);
        qf[c] = __builtin_bit_cast(QFrag, v);
    }

    // ---------------------------------------------------------------- the keys that rows see
    // Of the wave's rows: the first and last sample, and over the own keys that rows see the least and greatest begin
    // and end (greatest begin INT_MAX or least end 0 where a row sees none: no tile is whole for it).
    const int w_row = row0 + rw * 32, w_last = min(w_row + 32, a.R) - 1;
    const int w_s0 = w_row < a.R ? divide(divide(w_row, a.by_g), a.by_t) : 0x7fffffff;
    const int w_s1 = w_row < a.R ? divide(divide(w_last, a.by_g), a.by_t) : -1;
    const int s_first = divide(divide(row0, a.by_g), a.by_t), s_last = divide(divide(rows_end - 1, a.by_g), a.by_t);
    const int n0 = a.n0 == 0 ? 0 : (a.len0 ? min(max(a.len0[u], 0), a.n0) : a.n0);
    auto own_len = [&](int smp) __attribute__((always_inline)) {
        return a.n1 > 0 && a.len1 ? min(max(a.len1[static_cast<int64_t>(u) * a.per + smp], 0), a.n1) : a.n1;
    };
    auto causal_end = [&](int len, int t) __attribute__((always_inline)) {
        return min(max(len - a.T + t + 1, 0), len);
    };
    int r_lo, r_len;
    int w_maxlo = 0, w_minhi = 0x7fffffff, w_minlo = 0, w_maxhi = 0x7fffffff;
    int b_lo = 0, b_hi = 0;  // with spans: the keys that any of the workgroup's rows sees
    if (a.span) {
        const int2 *span = reinterpret_cast<const int2 *>(a.span) + static_cast<int64_t>(u) * a.T;
        w_maxlo = 0, w_minhi = 0x7fffffff, w_minlo = 0x7fffffff, w_maxhi = 0;
        const int2 sp = span[r_tok];
        const int lo = min(max(sp.x, 0), a.n1), end = min(max(sp.y, 0), a.n1);
        r_lo = lo;
        r_len = max(end - lo, 0);
        if (lo < end) {
            w_maxlo = max(w_maxlo, lo);
            w_minhi = min(w_minhi, end);
            w_minlo = min(w_minlo, lo);
            w_maxhi = max(w_maxhi, end);
        } else {
            w_maxlo = 0x7fffffff;
        }
        w_maxlo = wave_max(w_maxlo);
        w_minhi = wave_min(w_minhi);
        w_minlo = wave_min(w_minlo);
        w_maxhi = wave_max(w_maxhi);
        b_lo = w_minlo;
        b_hi = w_maxhi;
        if constexpr (RW > 1) {  // the other waves' rows
            int lo = 0x7fffffff, end = 0;
            const int t0 = divide(row0, a.by_g), t1 = divide(rows_end - 1, a.by_g);
            for (int t = t0 + lane; t <= t1; t += 64) {
                const int2 sp = span[t];
                const int x = min(max(sp.x, 0), a.n1), y = min(max(sp.y, 0), a.n1);
                if (x < y) {
                    lo = min(lo, x);
                    end = max(end, y);
                }
            }
            b_lo = wave_min(lo);
            b_hi = wave_max(end);
        }
        b_lo = min(b_lo, b_hi);
    } else {
        const int len = own_len(r_smp);
        r_lo = 0;
        r_len = a.causal ? causal_end(len, r_tok) : len;
        if (a.causal && w_s0 == w_s1) {  // (rows of several samples make every tile partial anyway)
            const int len = __builtin_amdgcn_readfirstlane(own_len(w_s0));
            w_minhi = causal_end(len, divide(w_row, a.by_g) - w_s0 * a.T);
        }
    }

    // ---------------------------------------------------------------- segments of keys
    auto seg_keys = [&](int sg, int &lo, int &end) __attribute__((always_inline)) {
        lo = 0;
        if (sg < 0) {
            end = n0;
        } else if (a.span) {
            lo = b_lo;
            end = b_hi;
        } else {
            end = __builtin_amdgcn_readfirstlane(own_len(sg));
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
    // The slices take the tiles by turns: of the shared keys' tiles followed by the samples', slice s takes those whose
    // number is s modulo the slices, so that each has its share of both.  Every other slice walks its samples' tiles
    // first: those come from far memory while the shared ones' are in the caches.
    const int turns = a.splits;
    const bool own_first = (split & 1) != 0;
    auto tiles_of = [&](int sg) __attribute__((always_inline)) {
        int lo, end;
        seg_keys(sg, lo, end);
        return (end - lo + KT - 1) / KT;
    };
    int64_t n_tiles = 0;
    for (int sg = -1; sg <= s_last; sg = sg < 0 ? s_first : sg + 1) n_tiles += tiles_of(sg);
    if (turns > 1) n_tiles = (n_tiles - split + turns - 1) / turns;
    // Goes to the slice's first tile of t.seg or, if it has none there, of a following segment; t.before: how many
    // tiles come before the segment, modulo the slices.
    auto enter = [&](Tile &t) __attribute__((always_inline)) {
        for (;;) {
            int lo, end;
            seg_keys(t.seg, lo, end);
            const int n = (end - lo + KT - 1) / KT;
            int skip = split - t.before;
            if (skip < 0) skip += turns;
            const bool final = t.seg == (own_first ? -1 : s_last);
            if (skip < n || final) {
                t.kb = lo + min(skip, n) * KT;
                t.end = end;
                break;
            }
            t.before = t.seg == s_last ? 0 : (turns > 1 ? (t.before + n) % turns : 0);
            t.seg = t.seg == s_last ? -1 : (t.seg < 0 ? s_first : t.seg + 1);
        }
        seg_base(t);
    };
    auto first_tile = [&](Tile &t) __attribute__((always_inline)) {
        t.seg = own_first ? s_first : -1;
        t.before = own_first ? tiles_of(-1) % turns : 0;
        enter(t);
    };
    auto advance = [&](Tile &t) __attribute__((always_inline)) {  // only called when another tile follows
        t.kb += turns * KT;
        if (t.kb < t.end) {
            t.k += turns * KT * t.kn;
            t.v += turns * KT * t.vn;
            return;
        }
        t.before = t.seg == s_last ? 0 : (turns > 1 ? (t.before + tiles_of(t.seg)) % turns : 0);
        t.seg = t.seg == s_last ? -1 : (t.seg < 0 ? s_first : t.seg + 1);
        enter(t);
    };

    // ---------------------------------------------------------------- staging
    // A key wave's buffers: NBUF times its keys of a tile, then its values; the RW waves that share them fill them.  A
    // row's 16-byte chunk c lies at c ^ swz(row), so that the lanes of a fragment read, 16 rows at one chunk, take
    // different banks (no conflict counted).  The load instruction n of a wave brings rows n STEP + (rw RPI +
    // lane / CPR); the two terms have no bits in common, so swz of the sum is swz of one ^ swz of the other.
    uint8_t *const lds_w = lds + kw * KWB;
    const uint32_t lds_at = rm_dma::lds_addr(lds_w) + rw * 1024;
    auto swz_k = [](int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; };
    auto swz_v = [](int row) {
        if constexpr (BF)
            return CPR == 8 ? 4 * ((row >> 1) & 1) : 4 * (row & 3);
        else
            return 8 * ((row >> 2) & 1);
    };
    const int lrow = rw * RPI + lane / CPR;
    const uint32_t chunk_k = (lane % CPR ^ swz_k(lrow)) * 16, chunk_v = (lane % CPR ^ swz_v(lrow)) * 16;
    // Loads of pair p of a matrix of tile t into buffer buf.  Rows past the last key are that key again (their scores
    // are masked) and columns past the head's its last ones (set to zero where they meet queries, or not written).
    // Token strides are below 2^24 bytes, so a tile's offsets fit in 32 bits.
    auto stage = [&](const Tile &t, int buf, bool values, int p, uint64_t mask) __attribute__((always_inline)) {
        const uint32_t sn = static_cast<uint32_t>(values ? t.vn : t.kn);
        const int last = t.end - 1 - t.kb;
        int row = kw * KPW + lrow;
        uint32_t chunk = values ? chunk_v : chunk_k;
        asm volatile("" : "+v"(row), "+v"(chunk));  // (else every instruction's offset is kept in a register)
        uint32_t off[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = 2 * p + i;
            uint32_t c = chunk ^ static_cast<uint32_t>((values ? swz_v(n * STEP) : swz_k(n * STEP)) * 16);
            if constexpr (PAD) c = min(c, static_cast<uint32_t>(a.D * ES - 16));
            off[i] = (static_cast<uint32_t>(min(row + n * STEP, last)) & 0xffffffu) * (sn & 0xffffffu) + c;
        }
        dma16_pair<RW * 1024>(values ? t.v : t.k, off[0], off[1],
                              __builtin_amdgcn_readfirstlane(lds_at + (buf * 2 + (values ? 1 : 0)) * TILEB +
                                                             2 * p * RW * 1024),
                              mask);
    };
    // Waits until all but this wave's last `N` loads are there and its LDS reads are done; where several waves share
    // the buffers, until that holds for all of them.
    auto sync = [&](auto n) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        if constexpr (RW > 1) rm_dma::wait_barrier<N>();
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    };
    // Loads in flight when a matrix is waited for: with two buffers the whole other matrix, with one the pairs of the
    // next keys that go out during the softmax.
    constexpr int NH = NBUF == 2 ? 0 : NP / 2;
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, NBUF == 2 ? 2 * NP : 2 * NH> Others;
    typedef std::integral_constant<int, 63> Any;  // reads only
    constexpr uint64_t kAll = ~0ull;

    // A slice without tiles (its row block sees few keys) leaves only its rows' empty maximum and sum.
    if (a.splits > 1 && n_tiles <= 0) {
        if (row < a.R && hi == 0 && kw == 0) {
            const int64_t prow = (static_cast<int64_t>(split) * a.U * a.Hk + ng) * a.R + row;
            a.part_ml[2 * prow] = -INFINITY;
            a.part_ml[2 * prow + 1] = 0.0f;
        }
        return;
    }

    Tile cur;
    first_tile(cur);
    auto start = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < NP; ++p) stage(cur, 0, false, p, kAll);
        if constexpr (NBUF == 2) {
#pragma unroll
            for (int p = 0; p < NP; ++p) stage(cur, 0, true, p, kAll);
        }
    };
    if (n_tiles > 0) start();

    // ---------------------------------------------------------------- fragment addresses
    const uint8_t *kb_ptr[8];  // keys: chunk 2 c + hi of row 32 ns + col, by c mod 8 (the rest are offsets)
#pragma unroll
    for (int c = 0; c < 8; ++c) kb_ptr[c] = lds_w + col * ROWB + (((2 * c + hi) ^ swz_k(col)) & (CPR - 1)) * 16;
    constexpr int VP = BF ? (DB < 4 ? DB : 4) : 2;
    const uint8_t *v_ptr[VP];
    if constexpr (BF) {
        const int i = (lane & 15) >> 2, inner = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
        for (int d = 0; d < VP; ++d)
            v_ptr[d] = lds_w + TILEB + (4 * hi + i) * ROWB + ((d * 64) ^ (swz_v(i) * 16)) + inner;
    } else {
#pragma unroll
        for (int d = 0; d < VP; ++d) v_ptr[d] = lds_w + TILEB + 4 * hi * ROWB + ((d * 128) ^ (hi * 128)) + col * 4;
    }

    rm_f32x16 o[DB];
    float m, l, r_slope;
    int r_pos;
    r_slope = a.slopes ? a.slopes[r_head] * kLog2e : 0.0f;
    // (Slopes: one sample a group.)  A row before the first key or after the last is as far from all keys as one at that
    // end, up to a constant, which the softmax does not see: rows that start farther off than they are long start there,
    // so that distances stay below N + T.
    r_pos = (a.slopes && a.q_start ? min(max(a.q_start[u], -a.T), a.n1) : 0) + r_tok;
    // The scores' registers hold s with score = sc s + off in powers of two: plain products, capped ones as tanh or
    // (LOW) -1 / (1 + e^2x), of which tanh x is 1 + 2 times; with a bias the scores themselves.
    const float sc = a.slopes ? 1.0f : a.cap != 0.0f ? (LOW ? 2.0f * a.cap : a.cap) : a.scale;
    const float off = LOW && a.cap != 0.0f && !a.slopes ? a.cap : 0.0f;

    // ---------------------------------------------------------------- tiles
    // One pass over the slice's tiles, the first one's loads under way.  Returns whether a tile had keys that some rows
    // see and others do not.  There 0 times an infinity or NaN may spoil the rows that do not see it, and a sum keeps
    // the NaN: a workgroup whose results then hold any (there is hardly ever one) makes three more passes.  kClean sets
    // the infinities and NaN among the values to 0 in LDS, the other sums staying as they are bit for bit; kPlus and
    // kMinus count, with weights of 1, the ones of either sign that a row sees, which are then added to its results.
    // So the values' contents bound the time: a call whose values are NaN throughout takes 5 to 12 times the usual (4096
    // causal rows of 16 heads of 128 109 -> 811 us, 850 rows of 256 columns 20 -> 237).
    auto pass = [&](const auto mode) __attribute__((always_inline)) -> bool {
        bool some = false;  // some tile had keys that not all rows see
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = rm_f32x16{};
        int buf = 0;
        // Queries and scalars are waited for here: the compiler would do so in front of their first use, in the loop, and
        // there on every tile for the tile's loads and LDS reads as well (256 single tokens on 1024 shared and 256 own
        // keys 56 -> 67 us, 850 rows on 850 keys 20.4 -> 20.9).
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
        for (int64_t n_left = n_tiles; n_left > 0; --n_left) {
            Tile nxt = cur;
            const bool more = n_left > 1;
            if (more) advance(nxt);
            const uint64_t next = more ? kAll : 0;           // the lanes that load the next tile
            const int at = NBUF == 2 ? buf * 2 * TILEB : 0;  // this tile's buffers
            if constexpr (NBUF == 2) buf ^= 1;
            sync(std::conditional_t<NBUF == 2, Others, None>{});  // the keys

            const int kbw = cur.kb + kw * KPW;
            bool mixed = kbw + KPW > cur.end || mode >= kPlus;  // keys that not all rows see
            if (cur.seg >= 0)
                mixed = mixed || cur.seg != w_s0 || cur.seg != w_s1 || kbw < w_maxlo || kbw + KPW > w_minhi;

            rm_f32x16 s[NS];
#pragma unroll
            for (int ns = 0; ns < NS; ++ns) s[ns] = rm_f32x16{};
            {  // S^T = K Q^T; with two buffers the next tile's keys go out meanwhile, with one this tile's values
                constexpr int X = QF * NS;
                QFrag kf[2 * AHEAD];
                auto read_k = [&](int x) __attribute__((always_inline)) {
                    const int c = x / NS, ns = x % NS;
                    QFrag f = *reinterpret_cast<const QFrag *>(kb_ptr[c & 7] + at + ns * 32 * ROWB + (c >> 3) * 256);
                    constexpr int E = 16 / ES;  // columns past the head's, not to meet the queries' zeros there
                    if (PAD && (2 * c + 2) * E > LEAST) f = (2 * c + hi) * E < a.D ? f : QFrag{};
                    kf[x % (2 * AHEAD)] = f;
                };
#pragma unroll
                for (int x = 0; x < AHEAD; ++x) read_k(x);
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (BF) {
                        s[x % NS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            kf[x % (2 * AHEAD)], qf[x / NS], s[x % NS], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            s[x % NS] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                                kf[x % (2 * AHEAD)][i], qf[x / NS][i], s[x % NS], 0, 0, 0);
                    }
                    if (x + AHEAD < X) read_k(x + AHEAD);
#pragma unroll
                    for (int p = x * NP / X; p < (x + 1) * NP / X; ++p) {
                        if constexpr (NBUF == 2) stage(nxt, buf, false, p, next);
                        else stage(cur, 0, true, p, kAll);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (NBUF == 1) sync(Any{});  // every wave has read the keys: the next ones may come
            auto interval = [&](int &lo, int &len) {  // the keys of this segment that the lane's row sees
                lo = cur.seg < 0 ? 0 : r_lo;
                len = cur.seg < 0 ? n0 : (r_smp == cur.seg ? r_len : 0);
            };
            if (a.cap != 0.0f) {  // (a.scale: the score's over the cap)
                const float x2 = a.scale * (2.0f * kLog2e);
#pragma unroll
                for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if constexpr (LOW)
                            s[ns][i] =
                                __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(s[ns][i] * x2));
                        else
                            s[ns][i] = BF ? tanh_relative(s[ns][i] * a.scale) : tanhf(s[ns][i] * a.scale);
                    }
            }
            if (a.slopes) {
                const float in = a.cap == 0.0f ? a.scale : LOW ? 2.0f * a.cap : a.cap;
                const float add = LOW ? a.cap : 0.0f;
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) {
                    const float d0 = static_cast<float>(r_pos - (kbw + 32 * ns + 4 * hi));
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[ns][i] = fmaf(
                            s[ns][i], in,
                            fmaf(-r_slope, fabsf(d0 - static_cast<float>(8 * (i >> 2) + (i & 3))), add));
                }
            }
            if (mixed) {
                int lo, len;
                interval(lo, len);
#pragma unroll
                for (int ns = 0; ns < NS; ++ns) {
                    const int d0 = kbw + 32 * ns + 4 * hi - lo;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[ns][i] =
                            static_cast<uint32_t>(d0 + 8 * (i >> 2) + (i & 3)) < static_cast<uint32_t>(len)
                                ? s[ns][i]
                                : -INFINITY;
                }
                if (__builtin_expect(mode >= kPlus, false)) {  // (sc 0 + off: a weight of 1)
#pragma unroll
                    for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[ns][i] = s[ns][i] == -INFINITY ? -INFINITY : 0.0f;
                }
            }
            float part[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
            for (int ns = 0; ns < NS; ++ns)
#pragma unroll
                for (int i = ns == 0 ? 4 : 0; i < 16; ++i) part[i & 3] = fmaxf(part[i & 3], s[ns][i]);
            float top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
            top = BF ? fmaf(xor32_max(top), sc, off) : xor32_max(top) * sc;
            // Raising the maximum of a row without sums so far (m = -inf) needs no rescaling.
            const bool raise = top > m + kRaise;  // (false for top = -inf)
            if (__any(raise)) {
                const float mn = raise ? top : m;
                const bool any = __any(raise && m != -INFINITY);
                const float f = raise ? __builtin_amdgcn_exp2f(m - mn) : 1.0f;
                m = mn;
                if (any) {
                    l *= f;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] *= f;
                }
            }
            const float ref = (m == -INFINITY ? 0.0f : m) - off;
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            constexpr int X = 4 * NS;
#pragma unroll
            for (int x = 0; x < X; ++x) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = s[x / 4][4 * (x % 4) + j];
                    // (float32 rounds the score first, as the maximum was: the largest weight is 1 exactly)
                    const float w = __builtin_amdgcn_exp2f(BF ? fmaf(e, sc, -ref) : scaled(e, sc) - ref);
                    s[x / 4][4 * (x % 4) + j] = w;
                    sum[j] += w;
                }
                if (NBUF == 1) {
#pragma unroll
                    for (int p = x * NH / X; p < (x + 1) * NH / X; ++p) stage(nxt, 0, false, p, next);
                }
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            if (more) sync(Others{});  // the values
            else sync(None{});
            if (__builtin_expect(mode != kFirst, false)) {
                for (int i = rw * 64 + lane; i < TILEB / 16; i += 64 * RW) {
                    rm_u32x4 *p = reinterpret_cast<rm_u32x4 *>(lds_w + TILEB + at) + i;
                    rm_u32x4 v = *p;
                    for (int e = 0; e < 4; ++e)
                        v[e] = BF ? marked<BF>(v[e] & 0xffffu, mode) | marked<BF>(v[e] >> 16, mode) << 16
                                  : marked<BF>(v[e], mode);
                    *p = v;
                }
                sync(Any{});
            }
            some = some || mixed;
            {  // O^T += V^T P^T; with two buffers the next tile's values go out meanwhile, with one the rest of its
               // keys.  The weights are rounded to bf16 like the values (2^-8 of each at most, of either sign); the sum
               // that divides them is not.
                constexpr int X = (BF ? 2 : 16) * NS * DB, NQ = NBUF == 2 ? NP : NP - NH;
                typedef typename std::conditional<BF, rm_bf16x8, float>::type VFrag;
                VFrag vf[2 * AHEAD];
                auto read_v = [&](int x) __attribute__((always_inline)) {
                    const int st = x / DB, d = x % DB;
                    if constexpr (BF)
                        vf[x % (2 * AHEAD)] = read_v_rows<ROWB>(v_ptr[d % VP] + at + (d / VP) * 256 + 16 * st * ROWB);
                    else
                        vf[x % (2 * AHEAD)] = *reinterpret_cast<const float *>(
                            v_ptr[d % VP] + at + (d / VP) * 256 +
                            (32 * (st / 16) + 8 * (st % 16 >> 2) + (st & 3)) * ROWB);
                };
                VFrag p;
#pragma unroll
                for (int x = 0; x < AHEAD; ++x) read_v(x);
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    __builtin_amdgcn_sched_barrier(0);
                    const int st = x / DB, d = x % DB;
                    if (d == 0) {
                        if constexpr (BF) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                p[i] = static_cast<__bf16>(s[st / 2][8 * (st % 2) + i]);
                        } else {
                            p = s[st / 16][st % 16];
                        }
                    }
                    const VFrag f = vf[x % (2 * AHEAD)];
                    if constexpr (BF)
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, p, o[d], 0, 0, 0);
                    else
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(f, p, o[d], 0, 0, 0);
                    if (x + AHEAD < X) read_v(x + AHEAD);
#pragma unroll
                    for (int q = x * NQ / X; q < (x + 1) * NQ / X; ++q) {
                        if constexpr (NBUF == 2) stage(nxt, buf, true, q, next);
                        else stage(nxt, 0, false, NH + q, next);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            cur = nxt;
        }
        return some;
    };

    // ---------------------------------------------------------------- join and write
    // Returns whether a result is not finite, or after kClean and kPlus that a pass follows: the same in every wave.
    auto write = [&](const auto mode) __attribute__((always_inline)) -> bool {
        // Of the blocks of 32 columns, wave kw joins those with number kw modulo KW: it has its own sums, the others'
        // come through LDS.
        float *join = reinterpret_cast<float *>(lds);
        float *ml = join + W * 32 * DC;  // [wave][2][32]
        auto slot = [&](int w, int d, int i) {
            return reinterpret_cast<rm_f32x4 *>(join + (((w * DB + d) * 4 + i) * 64 + lane) * 4);
        };
        auto quad = [&](int d, int i) {
            return rm_f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        };
        auto partial_row = [&](int r) { return (static_cast<int64_t>(split) * a.U * a.Hk + ng) * a.R + r; };
        auto out_row = [&](int t) {
            return a.o + (static_cast<int64_t>(u) * a.per + r_smp) * a.o_b + t * a.o_t + r_head * a.o_h;
        };
        if (__builtin_expect(mode >= kPlus, false)) {
            // The counts of all key waves, by way of LDS, to the results of the passes before, which this workgroup wrote
            // before the barrier between them.
            static_assert(LDSB >= W * 32 * DC * 4, "room for the counts");
            __syncthreads();  // every wave has read its last tile
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) *slot(wave, d, i) = quad(d, i);
            __syncthreads();
            const int64_t prow = partial_row(row);
            char *orow = out_row(r_tok);
            const float add = mode == kPlus ? INFINITY : -INFINITY;
#pragma unroll 1
            for (int d = kw; d < DB; d += KW)
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    const int c = 32 * d + 8 * i + 4 * hi;
                    if (row >= a.R || c >= a.D) continue;
                    rm_f32x4 n = {0.0f, 0.0f, 0.0f, 0.0f};
                    for (int k = 0; k < KW; ++k) n += *slot(k * RW + rw, d, i);
                    auto added = [&](auto *p) {
                        auto x = *p;
                        for (int e = 0; e < 4; ++e) x[e] = n[e] == 0.0f ? x[e] : x[e] + add;
                        *p = x;
                    };
                    if (a.splits > 1) added(reinterpret_cast<rm_f32x4 *>(a.part_o + prow * a.D + c));
                    else if constexpr (BF) added(reinterpret_cast<rm_bf16x4 *>(orow + c * 2));
                    else added(reinterpret_cast<rm_f32x4 *>(orow + c * 4));
                }
            __syncthreads();
            return mode == kPlus;
        }
        if constexpr (KW > 1) {
            __syncthreads();  // every wave has read its last tile
            const float sum = xor32_sum(l);
            if (hi == 0) {
                ml[(wave * 2 + 0) * 32 + col] = m;
                ml[(wave * 2 + 1) * 32 + col] = sum;
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
                if (d % KW != kw)
#pragma unroll
                    for (int i = 0; i < 4; ++i) *slot(wave, d, i) = quad(d, i);
            __syncthreads();
        }
        float nan = 0.0f;  // stays 0 unless a result is NaN (or infinite)
        float f[KW], top = m, sum = 0.0f;  // the key waves' factors
        if constexpr (KW > 1) {
            top = -INFINITY;
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                f[k] = ml[((k * RW + rw) * 2 + 0) * 32 + col];
                top = fmaxf(top, f[k]);
            }
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                f[k] = __builtin_amdgcn_exp2f(f[k] - ref);
                sum += ml[((k * RW + rw) * 2 + 1) * 32 + col] * f[k];
            }
        } else {
            sum = xor32_sum(l);
        }
        const int64_t prow = partial_row(row);
        char *orow = out_row(r_tok);
        const float inv = a.splits > 1 ? 1.0f : (sum == 0.0f ? 0.0f : 1.0f / sum);
        if (a.splits > 1 && row < a.R && hi == 0 && kw == 0) {
            a.part_ml[2 * prow] = top;
            a.part_ml[2 * prow + 1] = sum;
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if (KW > 1 && d % KW != kw) continue;
            rm_f32x4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = quad(d, i);
                if constexpr (KW > 1) {
                    v[i] *= f[d % KW];
#pragma unroll
                    for (int k = 0; k < KW; ++k)
                        if (k != d % KW) v[i] += *slot(k * RW + rw, d, i) * f[k];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) nan = fmaf(v[i][e], 0.0f, nan);
            }
            if (a.splits > 1 || !BF) {
                char *dst = a.splits > 1 ? reinterpret_cast<char *>(a.part_o + prow * a.D) : orow;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = 32 * d + 8 * i + 4 * hi;
                    if (row < a.R && (!PAD || c < a.D)) *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = v[i] * inv;
                }
            } else {
                // The lane halves have columns 8 i + {0..3} and + {4..7}: of two such groups each half takes one
                // whole.
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint32_t w[2][2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const rm_f32x4 y4 = v[i + e] * inv;
                        const rm_bf16x4 x = {static_cast<__bf16>(y4[0]), static_cast<__bf16>(y4[1]),
                                             static_cast<__bf16>(y4[2]), static_cast<__bf16>(y4[3])};
                        const uint2 y = __builtin_bit_cast(uint2, x);
                        w[e][0] = y.x, w[e][1] = y.y;
                    }
                    const auto p0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
                    const auto p1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                    const int c = 32 * d + 8 * (i + hi);
                    if (row < a.R && (!PAD || c < a.D))
                        *reinterpret_cast<rm_u32x4 *>(orow + c * 2) = rm_u32x4{p0[0], p1[0], p0[1], p1[1]};
                }
            }
        }
        return __builtin_amdgcn_readfirstlane(__syncthreads_or(!(nan == 0.0f))) != 0 || mode == kClean;
    };
    const std::integral_constant<int, kFirst> first;
    const bool some = pass(first);
    if (__builtin_expect(!write(first), true)) return;
    // Of any wave: the one that joins a column need not be the one whose keys spoiled it.
    if (!__builtin_amdgcn_readfirstlane(__syncthreads_or(some))) return;
    // A second copy of the code above: one copy for all passes costs the usual one up to 4 % (517 rows in float32 15.1 ->
    // 15.7 us, two copies 14.6).
#pragma unroll 1
    for (int mode = kClean;; ++mode) {
        first_tile(cur);
        start();
        pass(mode);
        if (!write(mode)) break;
    }
}

}  // namespace rm_attn
