// Attention of one new token over a paged cache (rm_paged_attention): the kernel that walks the pages, and the join of
// what several of its waves have of one token's head.
#include <algorithm>

#include "rm_attn.h"
#include "rm_serve.h"

namespace rm_serve {

namespace {

using rm_attn::divide;
using rm_attn::kRaise;

// A unit is one key head and up to QR of its query heads; a wave has one.  A token's keys are tiles of KT; the tiles of all
// tokens, one token after the other, are divided evenly among groups of waves, one wave a unit, whatever the lengths are:
// each wave reads the positions, finds the token where its group's share begins and goes on from token to token, the next
// tiles' keys, values, queries and table entries always under way.  So the waves of a group read the heads of the same rows
// at the same time.  A token whose tiles lie in one group's share is written by it; what several have is joined afterwards.
template <bool BF, int DH>
struct Shape {
    static constexpr int ES = BF ? 2 : 4, ROWB = DH * ES, CPR = ROWB / 16;
    static constexpr int RPI = 64 / CPR;                          // rows of a load instruction (1 KB)
    static constexpr int KT = ROWB <= 512 ? 8192 / ROWB : 16;     // keys of a tile
    static constexpr int NI = KT / RPI;                           // load instructions of a tile's keys or values
    static constexpr int TILEB = KT * ROWB;
};
constexpr int room(int columns) { return columns <= 64 ? 64 : columns <= 128 ? 128 : 256; }
template <bool BF, int DH, int QR>
constexpr int lds_bytes() { return 4 * Shape<BF, DH>::TILEB + QR * Shape<BF, DH>::ROWB + 512; }

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Four loads of 16 bytes a lane, to LDS at lds, lds + 1024 and so on, each from its own base in scalar registers and an
// offset a lane (as rm_attn::dma16_pair).  nt: keys and values are read once, and pass by the caches' other lines.
__device__ __forceinline__ void dma16_four(const char *const (&base)[4], const uint32_t (&off)[4], uint32_t lds) {
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %9\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5 nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6 nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %7 nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %8 nt\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base[0]), "s"(base[1]), "s"(base[2]), "s"(base[3]),
          "s"(lds)
        : "memory", "scc");
}
// The same with an address a lane.
__device__ __forceinline__ void dma16_four(const char *const (&at)[4], uint32_t lds) {
    uint32_t keep;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, off nt\n\t"
        "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, off nt\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(keep)
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(lds)
        : "memory", "scc");
}

// A load of 4 bytes a lane into LDS at lds + 4 lane (as rm_dma::dma16).
__device__ __forceinline__ void dma4(const void *g, uint32_t lds) {
    uint32_t keep;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(keep)
                 : "v"(g), "s"(lds)
                 : "memory");
}

// A whole number that is the same in every lane, read by way of the scalar cache: not among the loads that the waits count.
__device__ __forceinline__ int32_t scalar(const int32_t *p, int i) {
    typedef const __attribute__((address_space(4))) int32_t *constant;
    return *reinterpret_cast<constant>(reinterpret_cast<uintptr_t>(p) + static_cast<uintptr_t>(i) * 4);
}

// Joined over the lanes whose numbers are the same modulo 16.
__device__ __forceinline__ float rows_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return rm_attn::xor32_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float rows_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return rm_attn::xor32_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
    const int lo = __shfl(static_cast<int>(x), lane), hi = __shfl(static_cast<int>(x >> 32), lane);
    return static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo));
}

__device__ __forceinline__ int64_t at_lane(int64_t x, int lane) {  // (in scalar registers)
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(x), lane);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(x >> 32), lane);
    return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// The keys [lo, end) that a token at position p of table s sees.
__device__ __forceinline__ void seen(const PagedArgs &a, int p, int s, int &lo, int &end) {
    const int cap = a.per * a.page;
    end = p >= 0 && s >= 0 && s < a.seqs ? min(p, cap - 1) + 1 : 0;
    lo = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
    if (lo >= end) lo = end = 0;
}
template <int KT>
__device__ __forceinline__ int tiles(int lo, int end) {  // (one for a token that sees nothing: its zeros are written)
    return max(1, (end + KT - 1) / KT - lo / KT);
}

// Rows have room for DH columns in LDS; the products take DC of them.
template <bool BF, int DC, int QR>
__global__ __launch_bounds__(64, 1) void paged_kernel(PagedArgs a) {
    constexpr int DH = room(DC);
    typedef Shape<BF, DH> S;
    constexpr int ES = S::ES, ROWB = S::ROWB, CPR = S::CPR, RPI = S::RPI, KT = S::KT, NI = S::NI, TILEB = S::TILEB;
    constexpr int RT = QR > 16 ? 2 : 1;         // tiles of 16 query heads
    constexpr int NS = KT / 16, QF = DC * ES / 64, DB = DC / 16, NQ = QR / RPI;
    constexpr uint64_t kFull = KT == 64 ? ~0ull : (1ull << KT) - 1;
    static_assert(NQ >= 1 && NI >= 1, "load instructions");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[lds_bytes<BF, DH, QR>()];
    uint8_t *const lds_q = lds + 4 * TILEB;
    int32_t *const lds_t = reinterpret_cast<int32_t *>(lds_q + QR * ROWB);
    const uint32_t at_k = rm_dma::lds_addr(lds), at_q = rm_dma::lds_addr(lds_q);
    const uint32_t at_t = at_q + QR * ROWB;
    const int lane = threadIdx.x, m16 = lane & 15, h4 = lane >> 4;
    const int grp = divide(blockIdx.x, a.by_units), unit = blockIdx.x - grp * a.units;
    const int hk = divide(unit, a.by_q_tiles), g0 = (unit - hk * a.q_tiles) * QR;  // the unit's key and first query head
    const int heads = min(QR, a.G - g0);

    // ---------------------------------------------------------------- this group's share
    // Tokens in blocks of 64 times per, a lane's following each other: their positions, tables and tiles in registers.
    constexpr int MOST = 8;
    const int per = min(MOST, (a.N + 63) >> 6);
    int tp[MOST], ts[MOST], tw[MOST];
    auto fetch = [&](int n0) __attribute__((always_inline)) {
        int sum = 0;
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            tp[i] = -1, ts[i] = 0;
            const int n = n0 + lane * per + i;
            if (i < per && n < a.N) {
                tp[i] = a.pos[n];
                ts[i] = a.seq ? a.seq[n] : n;
            }
        }
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            int lo, end;
            seen(a, tp[i], ts[i], lo, end);
            tw[i] = i < per && n0 + lane * per + i < a.N ? tiles<KT>(lo, end) : 0;
            sum += tw[i];
        }
        return sum;
    };
    int total = 0, mine = 0;
    for (int n0 = 0; n0 < a.N; n0 += 64 * per) {
        mine = fetch(n0);
        total += mine;
    }
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o);
    total = __builtin_amdgcn_readfirstlane(total);
    const int share = max((total + a.groups - 1) / a.groups, a.least);
    const int64_t begin64 = static_cast<int64_t>(grp) * share;
    if (begin64 >= total) {
        if (!a.by_token && unit == 0 && lane == 0) a.info[grp] = make_int2(0, 0);
        return;
    }
    const int begin = static_cast<int>(begin64);
    int left = min(share, total - begin);  // tiles of the share that have not been staged
    // The token where it begins, the tiles before it, its position and table.
    int n = 0, before = 0, here_p = -1, here_s = 0;
    for (int n0 = 0; n0 < a.N; n0 += 64 * per) {
        if (a.N > 64 * MOST) mine = fetch(n0);
        int upto = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        const uint64_t past = __ballot(before + upto > begin);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            before += __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l);
            n = n0 + l * per;
            bool found = false;
#pragma unroll
            for (int i = 0; i < MOST; ++i) {
                const int each = __builtin_amdgcn_readlane(tw[i], l);
                if (found) continue;
                found = before + each > begin;
                here_p = __builtin_amdgcn_readlane(tp[i], l);
                here_s = __builtin_amdgcn_readlane(ts[i], l);
                if (!found) before += each, ++n;
            }
            break;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }

    // ---------------------------------------------------------------- tiles
    struct Tile {
        int n, lo, end, t, t0, t1;  // token, its keys and tiles
        int pos, seq;
        int base;                   // the token's first tile among all
    };
    auto enter = [&](Tile &c, int p, int s) __attribute__((always_inline)) {  // c.n's keys
        c.pos = p, c.seq = s;
        seen(a, p, s, c.lo, c.end);
        c.t = c.t0 = c.lo / KT;
        c.t1 = c.t0 + tiles<KT>(c.lo, c.end);
        if (c.end == 0) c.seq = 0;
    };
    int next_p, next_s;  // the next token's
    auto look_at = [&](int i) __attribute__((always_inline)) {
        i = min(i, a.N - 1);
        next_p = scalar(a.pos, i);
        next_s = a.seq ? scalar(a.seq, i) : i;
    };
    auto advance = [&](Tile &c) __attribute__((always_inline)) {
        if (++c.t < c.t1) return;
        c.base += c.t1 - c.t0;
        ++c.n;
        enter(c, next_p, next_s);
        look_at(c.n + 1);
    };

    const int lrow = lane / CPR;
    auto swz_k = [](int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; };
    auto swz_v = [](int row) {
        if constexpr (BF) return CPR == 8 ? 2 * ((row >> 1) & 3) : 2 * (row & 7);
        else return 4 * ((row >> 2) & 3);
    };
    const uint32_t last_chunk = a.D * ES / 16 - 1;
    const uint32_t chunk_k = lane % CPR ^ swz_k(lrow), chunk_v = lane % CPR ^ swz_v(lrow);
    auto fetch_table = [&](const Tile &c, int slot) __attribute__((always_inline)) {
        const int j = min(c.t * KT + (lane & (KT - 1)), max(c.end - 1, 0));
        dma4(a.table + static_cast<int64_t>(c.seq) * a.per + divide(j, a.by_page),
             __builtin_amdgcn_readfirstlane(at_t + slot * 256));
    };
    // Stages a tile whose table entries have come into a buffer, its unit's queries too if it is the first one here; says
    // which of its keys are seen.  The others' rows are the cache's first one.
    auto stage = [&](const Tile &c, int slot, int buf, bool queries) __attribute__((always_inline)) -> uint64_t {
        const int j = c.t * KT + (lane & (KT - 1)), jj = min(j, max(c.end - 1, 0));
        const int pg = lds_t[slot * 64 + lane];
        const bool is = static_cast<uint32_t>(pg) < static_cast<uint32_t>(a.n_pages), ok = is && j >= c.lo && j < c.end;
        // (Where a load instruction's rows are of one page, those behind the last key are that page's next rows.)
        const int at = a.whole ? j : jj;
        const int64_t p = is ? pg : 0, in_page = at - divide(at, a.by_page) * a.page;
        const int64_t ko = p * a.k_p + in_page * a.k_t, vo = p * a.v_p + in_page * a.v_t;
        if (queries) {
            const char *q = a.q + c.n * a.q_t;
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const uint32_t ch = min(chunk_k ^ static_cast<uint32_t>(swz_k(i * RPI)), last_chunk);
                rm_dma::dma16(q + (hk * a.G + g0 + min(i * RPI + lrow, heads - 1)) * a.q_h + ch * 16,
                              __builtin_amdgcn_readfirstlane(at_q + i * 1024));
            }
        }
        auto rows = [&](const char *base, int64_t from, int64_t step, bool values, uint32_t to) __attribute__((always_inline)) {
            auto chunk = [&](int i) {
                const uint32_t x = values ? chunk_v ^ static_cast<uint32_t>(swz_v(i * RPI))
                                          : chunk_k ^ static_cast<uint32_t>(swz_k(i * RPI));
                return min(x, last_chunk) * 16;
            };
            if (a.whole) {  // the rows of an instruction follow each other
                const uint32_t own = lrow * static_cast<uint32_t>(step);
#pragma unroll
                for (int i0 = 0; i0 < NI; i0 += 4) {
                    const char *b[4];
                    uint32_t off[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        b[i] = base + at_lane(from, (i0 + i) * RPI);
                        off[i] = own + chunk(i0 + i);
                    }
                    dma16_four(b, off, __builtin_amdgcn_readfirstlane(to + i0 * 1024));
                }
            } else {
#pragma unroll
                for (int i0 = 0; i0 < NI; i0 += 4) {
                    const char *b[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) b[i] = base + from_lane(from, (i0 + i) * RPI + lrow) + chunk(i0 + i);
                    dma16_four(b, __builtin_amdgcn_readfirstlane(to + i0 * 1024));
                }
            }
        };
        rows(a.k + hk * a.k_h, ko, a.k_t, false, at_k + buf * 2 * TILEB);
        rows(a.v + hk * a.v_h, vo, a.v_t, true, at_k + buf * 2 * TILEB + TILEB);
        return __ballot(ok) & kFull;
    };

    typedef typename std::conditional<BF, rm_bf16x8, rm_f32x4>::type Frag;
    // Chunk 4 c + h4 of row m16, by c mod 4 (the rest are offsets).
    uint32_t k_at[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) k_at[c] = m16 * ROWB + (((4 * c + h4) ^ swz_k(m16)) & (CPR - 1)) * 16;
    auto read_chunk = [&](const uint8_t *rows, int c) __attribute__((always_inline)) {
        Frag f = *reinterpret_cast<const Frag *>(rows + k_at[c & 3] + (c >> 2) * 256);
        // Columns past the head's are its last ones again, which must not meet each other.
        return static_cast<uint32_t>(4 * c + h4) <= last_chunk ? f : Frag{};
    };

    Tile cur;
    cur.n = n;
    look_at(n + 1);
    enter(cur, here_p, here_s);
    cur.base = before;
    cur.t += begin - before;
    fetch_table(cur, 0);
    wait_loads<0>();
    Tile nxt = cur;
    --left;
    if (left > 0) advance(nxt);
    fetch_table(nxt, 1);
    uint64_t vis = stage(cur, 0, 0, true), vis_next = 0;
    bool fresh = true;  // cur is the first tile of a token here

    Frag qf[RT][QF];
    rm_f32x4 o[RT][DB];
    float m[RT], l[RT], slope[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        slope[r] = a.slopes ? a.slopes[hk * a.G + g0 + min(r * 16 + m16, heads - 1)] * rm_attn::kLog2e : 0.0f;
    int2 end_info = make_int2(0, 0);
    for (int turn = 0;; turn ^= 1) {
        const bool more = left > 0, next_fresh = more && nxt.n != cur.n;
        wait_loads<2 * NI>();  // the next tile's table entries, and this one's queries
        if (fresh) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const uint8_t *rows = lds_q + r * 16 * ROWB;
#pragma unroll
                for (int c = 0; c < QF; ++c) {
                    // (QR = 8: rows 8 .. 15 are 0 .. 7 again, in the places that those have)
                    if constexpr (QR == 8) {
                        const int row = m16 & 7;
                        Frag f = *reinterpret_cast<const Frag *>(
                            lds_q + row * ROWB + ((((4 * (c & 3) + h4) ^ swz_k(row)) & (CPR - 1)) * 16) + (c >> 2) * 256);
                        qf[r][c] = static_cast<uint32_t>(4 * c + h4) <= last_chunk ? f : Frag{};
                    } else {
                        qf[r][c] = read_chunk(rows, c);
                    }
                }
                m[r] = -INFINITY;
                l[r] = 0.0f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[r][d] = rm_f32x4{};
            }
        }
        Tile after = nxt;
        const int buf = turn * 2 * TILEB;
        if (more) {
            wait_lds();  // the queries, and the tile before this one: their places are free
            if (left > 1) advance(after);
            // (Its entries go where this tile's were.)
            fetch_table(after, turn);
            vis_next = stage(nxt, turn ^ 1, turn ^ 1, next_fresh);
            if (next_fresh) wait_loads<3 * NI + 1 + NQ>();
            else wait_loads<3 * NI + 1>();
        } else {
            wait_loads<NI>();
        }

        // ---------------------------------------------------------------- S^T = K Q^T
        const uint8_t *const kt = lds + buf, *const vt = kt + TILEB;
        rm_f32x4 s[RT][NS];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < NS; ++i) s[r][i] = rm_f32x4{};
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int c = 0; c < QF; ++c) {
                const Frag kf = read_chunk(kt + i * 16 * ROWB, c);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    if constexpr (BF) {
                        s[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][c], s[r][i], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[r][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[r][c][e], s[r][i], 0, 0, 0);
                    }
                }
            }

        // ---------------------------------------------------------------- softmax
        const int j0 = cur.t * KT + 4 * h4;
        const uint64_t bits = vis >> (4 * h4);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[r][i][e] * a.scale;
                    if (a.cap != 0.0f) x = a.cap * (BF ? rm_attn::tanh_relative(x) : tanhf(x));
                    if (a.slopes) x = fmaf(-slope[r], static_cast<float>(cur.pos - (j0 + 16 * i + e)), x);
                    if (vis != kFull) x = (bits >> (16 * i + e)) & 1 ? x : -INFINITY;
                    s[r][i][e] = x;
                    top = fmaxf(top, x);
                }
            top = rows_max(top);
            const bool raise = top > m[r] + kRaise;  // (false for top = -inf)
            if (__any(raise)) {
                const float mn = raise ? top : m[r];
                const float f = raise ? __builtin_amdgcn_exp2f(m[r] - mn) : 1.0f;
                m[r] = mn;
                l[r] *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[r][d] *= f;
            }
            const float ref = m[r] == -INFINITY ? 0.0f : m[r];
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r][i][e] = __builtin_amdgcn_exp2f(s[r][i][e] - ref);
                    l[r] += s[r][i][e];
                }
        }

        // ---------------------------------------------------------------- O^T += V^T P^T
        if (more) {
            if (next_fresh) wait_loads<2 * NI + 1 + NQ>();
            else wait_loads<2 * NI + 1>();
        } else {
            wait_loads<0>();
        }
        if (vis != kFull) {  // values of keys that are not seen: 0 times an infinity or NaN is not 0
#pragma unroll
            for (int i = 0; i < TILEB / 1024; ++i) {
                const int at = i * 64 + lane;
                if (!((vis >> (at / CPR)) & 1)) *reinterpret_cast<rm_u32x4 *>(lds + buf + TILEB + at * 16) = rm_u32x4{0, 0, 0, 0};
            }
            wait_lds();
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            if constexpr (BF) {
                typedef __attribute__((address_space(3))) rm_s16x4 lds_s16x4;
                rm_s16x4 p[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const rm_bf16x4 b = {static_cast<__bf16>(s[r][i][0]), static_cast<__bf16>(s[r][i][1]),
                                         static_cast<__bf16>(s[r][i][2]), static_cast<__bf16>(s[r][i][3])};
                    p[r] = __builtin_bit_cast(rm_s16x4, b);
                }
                const int row = 4 * h4 + (m16 >> 2);
                const uint8_t *v = vt + (16 * i + row) * ROWB + (m16 & 3) * 8;
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const rm_s16x4 f = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_s16x4 *)(v + (((2 * d) & 15) ^ swz_v(row)) * 16 + (d >> 3) * 256));
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        o[r][d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(f, p[r], o[r][d], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = 16 * i + 4 * h4 + e;
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const float f = *reinterpret_cast<const float *>(
                            vt + row * ROWB + (((4 * d) & 15) ^ (4 * h4)) * 16 + (d >> 2) * 256 + m16 * 4);
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            o[r][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(f, s[r][i][e], o[r][d], 0, 0, 0);
                    }
                }
            }
        }

        // ---------------------------------------------------------------- the token's end, or the share's
        if (!more || next_fresh) {
            const bool starts = cur.base >= begin, ends = cur.t + 1 == cur.t1;
            if (starts) {
                const int parts = (cur.base + (cur.t1 - cur.t0) - 1) / share - grp + 1;
                if (a.by_token && unit == 0 && lane == 0) a.info[cur.n] = make_int2(grp, parts);
                if (!ends) end_info = make_int2(cur.n, parts);
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float sum = rows_sum(l[r]);
                const int g = r * 16 + m16;
                if (g >= heads) continue;
                if (starts && ends) {
                    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                    char *dst = a.o + cur.n * a.o_t + static_cast<int64_t>(hk * a.G + g0 + g) * a.o_h;
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const int c = 16 * d + 4 * h4;
                        if (c >= a.D) continue;
                        const rm_f32x4 y = o[r][d] * inv;
                        if constexpr (BF)
                            *reinterpret_cast<rm_bf16x4 *>(dst + c * 2) =
                                rm_bf16x4{static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1]), static_cast<__bf16>(y[2]),
                                          static_cast<__bf16>(y[3])};
                        else
                            *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = y;
                    }
                } else {
                    const int64_t row = ((2 * static_cast<int64_t>(grp) + starts) * a.units + unit) * QR + g;
                    if (h4 == 0) a.part_ml[row] = make_float2(m[r], sum);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const int c = 16 * d + 4 * h4;
                        if (c < a.D) *reinterpret_cast<rm_f32x4 *>(a.part_o + row * a.D + c) = o[r][d];
                    }
                }
            }
        }
        if (!more) break;
        cur = nxt;
        nxt = after;
        vis = vis_next;
        fresh = next_fresh;
        --left;
    }
    if (!a.by_token && unit == 0 && lane == 0) a.info[grp] = end_info;
}

// One workgroup an entry, unit and query head of it: the parts that groups of waves left of a token, in a fixed order.
template <bool BF, int LPR, int QR>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a) {
    constexpr int GR = 256 / LPR;
    __shared__ float tops[GR], sums[GR];
    __shared__ rm_f32x4 part[GR][LPR];
    const int each = a.units * a.rows, e = blockIdx.x / each, ur = blockIdx.x - e * each;
    const int u = ur / a.rows, r = ur - u * a.rows;
    const int2 info = a.info[e];
    const int parts = info.y, n = a.by_token ? e : info.x, first = a.by_token ? info.x : e;
    if (parts < 2) return;
    const int hk = u / a.q_tiles, g = (u - hk * a.q_tiles) * QR + r;
    if (g >= a.G) return;
    auto row = [&](int p) { return ((2 * static_cast<int64_t>(first + p) + (p == 0)) * a.units + u) * QR + r; };
    const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR;
    const int c = min(lane * 4, a.D - 4);
    rm_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;
    for (int p0 = grp; p0 < parts; p0 += 4 * GR) {
        float2 ml[4];
        rm_f32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = row(min(p0 + i * GR, parts - 1));
            ml[i] = a.part_ml[at];
            v[i] = *reinterpret_cast<const rm_f32x4 *>(a.part_o + at * a.D + c);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p0 + i * GR >= parts) ml[i] = make_float2(-INFINITY, 0.0f);
            top = fmaxf(top, ml[i].x);
        }
        const float ref = top == -INFINITY ? 0.0f : top;
        float f = __builtin_amdgcn_exp2f(m - ref);
        l *= f;
        o *= f;
        m = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (ml[i].y == 0.0f) continue;  // (no key with a weight: its sums are zeros)
            f = __builtin_amdgcn_exp2f(ml[i].x - ref);
            l += ml[i].y * f;
            o += v[i] * f;
        }
    }
    if (lane == 0) tops[grp] = m;
    __syncthreads();
    float top = tops[0];
#pragma unroll
    for (int i = 1; i < GR; ++i) top = fmaxf(top, tops[i]);
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    o *= f;
    l *= f;
    part[grp][lane] = o;
    if (lane == 0) sums[grp] = l;
    __syncthreads();
    if (grp != 0 || lane * 4 >= a.D) return;
    float sum = 0.0f;
    o = rm_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < GR; ++i) {
        sum += sums[i];
        o += part[i][lane];
    }
    o *= sum == 0.0f ? 0.0f : 1.0f / sum;
    char *dst = a.o + n * a.o_t + static_cast<int64_t>(hk * a.G + g) * a.o_h;
    if constexpr (BF)
        *reinterpret_cast<rm_bf16x4 *>(dst + c * 2) =
            rm_bf16x4{static_cast<__bf16>(o[0]), static_cast<__bf16>(o[1]), static_cast<__bf16>(o[2]), static_cast<__bf16>(o[3])};
    else
        *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = o;
}

template <bool BF, int DC, int QR>
hipError_t go(const PagedPlan &p, const PagedArgs &a, hipStream_t st) {
    paged_kernel<BF, DC, QR><<<dim3(static_cast<unsigned>(a.groups) * a.units), 64, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.join) return e;
    const unsigned entries = static_cast<unsigned>(std::min(a.N, a.groups));
    paged_join_kernel<BF, room(DC) / 4, QR><<<dim3(entries * a.units * a.rows), 256, 0, st>>>(a);
    return hipGetLastError();
}
template <bool BF, int DC>
hipError_t by_heads(const PagedPlan &p, const PagedArgs &a, hipStream_t st) {
    return p.qr == 8 ? go<BF, DC, 8>(p, a, st) : p.qr == 16 ? go<BF, DC, 16>(p, a, st) : go<BF, DC, 32>(p, a, st);
}
// The least of 64, 96, 128, 192 and 256 columns that hold the head.
template <bool BF>
hipError_t by_width(const PagedPlan &p, const PagedArgs &a, hipStream_t st) {
    if (a.D <= 64) return by_heads<BF, 64>(p, a, st);
    if (a.D <= 96) return by_heads<BF, 96>(p, a, st);
    if (a.D <= 128) return by_heads<BF, 128>(p, a, st);
    return a.D <= 192 ? by_heads<BF, 192>(p, a, st) : by_heads<BF, 256>(p, a, st);
}

template <bool BF, int DH>
void shape_of(PagedPlan &p) {
    const int bytes = p.qr == 8    ? lds_bytes<BF, DH, 8>()
                      : p.qr == 16 ? lds_bytes<BF, DH, 16>()
                                   : lds_bytes<BF, DH, 32>();
    p.kt = Shape<BF, DH>::KT;
    p.rpi = Shape<BF, DH>::RPI;
    p.per_cu = std::min(4, 160 * 1024 / bytes);
}

}  // namespace

void paged_shape(bool bf16, int D, int G, PagedPlan *p) {
    const int dh = room(D);
    p->qr = G <= 8 ? 8 : G <= 16 ? 16 : 32;
    if (bf16) dh == 64 ? shape_of<true, 64>(*p) : dh == 128 ? shape_of<true, 128>(*p) : shape_of<true, 256>(*p);
    else dh == 64 ? shape_of<false, 64>(*p) : dh == 128 ? shape_of<false, 128>(*p) : shape_of<false, 256>(*p);
}

hipError_t launch_paged(const PagedPlan &p, const PagedArgs &a, bool bf16, hipStream_t st) {
    return bf16 ? by_width<true>(p, a, st) : by_width<false>(p, a, st);
}

}  // namespace rm_serve
