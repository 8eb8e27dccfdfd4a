// Attention of one new token over a paged cache (rm_paged_attention; bf16 in paged_attn_bf16.hip, float32 in
// paged_attn_f32.hip): the kernel that walks the pages, and the join of what several of its waves have of one token's head.
//
// One pass over the keys with a running maximum and sum, as in rm_attn.h, but for rows that share their keys only with the
// few query heads of a key head: every byte of the cache is read once, and reading is what bounds it.  What that took, us for
// 64 tokens of 32 heads on 8 on up to 8192 keys (1.18 GB) / 4 of 32 on 4 on 131072 (1.06 GB), bf16, heads of 128 columns:
// a workgroup a query head 4998 / 67790; the kernel below with a wave a share of (token, head, key) 248 / 209; loads past the
// caches' other lines 191 / 180; waves of a group on the same rows at the same time, and what else is told below, 189 / 173:
// 6.2 and 6.1 TB/s (a read of one large buffer: 5.9).  Smaller calls are bound by round trips: launch, positions, table,
// keys, the parts' join: one token on 850 keys 11.3, on 8192 14.7.
#pragma once

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
//
// The wave is alone in its workgroup, so that nothing waits for another: 32 KB of LDS hold two tiles' keys and values, four
// waves to a compute unit, up to 128 KB under way for each, of which memory's latency needs about 50.  Tiles of half the size
// and twice the waves took 231 / 211 where these took 229 / 207, and 143 where these took 131 on 512 short sequences.
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

// Matrix-core layout (16x16 tiles): S^T = K Q^T, so a lane holds scores of query head lane % 16, keys 4 (lane / 16) + {0..3} of
// 16; O^T = V^T P^T takes them as they are, V's fragments read in the same order of keys.  A group of 8 heads fills half of
// a tile, which costs nothing in bf16 (the products take a sixth of the time that a tile's bytes do); in float32 they are a third
// of a step of 2.1 us, and issuing the loads half of it (37 tokens of 6 heads on 3, 72 columns, up to 1111 keys each: 25 us
// for 63 MB; a row has room for 128 columns in LDS, so that 14 of its 32 lanes fetch the last 16 bytes again).  Fragments of
// QR = 8 heads are kept in half the LDS, so that four waves fit.

// The value, as if it became known here only: what is made of it then stays where it is used, instead of taking registers
// and time in front of the loop.
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The kernel's arguments, to be read when they are used: kept from the start, they would take the scalar registers of the
// loop.
typedef const __attribute__((address_space(4))) PagedArgs *Arguments;
__device__ __forceinline__ Arguments again() {
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return (Arguments)p;
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

// Weights as the matrix cores take them, in two bf16 parts: what truncation leaves, and the rest, of which at most half a step
// is lost, 2^-8 of a value below 2^-7 of the weight.  In one part the loss was up to 2^-8 of each weight, as much as the
// rounding of the output (error of 64 bf16 tokens against 64 bits 2.0e-3, now 1.7e-3, what the output's rounding leaves).  The
// rest of a weight that is not 0 is not 0 either (at least 2^-100, or as much as such a small weight): times an infinite value
// it would be NaN.  The second product costs 64 tokens 0.5 of 199 us in a graph, 64 of 20 heads to a key head 0.5 of 26.4
// (with matrix instructions of 16 keys 1.0 and 2.7).
__device__ __forceinline__ void in_two(rm_f32x4 w, rm_s16x4 &high, rm_s16x4 &rest) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t bits = __float_as_uint(w[e]);
        const float r = fmaxf(w[e] - __uint_as_float(bits & 0xffff0000u), fminf(w[e], 0x1p-100f));
        high[e] = static_cast<short>(bits >> 16);
        rest[e] = __builtin_bit_cast(short, static_cast<__bf16>(r));
    }
}

// The sum of a value over the lanes up to the own one, in data-parallel steps along the rows of 16 lanes and across them.
__device__ __forceinline__ int running_sum(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return v;
}

// The keys [lo, end) that a token at position p of table s sees.
template <class A>
__device__ __forceinline__ void seen(const A &a, int p, int s, int &lo, int &end) {
    const int cap = a.per * a.page;
    const bool is = (p >= 0) & (static_cast<uint32_t>(s) < static_cast<uint32_t>(a.seqs));
    end = is ? min(p, cap - 1) + 1 : 0;
    const bool cut = (a.window > 0) & (p >= a.window);
    lo = cut ? p - a.window + 1 : 0;
    const bool any = lo < end;
    lo = any ? lo : 0;
    end = any ? end : 0;
}
template <int KT>
__device__ __forceinline__ int tiles(int lo, int end) {  // (one for a token that sees nothing: its zeros are written)
    return max(1, (end + KT - 1) / KT - lo / KT);
}

// Rows have room for DH columns in LDS; the products take DC of them.  WHOLE: the rows of a load instruction are of one page.
template <bool BF, bool WHOLE, int DC, int QR>
__global__ __launch_bounds__(64, 1) void paged_kernel(PagedArgs a) {
    constexpr int DH = room(DC);
    typedef Shape<BF, DH> S;
    constexpr int ES = S::ES, ROWB = S::ROWB, CPR = S::CPR, RPI = S::RPI, KT = S::KT, NI = S::NI, TILEB = S::TILEB;
    constexpr int RT = QR > 16 ? 2 : 1;         // tiles of 16 query heads
    constexpr int NS = KT / 16, QF = DC * ES / 64, DB = DC / 16, NQ = QR / RPI;
    constexpr uint64_t kFull = ~0ull >> (64 - KT);
    static_assert(NQ >= 1 && NI % 4 == 0 && DC / 16 % (NI / 4) == 0, "load instructions");
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
    int share, begin, left;       // tiles of a share, the first one's number, tiles that have not been staged
    int n, before;                // the token where it begins, and the tiles before it,
    int here_p, here_s, next_p, next_s;  // its position and table, and the next token's
    const int32_t *const seqs = a.seq ? a.seq : a.pos;  // (something to load from either way)
    auto look_at = [&](int i) __attribute__((always_inline)) {
        const Arguments b = again();
        const int32_t *pos = b->pos, *seq = b->seq;
        i = min(i, b->N - 1);
        next_p = scalar(pos, i);
        next_s = seq ? scalar(seq, i) : i;
    };
    auto divided = [&](int total) __attribute__((always_inline)) {  // false: there is nothing for this group
        share = max(divide(total + a.groups - 1, a.by_groups), 1);
        const int64_t first = static_cast<int64_t>(grp) * share;
        begin = static_cast<int>(min(first, static_cast<int64_t>(total)));
        left = min(share, total - begin);
        if (left <= 0 && a.info && !a.by_token && unit == 0 && lane == 0) a.info[grp] = make_int2(0, 0);
        return left > 0;
    };
    if (__builtin_expect(a.N <= 64, true)) {  // a token a lane
        const int i = min(lane, a.N - 1), p = a.pos[i], t = a.seq ? seqs[i] : i;
        int lo, end;
        seen(a, p, t, lo, end);
        const int mine = lane < a.N ? tiles<KT>(lo, end) : 0, upto = running_sum(mine);
        if (!divided(__builtin_amdgcn_readlane(upto, 63))) return;
        n = __builtin_ctzll(__ballot(upto > begin) | 1ull << 63);
        before = __builtin_amdgcn_readlane(upto, n) - __builtin_amdgcn_readlane(mine, n);
        here_p = __builtin_amdgcn_readlane(p, n), here_s = __builtin_amdgcn_readlane(t, n);
        next_p = __builtin_amdgcn_readlane(p, min(n + 1, 63)), next_s = __builtin_amdgcn_readlane(t, min(n + 1, 63));
    } else {  // blocks of 512 tokens, a lane's eight following each other
        constexpr int PER = 8;
        int tw[PER], mine = 0, total = 0;
        auto fetch = [&](int n0) __attribute__((always_inline)) {
            int tp[PER], ts[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = min(n0 + lane * PER + i, a.N - 1);
                tp[i] = a.pos[at];
                ts[i] = seqs[at];
            }
            mine = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                int lo, end;
                seen(a, tp[i], a.seq ? ts[i] : n0 + lane * PER + i, lo, end);
                tw[i] = n0 + lane * PER + i < a.N ? tiles<KT>(lo, end) : 0;
                mine += tw[i];
            }
        };
#pragma unroll 1
        for (int n0 = 0; n0 < a.N; n0 += 64 * PER) {
            fetch(n0);
            total += mine;
        }
        if (!divided(__builtin_amdgcn_readlane(running_sum(total), 63))) return;
        n = a.N - 1, before = 0;
#pragma unroll 1
        for (int n0 = 0; n0 < a.N; n0 += 64 * PER) {
            if (a.N > 64 * PER) fetch(n0);
            const int upto = running_sum(mine);
            const uint64_t past = __ballot(before + upto > begin);
            if (past != 0) {
                const int l = __builtin_ctzll(past);
                before += __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l);
                n = n0 + l * PER;
                bool found = false;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int each = __builtin_amdgcn_readlane(tw[i], l);
                    found = found || before + each > begin;
                    if (!found) before += each, ++n;
                }
                break;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
        look_at(n);
        here_p = next_p, here_s = next_s;
        look_at(n + 1);
    }

    // ---------------------------------------------------------------- tiles
    struct Tile {
        int n, lo, end, t, t0, t1;  // token, its keys and tiles
        int seq;
        int base;                   // the token's first tile among all
    };
    auto enter = [&](Tile &c, int p, int s) __attribute__((always_inline)) {  // c.n's keys
        c.seq = s;
        seen(*again(), p, s, c.lo, c.end);
        c.t = c.t0 = c.lo / KT;
        c.t1 = c.t0 + tiles<KT>(c.lo, c.end);
        if (c.end == 0) c.seq = 0;
    };
    auto advance = [&](Tile &c) __attribute__((always_inline)) {
        if (++c.t < c.t1) return;
        c.base += c.t1 - c.t0;
        c.n = min(c.n + 1, a.N - 1);
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
        const Arguments b = again();
        dma4(b->table + static_cast<int64_t>(c.seq) * b->per + divide(j, a.by_page),
             __builtin_amdgcn_readfirstlane(at_t + slot * 256));
    };
    // Of a tile whose table entries have come: where the lane's key and value are (from the head's first row on), and which
    // keys are seen.  A page that is none is taken for the first one.
    // WHOLE: in units of 16 bytes, of which a cache has fewer than 2^32.
    typedef typename std::conditional<WHOLE, uint32_t, int64_t>::type Offset;
    const uint32_t k_p16 = static_cast<uint32_t>(a.k_p >> 4), k_t16 = static_cast<uint32_t>(a.k_t >> 4);
    const uint32_t v_p16 = static_cast<uint32_t>(a.v_p >> 4), v_t16 = static_cast<uint32_t>(a.v_t >> 4);
    struct Place {
        Offset k, v;
        uint64_t vis;
    };
    auto place = [&](const Tile &c, int slot) __attribute__((always_inline)) {
        const int j = c.t * KT + (lane & (KT - 1)), jj = min(j, max(c.end - 1, 0));
        const int pg = lds_t[slot * 64 + lane];
        const bool is = static_cast<uint32_t>(pg) < static_cast<uint32_t>(a.n_pages), ok = is && j >= c.lo && j < c.end;
        // (WHOLE: rows behind the last key are its page's next ones, as far as the load instruction that has it goes.)
        const int at = WHOLE ? j : jj;
        const Offset p = is ? pg : 0, in_page = at - divide(at, a.by_page) * a.page;
        if constexpr (WHOLE)
            return Place{p * k_p16 + in_page * k_t16, p * v_p16 + in_page * v_t16, __ballot(ok) & kFull};
        else
            return Place{p * a.k_p + in_page * a.k_t, p * a.v_p + in_page * a.v_t, __ballot(ok) & kFull};
    };
    auto stage_queries = [&](const Tile &c) __attribute__((always_inline)) {
        const Arguments b = again();
        const char *q = b->q + c.n * b->q_t;
        const int own = here(lane), orow = own / CPR;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const uint32_t ch = min(static_cast<uint32_t>(own % CPR ^ swz_k(orow) ^ swz_k(i * RPI)), last_chunk);
            rm_dma::dma16(q + (hk * b->G + g0 + min(i * RPI + orow, heads - 1)) * b->q_h + ch * 16,
                          __builtin_amdgcn_readfirstlane(at_q + i * 1024));
        }
    };
    const char *const k_head = a.k + hk * a.k_h, *const v_head = a.v + hk * a.v_h;
    // Load instructions i0 .. i0 + 3 of a tile's keys or values into a buffer.
    auto stage = [&](const Place &at, bool values, int i0, int buf) __attribute__((always_inline)) {
        const char *const base = values ? v_head : k_head, *b[4];
        const Offset from = values ? at.v : at.k;
        const uint32_t to = __builtin_amdgcn_readfirstlane(at_k + (buf * 2 + values) * TILEB + i0 * 1024);
        auto chunk = [&](int i) {
            const uint32_t x = values ? chunk_v ^ static_cast<uint32_t>(swz_v(i * RPI))
                                      : chunk_k ^ static_cast<uint32_t>(swz_k(i * RPI));
            return min(x, last_chunk) * 16;
        };
        if constexpr (WHOLE) {  // the rows of an instruction follow each other
            uint32_t off[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b[i] = base + (static_cast<uint64_t>(__builtin_amdgcn_readlane(from, (i0 + i) * RPI)) << 4);
                off[i] = (lrow * (values ? v_t16 : k_t16) << 4) + chunk(i0 + i);
            }
            dma16_four(b, off, to);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = base + from_lane(from, (i0 + i) * RPI + lrow) + chunk(i0 + i);
            dma16_four(b, to);
        }
    };

    typedef typename std::conditional<BF, rm_bf16x8, rm_f32x4>::type Frag;
    // Chunk 4 c + h4 of row m16, by c mod 4 (the rest are offsets).
    uint32_t k_at[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) k_at[c] = m16 * ROWB + (((4 * c + h4) ^ swz_k(m16)) & (CPR - 1)) * 16;
    auto read_chunk = [&](const uint8_t *rows, int c) __attribute__((always_inline)) {
        return *reinterpret_cast<const Frag *>(rows + k_at[c & 3] + (c >> 2) * 256);
    };
    // Columns past the head's are its last ones again, which must not meet each other.
    const bool narrow = last_chunk + 1 < DC * ES / 16;
    auto own_columns = [&](Frag &f, int c) __attribute__((always_inline)) {
        f = static_cast<uint32_t>(4 * c + h4) <= last_chunk ? f : Frag{};
    };

    Tile cur, nxt;
    nxt.n = n;
    enter(nxt, here_p, here_s);
    nxt.base = before;
    nxt.t += begin - before;
    cur = nxt;
    fetch_table(nxt, 0);
    uint64_t vis = 0;
    bool fresh = true;  // cur is the first tile of a token here

    Frag qf[RT][QF];
    rm_f32x4 o[RT][DB];
    float m[RT], l[RT], slope[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        slope[r] = a.slopes ? a.slopes[hk * a.G + g0 + min(r * 16 + m16, heads - 1)] * rm_attn::kLog2e : 0.0f;
    const float sc = a.cap != 0.0f || a.slopes ? 1.0f : a.scale;
    int2 end_info = make_int2(0, 0);
    // A step stages a tile and takes the products of the one before it; the first has none before it.  The load
    // instructions go out between the products, since a wave that issues several in a row waits for the load unit.
    bool first = true;
    Place next = {0, 0, 0};
    for (int turn = 0;; turn ^= 1) {
        const bool more = left > 0, next_fresh = more && (first || nxt.n != cur.n);
        if (first) wait_loads<0>();
        else wait_loads<NI>();  // the next tile's table entries, this one's queries and keys
        const int buf = (turn ^ 1) * 2 * TILEB;
        const uint8_t *const kt = lds + buf, *const vt = kt + TILEB;
        if (!first && fresh) {
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
                        qf[r][c] = f;
                    } else {
                        qf[r][c] = read_chunk(rows, c);
                    }
                    own_columns(qf[r][c], c);
                }
                m[r] = -INFINITY;
                l[r] = 0.0f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[r][d] = rm_f32x4{};
            }
        }
        // ---------------------------------------------------------------- S^T = K Q^T
        Tile after = nxt;
        if (more) {
            if (left > 1) advance(after);
            next = place(nxt, turn);
            wait_lds();  // the queries, the table entries and the values of the tile before this one: their places are free
            fetch_table(after, turn ^ 1);
            if (next_fresh) stage_queries(nxt);
        }
        constexpr int CH = NS == 1 ? 2 : 1, GS = NI / 4;  // (two chains of sums where there is one tile of 16 keys)
        rm_f32x4 part[CH][RT][NS];
#pragma unroll
        for (int h = 0; h < CH; ++h)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < NS; ++i) part[h][r][i] = rm_f32x4{};
        // In as many groups as the loads: a group's reads from LDS, four load instructions, its products, so that a read's way
        // to LDS and back passes while the load unit is busy, and few fragments take registers.
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            constexpr int PER = (QF + GS - 1) / GS;
            const int c0 = g * QF / GS, c1 = (g + 1) * QF / GS;
            Frag kf[PER][NS];
            __builtin_amdgcn_sched_barrier(0);
            if (!first) {
#pragma unroll
                for (int c = c0; c < c1; ++c)
#pragma unroll
                    for (int i = 0; i < NS; ++i) kf[c - c0][i] = read_chunk(kt + i * 16 * ROWB, c);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) stage(next, false, 4 * g, turn);
            if (first) continue;
            if (narrow) {
#pragma unroll
                for (int c = c0; c < c1; ++c)
#pragma unroll
                    for (int i = 0; i < NS; ++i) own_columns(kf[c - c0][i], c);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = c0; c < c1; ++c)
#pragma unroll
                for (int i = 0; i < NS; ++i)
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        rm_f32x4 &x = part[c % CH][r][i];
                        if constexpr (BF) {
                            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c - c0][i], qf[r][c], x, 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c - c0][i][e], qf[r][c][e], x, 0, 0, 0);
                        }
                    }
        }
        if (first) {
#pragma unroll
            for (int g = 0; g < GS; ++g) stage(next, true, 4 * g, turn);
            cur = nxt, nxt = after, vis = next.vis, first = false;
            --left;
            continue;
        }
        rm_f32x4 s[RT][NS];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s[r][i] = part[0][r][i];
                if constexpr (CH > 1) s[r][i] += part[CH - 1][r][i];
            }

        // ---------------------------------------------------------------- softmax
        auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < NS; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r][i][e] = f(s[r][i][e], r, 16 * i + e);
        };
        // Scores in powers of two are sc times these: plain products, or with a cap or a bias the scores themselves.
        if (__builtin_expect(a.cap != 0.0f, false))
            each([&](float x, int, int) { return a.cap * (BF ? rm_attn::tanh_relative(x * a.scale) : tanhf(x * a.scale)); });
        // A bias is counted from the key that a token may see where it is highest (the last one, for a negative slope the first):
        // the same weights, and a position far behind the table costs them no digits.  Slope times distance may still be far
        // larger than what tells the weights apart, so it is rounded only after `off` is taken from it, about what it is where
        // it counts: the running maximum, or the highest bias of the tile, if that is more (a token's first tile, or the first
        // after missing pages).  Beyond 2^24 the maximum's own rounding would count; there the nearest key has the weight.
        float off[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) off[r] = 0.0f;
        if (__builtin_expect(a.slopes != nullptr, false)) {
            const float in = a.cap != 0.0f ? 1.0f : a.scale;
            int from[RT];  // distance of the tile's first key
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bool rises = slope[r] < 0.0f;  // (with the distance)
                from[r] = (rises ? cur.lo : cur.end - 1) - cur.t * KT;
                const int nearest = rises ? min(from[r], 0) : max(from[r] - (KT - 1), 0);
                const float about = fmaxf(m[r], -slope[r] * static_cast<float>(nearest));
                off[r] = fabsf(about) < 0x1p24f ? about : 0.0f;
            }
            const int own = 4 * here(h4);
            each([&](float x, int r, int j) {
                return fmaf(x, in, fmaf(-slope[r], static_cast<float>(from[r] - own - j), -off[r]));
            });
        }
        if (__builtin_expect(vis != kFull, false)) {
            const uint64_t bits = vis >> (4 * here(h4));
            each([&](float x, int, int j) { return (bits >> j) & 1 ? x : -INFINITY; });
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, s[r][i][e]);
            top = rows_max(top) * sc + off[r];
            const bool raise = top > m[r] + kRaise;  // (false for top = -inf)
            if (__any(raise)) {
                const float mn = raise ? top : m[r];
                const float f = raise ? __builtin_amdgcn_exp2f(m[r] - mn) : 1.0f;
                m[r] = mn;
                l[r] *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[r][d] *= f;
            }
            const float ref = (m[r] == -INFINITY ? 0.0f : m[r]) - off[r];
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // (float32 rounds the score first, as the maximum was: the largest weight is 1 exactly)
                    const float x = s[r][i][e];
                    s[r][i][e] = __builtin_amdgcn_exp2f(BF ? fmaf(x, sc, -ref) : rm_attn::scaled(x, sc) - ref);
                    l[r] += s[r][i][e];
                }
        }

        // ---------------------------------------------------------------- O^T += V^T P^T
        if (!more) wait_loads<0>();
        else if (next_fresh) wait_loads<NI + 1 + NQ>();
        else wait_loads<NI + 1>();
        if (__builtin_expect(vis != kFull, false)) {  // values of keys that are not seen: 0 times an infinity or NaN is not 0
            const int own = here(lane);
#pragma unroll
            for (int i = 0; i < TILEB / 1024; ++i) {
                const int at = i * 64 + own;
                if (!((vis >> (at / CPR)) & 1))
                    *reinterpret_cast<rm_u32x4 *>(lds + buf + TILEB + at * 16) = rm_u32x4{0, 0, 0, 0};
            }
            wait_lds();
        }
        if constexpr (BF) {
            typedef __attribute__((address_space(3))) rm_s16x4 lds_s16x4;
            // A matrix instruction takes 32 keys: two fours of a lane, once with the weights' first parts and once with their
            // rests, or where a tile has 16 keys, the one four with both at once.
            constexpr int PAIRS = (NS + 1) / 2, PER = PAIRS * DB / GS;
            const int row = 4 * h4 + (m16 >> 2);
            const uint8_t *v = vt + row * ROWB + (m16 & 3) * 8;
            auto both = [](rm_s16x4 x, rm_s16x4 y) __attribute__((always_inline)) {
                return __builtin_bit_cast(rm_bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
            };
            rm_bf16x8 w[NS == 1 ? 1 : 2][RT][PAIRS];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    rm_s16x4 high[2], rest[2];
                    in_two(s[r][2 * i], high[0], rest[0]);
                    if constexpr (NS == 1) {
                        w[0][r][i] = both(high[0], rest[0]);
                    } else {
                        in_two(s[r][2 * i + 1], high[1], rest[1]);
                        w[0][r][i] = both(high[0], high[1]);
                        w[1][r][i] = both(rest[0], rest[1]);
                    }
                }
#pragma unroll
            for (int g = 0; g < GS; ++g) {
                rm_s16x4 vf[PER][2];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < PER; ++x) {
                    const int i = (g * PER + x) / DB, d = (g * PER + x) % DB;
#pragma unroll
                    for (int j = 0; j < (NS == 1 ? 1 : 2); ++j)
                        vf[x][j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (lds_s16x4 *)(v + 16 * (2 * i + j) * ROWB + (((2 * d) & 15) ^ swz_v(row)) * 16 + (d >> 3) * 256));
                }
                __builtin_amdgcn_sched_barrier(0);
                if (more) stage(next, true, 4 * g, turn);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int part = 0; part < (NS == 1 ? 1 : 2); ++part)
#pragma unroll
                    for (int x = 0; x < PER; ++x) {
                        const int i = (g * PER + x) / DB, d = (g * PER + x) % DB;
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(both(vf[x][0], vf[x][NS == 1 ? 0 : 1]),
                                                                              w[part][r][i], o[r][d], 0, 0, 0);
                    }
            }
        } else {
            constexpr int PER = 4 * NS / GS;  // fours of keys, one of each lane row
#pragma unroll
            for (int g = 0; g < GS; ++g) {
                float vf[PER][DB];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < PER; ++x) {
                    const int row = 16 * ((g * PER + x) / 4) + 4 * h4 + (g * PER + x) % 4;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
                        vf[x][d] = *reinterpret_cast<const float *>(vt + row * ROWB + (((4 * d) & 15) ^ (4 * h4)) * 16 +
                                                                    (d >> 2) * 256 + m16 * 4);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (more) stage(next, true, 4 * g, turn);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < PER; ++x)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int d = 0; d < DB; ++d)
                            o[r][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                vf[x][d], s[r][(g * PER + x) / 4][(g * PER + x) % 4], o[r][d], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);

        // ---------------------------------------------------------------- the token's end, or the share's
        if (!more || next_fresh) {
            const Arguments b = again();
            const bool starts = cur.base >= begin, ends = cur.t + 1 == cur.t1;
            if (starts) {
                // (No more than there are groups, whatever else may write the positions meanwhile.)
                const int parts = min((cur.base + (cur.t1 - cur.t0) - 1) / share, b->groups - 1) - grp + 1;
                if (b->info && b->by_token && unit == 0 && lane == 0) b->info[cur.n] = make_int2(grp, parts);
                if (!ends) end_info = make_int2(cur.n, parts);
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float sum = rows_sum(l[r]);
                const int own = here(lane), g = r * 16 + (own & 15), c0 = 4 * (own >> 4);
                if (g >= heads) continue;
                if (starts && ends) {
                    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                    char *dst = b->o + cur.n * b->o_t + static_cast<int64_t>(hk * b->G + g0 + g) * b->o_h;
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const int c = 16 * d + c0;
                        if (c >= b->D) continue;
                        const rm_f32x4 y = o[r][d] * inv;
                        if constexpr (BF)
                            *reinterpret_cast<rm_bf16x4 *>(dst + c * 2) =
                                rm_bf16x4{static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1]), static_cast<__bf16>(y[2]),
                                          static_cast<__bf16>(y[3])};
                        else
                            *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = y;
                    }
                } else {
                    const int64_t row = ((2 * static_cast<int64_t>(grp) + starts) * b->units + unit) * QR + g;
                    if (c0 == 0) b->part_ml[row] = make_float2(m[r], sum);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const int c = 16 * d + c0;
                        if (c < b->D) *reinterpret_cast<rm_f32x4 *>(b->part_o + row * b->D + c) = o[r][d];
                    }
                }
            }
        }
        if (!more) break;
        cur = nxt;
        nxt = after;
        vis = next.vis;
        fresh = next_fresh;
        --left;
    }
    const Arguments b = again();
    if (b->info && !b->by_token && unit == 0 && lane == 0) b->info[grp] = end_info;
}

// The parts that groups of waves left of a token, joined in a fixed order: `share` lane groups (a power of two) divide the
// parts of one query head, and a workgroup takes as many heads of an entry and unit as it has such.  Bound by three round
// trips (the entry, the parts, the store).
constexpr int kJoinAtOnce = 8;  // parts of a lane group whose loads are in flight together
template <bool BF, int LPR, int QR>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, int share, int blocks) {
    constexpr int GR = 256 / LPR, AT = kJoinAtOnce;
    __shared__ float tops[GR], sums[GR];
    __shared__ rm_f32x4 part[GR][LPR];
    const int eu = blockIdx.x / blocks, block = blockIdx.x - eu * blocks, e = divide(eu, a.by_units), u = eu - e * a.units;
    const int2 info = a.info[e];
    const int parts = info.y, n = a.by_token ? e : info.x, first = a.by_token ? info.x : e;
    if (parts < 2) return;
    const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR, sub = grp & (share - 1);
    const int r = block * (GR / share) + grp / share, hk = divide(u, a.by_q_tiles), g = (u - hk * a.q_tiles) * QR + r;
    const bool is = r < QR && g < a.G;
    auto row = [&](int p) { return ((2 * static_cast<int64_t>(first + p) + (p == 0)) * a.units + u) * QR + r; };
    const int c = min(lane * 4, a.D - 4);
    rm_f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;
    for (int p0 = is ? sub : parts; p0 < parts; p0 += AT * share) {
        float2 ml[AT];
        rm_f32x4 v[AT];
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            ml[i] = make_float2(-INFINITY, 0.0f);
            v[i] = rm_f32x4{};
            if (p0 + i * share < parts) {
                const int64_t at = row(p0 + i * share);
                ml[i] = a.part_ml[at];
                v[i] = *reinterpret_cast<const rm_f32x4 *>(a.part_o + at * a.D + c);
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            top = fmaxf(top, ml[i].x);
        }
        const float ref = top == -INFINITY ? 0.0f : top;
        float f = __builtin_amdgcn_exp2f(m - ref);
        l *= f;
        o *= f;
        m = top;
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            if (ml[i].y == 0.0f) continue;  // (no key with a weight: its sums are zeros)
            f = __builtin_amdgcn_exp2f(ml[i].x - ref);
            l += ml[i].y * f;
            o += v[i] * f;
        }
    }
    if (share > 1) {
        if (lane == 0) tops[grp] = m;
        __syncthreads();
        float top = m;
        for (int i = 0; i < share; ++i) top = fmaxf(top, tops[grp - sub + i]);
        const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
        part[grp][lane] = o * f;
        if (lane == 0) sums[grp] = l * f;
        __syncthreads();
        if (sub != 0) return;
        l = 0.0f;
        o = rm_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = 0; i < share; ++i) {
            l += sums[grp + i];
            o += part[grp + i][lane];
        }
    }
    if (!is || lane * 4 >= a.D) return;
    o *= l == 0.0f ? 0.0f : 1.0f / l;
    char *dst = a.o + n * a.o_t + static_cast<int64_t>(hk * a.G + g) * a.o_h;
    if constexpr (BF)
        *reinterpret_cast<rm_bf16x4 *>(dst + c * 2) = rm_bf16x4{static_cast<__bf16>(o[0]), static_cast<__bf16>(o[1]),
                                                                static_cast<__bf16>(o[2]), static_cast<__bf16>(o[3])};
    else
        *reinterpret_cast<rm_f32x4 *>(dst + c * 4) = o;
}

template <bool BF, int DC, int QR>
hipError_t go(const PagedPlan &p, const PagedArgs &a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(a.groups) * a.units);
    if (p.whole) paged_kernel<BF, true, DC, QR><<<grid, 64, 0, st>>>(a);
    else paged_kernel<BF, false, DC, QR><<<grid, 64, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.join) return e;
    // A token has groups / N parts and two more where it begins and ends, if all are as long; lane groups
    // share them until one has at most four.
    constexpr int LPR = room(DC) / 4, GR = 256 / LPR;
    const int entries = std::min(a.N, a.groups), parts = a.groups / entries + 2;
    int share = 1;
    while (share < GR && share * 4 < parts) share *= 2;
    const int blocks = (a.rows * share + GR - 1) / GR;
    paged_join_kernel<BF, LPR, QR><<<dim3(static_cast<unsigned>(entries) * a.units * blocks), 256, 0, st>>>(a, share, blocks);
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
template <bool BF>
void shape_of(int D, int G, PagedPlan &p) {
    p.qr = G <= 8 ? 8 : G <= 16 ? 16 : 32;
    if (room(D) == 64) shape_of<BF, 64>(p);
    else if (room(D) == 128) shape_of<BF, 128>(p);
    else shape_of<BF, 256>(p);
}

}  // namespace

}  // namespace rm_serve
