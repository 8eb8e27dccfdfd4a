// Launch plan and kernel arguments of the attention calls, shared by the host code and the kernels.
#pragma once

#include <type_traits>

#include "rm_internal.h"

namespace rm_attn {

// One source of keys and values (strides in bytes).
struct Src {
    const char *k = nullptr, *v = nullptr;
    int64_t k_b = 0, k_n = 0, k_h = 0, v_b = 0, v_n = 0, v_h = 0;
};

// n / d for 0 <= n < 2^30: the high half of n mul, shifted (mul = 0: d = 1).  mul = ceil(2^(32 + shift) / d) with
// shift = max(0, ceil(log2 d) - 2) fits 32 bits and is off by less than d, which n < 2^30 keeps below one d-th.
struct Divisor {
    uint32_t mul = 0, shift = 0;
};
inline Divisor divisor(uint32_t d) {
    Divisor r;
    if (d <= 1) return r;
    uint32_t log = 0;
    while ((1ull << log) < d) ++log;
    r.shift = log > 2 ? log - 2 : 0;
    r.mul = static_cast<uint32_t>(((1ull << (32 + r.shift)) + d - 1) / d);
    return r;
}

// Up to this cap bf16 scores are capped through 1 / (1 + e^2x), whose error is one of the cap's size, at most 16
// roundings of it: 0.00024 at 256, a sixteenth of a weight's rounding to bf16.  Above it the tanh is as exact as the
// score, for a fifth to two fifths of a call's time (8192 rows on 8192 keys, 16 heads on 4: 64 columns 517 / 723 us, 128
// 671 / 807, 256 1275 / 1720).
constexpr float kLowCap = 256.0f;

struct Args {
    const char *q = nullptr;
    int64_t q_b = 0, q_t = 0, q_h = 0;  // bytes
    char *o = nullptr;
    int64_t o_b = 0, o_t = 0, o_h = 0;
    Src s0;                         // keys shared by a group's samples ([U] groups), seen by every row
    Src s1;                         // each sample's own keys
    const int32_t *len0 = nullptr;  // [U] or null: n0
    const int32_t *len1 = nullptr;  // [U per] or null: n1
    int n0 = 0, n1 = 0;
    const int32_t *span = nullptr;  // [U][T][2] own keys that a row sees (per = 1), or null
    const float *slopes = nullptr;  // [Hq] or null
    const int32_t *q_start = nullptr;
    int D = 0, Hk = 0, G = 0, T = 0, per = 0, U = 0, causal = 0;
    Divisor by_g, by_t, by_hk, by_splits;  // G, T, Hk and splits
    // The workgroups' order over the groups and key heads (of an XCD, by_xcd): by turns, or one after the other;
    // order: how many of them there are, or how many workgroups each has.
    int by_xcd = 0, turns = 0, order = 1;
    Divisor by_order;
    int R = 0;                      // rows of a group and key head: per T G
    int n_tiles = 0, splits = 1;    // row blocks, and workgroups that divide one's keys
    // Scores times scale in powers of two; with a cap: scale = score scale / cap, cap in powers of two.
    float scale = 0.0f, cap = 0.0f;
    float *part_o = nullptr, *part_ml = nullptr;  // [splits][U Hk][R][D] and [..][2], with splits > 1
};

struct Plan {
    int dh = 0;         // columns of a row in LDS (64, 128, 256)
    int kw = 1;         // key waves: 1 or several
    int rows = 0;       // rows of a workgroup
    int n_tiles = 0, splits = 1;
    size_t off_ml = 0, total = 0;
};

hipError_t launch_bf16(const Plan &p, const Args &a, hipStream_t st);
hipError_t launch_bf16_high_cap(const Plan &p, const Args &a, hipStream_t st);
hipError_t launch_f32(const Plan &p, const Args &a, hipStream_t st);
hipError_t launch_combine(bool bf16, const Args &a, hipStream_t st);

}  // namespace rm_attn
