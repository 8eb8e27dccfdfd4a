// C ABI entry points of the attention side: argument checks, launch plans and launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <numeric>

#include "rm_attn_plan.h"
#include "rm_checks.h"
#include "rm_rope.h"

#define RM_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using rm::api_fail;
using rm::api_ok;
using namespace rm_checks;

// The head vectors of a tensor of T x H, by byte offsets: `width` bytes at at + i step[0] + j step[1], the steps falling
// (0: no such axis); reach[n]: how far axis n and the later ones go.
struct Vectors {
    int64_t step[3] = {0, 0, 0}, reach[3] = {0, 0, 0};
};
Vectors vectors(const int64_t st[3], int64_t T, int64_t H, int64_t width) {
    Vectors v;
    const bool token_first = st[1] >= st[2];
    v.step[0] = st[token_first ? 1 : 2], v.step[1] = st[token_first ? 2 : 1];
    v.reach[2] = width;
    v.reach[1] = width + ((token_first ? H : T) - 1) * v.step[1];
    v.reach[0] = v.reach[1] + ((token_first ? T : H) - 1) * v.step[0];
    return v;
}

// Whether a's vectors, from axis i on, and b's, from axis j on and `at` bytes further, share no byte.  Of the larger step
// both are taken to repeat endlessly (or stand once); what they repeat fits into a step, so that only two of b's
// places can meet one of a's.  False where that does not decide it.
bool apart(const Vectors &a, int i, const Vectors &b, int j, int64_t at) {
    if (at >= a.reach[i] || at + b.reach[j] <= 0) return true;
    const int64_t step = std::max(a.step[i], b.step[j]);
    if (step == 0) return false;
    i += a.step[i] == step, j += b.step[j] == step;
    if (a.reach[i] > step || b.reach[j] > step) return false;
    const int64_t d = (at % step + step) % step;
    return apart(a, i, b, j, d) && apart(a, i, b, j, d - step);
}

// U groups of `per` samples of T tokens, n0 shared and n1 own keys.
rm_status attn_plan(const rm_attn_shape *s, int U, int per, int T, int n0, int n1, rm_attn::Plan *p) {
    const rm_status st = check_attn_shape(s);
    if (st != RM_OK) return st;
    if (U <= 0 || per <= 0 || T <= 0)
        return api_fail(RM_ERR_INVALID_ARG, "the numbers of samples and of tokens must be positive");
    if (n0 < 0 || n1 < 0 || n0 >= kMaxKeys || n1 >= kMaxKeys)
        return api_fail(RM_ERR_SHAPE, "numbers of keys must be in [0, 2^30)");
    rm_attn::Plan q;
    const int D = s->head_dim, G = s->n_q_heads / s->n_kv_heads;
    const bool bf = s->dtype == RM_BF16;
    const int64_t samples = static_cast<int64_t>(U) * per;
    const __int128 R = static_cast<__int128>(per) * T * G, groups = static_cast<__int128>(U) * s->n_kv_heads;
    if (R >= kMaxKeys || groups >= kMaxKeys || R * groups >= static_cast<__int128>(1) << 40 || samples >= kMaxKeys)
        return api_fail(RM_ERR_SHAPE, "too many query rows");
    const int64_t rows = static_cast<int64_t>(R), ng = static_cast<int64_t>(groups);
    q.dh = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    constexpr int64_t kCUs = 256;
    // Waves that divide 128 rows, or the keys of 32: the former once there are enough blocks of 128 rows.  Measured on
    // 2048 (512) keys, us, the latter / the former: bf16, 128 columns, 128 blocks 31 / 48 (13 / 17), 192 48 / 49
    // (20 / 17), 256 60 / 50 (24 / 18), 512 110 / 77; 64 columns alike; 256 columns (one workgroup to a compute unit)
    // 64 blocks 33 / 69 (14 / 23), 128 66 / 70 (26 / 24), 256 124 / 75.  Float32, 128 columns, 256 blocks 320 / 334
    // (97 / 90), 384 480 / 565, 512 639 / 568; 256 columns have too few registers for it (768 blocks: 1768 / 2841) and
    // waves that divide both.
    const int64_t blocks = ceil_div(rows, 128) * ng;
    bool key_waves = rows <= 32 || (bf ? blocks < (q.dh == 256 ? 128 : 192) : q.dh == 256 || blocks < 2 * kCUs);
    // Blocks that are at most half full: 256 of them (64 rows) on 2048 keys, bf16, 64 columns 26 / 39, 128 51 / 56, 256
    // 124 / 106.
    if (rows <= 64 && q.dh <= 128) key_waves = true;
    // Few blocks on many keys, where slices of the keys fill the compute units either way: bf16, 128 columns, 32 blocks
    // on 8192 keys 39 / 38, on 32768 111 / 89, 64 blocks on 32768 210 / 161; 64 columns, 32 on 8192 28 / 32, on 32768
    // 76 / 66; 256 columns, 8 on 8192 28 / 31, 32 on 8192 66 / 56, on 32768 221 / 156.  (A window that hides most of
    // the keys turns the second, 111 / 89, into 18 / 23: the plan does not know the spans.)
    // 4 (16) blocks of 96 rows on 131072: 64 columns 56 / 54 (166 / 143), 128 97 / 76 (300 / 216), 256 160 / 110
    // (545 / 383); of 64 rows: 64 columns 41 / 55 (130 / 141), 128 60 / 67 (240 / 209), 256 119 / 106 (414 / 381).
    auto keys = [&](int64_t r) {  // read by a block of r rows, which may hold rows of several samples
        return n0 + std::min<int64_t>(per, ceil_div(r, static_cast<int64_t>(T) * G)) * n1;
    };
    const int64_t many = int64_t{1} << (q.dh == 256 ? 18 : q.dh == 128 && rows > 64 ? 19 : 20);
    if (bf && rows > (q.dh == 64 ? 64 : 32) && keys(128) >= ceil_div(many, blocks)) key_waves = false;
    // Own keys that few of a block's rows see pass through all its waves: 1024 (256) single tokens of 8 (4) query heads
    // to a key head on 1024 shared and 64 (256) own keys, bf16, 128 columns 53 / 58 (57 / 90), 64 columns 38 / 48
    // (33 / 73), 256 columns 123 / 88 (116 / 186); float32, 2048 of 8 (4) on 1024 and 64 (256 and 128), 128 columns
    // 511 / 577 (505 / 1225), 64 columns 250 / 286 (247 / 590).
    if (2 * keys(128) > (q.dh == 256 ? 4 : 3) * keys(32)) key_waves = true;
    q.kw = key_waves ? 4 : 1;
    q.rows = key_waves ? (!bf && q.dh == 256 ? 64 : 32) : 128;
    q.n_tiles = static_cast<int>(ceil_div(rows, q.rows));
    const int64_t wgs = q.n_tiles * ng;
    if (wgs >= kMaxGroups) return api_fail(RM_ERR_SHAPE, "launch grid too large");
    // Few row blocks: several workgroups divide the keys, as many as fill the compute units once (two workgroups to
    // one, where their LDS allows it: heads up to 128 in bf16, 64 in float32), if the tiles that each of them then has
    // less pay for the second launch and the partial results.  Measured, us: a tile of 128 keys 0.9, 1.1 and 1.65 in
    // bf16 (rows of 64, 128 and 256 columns), 2.3, 4.1 and 14 in float32, 2.4 times that for 128 rows; the join 5 and
    // its traffic at 4 TB/s (one action chunk's 408 rows on 901 keys, D = 256: 20.2 us undivided, 14.2 in 8 slices;
    // 6528 rows 24.4 undivided, 38.7 in 2).
    // A row block walks the own keys of every sample it has rows of, (t + r - gcd(t, r)) / t of them on average for r
    // rows and t to a sample (32 single tokens of 8 heads on 8, 128 shared and 256 own keys: 65 tiles; one sample's
    // counted for all of them, 3, the call took 91 us undivided, 23 in slices).
    const int64_t t = static_cast<int64_t>(T) * G, own_tiles = ceil_div(n1, 128);
    const int64_t tiles =
        ceil_div(n0, 128) + std::min(per * own_tiles, own_tiles * (t + q.rows - std::gcd(t, int64_t{q.rows})) / t);
    const int64_t slots = kCUs * (q.dh * (bf ? 1 : 2) <= 128 ? 2 : 1);
    const double tile_us =
        (bf ? 0.65 + q.dh / 256.0 : q.dh == 256 ? 14.0 : 0.5 + q.dh / 36.0) * (key_waves ? 1.0 : 2.4);
    const double join_us = 5.0, part_us = static_cast<double>(rows) * ng * D * 8 / 4e6;  // one slice's results
    q.splits = 1;
    double best = tiles * tile_us;
    for (int64_t n = 2; n * wgs <= slots && n <= tiles; n += n < 16 ? 1 : n / 8) {
        const double us = ceil_div(tiles, n) * tile_us + join_us + n * part_us;
        if (us < best) best = us, q.splits = static_cast<int>(n);
    }
    if (q.splits > 1) {
        const size_t n = static_cast<size_t>(q.splits) * ng * rows;
        q.off_ml = align_up(n * D * 4, 256);
        q.total = align_up(q.off_ml + n * 8, 256);
    }
    *p = q;
    return RM_OK;
}

// Runs a planned call: the workspace checks, the kernel and the join of its slices.
rm_status attn_run(const rm_attn_shape *s, const rm_attn::Plan &p, rm_attn::Args &a, const Extent *in, int n_in,
                   const Extent &out, void *ws, size_t ws_bytes, void *stream) {
    if (p.total > 0) {
        if (!ws) return api_fail(RM_ERR_INVALID_ARG, "workspace is NULL");
        if (!aligned(ws, 256)) return api_fail(RM_ERR_ALIGN, "workspace must be 256-byte aligned");
        if (ws_bytes < p.total)
            return api_fail(RM_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", ws_bytes, p.total);
    }
    const Extent w{ws, p.total};
    if (overlap(w, out)) return api_fail(RM_ERR_INVALID_ARG, "the workspace overlaps the output");
    for (int i = 0; i < n_in; ++i)
        if (overlap(in[i], out) || overlap(in[i], w))
            return api_fail(RM_ERR_INVALID_ARG, "the output or the workspace overlaps an input");
    const float log2e = 1.4426950408889634f;
    if (s->softcap > 0.0f) {
        a.cap = s->softcap * log2e;
        a.scale = s->scale / s->softcap;
    } else {
        a.scale = s->scale * log2e;
    }
    a.by_g = rm_attn::divisor(a.G);
    a.by_t = rm_attn::divisor(a.T);
    a.by_hk = rm_attn::divisor(a.Hk);
    a.by_splits = rm_attn::divisor(p.splits);
    a.n_tiles = p.n_tiles;
    a.splits = p.splits;
    const int groups = a.U * a.Hk;
    a.by_xcd = groups % 8 == 0;
    const int of_xcd = a.by_xcd ? groups / 8 : groups;
    a.turns = of_xcd <= 8;
    a.order = a.turns ? of_xcd : p.n_tiles * p.splits;
    a.by_order = rm_attn::divisor(a.order);
    if (p.total > 0) {
        a.part_o = static_cast<float *>(ws);
        a.part_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + p.off_ml);
    }
    const auto hs = static_cast<hipStream_t>(stream);
    const bool bf = s->dtype == RM_BF16;
    hipError_t e = !bf                              ? rm_attn::launch_f32(p, a, hs)
                   : s->softcap <= rm_attn::kLowCap ? rm_attn::launch_bf16(p, a, hs)
                                                    : rm_attn::launch_bf16_high_cap(p, a, hs);
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "attention launch: %s", hipGetErrorString(e));
    if (p.splits > 1) e = rm_attn::launch_combine(bf, a, hs);
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "attention join launch: %s", hipGetErrorString(e));
    return api_ok();
}

}  // namespace

RM_EXPORT rm_status rm_qk_norm_rope(int32_t n_tok, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    int32_t in_dtype, int32_t out_dtype, const rm_heads *q, const rm_heads *k,
                                    const rm_heads *v, const rm_heads *q_out, const rm_heads *k_out,
                                    const rm_heads *v_out, int32_t rows, const int32_t *pos, const int32_t *slot,
                                    const float *inv_freq, int32_t rot, int32_t pairs, const float *gain_q,
                                    const float *gain_k, float eps, void *stream) {
    if (n_tok < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || rows < 0)
        return api_fail(RM_ERR_INVALID_ARG, "n_tok=%d and rows=%d must not be negative, the head counts positive", n_tok, rows);
    if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 256)
        return api_fail(RM_ERR_SHAPE, "head_dim=%d must be a multiple of 8 in [8, 256]", head_dim);
    if (rot < 0 || rot % 4 != 0 || rot > head_dim)
        return api_fail(RM_ERR_SHAPE, "rot=%d must be a multiple of 4 in [0, head_dim=%d]", rot, head_dim);
    if ((in_dtype != RM_F32 && in_dtype != RM_BF16) || (out_dtype != RM_F32 && out_dtype != RM_BF16))
        return api_fail(RM_ERR_DTYPE, "unknown dtype %d or %d", in_dtype, out_dtype);
    if (!(eps >= 0.0f)) return api_fail(RM_ERR_INVALID_ARG, "eps must be >= 0");
    if (!slot && rows < n_tok)
        return api_fail(RM_ERR_SHAPE, "rows=%d hold fewer than the n_tok=%d tokens (no slots given)", rows, n_tok);
    const bool values = v != nullptr && v->data != nullptr;
    const int64_t heads = static_cast<int64_t>(n_q_heads) + n_kv_heads * (values ? 2LL : 1LL);
    if (heads > 65535 || n_tok * heads >= (1LL << 30) || ceil_div(n_tok, 4) >= kMaxGroups)
        return api_fail(RM_ERR_SHAPE, "n_tok x heads = %d x %lld is too large", n_tok, static_cast<long long>(heads));
    const size_t ie = elem(in_dtype), oe = elem(out_dtype);
    Extent x[6];
    int64_t st[6][3] = {};
    rm_status r = check_heads("q", q, 1, n_tok, n_q_heads, head_dim, ie, false, INT64_MAX, &x[0], st[0]);
    if (r == RM_OK) r = check_heads("k", k, 1, n_tok, n_kv_heads, head_dim, ie, false, INT64_MAX, &x[1], st[1]);
    if (r == RM_OK) r = check_heads("q_out", q_out, 1, n_tok, n_q_heads, head_dim, oe, true, INT64_MAX, &x[3], st[3]);
    if (r == RM_OK) r = check_heads("k_out", k_out, 1, rows, n_kv_heads, head_dim, oe, true, INT64_MAX, &x[4], st[4]);
    if (r == RM_OK && values) {
        r = check_heads("v", v, 1, n_tok, n_kv_heads, head_dim, ie, false, INT64_MAX, &x[2], st[2]);
        if (r == RM_OK) r = check_heads("v_out", v_out, 1, rows, n_kv_heads, head_dim, oe, true, INT64_MAX, &x[5], st[5]);
    }
    if (r != RM_OK) return r;
    if (n_tok == 0) return api_ok();
    if (!pos || (rot > 0 && !inv_freq)) return api_fail(RM_ERR_INVALID_ARG, "pos or inv_freq is NULL");
    if (!aligned(pos, 4) || !aligned(slot, 4) || !aligned(inv_freq, 4) || !aligned(gain_q, 4) || !aligned(gain_k, 4))
        return api_fail(RM_ERR_ALIGN, "pos, slot, inv_freq and the gains must be 4-byte aligned");
    const size_t n4 = static_cast<size_t>(n_tok) * 4, g4 = static_cast<size_t>(head_dim) * 4;
    const Extent in[8] = {x[0], x[1], x[2], {pos, n4}, {slot, slot ? n4 : 0},
                          {inv_freq, static_cast<size_t>(rot) * 2}, {gain_q, gain_q ? g4 : 0}, {gain_k, gain_k ? g4 : 0}};
    const int64_t width = static_cast<int64_t>(head_dim) * static_cast<int64_t>(oe);
    const Vectors out[3] = {vectors(st[3], n_tok, n_q_heads, width), vectors(st[4], rows, n_kv_heads, width),
                            vectors(st[5], rows, n_kv_heads, width)};
    for (int o = 3; o < 6; ++o)
        for (int p = o + 1; p < 6; ++p)
            if (overlap(x[o], x[p]) && !apart(out[o - 3], 0, out[p - 3], 0,
                                              static_cast<int64_t>(reinterpret_cast<uintptr_t>(x[p].p) -
                                                                   reinterpret_cast<uintptr_t>(x[o].p))))
                return api_fail(RM_ERR_INVALID_ARG, "the outputs overlap each other");
    for (int o = 3; o < 6; ++o)
        for (const Extent &i : in)
            if (overlap(i, x[o])) return api_fail(RM_ERR_INVALID_ARG, "an output overlaps an input");
    rm::RopeArgs a;
    a.q = static_cast<const char *>(q->data);
    a.k = static_cast<const char *>(k->data);
    a.v = values ? static_cast<const char *>(v->data) : nullptr;
    a.q_t = st[0][1], a.q_h = st[0][2], a.k_t = st[1][1], a.k_h = st[1][2];
    a.q_out = static_cast<char *>(q_out->data);
    a.k_out = static_cast<char *>(k_out->data);
    a.qo_t = st[3][1], a.qo_h = st[3][2], a.ko_t = st[4][1], a.ko_h = st[4][2];
    if (values) {
        a.v_t = st[2][1], a.v_h = st[2][2];
        a.v_out = static_cast<char *>(v_out->data);
        a.vo_t = st[5][1], a.vo_h = st[5][2];
    }
    a.pos = pos, a.slot = slot, a.inv_freq = inv_freq, a.gain_q = gain_q, a.gain_k = gain_k;
    a.N = n_tok, a.D = head_dim, a.Hq = n_q_heads, a.Hk = n_kv_heads, a.H = static_cast<int>(heads);
    a.rot = rot, a.rows = rows, a.pairs = pairs != 0, a.eps = eps;
    const hipError_t e = rm::launch_qk_norm_rope(a, in_dtype == RM_BF16, out_dtype == RM_BF16,
                                                 static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "norm and rotation launch: %s", hipGetErrorString(e));
    return api_ok();
}

RM_EXPORT rm_status rm_attn_spans(int32_t B, int32_t T, int32_t N, int32_t causal, int32_t window,
                                  const int32_t *q_start, const int32_t *kv_len, const int32_t *prefix_len,
                                  const int32_t *doc, int32_t *span, void *stream) {
    if (B <= 0 || T <= 0 || N <= 0) return api_fail(RM_ERR_INVALID_ARG, "B=%d, T=%d and N=%d must be positive", B, T, N);
    if (N >= kMaxKeys || T >= kMaxKeys) return api_fail(RM_ERR_SHAPE, "T=%d and N=%d must be below 2^30", T, N);
    if (window < 0) return api_fail(RM_ERR_INVALID_ARG, "window=%d must not be negative", window);
    if (prefix_len && !causal) return api_fail(RM_ERR_INVALID_ARG, "prefix_len is given without causal");
    if (!span) return api_fail(RM_ERR_INVALID_ARG, "span is NULL");
    if (!aligned(q_start, 4) || !aligned(kv_len, 4) || !aligned(prefix_len, 4) || !aligned(doc, 4) || !aligned(span, 8))
        return api_fail(RM_ERR_ALIGN, "span must be 8-byte and the other pointers 4-byte aligned");
    if (ceil_div(T, 256) * B >= kMaxGroups) return api_fail(RM_ERR_SHAPE, "launch grid too large");
    const size_t b4 = static_cast<size_t>(B) * 4;
    const Extent out{span, static_cast<size_t>(B) * T * 8};
    const Extent in[4] = {{q_start, q_start ? b4 : 0}, {kv_len, kv_len ? b4 : 0}, {prefix_len, prefix_len ? b4 : 0},
                          {doc, doc ? b4 * N : 0}};
    for (const Extent &i : in)
        if (overlap(i, out)) return api_fail(RM_ERR_INVALID_ARG, "span overlaps an input");
    const hipError_t e = rm::launch_attn_spans(B, T, N, causal, window, q_start, kv_len, prefix_len, doc, span,
                                               static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "span launch: %s", hipGetErrorString(e));
    return api_ok();
}

RM_EXPORT rm_status rm_span_attention_workspace_size(const rm_attn_shape *s, int32_t B, int32_t T, int32_t N,
                                                     size_t *bytes) {
    if (!bytes) return api_fail(RM_ERR_INVALID_ARG, "bytes is NULL");
    rm_attn::Plan p;
    const rm_status st = attn_plan(s, B, 1, T, 0, N, &p);
    if (st != RM_OK) return st;
    *bytes = p.total;
    return api_ok();
}

RM_EXPORT rm_status rm_span_attention(const rm_attn_shape *s, int32_t B, int32_t T, int32_t N, const rm_heads *q,
                                      const rm_heads *k, const rm_heads *v, const rm_heads *out, const int32_t *span,
                                      const float *slopes, const int32_t *q_start, void *ws, size_t ws_bytes,
                                      void *stream) {
    rm_attn::Plan p;
    rm_status r = attn_plan(s, B, 1, T, 0, N, &p);
    if (r != RM_OK) return r;
    const int D = s->head_dim;
    const size_t es = elem(s->dtype);
    Extent x[4];
    int64_t st[4][3] = {};
    r = check_heads("q", q, B, T, s->n_q_heads, D, es, false, INT64_MAX, &x[0], st[0]);
    if (r == RM_OK) r = check_heads("k", k, B, N, s->n_kv_heads, D, es, false, kMaxTokenBytes, &x[1], st[1]);
    if (r == RM_OK) r = check_heads("v", v, B, N, s->n_kv_heads, D, es, false, kMaxTokenBytes, &x[2], st[2]);
    if (r == RM_OK) r = check_heads("out", out, B, T, s->n_q_heads, D, es, true, INT64_MAX, &x[3], st[3]);
    if (r != RM_OK) return r;
    if (!aligned(span, 8) || !aligned(slopes, 4) || !aligned(q_start, 4))
        return api_fail(RM_ERR_ALIGN, "span must be 8-byte, slopes and q_start 4-byte aligned");
    rm_attn::Args a;
    a.q = static_cast<const char *>(q->data);
    a.q_b = st[0][0], a.q_t = st[0][1], a.q_h = st[0][2];
    a.o = static_cast<char *>(out->data);
    a.o_b = st[3][0], a.o_t = st[3][1], a.o_h = st[3][2];
    a.s1.k = static_cast<const char *>(k->data), a.s1.v = static_cast<const char *>(v->data);
    a.s1.k_b = st[1][0], a.s1.k_n = st[1][1], a.s1.k_h = st[1][2];
    a.s1.v_b = st[2][0], a.s1.v_n = st[2][1], a.s1.v_h = st[2][2];
    a.n1 = N;
    a.span = span, a.slopes = slopes, a.q_start = slopes ? q_start : nullptr;
    a.D = D, a.Hk = s->n_kv_heads, a.G = s->n_q_heads / s->n_kv_heads, a.T = T, a.per = 1, a.U = B;
    a.R = T * a.G;
    const Extent in[6] = {x[0], x[1], x[2], {span, span ? static_cast<size_t>(B) * T * 8 : 0},
                          {slopes, slopes ? static_cast<size_t>(s->n_q_heads) * 4 : 0},
                          {q_start, slopes && q_start ? static_cast<size_t>(B) * 4 : 0}};
    return attn_run(s, p, a, in, 6, x[3], ws, ws_bytes, stream);
}

RM_EXPORT rm_status rm_prefix_attention_workspace_size(const rm_attn_shape *s, int32_t n_groups, int32_t per_group,
                                                       int32_t T, int32_t P, int32_t S, size_t *bytes) {
    if (!bytes) return api_fail(RM_ERR_INVALID_ARG, "bytes is NULL");
    rm_attn::Plan p;
    const rm_status st = attn_plan(s, n_groups, per_group, T, P, S, &p);
    if (st != RM_OK) return st;
    *bytes = p.total;
    return api_ok();
}

RM_EXPORT rm_status rm_prefix_attention(const rm_attn_shape *s, int32_t n_groups, int32_t per_group, int32_t T,
                                        int32_t P, int32_t S, const rm_heads *q, const rm_heads *k_prefix,
                                        const rm_heads *v_prefix, const int32_t *prefix_len, const rm_heads *k_own,
                                        const rm_heads *v_own, const int32_t *own_len, int32_t causal,
                                        const rm_heads *out, void *ws, size_t ws_bytes, void *stream) {
    rm_attn::Plan p;
    rm_status r = attn_plan(s, n_groups, per_group, T, P, S, &p);
    if (r != RM_OK) return r;
    const int D = s->head_dim, hk = s->n_kv_heads;
    const int64_t B = static_cast<int64_t>(n_groups) * per_group;
    const size_t es = elem(s->dtype);
    Extent x[6];
    int64_t st[6][3] = {};
    r = check_heads("q", q, B, T, s->n_q_heads, D, es, false, INT64_MAX, &x[0], st[0]);
    if (r == RM_OK) r = check_heads("k_prefix", k_prefix, n_groups, P, hk, D, es, false, kMaxTokenBytes, &x[1], st[1]);
    if (r == RM_OK) r = check_heads("v_prefix", v_prefix, n_groups, P, hk, D, es, false, kMaxTokenBytes, &x[2], st[2]);
    if (r == RM_OK) r = check_heads("k_own", k_own, B, S, hk, D, es, false, kMaxTokenBytes, &x[3], st[3]);
    if (r == RM_OK) r = check_heads("v_own", v_own, B, S, hk, D, es, false, kMaxTokenBytes, &x[4], st[4]);
    if (r == RM_OK) r = check_heads("out", out, B, T, s->n_q_heads, D, es, true, INT64_MAX, &x[5], st[5]);
    if (r != RM_OK) return r;
    if (!aligned(prefix_len, 4) || !aligned(own_len, 4))
        return api_fail(RM_ERR_ALIGN, "prefix_len and own_len must be 4-byte aligned");
    rm_attn::Args a;
    a.q = static_cast<const char *>(q->data);
    a.q_b = st[0][0], a.q_t = st[0][1], a.q_h = st[0][2];
    a.o = static_cast<char *>(out->data);
    a.o_b = st[5][0], a.o_t = st[5][1], a.o_h = st[5][2];
    a.s0.k = static_cast<const char *>(k_prefix->data), a.s0.v = static_cast<const char *>(v_prefix->data);
    a.s0.k_b = st[1][0], a.s0.k_n = st[1][1], a.s0.k_h = st[1][2];
    a.s0.v_b = st[2][0], a.s0.v_n = st[2][1], a.s0.v_h = st[2][2];
    a.s1.k = static_cast<const char *>(k_own->data), a.s1.v = static_cast<const char *>(v_own->data);
    a.s1.k_b = st[3][0], a.s1.k_n = st[3][1], a.s1.k_h = st[3][2];
    a.s1.v_b = st[4][0], a.s1.v_n = st[4][1], a.s1.v_h = st[4][2];
    a.len0 = prefix_len, a.len1 = own_len, a.n0 = P, a.n1 = S;
    a.D = D, a.Hk = hk, a.G = s->n_q_heads / hk, a.T = T, a.per = per_group, a.U = n_groups, a.causal = causal != 0;
    a.R = per_group * T * a.G;
    const Extent in[7] = {x[0], x[1], x[2], x[3], x[4],
                          {prefix_len, prefix_len ? static_cast<size_t>(n_groups) * 4 : 0},
                          {own_len, own_len ? static_cast<size_t>(B) * 4 : 0}};
    return attn_run(s, p, a, in, 7, x[5], ws, ws_bytes, stream);
}
