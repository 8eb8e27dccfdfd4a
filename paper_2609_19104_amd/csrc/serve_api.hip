// C ABI entry points of the serving step: slot maps, paged attention, block norm.
#include "rm_checks.h"
#include "rm_serve.h"

#define RM_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using rm::api_fail;
using rm::api_ok;
using namespace rm_checks;

// Whether every output is apart from every input and from the other outputs.
rm_status check_apart(const Extent *in, int n_in, const Extent *out, int n_out) {
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (overlap(out[i], in[j])) return api_fail(RM_ERR_INVALID_ARG, "an output overlaps an input");
        for (int j = i + 1; j < n_out; ++j)
            if (overlap(out[i], out[j])) return api_fail(RM_ERR_INVALID_ARG, "the outputs overlap each other");
    }
    return RM_OK;
}

// A cache of n_pages pages of `page` rows, and tables of max_pages pages.
rm_status check_pages(int page, int n_pages, int max_pages) {
    if (page <= 0 || n_pages <= 0 || max_pages <= 0)
        return api_fail(RM_ERR_INVALID_ARG, "page=%d, n_pages=%d and max_pages=%d must be positive", page, n_pages, max_pages);
    if (static_cast<int64_t>(n_pages) * page > INT32_MAX)
        return api_fail(RM_ERR_SHAPE, "n_pages x page = %d x %d rows are more than 2^31 - 1", n_pages, page);
    if (static_cast<int64_t>(max_pages) * page >= kMaxKeys)
        return api_fail(RM_ERR_SHAPE, "max_pages x page = %d x %d tokens are not below 2^30", max_pages, page);
    return RM_OK;
}

// Up to this many tiles one group has them all and no join follows (one token on 128 keys, 8 heads of 64 columns on 1, 6.2 us
// in a graph, in three groups 8.6).  Above, a tile a group pays (one token on 1024 keys, 8 heads of 64 columns on 8: a tile each
// 8.2, two each 10.4, four 14).  All before the weights' second part, which adds 0.1 to 0.2.
constexpr int64_t kOneGroup = 4;

rm_status paged_plan(const rm_attn_shape *s, int n_tok, int page, int max_pages, rm_serve::PagedPlan *p) {
    rm_status r = check_attn_shape(s);
    if (r == RM_OK) r = check_pages(page, 1, max_pages);
    if (r != RM_OK) return r;
    if (n_tok <= 0) return api_fail(RM_ERR_INVALID_ARG, "n_tok=%d must be positive", n_tok);
    if (static_cast<int64_t>(n_tok) * s->n_q_heads >= kMaxGroups)
        return api_fail(RM_ERR_SHAPE, "n_tok x n_q_heads = %d x %d is not below 2^24", n_tok, s->n_q_heads);
    const int G = s->n_q_heads / s->n_kv_heads;
    s->dtype == RM_BF16 ? rm_serve::paged_shape_bf16(s->head_dim, G, p) : rm_serve::paged_shape_f32(s->head_dim, G, p);
    p->q_tiles = static_cast<int>(ceil_div(G, p->qr));
    p->units = s->n_kv_heads * p->q_tiles;
    const int64_t most = n_tok * (ceil_div(static_cast<int64_t>(max_pages) * page, p->kt) + 1);  // tiles, at most
    if (most >= (1 << 30) - 2048)
        return api_fail(RM_ERR_SHAPE, "%lld tiles of keys are not below 2^30 - 2048", static_cast<long long>(most));
    // As many groups as fill 256 compute units once.
    const int64_t fill = std::max(1, 256 * p->per_cu / p->units);
    p->groups = most <= kOneGroup ? 1 : static_cast<int>(std::min(fill, most));
    p->by_token = n_tok <= p->groups;
    p->join = p->groups > 1;
    if (!p->join) return RM_OK;  // every token is one wave's
    const size_t rows = static_cast<size_t>(p->groups) * 2 * p->units * p->qr;
    p->off_ml = align_up(rows * s->head_dim * 4, 256);
    p->off_info = align_up(p->off_ml + rows * 8, 256);
    p->total = align_up(p->off_info + static_cast<size_t>(std::min(n_tok, p->groups)) * 8, 256);
    return RM_OK;
}

}  // namespace

RM_EXPORT rm_status rm_page_slots(int32_t n_seqs, int32_t max_tok, int32_t page, int32_t n_pages, int32_t max_pages,
                                  const int32_t *n_new, const int32_t *len, const int32_t *n_free, int32_t *table,
                                  int32_t *free_pages, int32_t *len_out, int32_t *n_free_out, int32_t *refused,
                                  int32_t *first, int32_t *start, int32_t *seq, int32_t *pos, int32_t *slot,
                                  void *stream) {
    if (n_seqs <= 0 || max_tok <= 0)
        return api_fail(RM_ERR_INVALID_ARG, "n_seqs=%d and max_tok=%d must be positive", n_seqs, max_tok);
    if (n_seqs > 1 << 20 || max_tok >= 1 << 30)
        return api_fail(RM_ERR_SHAPE, "n_seqs=%d is more than 2^20 or max_tok=%d not below 2^30", n_seqs, max_tok);
    const rm_status r = check_pages(page, n_pages, max_pages);
    if (r != RM_OK) return r;
    if (n_pages >= 1 << 30) return api_fail(RM_ERR_SHAPE, "n_pages=%d is not below 2^30", n_pages);
    const size_t b4 = static_cast<size_t>(n_seqs) * 4, t4 = static_cast<size_t>(max_tok) * 4;
    const Extent in[3] = {{n_new, b4}, {len, b4}, {n_free, 4}};
    const size_t p4 = static_cast<size_t>(n_pages) * 4;
    const Extent out[10] = {{len_out, b4}, {n_free_out, 4}, {table, b4 * max_pages}, {free_pages, p4}, {first, b4 + 4},
                            {start, b4}, {seq, t4}, {pos, t4}, {slot, t4}, {refused, refused ? 4u : 0u}};
    for (const Extent &e : in)
        if (!e.p) return api_fail(RM_ERR_INVALID_ARG, "n_new, len or n_free is NULL");
    for (const Extent &e : out)
        if (!e.p && e.n) return api_fail(RM_ERR_INVALID_ARG, "an output is NULL");
    for (const Extent &e : in)
        if (!aligned(e.p, 4)) return api_fail(RM_ERR_ALIGN, "every pointer must be 4-byte aligned");
    for (const Extent &e : out)
        if (!aligned(e.p, 4)) return api_fail(RM_ERR_ALIGN, "every pointer must be 4-byte aligned");
    // len_out may be len and n_free_out n_free: each thread reads its own first, the one count is read before the end.
    Extent rest[3] = {in[0], in[1], in[2]};
    if (len_out == len) rest[1].n = 0;
    if (n_free_out == n_free) rest[2].n = 0;
    const rm_status o = check_apart(rest, 3, out, 10);
    if (o != RM_OK) return o;
    rm_serve::SlotArgs a;
    a.B = n_seqs, a.max_tok = max_tok, a.page = page, a.n_pages = n_pages, a.per = max_pages;
    a.by_page = rm_attn::divisor(page);
    a.n_new = n_new, a.len = len, a.n_free = n_free, a.table = table, a.free_pages = free_pages;
    a.len_out = len_out, a.n_free_out = n_free_out, a.refused = refused;
    a.first = first, a.start = start, a.seq = seq, a.pos = pos, a.slot = slot;
    a.in_place = len_out == len || n_free_out == n_free;
    const hipError_t e = rm_serve::launch_page_slots(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "page slots launch: %s", hipGetErrorString(e));
    return api_ok();
}

RM_EXPORT rm_status rm_paged_attention_workspace_size(const rm_attn_shape *s, int32_t n_tok, int32_t page,
                                                      int32_t max_pages, size_t *bytes) {
    if (!bytes) return api_fail(RM_ERR_INVALID_ARG, "bytes is NULL");
    rm_serve::PagedPlan p;
    const rm_status r = paged_plan(s, n_tok, page, max_pages, &p);
    if (r != RM_OK) return r;
    *bytes = p.total;
    return api_ok();
}

RM_EXPORT rm_status rm_paged_attention(const rm_attn_shape *s, int32_t n_tok, int32_t n_seqs, int32_t page,
                                       int32_t n_pages, int32_t max_pages, const rm_heads *q, const rm_heads *k,
                                       const rm_heads *v, const rm_heads *out, const int32_t *table,
                                       const int32_t *seq, const int32_t *pos, int32_t window, const float *slopes,
                                       void *ws, size_t ws_bytes, void *stream) {
    rm_serve::PagedPlan p;
    rm_status r = paged_plan(s, n_tok, page, max_pages, &p);
    if (r == RM_OK) r = check_pages(page, n_pages, max_pages);
    if (r != RM_OK) return r;
    if (n_seqs <= 0) return api_fail(RM_ERR_INVALID_ARG, "n_seqs=%d must be positive", n_seqs);
    if (!seq && n_seqs < n_tok)
        return api_fail(RM_ERR_SHAPE, "n_seqs=%d tables are fewer than the n_tok=%d tokens (no seq given)", n_seqs, n_tok);
    if (window < 0) return api_fail(RM_ERR_INVALID_ARG, "window=%d must not be negative", window);
    const int D = s->head_dim;
    const size_t es = elem(s->dtype);
    Extent x[4];
    int64_t st[4][3] = {};
    r = check_heads("q", q, 1, n_tok, s->n_q_heads, D, es, false, INT64_MAX, &x[0], st[0]);
    if (r == RM_OK) r = check_heads("k", k, n_pages, page, s->n_kv_heads, D, es, false, INT64_MAX, &x[1], st[1]);
    if (r == RM_OK) r = check_heads("v", v, n_pages, page, s->n_kv_heads, D, es, false, INT64_MAX, &x[2], st[2]);
    if (r == RM_OK) r = check_heads("out", out, 1, n_tok, s->n_q_heads, D, es, true, INT64_MAX, &x[3], st[3]);
    if (r != RM_OK) return r;
    if (!table || !pos) return api_fail(RM_ERR_INVALID_ARG, "table or pos is NULL");
    if (!aligned(table, 4) || !aligned(pos, 4) || !aligned(seq, 4) || !aligned(slopes, 4))
        return api_fail(RM_ERR_ALIGN, "table, seq, pos and slopes must be 4-byte aligned");
    const size_t n4 = static_cast<size_t>(n_tok) * 4;
    const Extent in[7] = {x[0], x[1], x[2], {table, static_cast<size_t>(n_seqs) * max_pages * 4}, {seq, seq ? n4 : 0},
                          {pos, n4}, {slopes, slopes ? static_cast<size_t>(s->n_q_heads) * 4 : 0}};
    if (p.total > 0) {
        if (!ws) return api_fail(RM_ERR_INVALID_ARG, "workspace is NULL");
        if (!aligned(ws, 256)) return api_fail(RM_ERR_ALIGN, "workspace must be 256-byte aligned");
        if (ws_bytes < p.total)
            return api_fail(RM_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", ws_bytes, p.total);
    }
    const Extent written[2] = {x[3], {ws, p.total}};
    r = check_apart(in, 7, written, 2);
    if (r != RM_OK) return r;
    rm_serve::PagedArgs a;
    a.q = static_cast<const char *>(q->data), a.k = static_cast<const char *>(k->data);
    a.v = static_cast<const char *>(v->data), a.o = static_cast<char *>(out->data);
    a.q_t = st[0][1], a.q_h = st[0][2], a.o_t = st[3][1], a.o_h = st[3][2];
    a.k_p = st[1][0], a.k_t = st[1][1], a.k_h = st[1][2];
    a.v_p = st[2][0], a.v_t = st[2][1], a.v_h = st[2][2];
    a.table = table, a.seq = seq, a.pos = pos, a.slopes = slopes;
    a.N = n_tok, a.seqs = n_seqs, a.page = page, a.n_pages = n_pages, a.per = max_pages, a.window = window;
    a.D = D, a.G = s->n_q_heads / s->n_kv_heads;
    a.units = p.units, a.q_tiles = p.q_tiles, a.rows = std::min(a.G, p.qr);
    a.by_page = rm_attn::divisor(page), a.by_q_tiles = rm_attn::divisor(p.q_tiles);
    a.by_units = rm_attn::divisor(p.units), a.by_groups = rm_attn::divisor(p.groups);
    a.groups = p.groups, a.by_token = p.by_token;
    // (An instruction's rows from its first one in 32 bits, and rows of the cache in 32 bits of 16 bytes each.)
    const size_t wide = size_t{16} << 32;
    p.whole = page % p.rpi == 0 && a.k_t < 1 << 28 && a.v_t < 1 << 28 && x[1].n < wide && x[2].n < wide;
    if (p.total > 0) {
        a.part_o = static_cast<float *>(ws);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + p.off_ml);
        a.info = reinterpret_cast<int2 *>(static_cast<char *>(ws) + p.off_info);
    }
    const float log2e = 1.4426950408889634f;
    if (s->softcap > 0.0f) {
        a.cap = s->softcap * log2e;
        a.scale = s->scale / s->softcap;
    } else {
        a.scale = s->scale * log2e;
    }
    const auto hs = static_cast<hipStream_t>(stream);
    const hipError_t e = s->dtype == RM_BF16 ? rm_serve::launch_paged_bf16(p, a, hs) : rm_serve::launch_paged_f32(p, a, hs);
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "paged attention launch: %s", hipGetErrorString(e));
    return api_ok();
}

RM_EXPORT rm_status rm_block_norm(int32_t B, int32_t T, int32_t d, int32_t x_dtype, int32_t f_dtype,
                                  int32_t out_dtype, const void *x, const void *f, int32_t norm_post,
                                  const float *gain_post, const float *gate, int64_t gate_stride, float x_scale,
                                  float f_scale, void *y, const float *gain_pre, const float *scale,
                                  int64_t scale_stride, const float *shift, int64_t shift_stride, float eps, void *out,
                                  void *stream) {
    if (B <= 0 || T <= 0 || d <= 0) return api_fail(RM_ERR_INVALID_ARG, "B=%d, T=%d and d=%d must be positive", B, T, d);
    if (d % 8 != 0 || d > 32768) return api_fail(RM_ERR_SHAPE, "d=%d must be a multiple of 8 of at most 32768", d);
    const int64_t rows = static_cast<int64_t>(B) * T;
    if (rows >= kMaxGroups) return api_fail(RM_ERR_SHAPE, "B x T = %d x %d rows are not below 2^24", B, T);
    for (int t : {x_dtype, f_dtype, out_dtype})
        if (t != RM_F32 && t != RM_BF16) return api_fail(RM_ERR_DTYPE, "unknown dtype %d", t);
    if (!x) return api_fail(RM_ERR_INVALID_ARG, "x is NULL");
    if (!y && !out) return api_fail(RM_ERR_INVALID_ARG, "y and out are NULL");
    if (!f && (norm_post || gain_post || gate)) return api_fail(RM_ERR_INVALID_ARG, "norm_post, gain_post or gate without f");
    if (gain_post && !norm_post) return api_fail(RM_ERR_INVALID_ARG, "gain_post without norm_post");
    if (!out && (gain_pre || scale || shift)) return api_fail(RM_ERR_INVALID_ARG, "gain_pre, scale or shift without out");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return api_fail(RM_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (!std::isfinite(x_scale) || !std::isfinite(f_scale))
        return api_fail(RM_ERR_INVALID_ARG, "x_scale and f_scale must be finite");
    struct Mod {
        const char *name;
        const float *p;
        int64_t stride;
    };
    const Mod mod[3] = {{"gate", gate, gate_stride}, {"scale", scale, scale_stride}, {"shift", shift, shift_stride}};
    const size_t xe = elem(x_dtype), fe = elem(f_dtype), oe = elem(out_dtype), n = static_cast<size_t>(rows) * d;
    for (const void *p : {x, f, static_cast<const void *>(y), static_cast<const void *>(out)})
        if (!aligned(p, 16)) return api_fail(RM_ERR_ALIGN, "x, f, y and out must be 16-byte aligned");
    for (const float *p : {gain_post, gain_pre, gate, scale, shift})
        if (!aligned(p, 16)) return api_fail(RM_ERR_ALIGN, "gains, gate, scale and shift must be 16-byte aligned");
    const size_t d4 = static_cast<size_t>(d) * 4;
    Extent in[7] = {{x, n * xe}, {f, f ? n * fe : 0}, {gain_post, gain_post ? d4 : 0}, {gain_pre, gain_pre ? d4 : 0}};
    int64_t stride[3] = {0, 0, 0};
    for (int i = 0; i < 3; ++i) {
        if (!mod[i].p) continue;
        if (B > 1) {
            if (mod[i].stride < 0 || mod[i].stride > INT64_MAX / 16 / B)
                return api_fail(RM_ERR_SHAPE, "%s: a stride of %lld elements", mod[i].name,
                                static_cast<long long>(mod[i].stride));
            if (mod[i].stride % 4 != 0)
                return api_fail(RM_ERR_ALIGN, "%s: its stride must be a multiple of 16 bytes", mod[i].name);
            stride[i] = mod[i].stride;
        }
        in[4 + i] = {mod[i].p, static_cast<size_t>(stride[i]) * (B - 1) * 4 + d4};
    }
    // Every element of y and out is written by the lane that has read x's and f's in its place: y may be x, and out may
    // be f of the same type.
    const Extent yo{y, y ? n * xe : 0}, oo{out, out ? n * oe : 0};
    if (overlap(yo, oo)) return api_fail(RM_ERR_INVALID_ARG, "the outputs overlap each other");
    for (int i = 0; i < 7; ++i) {
        if (overlap(yo, in[i]) && !(i == 0 && y == x)) return api_fail(RM_ERR_INVALID_ARG, "y overlaps an input");
        if (overlap(oo, in[i]) && !(i == 1 && out == f && out_dtype == f_dtype))
            return api_fail(RM_ERR_INVALID_ARG, "out overlaps an input");
    }
    rm_serve::NormArgs a;
    a.x = static_cast<const char *>(x), a.f = static_cast<const char *>(f);
    a.y = static_cast<char *>(y), a.out = static_cast<char *>(out);
    a.gain_post = gain_post, a.gate = gate, a.gain_pre = gain_pre, a.scale = scale, a.shift = shift;
    a.gate_b = stride[0], a.scale_b = stride[1], a.shift_b = stride[2];
    a.rows = rows, a.T = T, a.d = d, a.norm_post = norm_post != 0;
    a.x_scale = x_scale, a.f_scale = f_scale, a.eps = eps;
    const hipError_t e = rm_serve::launch_block_norm(a, x_dtype == RM_BF16, f_dtype == RM_BF16, out_dtype == RM_BF16,
                                                     static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return api_fail(RM_ERR_HIP, "block norm launch: %s", hipGetErrorString(e));
    return api_ok();
}
