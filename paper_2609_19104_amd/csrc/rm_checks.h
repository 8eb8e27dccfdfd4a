// Argument checks shared by the entry points of the attention side and of the serving step.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "rm_internal.h"

namespace rm_checks {

using rm::api_fail;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t elem(int dtype) { return dtype == RM_BF16 ? 2 : 4; }

constexpr int kMaxKeys = 1 << 30;
constexpr int64_t kMaxGroups = 1 << 24;  // workgroups of 256 threads: a launch holds below 2^32 threads

struct Extent {
    const void *p = nullptr;
    size_t n = 0;
};
inline bool overlap(const Extent &a, const Extent &b) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    return a.n != 0 && b.n != 0 && pa < pb + b.n && pb < pa + a.n;
}

constexpr int64_t kMaxTokenBytes = 16 << 20;

// Checks one tensor of B x T x H head vectors of D elements of `es` bytes; gives its extent and its strides in bytes
// (0 for axes of size 1).  out: its elements must be distinct.  max_token: bound of the token stride in bytes.
inline rm_status check_heads(const char *name, const rm_heads *t, int64_t B, int64_t T, int64_t H, int D, size_t es, bool out,
                      int64_t max_token, Extent *ext, int64_t st[3]) {
    *ext = Extent{};
    st[0] = st[1] = st[2] = 0;
    if (t == nullptr) return api_fail(RM_ERR_INVALID_ARG, "%s is NULL", name);
    if (B == 0 || T == 0 || H == 0) return RM_OK;
    if (t->data == nullptr) return api_fail(RM_ERR_INVALID_ARG, "%s has no data", name);
    const int64_t size[3] = {B, T, H}, stride[3] = {t->batch, t->token, t->head};
    int64_t last = 0;  // offset of the last head vector, in bytes
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1) continue;
        if (stride[i] < 0) return api_fail(RM_ERR_SHAPE, "%s has a negative stride", name);
        if (stride[i] > (INT64_MAX >> 4) / size[i] / static_cast<int64_t>(es))
            return api_fail(RM_ERR_SHAPE, "%s spans more bytes than an address holds", name);
        st[i] = stride[i] * static_cast<int64_t>(es);
        if (st[i] % 16 != 0) return api_fail(RM_ERR_ALIGN, "%s: strides must be multiples of 16 bytes", name);
        last += (size[i] - 1) * st[i];
    }
    if (!aligned(t->data, 16)) return api_fail(RM_ERR_ALIGN, "%s must be 16-byte aligned", name);
    if (st[1] >= max_token)
        return api_fail(RM_ERR_SHAPE, "%s: a token stride of %lld bytes is not below %lld", name,
                        static_cast<long long>(st[1]), static_cast<long long>(max_token));
    if (out) {  // by rising stride, each axis must step over all of the ones before it
        int order[3] = {0, 1, 2};
        std::sort(order, order + 3, [&](int a, int b) { return st[a] < st[b]; });
        int64_t inner = D * static_cast<int64_t>(es);
        for (int i : order) {
            if (size[i] == 1) continue;
            if (st[i] < inner) return api_fail(RM_ERR_SHAPE, "%s: elements of an output must be distinct", name);
            inner = (size[i] - 1) * st[i] + inner;
        }
    }
    ext->p = t->data;
    ext->n = static_cast<size_t>(last) + D * es;
    return RM_OK;
}

inline rm_status check_attn_shape(const rm_attn_shape *s) {
    if (s == nullptr) return api_fail(RM_ERR_INVALID_ARG, "shape pointer is NULL");
    if (s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->n_q_heads % s->n_kv_heads != 0)
        return api_fail(RM_ERR_SHAPE, "n_q_heads=%d must be a positive multiple of n_kv_heads=%d", s->n_q_heads,
                        s->n_kv_heads);
    if (s->head_dim <= 0 || s->head_dim % 8 != 0 || s->head_dim > 256)
        return api_fail(RM_ERR_SHAPE, "head_dim=%d must be a multiple of 8 in [8, 256]", s->head_dim);
    if (s->dtype != RM_F32 && s->dtype != RM_BF16) return api_fail(RM_ERR_DTYPE, "unknown dtype %d", s->dtype);
    if (!(s->scale > 0.0f) || !std::isfinite(s->scale))
        return api_fail(RM_ERR_INVALID_ARG, "scale must be finite and positive");
    if (!(s->softcap >= 0.0f) || !std::isfinite(s->softcap))
        return api_fail(RM_ERR_INVALID_ARG, "softcap must be finite and not negative");
    if (s->softcap > 0.0f) {  // both factors of the capped score, scale / softcap and softcap log2 e, in float32
        const float x = s->scale / s->softcap;
        if (!(x >= FLT_MIN && x <= FLT_MAX / 4) || s->softcap > FLT_MAX / 2)
            return api_fail(RM_ERR_INVALID_ARG, "softcap=%g is out of float32's range at scale=%g",
                            static_cast<double>(s->softcap), static_cast<double>(s->scale));
    }
    return RM_OK;
}

}  // namespace rm_checks
