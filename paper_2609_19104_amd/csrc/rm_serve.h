// Arguments of the serving-step kernels (page_slots.hip, rm_paged.h, block_norm.hip).
#pragma once

#include "rm_attn_plan.h"

namespace rm_serve {

struct SlotArgs {
    int B = 0, max_tok = 0, page = 0, n_pages = 0, per = 0;  // per: table entries of a request
    bool in_place = false;  // len_out is len, or n_free_out is n_free
    rm_attn::Divisor by_page;
    const int32_t *n_new = nullptr, *len = nullptr, *n_free = nullptr;
    int32_t *table = nullptr, *free_pages = nullptr;
    int32_t *len_out = nullptr, *n_free_out = nullptr, *refused = nullptr;
    int32_t *first = nullptr, *start = nullptr, *seq = nullptr, *pos = nullptr, *slot = nullptr;
};
hipError_t launch_page_slots(const SlotArgs &a, hipStream_t st);

struct PagedArgs {
    const char *q = nullptr, *k = nullptr, *v = nullptr;  // strides in bytes
    char *o = nullptr;
    int64_t q_t = 0, q_h = 0, o_t = 0, o_h = 0;
    int64_t k_p = 0, k_t = 0, k_h = 0, v_p = 0, v_t = 0, v_h = 0;  // from page to page, row to row, head to head
    const int32_t *table = nullptr, *seq = nullptr, *pos = nullptr;
    const float *slopes = nullptr;
    int N = 0, seqs = 0, page = 0, n_pages = 0, per = 0, window = 0;
    rm_attn::Divisor by_page, by_q_tiles, by_units, by_groups;
    int D = 0, G = 0;
    // Units of a token: key heads times blocks of query heads; query heads of a block at most.
    int units = 0, q_tiles = 0, rows = 0;
    // Groups of waves, and where the parts of divided tokens are told: [N] or [groups].
    int groups = 0, by_token = 0;
    float scale = 0.0f, cap = 0.0f;  // scores in powers of two; with a cap: scale = score scale / cap
    float *part_o = nullptr;         // [groups][2][units][rows of a block][D]
    float2 *part_ml = nullptr;       // [groups][2][units][rows of a block]
    int2 *info = nullptr;
};
struct PagedPlan {
    int qr = 0, kt = 0;          // query heads of a block, keys of a tile
    int rpi = 0, per_cu = 0;     // rows of a load instruction, waves of a compute unit
    int groups = 0, units = 0, q_tiles = 0, by_token = 0;
    bool join = false, whole = false;  // whole: the rows of a load instruction are of one page
    size_t off_ml = 0, off_info = 0, total = 0;
};
void paged_shape_bf16(int D, int G, PagedPlan *p);  // qr, kt, rpi and per_cu
void paged_shape_f32(int D, int G, PagedPlan *p);
hipError_t launch_paged_bf16(const PagedPlan &p, const PagedArgs &a, hipStream_t st);
hipError_t launch_paged_f32(const PagedPlan &p, const PagedArgs &a, hipStream_t st);

struct NormArgs {
    const char *x = nullptr, *f = nullptr;
    char *y = nullptr, *out = nullptr;
    const float *gain_post = nullptr, *gate = nullptr, *gain_pre = nullptr, *scale = nullptr, *shift = nullptr;
    int64_t gate_b = 0, scale_b = 0, shift_b = 0;  // elements from sample to sample
    int64_t rows = 0, row0 = 0;  // row0: a launch's first
    int T = 0, d = 0, norm_post = 0;
    float x_scale = 1.0f, f_scale = 1.0f, eps = 0.0f;
};
hipError_t launch_block_norm(const NormArgs &a, bool x_bf16, bool f_bf16, bool out_bf16, hipStream_t st);

}  // namespace rm_serve
