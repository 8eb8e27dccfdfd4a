// Arguments of the norm-and-rotation kernel (qk_norm_rope.hip).
#pragma once

#include "rm_internal.h"

namespace rm {

struct RopeArgs {
    const char *q = nullptr, *k = nullptr, *v = nullptr;  // strides in bytes
    int64_t q_t = 0, q_h = 0, k_t = 0, k_h = 0, v_t = 0, v_h = 0;
    char *q_out = nullptr, *k_out = nullptr, *v_out = nullptr;
    int64_t qo_t = 0, qo_h = 0, ko_t = 0, ko_h = 0, vo_t = 0, vo_h = 0;
    const int32_t *pos = nullptr, *slot = nullptr;
    const float *inv_freq = nullptr, *gain_q = nullptr, *gain_k = nullptr;
    int N = 0, D = 0, Hq = 0, Hk = 0, H = 0, rot = 0, rows = 0, pairs = 0;  // H: all heads of a token (v's too, if any)
    float eps = 0.0f;
    int groups = 0, per = 0, lane_bits = 0;  // waves of a token, heads of a wave, logarithm of the lanes of a head
};
hipError_t launch_qk_norm_rope(const RopeArgs &a, bool in_bf16, bool out_bf16, hipStream_t st);
hipError_t launch_attn_spans(int B, int T, int N, int causal, int window, const int32_t *q_start,
                             const int32_t *kv_len, const int32_t *prefix_len, const int32_t *doc, int32_t *span,
                             hipStream_t st);

}  // namespace rm
