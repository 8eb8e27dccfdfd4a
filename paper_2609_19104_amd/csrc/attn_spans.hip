// Key intervals of the query rows from lengths, prefix lengths, a window and document ids (rm_attn_spans).
#include "rm_internal.h"

namespace rm {

namespace {

constexpr int kSpanRows = 256;  // rows per workgroup

// A document is a run of equal ids.  A workgroup's first row may lie inside a run that begins before its rows, and its
// last in one that ends after them: those two ends are searched for outwards, 8 ids a thread and step, and the runs in
// between come from a running maximum (minimum) of the positions where the id changes.  Bound by round trips (lengths,
// the search's loads, two joins of the workgroup): 8 x 16384 rows of 24 documents each take 7.3 us, 2.1 MB of ids and
// intervals; without documents 850 rows take 2.2.
__global__ __launch_bounds__(kSpanRows) void spans_kernel(int T, int N, int causal, int window,
                                                          const int32_t *__restrict__ q_start,
                                                          const int32_t *__restrict__ kv_len,
                                                          const int32_t *__restrict__ prefix_len,
                                                          const int32_t *__restrict__ doc, int32_t *__restrict__ span) {
    constexpr int kPer = 8, kStep = kSpanRows * kPer, kNone = -0x7fffffff;
    __shared__ int red[2][4];
    const int blocks = (T + kSpanRows - 1) / kSpanRows;
    const int b = blockIdx.x / blocks, i0 = (blockIdx.x - b * blocks) * kSpanRows;
    const int tid = threadIdx.x, i = i0 + tid;
    const int64_t start = q_start ? q_start[b] : 0;
    const int kv = kv_len ? min(max(kv_len[b], 0), N) : N;
    const int64_t p64 = start + i;
    int lo = 0, hi = kv;
    if (causal) {
        int64_t end = p64 + 1;
        if (prefix_len) end = max(end, static_cast<int64_t>(prefix_len[b]));
        hi = static_cast<int>(min(static_cast<int64_t>(kv), max(end, static_cast<int64_t>(0))));
    }
    if (window > 0) lo = static_cast<int>(min(max(p64 - window + 1, static_cast<int64_t>(0)), static_cast<int64_t>(N)));
    const bool inside = p64 >= 0 && p64 < kv;
    if (doc) {
        const int32_t *ids = doc + static_cast<int64_t>(b) * N;
        const int last_row = min(i0 + kSpanRows, T) - 1;
        const int pa = static_cast<int>(min(max(start + i0, static_cast<int64_t>(0)), static_cast<int64_t>(N - 1)));
        const int pb = static_cast<int>(min(max(start + last_row, static_cast<int64_t>(0)), static_cast<int64_t>(N - 1)));
        auto begins = [&](int j) { return j == 0 || ids[j] != ids[j - 1]; };  // a run begins at j in [0, N)
        // Both ends at a time: the greatest begin at or before pa, and minus the least one behind pb (N ends the last
        // run, position 0 begins the first, so both searches end).
        constexpr int64_t zero = 0;
        int first = -1, end = kNone;
        for (int64_t step = 0; first < 0 || end == kNone; step += kStep) {
            // All loads first (positions outside are read at the ends): in a branch each, every one would be a round
            // trip.
            int32_t at[2 * kPer], before[2 * kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int64_t i = pa - step - tid - k * kSpanRows, j = pb + 1 + step + tid + k * kSpanRows;
                at[2 * k] = ids[max(i, zero)];
                before[2 * k] = ids[max(i - 1, zero)];
                at[2 * k + 1] = ids[min(j, static_cast<int64_t>(N - 1))];
                before[2 * k + 1] = ids[min(j - 1, static_cast<int64_t>(N - 1))];
            }
            int best = -1, next = kNone;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int64_t i = pa - step - tid - k * kSpanRows, j = pb + 1 + step + tid + k * kSpanRows;
                if (i >= 0 && (i == 0 || at[2 * k] != before[2 * k])) best = max(best, static_cast<int>(i));
                if (j <= N && (j == N || at[2 * k + 1] != before[2 * k + 1])) next = max(next, static_cast<int>(-j));
            }
            for (int o = 32; o >= 1; o >>= 1) {
                best = max(best, __shfl_xor(best, o));
                next = max(next, __shfl_xor(next, o));
            }
            __syncthreads();
            if ((tid & 63) == 0) red[0][tid >> 6] = best, red[1][tid >> 6] = next;
            __syncthreads();
            if (first < 0) first = max(max(red[0][0], red[0][1]), max(red[0][2], red[0][3]));
            if (end == kNone) end = max(max(red[1][0], red[1][1]), max(red[1][2], red[1][3]));
        }
        // This row's run: the last begin at or before p, and the first after it.
        const int p = static_cast<int>(min(max(p64, static_cast<int64_t>(0)), static_cast<int64_t>(N - 1)));
        const bool row = i < T;
        int beg = row && begins(p) ? p : first;
        const int lane = tid & 63, wave = tid >> 6;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(beg, o);
            if (lane >= o) beg = max(beg, v);
        }
        // Negated, so that a running maximum from the last row backwards gives the first begin after p.
        int nxt = row && p + 1 < N && p < pb && begins(p + 1) ? -(p + 1) : end;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_down(nxt, o);
            if (lane + o < 64) nxt = max(nxt, v);
        }
        __shared__ int wbeg[4], wnxt[4];
        if (lane == 63) wbeg[wave] = beg;
        if (lane == 0) wnxt[wave] = nxt;
        __syncthreads();
        for (int w = 0; w < wave; ++w) beg = max(beg, wbeg[w]);
        for (int w = wave + 1; w < 4; ++w) nxt = max(nxt, wnxt[w]);
        lo = max(lo, beg);
        hi = min(hi, -nxt);
        if (row && ids[p] < 0) hi = 0;
    }
    if (i >= T) return;
    if (((causal || doc) && !inside) || hi <= lo) lo = hi = 0;
    reinterpret_cast<int2 *>(span)[static_cast<int64_t>(b) * T + i] = make_int2(lo, hi);
}

}  // namespace

hipError_t launch_attn_spans(int B, int T, int N, int causal, int window, const int32_t *q_start,
                             const int32_t *kv_len, const int32_t *prefix_len, const int32_t *doc, int32_t *span,
                             hipStream_t st) {
    const int blocks = (T + kSpanRows - 1) / kSpanRows;
    spans_kernel<<<dim3(static_cast<unsigned>(blocks) * B), kSpanRows, 0, st>>>(T, N, causal, window, q_start, kv_len,
                                                                              prefix_len, doc, span);
    return hipGetLastError();
}

}  // namespace rm
