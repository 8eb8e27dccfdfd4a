// A paged cache's tables and the cache row of every new token, from the requests' lengths (rm_page_slots).
#include "rm_serve.h"

namespace rm_serve {

namespace {

constexpr int kThreads = 1024;
// Running sums stop here, above every number of tokens or pages that a call takes; a sum that stops at its limit may
// still be taken in any order.
constexpr uint32_t kMost = 1u << 30;
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// Running sums of two values over the workgroup's threads, their own included; all gets the sums of everyone.
__device__ __forceinline__ uint2 scan(uint2 v, uint2 &all, uint2 (&wave_sum)[kThreads / 64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(v.x, o), y = __shfl_up(v.y, o);
        if (lane >= o) v = make_uint2(add(v.x, x), add(v.y, y));
    }
    __syncthreads();
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    all = make_uint2(0, 0);
    uint2 before = all;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w == wave) before = all;
        all = make_uint2(add(all.x, wave_sum[w].x), add(all.y, wave_sum[w].y));
    }
    return make_uint2(add(v.x, before.x), add(v.y, before.y));
}

// The first of n rising ends that is above x (n if none is).
__device__ __forceinline__ int find(const uint32_t *ends, int n, uint32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// One workgroup; requests in chunks of one a thread.
__global__ __launch_bounds__(kThreads) void page_slots_kernel(SlotArgs a) {
    __shared__ uint2 wave_sum[kThreads / 64];
    __shared__ uint32_t ends[kThreads], wants[kThreads];
    __shared__ int32_t held[kThreads], begins[kThreads];
    const int tid = threadIdx.x;
    const int64_t room = static_cast<int64_t>(a.per) * a.page;
    const uint32_t n_free = min(max(a.n_free[0], 0), a.n_pages);
    auto length = [&](int b) { return static_cast<int>(min(static_cast<int64_t>(max(a.len[b], 0)), room)); };
    auto pages = [&](int64_t tokens) { return static_cast<uint32_t>((tokens + a.page - 1) / a.page); };

    // Ended requests give their pages back.
    uint32_t back = n_free;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        uint2 mine = make_uint2(0, 0), all;
        if (b < a.B && a.n_new[b] < 0) mine.x = pages(length(b));
        const uint2 upto = scan(mine, all, wave_sum);
        ends[tid] = upto.x;
        __syncthreads();
        for (uint32_t k = tid; k < all.x; k += kThreads) {
            const int r = find(ends, kThreads, k);
            const uint32_t i = k - (r > 0 ? ends[r - 1] : 0), to = add(back, k);
            if (to < static_cast<uint32_t>(a.n_pages))
                a.free_pages[to] = a.table[static_cast<int64_t>(b0 + r) * a.per + i];
        }
        back = add(back, all.x);
        __syncthreads();
    }
    const uint32_t avail = min(back, static_cast<uint32_t>(a.n_pages));

    uint32_t tokens = 0, wanted = 0, taken = 0, refused = 0;  // (taken, refused: of this thread's requests)
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        const bool is = b < a.B;
        const int n = is ? a.n_new[b] : 0, old = is ? length(b) : 0;
        uint2 mine = make_uint2(static_cast<uint32_t>(min(max(n, 0), static_cast<int>(kMost))), 0), all;
        // The tokens' ends first: they decide which requests fit.
        uint2 upto = scan(mine, all, wave_sum);
        const uint32_t end = add(tokens, upto.x), n_all = all.x;
        const bool fits = n >= 0 && static_cast<int64_t>(old) + n <= room && (n == 0 || end <= static_cast<uint32_t>(a.max_tok));
        const uint32_t have = pages(old);
        mine.x = fits ? pages(static_cast<int64_t>(old) + n) - have : 0;
        upto = scan(mine, all, wave_sum);
        const bool served = fits && (mine.x == 0 || add(wanted, upto.x) <= avail);
        ends[tid] = end;
        wants[tid] = upto.x;
        held[tid] = have;
        begins[tid] = served ? old : -1;
        if (served) taken += mine.x;
        if (is) {
            if (n >= 0 && !served) ++refused;
            a.len_out[b] = n < 0 ? 0 : served ? old + n : old;
            a.start[b] = served ? old : -1;
            a.first[b + 1] = static_cast<int32_t>(end);
            if (b == 0) a.first[0] = 0;
        }
        __syncthreads();
        for (uint32_t k = tid; k < all.x; k += kThreads) {
            const int r = find(wants, kThreads, k);
            const uint32_t at = add(wanted, k);
            if (begins[r] < 0 || at >= avail) continue;
            const uint32_t i = held[r] + k - (r > 0 ? wants[r - 1] : 0);
            a.table[static_cast<int64_t>(b0 + r) * a.per + i] = a.free_pages[avail - 1 - at];
        }
        __syncthreads();
        const uint32_t last = min(add(tokens, n_all), static_cast<uint32_t>(a.max_tok));
        for (uint32_t t = tokens + tid; t < last; t += kThreads) {
            const int r = find(ends, kThreads, t);
            const int p = begins[r] < 0 ? -1 : static_cast<int>(begins[r] + (t - (r > 0 ? ends[r - 1] : tokens)));
            int row = -1;
            if (p >= 0) {
                const int pg = a.table[static_cast<int64_t>(b0 + r) * a.per + p / a.page];
                if (pg >= 0 && pg < a.n_pages) row = pg * a.page + p % a.page;
            }
            a.seq[t] = b0 + r;
            a.pos[t] = p;
            a.slot[t] = row;
        }
        tokens = add(tokens, n_all);
        wanted = add(wanted, all.x);
        __syncthreads();
    }
    for (uint32_t t = tokens + tid; t < static_cast<uint32_t>(a.max_tok); t += kThreads) a.seq[t] = a.pos[t] = a.slot[t] = -1;
    uint2 all;
    scan(make_uint2(taken, refused), all, wave_sum);
    if (tid == 0) {
        a.n_free_out[0] = static_cast<int32_t>(avail - all.x);
        if (a.refused) a.refused[0] = static_cast<int32_t>(all.y);
    }
}

}  // namespace

hipError_t launch_page_slots(const SlotArgs &a, hipStream_t st) {
    page_slots_kernel<<<1, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rm_serve
