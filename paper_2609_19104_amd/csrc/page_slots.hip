// A paged cache's tables and the cache row of every new token, from the requests' lengths (rm_page_slots).
#include <algorithm>

#include "rm_serve.h"

namespace rm_serve {

namespace {

constexpr int kThreads = 1024;
constexpr int kAtOnce = 4;  // pages of a thread whose loads are in flight together
// Running sums stop here, above every number of tokens or pages that a call takes; a sum that stops at its limit may
// still be taken in any order.
constexpr uint32_t kMost = 1u << 30;
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, kMost); }

__device__ __forceinline__ int divide(int n, rm_attn::Divisor d) {  // n < 2^30
    return d.mul == 0 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), d.mul) >> d.shift);
}

// v added to by the lane CTRL of a data-parallel step says, in the rows of lanes of MASK.
template <int CTRL, int MASK>
__device__ __forceinline__ uint2 step(uint2 v) {
    return make_uint2(add(v.x, __builtin_amdgcn_update_dpp(0, static_cast<int>(v.x), CTRL, MASK, 0xf, false)),
                      add(v.y, __builtin_amdgcn_update_dpp(0, static_cast<int>(v.y), CTRL, MASK, 0xf, false)));
}
__device__ __forceinline__ uint2 scan16(uint2 v) {  // along the rows of 16 lanes
    return step<0x118, 0xf>(step<0x114, 0xf>(step<0x112, 0xf>(step<0x111, 0xf>(v))));
}
__device__ __forceinline__ uint2 of_lane(uint2 v, int lane) {
    return make_uint2(__builtin_amdgcn_readlane(v.x, lane), __builtin_amdgcn_readlane(v.y, lane));
}

// Running sums of two values over the workgroup's threads, their own included; all gets the sums of everyone.
__device__ __forceinline__ uint2 scan(uint2 v, uint2 &all, uint2 (&wave_sum)[kThreads / 64]) {
    static_assert(kThreads == 1024, "a row of lanes has the sums of 16 waves");
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    v = step<0x143, 0xc>(step<0x142, 0xa>(scan16(v)));
    if (waves == 1) {
        all = of_lane(v, 63);
        return v;
    }
    __syncthreads();
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    const uint2 sums = scan16(lane < waves ? wave_sum[lane] : make_uint2(0, 0));
    all = of_lane(sums, waves - 1);
    if (wave == 0) return v;
    const uint2 before = of_lane(sums, wave - 1);
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

// The row of position p in a request's table (-1: none).
__device__ __forceinline__ int row_of(const SlotArgs &a, const int32_t *table, int p) {
    const int i = divide(p, a.by_page), pg = table[i];
    return pg >= 0 && pg < a.n_pages ? pg * a.page + p - i * a.page : -1;
}

// One workgroup, since every page taken depends on all requests before: running sums over the requests, a thread each
// (chunks of them where they are more than threads), give each its tokens' and pages' numbers; then threads take single
// pages and tokens, whose request is the first with an end above their number.  Bound by round trips, not by its few bytes:
// lengths, tables and free list, the stores; 64 requests of a token each take 3.0 us in a graph, an empty kernel 1.6.
// fill: it writes the tokens too, up to most_fill of them (a thousand threads write 4 KB at a time: 131072 tokens took 79 us
// here, 5 in the kernel below and 7 for the rest; 17152 20, then 4.8 and 10.9).
__global__ __launch_bounds__(kThreads) void page_slots_kernel(SlotArgs a, int fill) {
    __shared__ uint2 wave_sum[kThreads / 64];
    __shared__ uint32_t ends[kThreads], wants[kThreads];
    __shared__ int32_t held[kThreads], begins[kThreads];
    const int tid = threadIdx.x, threads = blockDim.x;
    const int room = a.per * a.page;
    const bool once = a.B <= threads;  // one chunk: everything is read once
    auto pages = [&](int tokens) { return tokens > 0 ? static_cast<uint32_t>(divide(tokens - 1, a.by_page) + 1) : 0u; };
    int n = 0, old = 0;
    auto fetch = [&](int b) {
        n = b < a.B ? a.n_new[b] : 0;
        old = b < a.B ? min(max(a.len[b], 0), room) : 0;
    };
    fetch(tid);
    const uint32_t n_free = min(max(a.n_free[0], 0), a.n_pages);

    // Ended requests give their pages back.
    uint32_t back = n_free;
    for (int b0 = 0; b0 < a.B; b0 += threads) {
        if (b0 > 0) fetch(b0 + tid);
        if (!__syncthreads_or(n < 0)) continue;
        uint2 all;
        const uint2 upto = scan(make_uint2(n < 0 ? pages(old) : 0, 0), all, wave_sum);
        ends[tid] = upto.x;
        __syncthreads();
        for (uint32_t k0 = tid; k0 < all.x; k0 += kAtOnce * threads) {
            int32_t pg[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const uint32_t k = min(k0 + j * threads, all.x - 1);
                const int r = find(ends, threads, k);
                pg[j] = a.table[static_cast<int64_t>(b0 + r) * a.per + (k - (r > 0 ? ends[r - 1] : 0))];
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const uint32_t k = k0 + j * threads, to = add(back, k);
                if (k < all.x && to < static_cast<uint32_t>(a.n_pages)) a.free_pages[to] = pg[j];
            }
        }
        back = add(back, all.x);
        __syncthreads();
    }
    const uint32_t avail = min(back, static_cast<uint32_t>(a.n_pages)), max_tok = a.max_tok;

    uint32_t tokens = 0, wanted = 0, taken = 0, refused = 0;  // (taken, refused: of this thread's requests)
    for (int b0 = 0; b0 < a.B; b0 += threads) {
        const int b = b0 + tid;
        if (!once) fetch(b);
        const bool is = b < a.B;
        const uint32_t have = pages(old);
        bool fits = n >= 0 && n <= room - old;
        uint2 mine;
        mine.x = static_cast<uint32_t>(min(max(n, 0), static_cast<int>(kMost)));
        mine.y = fits ? pages(old + n) - have : 0;
        uint2 all, upto = scan(mine, all, wave_sum);
        const uint32_t end = add(tokens, upto.x), n_all = all.x;
        if (add(tokens, n_all) > max_tok) {  // tokens past the batch's room want no pages
            fits = fits && (n == 0 || end <= max_tok);
            if (!fits) mine.y = 0;
            upto.y = scan(mine, all, wave_sum).y;
        }
        const bool served = fits && (mine.y == 0 || add(wanted, upto.y) <= avail);
        const uint32_t first_want = add(wanted, upto.y - mine.y);  // (exact where it is served)
        const int start = served ? old : -1;
        if (served) taken += mine.y;
        if (is) {
            if (n >= 0 && !served) ++refused;
            a.len_out[b] = n < 0 ? 0 : served ? old + n : old;
            a.start[b] = start;
            a.first[b + 1] = static_cast<int32_t>(end);
            if (b == 0) a.first[0] = 0;
        }
        int32_t *const table = a.table + static_cast<int64_t>(is ? b : 0) * a.per;
        if (!__syncthreads_or(n > 1)) {
            // One token of every request at most: each thread has its own token and its page.
            if (served && n == 1) {
                int pg;
                if (mine.y != 0) {
                    pg = a.free_pages[avail - 1 - first_want];
                    table[have] = pg;
                } else {
                    pg = table[divide(old, a.by_page)];
                }
                if (fill) {
                    const int in_page = old - divide(old, a.by_page) * a.page;
                    a.slot[end - 1] = pg >= 0 && pg < a.n_pages ? pg * a.page + in_page : -1;
                }
            }
            if (fill && n == 1 && end <= max_tok) {
                a.seq[end - 1] = b;
                a.pos[end - 1] = start;
                if (!served) a.slot[end - 1] = -1;
            }
        } else {
            ends[tid] = end;
            wants[tid] = upto.y;
            held[tid] = have;
            begins[tid] = start;
            __syncthreads();
            // (Pages from avail - wanted on are the served requests' and perhaps a refused one's.)
            const uint32_t some = min(all.y, avail - min(avail, wanted));
            for (uint32_t k0 = tid; k0 < some; k0 += kAtOnce * threads) {
                int32_t pg[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    pg[j] = a.free_pages[avail - 1 - wanted - min(k0 + j * threads, some - 1)];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const uint32_t k = k0 + j * threads;
                    if (k >= some) break;
                    const int r = find(wants, threads, k);
                    if (begins[r] >= 0)
                        a.table[static_cast<int64_t>(b0 + r) * a.per + held[r] + k - (r > 0 ? wants[r - 1] : 0)] = pg[j];
                }
            }
            if (fill) {
                __syncthreads();
                const uint32_t last = min(add(tokens, n_all), max_tok);
                for (uint32_t t = tokens + tid; t < last; t += threads) {
                    const int r = find(ends, threads, t);
                    const int p = begins[r] < 0 ? -1 : static_cast<int>(begins[r] + (t - (r > 0 ? ends[r - 1] : tokens)));
                    a.seq[t] = b0 + r;
                    a.pos[t] = p;
                    a.slot[t] = p < 0 ? -1 : row_of(a, a.table + static_cast<int64_t>(b0 + r) * a.per, p);
                }
            }
        }
        tokens = add(tokens, n_all);
        wanted = add(wanted, all.y);
        if (!once) __syncthreads();
    }
    if (fill)
        for (uint32_t t = tokens + tid; t < max_tok; t += threads) a.seq[t] = a.pos[t] = a.slot[t] = -1;
    uint2 all;
    scan(make_uint2(taken, refused), all, wave_sum);
    if (tid == 0) {
        a.n_free_out[0] = static_cast<int32_t>(avail - all.x);
        if (a.refused) a.refused[0] = static_cast<int32_t>(all.y);
    }
}

constexpr int kFillThreads = 256, kFillTokens = 512;

// The tokens of a batch that one workgroup would be long about, after the kernel above: a workgroup takes kFillTokens of
// them.  It finds its first token's request by whole workgroups of comparisons (two rounds for up to 65536 requests, where
// halving takes sixteen), the others' from there on in LDS.  131072 tokens take 5.4 us, as few take: trips to memory.
__global__ __launch_bounds__(kFillThreads) void fill_kernel(SlotArgs a) {
    __shared__ uint32_t ends[kFillTokens];
    __shared__ int32_t begins[kFillTokens];
    const int tid = threadIdx.x;
    const uint32_t t0 = blockIdx.x * kFillTokens;
    const int32_t *const end_of = a.first + 1;
    int lo = 0, n = a.B + 1;  // the first request that ends above t0 is in [lo, lo + n), a.B if none does
    while (n > 1) {
        const int step = (n + kFillThreads - 1) / kFillThreads, i = lo + (tid + 1) * step - 1;
        const bool below = (tid + 1) * step <= n && i < a.B && static_cast<uint32_t>(end_of[i]) <= t0;
        const int done = __syncthreads_count(below) * step;
        lo += done;
        n = min(n - done, step);
    }
    const int count = min(kFillTokens, a.B - lo);  // requests in LDS
    for (int i = tid; i < count; i += kFillThreads) {
        ends[i] = end_of[lo + i];
        begins[i] = a.start[lo + i];
    }
    const uint32_t base = lo < a.B ? a.first[lo] : 0;
    __syncthreads();
    for (uint32_t t = t0 + tid; t < min(t0 + kFillTokens, static_cast<uint32_t>(a.max_tok)); t += kFillThreads) {
        int r = find(ends, count, t), b = lo + r, start = -1;
        uint32_t from = 0;
        if (r < count) {
            start = begins[r];
            from = r > 0 ? ends[r - 1] : base;
        } else {  // behind those (requests without tokens are many here), or behind the last
            b += find(reinterpret_cast<const uint32_t *>(end_of) + b, a.B - b, t);
            if (b < a.B) start = a.start[b], from = a.first[b];
        }
        const int p = start < 0 ? -1 : static_cast<int>(start + (t - from));
        a.seq[t] = b < a.B ? b : -1;
        a.pos[t] = p;
        a.slot[t] = p < 0 ? -1 : row_of(a, a.table + static_cast<int64_t>(b) * a.per, p);
    }
}

}  // namespace

hipError_t launch_page_slots(const SlotArgs &a, hipStream_t st) {
    const bool fill = a.max_tok <= a.most_fill;
    const int threads = std::min(kThreads, (std::max(a.B, std::min(a.max_tok, kThreads)) + 63) / 64 * 64);
    page_slots_kernel<<<1, threads, 0, st>>>(a, fill);
    if (!fill) fill_kernel<<<(a.max_tok + kFillTokens - 1) / kFillTokens, kFillThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rm_serve
