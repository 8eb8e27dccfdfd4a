// A paged cache's tables and the cache row of every new token, from the requests' lengths (rm_page_slots).
#include <algorithm>

#include "rm_serve.h"

namespace rm_serve {

namespace {

constexpr int kThreads = 1024;
constexpr int kAtOnce = 4;  // pages or tokens of a thread whose loads are in flight together
// Running sums stop here, above every number of tokens or pages that a call takes; a sum that stops at its limit may
// still be taken in any order.
constexpr uint32_t kMost = 1u << 30;
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return min(a + b, kMost); }

__device__ __forceinline__ int divide(int n, rm_attn::Divisor d) {  // n < 2^30
    return d.mul == 0 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), d.mul) >> d.shift);
}

struct Sums {
    uint32_t x, y, z;
};
__device__ __forceinline__ Sums add(Sums a, Sums b) { return {add(a.x, b.x), add(a.y, b.y), add(a.z, b.z)}; }

// v added to by the lane CTRL of a data-parallel step says, in the rows of lanes of MASK.
template <int CTRL, int MASK>
__device__ __forceinline__ Sums step(Sums v) {
    auto moved = [](uint32_t x) -> uint32_t {
        return __builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, MASK, 0xf, false);
    };
    return add(v, {moved(v.x), moved(v.y), moved(v.z)});
}
__device__ __forceinline__ Sums scan16(Sums v) {  // along the rows of 16 lanes
    return step<0x118, 0xf>(step<0x114, 0xf>(step<0x112, 0xf>(step<0x111, 0xf>(v))));
}
__device__ __forceinline__ Sums of_lane(Sums v, int lane) {
    return {static_cast<uint32_t>(__builtin_amdgcn_readlane(v.x, lane)), static_cast<uint32_t>(__builtin_amdgcn_readlane(v.y, lane)),
            static_cast<uint32_t>(__builtin_amdgcn_readlane(v.z, lane))};
}

// Running sums of three values over the workgroup's threads, their own included; all gets the sums of everyone.
__device__ __forceinline__ Sums scan(Sums v, Sums &all, Sums (&wave_sum)[kThreads / 64]) {
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
    const Sums sums = scan16(lane < waves ? wave_sum[lane] : Sums{0, 0, 0});
    all = of_lane(sums, waves - 1);
    return wave == 0 ? v : add(v, of_lane(sums, wave - 1));
}

// The first of n rising ends that is above x (n if none is), for several x side by side: one after the other, each would
// cost ten trips to LDS.
template <int K>
__device__ __forceinline__ void find(const uint32_t *ends, int n, const uint32_t (&x)[K], int (&r)[K]) {
#pragma unroll
    for (int i = 0; i < K; ++i) r[i] = 0;
    for (int step = n > 0 ? 1 << (31 - __builtin_clz(n)) : 0; step >= 1; step >>= 1)
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int at = r[i] + step;
            if (ends[min(at, n) - 1] <= x[i] && at <= n) r[i] = at;
        }
}
__device__ __forceinline__ int find(const uint32_t *ends, int n, uint32_t x) {
    const uint32_t one[1] = {x};
    int r[1];
    find(ends, n, one, r);
    return r[0];
}

// The row of position p in a request's table (-1: none).
__device__ __forceinline__ int row_of(const SlotArgs &a, const int32_t *table, int p) {
    const int i = divide(p, a.by_page), pg = table[i];
    return pg >= 0 && pg < a.n_pages ? pg * a.page + p - i * a.page : -1;
}

// One workgroup, since every page taken depends on all requests before: running sums over the requests, a thread each
// (chunks of them where they are more than threads), give each its tokens' and pages' numbers; then threads take single
// pages and tokens, whose request is the first with an end above their number.  Bound by round trips, not by its few bytes:
// lengths, tables and free list, the stores; 64 requests of a token each take 2.7 us in a graph, an empty kernel 1.6.  A page
// that one request gives back and another takes in the same step is read from the ended request's table, since through the
// free list it would wait for a store and a barrier.
// fill: it writes the tokens too, where they are few (a thousand threads write 4 KB at a time: 131072 tokens took 79 us here,
// 17152 20).
//
// MANY: the same by many workgroups, for more tokens of no more requests than a workgroup has threads.  Each makes all
// running sums; the first page_blocks of them move pages, the others write tokens, whose new pages they take from where they
// lie, not from the tables.  So nobody reads what another writes: of the free list what was free, of the tables what a
// request had; lengths and count, where they are updated in place, are left to finish_kernel.  256 requests with 8 thousand
// tokens 5.2 us (one workgroup for the pages and, after it, many for the tokens 13.1), 1024 with 66 thousand 5.4 (10.3).
template <bool MANY>
__global__ __launch_bounds__(kThreads) void page_slots_kernel(SlotArgs a, int fill, int page_blocks) {
    __shared__ Sums wave_sum[kThreads / 64];
    __shared__ uint32_t ends[kThreads], wants[kThreads], backs[kThreads];
    __shared__ int32_t held[kThreads], begins[kThreads];
    const int tid = threadIdx.x, threads = blockDim.x;
    const int room = a.per * a.page;
    const bool once = MANY || a.B <= threads;  // one chunk: everything is read once
    const bool tells = !MANY || blockIdx.x == 0;
    auto pages = [&](int tokens) { return tokens > 0 ? static_cast<uint32_t>(divide(tokens - 1, a.by_page) + 1) : 0u; };
    int n = 0, old = 0;
    auto fetch = [&](int b) {
        n = b < a.B ? a.n_new[b] : 0;
        old = b < a.B ? min(max(a.len[b], 0), room) : 0;
    };
    fetch(tid);
    const uint32_t n_free = min(max(a.n_free[0], 0), a.n_pages), n_pages = a.n_pages, max_tok = a.max_tok;
    // Where page number k lies that the ended requests of the chunk at b0 give back, r the one that has it.
    auto given = [&](int b0, uint32_t k, int r) {
        return a.table + static_cast<int64_t>(b0 + r) * a.per + (k - (r > 0 ? backs[r - 1] : 0));
    };

    // Ended requests give their pages back before anyone takes pages: with several chunks in a pass of its own.
    uint32_t back = n_free;
    for (int b0 = once ? a.B : 0; b0 < a.B; b0 += threads) {
        if (b0 > 0) fetch(b0 + tid);
        Sums all;
        backs[tid] = scan({0, 0, n < 0 ? pages(old) : 0}, all, wave_sum).z;
        __syncthreads();
        for (uint32_t k = tid; k < all.z; k += threads) {
            const uint32_t to = add(back, k);
            if (to < n_pages) a.free_pages[to] = *given(b0, k, find(backs, threads, k));
        }
        back = add(back, all.z);
        __syncthreads();
    }

    uint32_t tokens = 0, wanted = 0, taken = 0, refused = 0, avail = 0;  // (taken, refused: of this thread's requests)
    for (int b0 = 0; b0 < a.B; b0 += threads) {
        const int b = b0 + tid;
        if (!once) fetch(b);
        const bool is = b < a.B;
        const uint32_t have = pages(old);
        bool fits = n >= 0 && n <= room - old;
        Sums mine, all;
        mine.x = static_cast<uint32_t>(min(max(n, 0), static_cast<int>(kMost)));
        mine.y = fits ? pages(old + n) - have : 0;
        mine.z = once && n < 0 ? have : 0;
        Sums upto = scan(mine, all, wave_sum);
        const uint32_t end = add(tokens, upto.x), n_all = all.x;
        if (add(tokens, n_all) > max_tok) {  // tokens past the batch's room want no pages
            fits = fits && (n == 0 || end <= max_tok);
            if (!fits) mine.y = 0;
            upto.y = scan(mine, all, wave_sum).y;
        }
        const uint32_t n_back = all.z;
        avail = min(add(back, n_back), n_pages);
        const bool served = fits && (mine.y == 0 || add(wanted, upto.y) <= avail);
        const uint32_t first_want = add(wanted, upto.y - mine.y);  // (exact where it is served)
        const int start = served ? old : -1;
        if (served) taken += mine.y;
        if (is && n >= 0 && !served) ++refused;
        if (is && tells) {
            if (!MANY || !a.in_place) a.len_out[b] = n < 0 ? 0 : served ? old + n : old;
            a.start[b] = start;
            a.first[b + 1] = static_cast<int32_t>(end);
            if (b == 0) a.first[0] = 0;
        }
        ends[tid] = end;
        wants[tid] = upto.y;
        backs[tid] = upto.z;
        held[tid] = have;
        begins[tid] = start;
        const bool ones = !__syncthreads_or(n > 1) && !MANY;  // one token of every request at most
        // Where the page lies that is taken as number k of all: at the top of the free list, or if this step's ended requests
        // give it back, still in their tables.
        auto page_of = [&](uint32_t k) {
            const uint32_t i = avail - 1 - k;
            return i < back || n_back == 0 ? a.free_pages + i : given(b0, i - back, find(backs, threads, i - back));
        };
        // Pages given back go to the free list, pages taken (from avail - wanted on they are the served requests' and perhaps
        // a refused one's) into the tables: all loads of a turn, then its stores.
        const uint32_t some = ones ? 0 : min(all.y, avail - min(avail, wanted));
        int pg_own = -1;
        int32_t *const table = a.table + static_cast<int64_t>(is ? b : 0) * a.per;
        if (ones && served && n == 1) {
            pg_own = mine.y != 0 ? *page_of(first_want) : table[divide(old, a.by_page)];
        }
        constexpr int AT = MANY ? 1 : kAtOnce;
        const uint32_t movers = MANY ? page_blocks * threads : threads;
        for (uint32_t k0 = MANY ? blockIdx.x * threads + tid : tid; k0 < max(n_back, some); k0 += AT * movers) {
            if (MANY && static_cast<int>(blockIdx.x) >= page_blocks) break;
            int32_t from_ended[AT], from_free[AT];
            uint32_t k[AT];
            int r[AT];
#pragma unroll
            for (int j = 0; j < AT; ++j) k[j] = k0 + j * movers;
            if (k0 < n_back) find(backs, threads, k, r);
#pragma unroll
            for (int j = 0; j < AT; ++j) {
                from_ended[j] = k[j] < n_back ? *given(b0, k[j], r[j]) : 0;
                from_free[j] = k[j] < some ? *page_of(wanted + k[j]) : 0;
            }
#pragma unroll
            for (int j = 0; j < AT; ++j) {
                const uint32_t to = add(back, k[j]);
                if (k[j] < n_back && to < n_pages) a.free_pages[to] = from_ended[j];
                if (k[j] < some) {
                    const int q = find(wants, threads, k[j]);
                    if (begins[q] >= 0)
                        a.table[static_cast<int64_t>(b0 + q) * a.per + held[q] + k[j] - (q > 0 ? wants[q - 1] : 0)] = from_free[j];
                }
            }
        }
        if constexpr (MANY) {
            const uint32_t last = min(n_all, max_tok), writers = (gridDim.x - page_blocks) * threads;
            if (static_cast<int>(blockIdx.x) >= page_blocks)
                for (uint32_t t = (blockIdx.x - page_blocks) * threads + tid; t < max_tok; t += writers) {
                    int r = -1, p = -1, row = -1;
                    if (t < last) {
                        r = find(ends, threads, t);
                        if (begins[r] >= 0) {
                            p = static_cast<int>(begins[r] + (t - (r > 0 ? ends[r - 1] : 0)));
                            const uint32_t i = divide(p, a.by_page), own = held[r];
                            const int pg = i < own ? a.table[static_cast<int64_t>(r) * a.per + i]
                                                   : *page_of((r > 0 ? wants[r - 1] : 0) + i - own);
                            if (pg >= 0 && pg < a.n_pages) row = pg * a.page + p - static_cast<int>(i) * a.page;
                        }
                    }
                    a.seq[t] = r;
                    a.pos[t] = p;
                    a.slot[t] = row;
                }
        } else if (ones) {  // each thread has its own token
            if (served && n == 1 && mine.y != 0) table[have] = pg_own;
            if (fill && n == 1 && end <= max_tok) {
                const int in_page = old - divide(old, a.by_page) * a.page;
                a.seq[end - 1] = b;
                a.pos[end - 1] = start;
                a.slot[end - 1] = pg_own >= 0 && pg_own < a.n_pages ? pg_own * a.page + in_page : -1;
            }
        } else if (fill) {
            __syncthreads();
            const uint32_t last = min(add(tokens, n_all), max_tok);
            for (uint32_t t0 = tokens + tid; t0 < last; t0 += kAtOnce * threads) {
                uint32_t t[kAtOnce];
                int r[kAtOnce], p[kAtOnce], row[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) t[j] = t0 + j * threads;
                find(ends, threads, t, r);
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int q = min(r[j], threads - 1);
                    p[j] = t[j] >= last || begins[q] < 0 ? -1 : static_cast<int>(begins[q] + (t[j] - (q > 0 ? ends[q - 1] : tokens)));
                    row[j] = p[j] < 0 ? -1 : row_of(a, a.table + static_cast<int64_t>(b0 + q) * a.per, p[j]);
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (t[j] < last) a.seq[t[j]] = b0 + r[j], a.pos[t[j]] = p[j], a.slot[t[j]] = row[j];
            }
        }
        tokens = add(tokens, n_all);
        wanted = add(wanted, all.y);
        if (!once) __syncthreads();
    }
    if (!MANY && fill)
        for (uint32_t t = tokens + tid; t < max_tok; t += threads) a.seq[t] = a.pos[t] = a.slot[t] = -1;
    if (!tells) return;
    Sums all;
    scan({taken, refused, 0}, all, wave_sum);
    if (tid == 0) {
        if (!MANY || !a.in_place) a.n_free_out[0] = static_cast<int32_t>(avail - all.x);
        if (a.refused) a.refused[0] = static_cast<int32_t>(all.y);
    }
}

// The lengths and the count, from where the requests start and what they were, after workgroups that all read the old ones.
__global__ __launch_bounds__(kThreads) void finish_kernel(SlotArgs a) {
    __shared__ Sums wave_sum[kThreads / 64];
    const int b = threadIdx.x;
    const uint32_t n_free = min(max(a.n_free[0], 0), a.n_pages);
    auto pages = [&](int tokens) { return tokens > 0 ? static_cast<uint32_t>(divide(tokens - 1, a.by_page) + 1) : 0u; };
    Sums mine = {0, 0, 0}, all;
    if (b < a.B) {
        const int n = a.n_new[b], old = min(max(a.len[b], 0), a.per * a.page), start = a.start[b];
        a.len_out[b] = n < 0 ? 0 : start >= 0 ? start + n : old;
        if (n < 0) mine.x = pages(old);
        else if (start >= 0) mine.y = pages(start + n) - pages(start);
    }
    scan(mine, all, wave_sum);
    if (b == 0) a.n_free_out[0] = static_cast<int32_t>(min(add(n_free, all.x), static_cast<uint32_t>(a.n_pages)) - all.y);
}

constexpr int kFillThreads = 256, kFillTokens = 512;

// The tokens of more requests than a workgroup has threads, after the kernel above by one: a workgroup takes kFillTokens of
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
    constexpr int K = kFillTokens / kFillThreads;
    uint32_t t[K];
    int r[K], b[K], p[K], row[K];
#pragma unroll
    for (int j = 0; j < K; ++j) t[j] = t0 + tid + j * kFillThreads;
    find(ends, count, t, r);
#pragma unroll
    for (int j = 0; j < K; ++j) {
        int start = -1;
        uint32_t from = 0;
        b[j] = lo + r[j];
        if (r[j] < count) {
            start = begins[r[j]];
            from = r[j] > 0 ? ends[r[j] - 1] : base;
        } else {  // behind those (requests without tokens are many here), or behind the last
            b[j] += find(reinterpret_cast<const uint32_t *>(end_of) + b[j], a.B - b[j], t[j]);
            if (b[j] < a.B) start = a.start[b[j]], from = a.first[b[j]];
        }
        p[j] = start < 0 || t[j] >= static_cast<uint32_t>(a.max_tok) ? -1 : static_cast<int>(start + (t[j] - from));
        row[j] = p[j] < 0 ? -1 : row_of(a, a.table + static_cast<int64_t>(b[j]) * a.per, p[j]);
    }
#pragma unroll
    for (int j = 0; j < K; ++j)
        if (t[j] < static_cast<uint32_t>(a.max_tok)) {
            a.seq[t[j]] = b[j] < a.B ? b[j] : -1;
            a.pos[t[j]] = p[j];
            a.slot[t[j]] = row[j];
        }
}

}  // namespace

// One workgroup for a token each (64 requests of which some end 4.7 us, by many workgroups 5.1) and for few tokens.  Else many,
// from 257 tokens on (a prompt of 500 6.6 and 4.0, 256 requests of 4 tokens 10.6 and 5.3, of one 6.9 and 5.3); where lengths and
// count are updated in place from 4097 on: that takes a second launch, which costs the host 2 us, so that many are faster only
// in graphs and with prompts (64 requests of 32 tokens 7.7 and 5.4; 256 of one, with room for 2048, 4.6 and 5.9).
hipError_t launch_page_slots(const SlotArgs &a, hipStream_t st) {
    const bool fill = a.max_tok <= (a.in_place || a.B > kThreads ? 4096 : std::max(256, a.B));
    const int wide = (a.B + 63) / 64 * 64;
    if (!fill && a.B <= kThreads) {
        const int threads = std::max(256, wide);
        // A thread for each page that the tokens take and for one in 16 of the tables', as ended requests may give back
        // (with threads for the first only, 16 of 256 requests ending, 512 pages at most each, 7.0 us).
        const int64_t pages = a.max_tok / a.page + a.B + static_cast<int64_t>(a.B) * a.per / 16;
        const int movers = static_cast<int>(std::min<int64_t>(64, pages / threads + 1));
        const int writers = std::min((a.max_tok + threads - 1) / threads, 256 * 2048 / threads);
        page_slots_kernel<true><<<movers + writers, threads, 0, st>>>(a, 0, movers);
        if (a.in_place) finish_kernel<<<1, wide, 0, st>>>(a);
        return hipGetLastError();
    }
    const int threads = std::min(kThreads, std::max(wide, (std::min(a.max_tok, kThreads) + 63) / 64 * 64));
    page_slots_kernel<false><<<1, threads, 0, st>>>(a, fill, 0);
    if (!fill) fill_kernel<<<(a.max_tok + kFillTokens - 1) / kFillTokens, kFillThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rm_serve
