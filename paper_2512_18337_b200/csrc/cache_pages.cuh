// Page bookkeeping of the 4-bit cache: reserve (with copy on write), commit / roll back, fork, compact, whole-page copies.
//
// Every result is independent of timing: pages are handed out and given back by prefix sums over rows and positions, and
// where several rows name one page, integer atomics decide by row number.
//
// The bookkeeping is a few kilobytes: what it costs is chains of dependent loads (about 700 ns each) and launches, so a call is one
// block (288 rows: reserve 7 us, commit 9 us, a commit that gives 3,800 pages back 25 us).  Page contents move at 5.6 TB/s.
#pragma once

#include "cache_format.cuh"

namespace samb200 {

constexpr int kPageThreads = 1024;
constexpr int kStatusOutOfPages = 1, kStatusTableFull = 2, kStatusBadFork = 4;
constexpr int kClaim = 1 << 30;

// Scratch words: 0 = number of copies, then per-row words and lists.
constexpr int kScratchHead = 64;
struct PageScratch {
    int32_t* count;     // copies listed
    int32_t* row_a;     // [n_streams]
    int32_t* row_b;     // [n_streams]
    int32_t* row_c;     // [n_streams]
    int32_t* from;      // [max(n_streams, n_pages)]
    int32_t* to;
    int32_t* remap;     // [n_pages]
};
__host__ __device__ inline int64_t page_scratch_ints(int64_t n_streams, int64_t n_pages) {
    const int64_t list = n_streams > n_pages ? n_streams : n_pages;
    return kScratchHead + 3 * n_streams + 2 * list + n_pages;
}
__device__ __forceinline__ PageScratch page_scratch(const CacheView& c) {
    const int64_t list = max(c.n_streams, c.n_pages);
    PageScratch s;
    s.count = c.scratch;
    s.row_a = c.scratch + kScratchHead;
    s.row_b = s.row_a + c.n_streams;
    s.row_c = s.row_b + c.n_streams;
    s.from = s.row_c + c.n_streams;
    s.to = s.from + list;
    s.remap = s.to + list;
    return s;
}

// Exclusive prefix sum over the block; *total gets the sum.  All threads call it.
__device__ __forceinline__ int block_scan(int x, int* total) {
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, y, d);
        if (lane >= d) y += up;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = y;
    __syncthreads();
    if (warp == 0) {
        int z = lane < static_cast<int>(blockDim.x >> 5) ? sums[lane] : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, z, d);
            if (lane >= d) z += up;
        }
        sums[lane] = z;
    }
    __syncthreads();
    *total = sums[(blockDim.x >> 5) - 1];
    return y - x + (warp ? sums[warp - 1] : 0);
}

// Sum over the block, known to all threads.
__device__ __forceinline__ int block_sum(int x) {
    __shared__ int sums[32];
    x = __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = x;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, (threadIdx.x & 31) < (blockDim.x >> 5) ? sums[threadIdx.x & 31] : 0);
}

__global__ void cache_init_kernel(CacheView c) {
    const int64_t i0 = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t i = i0; i < static_cast<int64_t>(c.n_streams) * c.max_pages; i += step) c.table[i] = -1;
    for (int64_t i = i0; i < c.n_streams; i += step) c.seq_len[i] = 0;
    for (int64_t i = i0; i < c.n_pages; i += step) {
        c.ref[i] = 0;
        c.free_list[i] = c.n_pages - 1 - static_cast<int>(i);
    }
    if (i0 < 4) c.meta[i0] = i0 == 0 ? c.n_pages : 0;
}

struct RowNeed {
    int s, n, first, want, page0;   // page0: the partly filled page that will be written to, or -1
};
__device__ __forceinline__ RowNeed row_need(const CacheView& c, const int32_t* streams, const int32_t* n_new, int b) {
    RowNeed r;
    r.s = c.stream_of(streams, b);
    r.n = r.s < 0 ? 0 : max(n_new[b], 0);
    r.first = r.want = 0;
    r.page0 = -1;
    if (r.n == 0) return r;
    const int len = c.length_of(r.s);
    r.first = len >> c.log_p;
    r.want = static_cast<int>((static_cast<int64_t>(len) + r.n + c.page_tokens() - 1) >> c.log_p);
    if ((len & (c.page_tokens() - 1)) && r.first < c.max_pages) r.page0 = c.page_at(r.s, r.first);
    return r;
}

// One block; a thread looks after up to four rows and keeps them in registers.  What a step costs is the chain of dependent
// loads (stream, length, table, counts), so each of them is made once.  Rows that need room for many pages (a prompt) are
// counted and filled by the whole block, one after the other.
constexpr int kRowsPerThread = 4;   // SAM_CACHE_MAX_B / kPageThreads
constexpr int kLongSpan = 8;        // pages that a thread looks at by itself
__global__ void __launch_bounds__(kPageThreads) reserve_kernel(CacheView c, int B, const int32_t* streams, const int32_t* n_new) {
    const PageScratch sc = page_scratch(c);
    __shared__ int bad, copies, n_long;
    if (threadIdx.x == 0) bad = copies = n_long = 0;
    __syncthreads();
    const int n_free = c.meta[0];
    RowNeed r[kRowsPerThread];
    auto is_long = [](const RowNeed& x) { return x.want - x.first > kLongSpan; };
    int need[kRowsPerThread];
    bool sole[kRowsPerThread], keeper[kRowsPerThread];
    // writers of a page leave it: a count of zero means that all its holders write
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
        const int b = u * kPageThreads + threadIdx.x;
        r[u].s = r[u].page0 = -1;
        r[u].first = r[u].want = need[u] = 0;
        if (b >= B) continue;
        r[u] = row_need(c, streams, n_new, b);
        if (r[u].want > c.max_pages) bad = 1;
        if (r[u].page0 >= 0) atomicSub(&c.ref[r[u].page0], 1);
        if (is_long(r[u])) sc.row_a[atomicAdd(&n_long, 1)] = b;   // in any order: each is dealt with by itself
        else
            for (int i = r[u].first; i < min(r[u].want, c.max_pages); ++i) need[u] += c.page_at(r[u].s, i) < 0;
    }
    __syncthreads();
    for (int j = 0; j < n_long; ++j) {
        const int b = sc.row_a[j];
        const RowNeed x = row_need(c, streams, n_new, b);
        int missing = 0;
        for (int i = x.first + threadIdx.x; i < min(x.want, c.max_pages); i += kPageThreads) missing += c.page_at(x.s, i) < 0;
        missing = block_sum(missing);
        if (threadIdx.x == 0) sc.row_b[b] = missing;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u)
        if (is_long(r[u])) need[u] = sc.row_b[u * kPageThreads + threadIdx.x];
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) sole[u] = r[u].page0 >= 0 && __ldcg(&c.ref[r[u].page0]) == 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u)
        if (sole[u]) atomicMax(&c.ref[r[u].page0], u * kPageThreads + threadIdx.x + 1);
    __syncthreads();
    int mine = 0;
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
        // the last of the rows that write keeps the page
        keeper[u] = sole[u] && __ldcg(&c.ref[r[u].page0]) == static_cast<int>(u * kPageThreads + threadIdx.x + 1);
        need[u] += r[u].page0 >= 0 && !keeper[u];
        mine += need[u];
    }
    const int need_all = block_sum(mine);
    if (bad || need_all > n_free) {   // put the counts back
#pragma unroll
        for (int u = 0; u < kRowsPerThread; ++u)
            if (keeper[u]) c.ref[r[u].page0] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kRowsPerThread; ++u)
            if (r[u].page0 >= 0) atomicAdd(&c.ref[r[u].page0], 1);
        if (threadIdx.x == 0) {
            c.meta[1] |= bad ? kStatusTableFull : kStatusOutOfPages;
            *sc.count = 0;
        }
        return;
    }
    int before = 0;
#pragma unroll
    for (int u = 0; u < kRowsPerThread; ++u) {
        if (u * kPageThreads >= B) break;
        int total;
        int at = n_free - 1 - before - block_scan(need[u], &total);
        before += total;
        if (keeper[u]) c.ref[r[u].page0] = 1;
        const bool copy = r[u].page0 >= 0 && !keeper[u];
        if (need[u] == 0) continue;
        auto hand_out = [&](int i, int page) {
            c.row(r[u].s)[i] = page;
            if (static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages)) c.ref[page] = 1;
        };
        if (copy) {
            const int page = c.free_list[at--], k = atomicAdd(&copies, 1);   // the order of the copies does not matter
            sc.from[k] = r[u].page0;
            sc.to[k] = page;
            hand_out(r[u].first, page);
        }
        if (is_long(r[u])) sc.row_c[u * kPageThreads + threadIdx.x] = at;
        else
            for (int i = r[u].first; i < r[u].want; ++i)
                if (c.page_at(r[u].s, i) < 0) hand_out(i, c.free_list[at--]);
    }
    __syncthreads();
    for (int j = 0; j < n_long; ++j) {
        const int b = sc.row_a[j];
        const RowNeed x = row_need(c, streams, n_new, b);
        int at = sc.row_c[b];
        if (sc.row_b[b] == 0) continue;
        for (int i0 = x.first; i0 < x.want; i0 += kPageThreads) {
            const int i = i0 + threadIdx.x;
            const bool missing = i < x.want && c.page_at(x.s, i) < 0;
            int total;
            const int mine_at = at - block_scan(missing, &total);
            at -= total;
            if (!missing) continue;
            const int page = c.free_list[mine_at];
            c.row(x.s)[i] = page;
            if (static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages)) c.ref[page] = 1;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        c.meta[0] = n_free - need_all;
        *sc.count = copies;
    }
}

// Copies count pages src[from[k]] -> dst[to[k]]; a block takes 16 KB pieces.
constexpr int kCopyPiece = 16384, kCopyThreads = 256;
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const uint8_t* src, uint8_t* dst, int64_t page_bytes, int src_pages, int dst_pages,
                                                                  const int32_t* count, int n, const int32_t* from, const int32_t* to) {
    if (count) n = *count;
    const int64_t per_page = (page_bytes + kCopyPiece - 1) / kCopyPiece;
    for (int64_t w = blockIdx.x; w < n * per_page; w += gridDim.x) {
        const int k = static_cast<int>(w / per_page);
        const int64_t off = (w % per_page) * kCopyPiece;
        const int f = from[k], t = to[k];
        if (static_cast<unsigned>(f) >= static_cast<unsigned>(src_pages) || static_cast<unsigned>(t) >= static_cast<unsigned>(dst_pages)) continue;
        const int units = static_cast<int>(min(static_cast<int64_t>(kCopyPiece), page_bytes - off) >> 4);
        const uint4* a = reinterpret_cast<const uint4*>(src + f * page_bytes + off);
        uint4* z = reinterpret_cast<uint4*>(dst + t * page_bytes + off);
        uint4 x[kCopyPiece / 16 / kCopyThreads];
#pragma unroll
        for (int i = 0; i < kCopyPiece / 16 / kCopyThreads; ++i)
            if (i * kCopyThreads + static_cast<int>(threadIdx.x) < units) x[i] = __ldcs(a + i * kCopyThreads + threadIdx.x);
#pragma unroll
        for (int i = 0; i < kCopyPiece / 16 / kCopyThreads; ++i)
            if (i * kCopyThreads + static_cast<int>(threadIdx.x) < units) __stcs(z + i * kCopyThreads + threadIdx.x, x[i]);
    }
}

// One block.  The table entries that rows give up are numbered in order of rows, then of positions; a page whose count reaches
// zero is pushed by its lowest number, which an atomic minimum in the count itself finds.  First a thread per row moves the
// lengths on and looks whether there is anything behind them: mostly there is not, and the call ends after one chain of loads.
// Otherwise the given-up entries are worked on one per thread, found by a binary search among the rows' first numbers.
//
// Between the new and the old length any entry may be absent (positions committed after a refused reserve, pages that the caller
// evicted), so all of them are given up.  What lies behind the old length was reserved from there on without a gap, so its end is
// the first absent entry, and the rest of the table is not read.
__global__ void __launch_bounds__(kPageThreads) commit_kernel(CacheView c, int B, const int32_t* streams, const int32_t* n_keep) {
    const PageScratch sc = page_scratch(c);
    extern __shared__ int begin[];          // [rows that give up pages + 1]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_free = c.meta[0];
    int rows = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        const int s = b < B ? c.stream_of(streams, b) : -1;
        int keep = c.max_pages, held = 0;
        bool gives = false;
        if (s >= 0) {
            const int old = c.length_of(s);
            const int64_t len = min(max(static_cast<int64_t>(old) + n_keep[b], int64_t(0)), static_cast<int64_t>(c.capacity()));
            keep = static_cast<int>((len + c.page_tokens() - 1) >> c.log_p);
            held = (old + c.page_tokens() - 1) >> c.log_p;
            gives = keep < held || (keep < c.max_pages && c.page_at(s, keep) >= 0);
            c.seq_len[s] = static_cast<int>(len);
        }
        if (!__syncthreads_or(gives)) continue;
        int total;
        const int at = rows + block_scan(gives, &total);
        if (gives) {
            sc.row_a[at] = s;
            sc.row_b[at] = keep;
            sc.row_c[at] = max(keep, held);
        }
        rows += total;
    }
    if (rows == 0) return;
    __syncthreads();
    // how many: up to the old length, and behind it up to the first absent entry
    for (int k = warp; k < rows; k += kPageThreads / 32) {
        const int s = sc.row_a[k], held = sc.row_c[k];
        int gone = held - sc.row_b[k];
        for (int i0 = held; i0 < c.max_pages; i0 += 128) {
            unsigned none[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * 32 + lane;
                none[u] = __ballot_sync(0xffffffffu, i >= c.max_pages || c.page_at(s, min(i, c.max_pages - 1)) < 0);
            }
            int n = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (n == u * 32) n += none[u] ? __ffs(none[u]) - 1 : 32;
            gone += n;
            if (n < 128) break;
        }
        if (lane == 0) begin[k] = gone;
    }
    __syncthreads();
    int all = 0;
    for (int k0 = 0; k0 < rows; k0 += kPageThreads) {
        const int k = k0 + threadIdx.x;
        int total;
        const int at = block_scan(k < rows ? begin[k] : 0, &total);
        if (k < rows) begin[k] = all + at;
        all += total;
    }
    if (threadIdx.x == 0) begin[rows] = all;
    __syncthreads();
    auto entry = [&](int e) -> int32_t* {   // given-up table entry e
        int lo = 0, hi = rows - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (begin[mid] <= e) lo = mid;
            else hi = mid - 1;
        }
        return c.row(sc.row_a[lo]) + sc.row_b[lo] + (e - begin[lo]);
    };
    auto page_of = [&](const int32_t* at) -> int {   // -1: absent
        const int page = *at;
        return static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages) ? page : -1;
    };
#pragma unroll 4
    for (int e = threadIdx.x; e < all; e += kPageThreads) {
        const int page = page_of(entry(e));
        if (page >= 0) atomicSub(&c.ref[page], 1);
    }
    __syncthreads();
#pragma unroll 4
    for (int e = threadIdx.x; e < all; e += kPageThreads) {
        const int page = page_of(entry(e));
        if (page >= 0 && __ldcg(&c.ref[page]) <= 0) atomicMin(&c.ref[page], e - kClaim);
    }
    __syncthreads();
    int pushed = 0;
    for (int e0 = 0; e0 < all; e0 += kPageThreads) {
        const int e = e0 + threadIdx.x;
        const int page = e < all ? page_of(entry(e)) : -1;
        const bool mine = page >= 0 && __ldcg(&c.ref[page]) == e - kClaim;
        int total;
        const int at = n_free + pushed + block_scan(mine, &total);
        if (mine && at < c.n_pages) c.free_list[at] = page;
        pushed += total;
    }
    __syncthreads();
#pragma unroll 4
    for (int e = threadIdx.x; e < all; e += kPageThreads) {
        int32_t* at = entry(e);
        const int page = page_of(at);
        if (page >= 0 && __ldcg(&c.ref[page]) < 0) c.ref[page] = 0;
        *at = -1;
    }
    if (threadIdx.x == 0) c.meta[0] = min(n_free + pushed, c.n_pages);
}

// One block per pair.
__global__ void __launch_bounds__(256) fork_kernel(CacheView c, const int32_t* src, const int32_t* dst) {
    const int a = src[blockIdx.x], z = dst[blockIdx.x];
    const bool known = static_cast<unsigned>(a) < static_cast<unsigned>(c.n_streams) && static_cast<unsigned>(z) < static_cast<unsigned>(c.n_streams);
    bool taken = !known || a == z || c.seq_len[z] != 0;
    if (!taken) {   // a page anywhere in the row would be lost
#pragma unroll 4
        for (int i = threadIdx.x; i < c.max_pages; i += blockDim.x) taken |= c.row(z)[i] != -1;
    }
    const int len = known ? c.length_of(a) : 0, held = (len + c.page_tokens() - 1) >> c.log_p;
    if (__syncthreads_or(taken)) {
        if (threadIdx.x == 0) atomicOr(&c.meta[1], kStatusBadFork);
        return;
    }
    for (int i = threadIdx.x; i < held; i += blockDim.x) {
        const int page = c.page_at(a, i);
        c.row(z)[i] = page;
        if (page >= 0) atomicAdd(&c.ref[page], 1);
    }
    if (threadIdx.x == 0) c.seq_len[z] = len;
}

// One block: ranks the pages, lists the moves and where each page will be, and moves the counts.  A thread has eight pages in
// each round, so that a pool of 30,000 pages takes four.
constexpr int kPlanPages = 8;
__global__ void __launch_bounds__(kPageThreads) compact_plan_kernel(CacheView c) {
    const PageScratch sc = page_scratch(c);
    __shared__ int boundary;
    constexpr int kRound = kPageThreads * kPlanPages;
    auto live_bits = [&](int p) {          // of pages p .. p + 7
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < kPlanPages; ++i) m |= static_cast<unsigned>(p + i < c.n_pages && c.ref[min(p + i, c.n_pages - 1)] > 0) << i;
        return m;
    };
    int mine = 0;
    for (int p0 = 0; p0 < c.n_pages; p0 += kRound) mine += __popc(live_bits(p0 + threadIdx.x * kPlanPages));
    const int live = block_sum(mine);
    if (threadIdx.x == 0) boundary = live;  // live pages below page `live`; that many when there is no such page
    int below = 0;
    for (int p0 = 0; p0 < c.n_pages; p0 += kRound) {
        const int p = p0 + threadIdx.x * kPlanPages;
        const unsigned m = live_bits(p);
        int total;
        const int rank = below + block_scan(__popc(m), &total);   // live pages below p
        if (p <= live && live < p + kPlanPages) boundary = rank + __popc(m & ((1u << (live - p)) - 1));
        __syncthreads();
        const int edge = boundary;
#pragma unroll
        for (int i = 0; i < kPlanPages; ++i) {
            if (p + i >= c.n_pages) break;
            const int r = rank + __popc(m & ((1u << i) - 1));
            const bool on = (m >> i) & 1;
            if (on && p + i >= live) sc.from[r - edge] = p + i;
            if (!on && p + i < live) sc.to[p + i - r] = p + i;
            sc.remap[p + i] = p + i;
        }
        below += total;
    }
    __syncthreads();
    const int moves = live - boundary;
    for (int k = threadIdx.x; k < moves; k += kPageThreads) {
        const int f = sc.from[k], t = sc.to[k];
        sc.remap[f] = t;
        c.ref[t] = c.ref[f];
        c.ref[f] = 0;
    }
    const int n_free = c.n_pages - live;
    for (int i = threadIdx.x; i < n_free; i += kPageThreads) c.free_list[i] = c.n_pages - 1 - i;
    if (threadIdx.x == 0) {
        c.meta[0] = n_free;
        *sc.count = moves;
    }
}

__global__ void __launch_bounds__(256) compact_tables_kernel(CacheView c) {
    const PageScratch sc = page_scratch(c);
    const int64_t n = static_cast<int64_t>(c.n_streams) * c.max_pages;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
        const int p = c.table[i];
        if (static_cast<unsigned>(p) < static_cast<unsigned>(c.n_pages)) c.table[i] = sc.remap[p];
    }
}

}  // namespace samb200
