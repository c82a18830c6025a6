// Page bookkeeping of the 4-bit cache: reserve (with copy on write), commit / roll back, fork, compact, whole-page copies.
//
// Every result is independent of timing: pages are handed out and given back by prefix sums over rows and positions, and
// where several rows name one page, integer atomics decide by row number.
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
    int32_t* from;      // [max(n_streams, n_pages)]
    int32_t* to;
    int32_t* remap;     // [n_pages]
};
__host__ __device__ inline int64_t page_scratch_ints(int64_t n_streams, int64_t n_pages) {
    const int64_t list = n_streams > n_pages ? n_streams : n_pages;
    return kScratchHead + 2 * n_streams + 2 * list + n_pages;
}
__device__ __forceinline__ PageScratch page_scratch(const CacheView& c) {
    const int64_t list = max(c.n_streams, c.n_pages);
    PageScratch s;
    s.count = c.scratch;
    s.row_a = c.scratch + kScratchHead;
    s.row_b = s.row_a + c.n_streams;
    s.from = s.row_b + c.n_streams;
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

// One block.  Row state kept in scratch between the phases: row_a = the page to be copied (or -1), row_b = 1 when this
// row keeps a page whose count the phases have taken to zero.
__global__ void __launch_bounds__(kPageThreads) reserve_kernel(CacheView c, int B, const int32_t* streams, const int32_t* n_new) {
    const PageScratch sc = page_scratch(c);
    __shared__ int bad, copies;
    if (threadIdx.x == 0) bad = copies = 0;
    __syncthreads();
    // writers of a page leave it: a count of zero means that all its holders write
    for (int b = threadIdx.x; b < B; b += kPageThreads) {
        const RowNeed r = row_need(c, streams, n_new, b);
        if (r.want > c.max_pages) bad = 1;
        if (r.page0 >= 0) atomicSub(&c.ref[r.page0], 1);
        sc.row_a[b] = r.page0;
    }
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += kPageThreads) sc.row_b[b] = sc.row_a[b] >= 0 && __ldcg(&c.ref[sc.row_a[b]]) == 0;
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += kPageThreads)
        if (sc.row_b[b]) atomicMax(&c.ref[sc.row_a[b]], b + 1);
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += kPageThreads)
        if (sc.row_b[b]) sc.row_b[b] = __ldcg(&c.ref[sc.row_a[b]]) == b + 1 ? 2 : 1;   // 2: the last of them, which keeps the page
    __syncthreads();
    int need_all = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        int need = 0;
        if (b < B) {
            const RowNeed r = row_need(c, streams, n_new, b);
            need = r.page0 >= 0 && sc.row_b[b] != 2;
            for (int i = r.first; i < min(r.want, c.max_pages); ++i) need += c.page_at(r.s, i) < 0;
        }
        int total;
        block_scan(need, &total);
        need_all += total;
    }
    const int n_free = c.meta[0];
    const bool ok = !bad && need_all <= n_free;
    __syncthreads();
    if (!ok) {   // put the counts back
        for (int b = threadIdx.x; b < B; b += kPageThreads)
            if (sc.row_b[b] == 2) c.ref[sc.row_a[b]] = 0;
        __syncthreads();
        for (int b = threadIdx.x; b < B; b += kPageThreads)
            if (sc.row_a[b] >= 0) atomicAdd(&c.ref[sc.row_a[b]], 1);
        if (threadIdx.x == 0) {
            c.meta[1] |= bad ? kStatusTableFull : kStatusOutOfPages;
            *sc.count = 0;
        }
        return;
    }
    int before = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        RowNeed r;
        r.s = -1;
        r.first = r.want = 0;
        int need = 0;
        bool copy = false;
        if (b < B) {
            r = row_need(c, streams, n_new, b);
            if (r.page0 >= 0 && sc.row_b[b] == 2) c.ref[r.page0] = 1;
            copy = r.page0 >= 0 && sc.row_b[b] != 2;
            need = copy;
            for (int i = r.first; i < r.want; ++i) need += c.page_at(r.s, i) < 0;
        }
        int total;
        int at = n_free - 1 - before - block_scan(need, &total);
        before += total;
        for (int i = r.first; i < r.want; ++i) {
            const bool replace = copy && i == r.first;
            if (!replace && c.page_at(r.s, i) >= 0) continue;
            const int page = c.free_list[at--];
            if (replace) {
                const int k = atomicAdd(&copies, 1);   // the order of the copies does not matter
                sc.from[k] = r.page0;
                sc.to[k] = page;
            }
            c.row(r.s)[i] = page;
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

// One block, a warp per row.  The pages that a row gives up are numbered in order of rows, then of positions; a page
// whose count reaches zero is pushed by its lowest number, which the warps find by an atomic minimum in the count itself.
__global__ void __launch_bounds__(kPageThreads) commit_kernel(CacheView c, int B, const int32_t* streams, const int32_t* n_keep) {
    const PageScratch sc = page_scratch(c);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kPageThreads / 32;
    auto keep_pages = [&](int s) { return (c.seq_len[s] + c.page_tokens() - 1) >> c.log_p; };

    for (int b = warp; b < B; b += kWarps) {
        const int s = c.stream_of(streams, b);
        int gone = 0;
        if (s >= 0) {
            const int64_t len = min(max(static_cast<int64_t>(c.length_of(s)) + n_keep[b], int64_t(0)), static_cast<int64_t>(c.capacity()));
            __syncwarp();
            if (lane == 0) c.seq_len[s] = static_cast<int>(len);
            const int keep = static_cast<int>((len + c.page_tokens() - 1) >> c.log_p);
            for (int i0 = keep; i0 < c.max_pages; i0 += 32) {
                const int page = i0 + lane < c.max_pages ? c.page_at(s, i0 + lane) : -1;
                const unsigned none = __ballot_sync(0xffffffffu, page < 0);
                const int n = none ? __ffs(none) - 1 : 32;
                if (lane < n) atomicSub(&c.ref[page], 1);
                gone += n;
                if (n < 32) break;
            }
        }
        if (lane == 0) sc.row_a[b] = gone;
    }
    __syncthreads();
    // numbers of the rows' first given-up pages
    int base = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        int total;
        const int at = block_scan(b < B ? sc.row_a[b] : 0, &total);
        if (b < B) sc.row_b[b] = base + at;
        base += total;
    }
    if (base == 0) return;
    __syncthreads();
    for (int b = warp; b < B; b += kWarps) {
        const int gone = sc.row_a[b];
        if (!gone) continue;
        const int s = c.stream_of(streams, b), keep = keep_pages(s);
        for (int i = lane; i < gone; i += 32) {
            const int page = c.page_at(s, keep + i);
            if (__ldcg(&c.ref[page]) <= 0) atomicMin(&c.ref[page], sc.row_b[b] + i - kClaim);
        }
    }
    __syncthreads();
    for (int b = warp; b < B; b += kWarps) {
        const int gone = sc.row_a[b];
        int freed = 0;
        if (gone) {
            const int s = c.stream_of(streams, b), keep = keep_pages(s);
            for (int i = lane; i < gone; i += 32) freed += __ldcg(&c.ref[c.page_at(s, keep + i)]) == sc.row_b[b] + i - kClaim;
            freed = __reduce_add_sync(0xffffffffu, freed);
        }
        if (lane == 0) sc.to[b] = freed;
    }
    __syncthreads();
    const int n_free = c.meta[0];
    int pushed = 0;
    for (int b0 = 0; b0 < B; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        int total;
        const int at = block_scan(b < B ? sc.to[b] : 0, &total);
        if (b < B) sc.from[b] = n_free + pushed + at;
        pushed += total;
    }
    __syncthreads();
    for (int b = warp; b < B; b += kWarps) {
        const int gone = sc.row_a[b];
        if (!gone) continue;
        const int s = c.stream_of(streams, b), keep = keep_pages(s);
        int at = sc.from[b];
        for (int i0 = 0; i0 < gone; i0 += 32) {
            const int i = i0 + lane;
            const int page = i < gone ? c.page_at(s, keep + i) : -1;
            const bool mine = page >= 0 && __ldcg(&c.ref[page]) == sc.row_b[b] + i - kClaim;
            const unsigned m = __ballot_sync(0xffffffffu, mine);
            const int k = at + __popc(m & ((1u << lane) - 1));
            if (mine && k < c.n_pages) c.free_list[k] = page;
            at += __popc(m);
        }
    }
    __syncthreads();
    for (int b = warp; b < B; b += kWarps) {
        const int gone = sc.row_a[b];
        if (!gone) continue;
        const int s = c.stream_of(streams, b), keep = keep_pages(s);
        for (int i = lane; i < gone; i += 32) {
            const int page = c.page_at(s, keep + i);
            if (__ldcg(&c.ref[page]) < 0) c.ref[page] = 0;
            c.row(s)[keep + i] = -1;
        }
    }
    if (threadIdx.x == 0) c.meta[0] = min(n_free + pushed, c.n_pages);
}

// One block per pair.
__global__ void __launch_bounds__(256) fork_kernel(CacheView c, const int32_t* src, const int32_t* dst) {
    const int a = src[blockIdx.x], z = dst[blockIdx.x];
    const bool known = static_cast<unsigned>(a) < static_cast<unsigned>(c.n_streams) && static_cast<unsigned>(z) < static_cast<unsigned>(c.n_streams);
    if (!known || a == z || c.seq_len[z] != 0 || c.row(z)[0] != -1) {
        if (threadIdx.x == 0) atomicOr(&c.meta[1], kStatusBadFork);
        return;
    }
    const int len = c.length_of(a), held = (len + c.page_tokens() - 1) >> c.log_p;
    __syncthreads();
    for (int i = threadIdx.x; i < held; i += blockDim.x) {
        const int page = c.page_at(a, i);
        c.row(z)[i] = page;
        if (page >= 0) atomicAdd(&c.ref[page], 1);
    }
    if (threadIdx.x == 0) c.seq_len[z] = len;
}

// One block: ranks the pages, lists the moves and where each page will be, and moves the counts.
__global__ void __launch_bounds__(kPageThreads) compact_plan_kernel(CacheView c) {
    const PageScratch sc = page_scratch(c);
    int live = 0;
    for (int p0 = 0; p0 < c.n_pages; p0 += kPageThreads) {
        const int p = p0 + threadIdx.x;
        live += __syncthreads_count(p < c.n_pages && c.ref[p] > 0);
    }
    int below = 0, at_boundary = 0;   // live pages below p0; below `live`
    for (int p0 = 0; p0 < c.n_pages; p0 += kPageThreads) {
        const int p = p0 + threadIdx.x;
        const bool on = p < c.n_pages && c.ref[p] > 0;
        int total;
        const int rank = below + block_scan(on, &total);   // live pages below p
        if (live >= p0 && live < p0 + kPageThreads) {
            __shared__ int r;
            if (p == live) r = rank;
            __syncthreads();
            at_boundary = r;
        }
        if (p < c.n_pages) {
            if (on && p >= live) sc.from[rank - at_boundary] = p;
            if (!on && p < live) sc.to[p - rank] = p;
            sc.remap[p] = p;
        }
        below += total;
    }
    __syncthreads();
    const int moves = live == c.n_pages ? 0 : live - at_boundary;
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
