// Which blocks (pages) of its context a query reads: bounds of the keys of each page, a score from them, the best pages.
//
// Bounds: for a page, layer and head the largest and the smallest key of every channel as 8-bit codes with one power of two,
// the largest rounded up and the smallest down.  A channel adds at most max(q max, q min) to q.k; with q in 8 bits too, the sum
// over the channels is <q+, max> + <q-, min> (q+ and q- the positive and the negative part): a product of whole numbers below
// 2^22 in magnitude, exact in 32 bits, so that equal scores are equal wherever and in whatever order they are computed.
#pragma once

#include "cache_attend.cuh"
#include "cache_format.cuh"

namespace samb200 {

constexpr int kNanPage = 127;            // exponent of a page with a NaN among its keys
constexpr uint32_t kForced = 0xffffffffu, kNanKey = 0xfffffffeu;   // keys of pages that are listed before all others

struct BoundsView {
    int8_t* codes;     // [n_pages, n_layers, n_kv, 2, D]: largest, smallest
    int8_t* exps;      // [n_pages, n_layers, n_kv]
};

// ---- bounds
constexpr int kBoundThreads = 128;

// e with amax <= 127 * 2^e, amax > 63 * 2^e, from the bits of a positive normal number.
__device__ __forceinline__ int eight_bit_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    return static_cast<int>(u >> 23) - 126 - 6 - ((u & 0x7fffff) <= 0x7e0000);
}

// Bounds of one page, layer and head, by the whole block.  A thread has eight channels of every (16 or 32 threads apart) token.
__device__ __forceinline__ void bound_page(const CacheView& c, const BoundsView& o, int page, int layer, int head) {
    __shared__ __half2 high[kBoundThreads][5], low[kBoundThreads][5];
    const int words = c.D >> 3, groups = kBoundThreads / words, w = threadIdx.x % words, g = threadIdx.x / words;
    const uint8_t* tiles = c.head_tiles(page, layer, head);
    __half2 hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        hi[i] = __half2half2(__ushort_as_half(0xfc00));   // -inf
        lo[i] = __half2half2(__ushort_as_half(0x7c00));
    }
    bool nan = false;
#pragma unroll 4
    for (int t = g; t < c.page_tokens(); t += groups) {
        const uint8_t* tile = tiles + (t >> 4) * c.tile_bytes();
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(tile + (t & 15) * (c.D >> 1) + w * 4);
        const uint32_t scale = tile[16 * c.D + (t & 15) * (c.D >> 4) + (w >> 1)];
        nan |= (scale & 0x7f) == 0x7f;
        uint32_t x[4];
        e2m1x8_to_half2(codes, x);
        const uint32_t f = e4m3x2_to_half2(scale * 0x0101u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&x[i]), *reinterpret_cast<const __half2*>(&f));   // exact
            hi[i] = __hmax2(hi[i], y);
            lo[i] = __hmin2(lo[i], y);
        }
    }
    __syncthreads();                                      // the last page's are read
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        high[threadIdx.x][i] = hi[i];
        low[threadIdx.x][i] = lo[i];
    }
    nan = __syncthreads_or(nan);
    float amax = 0.f;
    if (threadIdx.x < words) {
        for (int k = 1; k < groups; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[i] = __hmax2(hi[i], high[k * words + w][i]);
                lo[i] = __hmin2(lo[i], low[k * words + w][i]);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 y = __half22float2(hi[i]), z = __half22float2(lo[i]);
            amax = fmaxf(amax, fmaxf(fmaxf(fabsf(y.x), fabsf(y.y)), fmaxf(fabsf(z.x), fabsf(z.y))));
        }
    }
    if (threadIdx.x < 32) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
        const int64_t at = (static_cast<int64_t>(page) * c.n_layers + layer) * c.n_kv + head;
        const int e = amax > 0.f ? eight_bit_exponent(amax) : 0;
        const float down = nan ? 0.f : pow2(-e);
        if (threadIdx.x < words) {
            uint32_t up[2] = {0, 0}, dn[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = __half22float2(hi[i]), z = __half22float2(lo[i]);
                if (!nan) {
                    up[i >> 1] |= ((static_cast<int>(ceilf(y.x * down)) & 255) | (static_cast<int>(ceilf(y.y * down)) & 255) << 8) << (16 * (i & 1));
                    dn[i >> 1] |= ((static_cast<int>(floorf(z.x * down)) & 255) | (static_cast<int>(floorf(z.y * down)) & 255) << 8) << (16 * (i & 1));
                }
            }
            uint2* out = reinterpret_cast<uint2*>(o.codes + at * 2 * c.D);
            out[w] = make_uint2(up[0], up[1]);
            out[words + w] = make_uint2(dn[0], dn[1]);
        }
        if (threadIdx.x == 0) o.exps[at] = static_cast<int8_t>(nan ? kNanPage : amax > 0.f ? e + c.k_exp : 0);
    }
}

// Pages that the new tokens fill up.  Grid: (heads, rows, pages of a row).
__global__ void __launch_bounds__(kBoundThreads) bounds_update_kernel(CacheView c, BoundsView o, int layer, int Q, const int32_t* streams, const int32_t* n_new) {
    const int b = blockIdx.y;
    const int s = c.stream_of(streams, b);
    if (s < 0) return;
    const int n = max(n_new ? min(n_new[b], Q) : Q, 0), len = c.length_of(s);
    const int end = static_cast<int>(min(static_cast<int64_t>(len) + n, static_cast<int64_t>(c.capacity()))) >> c.log_p;
    for (int i = (len >> c.log_p) + blockIdx.z; i < end; i += gridDim.z) {
        const int page = c.page_at(s, i);
        if (page >= 0) bound_page(c, o, page, layer, blockIdx.x);
    }
}

// All layers and heads of listed pages (null: of every page).  Grid: any.
__global__ void __launch_bounds__(kBoundThreads) bounds_rebuild_kernel(CacheView c, BoundsView o, int n, const int32_t* pages) {
    const int64_t all = static_cast<int64_t>(n) * c.n_layers * c.n_kv;
    for (int64_t e = blockIdx.x; e < all; e += gridDim.x) {
        const int head = static_cast<int>(e % c.n_kv), layer = static_cast<int>(e / c.n_kv % c.n_layers), i = static_cast<int>(e / c.n_kv / c.n_layers);
        const int page = pages ? pages[i] : i;
        if (static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages)) bound_page(c, o, page, layer, head);
    }
}

// ---- scores
struct SelectArgs {
    CacheView c;
    BoundsView o;
    const void* q;
    const int32_t* streams;
    const int32_t* n_new;
    int64_t q_row, q_token, q_head;
    int32_t layer, B, Q, H, group;
    int32_t lists, share, n_blocks, n_sink, n_recent;
    int64_t first_run;           // of this launch: run v is list v % lists of row v / lists
    int32_t runs;
    uint32_t* keys;              // [runs, n_kv, max_pages]
    int32_t* out;                // [B, lists, n_kv, n_blocks]
    bool q_wide;
};

// A run of query tokens with a list in common.
struct SelectRun {
    int s, n;          // stream, -1 = unknown; query tokens in use
    int pages;         // blocks up to the last query's own, within the table
    int old;           // blocks [n_sink, old) are scored, those behind are listed
    int b, i0;
};
__device__ __forceinline__ SelectRun select_run(const SelectArgs& a, int64_t v) {
    SelectRun r;
    r.b = static_cast<int>(quotient(v, a.lists));
    r.i0 = static_cast<int>(v - static_cast<int64_t>(r.b) * a.lists) * a.share;
    r.s = a.c.stream_of(a.streams, r.b);
    r.n = r.s < 0 ? 0 : min(max((a.n_new ? min(a.n_new[r.b], a.Q) : a.Q) - r.i0, 0), a.share);
    const int64_t first = r.s < 0 ? 0 : static_cast<int64_t>(a.c.length_of(r.s)) + r.i0;
    r.pages = r.n > 0 ? static_cast<int>(min(((first + r.n - 1) >> a.c.log_p) + 1, static_cast<int64_t>(a.c.max_pages))) : 0;
    r.old = static_cast<int>(min(max((first >> a.c.log_p) + 1 - a.n_recent, int64_t(0)), static_cast<int64_t>(r.pages)));
    return r;
}

// Monotone in the float: larger keys for larger scores; 1 or more, and below the keys that go first.
__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int kScoreThreads = 256, kScoreColumns = 64;   // query rows in shared memory at a time

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Keys of the pages of one run and head: sixteen pages of a warp are the M side, eight query rows the N side.
// Grid: (shares of the pages, heads, runs).
template <typename T, int D>
__global__ void __launch_bounds__(kScoreThreads) select_score_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int kStride = 2 * D + 64;                   // of a column in shared memory: two columns fill all banks
    constexpr int kParts = 2 * D / 64;                    // sixteen-byte parts of a row or column that a thread has
    __shared__ alignas(16) uint8_t columns[kScoreColumns * kStride];
    __shared__ float unit[kScoreColumns];
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, j = lane & 3;
    const int head = blockIdx.y;
    const SelectRun run = select_run(a, a.first_run + blockIdx.z);
    if (run.pages == 0) return;
    const bool scored = run.pages > a.n_blocks;           // else all of them are listed
    uint32_t* keys = a.keys + (static_cast<int64_t>(blockIdx.z) * c.n_kv + head) * c.max_pages;
    const int rows = run.n * a.group, step = gridDim.x * (kScoreThreads / 2);
    for (int col0 = 0; col0 == 0 || (scored && col0 < rows); col0 += kScoreColumns) {
        const int cols = min(rows - col0, kScoreColumns), tiles = (cols + 7) >> 3;
        __syncthreads();
        if (scored) {
            // queries in eight bits, their positive and their negative parts: a warp takes a row
            for (int n = warp; n < tiles * 8; n += kScoreThreads / 32) {
                float x[D / 32];
#pragma unroll
                for (int k = 0; k < D / 32; ++k) x[k] = 0.f;
                if (n < cols) {
                    const int rho = col0 + n;
                    const T* q = static_cast<const T*>(a.q) + run.b * a.q_row + (run.i0 + rho / a.group) * a.q_token +
                                 (head * a.group + rho % a.group) * a.q_head + lane * (D / 32);
                    if (a.q_wide) {
                        alignas(8) T y[D / 32];
                        if constexpr (D == 128) *reinterpret_cast<uint2*>(y) = __ldg(reinterpret_cast<const uint2*>(q));
                        else *reinterpret_cast<uint32_t*>(y) = __ldg(reinterpret_cast<const uint32_t*>(q));
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) x[k] = Elem<T>::to_float(y[k]);
                    } else {
#pragma unroll
                        for (int k = 0; k < D / 32; ++k) x[k] = Elem<T>::to_float(q[k]);
                    }
                }
                float big = 0.f;                          // of the finite ones
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const float y = fabsf(x[k]);
                    if (y < INFINITY) big = fmaxf(big, y);
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
                const int e = big >= 1.17549435e-38f ? max(eight_bit_exponent(big), -100) : 0;
                uint32_t up = 0, dn = 0;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    const int y = x[k] == x[k] ? __float2int_rn(fminf(fmaxf(x[k] * pow2(-e), -127.f), 127.f)) : 0;
                    up |= static_cast<uint32_t>(max(y, 0)) << (8 * k);
                    dn |= static_cast<uint32_t>(min(y, 0) & 255) << (8 * k);
                }
                uint8_t* col = columns + n * kStride + lane * (D / 32);
                if constexpr (D == 128) {
                    *reinterpret_cast<uint32_t*>(col) = up;
                    *reinterpret_cast<uint32_t*>(col + D) = dn;
                } else {
                    *reinterpret_cast<uint16_t*>(col) = static_cast<uint16_t>(up);
                    *reinterpret_cast<uint16_t*>(col + D) = static_cast<uint16_t>(dn);
                }
                if (lane == 0) unit[n] = n < cols ? pow2(e) : 0.f;
            }
            __syncthreads();
        }
        for (int i0 = (blockIdx.x * (kScoreThreads / 32) + warp) * 16; i0 < run.pages; i0 += step) {
            // pages i0 + r and + 8: what there is, and their keys
            int page[2];
            uint32_t key[2];
            float size[2];
            uint4 x[2][kParts];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = i0 + r + 8 * h;
                page[h] = i < run.pages ? c.page_at(run.s, i) : -1;
                key[h] = page[h] < 0 ? 0u : !scored || i < a.n_sink || i >= run.old ? kForced : 1u;
                size[h] = 0.f;
                const int64_t at = (static_cast<int64_t>(max(page[h], 0)) * c.n_layers + a.layer) * c.n_kv + head;
#pragma unroll
                for (int k = 0; k < kParts; ++k) x[h][k] = make_uint4(0, 0, 0, 0);
                if (key[h] == 1u) {
                    const int e = a.o.exps[at];
                    if (e == kNanPage) key[h] = kNanKey;
                    size[h] = pow2(e == kNanPage ? 0 : e);
#pragma unroll
                    for (int k = 0; k < kParts; ++k) x[h][k] = __ldg(reinterpret_cast<const uint4*>(a.o.codes + at * 2 * D) + k * 4 + j);
                }
            }
            if (__any_sync(0xffffffffu, key[0] == 1u || key[1] == 1u)) {
                float best[2] = {-INFINITY, -INFINITY};
                for (int t = 0; t < tiles; ++t) {
                    int acc[4] = {0, 0, 0, 0};
                    const uint8_t* col = columns + (t * 8 + r) * kStride + j * 16;
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        const uint4 y = *reinterpret_cast<const uint4*>(col + k * 64);
                        mma_s8(acc, x[0][k].x, x[1][k].x, x[0][k].y, x[1][k].y, y.x, y.y);
                        mma_s8(acc, x[0][k].z, x[1][k].z, x[0][k].w, x[1][k].w, y.z, y.w);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int n = t * 8 + 2 * j + k;
                        if (n < cols) {
                            best[0] = fmaxf(best[0], static_cast<float>(acc[k]) * unit[n]);
                            best[1] = fmaxf(best[1], static_cast<float>(acc[2 + k]) * unit[n]);
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    best[h] = fmaxf(best[h], __shfl_xor_sync(0xffffffffu, best[h], 1));
                    best[h] = fmaxf(best[h], __shfl_xor_sync(0xffffffffu, best[h], 2));
                    if (key[h] == 1u) key[h] = score_key(best[h] * size[h]);
                }
            }
            if (j < 2) {                                  // lane j = 0: page r, j = 1: page r + 8
                const int i = i0 + r + 8 * j;
                const uint32_t y = j ? key[1] : key[0];
                if (i < run.pages) keys[i] = col0 == 0 ? y : max(keys[i], y);
            }
        }
    }
}

// ---- the best pages of a run and head: the n_blocks-th largest key by eight bits at a time, then all pages above it and the first of
// those that equal it, in order.
constexpr int kPickThreads = 256, kPickKeep = 4096;      // keys in shared memory

// Exclusive prefix sum of two counts below 2^31 over the block; *total gets the sums.
__device__ __forceinline__ int2 block_scan2(int2 x, int2* total) {
    __shared__ int2 sums[kPickThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, y.x, d), v = __shfl_up_sync(0xffffffffu, y.y, d);
        if (lane >= d) {
            y.x += u;
            y.y += v;
        }
    }
    __syncthreads();
    if (lane == 31) sums[warp] = y;
    __syncthreads();
    int2 before = make_int2(0, 0), all = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < kPickThreads / 32; ++w) {
        if (w == warp) before = all;
        all.x += sums[w].x;
        all.y += sums[w].y;
    }
    *total = all;
    return make_int2(before.x + y.x - x.x, before.y + y.y - x.y);
}

// Grid: (heads, runs).
__global__ void __launch_bounds__(kPickThreads) select_pick_kernel(const __grid_constant__ SelectArgs a) {
    __shared__ uint32_t kept[kPickKeep];
    __shared__ int bins[256];
    __shared__ uint32_t chosen;
    __shared__ int above;
    const CacheView& c = a.c;
    const int tid = threadIdx.x, head = blockIdx.x;
    const SelectRun run = select_run(a, a.first_run + blockIdx.y);
    int32_t* out = a.out + ((a.first_run + blockIdx.y) * c.n_kv + head) * a.n_blocks;
    const uint32_t* keys = a.keys + (static_cast<int64_t>(blockIdx.y) * c.n_kv + head) * c.max_pages;
    const int n = run.pages;
    const bool keep = n <= kPickKeep;
    if (keep)
        for (int i = tid; i < n; i += kPickThreads) kept[i] = keys[i];
    __syncthreads();
    auto key = [&](int i) { return keep ? kept[i] : keys[i]; };
    // the key of the last page that is listed, and how many with that key are
    uint32_t limit = 1;
    int ties = a.n_blocks;
    if (n > a.n_blocks) {
        uint32_t prefix = 0, mask = 0;
        int want = a.n_blocks;                            // from the keys that begin with the prefix
        for (int shift = 24; shift >= 0; shift -= 8) {
            bins[tid] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += kPickThreads) {
                const uint32_t k = key(i);
                if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & 255], 1);
            }
            __syncthreads();
            int2 total;
            const int mine = bins[255 - tid];
            const int before = block_scan2(make_int2(mine, 0), &total).x;   // keys in higher bins
            if (before < want && before + mine >= want) {
                chosen = 255 - tid;
                above = before;
            }
            __syncthreads();
            prefix |= chosen << shift;
            mask |= 255u << shift;
            want -= above;
            __syncthreads();
        }
        limit = prefix;
        ties = want;
        if (limit == 0) {                                 // fewer pages present than wanted
            limit = 1;
            ties = a.n_blocks;
        }
    }
    // in order: a thread takes neighbouring pages
    const int each = (n + kPickThreads - 1) / kPickThreads, i0 = min(tid * each, n), i1 = min(i0 + each, n);
    int2 count = make_int2(0, 0);
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = key(i);
        count.x += k > limit;
        count.y += k == limit;
    }
    int2 total;
    const int2 before = block_scan2(count, &total);
    int greater = before.x, equal = before.y;
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = key(i);
        if (k > limit || (k == limit && equal < ties)) {
            const int at = greater + min(equal, ties);
            if (at < a.n_blocks) out[at] = i;
        }
        greater += k > limit;
        equal += k == limit;
    }
    const int used = min(total.x + min(total.y, ties), a.n_blocks);
    for (int i = used + tid; i < a.n_blocks; i += kPickThreads) out[i] = -1;
}

}  // namespace samb200
