// Which blocks (pages) of its context a query reads: bounds of the keys of each page, a score from them, the best pages.
//
// Bounds: for a page, layer and head the largest and the smallest key of every channel as 8-bit codes with one power of two,
// the largest rounded up and the smallest down.  A channel adds at most max(q max, q min) to q.k; with q in 8 bits too, the sum
// over the channels is <q+, max> + <q-, min> (q+ and q- the positive and the negative part): a product of whole numbers below
// 2^22 in magnitude, exact in 32 bits, so that equal scores are equal wherever and in whatever order they are computed.
#pragma once

#include "attend_wide.cuh"
#include "cache_attend.cuh"
#include "cache_format.cuh"
#include "cache_io.cuh"

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
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the scores' kernel may be placed; it waits for the end of this one
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
    int32_t team, teams;         // lists of a row that are scored together; such teams in a row
    int64_t first_team;          // of this launch
    int64_t key_stride;          // of a list and head: max_pages, rounded up to a multiple of 4
    uint32_t* keys;              // [teams of the launch, team, n_kv, key_stride]
    int32_t* out;                // [B, lists, n_kv, n_blocks]
    bool q_wide;
};

// The kernels of a selection are placed while the one before them ends.  Scores wait for everything before them and only then let
// the picks be placed, so that picks may read whatever scores do not write before they wait themselves.  (64 streams, contexts to 32,768: 40 us -> 35
// with the bounds of their new pages.)
__device__ __forceinline__ void await_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void await_and_release() {
    await_before();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A run of query tokens with a list in common: list l of row b.
struct SelectRun {
    int s, n;          // stream, -1 = unknown; query tokens in use
    int pages;         // blocks up to the last query's own, within the table
    int old;           // blocks [n_sink, old) are scored, those behind are listed
};
__device__ __forceinline__ SelectRun select_run(const SelectArgs& a, int b, int l) {
    SelectRun r;
    const int i0 = l * a.share;
    r.s = a.c.stream_of(a.streams, b);
    r.n = r.s < 0 ? 0 : min(max((a.n_new ? min(a.n_new[b], a.Q) : a.Q) - i0, 0), a.share);
    const int64_t first = r.s < 0 ? 0 : static_cast<int64_t>(a.c.length_of(r.s)) + i0;
    r.pages = r.n > 0 ? static_cast<int>(min(((first + r.n - 1) >> a.c.log_p) + 1, static_cast<int64_t>(a.c.max_pages))) : 0;
    r.old = static_cast<int>(min(max((first >> a.c.log_p) + 1 - a.n_recent, int64_t(0)), static_cast<int64_t>(r.pages)));
    return r;
}

// Monotone in the float: larger keys for larger scores; above 1, and below the keys that go first.
__device__ __forceinline__ uint32_t score_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight bits for a query row of which every one of kLanes lanes has eight channels: codes of the positive and of the negative parts;
// returns the power of two.
template <typename T, int kLanes>
__device__ __forceinline__ int query_codes(const uint4& raw, uint32_t (&up)[2], uint32_t (&dn)[2]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    float x[8], big = 0.f;                                // big: of the finite ones
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = i & 1 ? Pair<T>::hi(w[i >> 1]) : Pair<T>::lo(w[i >> 1]);
        if (fabsf(x[i]) < INFINITY) big = fmaxf(big, fabsf(x[i]));
    }
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
    const int e = big >= 1.17549435e-38f ? max(eight_bit_exponent(big), -100) : 0;
    const float down = pow2(-e);
    up[0] = up[1] = dn[0] = dn[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int y = x[i] == x[i] ? __float2int_rn(fminf(fmaxf(x[i] * down, -127.f), 127.f)) : 0;
        up[i >> 2] |= static_cast<uint32_t>(max(y, 0)) << (8 * (i & 3));
        dn[i >> 2] |= static_cast<uint32_t>(min(y, 0) & 255) << (8 * (i & 3));
    }
    return e;
}
// Eight channels of a query row of a run, from channel `at` on.
template <typename T>
__device__ __forceinline__ uint4 query_part(const SelectArgs& a, int b, int i0, int head, int rho, int at) {
    const T* q = static_cast<const T*>(a.q) + b * a.q_row + (static_cast<int64_t>(i0) + rho / a.group) * a.q_token + (head * a.group + rho % a.group) * a.q_head + at;
    if (a.q_wide) return __ldg(reinterpret_cast<const uint4*>(q));
    const uint16_t* h = reinterpret_cast<const uint16_t*>(q);
    return make_uint4(h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16, h[4] | static_cast<uint32_t>(h[5]) << 16,
                      h[6] | static_cast<uint32_t>(h[7]) << 16);
}

// Keys of the pages of a list and head with up to kFewColumns query rows: the bounds come straight from memory into the fragments of
// m16n8k32 (sixteen pages of a warp are the M side; the order of the summed index is free, so that a thread has sixteen neighbouring
// bytes at a time), the next sixteen pages' while these are multiplied.  A product takes 26 clocks, which is why more rows go another way.
// 64 streams of up to 2,048 pages of 8 heads, four query rows each (148 MB): 24 us.
// Grid: (shares of the pages, heads, lists).
constexpr int kFewThreads = 256, kFewColumns = 16;
template <typename T, int D>
__global__ void __launch_bounds__(kFewThreads) select_score_few_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int kStride = 2 * D + 64;                   // of a column in shared memory: two columns fill all banks
    constexpr int kParts = 2 * D / 64, kLanes = D / 8;    // sixteen-byte parts of a row or column that a thread has; lanes of a query row
    __shared__ alignas(16) uint8_t columns[kFewColumns * kStride];
    __shared__ alignas(8) float unit[kFewColumns];
    await_and_release();
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, j = lane & 3, head = blockIdx.y;
    const int64_t v = a.first_team + blockIdx.z;
    const int b = static_cast<int>(quotient(v, a.lists)), l = static_cast<int>(v - static_cast<int64_t>(b) * a.lists);
    const SelectRun run = select_run(a, b, l);
    const int first = (blockIdx.x * (kFewThreads / 32) + warp) * 16, step = gridDim.x * (kFewThreads / 2);
    const bool scored = run.pages > a.n_blocks;           // else all blocks are listed
    uint32_t* const keys = a.keys + (static_cast<int64_t>(blockIdx.z) * c.n_kv + head) * a.key_stride;
    auto page_of = [&](int i) { return i < run.pages ? c.page_at(run.s, i) : -1; };
    auto fetch = [&](const int (&page)[2], uint4 (&x)[2][kParts], int (&e)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (static_cast<int64_t>(max(page[h], 0)) * c.n_layers + a.layer) * c.n_kv + head;
            e[h] = page[h] < 0 ? 0 : a.o.exps[at];
#pragma unroll
            for (int k = 0; k < kParts; ++k)
                x[h][k] = page[h] < 0 ? make_uint4(0, 0, 0, 0) : __ldg(reinterpret_cast<const uint4*>(a.o.codes + at * 2 * D) + k * 4 + j);
        }
    };
    uint4 next[2][kParts];
    int page[2], next_e[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) page[h] = page_of(first + r + 8 * h);
    if (scored) fetch(page, next, next_e);
    const int rows = run.n * a.group, tiles = (a.share * a.group + 7) >> 3;
    if (scored) {
        // queries in eight bits, their positive and their negative parts: eight channels a lane
        const int n = threadIdx.x / kLanes, part = threadIdx.x % kLanes;
        if (n < kFewColumns) {                            // whole warps
            uint32_t up[2], dn[2];
            const int e = query_codes<T, kLanes>(n < rows ? query_part<T>(a, b, l * a.share, head, n, part * 8) : make_uint4(0, 0, 0, 0), up, dn);
            *reinterpret_cast<uint2*>(columns + n * kStride + part * 8) = make_uint2(up[0], up[1]);
            *reinterpret_cast<uint2*>(columns + n * kStride + D + part * 8) = make_uint2(dn[0], dn[1]);
            if (part == 0) unit[n] = n < rows ? pow2(e) : __int_as_float(0x7fffffff);   // a NaN drops out of the maximum
        }
    }
    __syncthreads();
    for (int i0 = first; i0 < run.pages; i0 += step) {
        // pages i0 + r and + 8, and the next ones
        uint4 x[2][kParts];
        float size[2], best[2] = {-INFINITY, -INFINITY};
        bool nan[2];
        const int here[2] = {page[0], page[1]};
        if (scored) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                nan[h] = next_e[h] == kNanPage;
                size[h] = pow2(nan[h] ? 0 : next_e[h]);
#pragma unroll
                for (int k = 0; k < kParts; ++k) x[h][k] = next[h][k];
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) page[h] = page_of(i0 + step + r + 8 * h);
        if (scored && i0 + step < run.pages) fetch(page, next, next_e);
        if (scored) {
            for (int t = 0; t < tiles; ++t) {
                int acc[4] = {0, 0, 0, 0};
                const uint8_t* col = columns + (t * 8 + r) * kStride + j * 16;
#pragma unroll
                for (int k = 0; k < kParts; ++k) {
                    const uint4 y = *reinterpret_cast<const uint4*>(col + k * 64);
                    mma_s8(acc, x[0][k].x, x[1][k].x, x[0][k].y, x[1][k].y, y.x, y.y);
                    mma_s8(acc, x[0][k].z, x[1][k].z, x[0][k].w, x[1][k].w, y.z, y.w);
                }
                const float2 u = *reinterpret_cast<const float2*>(&unit[t * 8 + 2 * j]);
                best[0] = fmaxf(best[0], fmaxf(static_cast<float>(acc[0]) * u.x, static_cast<float>(acc[1]) * u.y));
                best[1] = fmaxf(best[1], fmaxf(static_cast<float>(acc[2]) * u.x, static_cast<float>(acc[3]) * u.y));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                best[h] = fmaxf(best[h], __shfl_xor_sync(0xffffffffu, best[h], 1));
                best[h] = fmaxf(best[h], __shfl_xor_sync(0xffffffffu, best[h], 2));
            }
        }
        const int i = i0 + r + 8 * j;                     // lane j = 0: page r, j = 1: page r + 8
        if (j < 2 && i < run.pages) {
            uint32_t key = 0;
            if ((j ? here[1] : here[0]) >= 0)
                key = !scored || i < a.n_sink || i >= run.old ? kForced : (j ? nan[1] : nan[0]) ? kNanKey : score_key(j ? best[1] * size[1] : best[0] * size[0]);
            keys[i] = key;
        }
    }
}

constexpr int kScorePages = 128, kScoreColumns = 128, kScoreTeam = kScoreColumns / 8;   // pages of a tile; query rows at a time; most lists of a team
constexpr int kScoreThreads = 512, kScoreGroups = kScoreThreads / kScorePages;   // threads of a page
constexpr int kScoreStages = 2;
template <int D>
constexpr int score_smem(int columns) { return kScoreStages * kScorePages * 2 * D + columns * 2 * D + 1024; }   // and room to start on a 1024-byte boundary

__device__ __forceinline__ void tc_mma_s8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
// s32 accumulator, s8 operands, both with the summed index innermost.
__device__ __forceinline__ uint32_t score_desc(int n) { return 2u << 4 | 1u << 7 | 1u << 10 | static_cast<uint32_t>(n >> 3) << 17 | 8u << 24; }
__device__ __forceinline__ void tmem_load8(uint32_t at, uint32_t (&x)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]) : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait(uint32_t (&x)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]) :: "memory");
}

// Keys of the pages of a team of lists and a head: 128 pages are the M side, the query rows of all lists of the team the N side.  A thread
// then has all products of its page, and the largest of a list's needs no exchange.  Bounds are gathered two tiles ahead, 16 bytes a copy;
// nothing else runs ahead in a block, that is what the other blocks of the SM are for.
// 48 streams' proposals of 17, 28/4 heads, 750 pages each: 30 us (the kernel above took 52); 1,024 lists of 28/4 heads over 939 pages: 44 us (125).  Half of it goes into the
// queries and the first tiles of a block, a quarter into taking maxima: both are chains of instructions, and the tensor cores wait.
// Grid: (shares of the pages, heads, teams).
template <typename T, int D>
__global__ void __launch_bounds__(kScoreThreads, 2) select_score_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int kTile = kScorePages * 2 * D;            // bytes
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(16) float unit[kScoreColumns];
    __shared__ SelectRun runs[kScoreTeam];
    __shared__ int ids[3][kScorePages];                   // pages of the tiles that are copied next
    __shared__ float part_best[kScoreGroups][kScorePages];   // where one list is all there is
    __shared__ uint64_t done;
    __shared__ uint32_t tmem_base;
    await_and_release();
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, head = blockIdx.y;
    const int own = tid % kScorePages, group = tid / kScorePages;   // the thread's page of a tile
    const int64_t team = a.first_team + blockIdx.z;
    const int b = static_cast<int>(quotient(team, a.teams)), l0 = static_cast<int>(team - static_cast<int64_t>(b) * a.teams) * a.team;
    if (tid < a.team) {
        SelectRun run{-1, 0, 0, 0};
        if (l0 + tid < a.lists) run = select_run(a, b, l0 + tid);
        runs[tid] = run;
    }
    if (tid == 0) barrier_init(shared_addr(&done), 1);
    barrier_init_fence();
    __syncthreads();
    int most = 0, s = -1;                                 // pages of the list that has most
    for (int l = 0; l < a.team; ++l) {
        most = max(most, runs[l].pages);
        if (runs[l].n > 0) s = runs[l].s;
    }
    uint32_t* const keys = a.keys + (static_cast<int64_t>(blockIdx.z) * a.team * c.n_kv + head) * a.key_stride;
    const int64_t list_stride = c.n_kv * a.key_stride;
    const int begin = blockIdx.x * kScorePages, step = gridDim.x * kScorePages;
    if (begin >= most) return;
    auto page_of = [&](int i) { return i < most ? c.page_at(s, i) : -1; };   // of the thread's own row
    auto row_at = [&](int page) { return (static_cast<int64_t>(page) * c.n_layers + a.layer) * c.n_kv + head; };
    if (most <= a.n_blocks) {                             // all blocks are listed
        for (int i0 = begin; i0 < most; i0 += step) {
            const int i = i0 + own, page = page_of(i);
            for (int l = group; l < a.team; l += kScoreGroups)
                if (i < runs[l].pages) keys[l * list_stride + i] = page < 0 ? 0u : kForced;
        }
        return;
    }
    const int each = a.share * a.group, padded = (each + 7) & ~7;   // columns of a list; more than fit are taken in turns
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t tiles_at = shared_addr(smem), columns_at = tiles_at + kScoreStages * kTile, bar = shared_addr(&done);
    const int most_columns = (min(a.team * padded, kScoreColumns) + 15) & ~15;   // what there is room for
    const uint32_t tmem_columns = most_columns <= 32 ? 32u : most_columns <= 64 ? 64u : 128u;
    if (warp == 0) tmem_alloc(shared_addr(&tmem_base), tmem_columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    // the tile of 128 pages of which ids[from] has the numbers into a stage: sixteen bytes of neighbouring rows or of one row a thread
    auto copy = [&](int stage, const int* from, bool on) {
        if (on) {
            constexpr int kUnits = D / 8;                 // of a row
            const int u = tid % kUnits;
#pragma unroll 4
            for (int r = tid / kUnits; r < kScorePages; r += kScoreThreads / kUnits) {
                const int page = from[r];
                if (page >= 0)
                    async_copy16(tiles_at + stage * kTile + (u >> 3) * (kScorePages * 128) + r * 128 + (((u & 7) ^ (r & 7)) << 4),
                                 a.o.codes + row_at(page) * 2 * D + u * 16);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    uint32_t products = 0;                                // so far
    bool late = false;
    for (int col0 = 0; col0 < each && !late; col0 += kScoreColumns) {
        const int per_list = min(padded - col0, kScoreColumns);   // columns of a list; more than one list only if all of its columns fit
        const int columns = (a.team * per_list + 15) & ~15;
        // ---- pages of the first tiles
        int page[2], e[2];                                // of the thread's row: this tile and the next
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            page[k] = page_of(begin + k * step + own);
            if (group == 0) ids[k][own] = page[k];
        }
        int ahead = page_of(begin + 2 * step + own);
        __syncthreads();
        copy(0, ids[0], true);
        copy(1, ids[1], begin + step < most);
#pragma unroll
        for (int k = 0; k < 2; ++k) e[k] = page[k] < 0 ? 0 : a.o.exps[row_at(page[k])];
        // ---- queries in eight bits, their positive and their negative parts: eight channels a lane, a few rows a warp under way together
        constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes, kRound = 2;
        const int part = lane % kLanes;
        for (int n0 = warp * (kAtOnce * kRound); n0 < columns; n0 += kScoreThreads / 32 * (kAtOnce * kRound)) {
            uint4 raw[kRound];
            bool used[kRound];
#pragma unroll
            for (int k = 0; k < kRound; ++k) {
                const int n = n0 + k * kAtOnce + lane / kLanes, l = n / per_list, rho = col0 + n - l * per_list;
                used[k] = n < columns && l < a.team && rho < runs[min(l, kScoreTeam - 1)].n * a.group;
                raw[k] = used[k] ? query_part<T>(a, b, (l0 + l) * a.share, head, rho, part * 8) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < kRound; ++k) {
                const int n = n0 + k * kAtOnce + lane / kLanes;
                uint32_t up[2], dn[2];
                const int ex = query_codes<T, kLanes>(raw[k], up, dn);
                if (n >= columns) continue;
                // rows of 128 bytes, sixteen-byte units swapped by the row's number
                auto put = [&](int at, const uint32_t (&bytes)[2]) {
                    uint8_t* to = smem + kScoreStages * kTile + (at >> 7) * (columns * 128) + n * 128 + ((at & 127) ^ ((n & 7) << 4));
                    *reinterpret_cast<uint2*>(to) = make_uint2(bytes[0], bytes[1]);
                };
                put(part * 8, up);
                put(D + part * 8, dn);
                if (part == 0) unit[n] = used[k] ? pow2(ex) : __int_as_float(0x7fffffff);   // a NaN drops out of the maximum
            }
        }
        // ---- tiles
        int stage = 0, slot = 0;                          // slot: of ids, the tile's
        for (int i0 = begin; i0 < most; i0 += step, stage ^= 1) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            async_proxy_fence();
            __syncthreads();
            if (tid == 0) {
                tc_fence_after();
                const uint64_t rows = operand_desc(tiles_at + stage * kTile, 16, 1024), cols = operand_desc(columns_at, 16, 1024);
#pragma unroll
                for (int x = 0; x < D / 16; ++x)
                    tc_mma_s8(tmem, rows + (((x >> 2) * (kScorePages * 128) + (x & 3) * 32) >> 4), cols + (((x >> 2) * (columns * 128) + (x & 3) * 32) >> 4), score_desc(columns), x > 0);
                tc_commit(bar);
            }
            __syncwarp();
            slot = slot == 2 ? 0 : slot + 1;
            const int after = slot == 2 ? 0 : slot + 1;   // of the tile after the next
            if (group == 0) ids[after][own] = ahead;
            const int here = page[0], e_here = e[0];
            page[0] = page[1], e[0] = e[1];
            page[1] = ahead;
            e[1] = ahead < 0 ? 0 : a.o.exps[row_at(ahead)];
            ahead = page_of(i0 + 3 * step + own);
            late |= !poll([&] { return barrier_try(bar, products & 1); });
            __syncwarp();
            ++products;
            tc_fence_after();
            const int i = i0 + own;
            const bool nan = e_here == kNanPage;
            const float size = pow2(nan ? 0 : e_here);
            const uint32_t from = tmem + (static_cast<uint32_t>(warp & 3) << 21);
            // the largest of the columns n0 .. n1 - 1, eight at a time
            auto largest = [&](int n0, int n1) {
                float best = -INFINITY;
                for (int n = n0; n < n1; n += 8) {
                    uint32_t x[8];
                    tmem_load8(from + n, x);
                    const float4 u0 = *reinterpret_cast<const float4*>(&unit[n]), u1 = *reinterpret_cast<const float4*>(&unit[n + 4]);
                    const float u[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
                    tmem_load_wait(x);
#pragma unroll
                    for (int w = 0; w < 8; ++w) best = fmaxf(best, static_cast<float>(static_cast<int>(x[w])) * u[w]);
                }
                return best;
            };
            auto write = [&](int l, float best) {
                const int pages = runs[l].pages, old = runs[l].old;
                if (i < pages) {
                    uint32_t key = 0;
                    if (here >= 0) key = pages <= a.n_blocks || i < a.n_sink || i >= old ? kForced : nan ? kNanKey : score_key(best * size);
                    uint32_t* at = keys + l * list_stride + i;
                    *at = col0 == 0 ? key : max(*at, key);
                }
                __syncwarp();                             // the loads from tensor memory want the warp together
            };
            if (a.team == 1) {                            // a share of its columns for each thread of the page
                const int eighths = per_list >> 3;
                const float best = largest(eighths * group / kScoreGroups * 8, eighths * (group + 1) / kScoreGroups * 8);
                if (per_list > 8) {
                    part_best[group][own] = best;
                    __syncthreads();
                    if (group == 0) write(0, fmaxf(fmaxf(best, part_best[1][own]), fmaxf(part_best[2][own], part_best[3][own])));
                } else if (eighths * (group + 1) / kScoreGroups > eighths * group / kScoreGroups) {
                    write(0, best);
                }
            } else {
                for (int l = group; l < a.team; l += kScoreGroups) write(l, largest(l * per_list, (l + 1) * per_list));
            }
            tc_fence_before();
            late = __syncthreads_or(late);                // the products are read, the stage is free
            if (late) break;
            copy(stage, ids[after], i0 + 2 * step < most);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                                  // the columns may be written again
    }
    if (late) {
        __nanosleep(100000);                              // products still under way
        if (tid == 0 && c.meta) atomicOr(&c.meta[1], kStatusGaveUp);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_free(tmem, tmem_columns);
}

// ---- the best pages of a list: the keys lie in registers, kKeys neighbouring ones a thread; the n_blocks-th largest is found bit by bit,
// and listed are all pages above it and the first of those that equal it, in order.  A list is a warp's or a block's.
constexpr int kPickThreads = 256;

template <int kTeam>
struct PickTeam {
    static constexpr int kWarps = kTeam / 32;
    int2 (*sums)[kWarps > 1 ? kWarps : 1];   // [2][warps]
    int flip = 0;
    // Sums of two counts over the team; *before: over its earlier threads.
    __device__ __forceinline__ int2 scan(int2 x, int2* before) {
        const int lane = threadIdx.x & 31;
        int2 y = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, y.x, d), v = __shfl_up_sync(0xffffffffu, y.y, d);
            if (lane >= d) {
                y.x += u;
                y.y += v;
            }
        }
        int2 all = make_int2(__shfl_sync(0xffffffffu, y.x, 31), __shfl_sync(0xffffffffu, y.y, 31)), earlier = make_int2(0, 0);
        if constexpr (kWarps > 1) {
            const int warp = threadIdx.x >> 5;
            if (lane == 0) sums[flip][warp] = all;
            __syncthreads();
            all = make_int2(0, 0);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                if (w == warp) earlier = all;
                all.x += sums[flip][w].x;
                all.y += sums[flip][w].y;
            }
            flip ^= 1;
        }
        *before = make_int2(earlier.x + y.x - x.x, earlier.y + y.y - x.y);
        return all;
    }
    __device__ __forceinline__ int sum(int x) {
        int all = __reduce_add_sync(0xffffffffu, x);
        if constexpr (kWarps > 1) {
            if ((threadIdx.x & 31) == 0) sums[flip][threadIdx.x >> 5].x = all;
            __syncthreads();
            all = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) all += sums[flip][w].x;
            flip ^= 1;
        }
        return all;
    }
    // Bitwise "or" and "and" over the team.
    __device__ __forceinline__ void bits(uint32_t& any, uint32_t& every) {
        any = __reduce_or_sync(0xffffffffu, any);
        every = __reduce_and_sync(0xffffffffu, every);
        if constexpr (kWarps > 1) {
            if ((threadIdx.x & 31) == 0) sums[flip][threadIdx.x >> 5] = make_int2(static_cast<int>(any), static_cast<int>(every));
            __syncthreads();
            any = 0;
            every = 0xffffffffu;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                any |= static_cast<uint32_t>(sums[flip][w].x);
                every &= static_cast<uint32_t>(sums[flip][w].y);
            }
            flip ^= 1;
        }
    }
};

// kKeys = 0: any number of pages, the keys read again each time.  Grid: (lists and heads of the launch in runs of kPickThreads / kTeam).
template <int kTeam, int kKeys>
__global__ void __launch_bounds__(kPickThreads) select_pick_kernel(const __grid_constant__ SelectArgs a, int64_t n_lists) {
    using Team = PickTeam<kTeam>;
    __shared__ int2 sums[2][Team::kWarps];
    Team team{sums};
    const CacheView& c = a.c;
    const int t = threadIdx.x % kTeam;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kPickThreads / kTeam) + threadIdx.x / kTeam;   // of the keys
    if (row >= n_lists) {                                 // the whole team
        await_before();
        return;
    }
    const int64_t g = quotient(row, c.n_kv), w = quotient(g, a.team), v = a.first_team + w;
    const int head = static_cast<int>(row - g * c.n_kv), b = static_cast<int>(quotient(v, a.teams));
    const int l = static_cast<int>(v - static_cast<int64_t>(b) * a.teams) * a.team + static_cast<int>(g - w * a.team);
    const int n = l < a.lists ? select_run(a, b, l).pages : 0;
    await_before();
    if (l >= a.lists) return;
    int32_t* const out = a.out + ((static_cast<int64_t>(b) * a.lists + l) * c.n_kv + head) * a.n_blocks;
    const uint32_t* const keys = a.keys + row * a.key_stride;
    const int each = kKeys ? kKeys : (n + kTeam - 1) / kTeam, i0 = t * each;   // the thread's pages: i0 .. i0 + each - 1
    uint32_t kept[kKeys ? kKeys : 1];
    if constexpr (kKeys > 0) {
#pragma unroll
        for (int k = 0; k < kKeys; k += 4) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (i0 + k < n) x = *reinterpret_cast<const uint4*>(keys + i0 + k);
            kept[k] = i0 + k < n ? x.x : 0u;
            kept[k + 1] = i0 + k + 1 < n ? x.y : 0u;
            kept[k + 2] = i0 + k + 2 < n ? x.z : 0u;
            kept[k + 3] = i0 + k + 3 < n ? x.w : 0u;
        }
    }
    auto for_keys = [&](auto f) {
        if constexpr (kKeys > 0) {
#pragma unroll
            for (int k = 0; k < kKeys; ++k) f(kept[k], i0 + k);
        } else {
            for (int k = 0; k < each; ++k)
                if (i0 + k < n) f(keys[i0 + k], i0 + k);
        }
    };
    // the key of the last page that is listed: the largest for which n_blocks pages reach it, 1 if fewer are present
    uint32_t limit = 1;
    if (n > a.n_blocks) {
        int present = 0, forced = 0;
        uint32_t any = 0, every = 0xffffffffu;            // bits of the keys in between
        for_keys([&](uint32_t k, int) {
            present += k != 0;
            forced += k == kForced;
            if (k != 0 && k != kForced) {
                any |= k;
                every &= k;
            }
        });
        int2 unused;
        const int2 all = team.scan(make_int2(present, forced), &unused);
        team.bits(any, every);
        const int want = a.n_blocks - all.y;              // of them: forced ones always fit
        if (all.x > a.n_blocks) {
            if (want <= 0) {
                limit = kForced;
            } else {
                uint32_t differ = any & ~every;           // where they are not all alike
                limit = every;
                while (differ) {
                    const uint32_t bit = 0x80000000u >> __clz(differ);
                    differ &= ~bit;
                    const uint32_t to = limit | bit;
                    int count = 0;
                    for_keys([&](uint32_t k, int) { count += k >= to; });
                    count = team.sum(count) - all.y;
                    if (count >= want) limit = to;
                    if (count == want) {                  // exactly those
                        --limit;
                        break;
                    }
                }
            }
        }
    }
    int2 count = make_int2(0, 0);
    for_keys([&](uint32_t k, int) {
        count.x += k > limit;
        count.y += k == limit;
    });
    int2 before;
    const int2 total = team.scan(count, &before);
    const int ties = a.n_blocks - total.x;                // so many of the pages at the limit
    int at = before.x + min(before.y, ties), equal = before.y;
    for_keys([&](uint32_t k, int i) {
        const bool on = k > limit || (k == limit && equal < ties);
        if (on && at < a.n_blocks) out[at] = i;
        at += on;
        equal += k == limit;
    });
    for (int i = min(total.x + min(total.y, ties), a.n_blocks) + t; i < a.n_blocks; i += kTeam) out[i] = -1;
}

}  // namespace samb200
