// Attention for many query rows per key/value head (proposals of several heads, prompt chunks): tcgen05 products.
//
// S = Q K^T and O += P V on a tile of 128 query rows, with 128 tokens a step.  Sixteen warps expand the 4-bit tiles into two stages
// of fp16 keys and two of fp16 values in shared memory (exact: a value has six significant bits).  Q, two tiles of scores and the
// sums O lie in tensor memory.  Two threads of the eight softmax warps share a query row, each with half of a step's tokens; they
// write P as fp16 over S, from where the second product takes it.  While they work on one step's scores, the products of the step
// before and of the step after run.
//
// Q is read from tensor memory, not from shared memory: a 128 x 128 product with both operands in shared memory takes all of its
// bandwidth, and beside it a warp gets half the stores and a tenth of the loads through (barriers are loads) that it gets beside
// products with one operand there.
//
// What it measured: a step takes 2,370 to 2,450 clocks (2,048 query tokens over 20,011 positions, 28/4 heads of 128: 715 us,
// 865 TFLOP/s), of which the products are 1,024 and the exponentials 1,024.  It is bound by the chain scores - exponentials -
// weights - products, of which two are in flight: no pipe is full.  Tried and slower: two row tiles a CTA with the expanded operands
// shared and Q in shared memory (2,450 clocks for a tile's step, but only with more than 128 query rows); one softmax warp per
// scheduler with whole rows (2,640); the scores in two halves; three waits a step for the issuing warp instead of one (2,520).
//
// Keys and values have the same layout in shared memory, [token][64 channels] in 128-byte rows with the 128-byte swizzle: for
// the first product it is read with the channels (the summed index) innermost, for the second with the channels as the N side.
//
// Weights are 2^(score - reference), with a reference that lies 8 below the largest score when it is set.  It is raised, and the
// row's sums rescaled, only when the weights of a step add up to more than 2^15: as long as they do not, each of them is within
// fp16, and the maximum of a step need not be known.  Weights down to 2^-22 of the largest keep all 11 bits.
//
// What the warps of an SM run has to stay within the instruction caches: the roles are small loops, and masked steps have code of
// their own.
#pragma once

#include "attend_stream.cuh"

namespace samb200 {

constexpr int kWideUnit = 128;                     // tokens of a step
constexpr int kWideRows = 128;                     // query rows of a segment
constexpr int kWideWarps = 28, kWideThreads = kWideWarps * 32;   // eight softmax warps, sixteen expanding ones, an issuing one (and three that idle)
constexpr int kWideMaxCtas = 160;
// How far below the largest score the reference is set, and what a thread's 64 weights of a step may add up to before it is raised.  Pages
// out of a list differ more from one another than neighbours do, so that it is raised more often: with lists it takes the largest
// of all scores of the first step, not of a quarter, the sum may be all that a single fp16 weight can, and the reference lies 7 below, so that weights keep
// all 11 bits down to 2^-21 of the largest, as in the streaming kernel.  (48 proposals of 17 over 64 blocks of 32, and 2,048 queries, every sixteen over 32 blocks of
// 64: 143 and 114 us; as without lists 162 and 139, so but 8 below 148 and 123, 6 below 142 and 108.)
template <bool kListed> constexpr float kWideAbove = kListed ? 7.f : 8.f;
template <bool kListed> constexpr float kTotalMax = kListed ? 65504.f : 32768.f;
// columns of tensor memory
constexpr uint32_t kColQ = 0, kColS = 64, kColO = 320;

template <int D>
struct WidePlan {
    static constexpr int kTileBytes = 128 * D * 2;                      // a [128][D] fp16 operand
    static constexpr int kChunkBytes = 128 * 128;                       // 64 channels of it
    static constexpr int kK = 0, kV = 2 * kTileBytes;
    static constexpr int kRaw = kV + 2 * kTileBytes;                    // slots of the expanding warps: two tiles' keys or values each
    static constexpr int kRawSlots = 2, kRawHalf = 18 * D;
    static constexpr int kSmem = kRaw + 16 * kRawSlots * kRawHalf + 1024;   // and room to start on a 1024-byte boundary
    static constexpr int kPart = 128 * D + 2 * 128;                     // floats of a partial result
};

// ---- tensor memory and tcgen05
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
#define SAM_R8(x, o) "=r"(x[o]), "=r"(x[o + 1]), "=r"(x[o + 2]), "=r"(x[o + 3]), "=r"(x[o + 4]), "=r"(x[o + 5]), "=r"(x[o + 6]), "=r"(x[o + 7])
#define SAM_S8(x, o) "r"(x[o]), "r"(x[o + 1]), "r"(x[o + 2]), "r"(x[o + 3]), "r"(x[o + 4]), "r"(x[o + 5]), "r"(x[o + 6]), "r"(x[o + 7])
// 32 columns of the warp's 32 lanes: thread = lane, register = column.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&x)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
                 "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : SAM_R8(x, 0), SAM_R8(x, 8), SAM_R8(x, 16), SAM_R8(x, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait(uint32_t (&x)[32]) {   // ties the registers to the wait
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
                 "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]) :: "memory");
    asm volatile("" : "+r"(x[16]), "+r"(x[17]), "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]),
                 "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]), "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31]));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t (&x)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : SAM_R8(x, 0), SAM_R8(x, 8) : "r"(at));
}
__device__ __forceinline__ void tmem_load_wait(uint32_t (&x)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
                 "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]) :: "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), SAM_S8(x, 0), SAM_S8(x, 8) : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
#undef SAM_R8
#undef SAM_S8
__device__ __forceinline__ void async_copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Descriptor of a 128-byte swizzled operand at `at` (shared address): bytes between 64-element groups of the M/N side (used when
// that side is innermost) and between groups of eight rows.
__device__ __forceinline__ uint64_t operand_desc(uint32_t at, uint32_t lead, uint32_t stride) {
    return static_cast<uint64_t>((at & 0x3ffff) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 | static_cast<uint64_t>(stride >> 4) << 32 |
           1ull << 46 | 2ull << 61;
}
// f32 accumulator, f16 operands, A with the summed index innermost.
__host__ __device__ constexpr uint32_t product_desc(int m, int n, bool b_n_innermost) {
    return 1u << 4 | static_cast<uint32_t>(b_n_innermost) << 16 | static_cast<uint32_t>(n >> 3) << 17 | static_cast<uint32_t>(m >> 4) << 24;
}

__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
    float2 w;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(w.x), "=f"(w.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
    return w;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
    float2 w;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(w.x), "=f"(w.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return w;
}

// A segment: one row of the batch, one tile of kWideRows query rows, one key/value head; its steps cover the tokens that some
// query row of it sees.  Segments are numbered by row, row tile, head.
struct WideSegment {
    RowInfo ri;          // lo, hi: of this row tile
    int b, rt, head, steps;
    int rows;            // query rows of the tile
    int first_pos, last_pos;
    int end;             // listed: first position that none of them sees
    int64_t begin;       // number of its first unit
};
template <bool kListed>
__device__ __forceinline__ void wide_tile(const AttendArgs& a, int tiles, int64_t e, WideSegment& g) {   // e = b * tiles + rt
    g.b = static_cast<int>(quotient(e, tiles));
    g.rt = static_cast<int>(e - static_cast<int64_t>(g.b) * tiles);
    g.ri = row_info<kWideUnit, kListed>(a, g.b);
    g.rows = min(run_rows<kListed>(a, g.ri.n) - g.rt * kWideRows, kWideRows);   // a launch of this kernel begins with row 0
    g.steps = 0;
    if (g.rows <= 0) return;
    const int i0 = g.rt * kWideRows / a.group, i1 = (g.rt * kWideRows + g.rows - 1) / a.group, cap = a.c.capacity();
    g.first_pos = g.ri.len + i0;
    g.last_pos = g.ri.len + i1;
    g.end = static_cast<int>(min(static_cast<int64_t>(g.ri.len) + i1 + 1, static_cast<int64_t>(cap)));
    if constexpr (kListed) {
        g.steps = (g.ri.hi + kWideUnit - 1) / kWideUnit;
        return;
    }
    g.ri.hi = g.end;
    g.ri.lo = a.window > 0 ? min(max(g.first_pos - a.window + 1, 0), cap - 1) & ~(kWideUnit - 1) : 0;
    g.steps = max((g.ri.hi - g.ri.lo + kWideUnit - 1) / kWideUnit, 1);
}

// kListed: over listed blocks.  The tokens of a segment are then the places of its list; the expanding warps say where the tiles of a
// step really begin, and whether every row sees all of them.
template <typename T, int D, bool kListed>
__global__ void __launch_bounds__(kWideThreads, 1) attend_wide_kernel(const __grid_constant__ AttendArgs a) {
    using Plan = WidePlan<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[15];
    __shared__ uint32_t tmem_base;
    __shared__ int64_t scan[kWideWarps], start_e, start_begin;
    __shared__ alignas(4) uint8_t tile_there[4][4];    // per step (mod 4) and expanding warp: which of its two tiles are there
    __shared__ alignas(4) uint8_t nan_flag[4][4];      // NaN among the values of the warp's tokens (written where there are masks)
    __shared__ uint8_t nan_block[4][128];              // which 16-channel blocks of a token's values are NaN
    __shared__ alignas(4) uint8_t tile_all[4][4];      // listed: every row sees all of the warp's two tiles
    __shared__ int tile_begin[kListed ? 4 : 1][8];     // listed: positions of the first tokens of the step's tiles
    __shared__ int2 slot_begin[kListed ? 16 : 1][Plan::kRawSlots];   // listed: of the tiles in an expanding warp's slots
    __shared__ float shared_row[2][128];               // what the two threads of a query row tell each other
    __shared__ int last_here;
    __shared__ volatile int abort_flag;

    if constexpr (kListed) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the streaming kernel for rows behind the last full tile
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sm = shared_addr(smem), bar = shared_addr(bars);
    // barriers, two each: scores ready, first keys ready, product done, step ready; and queries ready
    auto score_bar = [&](int i) { return bar + 8 * i; };
    auto k_first = [&](int i) { return bar + 16 + 8 * i; };
    auto product_bar = [&](int i) { return bar + 80 + 8 * i; };
    // Step n may go on when its weights (eight warps), its values (four) and the keys of step n + 2 (four) are there: one wait of the
    // issuing warp, where three of them took as long as the products themselves.
    auto ready_bar = [&](int i) { return bar + 96 + 8 * i; };
    const uint32_t query_bar = bar + 112;
    // Gives up after kCachePolls polls, and at once when some wait of the CTA has: everybody then runs on without waiting, the
    // results are not valid, and the status says so.
    auto wait = [&](uint32_t b, uint32_t parity) {
        for (uint32_t i = 0; i < kCachePolls; ++i) {
            if (barrier_try(b, parity)) return;
            if ((i & 15) == 15 && abort_flag) return;
        }
        abort_flag = 1;
    };
    // For whole warps.  Lanes leave a wait, and a branch of their own, one by one; what follows in tensor memory and at the hardware
    // barriers wants the warp together, so it is brought together there, here and below.
    auto wait_warp = [&](uint32_t b, uint32_t parity) {
        wait(b, parity);
        __syncwarp();
    };
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            barrier_init(score_bar(i), 1);
            barrier_init(k_first(i), 4);
            barrier_init(product_bar(i), 1);
            barrier_init(ready_bar(i), 16);
        }
        barrier_init(query_bar, 8);
        abort_flag = 0;
    }
    barrier_init_fence();

    // ---- how many units there are, and where our share begins
    const int tiles = static_cast<int>(((kListed ? a.row1 : static_cast<int64_t>(a.share) * a.group) + kWideRows - 1) / kWideRows);
    const int64_t n_tiles = static_cast<int64_t>(a.runs) * tiles;
    auto block_sum = [&](int64_t x, int64_t* before) -> int64_t {
        int64_t y = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t up = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) y += up;
        }
        __syncthreads();
        if (lane == 31) scan[warp] = y;
        __syncthreads();
        int64_t all = 0, first = 0;
        for (int w = 0; w < kWideWarps; ++w) {
            if (w == warp) first = all;
            all += scan[w];
        }
        *before = first + y - x;
        return all;
    };
    auto units_of = [&](int64_t e) -> int64_t {
        if (e >= n_tiles) return 0;
        WideSegment g;
        wide_tile<kListed>(a, tiles, e, g);
        return static_cast<int64_t>(g.steps) * c.n_kv;
    };
    int64_t units = 0, mine = 0, before = 0;
    for (int64_t e0 = 0; e0 < n_tiles; e0 += kWideThreads) {
        mine = units_of(e0 + tid);
        units += block_sum(mine, &before);
    }
    const int ctas = static_cast<int>(min(units, static_cast<int64_t>(gridDim.x))), cta = blockIdx.x;
    const Shares shares(units, max(ctas, 1));
    const bool busy = cta < ctas;
    const int64_t u0 = busy ? shares.begin(cta) : 0, u1 = busy ? shares.begin(cta + 1) : 0;
    if (busy) {
        int64_t sum = 0;
        for (int64_t e0 = 0; e0 < n_tiles; e0 += kWideThreads) {
            if (n_tiles > kWideThreads) {
                mine = units_of(e0 + tid);
                const int64_t all = block_sum(mine, &before);
                before += sum;
                sum += all;
            }
            if (u0 >= before && u0 < before + mine) {
                start_e = e0 + tid;
                start_begin = before;
            }
        }
    }
    clear_unused_rows<T, D>(a, cta, gridDim.x);
    if (!busy) return;
    __syncwarp();
    if (warp == 24) tmem_alloc(shared_addr(&tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    // Runs f(segment, first step, steps) over the pieces of our share.
    auto for_pieces = [&](auto f) {
        WideSegment g;
        int64_t e = start_e;
        wide_tile<kListed>(a, tiles, e, g);
        const int64_t rel = u0 - start_begin;
        g.head = static_cast<int>(quotient(rel, g.steps));
        g.begin = start_begin + static_cast<int64_t>(g.head) * g.steps;
        int64_t u = u0;
        for (;;) {
            const int s0 = static_cast<int>(u - g.begin);
            const int count = static_cast<int>(min(u1 - u, static_cast<int64_t>(g.steps - s0)));
            f(g, s0, count);
            u += count;
            if (u >= u1) return;
            g.begin += g.steps;
            if (++g.head == c.n_kv) {
                g.head = 0;
                const int64_t next = g.begin;
                do wide_tile<kListed>(a, tiles, ++e, g);
                while (g.steps == 0 && e + 1 < n_tiles);
                g.begin = next;
            }
        }
    };
    // Steps that begin at or before the first number and after the second are seen by all rows of the segment.
    auto all_until = [&](const WideSegment& g) { return g.first_pos - (kWideUnit - 1); };
    auto all_after = [&](const WideSegment& g) { return a.window == 0 ? -1 : g.last_pos - a.window; };

    // Registers go where they are needed: 256 threads x 96, 512 x 64, 128 x 48, of 896 x 72 at launch.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
        // ================= softmax warps
        const int row = tid & 127, part_no = warp >> 2, pair = warp & 3;     // tokens 64 part_no ... of a step
        const uint32_t lanes = tmem + (static_cast<uint32_t>(pair) << 21);   // the warp's quarter of the lanes
        uint32_t n = 0;                                 // steps so far
        auto meet_pair = [&]() { asm volatile("barrier.cta.sync.aligned %0, 64;" ::"r"(1 + pair) : "memory"); };
        auto any_of_pair = [&](bool x) -> bool {        // true if x is for any of the pair's threads
            uint32_t y;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred.aligned q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(y) : "r"(static_cast<uint32_t>(x)), "r"(1 + pair) : "memory");
            return y != 0;
        };
        auto meet = [&]() { asm volatile("barrier.cta.sync.aligned 5, 256;" ::: "memory"); };
        auto larger = [&](float x) -> float {           // the larger of the two threads' values
            shared_row[part_no][row] = x;
            meet_pair();
            const float y = static_cast<volatile float*>(shared_row[part_no ^ 1])[row];
            meet_pair();                                // the places are free again
            return fmaxf(x, y);
        };
        // Product n complete.  Asked for when the scores of step n + 1 are there, or none are to come: the product before n has been
        // complete since, so that the parity of n's barrier tells.
        auto product = [&](uint32_t i) {
            wait_warp(product_bar(i & 1), (i >> 1) & 1);
            tc_fence_after();
        };
        for_pieces([&](const WideSegment& seg, int s0, int count) {
            // ---- queries into tensor memory
            const bool mine = row < seg.rows;
            const RunPlace place = run_place<kListed>(a, seg.b);
            const int rho = seg.rt * kWideRows + row, qi = place.i0 + rho / a.group, qh = seg.head * a.group + rho % a.group;
            float factor;
            {
                const T* q = static_cast<const T*>(a.q) + place.b * a.q_row + static_cast<int64_t>(qi) * a.q_token + static_cast<int64_t>(qh) * a.q_head;
                constexpr int kHalf = D / 2;            // channels of a thread; the size of the row is taken over all of them
                uint32_t x[kHalf / 2];
                auto load8 = [&](int d, uint32_t (&w)[4]) {
                    alignas(16) T y[8];
                    if (mine && a.q_wide) {
                        *reinterpret_cast<uint4*>(y) = __ldg(reinterpret_cast<const uint4*>(q + d));
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = mine ? q[d + i] : Elem<T>::from_float(0.f);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t*>(y)[i];
                };
#pragma unroll
                for (int d = 0; d < kHalf; d += 8) load8(part_no * kHalf + d, reinterpret_cast<uint32_t(&)[4]>(x[d / 2]));
                __syncwarp();
                int e = 0;
                if constexpr (!std::is_same<T, __half>::value) {
                    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
                    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
                    float big = 0.f;
#pragma unroll
                    for (int i = 0; i < kHalf / 2; ++i) big = fmaxf(big, fmaxf(fabsf(lo(x[i])), fabsf(hi(x[i]))));
                    big = larger(big);
                    e = big > 0.f ? min(14 - (static_cast<int>(__float_as_uint(big) >> 23) - 127), 126) : 0;
                    const float up = pow2(e);
#pragma unroll
                    for (int i = 0; i < kHalf / 2; ++i) x[i] = pack_half2(lo(x[i]) * up, hi(x[i]) * up);
                }
                if (a.scale < 0.f) {                    // so that the largest score is the largest product
#pragma unroll
                    for (int i = 0; i < kHalf / 2; ++i) x[i] ^= 0x80008000u;
                }
                factor = score_factor(a.scale, c.k_exp - e);
#pragma unroll
                for (int i = 0; i < kHalf / 2; i += 16) tmem_store16(lanes + kColQ + part_no * (kHalf / 2) + i, reinterpret_cast<const uint32_t(&)[16]>(x[i]));
                tmem_store_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(query_bar);
                __syncwarp();
            }
            const int pos = mine ? seg.ri.len + rho / a.group : -1;
            const bool idle = !__any_sync(0xffffffffu, mine);
            float m = -INFINITY, l = 0.f;
            uint32_t nan_blocks = 0;

            // ---- steps
            const int until = all_until(seg), after = all_after(seg), base = seg.ri.lo + s0 * kWideUnit;
            auto hand_over = [&](uint32_t i) {           // the weights of step i to the second product
                tmem_store_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(ready_bar(i & 1));
                __syncwarp();
            };
#pragma unroll 1
            for (int k = 0; k < count; ++k, ++n) {
                const uint32_t s_at = lanes + kColS + (n & 1) * 128 + part_no * 64;
                wait_warp(score_bar(n & 1), (n >> 1) & 1);
                if (k > 0) hand_over(n - 1);             // the weights of the step before are stored by now
                tc_fence_after();
                const int t0 = base + k * kWideUnit, ring = n & 3;
                uint32_t on = *reinterpret_cast<volatile uint32_t*>(tile_there[ring]);
                on = (on * 0x01041040u) >> 24;            // two bits of each byte, side by side
                const bool all = kListed ? *reinterpret_cast<volatile uint32_t*>(tile_all[ring]) == 0x01010101u : t0 <= until && t0 > after;
                // Weights with the reference at hand, in one pass: a sum of at most kTotalMax means that each of them is within fp16.
                // Where that fails, and where there are masks or absent tiles, the step is done in two passes, the largest score first.
                bool done = idle;                        // a quarter without query rows hands nothing over: its sums are nobody's
                if (all && on == 0xff && !idle) {        // absent tiles read as scores of zero, which must not make a reference
                    float2 total = make_float2(0.f, 0.f);
                    uint32_t x[2][16], p[2][16];
                    tmem_load16(s_at, x[0]);
                    if (__any_sync(0xffffffffu, m == -INFINITY)) {   // a first reference from some of the scores; with lists, from all
                        tmem_load_wait(x[0]);
                        float top = -INFINITY;
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = fmaxf(top, __uint_as_float(x[0][i]));
                        if constexpr (kListed) {
#pragma unroll 1
                            for (int q = 1; q < 4; ++q) {
                                tmem_load16(s_at + q * 16, x[1]);
                                tmem_load_wait(x[1]);
#pragma unroll
                                for (int i = 0; i < 16; ++i) top = fmaxf(top, __uint_as_float(x[1][i]));
                            }
                        }
                        top = larger(top);
                        if (m == -INFINITY) m = top * factor - kWideAbove<kListed>;
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t(&y)[16] = x[q & 1];
                        tmem_load_wait(y);
                        if (q < 3) tmem_load16(s_at + (q + 1) * 16, x[(q + 1) & 1]);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float2 z = fma2(make_float2(__uint_as_float(y[i]), __uint_as_float(y[i + 1])), make_float2(factor, factor), make_float2(-ref, -ref));
                            z.x = exp2_fast(z.x);
                            z.y = exp2_fast(z.y);
                            total = add2(total, z);
                            p[q >> 1][(q & 1) * 8 + i / 2] = pack_half2(z.x, z.y);
                        }
                    }
                    const float sum = total.x + total.y;
                    done = !any_of_pair(sum > kTotalMax<kListed>);
                    if (done) {
                        l += sum;
                        tmem_store16(s_at, p[0]);
                        tmem_store16(s_at + 16, p[1]);
                    }
                }
                if (!done) {
                    if (!all && *reinterpret_cast<volatile uint32_t*>(nan_flag[ring])) {
                        for (int t = 0; t < kWideUnit; ++t)
                            if (static_cast<volatile uint8_t*>(nan_flag[ring])[t >> 5] &&
                                (kListed ? static_cast<volatile int*>(tile_begin[kListed ? ring : 0])[t >> 4] + (t & 15) <= pos : t0 + t <= pos && (a.window == 0 || t0 + t > pos - a.window)))
                                nan_blocks |= static_cast<volatile uint8_t*>(nan_block[ring])[t];
                        __syncwarp();
                    }
                    // which of 32 columns a row sees, as bits; q: 0 .. 3 over the step
                    const int from = a.window > 0 ? max(pos - a.window + 1 - t0, 0) : 0, to_col = min(pos - t0, kWideUnit - 1);
                    auto seen = [&](int q) -> uint32_t {
                        if constexpr (kListed) {
                            uint32_t bits = 0;
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const int last = min(pos - static_cast<volatile int*>(tile_begin[ring])[2 * q + x], 15);   // of the tile's tokens
                                if (last >= 0 && ((on >> (2 * q + x)) & 1)) bits |= ((2u << last) - 1) << (16 * x);
                            }
                            return bits;
                        }
                        const int lo = max(from - q * 32, 0), hi = to_col - q * 32;
                        uint32_t bits = hi < 0 || lo > 31 ? 0u : (0xffffffffu >> (31 - min(hi, 31))) & (0xffffffffu << lo);
                        if (!((on >> (2 * q)) & 1)) bits &= 0xffff0000u;
                        if (!((on >> (2 * q)) & 2)) bits &= 0x0000ffffu;
                        return bits;
                    };
                    uint32_t x[32];
                    float top = -INFINITY;
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {
                        tmem_load32(s_at + q * 32, x);
                        tmem_load_wait(x);
                        const uint32_t bits = seen(part_no * 2 + q);
#pragma unroll
                        for (int i = 0; i < 32; ++i) top = fmaxf(top, (bits >> i) & 1 ? __uint_as_float(x[i]) : -INFINITY);
                    }
                    top = larger(top) * factor;
                    if (__any_sync(0xffffffffu, top > m + kWideAbove<kListed>)) {
                        const float to = top > m + kWideAbove<kListed> ? top - kWideAbove<kListed> : m;
                        const float keep = m == -INFINITY ? 0.f : exp2_fast(m - to);
                        if (k > 0) {                     // the sums so far
                            product(n - 1);
#pragma unroll 1
                            for (int q = part_no * (D / 32); q < (part_no + 1) * (D / 32); ++q) {
                                uint32_t o[16];
                                tmem_load16(lanes + kColO + q * 16, o);
                                tmem_load_wait(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
                                tmem_store16(lanes + kColO + q * 16, o);
                            }
                        }
                        l *= keep;
                        m = to;
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {
                        tmem_load32(s_at + q * 32, x);
                        tmem_load_wait(x);
                        const uint32_t bits = seen(part_no * 2 + q);
                        uint32_t p[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float y0 = fmaf(__uint_as_float(x[i]), factor, -ref), y1 = fmaf(__uint_as_float(x[i + 1]), factor, -ref);
                            const float e0 = exp2_fast((bits >> i) & 1 ? y0 : -INFINITY), e1 = exp2_fast((bits >> i) & 2 ? y1 : -INFINITY);
                            l += e0 + e1;
                            p[i / 2] = pack_half2(e0, e1);
                        }
                        tmem_store16(s_at + q * 16, p);      // behind the scores that are still to be read
                    }
                }
            }
            hand_over(n - 1);

            // ---- the piece's result
            product(n - 1);
            {   // the row's total
                shared_row[part_no][row] = l;
                meet_pair();
                l = static_cast<volatile float*>(shared_row[0])[row] + static_cast<volatile float*>(shared_row[1])[row];
                meet_pair();
            }
            const bool begins = s0 == 0, ends = s0 + count == seg.steps;
            const int col0 = part_no * (D / 2), col1 = col0 + D / 2;
            auto sums = [&](int col, float (&y)[32]) {  // 32 channels
                uint32_t x[32];
                tmem_load32(lanes + kColO + col, x);
                tmem_load_wait(x);
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = (nan_blocks >> ((col + i) >> 4)) & 1 ? __int_as_float(0x7fffffff) : __uint_as_float(x[i]);
            };
            auto finish = [&](int col, float (&y)[32], float m_all, float l_all) {
                const float f = finish_factor(l_all, c.v_exp);
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = l_all == 0.f ? 0.f : y[i] * f;
                store_row<T>(static_cast<T*>(a.out) + place.b * a.o_row + static_cast<int64_t>(qi) * a.o_token + static_cast<int64_t>(qh) * a.o_head + col, y, a.o_wide);
                if (a.lse && col == 0) a.lse[(static_cast<int64_t>(place.b) * a.Q + qi) * a.H + qh] = finish_lse(m_all, l_all);
            };
            if (begins && ends) {
#pragma unroll 1
                for (int col = col0; col < col1; col += 32) {
                    float y[32];
                    sums(col, y);
                    if (mine) finish(col, y, m, l);
                    __syncwarp();
                }
            } else {
                // [D / 4][128] float4, then references and totals
                auto part = [&](int owner, bool first_piece) { return a.partials + (2ll * owner + first_piece) * Plan::kPart; };
                float* out = part(cta, begins);
#pragma unroll 1
                for (int col = col0; col < col1; col += 32) {
                    float y[32];
                    sums(col, y);
                    if (mine) {                          // unused rows are not written, nor read below
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            reinterpret_cast<float4*>(out)[((col + i) >> 2) * 128 + row] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                    }
                    __syncwarp();
                }
                if (part_no == 0) {
                    out[128 * D + row] = m;
                    out[128 * D + 128 + row] = l;
                }
                __threadfence();
                meet();
                const int c0 = shares.owner(seg.begin), c1 = shares.owner(seg.begin + seg.steps - 1);
                if (tid == 0) {
                    last_here = atomicAdd(&a.counters[c0], 1) == c1 - c0;
                    if (last_here) a.counters[c0] = 0;
                    __threadfence();
                }
                __syncwarp();
                meet();
                if (*static_cast<volatile int*>(&last_here) && mine) {
                    __threadfence();
                    const int parts = c1 - c0 + 1;
                    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll 4
                    for (int i = 0; i < parts; ++i) m_all = fmaxf(m_all, __ldcg(part(c0 + i, i == 0) + 128 * D + row));
#pragma unroll 4
                    for (int i = 0; i < parts; ++i) {
                        const float* p = part(c0 + i, i == 0) + 128 * D + row;
                        l_all += join_weight(__ldcg(p), m_all) * __ldcg(p + 128);
                    }
#pragma unroll 1
                    for (int col = col0; col < col1; col += 32) {
                        float y[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = 0.f;
#pragma unroll 2
                        for (int i = 0; i < parts; ++i) {
                            const float* p = part(c0 + i, i == 0);
                            const float wt = join_weight(__ldcg(p + 128 * D + row), m_all);
#pragma unroll
                            for (int d = 0; d < 32; d += 4) {
                                const float4 v = __ldcg(reinterpret_cast<const float4*>(p) + ((col + d) >> 2) * 128 + row);
                                y[d] += wt * v.x;
                                y[d + 1] += wt * v.y;
                                y[d + 2] += wt * v.z;
                                y[d + 3] += wt * v.w;
                            }
                        }
                        finish(col, y, m_all, l_all);
                    }
                }
                __syncwarp();
                meet();                // `last_here` is free again
            }
            tc_fence_before();
        });
    } else if (warp < 24) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ================= expanding warps: 4-bit tiles -> fp16 operands; eight warps for the keys, eight for the values
        // Four of the eight take a step, the other four the next one: half of a warp's time goes into waiting (a round of
        // barriers and copies takes 1,650 clocks, expanding a tile 320).  A warp takes two tiles and brings them itself, a few steps ahead, into slots of its own (sixteen bytes a thread and
        // copy: a bulk copy costs some 100 clocks to issue, however small).  A thread expands a quarter of the channels of tokens
        // lane / 4 and + 8: its reads are contiguous over the warp, and with the halves of the upper two quarters swapped its writes
        // fall into eight different 16-byte columns of the swizzled rows.
        const bool values = warp >= 16;
        const uint32_t stage = (warp >> 2) & 1;            // the steps that this warp takes, and where it puts them
        const int w = warp & 3, tok = lane >> 2, quarter = lane & 3;
        constexpr int QB = D / 8;                          // bytes of codes of a quarter
        constexpr int QW = D / 32, HW = QW / 2;            // words of it, and of half of it
        constexpr int R = Plan::kRawSlots;
        const int swap = D == 128 && quarter >= 2;
        uint32_t column[QW];                               // where the thread's 16-byte columns go, in a warp's share of a stage
#pragma unroll
        for (int k = 0; k < QW; ++k) {
            const int col = quarter * QW + (swap ? k ^ HW : k);
            column[k] = sm + (values ? Plan::kV : Plan::kK) + stage * Plan::kTileBytes + (col >> 3) * Plan::kChunkBytes + (w * 32 + tok) * 128 + (((col & 7) ^ tok) << 4);
        }
        const uint32_t raw = sm + Plan::kRaw + (warp - 8) * R * Plan::kRawHalf;
        const uint32_t codes_at = raw + tok * (D / 2) + quarter * QB, scales_at = raw + 8 * D + (D == 128 ? tok * 8 + quarter * 2 : tok * 4 + quarter);
        const uint32_t half0 = codes_at + (swap ? QB / 2 : 0), half1 = codes_at + (swap ? 0 : QB / 2);
        const uint32_t sel0 = D == 64 || !swap ? 0x1010 : 0x3232, sel1 = D == 64 || swap ? 0x1010 : 0x3232;
        constexpr int kCodeParts = 8 * D / 512;            // warp-wide copies of a tile's codes
        constexpr int kScaleLanes = D / 16;                // sixteen-byte parts of a tile's scales
        const uint32_t full_bar = ready_bar(stage), empty_bar = (values ? product_bar(0) : score_bar(0)) + 8 * stage;   // done with: by the products
        const int tile_mask = (c.page_tokens() >> 4) - 1;
        const uint32_t page_bytes = static_cast<uint32_t>(c.page_bytes >> 7);   // pages are multiples of 128 bytes
        uint32_t n = 0;                                    // steps in earlier pieces
        for_pieces([&](const WideSegment& g, int s0, int count) {
            const uint8_t* const head = c.head_tiles(0, a.layer, g.head) + (values ? 8 * D : 0) + lane * 16;
            const int until = all_until(g), after = all_after(g), base = g.ri.lo + s0 * kWideUnit, hi_token = kListed ? g.end : g.ri.hi;
            const int32_t* const list = kListed ? a.blocks + (static_cast<int64_t>(g.b) * c.n_kv + g.head) * a.n_blocks : nullptr;
            int begin_of = 0;                              // listed: positions of the first tokens of those tiles
            const int tile0 = (g.ri.lo >> 4) + w * 2;      // number of the warp's first tile of step 0
            int page_base = -16, page_of = -1;              // pages of the warp's tiles of sixteen steps: lane = 2 * (step - page_base) + tile
            const int first = (n ^ stage) & 1;             // our first step of the piece
            uint32_t present = 0;                          // two bits per slot
            auto fill = [&](int step, int slot) {          // the step's tiles into the slot, if it is one of ours
                if (step < s0 + count) {
                    if (step - page_base >= 16) {
                        page_base = step;
                        const int t = g.ri.lo + (step + (lane >> 1)) * kWideUnit + (w * 2 + (lane & 1)) * 16;
                        if constexpr (kListed) {
                            const int block = t < g.ri.hi && t >= 0 ? list[t >> c.log_p] : -1;
                            page_of = -1;
                            if (static_cast<unsigned>(block) < static_cast<unsigned>(c.max_pages)) {
                                begin_of = (block << c.log_p) + (t & (c.page_tokens() - 1));
                                if (begin_of < hi_token) page_of = c.page_at(g.ri.s, block);
                            }
                        } else {
                            page_of = t < g.ri.hi && t >= 0 ? c.page_at(g.ri.s, t >> c.log_p) : -1;
                        }
                    }
                    const uint32_t dst = raw + slot * Plan::kRawHalf + lane * 16;
                    uint32_t on = 0;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int page = __shfl_sync(0xffffffffu, page_of, 2 * (step - page_base) + x);
                        const int tile = (tile0 + step * 8 + x) & tile_mask;
                        if (page >= 0) {
                            on |= 1u << x;
                            const uint8_t* src = head + static_cast<uint64_t>(page) * page_bytes * 128 + tile * (18 * D);
#pragma unroll
                            for (int y = 0; y < kCodeParts; ++y) async_copy16(dst + x * (9 * D) + y * 512, src + y * 512);
                            if (lane < kScaleLanes) async_copy16(dst + x * (9 * D) + 8 * D, src + (values ? 9 * D : 16 * D));
                        }
                    }
                    present = (present & ~(3u << (2 * slot))) | on << (2 * slot);
                    if constexpr (kListed) {
                        const int begin0 = __shfl_sync(0xffffffffu, begin_of, 2 * (step - page_base)), begin1 = __shfl_sync(0xffffffffu, begin_of, 2 * (step - page_base) + 1);
                        if (lane == 0) slot_begin[warp - 8][slot] = make_int2(begin0, begin1);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll 1
            for (int k = 0; k < R; ++k) fill(s0 + first + 2 * k, k);
            int slot = 0;
#pragma unroll 1
            for (int k = first; k < count; k += 2) {
                asm volatile("cp.async.wait_group %0;" ::"n"(R - 1) : "memory");
                __syncwarp();
                const uint32_t there = (present >> (2 * slot)) & 3, from = slot * Plan::kRawHalf;
                uint32_t codes[4][2][HW], scales[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t at = from + (x >> 1) * (9 * D);
                    lds_words<HW>(at + half0 + (x & 1) * 8 * (D / 2), codes[x][0]);
                    lds_words<HW>(at + half1 + (x & 1) * 8 * (D / 2), codes[x][1]);
                    if constexpr (D == 128) {
                        uint16_t y;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(at + scales_at + (x & 1) * 64));
                        scales[x] = y;
                    } else {
                        scales[x] = lds8(at + scales_at + (x & 1) * 32) * 0x0101u;
                    }
                }
                int t0, t1;                                // positions of the first tokens of the two tiles
                if constexpr (kListed) {
                    const int2 begin = slot_begin[warp - 8][slot];
                    t0 = begin.x;
                    t1 = begin.y;
                }
                __syncwarp();
                fill(s0 + k + 2 * R, slot);
                if (++slot == R) slot = 0;
                const int first_token = base + k * kWideUnit;
                bool all;                                  // every row sees all of the step; listed: of the two tiles
                if constexpr (kListed) {
                    all = there == 3 && max(t0, t1) + 15 <= g.first_pos;
                } else {
                    t0 = first_token + w * 32;
                    t1 = t0 + 16;
                    all = first_token <= until && first_token > after;
                }
                if (!all || there != 3) {                  // what is absent or masked must not be multiplied with
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if (!((there >> (x >> 1)) & 1) || (values && (x < 2 ? t0 : t1) + (x & 1) * 8 + tok >= hi_token)) scales[x] = 0;
                        if (values && !all) {
                            if ((scales[x] & 0x7f) == 0x7f) scales[x] &= 0xff00;
                            if ((scales[x] & 0x7f00) == 0x7f00) scales[x] &= 0x00ff;
                        }
                    }
                }
                const uint32_t i = n + k;                  // number of the step in this CTA
                if (i >= 2) wait(empty_bar, ((i >> 1) - 1) & 1);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t f = e4m3x2_to_half2(scales[x]);
                    const uint32_t f0 = __byte_perm(f, f, sel0), f1 = __byte_perm(f, f, sel1);
#pragma unroll
                    for (int q = 0; q < QW; ++q) {
                        uint32_t y[4];
                        e2m1x8_to_half2(codes[x][q / HW][q % HW], y);
#pragma unroll
                        for (int z = 0; z < 4; ++z) y[z] = mul_half2(y[z], q < HW ? f0 : f1);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                     ::"r"(column[q] + x * 1024), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                    }
                }
                if (!values) {
                    const int ring = i & 3;
                    if (lane == 0) {
                        tile_there[ring][w] = static_cast<uint8_t>(there);
                        if constexpr (kListed) {
                            tile_all[ring][w] = all;
                            tile_begin[ring][2 * w] = t0;
                            tile_begin[ring][2 * w + 1] = t1;
                            if (all) nan_flag[ring][w] = 0;   // others' tiles may make the step one with masks
                        }
                    }
                    if (!all) {
                        // NaN among the values of these tokens, for the rows that do see them
                        uint32_t nans = 0;
#pragma unroll 1
                        for (int x = 0; x < 4; ++x) {
                            const int t = (x < 2 ? t0 : t1) + (x & 1) * 8 + tok;
                            if (!((there >> (x >> 1)) & 1) || t >= hi_token) continue;
                            const uint8_t* z = c.tile(c.page_at(g.ri.s, t >> c.log_p), a.layer, g.head, t & (c.page_tokens() - 1)) + 17 * D +
                                               ((x & 1) * 8 + tok) * (D / 16) + (D == 128 ? quarter * 2 : quarter);
                            const uint32_t s = D == 128 ? __ldg(reinterpret_cast<const uint16_t*>(z)) : __ldg(z);
                            if ((s & 0x7f) == 0x7f) nans |= 1u << (2 * x);
                            if (D == 128 && (s & 0x7f00) == 0x7f00) nans |= 2u << (2 * x);
                        }
                        const uint32_t flagged = __ballot_sync(0xffffffffu, nans != 0);
                        if (flagged) {
#pragma unroll 1
                            for (int x = 0; x < 4; ++x) {
                                // blocks of a quarter: two at 128 channels, one at 64
                                uint32_t m = D == 128 ? ((nans >> (2 * x)) & 3) << (2 * quarter) : ((nans >> (2 * x)) & 1) << quarter;
                                m |= __shfl_xor_sync(0xffffffffu, m, 1);
                                m |= __shfl_xor_sync(0xffffffffu, m, 2);
                                if (quarter == 0) nan_block[ring][w * 32 + x * 8 + tok] = static_cast<uint8_t>(m);
                            }
                        }
                        if (lane == 0) nan_flag[ring][w] = flagged != 0;
                    }
                }
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) barrier_arrive(!values && i < 2 ? k_first(stage) : full_bar);
            }
            n += count;
        });
        // the last two steps wait for keys as the others do
        const uint32_t beyond = n + ((n ^ stage) & 1);
        if (!values && beyond >= 2) {
            wait(empty_bar, ((beyond >> 1) - 1) & 1);
            if (lane == 0) barrier_arrive(full_bar);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (warp == 24) {
        // ================= issuing warp
        if (lane == 0) {
            constexpr uint32_t kScoreDesc = product_desc(128, 128, false), kSumDesc = product_desc(128, D, true);
            const uint64_t k_desc = operand_desc(sm + Plan::kK, 16, 1024), v_desc = operand_desc(sm + Plan::kV, Plan::kChunkBytes, 1024);
            uint32_t n = 0, n_query = 0;                 // steps in earlier pieces
            for_pieces([&](const WideSegment&, int, int count) {
                auto scores = [&](uint32_t i) {          // S of step i
                    const int stage = i & 1;
                    const uint64_t k = k_desc + stage * (Plan::kTileBytes >> 4);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        tc_mma_ts(tmem + kColS + stage * 128, tmem + kColQ + x * 8, k + (((x >> 2) * Plan::kChunkBytes + (x & 3) * 32) >> 4), kScoreDesc, x > 0);
                    tc_commit(score_bar(stage));
                };
                wait(query_bar, n_query++ & 1);
                for (int k = 0; k < 2 && k < count; ++k) {
                    if (n + k < 2) wait(k_first(n + k), 0);
                    tc_fence_after();
                    scores(n + k);
                }
#pragma unroll 1
                for (int k = 0; k < count; ++k, ++n) {
                    const int stage = n & 1;
                    wait(ready_bar(stage), (n >> 1) & 1);
                    tc_fence_after();
                    const uint64_t v = v_desc + stage * (Plan::kTileBytes >> 4);
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        tc_mma_ts(tmem + kColO, tmem + kColS + stage * 128 + (x >> 2) * 64 + (x & 3) * 8, v + x * (2048 >> 4), kSumDesc, k > 0 || x > 0);
                    tc_commit(product_bar(stage));
                    if (k + 2 < count) scores(n + 2);
                }
            });
        }
        __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (abort_flag) __nanosleep(100000);               // products still under way
    if (warp == 24) tmem_free(tmem, 512);
    if (tid == 0 && abort_flag && c.meta) atomicOr(&c.meta[1], kStatusGaveUp);
}

}  // namespace samb200
