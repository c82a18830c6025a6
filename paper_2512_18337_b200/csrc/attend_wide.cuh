// Attention for many query rows per key/value head (proposals of several heads, prompt chunks): tcgen05 products.
//
// S = Q K^T and O += P V on 128-row tiles, with 128 tokens a step.  Four warps expand the 4-bit tiles into two stages of fp16
// keys and two of fp16 values in shared memory (exact: a value has six significant bits); Q lies there too, S and O in tensor
// memory.  A thread of a softmax group owns one query row, so its maximum and its sum need no exchange; it writes P as fp16
// over S, from where the second product takes it.  Two groups alternate, so that one group's exponentials run under the other's
// products: with more than 128 query rows they hold two row tiles that share the expanded keys and values (kPair), otherwise
// they take the steps of one row tile in turn and are joined at the end of the segment.
//
// Keys and values have the same layout in shared memory, [token][64 channels] in 128-byte rows with the 128-byte swizzle: for
// the first product it is read with the channels (the summed index) innermost, for the second with the channels as the N side.
//
// The reference of the weights follows the rule of attend_stream.cuh: a row's sums are rescaled only when a score lies 15
// (powers of two) above it.
#pragma once

#include "attend_stream.cuh"

namespace samb200 {

constexpr int kWideUnit = 128;                     // tokens of a step
constexpr int kWideWarps = 20, kWideThreads = kWideWarps * 32;   // two softmax groups and two expanding groups of four warps, one issuing warp (and three that idle)
constexpr int kWideMaxCtas = 160;

template <int D, bool kPair>
struct WidePlan {
    static constexpr int kRows = kPair ? 256 : 128;                     // query rows of a segment
    static constexpr int kTileBytes = 128 * D * 2;                      // a [128][D] fp16 operand
    static constexpr int kChunkBytes = 128 * 128;                       // 64 channels of it
    static constexpr int kQ = 0, kK = (kPair ? 2 : 1) * kTileBytes, kV = kK + 2 * kTileBytes;
    static constexpr int kRaw = kV + 2 * kTileBytes;                    // slots of the expanding warps: two tiles' keys or values each
    static constexpr int kRawSlots = kPair && D == 128 ? 1 : 3, kRawHalf = 18 * D;
    static constexpr int kSmem = kRaw + 8 * kRawSlots * kRawHalf + 1024;   // and room to start on a 1024-byte boundary
    static constexpr int kPartTile = 128 * D + 2 * 128;                 // floats of a row tile's partial result
    static constexpr int kPart = (kPair ? 2 : 1) * kPartTile;
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
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
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

// A segment: one row of the batch, one row tile (kRows query rows), one key/value head; its steps cover the tokens that some
// query row of it sees.  Segments are numbered by row, row tile, head.
struct WideSegment {
    RowInfo ri;          // lo, hi: of this row tile
    int b, rt, head, steps;
    int rows;            // query rows of the tile
    int first_pos, last_pos;
    int64_t begin;       // number of its first unit
};
template <int kRows>
__device__ __forceinline__ void wide_tile(const AttendArgs& a, int tiles, int64_t e, WideSegment& g) {   // e = b * tiles + rt
    g.b = static_cast<int>(e / tiles);
    g.rt = static_cast<int>(e % tiles);
    g.ri = row_info<kWideUnit>(a, g.b);
    g.rows = min(g.ri.n * a.group - g.rt * kRows, kRows);
    g.steps = 0;
    if (g.rows <= 0) return;
    const int i0 = g.rt * kRows / a.group, i1 = (g.rt * kRows + g.rows - 1) / a.group, cap = a.c.capacity();
    g.first_pos = g.ri.len + i0;
    g.last_pos = g.ri.len + i1;
    g.ri.hi = static_cast<int>(min(static_cast<int64_t>(g.ri.len) + i1 + 1, static_cast<int64_t>(cap)));
    g.ri.lo = a.window > 0 ? min(max(g.first_pos - a.window + 1, 0), cap - 1) & ~(kWideUnit - 1) : 0;
    g.steps = max((g.ri.hi - g.ri.lo + kWideUnit - 1) / kWideUnit, 1);
}

template <typename T, int D, bool kPair>
__global__ void __launch_bounds__(kWideThreads, 1) attend_wide_kernel(const __grid_constant__ AttendArgs a) {
    using Plan = WidePlan<D, kPair>;
    constexpr int kRows = Plan::kRows;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[14];
    __shared__ uint32_t tmem_base;
    __shared__ int64_t scan[kWideWarps], start_e, start_begin;
    __shared__ float2 stats[2][128];
    __shared__ uint32_t stat_nan[2][128];
    __shared__ alignas(4) uint8_t tile_there[4][4];    // per step (mod 4) and expanding warp: which of its two tiles are there
    __shared__ uint32_t nan_flag[4][4];                // per step and expanding warp: NaN among the values of its tokens
    __shared__ uint8_t nan_block[4][128];              // which 16-channel blocks of a token's values are NaN
    __shared__ int last_here;
    __shared__ volatile int abort_flag;

    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sm = shared_addr(smem), bar = shared_addr(bars);
    // barriers: scores ready / weights ready per group, keys and values full / empty per stage, queries ready, both groups
    auto score_bar = [&](int g) { return bar + 8 * g; };
    auto weight_bar = [&](int g) { return bar + 16 + 8 * g; };
    auto k_full = [&](int s) { return bar + 32 + 8 * s; };
    auto k_empty = [&](int s) { return bar + 48 + 8 * s; };
    auto v_full = [&](int s) { return bar + 64 + 8 * s; };
    auto v_empty = [&](int s) { return bar + 80 + 8 * s; };
    const uint32_t query_bar = bar + 96, both_bar = bar + 104;
    auto wait = [&](uint32_t b, uint32_t parity) {     // false: give up (here or elsewhere in the CTA)
        for (uint32_t i = 0; i < kCachePolls; ++i) {
            if (barrier_try(b, parity)) return true;
            if ((i & 63) == 63 && abort_flag) return false;
        }
        abort_flag = 1;
        return false;
    };

    if (tid == 0) {
        for (int g = 0; g < 2; ++g) {
            barrier_init(score_bar(g), 1);
            barrier_init(weight_bar(g), 4);
            barrier_init(k_full(g), 4);
            barrier_init(k_empty(g), 1);
            barrier_init(v_full(g), 4);
            barrier_init(v_empty(g), 1);
        }
        barrier_init(query_bar, 8);
        barrier_init(both_bar, 8);
        abort_flag = 0;
    }
    barrier_init_fence();

    // ---- how many units there are, and where our share begins
    const int tiles = static_cast<int>((static_cast<int64_t>(a.Q) * a.group + kRows - 1) / kRows);
    const int64_t n_tiles = static_cast<int64_t>(a.B) * tiles;
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
        wide_tile<kRows>(a, tiles, e, g);
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
    if (warp == 16) tmem_alloc(shared_addr(&tmem_base), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    // Runs f(segment, first step, steps, index) over the pieces of our share; f returns false to stop.
    auto for_pieces = [&](auto f) {
        WideSegment g;
        int64_t e = start_e;
        wide_tile<kRows>(a, tiles, e, g);
        const int64_t rel = u0 - start_begin;
        g.head = static_cast<int>(rel / g.steps);
        g.begin = start_begin + static_cast<int64_t>(g.head) * g.steps;
        int64_t u = u0;
        for (int index = 0;; ++index) {
            const int s0 = static_cast<int>(u - g.begin);
            const int count = static_cast<int>(min(u1 - u, static_cast<int64_t>(g.steps - s0)));
            if (!f(g, s0, count)) return;
            u += count;
            if (u >= u1) return;
            g.begin += g.steps;
            if (++g.head == c.n_kv) {
                g.head = 0;
                const int64_t next = g.begin;
                do wide_tile<kRows>(a, tiles, ++e, g);
                while (g.steps == 0 && e + 1 < n_tiles);
                g.begin = next;
            }
        }
    };
    auto seen_by_all = [&](const WideSegment& g, int t0) {
        return t0 + kWideUnit - 1 <= g.first_pos && (a.window == 0 || t0 > g.last_pos - a.window);
    };

    // Registers go where they are needed: 2 x 128 threads x 136, 2 x 128 x 72, 128 x 64, of 640 x 96 at launch.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        // ================= softmax groups
        const int g = warp >> 2, row = tid & 127, quarter_lane = (warp & 3) << 21;   // lane quarter in the tensor-memory address
        const uint32_t s_at = tmem + quarter_lane + g * 128, o_at = tmem + quarter_lane + 256 + g * 128;
        uint32_t n_score = 0, n_both = 0, kt = 0;
        auto both = [&]() -> bool {                     // meets the other group
            __syncwarp();
            if (lane == 0) barrier_arrive(both_bar);
            return wait(both_bar, n_both++ & 1);
        };
        for_pieces([&](const WideSegment& seg, int s0, int count) {
            // ---- queries into shared memory
            const int rho_tile = seg.rt * kRows + (kPair ? g * 128 : 0);     // first query row of this group's tile
            const bool mine = (kPair ? g * 128 : 0) + row < seg.rows;
            const int rho = rho_tile + row, qi = rho / a.group, qh = seg.head * a.group + rho % a.group;
            float factor;
            {
                // without a pair both groups hold the same rows and write half the channels each
                constexpr int kPart = kPair ? D : D / 2;
                const T* q = static_cast<const T*>(a.q) + seg.b * a.q_row + static_cast<int64_t>(qi) * a.q_token + static_cast<int64_t>(qh) * a.q_head;
                int e = 0;
                float up = 1.f;
                if constexpr (!std::is_same<T, __half>::value) {
                    float big = 0.f;
                    if (mine)
                        for (int d = 0; d < D; d += 8) {
                            alignas(16) T x[8];
                            if (a.q_wide) *reinterpret_cast<uint4*>(x) = __ldg(reinterpret_cast<const uint4*>(q + d));
                            else
                                for (int i = 0; i < 8; ++i) x[i] = q[d + i];
#pragma unroll
                            for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(Elem<T>::to_float(x[i])));
                        }
                    e = big > 0.f ? min(14 - (static_cast<int>(__float_as_uint(big) >> 23) - 127), 126) : 0;
                    up = pow2(e);
                }
                if (a.scale < 0.f) up = -up;                 // so that the largest score is the largest product
                factor = scale_pow2(fabsf(a.scale) * 1.4426950408889634f, c.k_exp - e);
                const uint32_t base = sm + Plan::kQ + (kPair ? g : 0) * Plan::kTileBytes + row * 128;
                const int d0 = kPair ? 0 : g * kPart;
#pragma unroll 4
                for (int d = d0; d < d0 + kPart; d += 8) {
                    uint32_t y[4] = {0, 0, 0, 0};
                    if (mine) {
                        alignas(16) T x[8];
                        if (a.q_wide) *reinterpret_cast<uint4*>(x) = __ldg(reinterpret_cast<const uint4*>(q + d));
                        else
                            for (int i = 0; i < 8; ++i) x[i] = q[d + i];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (std::is_same<T, __half>::value) y[i] = reinterpret_cast<const uint32_t*>(x)[i] ^ (up < 0.f ? 0x80008000u : 0u);
                            else y[i] = pack_half2(Elem<T>::to_float(x[2 * i]) * up, Elem<T>::to_float(x[2 * i + 1]) * up);
                        }
                    }
                    const uint32_t at = base + (d >> 6) * Plan::kChunkBytes + ((((d & 63) >> 3) ^ (row & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                }
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) barrier_arrive(query_bar);
            }
            const int pos = mine ? seg.ri.len + qi : -1;
            float m = -INFINITY, l = 0.f;
            uint32_t nan_blocks = 0;

            // ---- steps
            const int first = kPair ? 0 : g, by = kPair ? 1 : 2;
            for (int k = first; k < count; k += by) {
                if (!wait(score_bar(g), n_score++ & 1)) return false;
                tc_fence_after();
                const int t0 = seg.ri.lo + (s0 + k) * kWideUnit, ring = (kt + k) & 3;
                uint32_t on = *reinterpret_cast<volatile uint32_t*>(tile_there[ring]);
                on = (on & 3) | (on >> 6 & 0xc) | (on >> 12 & 0x30) | (on >> 18 & 0xc0);
                const bool all = seen_by_all(seg, t0);
                const bool full = all && on == 0xff;
                if (!all) {
                    volatile uint32_t* flags = nan_flag[ring];
                    if (flags[0] | flags[1] | flags[2] | flags[3])
                        for (int t = 0; t < kWideUnit; ++t)
                            if (flags[t >> 5] && t0 + t <= pos && (a.window == 0 || t0 + t > pos - a.window)) nan_blocks |= static_cast<volatile uint8_t*>(nan_block[ring])[t];
                }
                // Both passes over the scores (their largest; their weights) exist twice: without masks in one straight run, with the
                // next 32 columns on the way, and with masks as a small loop - a run of masked code does not fit the instruction cache.
                auto seen = [&](int t) { return ((on >> (t >> 4)) & 1) && t0 + t <= pos && (a.window == 0 || t0 + t > pos - a.window); };
                float top = -INFINITY;
                uint32_t x[2][32];
                if (full) {
                    tmem_load32(s_at, x[0]);
#pragma unroll 1
                    for (int q = 0; q < 128; q += 64) {
                        tmem_load_wait(x[0]);
                        tmem_load32(s_at + q + 32, x[1]);
#pragma unroll
                        for (int i = 0; i < 32; i += 2) top = fmaxf(fmaxf(top, __uint_as_float(x[0][i])), __uint_as_float(x[0][i + 1]));
                        tmem_load_wait(x[1]);
                        tmem_load32(s_at + (q ^ 64), x[0]);          // the last one is the first of the second pass
#pragma unroll
                        for (int i = 0; i < 32; i += 2) top = fmaxf(fmaxf(top, __uint_as_float(x[1][i])), __uint_as_float(x[1][i + 1]));
                    }
                } else {
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        tmem_load32(s_at + q * 32, x[0]);
                        tmem_load_wait(x[0]);
#pragma unroll
                        for (int i = 0; i < 32; ++i) top = fmaxf(top, seen(q * 32 + i) ? __uint_as_float(x[0][i]) : -INFINITY);
                    }
                }
                top *= factor;
                if (__any_sync(0xffffffffu, top > m + kRaiseAt)) {
                    const float to = top > m + kRaiseAt ? top - kAbove : m;
                    const float keep = m == -INFINITY ? 0.f : exp2_fast(m - to);
                    if (k >= first + by) {               // the sums so far; the group's last product is complete (it came before these scores)
#pragma unroll 1
                        for (int q = 0; q < D / 16; ++q) {
                            uint32_t o[16];
                            tmem_load16(o_at + q * 16, o);
                            tmem_load_wait(o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
                            tmem_store16(o_at + q * 16, o);
                        }
                    }
                    l *= keep;
                    m = to;
                }
                const float ref = m == -INFINITY ? 0.f : m;
                float2 total = make_float2(0.f, 0.f);
                if (full) {
                    auto weights = [&](const uint32_t (&s)[32], int at) {
                        uint32_t p[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float2 y = fma2(make_float2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), make_float2(factor, factor), make_float2(-ref, -ref));
                            y.x = exp2_fast(y.x);
                            y.y = exp2_fast(y.y);
                            total = add2(total, y);
                            p[i / 2] = pack_half2(y.x, y.y);
                        }
                        tmem_store16(s_at + at, p);                  // behind the scores that are still to be read
                    };
#pragma unroll 1
                    for (int q = 0; q < 128; q += 64) {
                        tmem_load_wait(x[0]);
                        tmem_load32(s_at + q + 32, x[1]);
                        weights(x[0], q / 2);
                        tmem_load_wait(x[1]);
                        if (q == 0) tmem_load32(s_at + 64, x[0]);
                        weights(x[1], q / 2 + 16);
                    }
                } else {
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        tmem_load32(s_at + q * 32, x[0]);
                        tmem_load_wait(x[0]);
                        uint32_t p[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float2 y = make_float2(fmaf(__uint_as_float(x[0][i]), factor, -ref), fmaf(__uint_as_float(x[0][i + 1]), factor, -ref));
                            y.x = exp2_fast(seen(q * 32 + i) ? y.x : -INFINITY);
                            y.y = exp2_fast(seen(q * 32 + i + 1) ? y.y : -INFINITY);
                            total = add2(total, y);
                            p[i / 2] = pack_half2(y.x, y.y);
                        }
                        tmem_store16(s_at + q * 16, p);
                    }
                }
                l += total.x + total.y;
                tmem_store_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(weight_bar(g));
            }
            kt += count;

            // ---- the piece's result
            const bool worked = first < count;
            if (worked) {
                if (!wait(score_bar(g), n_score++ & 1)) return false;
                tc_fence_after();
            }
            const bool begins = s0 == 0, ends = s0 + count == seg.steps;
            float m2 = -INFINITY, w1 = 1.f, w2 = 0.f, top = m, tot = l;
            bool have1 = true, have2 = false;
            if (!kPair) {
                stats[g][row] = make_float2(m, l);
                stat_nan[g][row] = nan_blocks;
                if (!both()) return false;
                tc_fence_after();
                const float2 s1 = stats[0][row], s2 = stats[1][row];
                nan_blocks = stat_nan[0][row] | stat_nan[1][row];
                m2 = s2.x;
                top = fmaxf(s1.x, m2);
                w1 = join_weight(s1.x, top);
                w2 = join_weight(m2, top);
                tot = w1 * s1.y + w2 * s2.y;
                have2 = count > 1;
            }
            (void)have1;
            const uint32_t o1 = tmem + quarter_lane + 256 + (kPair ? g * 128 : 0), o2 = tmem + quarter_lane + 256 + 128;
            constexpr int kCols = kPair ? D : D / 2;
            const int col0 = kPair ? 0 : g * kCols;
            // sums of 32 channels
            auto sums = [&](int col, float (&y)[32]) {
                uint32_t x[32];
                tmem_load32(o1 + col, x);
                tmem_load_wait(x);
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = kPair ? __uint_as_float(x[i]) : __uint_as_float(x[i]) * w1;
                if (have2) {
                    tmem_load32(o2 + col, x);
                    tmem_load_wait(x);
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i] += __uint_as_float(x[i]) * w2;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if ((nan_blocks >> ((col + i) >> 4)) & 1) y[i] = __int_as_float(0x7fffffff);
            };
            auto finish = [&](int col, float (&y)[32], float m_all, float l_all) {
                const float f = finish_factor(l_all, c.v_exp);
#pragma unroll
                for (int i = 0; i < 32; ++i) y[i] = l_all == 0.f ? 0.f : y[i] * f;
                store_row<T>(static_cast<T*>(a.out) + seg.b * a.o_row + static_cast<int64_t>(qi) * a.o_token + static_cast<int64_t>(qh) * a.o_head + col, y, a.o_wide);
                if (a.lse && col == 0) a.lse[(static_cast<int64_t>(seg.b) * a.Q + qi) * a.H + qh] = finish_lse(m_all, l_all);
            };
            if (begins && ends) {
#pragma unroll 1
                for (int col = col0; col < col0 + kCols; col += 32) {
                    float y[32];
                    sums(col, y);
                    if (mine) finish(col, y, top, tot);
                }
            } else {
                // [D / 4][128] float4, then references and totals
                auto part = [&](int owner, bool first_piece) {
                    return a.partials + (2ll * owner + first_piece) * Plan::kPart + (kPair ? g * Plan::kPartTile : 0);
                };
                float* out = part(cta, begins);
#pragma unroll 1
                for (int col = col0; col < col0 + kCols; col += 32) {
                    float y[32];
                    sums(col, y);
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        reinterpret_cast<float4*>(out)[((col + i) >> 2) * 128 + row] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                }
                if (col0 == 0) {
                    out[128 * D + row] = top;
                    out[128 * D + 128 + row] = tot;
                }
                __threadfence();
                if (!both()) return false;
                const int c0 = shares.owner(seg.begin), c1 = shares.owner(seg.begin + seg.steps - 1);
                if (tid == 0) {
                    last_here = atomicAdd(&a.counters[c0], 1) == c1 - c0;
                    if (last_here) a.counters[c0] = 0;
                    __threadfence();
                }
                if (!both()) return false;
                if (*static_cast<volatile int*>(&last_here)) {
                    __threadfence();
                    const int n = c1 - c0 + 1;
                    float m_all = -INFINITY, l_all = 0.f;
#pragma unroll 4
                    for (int i = 0; i < n; ++i) m_all = fmaxf(m_all, __ldcg(part(c0 + i, i == 0) + 128 * D + row));
#pragma unroll 4
                    for (int i = 0; i < n; ++i) {
                        const float* p = part(c0 + i, i == 0) + 128 * D + row;
                        l_all += join_weight(__ldcg(p), m_all) * __ldcg(p + 128);
                    }
#pragma unroll 1
                    for (int col = col0; col < col0 + kCols; col += 32) {
                        float y[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = 0.f;
#pragma unroll 1
                        for (int i = 0; i < n; ++i) {
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
                        if (mine) finish(col, y, m_all, l_all);
                    }
                }
            }
            // the next piece writes the queries and the sums anew: both groups are through with these
            tc_fence_before();
            return both();
        });
    } else if (warp < 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        // ================= expanding warps: 4-bit tiles -> fp16 operands; four warps for the keys, four for the values
        // A warp takes two tiles of a step and brings them itself, a few steps ahead, into slots of its own (sixteen bytes a thread and
        // copy: a bulk copy costs some 100 clocks to issue, however small).  A thread expands a quarter of the channels of tokens
        // lane / 4 and + 8: its reads are contiguous over the warp, and with the words of the upper two quarters swapped its writes
        // fall into eight different 16-byte columns of the swizzled rows.
        const bool values = warp >= 12;
        const int w = warp & 3, tok = lane >> 2, quarter = lane & 3;
        constexpr int QB = D / 8;                          // bytes of codes of a quarter
        constexpr int QW = D / 32;                         // words
        constexpr int R = Plan::kRawSlots;
        const bool swap = D == 128 && quarter >= 2;
        uint32_t column[QW];                               // where the thread's 16-byte columns go, in a warp's share of a stage
#pragma unroll
        for (int k = 0; k < QW; ++k) {
            const int col = quarter * QW + (swap ? k ^ 2 : k);
            column[k] = sm + (values ? Plan::kV : Plan::kK) + (col >> 3) * Plan::kChunkBytes + (w * 32 + tok) * 128 + (((col & 7) ^ tok) << 4);
        }
        const uint32_t raw = sm + Plan::kRaw + (warp - 8) * R * Plan::kRawHalf;
        const uint32_t codes_at = raw + tok * (D / 2) + quarter * QB, scales_at = raw + 8 * D + (D == 128 ? tok * 8 + quarter * 2 : tok * 4 + quarter);
        constexpr int kCodeParts = 8 * D / 512;            // warp-wide copies of a tile's codes
        constexpr int kScaleLanes = D / 16;                // sixteen-byte parts of a tile's scales
        uint32_t n = 0;                                    // halves expanded so far
        for_pieces([&](const WideSegment& g, int s0, int count) {
            const uint8_t* const head = c.head_tiles(0, a.layer, g.head) + (values ? 8 * D : 0);
            // pages of the warp's tiles of sixteen steps: lane = 2 * (step - page_base) + tile
            int page_base = s0, page_of = -1, slot = 0;
            uint32_t present = 0;                          // two bits per slot
            auto fill = [&](int step) {                    // the step's tiles into the slot, if it is one of ours
                if (step < s0 + count) {
                    if (step - page_base >= 16 || step == s0) {
                        page_base = step;
                        const int t = g.ri.lo + (step + (lane >> 1)) * kWideUnit + (w * 2 + (lane & 1)) * 16;
                        page_of = t < g.ri.hi && t >= 0 ? c.page_at(g.ri.s, t >> c.log_p) : -1;
                    }
                    const int t0 = g.ri.lo + step * kWideUnit + w * 32;
                    const uint32_t dst = raw + slot * Plan::kRawHalf + lane * 16;
                    present &= ~(3u << (2 * slot));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int page = __shfl_sync(0xffffffffu, page_of, 2 * (step - page_base) + x);
                        if (page < 0) continue;
                        present |= 1u << (2 * slot + x);
                        const uint8_t* src = head + page * c.page_bytes + (((t0 + x * 16) & (c.page_tokens() - 1)) >> 4) * (18 * D) + lane * 16;
#pragma unroll
                        for (int y = 0; y < kCodeParts; ++y) async_copy16(dst + x * (9 * D) + y * 512, src + y * 512);
                        // scales: D bytes, 8 D (values) or 15 D further on for keys
                        if (lane < kScaleLanes) async_copy16(dst + x * (9 * D) + 8 * D, src + (values ? 9 * D : 16 * D));
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll 1
            for (int k = 0; k < R; ++k, ++slot) fill(s0 + k);
            slot = 0;
#pragma unroll 1
            for (int k = 0; k < count; ++k, ++n) {
                asm volatile("cp.async.wait_group %0;" ::"n"(R - 1) : "memory");
                __syncwarp();
                const int stage = n & 1;
                const uint32_t there = present >> (2 * slot);
                uint32_t codes[4][QW], scales[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t at = slot * Plan::kRawHalf + (x >> 1) * (9 * D);
                    lds_words<QW>(at + codes_at + (x & 1) * 8 * (D / 2), codes[x]);
                    if constexpr (D == 128) {
                        uint16_t y;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(at + scales_at + (x & 1) * 64));
                        scales[x] = y;
                    } else {
                        scales[x] = lds8(at + scales_at + (x & 1) * 32);
                    }
                }
                __syncwarp();
                fill(s0 + k + R);
                if (++slot == R) slot = 0;
                if (n >= 2 && !wait(values ? v_empty(stage) : k_empty(stage), ((n >> 1) - 1) & 1)) return false;
                const int t0 = g.ri.lo + (s0 + k) * kWideUnit + w * 32;
                const bool all = seen_by_all(g, g.ri.lo + (s0 + k) * kWideUnit);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    uint32_t s = (there >> (x >> 1)) & 1 ? scales[x] : 0;
                    if (values && !all) {   // what is masked must not be multiplied with
                        if (t0 + x * 8 + tok >= g.ri.hi) s = 0;
                        if ((s & 0x7f) == 0x7f) s &= 0xff00;
                        if ((s & 0x7f00) == 0x7f00) s &= 0x00ff;
                    }
                    const uint32_t f = e4m3x2_to_half2(D == 128 ? s : s * 0x0101u);
                    const uint32_t f0 = D == 128 ? __byte_perm(f, f, swap ? 0x3232 : 0x1010) : f, f1 = D == 128 ? __byte_perm(f, f, swap ? 0x1010 : 0x3232) : f;
#pragma unroll
                    for (int q = 0; q < QW; ++q) {
                        uint32_t y[4];
                        e2m1x8_to_half2(D == 128 && swap ? codes[x][q ^ (QW / 2)] : codes[x][q], y);
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = mul_half2(y[i], q < QW / 2 ? f0 : f1);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                     ::"r"(column[q] + stage * Plan::kTileBytes + x * 1024), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                    }
                }
                if (!values) {
                    const int ring = n & 3;
                    uint32_t flagged = 0;
                    if (!all) {
                        // NaN among the values of these tokens, for the rows that do see them
                        uint32_t nans = 0;
#pragma unroll 1
                        for (int x = 0; x < 4; ++x) {
                            const int t = t0 + x * 8 + tok;
                            if (!((there >> (x >> 1)) & 1) || t >= g.ri.hi) continue;
                            const uint8_t* z = c.tile(c.page_at(g.ri.s, t >> c.log_p), a.layer, g.head, t & (c.page_tokens() - 1)) + 17 * D +
                                               ((x & 1) * 8 + tok) * (D / 16) + (D == 128 ? quarter * 2 : quarter);
                            const uint32_t s = D == 128 ? __ldg(reinterpret_cast<const uint16_t*>(z)) : __ldg(z);
                            if ((s & 0x7f) == 0x7f) nans |= 1u << (2 * x);
                            if (D == 128 && (s & 0x7f00) == 0x7f00) nans |= 2u << (2 * x);
                        }
                        flagged = __ballot_sync(0xffffffffu, nans != 0);
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
                    }
                    if (lane == 0) {
                        nan_flag[ring][w] = flagged;
                        tile_there[ring][w] = static_cast<uint8_t>(there & 3);
                    }
                }
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) barrier_arrive(values ? v_full(stage) : k_full(stage));
            }
            return true;
        });
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 16) {
        // ================= issuing warp
        if (lane == 0) {
            constexpr uint32_t kScoreDesc = product_desc(128, 128, false), kSumDesc = product_desc(128, D, true);
            const uint64_t q_desc = operand_desc(sm + Plan::kQ, 16, 1024), k_desc = operand_desc(sm + Plan::kK, 16, 1024);
            const uint64_t v_desc = operand_desc(sm + Plan::kV, Plan::kChunkBytes, 1024);
            uint32_t kt = 0, vt = 0, n_query = 0, n_weight[2] = {0, 0};
            for_pieces([&](const WideSegment&, int, int count) {
                const int jobs = kPair ? 2 * count : count;
                if (!wait(query_bar, n_query++ & 1)) return false;
                tc_fence_after();
                auto scores = [&](int n) -> bool {      // S of job n
                    const int g = n & 1, tile = kPair ? n >> 1 : n, stage = (kt + tile) & 1;
                    if ((!kPair || g == 0) && !wait(k_full(stage), ((kt + tile) >> 1) & 1)) return false;
                    tc_fence_after();
                    const uint64_t q = q_desc + (kPair ? g : 0) * (Plan::kTileBytes >> 4), k = k_desc + stage * (Plan::kTileBytes >> 4);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t off = ((i >> 2) * Plan::kChunkBytes + (i & 3) * 32) >> 4;
                        tc_mma_ss(tmem + g * 128, q + off, k + off, kScoreDesc, i > 0);
                    }
                    tc_commit(score_bar(g));
                    if (!kPair || g == 1) tc_commit(k_empty(stage));
                    return true;
                };
                if (!scores(0)) return false;
                for (int n = 0; n < jobs; ++n) {
                    if (n + 1 < jobs && !scores(n + 1)) return false;
                    const int g = n & 1, tile = kPair ? n >> 1 : n, stage = (vt + tile) & 1;
                    if ((!kPair || g == 0) && !wait(v_full(stage), ((vt + tile) >> 1) & 1)) return false;
                    if (!wait(weight_bar(g), n_weight[g]++ & 1)) return false;
                    tc_fence_after();
                    const uint64_t v = v_desc + stage * (Plan::kTileBytes >> 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) tc_mma_ts(tmem + 256 + g * 128, tmem + g * 128 + i * 8, v + i * (2048 >> 4), kSumDesc, n > 1 || i > 0);
                    if (!kPair || g == 1) tc_commit(v_empty(stage));
                    if (n + 2 >= jobs) tc_commit(score_bar(g));   // the group's last: its sums are complete
                }
                kt += count;
                vt += count;
                return true;
            });
        }
        __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 16) tmem_free(tmem, 512);
    if (tid == 0 && abort_flag && c.meta) atomicOr(&c.meta[1], kStatusGaveUp);
}

}  // namespace samb200
