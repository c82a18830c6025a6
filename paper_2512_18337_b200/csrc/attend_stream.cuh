// Attention for few query rows per key/value head (a token, a short proposal): streams the cache through the tensor cores.
//
// The scores are computed transposed, S^T = K Q^T with m16n8k16: sixteen tokens make the M side and eight query rows the
// N side, so one query row wastes 7/8 of the products instead of 15/16, and products are not what bounds it.  A thread reads
// its A fragment of K (two tokens, a quarter of the channels) straight out of the 4-bit tile, expands it to fp16 in registers
// (exact: a code has two significant bits and a scale four) and feeds it to the tensor core; the order of the channels inside
// a product is free, so no shuffle is needed.  O^T = V^T P^T takes P^T from S^T's accumulator through a register transpose
// (movmatrix) and V^T by interleaving the nibbles of two tokens before they are expanded.  Scales, statistics and sums are
// 32-bit; the only rounding beyond the result's is that of the weights to fp16.  bf16 queries are scaled per row by a power of
// two into fp16's range, which keeps every bit that reaches 2^-28 of the row's largest.
//
// Weights are 2^(score - reference) with a reference that is set 11 below the largest score and raised again only when some
// score comes 15 above it: one vote per 32 tokens instead of three shuffles per query row.  Weights then lie below 2^15, within
// fp16, and those down to 2^-21 of the largest keep all 11 bits.
//
// A warp is on its own: it has a ring of kStages units (32 tokens, 4.6 KB at 128 channels) filled by bulk copies, and runs
// from unit to unit, over the ends of segments.  Results of segments that end inside the warp's share are written directly;
// the others meet in shared memory, and through global memory where a segment crosses CTAs.
//
// What it measured, from clocks that its warps wrote down: two streams of 250,001 positions, 64/8 heads of 128: 143 us, 4.0 TB/s.
// The first tiles are there after 8 us (numbering, then a chain of dependent loads), half of the warps are through after 112, the
// last after 125, and joining takes the other 18.  Until then 5.6 TB/s are read, 0.85 of the copy rate, with 0.7 of the issue slots
// (677 instructions per unit).  32 streams of 4,400 on average: 57 us for 159 MB, 8 + 32 (at 5.0 TB/s) + 7 until the last warp + 10
// for joining.  So it is the ends that bound it: the start, warps that are not through together, and the joining.
#pragma once

#include <type_traits>

#include "cache_attend.cuh"

namespace samb200 {

constexpr int kStreamWarps = 8, kStreamThreads = kStreamWarps * 32;
constexpr int kStreamUnit = 32;       // tokens of a unit: two tiles
constexpr float kAbove = 11.f, kRaiseAt = 15.f;   // log2 of the largest weight after the reference was set, and at most

template <int D, int NT>
struct StreamPlan {
    static constexpr int kTile = 18 * D, kUnitBytes = 2 * kTile;
    static constexpr int kRows = 8 * NT;
    static constexpr int kPiece = kRows * D + 2 * kRows;                 // floats of a partial result: sums, references, totals
    static constexpr int kCtasPerSm = D * NT <= 128 ? 2 : 1;
    static constexpr int kStages = D == 128 && NT == 1 ? 2 : 4;
    static constexpr int kRing = kStages * kUnitBytes;                   // per warp
    static constexpr int kPerWarp = kRing + kPiece * 4;                  // the ring, and the partial result of its first segment
    static_assert(kPiece * 4 <= kRing, "the partial result of a warp's last segment replaces its ring");
    static constexpr int kSmem = kStreamWarps * kPerWarp;
};

// A partial result in shared memory: of a segment that began in an earlier warp (slot 0), or begins in this one and goes on
// in the next (slot 1).
struct StreamPiece {
    int64_t seg_begin;   // number of the segment's first unit
    int b, head, rt, steps, len, n;
    int used, open;      // open: the segment goes on in the next warp
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t x, uint32_t y) {
    uint32_t z;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
    return z;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t z;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(z) : "f"(hi), "f"(lo));
    return z;
}
__device__ __forceinline__ uint32_t lds32(uint32_t p) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(p));
    return x;
}
__device__ __forceinline__ uint32_t lds8(uint32_t p) {
    uint32_t x;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(p));
    return x;
}
template <int W>
__device__ __forceinline__ void lds_words(uint32_t p, uint32_t (&w)[W]) {
    if constexpr (W == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(p));
    else if constexpr (W == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(p));
    else w[0] = lds32(p);
}

// The weight of a partial result with reference m against the largest reference.
__device__ __forceinline__ float join_weight(float m, float top) { return m == -INFINITY ? 0.f : exp2_fast(m - top); }

// A finished query row: out and lse from its sums, reference (log2) and total.
__device__ __forceinline__ float finish_factor(float l, int v_exp) { return l == 0.f ? 0.f : scale_pow2(1.f / l, v_exp); }
__device__ __forceinline__ float finish_lse(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }

// Where a warp is in the numbering of the units.
struct StreamCursor {
    int64_t base;        // number of the row's first unit
    RowInfo ri;
    int b, steps, tiles, head, rt, step;

    template <int kRows>
    __device__ __forceinline__ void enter(const AttendArgs& a, int row, const RowInfo& info) {
        b = row;
        ri = info;
        steps = row_steps<kStreamUnit>(ri);
        tiles = (ri.n * a.group + kRows - 1) / kRows;
    }
    template <int kRows>
    __device__ __forceinline__ void seek(const AttendArgs& a, int row, const RowInfo& info, int64_t row_begin, int64_t u) {
        enter<kRows>(a, row, info);
        base = row_begin;
        const int64_t rel = u - base;
        const int seg = static_cast<int>(quotient(rel, steps));
        step = static_cast<int>(rel - static_cast<int64_t>(seg) * steps);
        head = seg / tiles;
        rt = seg % tiles;
    }
    __device__ __forceinline__ int64_t seg_begin() const { return base + (static_cast<int64_t>(head) * tiles + rt) * steps; }
    // To the first unit of the next segment; the caller knows that there is one.
    template <int kRows>
    __device__ __forceinline__ void next_segment(const AttendArgs& a) {
        step = 0;
        if (++rt < tiles) return;
        rt = 0;
        if (++head < a.c.n_kv) return;
        head = 0;
        base += static_cast<int64_t>(steps) * tiles * a.c.n_kv;
        do enter<kRows>(a, b + 1, row_info<kStreamUnit>(a, b + 1));
        while (steps == 0 && b + 1 < a.B);
    }
};

// Joins `count` partial results (get(k): sums [kRows][D], references [kRows], totals [kRows]) and hands every four channels
// of a row to put(n, d, sums, reference, total).
// kGlobal: they were written by other CTAs.
template <int D, int kRows, bool kGlobal, typename Get, typename Put>
__device__ __forceinline__ void join_partials(int count, Get get, Put put) {
    auto load = [](const float* p) { return kGlobal ? __ldcg(p) : *p; };
    for (int e = threadIdx.x; e < kRows * (D / 4); e += kStreamThreads) {
        const int n = e / (D / 4), d = e % (D / 4) * 4;
        float top = -INFINITY, l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < count; ++k) top = fmaxf(top, load(get(k) + kRows * D + n));
#pragma unroll 4
        for (int k = 0; k < count; ++k) {
            const float* p = get(k);
            const float w = join_weight(load(p + kRows * D + n), top);
            const float4* at = reinterpret_cast<const float4*>(p + n * D + d);
            const float4 y = kGlobal ? __ldcg(at) : *at;
            l += w * load(p + kRows * D + kRows + n);
            x.x += w * y.x;
            x.y += w * y.y;
            x.z += w * y.z;
            x.w += w * y.w;
        }
        put(n, d, x, top, l);
    }
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kStreamThreads, StreamPlan<D, NT>::kCtasPerSm) attend_stream_kernel(const __grid_constant__ AttendArgs a) {
    using Plan = StreamPlan<D, NT>;
    constexpr int KW = D / 32, VW = D / 64, MT = D / 16;     // words of a token that a thread reads: keys, values; M tiles of O^T
    constexpr int kStages = Plan::kStages, kRows = Plan::kRows;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t bars[kStreamWarps][kStages];
    __shared__ int64_t scan[kStreamWarps], row_base[kStreamWarps];
    __shared__ int row_of[kStreamWarps];
    __shared__ RowInfo row_found[kStreamWarps];
    __shared__ StreamPiece pieces[kStreamWarps][2];
    __shared__ int last_here;
    __shared__ bool gave_up[kStreamWarps];

    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = lane >> 2, j = lane & 3;

    // ---- how many units there are, and where our share begins
    int64_t segments = 0;
    bool count_segments = true;
    RowInfo ri{};                                          // of the row that the thread looked at last
    auto units_of = [&](int b) -> int64_t {
        ri = row_info<kStreamUnit>(a, b);
        const int tiles = (ri.n * a.group + kRows - 1) / kRows;
        if (count_segments) segments += tiles * c.n_kv;
        return static_cast<int64_t>(row_steps<kStreamUnit>(ri)) * tiles * c.n_kv;
    };
    auto block_sum = [&](int64_t x, int64_t* before) -> int64_t {   // the total, and the sum over earlier threads
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
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) {
            if (w == warp) first = all;
            all += scan[w];
        }
        *before = first + y - x;
        return all;
    };
    if (tid < kStreamWarps * kStages) barrier_init(shared_addr(&bars[0][0]) + tid * 8, 1);
    if (tid < kStreamWarps * 2) pieces[tid >> 1][tid & 1].used = 0;
    if (tid < kStreamWarps) gave_up[tid] = false;
    barrier_init_fence();
    int64_t units = 0, mine = 0, before = 0, unused;
    for (int b0 = 0; b0 < a.B; b0 += kStreamThreads) {
        mine = b0 + tid < a.B ? units_of(b0 + tid) : 0;
        units += block_sum(mine, &before);
    }
    count_segments = false;
    segments = block_sum(segments, &unused);
    // About a unit a warp at least.  With up to two units a warp in a segment, a CTA
    // per segment: one more unit costs less than joining results across CTAs (one stream, 333 positions: 16.4 -> 11.6 us).
    const int64_t wanted = segments <= gridDim.x && units <= segments * kStreamWarps * 2 ? segments : (units + kStreamWarps - 1) / kStreamWarps;
    const int ctas = static_cast<int>(min(wanted, static_cast<int64_t>(gridDim.x)));
    const int cta = blockIdx.x;
    const bool busy = cta < ctas;
    const Shares shares(units, max(ctas, 1));              // of the CTAs, and of this one's warps
    const int64_t cta_begin = busy ? shares.begin(cta) : 0, cta_units = busy ? shares.begin(cta + 1) - cta_begin : 0;
    const Shares warp_shares(cta_units, kStreamWarps);
    if (busy) {
        const bool once = a.B <= kStreamThreads;
        int64_t sum = 0;
        for (int b0 = 0; b0 < a.B; b0 += kStreamThreads) {
            if (!once) {
                mine = b0 + tid < a.B ? units_of(b0 + tid) : 0;
                const int64_t all = block_sum(mine, &before);
                before += sum;
                sum += all;
            }
            for (int w = 0; w < kStreamWarps; ++w) {
                const int64_t u = cta_begin + warp_shares.begin(w);
                if (u >= before && u < before + mine) {
                    row_of[w] = b0 + tid;
                    row_base[w] = before;
                    row_found[w] = ri;
                }
            }
        }
    }
    __syncthreads();

    uint8_t* const own = smem + warp * Plan::kPerWarp;
    const uint32_t ring = shared_addr(own), bar0 = shared_addr(&bars[warp][0]);
    const int64_t u0 = cta_begin + warp_shares.begin(warp), u1 = cta_begin + warp_shares.begin(warp + 1);
    int64_t left = u1 - u0, to_load = left;
    const RingWaits waits{&gave_up[warp]};

    // ---- the filling side of the ring: lane l knows where the tiles of step page_step + l are, and issues their copies
    StreamCursor in{}, cur{};
    uint32_t present = 0;              // two bits per stage: which of the unit's tiles are there
    const uint8_t* from0 = nullptr;    // the two tiles of the lane's step
    const uint8_t* from1 = nullptr;
    uint32_t have0 = 0, have1 = 0;     // bit l: lane l has them
    int page_step = -1;
    auto fill = [&](int stage) {
        if (to_load == 0) return;
        if (page_step < 0 || in.step - page_step >= 32) {
            page_step = in.step;
            const int t = in.ri.lo + (page_step + lane) * kStreamUnit, i = t >> c.log_p, slot = t & (c.page_tokens() - 1);
            const int page0 = t < in.ri.hi && t >= 0 ? c.page_at(in.ri.s, i) : -1;
            const int page1 = t + 16 >= in.ri.hi || t < 0 ? -1 : c.log_p > 4 ? page0 : c.page_at(in.ri.s, i + 1);
            from0 = c.tile(max(page0, 0), a.layer, in.head, slot);
            from1 = c.tile(max(page1, 0), a.layer, in.head, c.log_p > 4 ? slot + 16 : 0);
            have0 = __ballot_sync(0xffffffffu, page0 >= 0);
            have1 = __ballot_sync(0xffffffffu, page1 >= 0);
        }
        const int l = in.step - page_step;
        const uint32_t on = ((have0 >> l) & 1) | ((have1 >> l) & 1) << 1;
        present = (present & ~(3u << (2 * stage))) | on << (2 * stage);
        if (lane == l) {
            const uint32_t dst = ring + stage * Plan::kUnitBytes, bar = bar0 + stage * 8;
            barrier_expect(bar, __popc(on) * Plan::kTile);
            if (on == 3 && c.log_p > 4) {
                bulk_load(dst, from0, Plan::kUnitBytes, bar);
            } else {
                if (on & 1) bulk_load(dst, from0, Plan::kTile, bar);
                if (on & 2) bulk_load(dst + Plan::kTile, from1, Plan::kTile, bar);
            }
        }
        --to_load;
        if (++in.step == in.steps && to_load) {
            in.next_segment<kRows>(a);
            page_step = -1;
        }
    };
    if (left > 0) {
        in.seek<kRows>(a, row_of[warp], row_found[warp], row_base[warp], u0);
        cur = in;
        for (int s = 0; s < kStages; ++s) fill(s);
    }
    clear_unused_rows<T, D>(a, cta, gridDim.x);

    // token of M row r (and r + 8) of a tile: neighbours r, r + 1 and every second r fall into different banks below
    const int tok = (r & 1) ? 4 + ((r >> 1) ^ 1) : r >> 1;
    const int tok_a = j, tok_b = 4 + (j ^ 1);                // tokens of K-slots 2j, 2j + 1 (and + 8) of P^T: the same map
    int it = 0;
    while (left > 0) {
        // ---- a piece: the units of one segment that are ours
        const int s0 = cur.step;
        const int count = static_cast<int>(min(left, static_cast<int64_t>(cur.steps - s0)));
        const int rows = cur.ri.n * a.group - cur.rt * kRows;   // query rows of the segment (more than kRows: kRows)
        uint32_t qf[NT][KW][4];
        float factor[NT][2], m[NT][2], limit[NT][2], l[NT][2], o[MT][NT][4];   // limit: m + kRaiseAt
        int pos[NT][2];
        int first_pos, last_pos;
        {
            const int row0 = cur.rt * kRows;
            first_pos = cur.ri.len + row0 / a.group;
            last_pos = cur.ri.len + min(row0 + kRows - 1, cur.ri.n * a.group - 1) / a.group;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = nt * 8 + r, rho = cur.rt * kRows + n;
            float e_scale = 1.f;
            int e_row = 0;
            alignas(16) T x[KW * 8];
            if (n < rows) {
                const T* q = static_cast<const T*>(a.q) + cur.b * a.q_row + rho / a.group * a.q_token +
                             (cur.head * a.group + rho % a.group) * a.q_head + j * (D / 4);
                if (a.q_wide) {
#pragma unroll
                    for (int w = 0; w < KW; ++w) reinterpret_cast<uint4*>(x)[w] = __ldg(reinterpret_cast<const uint4*>(q) + w);
                } else {
#pragma unroll
                    for (int w = 0; w < KW * 8; ++w) x[w] = q[w];
                }
            } else {
#pragma unroll
                for (int w = 0; w < KW * 8; ++w) x[w] = Elem<T>::from_float(0.f);
            }
            if constexpr (sizeof(T) == 2 && !std::is_same<T, __half>::value) {
                float big = 0.f;
#pragma unroll
                for (int w = 0; w < KW * 8; ++w) big = fmaxf(big, fabsf(Elem<T>::to_float(x[w])));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                e_row = big > 0.f ? 14 - (static_cast<int>(__float_as_uint(big) >> 23) - 127) : 0;
                e_row = min(e_row, 126);
                e_scale = a.scale < 0.f ? -pow2(e_row) : pow2(e_row);   // so that the largest score is the largest product
#pragma unroll
                for (int w = 0; w < KW; ++w)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        qf[nt][w][k] = pack_half2(Elem<T>::to_float(x[w * 8 + 2 * k]) * e_scale, Elem<T>::to_float(x[w * 8 + 2 * k + 1]) * e_scale);
            } else {
#pragma unroll
                for (int w = 0; w < KW; ++w)
#pragma unroll
                    for (int k = 0; k < 4; ++k) qf[nt][w][k] = reinterpret_cast<const uint32_t*>(x)[w * 4 + k] ^ (a.scale < 0.f ? 0x80008000u : 0u);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e_col = __shfl_sync(0xffffffffu, e_row, (2 * j + h) * 4);
                factor[nt][h] = score_factor(a.scale, c.k_exp - e_col);
                const int col = nt * 8 + 2 * j + h;
                pos[nt][h] = col < rows ? cur.ri.len + (cur.rt * kRows + col) / a.group : -1;
                m[nt][h] = limit[nt][h] = -INFINITY;
                l[nt][h] = 0.f;
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[mt][nt][k] = 0.f;
        }

        for (int k = 0; k < count; ++k) {
            const int stage = it % kStages;
            const bool late = !waits.unit([&] { return barrier_try(bar0 + stage * 8, (it / kStages) & 1); });
            // (kept for the vote further down instead: two streams of 250,001 positions 142.7 -> 144.0 us, registers spilled)
            if (__any_sync(0xffffffffu, late)) {
                waits.give_up(static_cast<int>(min(left - k - to_load, static_cast<int64_t>(kStages))),
                              [&](int i) { return barrier_try(bar0 + (it + i) % kStages * 8, ((it + i) / kStages) & 1); });
                to_load = 0;
            }
            const int t0 = cur.ri.lo + (s0 + k) * kStreamUnit;
            const uint32_t unit = ring + stage * Plan::kUnitBytes;
            const uint32_t here = (present >> (2 * stage)) & 3;
            const bool full = here == 3 && t0 + kStreamUnit - 1 <= first_pos && (a.window == 0 || t0 > last_pos - a.window);

            // ---- S^T = K Q^T
            float s[2][NT][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t tile = unit + h * Plan::kTile;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) s[h][nt][x] = 0.f;
                uint32_t k0[KW], k1[KW];
                lds_words<KW>(tile + tok * (D / 2) + j * (D / 8), k0);
                lds_words<KW>(tile + (tok + 8) * (D / 2) + j * (D / 8), k1);
                uint32_t c0, c1;   // scales of the two tokens, as pairs
                if constexpr (D == 128) {
                    uint16_t x0, x1;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x0) : "r"(tile + 16 * D + tok * 8 + 2 * j));
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x1) : "r"(tile + 16 * D + (tok + 8) * 8 + 2 * j));
                    c0 = e4m3x2_to_half2(x0);
                    c1 = e4m3x2_to_half2(x1);
                } else {
                    c0 = e4m3x2_to_half2(lds8(tile + 16 * D + tok * 4 + j) * 0x0101u);
                    c1 = e4m3x2_to_half2(lds8(tile + 16 * D + (tok + 8) * 4 + j) * 0x0101u);
                }
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const uint32_t sel = w < KW / 2 || D == 64 ? 0x1010u : 0x3232u;
                    const uint32_t f0 = D == 64 ? c0 : __byte_perm(c0, c0, sel), f1 = D == 64 ? c1 : __byte_perm(c1, c1, sel);
                    uint32_t x0[4], x1[4];
                    e2m1x8_to_half2(k0[w], x0);
                    e2m1x8_to_half2(k1[w], x1);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        x0[x] = mul_half2(x0[x], f0);
                        x1[x] = mul_half2(x1[x], f1);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_16816(s[h][nt], x0[0], x1[0], x0[1], x1[1], qf[nt][w][0], qf[nt][w][1]);
                        mma_16816(s[h][nt], x0[2], x1[2], x0[3], x1[3], qf[nt][w][2], qf[nt][w][3]);
                    }
                }
            }
            // ---- softmax over the tokens of the unit
            if (!full) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int t = t0 + h * 16 + tok + (x >> 1) * 8, p = pos[nt][x & 1];
                            const bool seen = ((here >> h) & 1) && t <= p && (a.window == 0 || t > p - a.window);
                            s[h][nt][x] = seen ? s[h][nt][x] : -INFINITY;
                        }
            }
            // the largest score of the thread's two columns, against what the reference allows
            bool raise = false;
            float top[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    top[nt][x] = fmaxf(fmaxf(s[0][nt][x], s[0][nt][x + 2]), fmaxf(s[1][nt][x], s[1][nt][x + 2])) * factor[nt][x];
                    raise |= top[nt][x] > limit[nt][x];
                }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float y = top[nt][x];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, d));
                        y = fmaxf(y - kAbove, m[nt][x]);
                        const float keep = m[nt][x] == -INFINITY ? 0.f : exp2_fast(m[nt][x] - y);
                        m[nt][x] = y;
                        limit[nt][x] = y + kRaiseAt;
                        l[nt][x] *= keep;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            o[mt][nt][x] *= keep;
                            o[mt][nt][x + 2] *= keep;
                        }
                    }
            }
            uint32_t p[2][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float z0 = m[nt][0] == -INFINITY ? 0.f : -m[nt][0], z1 = m[nt][1] == -INFINITY ? 0.f : -m[nt][1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float e0 = exp2_fast(fmaf(s[h][nt][0], factor[nt][0], z0)), e1 = exp2_fast(fmaf(s[h][nt][1], factor[nt][1], z1));
                    const float e2 = exp2_fast(fmaf(s[h][nt][2], factor[nt][0], z0)), e3 = exp2_fast(fmaf(s[h][nt][3], factor[nt][1], z1));
                    l[nt][0] += e0 + e2;
                    l[nt][1] += e1 + e3;
                    p[h][nt][0] = transpose_8x8(pack_half2(e0, e1));
                    p[h][nt][1] = transpose_8x8(pack_half2(e2, e3));
                }
            }
            // ---- O^T += V^T P^T
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t tile = unit + h * Plan::kTile + 8 * D;
                uint32_t va[VW], vb[VW], vc[VW], vd[VW];
                lds_words<VW>(tile + tok_a * (D / 2) + r * (D / 16), va);
                lds_words<VW>(tile + tok_b * (D / 2) + r * (D / 16), vb);
                lds_words<VW>(tile + (tok_a + 8) * (D / 2) + r * (D / 16), vc);
                lds_words<VW>(tile + (tok_b + 8) * (D / 2) + r * (D / 16), vd);
                const uint32_t sc = tile + 9 * D + (D == 128 ? r : r >> 1);
                uint32_t b0 = lds8(sc + tok_a * (D / 16)), b1 = lds8(sc + tok_b * (D / 16));
                uint32_t b2 = lds8(sc + (tok_a + 8) * (D / 16)), b3 = lds8(sc + (tok_b + 8) * (D / 16));
                if (!full) {
                    // what is masked must not be multiplied with: absent tiles and tokens behind the last get a zero scale; a NaN
                    // that only some rows see is taken out here and given to those rows
                    const int t = t0 + h * 16;
                    const bool on = (here >> h) & 1;
                    uint32_t nans = 0;
                    auto clean = [&](uint32_t& b, int token, int bit) {
                        if (!on || t + token >= cur.ri.hi) b = 0;
                        if ((b & 0x7f) == 0x7f) {
                            b = 0;
                            nans |= 1u << bit;
                        }
                    };
                    clean(b0, tok_a, 0);
                    clean(b1, tok_b, 1);
                    clean(b2, tok_a + 8, 2);
                    clean(b3, tok_b + 8, 3);
                    if (__any_sync(0xffffffffu, nans != 0)) {
                        for (int jj = 0; jj < 4; ++jj) {
                            const uint32_t theirs = __shfl_sync(0xffffffffu, nans, (lane & ~3) | jj);
                            for (int bit = 0; bit < 4; ++bit) {
                                if (!((theirs >> bit) & 1)) continue;
                                const int token = t + ((bit & 1) ? 4 + (jj ^ 1) : jj) + (bit >> 1) * 8;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int x = 0; x < 2; ++x)
                                        if (token <= pos[nt][x] && (a.window == 0 || token > pos[nt][x] - a.window))
#pragma unroll
                                            for (int mt = 0; mt < MT; ++mt) o[mt][nt][x] = o[mt][nt][x + 2] = __int_as_float(0x7fffffff);
                            }
                        }
                        __syncwarp();                        // the products below want the warp together
                    }
                }
                const uint32_t f0 = e4m3x2_to_half2(b0 | b1 << 8), f1 = e4m3x2_to_half2(b2 | b3 << 8);
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    // pairs (token, next token) of the even and the odd channels of the word
                    constexpr uint32_t kLow = 0x0f0f0f0fu;
                    uint32_t ev0[4], od0[4], ev1[4], od1[4];
                    e2m1x8_to_half2((va[w] & kLow) | ((vb[w] << 4) & ~kLow), ev0);
                    e2m1x8_to_half2(((va[w] >> 4) & kLow) | (vb[w] & ~kLow), od0);
                    e2m1x8_to_half2((vc[w] & kLow) | ((vd[w] << 4) & ~kLow), ev1);
                    e2m1x8_to_half2(((vc[w] >> 4) & kLow) | (vd[w] & ~kLow), od1);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        ev0[x] = mul_half2(ev0[x], f0);
                        od0[x] = mul_half2(od0[x], f0);
                        ev1[x] = mul_half2(ev1[x], f1);
                        od1[x] = mul_half2(od1[x], f1);
                    }
                    // M rows r and r + 8 of tile mt: channels 2 mt and 2 mt + 1 of the thread's group r
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int x = 0; x < 4; ++x) mma_16816(o[w * 4 + x][nt], ev0[x], od0[x], ev1[x], od1[x], p[h][nt][0], p[h][nt][1]);
                }
            }
            __syncwarp();
            fill(stage);
            ++it;
        }

        // ---- the piece's result
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][x] += __shfl_xor_sync(0xffffffffu, l[nt][x], d);
        const bool begins = s0 == 0, ends = s0 + count == cur.steps;
        float* const piece = reinterpret_cast<float*>(begins ? own : own + Plan::kRing);
        if (!(begins && ends)) __syncwarp();   // the ring is drained when a last piece takes its place
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int n = nt * 8 + 2 * j + x;
                float y[MT * 2];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    y[2 * mt] = o[mt][nt][x];
                    y[2 * mt + 1] = o[mt][nt][x + 2];
                }
                if (begins && ends) {
                    if (n < rows) {
                        const int rho = cur.rt * kRows + n, i = rho / a.group, h = cur.head * a.group + rho % a.group;
                        const float f = finish_factor(l[nt][x], c.v_exp);
#pragma unroll
                        for (int d = 0; d < MT * 2; ++d) y[d] = l[nt][x] == 0.f ? 0.f : y[d] * f;
                        store_row<T>(static_cast<T*>(a.out) + cur.b * a.o_row + i * a.o_token + h * a.o_head + r * (MT * 2), y, a.o_wide);
                        if (a.lse && r == 0) a.lse[(static_cast<int64_t>(cur.b) * a.Q + i) * a.H + h] = finish_lse(m[nt][x], l[nt][x]);
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < MT * 2; d += 4)
                        *reinterpret_cast<float4*>(piece + n * D + r * (MT * 2) + d) = make_float4(y[d], y[d + 1], y[d + 2], y[d + 3]);
                    if (r == 0) {
                        piece[kRows * D + n] = m[nt][x];
                        piece[kRows * D + kRows + n] = l[nt][x];
                    }
                }
            }
        if (!(begins && ends) && lane == 0) {
            StreamPiece& d = pieces[warp][begins];
            d.seg_begin = cur.seg_begin();
            d.b = cur.b;
            d.head = cur.head;
            d.rt = cur.rt;
            d.steps = cur.steps;
            d.len = cur.ri.len;
            d.n = cur.ri.n;
            d.open = !ends;
            d.used = 1;
        }
        left -= count;
        cur.step += count;
        if (left) cur.next_segment<kRows>(a);
    }
    if (gave_up[warp] && c.meta && lane == 0) atomicOr(&c.meta[1], kStatusGaveUp);
    if (!busy) return;
    __syncthreads();

    // ---- join the pieces of segments that several warps hold; those that several CTAs hold go on through global memory
    auto write_row = [&](const StreamPiece& d, int n, int ch, float4 x, float top, float l) {
        const int rho = d.rt * kRows + n;
        if (rho >= d.n * a.group) return;
        const int i = rho / a.group, h = d.head * a.group + rho % a.group;
        const float f = finish_factor(l, c.v_exp);
        T* out = static_cast<T*>(a.out) + d.b * a.o_row + i * a.o_token + h * a.o_head + ch;
        const float y[4] = {l == 0.f ? 0.f : x.x * f, l == 0.f ? 0.f : x.y * f, l == 0.f ? 0.f : x.z * f, l == 0.f ? 0.f : x.w * f};
        alignas(8) T e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = Elem<T>::from_float(y[k]);
        if (a.o_wide) {
            *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(e);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = e[k];
        }
        if (a.lse && ch == 0) a.lse[(static_cast<int64_t>(d.b) * a.Q + i) * a.H + h] = finish_lse(top, l);
    };
    int crossing = -1, crossing2 = -1;   // first pieces of the segments that cross CTAs (at most two): warp * 2 + slot
    for (int w0 = 0; w0 < kStreamWarps; ++w0)
        for (int slot = w0 == 0 ? 0 : 1; slot < 2; ++slot) {
            if (!pieces[w0][slot].used) continue;
            const StreamPiece& d = pieces[w0][slot];
            int w1 = w0;
            bool open = d.open;
            while (open && w1 + 1 < kStreamWarps && pieces[w1 + 1][0].used) open = pieces[++w1][0].open;
            auto get = [&](int k) {
                return reinterpret_cast<const float*>(smem + (w0 + k) * Plan::kPerWarp + (k == 0 && slot == 1 ? 0 : Plan::kRing));
            };
            if (slot == 1 && !open) {
                join_partials<D, kRows, false>(w1 - w0 + 1, get, [&](int n, int ch, float4 x, float top, float l) { write_row(d, n, ch, x, top, l); });
            } else {
                (crossing < 0 ? crossing : crossing2) = w0 * 2 + slot;
                float* part = a.partials + (2ll * cta + slot) * Plan::kPiece;
                join_partials<D, kRows, false>(w1 - w0 + 1, get, [&](int n, int ch, float4 x, float top, float l) {
                    *reinterpret_cast<float4*>(part + n * D + ch) = x;
                    if (ch == 0) {
                        part[kRows * D + n] = top;
                        part[kRows * D + kRows + n] = l;
                    }
                });
            }
        }
    for (int k = 0; k < 2; ++k) {
        const int at = k ? crossing2 : crossing;
        if (at < 0) break;
        const StreamPiece& d = pieces[at >> 1][at & 1];
        const int c0 = shares.owner(d.seg_begin), c1 = shares.owner(d.seg_begin + d.steps - 1);
        __threadfence();
        __syncthreads();
        if (tid == 0) last_here = atomicAdd(&a.counters[c0], 1) == c1 - c0;
        __syncthreads();
        if (!last_here) continue;
        __threadfence();
        if (tid == 0) a.counters[c0] = 0;
        join_partials<D, kRows, true>(c1 - c0 + 1, [&](int i) { return const_cast<const float*>(a.partials + (2ll * (c0 + i) + (i == 0)) * Plan::kPiece); },
                                [&](int n, int ch, float4 x, float top, float l) { write_row(d, n, ch, x, top, l); });
    }
}

}  // namespace samb200
