// Attention over the 4-bit cache: arguments, work division, and the joining of partial results.
//
// The work is cut along the context: a segment is one row of the batch, one key/value head and one tile of its query rows;
// a unit is kUnit tokens of a segment.  All units of all segments are numbered, and the CTAs take equal shares of the
// numbers, so that a batch of one long and many short contexts keeps every SM busy.  A segment that several CTAs hold is
// joined by the last of them to finish, always in the order of the tokens: the result does not depend on who that is.
#pragma once

#include "cache_async.cuh"
#include "cache_format.cuh"

namespace samb200 {

constexpr int kStatusGaveUp = 8;

struct AttendArgs {
    CacheView c;
    const void* q;
    void* out;
    float* lse;
    const int32_t* streams;
    const int32_t* n_new;
    int64_t q_row, q_token, q_head, o_row, o_token, o_head;   // strides in elements
    int32_t layer, B, Q, H, window;
    int32_t group;            // query heads per key/value head
    float scale;
    bool q_wide, o_wide;      // every row starts on a 16-byte boundary
    int32_t* counters;        // [grid], zero between calls
    float* partials;          // [2 * grid] partial results
};

// One row of the batch as every kernel sees it.
struct RowInfo {
    int s;          // stream, -1 = unknown
    int len, n;     // committed tokens; query rows that are computed
    int lo, hi;     // tokens [lo, hi) may be seen by one of the query rows; lo is a multiple of the unit
};
template <int kUnit>
__device__ __forceinline__ RowInfo row_info(const AttendArgs& a, int b) {
    RowInfo r;
    r.s = a.c.stream_of(a.streams, b);
    r.n = r.s < 0 ? 0 : max(a.n_new ? min(a.n_new[b], a.Q) : a.Q, 0);
    r.len = r.s < 0 ? 0 : a.c.length_of(r.s);
    const int cap = a.c.capacity();
    r.hi = static_cast<int>(min(static_cast<int64_t>(r.len) + r.n, static_cast<int64_t>(cap)));
    r.lo = a.window > 0 ? max(r.len - a.window + 1, 0) : 0;
    r.lo = min(r.lo, cap - 1) & ~(kUnit - 1);
    return r;
}
// Units of a row: at least one per segment, so that somebody writes its result.
template <int kUnit>
__device__ __forceinline__ int row_steps(const RowInfo& r) { return r.n > 0 ? max((r.hi - r.lo + kUnit - 1) / kUnit, 1) : 0; }

// 64-bit quotients of numbers that nearly always fit 32 bits (a 64-bit division is a subroutine of over a hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((a | b) >> 31) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Shares of T units among W workers: the first T mod W have one more.
struct Shares {
    int64_t base, rem;
    __device__ __forceinline__ Shares(int64_t T, int W) : base(quotient(T, W)), rem(T - base * W) {}
    __device__ __forceinline__ int64_t begin(int w) const { return w * base + min(static_cast<int64_t>(w), rem); }
    __device__ __forceinline__ int owner(int64_t u) const {
        const int64_t first = rem * (base + 1);
        return static_cast<int>(u < first ? quotient(u, base + 1) : rem + quotient(u - first, base));
    }
};

// 2^e for any e that matters, in two exact steps.
__device__ __forceinline__ float scale_pow2(float x, int e) {
    const int h = min(max(e, -250), 250) / 2;
    return x * pow2(h) * pow2(min(max(e, -250), 250) - h);
}

// From a product of queries and keys (scaled by 2^-e, with the sign of the scale in it) to a score in powers of two.  Never zero,
// so that a masked score of minus infinity stays one; the least value leaves nothing of any product.
__device__ __forceinline__ float score_factor(float scale, int e) {
    return fmaxf(scale_pow2(fabsf(scale) * 1.4426950408889634f, e), 1.17549435e-38f);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Sixteen-byte store of eight results, or eight single ones.
template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const float (&x)[N], bool wide) {
    alignas(16) T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = Elem<T>::from_float(x[i]);
    if (wide) {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = e[i];
    }
}

// Query rows that are not computed (i >= n): out = 0, lse = -inf.  CTA `cta` of `ctas` takes its share of the batch.
template <typename T, int D>
__device__ __forceinline__ void clear_unused_rows(const AttendArgs& a, int cta, int ctas) {
    for (int b = cta; b < a.B; b += ctas) {
        const int s = a.c.stream_of(a.streams, b);
        const int n = s < 0 ? 0 : max(a.n_new ? min(a.n_new[b], a.Q) : a.Q, 0);
        const int64_t rows = static_cast<int64_t>(a.Q - n) * a.H;
        for (int64_t e = threadIdx.x; e < rows * (D / 8); e += blockDim.x) {
            const int64_t r = e / (D / 8);
            const int i = n + static_cast<int>(r / a.H), h = static_cast<int>(r % a.H);
            const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            store_row<T, 8>(static_cast<T*>(a.out) + b * a.o_row + i * a.o_token + h * a.o_head + e % (D / 8) * 8, zero, a.o_wide);
            if (a.lse && e % (D / 8) == 0) a.lse[(static_cast<int64_t>(b) * a.Q + i) * a.H + h] = -INFINITY;
        }
    }
}

}  // namespace samb200
