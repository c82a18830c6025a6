// Greedy choice of logits rows under penalties for repeated tokens, biases and masks; and the counts behind the penalties.
//
// Every logit is read once and nothing is written back: the values that a row is shaped to exist in registers only.  Few tokens
// of a row are anything but their logit ("special": said before, biased, or a draft before the row); which ones, and which are
// allowed at all, comes as bits, 1/16 of the logits' bytes each.
#pragma once

#include "sam_kernels.cuh"

namespace samb200 {

struct ShapeArgs {
    const __nv_bfloat16* logits;
    long long stride;
    const int32_t* drafts;            // [B, K]
    const int32_t* streams;           // [B] or null
    const int32_t* counts;            // [n_streams, V]: times said, sign bit: told
    const uint32_t* seen;             // [n_streams, words]: counts != 0
    const float* repetition;          // [B], or null
    const float* presence;
    const float* frequency;
    const int32_t* bias_tokens;       // [B, max_bias]
    const float* bias_values;
    const int32_t* n_bias;            // [B], or null: max_bias
    const uint32_t* masks;            // [n_masks, words]
    const int32_t* mask_of;           // [B, K + 1]
    unsigned long long* keys;         // [B * (K + 1)]
    int32_t B, K, V, words, n_streams, max_bias, n_masks, tiles_per_row;
};

constexpr int kShapeCtasPerSm = 4;
constexpr int kShapeThreads = 256, kShapeVecs = 4, kShapeTile = kShapeThreads * kShapeVecs * 8;   // logits of a tile
constexpr int kShapeWords = kShapeTile / 32 + 2;

// Larger for larger numbers, as an unsigned number; the two zeros alike.
__device__ __forceinline__ unsigned ordered_key32(float x) {
    const unsigned b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr unsigned kKeyNothing = 0x007fffffu;                      // of minus infinity
constexpr unsigned long long kKeyNoneAllowed = 1ull << 32;         // decodes to index -1

// What is shaped to what, in the order and the roundings that the interface promises.
__device__ __forceinline__ float shaped_value(float x, bool told, int said, float rep, float pres, float freq, float bias) {
    if (told || said > 0) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
    if (said > 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, static_cast<float>(said))), pres);
    return __fadd_rn(x, bias);
}

// Persistent CTAs take equal shares of the tiles of all rows.
__global__ void __launch_bounds__(kShapeThreads, kShapeCtasPerSm) argmax_shaped_kernel(const __grid_constant__ ShapeArgs a) {
    __shared__ uint32_t allowed[kShapeWords], special[kShapeWords], biased[kShapeWords];
    const int tid = threadIdx.x, lane = tid & 31, K1 = a.K + 1;
    const long long total = static_cast<long long>(a.B) * K1 * a.tiles_per_row;
    const long long t0 = total * blockIdx.x / gridDim.x, t1 = total * (blockIdx.x + 1) / gridDim.x;
    const bool penalties = a.repetition || a.presence || a.frequency;
    long long cur = -1;
    int b = 0, j = 0, n_bias = 0, fallback = -1;
    RowView rv{};
    float best = -INFINITY, rep = 1.f, pres = 0.f, freq = 0.f;
    unsigned best_at = 0;
    bool raising = false;
    const uint32_t* mask = nullptr;
    const uint32_t* seen = nullptr;
    const int32_t* counts = nullptr;
    auto flush = [&]() {
        if (cur < 0) return;
        unsigned long long k = kKeyNoneAllowed;
        if (fallback >= 0) k = static_cast<unsigned long long>(kKeyNothing) << 32 | (0xffffffffu - static_cast<unsigned>(fallback));
        if (best > -INFINITY) k = static_cast<unsigned long long>(ordered_key32(best)) << 32 | (0xffffffffu - best_at);
        k = warp_max_u64(k);
        if (lane == 0) atomicMax(a.keys + cur, k);
    };
    for (long long t = t0; t < t1; ++t) {
        const long long row = t / a.tiles_per_row;
        const int tile = static_cast<int>(t - row * a.tiles_per_row);
        if (row != cur) {
            flush();
            cur = row;
            b = static_cast<int>(row / K1);
            j = static_cast<int>(row - static_cast<long long>(b) * K1);
            rv = row_view(a.logits, a.stride, row, a.V);
            best = -INFINITY;
            fallback = -1;
            const int s = a.streams ? a.streams[b] : b;
            const bool known = static_cast<unsigned>(s) < static_cast<unsigned>(a.n_streams);
            counts = penalties && a.counts && known ? a.counts + static_cast<long long>(s) * a.V : nullptr;
            seen = counts ? a.seen + static_cast<long long>(s) * a.words : nullptr;
            rep = a.repetition ? a.repetition[b] : 1.f;
            pres = a.presence ? a.presence[b] : 0.f;
            freq = a.frequency ? a.frequency[b] : 0.f;
            raising = !(rep >= 1.f && pres >= 0.f && freq >= 0.f);
            n_bias = a.max_bias ? min(max(a.n_bias ? a.n_bias[b] : a.max_bias, 0), a.max_bias) : 0;
            const int m = a.masks ? a.mask_of[row] : -1;
            mask = static_cast<unsigned>(m) < static_cast<unsigned>(a.n_masks) ? a.masks + static_cast<long long>(m) * a.words : nullptr;
        }
        // ---- the tile's bits: words w0 .. of the vocabulary
        const int e0 = tile * kShapeTile - rv.off, w0 = e0 >> 5;   // first token; below zero in front of an unaligned row
        uint4 v[kShapeVecs];
        const int q0 = tile * (kShapeTile / 8) + tid;
#pragma unroll
        for (int i = 0; i < kShapeVecs; ++i) {
            const int q = q0 + i * kShapeThreads;
            v[i] = make_uint4(kNaN2, kNaN2, kNaN2, kNaN2);
            if (q < rv.nvec) v[i] = ld_stream(rv.vec + q);
        }
        __syncthreads();
        for (int w = tid; w < kShapeWords; w += kShapeThreads) {
            const int at = w0 + w;
            const bool in = at >= 0 && at < a.words;
            uint32_t ok = in ? (mask ? mask[at] : 0xffffffffu) : 0u;
            if (at == a.words - 1 && (a.V & 31)) ok &= (1u << (a.V & 31)) - 1;
            allowed[w] = ok;
            special[w] = in && seen ? seen[at] : 0u;
            biased[w] = 0;
        }
        __syncthreads();
        auto mark = [&](uint32_t* bits, int token) {
            if (static_cast<unsigned>(token) >= static_cast<unsigned>(a.V)) return;
            const int w = (token >> 5) - w0;
            if (static_cast<unsigned>(w) < static_cast<unsigned>(kShapeWords)) atomicOr(&bits[w], 1u << (token & 31));
        };
        for (int i = tid; i < n_bias; i += kShapeThreads) {
            const int token = a.bias_tokens[static_cast<long long>(b) * a.max_bias + i];
            mark(special, token);
            mark(biased, token);
        }
        if (penalties && tid < j) mark(special, a.drafts[static_cast<long long>(b) * a.K + tid]);
        __syncthreads();
        // ---- tokens that are their logit
        uint32_t odd[kShapeVecs];                          // special and allowed tokens of the vectors
        auto bits_at = [&](const uint32_t* bits, int e) { return __funnelshift_r(bits[(e >> 5) - w0], bits[(e >> 5) - w0 + 1], e & 31) & 0xffu; };
#pragma unroll
        for (int i = 0; i < kShapeVecs; ++i) {
            const int q = q0 + i * kShapeThreads, e = q * 8 - rv.off;
            odd[i] = 0;
            if (q >= rv.nvec) continue;
            const uint32_t ok = bits_at(allowed, e), sp = bits_at(special, e) & ok, plain = ok & ~sp;
            odd[i] = sp;
            if (ok && fallback < 0) fallback = e + __ffs(ok) - 1;
            uint4 x = v[i];
            unsigned w[4] = {x.x, x.y, x.z, x.w};
            if (plain != 0xff) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] |= ((plain >> (2 * k)) & 1 ? 0u : 0xffffu) | ((plain >> (2 * k)) & 2 ? 0u : 0xffff0000u);   // NaN
            }
            x = make_uint4(w[0], w[1], w[2], w[3]);
            const float m = vec_max(x);
            if (m > best) {
                best = m;
                best_at = e + first_equal(x, m);
            }
        }
        // ---- special tokens: no penalty makes them more than their logit (or all are looked at)
        float bound = best;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) bound = fmaxf(bound, __shfl_xor_sync(kFull, bound, d));
#pragma unroll
        for (int i = 0; i < kShapeVecs; ++i) {
            const int e = (q0 + i * kShapeThreads) * 8 - rv.off;
            const unsigned w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            const uint32_t bi = odd[i] ? bits_at(biased, e) : 0u;
            for (uint32_t left = odd[i]; left; left &= left - 1) {
                const int k = __ffs(left) - 1, token = e + k;
                const unsigned pair = k < 4 ? (k < 2 ? w[0] : w[1]) : (k < 6 ? w[2] : w[3]);
                const float x = (k & 1) ? bf16hi(pair) : bf16lo(pair);
                const bool has_bias = (bi >> k) & 1;
                if (!raising && !has_bias && !(x >= bound)) continue;
                const int c = counts ? counts[token] : 0;
                int said = c & 0x7fffffff;
                if (penalties)
                    for (int d = 0; d < j; ++d) said += a.drafts[static_cast<long long>(b) * a.K + d] == token;
                float bias = 0.f;
                if (has_bias)
                    for (int d = 0; d < n_bias; ++d)
                        if (a.bias_tokens[static_cast<long long>(b) * a.max_bias + d] == token) bias = __fadd_rn(bias, a.bias_values[static_cast<long long>(b) * a.max_bias + d]);
                const float y = shaped_value(x, c < 0, said, rep, pres, freq, bias);
                if (y > best || (y == best && y > -INFINITY && static_cast<unsigned>(token) < best_at)) {
                    best = y;
                    best_at = token;
                }
            }
        }
    }
    flush();
}

// ---- what was told and said
__global__ void __launch_bounds__(256) history_add_kernel(int32_t* counts, uint32_t* seen, int n_streams, int V, int words, int B, const int32_t* streams,
                                                          const int32_t* tokens, int ld, const int32_t* n, bool told) {
    const int b = blockIdx.y, s = streams ? streams[b] : b;
    if (static_cast<unsigned>(s) >= static_cast<unsigned>(n_streams)) return;
    const int count = n ? min(n[b], ld) : ld;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < count; i += gridDim.x * 256) {
        const int t = tokens[static_cast<long long>(b) * ld + i];
        if (static_cast<unsigned>(t) >= static_cast<unsigned>(V)) continue;
        int32_t* at = counts + static_cast<long long>(s) * V + t;
        if (told) atomicOr(at, static_cast<int>(0x80000000u));
        else atomicAdd(at, 1);
        atomicOr(seen + static_cast<long long>(s) * words + (t >> 5), 1u << (t & 31));
    }
}

// Rows dst[i] become rows src[i] (src null: empty).
__global__ void __launch_bounds__(256) history_copy_kernel(int32_t* counts, uint32_t* seen, int n_streams, int V, int words, const int32_t* src, const int32_t* dst) {
    const int z = dst[blockIdx.y], s = src ? src[blockIdx.y] : 0;
    if (static_cast<unsigned>(z) >= static_cast<unsigned>(n_streams) || static_cast<unsigned>(s) >= static_cast<unsigned>(n_streams) || (src && s == z)) return;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < V; i += gridDim.x * 256)
        counts[static_cast<long long>(z) * V + i] = src ? counts[static_cast<long long>(s) * V + i] : 0;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < words; i += gridDim.x * 256)
        seen[static_cast<long long>(z) * words + i] = src ? seen[static_cast<long long>(s) * words + i] : 0u;
}

}  // namespace samb200
