// Greedy choice of logits rows under penalties for repeated tokens, biases and masks; and the counts behind the penalties.
//
// Every logit is read once and nothing is written back: the values that a row is shaped to exist in registers only.  Few tokens
// of a row are anything but their logit ("special": said before, or a draft; and biased ones); which ones, and which are
// allowed at all, comes as bits, 1/16 of the logits' bytes each.  The others take part in a maximum of pairs of bf16; a special token is worked
// out only where its logit reaches the best so far, which no usual penalty can raise.
//
// 192 streams of 17 rows of 151,936 logits with 6,000 tokens said and up to 64 biases each (1.0 GB): 180 to 184 us, 5.4 TB/s (without penalties
// and biases 160, the plain argmax 146).  What it took: every token of a row looked at with its bits, loads into registers: 742 us; bits
// once for all rows of a tile: 430; copies to shared memory some rows ahead by the threads that read them: 265; special tokens
// in the order of their tiles and by one lane: 193; a lane for each token: 184.  All of it fits 80 registers a thread, which
// three CTAs an SM need; forms that spilled took 215 to 330.  Warps that run on their own over slices of 1,024 tokens: 206.
//
// Rows whose stride is no multiple of eight begin at different places of a vector, and every row is then a tile of its own: bits, marks and
// six block barriers for each.  192 streams of 17 rows of 50,257 packed logits: 110 us (64 with rows 50,264 apart), with penalties
// 179 (76), with 64 biases too 230 (86).
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

constexpr int kShapeThreads = 256, kShapeVecs = 4, kShapeTile = kShapeThreads * kShapeVecs * 8;   // tokens of a tile: 1,024 a warp

// Larger for larger numbers, as an unsigned number; the two zeros alike.
__device__ __forceinline__ unsigned ordered_key32(float x) {
    const unsigned b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr unsigned kKeyNothing = 0x007fffffu;                      // of minus infinity
constexpr unsigned long long kKeyNoneAllowed = 1ull << 32;         // decodes to index -1
__device__ __forceinline__ unsigned long long shaped_candidate(unsigned key, int token) {
    return static_cast<unsigned long long>(key) << 32 | (0xffffffffu - static_cast<unsigned>(token));
}

// What is shaped to what, in the order and the roundings that the interface promises.
__device__ __forceinline__ float shaped_value(float x, bool told, int said, float rep, float pres, float freq, float bias) {
    if (told || said > 0) x = x > 0.f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
    if (said > 0) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, static_cast<float>(said))), pres);
    return __fadd_rn(x, bias);
}

// 32 bits from bit `at` of a row of words; what lies outside reads as zero.
__device__ __forceinline__ uint32_t bits_from(const uint32_t* row, int words, int at) {
    const int w = at >> 5;
    const uint32_t lo = w >= 0 && w < words ? __ldg(row + w) : 0u;
    if (!(at & 31)) return lo;
    const uint32_t hi = w + 1 >= 0 && w + 1 < words ? __ldg(row + w + 1) : 0u;
    return __funnelshift_r(lo, hi, at & 31);
}

// Eight bits -> the pairs of a vector, 0xffff (a NaN) where a bit is clear.
__device__ __forceinline__ void nan_where_clear(uint32_t bits, uint32_t (&w)[4]) {
    const uint32_t lo = (~bits & 15u) * 0x10204080u, hi = (~bits >> 4 & 15u) * 0x10204080u;   // bit k to the sign of byte k
    auto signs = [](uint32_t x, uint32_t which) {          // each byte the sign of one of x's bytes, eight times
        uint32_t y;
        asm("prmt.b32 %0, %1, 0, %2;" : "=r"(y) : "r"(x), "r"(which));
        return y;
    };
    w[0] = signs(lo, 0x9988);
    w[1] = signs(lo, 0xbbaa);
    w[2] = signs(hi, 0x9988);
    w[3] = signs(hi, 0xbbaa);
}

constexpr int kShapeCtasPerSm = 3, kShapeStages = 4, kShapeBias = SAM_MAX_BIAS, kShapeWaiting = 64, kShapeFew = 6;
static_assert(kShapeVecs == 4 && kShapeTile / 32 == kShapeThreads, "a thread has 32 tokens of a tile");
constexpr int shape_smem(bool masks) { return kShapeStages * kShapeThreads * (kShapeVecs * 16 + (masks ? 4 : 0)); }   // the ring: vectors, and words of allowed tokens

// One row of one tile.  The last tile of a stream comes first: what is said often are tokens of low numbers, and by then the best
// of the others is known.
struct ShapeItem {
    int b, tile, j;
    __device__ __forceinline__ bool next(const ShapeArgs& a) {   // true: in another tile
        if (++j <= a.K) return false;
        j = 0;
        if (--tile >= 0) return true;
        tile = a.tiles_per_row - 1;
        ++b;
        return true;
    }
};

// The lane's vectors of a row, as far as their bits are set.
template <int kFirst>
__device__ __forceinline__ void copy_vectors(uint32_t to, const uint4* from, uint32_t bits) {
    if constexpr (kFirst < kShapeVecs) {
        if (bits & (1u << kFirst))
            asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16;"
                         ::"r"(to), "l"(from), "n"(kFirst * kShapeThreads * 16), "n"(kFirst * 512) : "memory");
        copy_vectors<kFirst + 1>(to, from, bits);
    }
}

// A tile is 8,192 tokens of a stream, and all its rows are asked about them one after the other: which tokens are special is worked
// out once for the rows of a tile, and lies in registers as the pairs of NaN that take them out of a row's maximum.  CTAs take equal
// shares of the rows of all tiles, in the order streams, tiles, rows.  Every thread copies the vectors that it will look at
// into shared memory itself, kShapeStages - 1 rows ahead and over the ends of tiles: nobody waits for anybody but where tiles
// change, and copies are under way even then.  Vectors of which the mask leaves nothing are not copied; the words of a mask come
// a row before the copies that depend on them.
template <bool kMasks>
__global__ void __launch_bounds__(kShapeThreads, kShapeCtasPerSm) argmax_shaped_kernel(const __grid_constant__ ShapeArgs a) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ unsigned long long best[SAM_K_MAX + 1];     // of the current stream's rows, so far
    __shared__ int drafts[SAM_K_MAX];
    __shared__ uint32_t marked[kShapeTile / 32];           // biased tokens of the tile
    __shared__ int bias_token[kShapeBias];                 // the stream's: -1 for what is no token, or was mentioned before
    __shared__ float bias_sum[kShapeBias];
    __shared__ uint16_t listed[kShapeThreads];             // biases of the tile
    __shared__ int n_listed, n_waiting;
    __shared__ int2 waiting[kShapeWaiting];                // token; its logit, and below it the row
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K1 = a.K + 1;
    const long long total = static_cast<long long>(a.B) * K1 * a.tiles_per_row;
    const long long i0 = total * blockIdx.x / gridDim.x, i1 = total * (blockIdx.x + 1) / gridDim.x;
    const bool penalties = a.repetition || a.presence || a.frequency;
    uint4* const slots = reinterpret_cast<uint4*>(ring) + tid;                      // stage s, vector i: [(s * kShapeVecs + i) * kShapeThreads]
    uint32_t* const words = reinterpret_cast<uint32_t*>(ring + kShapeStages * kShapeThreads * kShapeVecs * 16) + tid;
    auto byte_of = [&](uint32_t word, int i) { return (__shfl_sync(kFull, word, i * 8 + (lane >> 2)) >> (8 * (lane & 3))) & 0xffu; };
    auto row_of = [&](const ShapeItem& x) { return a.logits + (static_cast<long long>(x.b) * K1 + x.j) * a.stride; };
    auto offset_of = [&](const __nv_bfloat16* row) { return static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) >> 1); };
    // first of the 32 tokens whose bits the lane has, and which of them there are
    auto own_of = [&](int tile, int off) { return tile * kShapeTile - off + warp * 1024 + lane * 32; };
    auto valid_of = [&](int own) {
        uint32_t v = 0xffffffffu;
        if (own < 0) v &= own > -32 ? 0xffffffffu << -own : 0u;
        if (own + 32 > a.V) v &= own < a.V ? 0xffffffffu >> (own + 32 - a.V) : 0u;
        return v;
    };

    // ---- the filling side: the mask of an item, then its allowed tokens, then its copies
    ShapeItem x;
    {
        const long long unit = i0 / K1;
        x.j = static_cast<int>(i0 - unit * K1);
        x.b = static_cast<int>(unit / a.tiles_per_row);
        x.tile = a.tiles_per_row - 1 - static_cast<int>(unit - static_cast<long long>(x.b) * a.tiles_per_row);
    }
    const bool ragged = a.stride & 7;                      // rows begin at different places of a vector
    const int n_items = static_cast<int>(min(i1 - i0, 0x7fffffffll));
    ShapeItem mask_item = x, copy_item = x;
    int to_mask = n_items, to_load = n_items, mask_now = -1, mask_next = -1, stage_in = 0, own_in = 0;
    uint32_t valid_in = 0, mask_lo = 0, mask_hi = 0;       // of the item that is copied next
    const uint4* src = nullptr;
    auto fetch_mask = [&]() {
        mask_now = mask_next;
        if (kMasks && to_mask > 0) {
            mask_next = __ldg(a.mask_of + static_cast<long long>(mask_item.b) * K1 + mask_item.j);
            --to_mask;
            mask_item.next(a);
        }
    };
    auto seek = [&]() {                                    // to the item's tile
        const __nv_bfloat16* row = row_of(copy_item);
        src = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(15)) + copy_item.tile * (kShapeTile / 8) + warp * 128 + lane;
        own_in = own_of(copy_item.tile, offset_of(row));
        valid_in = valid_of(own_in);
    };
    // which vectors of the lane have an allowed token
    auto vectors_of = [&](uint32_t word) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < kShapeVecs; ++i) n |= (byte_of(word, i) != 0) << i;
        return n;
    };
    uint32_t vectors_in = 0;
    auto fetch_word = [&](bool moved) {
        if (moved) {
            seek();
            if (!kMasks) vectors_in = vectors_of(valid_in);
        }
        if (kMasks) {                                      // loaded here, looked at when the row is copied
            mask_lo = mask_hi = 0xffffffffu;
            if (static_cast<unsigned>(mask_now) < static_cast<unsigned>(a.n_masks)) {
                const uint32_t* m = a.masks + static_cast<long long>(mask_now) * a.words;
                const int w = own_in >> 5;
                mask_lo = mask_hi = 0;
                if (w >= 0 && w < a.words) mask_lo = __ldg(m + w);
                if ((own_in & 31) && w + 1 >= 0 && w + 1 < a.words) mask_hi = __ldg(m + w + 1);
            }
        }
    };
    auto copy = [&]() {
        if (to_load > 0) {
            if (kMasks) {
                const uint32_t word = valid_in & __funnelshift_r(mask_lo, mask_hi, own_in & 31);
                vectors_in = vectors_of(word);
                words[stage_in * kShapeThreads] = word;
            }
            const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(slots)) + stage_in * (kShapeVecs * kShapeThreads * 16);
            copy_vectors<0>(to, src, vectors_in);
            if (--to_load > 0) {
                const bool moved = copy_item.next(a) || ragged;
                if (!moved) src += a.stride >> 3;
                fetch_mask();
                fetch_word(moved);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage_in == kShapeStages) stage_in = 0;
    };
    fetch_mask();
    fetch_mask();
    fetch_word(true);
    for (int s = 0; s < kShapeStages - 1; ++s) copy();

    // ---- the stream's and the tile's facts
    int cur_b = -1, n_bias = 0, first = 0;
    uint32_t valid = 0, plain = 0;                         // which of the lane's 32 tokens there are, and which are their logit
    float rep = 1.f, pres = 0.f, freq = 0.f;
    bool raising = false, any_odd = false;
    const uint32_t* seen = nullptr;
    const int32_t* counts = nullptr;
    constexpr int kNowhere = -0x7fffffff;
    int seen_at = kNowhere;
    uint32_t seen_next = 0;
    uint32_t out[kShapeVecs][4], odd = 0;                  // what takes tokens out of the maximum; special tokens of the vectors
    auto flush = [&]() {
        asm volatile("griddepcontrol.wait;" ::: "memory");   // the keys are cleared
        __syncthreads();
        if (cur_b >= 0 && tid < K1 && best[tid]) atomicMax(a.keys + static_cast<long long>(cur_b) * K1 + tid, best[tid]);
        __syncthreads();
    };
    // what token t, of raw value x, comes to in row j
    auto shaped = [&](int t, float x, int j, float bias) {
        const int c = counts ? __ldg(counts + t) : 0;
        int said = c & 0x7fffffff;
        if (penalties)
            for (int d = 0; d < j; ++d) said += drafts[d] == t;
        return shaped_value(x, c < 0, said, rep, pres, freq, bias);
    };
    auto look_at = [&](int t, float x, int j, float bias) {
        const float y = shaped(t, x, j, bias);
        if (y > -INFINITY) atomicMax(&best[j], shaped_candidate(ordered_key32(y), t));
    };
    // special tokens that a tile's rows want to be looked at, all together
    auto settle = [&]() {
        __syncthreads();
        if (tid < min(n_waiting, kShapeWaiting)) look_at(waiting[tid].x, __uint_as_float(waiting[tid].y & 0xffff0000u), waiting[tid].y & 0xffff, 0.f);
        __syncthreads();
        if (tid == 0) n_waiting = 0;
    };
    auto enter_stream = [&](int b) {
        if (cur_b >= 0) flush();                           // the first stream's facts need no wait for the keys
        cur_b = b;
        if (tid < K1) best[tid] = 0;
        if (tid < a.K) drafts[tid] = a.drafts[static_cast<long long>(b) * a.K + tid];
        const int s = a.streams ? a.streams[b] : b;
        const bool known = static_cast<unsigned>(s) < static_cast<unsigned>(a.n_streams);
        counts = penalties && a.counts && known ? a.counts + static_cast<long long>(s) * a.V : nullptr;
        seen = counts ? a.seen + static_cast<long long>(s) * a.words : nullptr;
        seen_at = kNowhere;
        rep = a.repetition ? a.repetition[b] : 1.f;
        pres = a.presence ? a.presence[b] : 0.f;
        freq = a.frequency ? a.frequency[b] : 0.f;
        raising = !(rep >= 1.f && pres >= 0.f && freq >= 0.f);   // a penalty may make a token more than its logit
        n_bias = a.max_bias ? min(max(a.n_bias ? a.n_bias[b] : a.max_bias, 0), a.max_bias) : 0;
        if (n_bias == 0) return;
        for (int i = tid; i < n_bias; i += kShapeThreads) {
            const int t = a.bias_tokens[static_cast<long long>(b) * a.max_bias + i];
            bias_token[i] = static_cast<unsigned>(t) < static_cast<unsigned>(a.V) ? t : -1;
            bias_sum[i] = a.bias_values[static_cast<long long>(b) * a.max_bias + i];
        }
        __syncthreads();
        // the first mention of a token gets the sum of all, in their order
        int t[kShapeBias / kShapeThreads];
        float sum[kShapeBias / kShapeThreads];
#pragma unroll
        for (int r = 0; r < kShapeBias / kShapeThreads; ++r) {
            const int i = tid + r * kShapeThreads;
            t[r] = i < n_bias ? bias_token[i] : -1;
            sum[r] = 0.f;
            if (t[r] < 0) continue;
            bool earlier = false;
#pragma unroll 8
            for (int k = 0; k < n_bias; ++k)
                if (bias_token[k] == t[r]) {
                    earlier |= k < i;
                    sum[r] = __fadd_rn(sum[r], bias_sum[k]);
                }
            if (earlier) t[r] = -1;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kShapeBias / kShapeThreads; ++r) {
            const int i = tid + r * kShapeThreads;
            if (i < n_bias) {
                bias_token[i] = t[r];
                bias_sum[i] = sum[r];
            }
        }
    };
    // rows: how many rows of the tile this CTA has from here on that begin at the same place of a vector
    auto enter_tile = [&](const ShapeItem& x, int rows) {
        __syncthreads();                                   // the last tile's marks are read, the stream's facts written
        const __nv_bfloat16* const logits = row_of(x);
        const int off = offset_of(logits), own = own_of(x.tile, off);
        first = x.tile * kShapeTile - off;                 // the tile's first token; below zero in front of an unaligned row
        // what was seen of this tile came with the last one, if that was of the same stream
        const uint32_t said = seen_at == own ? seen_next : seen ? bits_from(seen, a.words, own) : 0u;
        if (seen) {
            seen_at = own - kShapeTile;
            seen_next = bits_from(seen, a.words, seen_at);
        }
        marked[tid] = 0;
        if (tid == 0) n_listed = 0;
        __syncthreads();
        auto mark = [&](int token) {
            const int at = token - first;
            if (token < 0 || static_cast<unsigned>(at) >= static_cast<unsigned>(kShapeTile)) return false;
            atomicOr(&marked[at >> 5], 1u << (at & 31));
            return true;
        };
        for (int i0 = 0; i0 < n_bias; i0 += kShapeThreads) {   // once, but for more biases than threads
            if (i0 + tid < n_bias && mark(bias_token[i0 + tid])) listed[atomicAdd(&n_listed, 1)] = static_cast<uint16_t>(i0 + tid);
            __syncthreads();
            // biased tokens, whatever their logits
            const int n = n_listed;
            for (int e = tid; e < n * rows; e += kShapeThreads) {
                const int r = e / n, at = listed[e - r * n], t = bias_token[at], j = x.j + r;
                if (kMasks) {
                    const int m = a.mask_of[static_cast<long long>(x.b) * K1 + j];
                    if (static_cast<unsigned>(m) < static_cast<unsigned>(a.n_masks) && !((a.masks[static_cast<long long>(m) * a.words + (t >> 5)] >> (t & 31)) & 1)) continue;
                }
                look_at(t, __bfloat162float(logits[r * a.stride + t]), j, bias_sum[at]);
            }
            if (i0 + kShapeThreads < n_bias) {
                __syncthreads();
                if (tid == 0) n_listed = 0;
                __syncthreads();
            }
        }
        __syncthreads();
        const uint32_t biased = marked[tid];
        valid = valid_of(own);
        uint32_t special = said;
        if (penalties)
            for (int d = 0; d < a.K; ++d)
                if (static_cast<unsigned>(drafts[d] - own) < 32u) special |= 1u << (drafts[d] - own);
        special &= valid & ~biased;
        plain = valid & ~special & ~biased;
        odd = 0;
#pragma unroll
        for (int i = 0; i < kShapeVecs; ++i) {
            nan_where_clear(byte_of(plain, i), out[i]);
            odd |= byte_of(special, i) << (8 * i);
        }
        any_odd = __any_sync(kFull, odd != 0);
    };

    // ---- the rows
    if (tid == 0) n_waiting = 0;
    int stage = 0;
    bool moved = true;
    for (int it = 0; it < n_items; ++it, moved = x.next(a) || ragged) {
        if (moved) {
            settle();
            if (x.b != cur_b) enter_stream(x.b);
            enter_tile(x, ragged ? 1 : min(K1 - x.j, n_items - it));
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kShapeStages - 2) : "memory");
        copy();
        const int j = x.j;
        const uint32_t here = kMasks ? words[stage * kShapeThreads] : valid;
        // The block's other warps raise it meanwhile, and lanes that load it apart may find different values.  Whole-warp steps below
        // depend on it: it is lane 0's for all, and the shuffle brings the warp together.
        const unsigned so_far = __shfl_sync(kFull, static_cast<unsigned>(*reinterpret_cast<volatile unsigned long long*>(&best[j]) >> 32), 0);
        unsigned bound = so_far;
        auto element = [&](int vector, int l, int k) {     // of what lane l copied: the bits of a float
            return static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(slots - lane + l + (stage * kShapeVecs + vector) * kShapeThreads)[k]) << 16;
        };
        auto look_later = [&](int t, uint32_t z) {
            const int at = atomicAdd(&n_waiting, 1);
            if (at < kShapeWaiting) waiting[at] = make_int2(t, z | j);
            else look_at(t, __uint_as_float(z), j, 0.f);
        };
        const unsigned who = kMasks ? __ballot_sync(kFull, here != 0) : kFull;
        if (kMasks && __popc(who) <= kShapeFew) {
            // a mask that leaves next to nothing: word by word, a lane for a token
            unsigned key = 0, token = 0xffffffffu;
            __syncwarp();                                  // what the other lanes copied is there, too
            for (unsigned lanes = who; lanes; lanes &= lanes - 1) {
                const int l = __ffs(lanes) - 1;
                const uint32_t bits = __shfl_sync(kFull, here, l), their = __shfl_sync(kFull, plain, l);
                if (!((bits >> lane) & 1)) continue;
                const int e = l * 32 + lane, t = first + warp * 1024 + e;
                const uint32_t z = element(e >> 8, (e >> 3) & 31, e & 7);
                if (!(__uint_as_float(z) > -INFINITY)) continue;
                const unsigned k = ordered_key32(__uint_as_float(z));
                if ((their >> lane) & 1) {
                    if (k > key) {
                        key = k;
                        token = t;
                    }
                } else if (!((marked[warp * 32 + l] >> lane) & 1)) {
                    if (raising) look_at(t, __uint_as_float(z), j, 0.f);
                    else if (k >= so_far) look_later(t, z);
                }
            }
            __syncwarp();
            const unsigned warp_key = __reduce_max_sync(kFull, key);
            if (warp_key && warp_key >= so_far) {
                token = __reduce_min_sync(kFull, key == warp_key ? token : 0xffffffffu);
                if (lane == 0) atomicMax(&best[j], shaped_candidate(warp_key, token));
            }
            bound = max(so_far, warp_key);
        } else {
            uint32_t y[kShapeVecs][4];
#pragma unroll
            for (int i = 0; i < kShapeVecs; ++i) {
                const uint4 v = slots[(stage * kShapeVecs + i) * kShapeThreads];
                y[i][0] = v.x, y[i][1] = v.y, y[i][2] = v.z, y[i][3] = v.w;
            }
            // tokens that are their logit
            if (kMasks) {
#pragma unroll
                for (int i = 0; i < kShapeVecs; ++i) {
                    uint32_t n[4];
                    nan_where_clear(byte_of(here, i), n);
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[i][k] |= n[k];
                }
            }
            uint32_t top = 0xffffffffu;                        // NaN
#pragma unroll
            for (int i = 0; i < kShapeVecs; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) top = hmax2u(top, y[i][k] | out[i][k]);
            const float most = fmaxf(bf16lo(top), bf16hi(top));
            const unsigned key = most > -INFINITY ? ordered_key32(most) : 0u;
            const unsigned warp_key = __reduce_max_sync(kFull, key);
            if (warp_key && warp_key >= so_far) {
                unsigned token = 0xffffffffu;
                if (key == warp_key) {
#pragma unroll
                    for (int i = kShapeVecs - 1; i >= 0; --i) {
                        const int e = first_equal(make_uint4(y[i][0] | out[i][0], y[i][1] | out[i][1], y[i][2] | out[i][2], y[i][3] | out[i][3]), most);
                        if (e < 8) token = first + warp * 1024 + i * 256 + lane * 8 + e;
                    }
                }
                token = __reduce_min_sync(kFull, token);
                if (lane == 0) atomicMax(&best[j], shaped_candidate(warp_key, token));
            }
            bound = max(so_far, warp_key);
            // special tokens: looked at where their logit reaches the best so far (all of them, if a penalty may raise them)
            if (any_odd) {
                uint32_t odd_top = 0xffffffffu;
#pragma unroll
                for (int i = 0; i < kShapeVecs; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) odd_top = hmax2u(odd_top, y[i][k] | ~out[i][k]);
                const float odd_most = fmaxf(bf16lo(odd_top), bf16hi(odd_top));
                uint32_t lanes = __ballot_sync(kFull, odd && (raising || (odd_most > -INFINITY && ordered_key32(odd_most) >= bound)));
                if (lanes) {
                    __syncwarp();                              // what the other lanes copied is there, too
                    uint32_t left = odd;
                    if (kMasks) {
#pragma unroll
                        for (int i = 0; i < kShapeVecs; ++i) left &= byte_of(here, i) << (8 * i) | ~(0xffu << (8 * i));
                    }
                    for (; lanes; lanes &= lanes - 1) {        // lane k looks at token k of the lane's vectors
                        const int l = __ffs(lanes) - 1;
                        if (!((__shfl_sync(kFull, left, l) >> lane) & 1)) continue;
                        const int t = first + warp * 1024 + (lane >> 3) * 256 + l * 8 + (lane & 7);
                        const uint32_t z = element(lane >> 3, l, lane & 7);
                        if (raising) {
                            look_at(t, __uint_as_float(z), j, 0.f);
                        } else if (__uint_as_float(z) > -INFINITY && ordered_key32(__uint_as_float(z)) >= bound) {
                            look_later(t, z);
                        }
                    }
                }
                __syncwarp();
            }
        }
        // nothing above minus infinity so far: the lowest allowed token
        if (bound <= kKeyNothing) {
            const int t = __reduce_min_sync(kFull, here ? first + warp * 1024 + lane * 32 + __ffs(here) - 1 : 0x7fffffff);
            if (lane == 0) atomicMax(&best[j], t == 0x7fffffff ? kKeyNoneAllowed : shaped_candidate(kKeyNothing, t));
        }
        if (++stage == kShapeStages) stage = 0;
    }
    settle();
    flush();
}

// The kernel above is placed while this one ends: it needs no key before it has its first result, and all that came before this one
// has ended when this one begins.
__global__ void __launch_bounds__(256) clear_keys_kernel(unsigned long long* keys, long long n) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) keys[i] = 0;
}

// Accepts from keys; placed while the kernel before it ends, whatever that is, and waits for that end first of all.  (4 streams of three
// drafts, 151,936 logits: 10.5 us for the three kernels, 14.4 with a fill and kernels that are placed one after the other.)
__global__ void __launch_bounds__(128) verify_keys_kernel(AcceptArgs p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (b < p.B) accept_stream<kTailVerifyOnly, false>(DeviceSam{}, p, b, threadIdx.x & 31);
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
