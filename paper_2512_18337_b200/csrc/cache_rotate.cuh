// Queries and keys turned to their positions, and keys and values into the 4-bit cache, in one pass.
//
// Channel pairs (a, b) of a token at position p become (a cos - b sin, b cos + a sin) with the angle p f_i.  The angle is held as
// a fraction of a turn in 64 bits, so that p times the turn's fraction, modulo 2^64, is exact for every position; what is left
// to round is the fraction's top 32 bits to a float, 2^-25 of a half turn.  Products and sums are in 32 bits; a query is rounded once, to its
// own type, and a key once, to its code: it does not pass through 16 bits in between.
//
// A CTA takes a few tokens: their sines and cosines go to shared memory once and serve all heads.  Then a thread takes two pieces
// of eight channels of a head, which hold both halves of their pairs; neighbouring threads take neighbouring pieces, so that loads and stores
// fill sectors, and share the scale of their sixteen channels.
//
// 256 streams of up to 17 tokens, 32/8 heads of 128 (80 MB): 27 us; 20,000 tokens, 28/4 heads (338 MB): 70 us, 4.8 TB/s.  Bound by
// instructions: 308 and 279 for the sixteen channels of a thread, 0.7 of the issue slots, most of them to find out where a unit lies.  Tried: two
// blocks of 16 channels a thread (half-filled sectors: 29 and 74 us), the next unit's loads ahead of this one's products (30 and 84), a
// thread that keeps to its channels token after token (29 and 85: keys and values become a chain of a few microseconds).
#pragma once

#include "cache_io.cuh"

namespace samb200 {

constexpr int kTurnThreads = 128, kTurnTokens = 8, kTurnCtasPerSm = 10;   // most tokens of a CTA

struct TurnArgs {
    CacheView c;
    const void* q;
    const void* k;
    const void* v;
    void* q_out;
    KvStrides qs, ks, os;          // of queries; of keys and values; of the turned queries
    const uint64_t* turns;         // [rotary / 2] turns per position, in 2^-64
    const int32_t* positions;      // [B, Q], or null: behind the committed tokens
    const int32_t* streams;
    const int32_t* n_new;
    float factor;                  // of sines and cosines
    int32_t layer, B, Q, H, rotary, interleaved, tokens;   // tokens: of a CTA
    uint32_t magic;                // ceil(2^32 / (H + 2 n_kv))
    bool q_wide, k_wide, o_wide;
};

// Eight 32-bit values of a block whose other eight the neighbouring lane has -> four bytes of codes, and the block's scale byte.  The
// quotient by the scale is a product with its reciprocal, off by less than two units in the last place: rounded to 22 bits, one that is a
// tie between two codes is that tie (ties have three bits).
__device__ __forceinline__ uint32_t quantise_half(const float (&x)[8], int exp, uint8_t* scale) {
    uint32_t big = 0;                                     // magnitudes in the order of their bits, NaN above all
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(x[i]) & 0x7fffffffu);
    big = max(big, __shfl_xor_sync(3u << (threadIdx.x & 30), big, 1));
    const float down = pow2(-exp);
    const bool nan = big > 0x7f800000u;
    const uint8_t s8 = nan ? 0x7f : float_to_e4m3(__fdiv_rn(__uint_as_float(big) * down, 6.f));
    *scale = s8;
    if (nan || s8 == 0) return 0;
    const float r = __frcp_rn(e4m3_to_float(s8)) * down;
    auto rounded = [&](float y) { return __uint_as_float((__float_as_uint(y * r) + 2u) & ~3u); };
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) codes |= float2_to_e2m1(rounded(x[2 * i]), rounded(x[2 * i + 1])) << (8 * i);
    return codes;
}

// Eight channels, by ordinary loads: the turned queries may take the place of the queries.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* p, bool wide) {
    if (wide) return *reinterpret_cast<const uint4*>(p);
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    return make_uint4(h[0] | static_cast<uint32_t>(h[1]) << 16, h[2] | static_cast<uint32_t>(h[3]) << 16, h[4] | static_cast<uint32_t>(h[5]) << 16,
                      h[6] | static_cast<uint32_t>(h[7]) << 16);
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, bool wide, const float (&x)[8]) {
    const uint4 y = make_uint4(Pair<T>::pack(x[0], x[1]), Pair<T>::pack(x[2], x[3]), Pair<T>::pack(x[4], x[5]), Pair<T>::pack(x[6], x[7]));
    if (wide) {
        *reinterpret_cast<uint4*>(p) = y;
    } else {
        uint16_t* h = reinterpret_cast<uint16_t*>(p);
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[2 * i] = static_cast<uint16_t>(w[i]);
            h[2 * i + 1] = static_cast<uint16_t>(w[i] >> 16);
        }
    }
}

// Grid: (runs of tokens, rows).
template <typename T, int D>
__global__ void __launch_bounds__(kTurnThreads, kTurnCtasPerSm) append_rotated_kernel(const __grid_constant__ TurnArgs a) {
    constexpr int kUnits = D / 16;                        // of a head
    __shared__ alignas(16) float2 turn[kTurnTokens][D / 2];   // cosine, sine
    const CacheView& c = a.c;
    const int b = blockIdx.y;
    const int s = c.stream_of(a.streams, b);
    const int n = s < 0 ? 0 : min(a.n_new ? a.n_new[b] : a.Q, a.Q), len = s < 0 ? 0 : c.length_of(s);
    const int i0 = static_cast<int>(blockIdx.x) * a.tokens, here = min(a.tokens, a.Q - i0), half = a.rotary >> 1;
    for (int e = threadIdx.x; e < here * half; e += kTurnThreads) {
        const int t = e / half, f = e - t * half, i = i0 + t;
        if (i >= n) break;
        const int64_t p = a.positions ? a.positions[static_cast<int64_t>(b) * a.Q + i] : static_cast<int64_t>(len) + i;
        const int part = static_cast<int>((static_cast<uint64_t>(p) * a.turns[f]) >> 32);   // of a turn, in 2^-32, signed
        float2 y;
        sincospif(static_cast<float>(part) * 4.656612873077393e-10f, &y.y, &y.x);
        turn[t][f] = make_float2(y.x * a.factor, y.y * a.factor);
    }
    __syncthreads();
    const int heads = a.H + 2 * c.n_kv, turned = a.rotary >> 4;   // units of a head that hold pairs of halves
    for (int e = threadIdx.x; e < here * heads * kUnits; e += kTurnThreads) {
        const uint32_t g = e / kUnits, t = __umulhi(g, a.magic);
        const int head = g - t * heads, u = e % kUnits, i = i0 + t;
        const bool on = i < n, is_q = head < a.H, is_v = head >= a.H + c.n_kv;
        // the unit's two pieces of eight channels
        int piece0 = u, piece1 = u + kUnits;
        if (!a.interleaved) {
            piece0 = u < turned ? u : u + turned;
            piece1 = u < turned ? u + turned : u + kUnits;
        }
        uint8_t* tile = nullptr;
        const int64_t at = static_cast<int64_t>(len) + i;
        const int slot = static_cast<int>(at) & (c.page_tokens() - 1), kv = is_v ? head - a.H - c.n_kv : head - a.H;
        if (!is_q) {
            if (!on || at >= c.capacity()) continue;
            const int page = c.page_at(s, static_cast<int>(at >> c.log_p));
            if (page < 0) continue;
            tile = c.tile(page, a.layer, kv, slot);
        }
        uint4 r0 = make_uint4(0, 0, 0, 0), r1 = r0;
        if (on) {
            const T* src = is_q ? static_cast<const T*>(a.q) + b * a.qs.row + i * a.qs.token + head * a.qs.head
                                : static_cast<const T*>(is_v ? a.v : a.k) + b * a.ks.row + i * a.ks.token + kv * a.ks.head;
            r0 = load_piece(src + piece0 * 8, is_q ? a.q_wide : a.k_wide);
            r1 = load_piece(src + piece1 * 8, is_q ? a.q_wide : a.k_wide);
        }
        const uint32_t w0[4] = {r0.x, r0.y, r0.z, r0.w}, w1[4] = {r1.x, r1.y, r1.z, r1.w};
        float y0[8], y1[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y0[2 * k] = Pair<T>::lo(w0[k]), y0[2 * k + 1] = Pair<T>::hi(w0[k]);
            y1[2 * k] = Pair<T>::lo(w1[k]), y1[2 * k + 1] = Pair<T>::hi(w1[k]);
        }
        if (on && !is_v) {
            if (a.interleaved) {
                auto turn_pairs = [&](float (&y)[8], int piece) {
                    if (piece >= 2 * turned) return;
                    const float4* w = reinterpret_cast<const float4*>(turn[t] + piece * 4);   // two angles each
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float4 r = w[k];
                        const float p0 = y[4 * k], p1 = y[4 * k + 2];
                        y[4 * k] = p0 * r.x - y[4 * k + 1] * r.y;
                        y[4 * k + 1] = y[4 * k + 1] * r.x + p0 * r.y;
                        y[4 * k + 2] = p1 * r.z - y[4 * k + 3] * r.w;
                        y[4 * k + 3] = y[4 * k + 3] * r.z + p1 * r.w;
                    }
                };
                turn_pairs(y0, piece0);
                turn_pairs(y1, piece1);
            } else if (u < turned) {
                const float4* w = reinterpret_cast<const float4*>(turn[t] + u * 8);
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const float4 r = w[k >> 1];
                    const float p0 = y0[k], p1 = y0[k + 1];
                    y0[k] = p0 * r.x - y1[k] * r.y;
                    y1[k] = y1[k] * r.x + p0 * r.y;
                    y0[k + 1] = p1 * r.z - y1[k + 1] * r.w;
                    y1[k + 1] = y1[k + 1] * r.z + p1 * r.w;
                }
            }
        }
        if (is_q) {
            T* out = static_cast<T*>(a.q_out) + b * a.os.row + i * a.os.token + head * a.os.head;
            store_piece(out + piece0 * 8, a.o_wide, y0);
            store_piece(out + piece1 * 8, a.o_wide, y1);
        } else {
            uint8_t s0, s1;
            uint8_t* codes = tile + (is_v ? 8 * D : 0) + (slot & 15) * (D / 2);
            uint8_t* scales = tile + (is_v ? 17 : 16) * D + (slot & 15) * (D / 16);
            const int exp = is_v ? c.v_exp : c.k_exp;
            *reinterpret_cast<uint32_t*>(codes + piece0 * 4) = quantise_half(y0, exp, &s0);
            *reinterpret_cast<uint32_t*>(codes + piece1 * 4) = quantise_half(y1, exp, &s1);
            if (!(u & 1)) {
                scales[piece0 >> 1] = s0;
                scales[piece1 >> 1] = s1;
            }
        }
    }
}

}  // namespace samb200
