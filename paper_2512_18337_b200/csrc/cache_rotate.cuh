// Queries and keys turned to their positions, and keys and values into the 4-bit cache, in one pass.
//
// Channel pairs (a, b) of a token at position p become (a cos - b sin, b cos + a sin) with the angle p f_i.  The angle is held as
// a fraction of a turn in 64 bits, so that p times the turn's fraction, modulo 2^64, is exact for every position; what is left
// to round is the fraction's top 32 bits to a float, 2^-25 of a half turn.  Products and sums are in 32 bits; a query is rounded once, to its
// own type, and a key once, to its code: it does not pass through 16 bits in between.
//
// A CTA takes a few tokens: their sines and cosines go to shared memory once and serve all heads.  Then a thread takes 32
// channels of a head: two blocks of 16, which hold both halves of their pairs.
#pragma once

#include "cache_io.cuh"

namespace samb200 {

constexpr int kTurnThreads = 256, kTurnTokens = 8;   // most tokens of a CTA

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

// Sixteen 32-bit values -> codes and a scale byte.  The quotient by the scale is a product with its reciprocal, off by less than two
// units in the last place: rounded to 22 bits, one that is a tie between two codes is that tie (ties have three bits).
__device__ __forceinline__ uint2 quantise_block32(const float (&x)[16], int exp, uint8_t* scale) {
    float big = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        big = fmaxf(big, fabsf(x[i]));
        nan |= x[i] != x[i];
    }
    const float down = pow2(-exp);
    const uint8_t s8 = nan ? 0x7f : float_to_e4m3(__fdiv_rn(big * down, 6.f));
    *scale = s8;
    if (nan || s8 == 0) return make_uint2(0, 0);
    const float r = __frcp_rn(e4m3_to_float(s8)) * down;
    auto rounded = [&](float y) { return __uint_as_float((__float_as_uint(y * r) + 2u) & ~3u); };
    uint32_t byte[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) byte[i] = float2_to_e2m1(rounded(x[2 * i]), rounded(x[2 * i + 1]));
    return make_uint2(byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24, byte[4] | byte[5] << 8 | byte[6] << 16 | byte[7] << 24);
}

template <typename T>
__device__ __forceinline__ void store_block(T* p, bool wide, const uint32_t (&x)[8]) {
    if (wide) {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(x[4], x[5], x[6], x[7]);
    } else {
        uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[2 * i] = static_cast<uint16_t>(x[i]);
            h[2 * i + 1] = static_cast<uint16_t>(x[i] >> 16);
        }
    }
}

// Sixteen elements by ordinary loads: the turned queries may take the place of the queries.
template <typename T>
__device__ __forceinline__ void load_block_in_place(const T* p, bool wide, uint32_t (&x)[8]) {
    if (wide) {
        const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = h[2 * i] | static_cast<uint32_t>(h[2 * i + 1]) << 16;
    }
}

// Grid: (runs of tokens, rows).
template <typename T>
__global__ void __launch_bounds__(kTurnThreads) append_rotated_kernel(const __grid_constant__ TurnArgs a) {
    __shared__ float2 turn[kTurnTokens][64];            // cosine, sine
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
    const int log_d = c.D == 128 ? 2 : 1, heads = a.H + 2 * c.n_kv, turned = a.rotary >> 5;   // units of a head; of them turned
    for (int e = threadIdx.x; e < (here * heads) << log_d; e += kTurnThreads) {
        const uint32_t g = e >> log_d, t = __umulhi(g, a.magic);
        const int head = g - t * heads, u = e & ((1 << log_d) - 1), i = i0 + t;
        const bool on = i < n, is_q = head < a.H, is_v = head >= a.H + c.n_kv, turns = !is_v && u < turned;
        // the unit's two blocks
        const int block0 = turns && !a.interleaved ? u : 2 * u, block1 = turns && !a.interleaved ? u + turned : 2 * u + 1;
        uint8_t* tile = nullptr;
        const int64_t at = static_cast<int64_t>(len) + i;
        const int slot = static_cast<int>(at) & (c.page_tokens() - 1), kv = is_v ? head - a.H - c.n_kv : head - a.H;
        if (!is_q) {
            if (!on || at >= c.capacity()) continue;
            const int page = c.page_at(s, static_cast<int>(at >> c.log_p));
            if (page < 0) continue;
            tile = c.tile(page, a.layer, kv, slot);
        }
        uint32_t x0[8] = {}, x1[8] = {};
        if (on) {
            const T* src = is_q ? static_cast<const T*>(a.q) + b * a.qs.row + i * a.qs.token + head * a.qs.head
                                : static_cast<const T*>(is_v ? a.v : a.k) + b * a.ks.row + i * a.ks.token + kv * a.ks.head;
            load_block_in_place(src + block0 * 16, is_q ? a.q_wide : a.k_wide, x0);
            load_block_in_place(src + block1 * 16, is_q ? a.q_wide : a.k_wide, x1);
        }
        if (!is_v) {
            float y0[16], y1[16];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                y0[2 * k] = Pair<T>::lo(x0[k]), y0[2 * k + 1] = Pair<T>::hi(x0[k]);
                y1[2 * k] = Pair<T>::lo(x1[k]), y1[2 * k + 1] = Pair<T>::hi(x1[k]);
            }
            if (turns && on) {
                const float2* w = turn[t] + u * 16;
                if (a.interleaved) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 r0 = w[k], r1 = w[8 + k];
                        const float p0 = y0[2 * k], p1 = y0[2 * k + 1], p2 = y1[2 * k], p3 = y1[2 * k + 1];
                        y0[2 * k] = p0 * r0.x - p1 * r0.y;
                        y0[2 * k + 1] = p1 * r0.x + p0 * r0.y;
                        y1[2 * k] = p2 * r1.x - p3 * r1.y;
                        y1[2 * k + 1] = p3 * r1.x + p2 * r1.y;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 r = w[k];
                        const float p0 = y0[k], p1 = y1[k];
                        y0[k] = p0 * r.x - p1 * r.y;
                        y1[k] = p1 * r.x + p0 * r.y;
                    }
                }
            }
            if (is_q) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x0[k] = Pair<T>::pack(y0[2 * k], y0[2 * k + 1]);
                    x1[k] = Pair<T>::pack(y1[2 * k], y1[2 * k + 1]);
                }
                T* out = static_cast<T*>(a.q_out) + b * a.os.row + i * a.os.token + head * a.os.head;
                store_block(out + block0 * 16, a.o_wide, x0);
                store_block(out + block1 * 16, a.o_wide, x1);
                continue;
            }
            uint8_t s0, s1;
            uint8_t* codes = tile + (slot & 15) * (c.D >> 1);
            uint8_t* scales = tile + 16 * c.D + (slot & 15) * (c.D >> 4);
            *reinterpret_cast<uint2*>(codes + block0 * 8) = quantise_block32(y0, c.k_exp, &s0);
            *reinterpret_cast<uint2*>(codes + block1 * 8) = quantise_block32(y1, c.k_exp, &s1);
            scales[block0] = s0;
            scales[block1] = s1;
        } else {
            uint8_t s0, s1;
            uint8_t* codes = tile + 8 * c.D + (slot & 15) * (c.D >> 1);
            uint8_t* scales = tile + 17 * c.D + (slot & 15) * (c.D >> 4);
            *reinterpret_cast<uint2*>(codes + block0 * 8) = quantise_block<T>(x0, c.v_exp, &s0);
            *reinterpret_cast<uint2*>(codes + block1 * 8) = quantise_block<T>(x1, c.v_exp, &s1);
            scales[block0] = s0;
            scales[block1] = s1;
        }
    }
}

}  // namespace samb200
