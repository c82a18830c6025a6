// Keys and values into the 4-bit cache (append) and back (read): one thread per 16-channel block.
//
// A prompt of 49,152 tokens, 8 heads of 128, is 258 MB each way: append 62 us (4.2 TB/s), read 53 us (4.9 TB/s).  append is bound
// by instructions: 288 for the 32 blocks of a warp, 0.84 of the issue slots (with 64-bit divisions for the position, a correctly
// rounded division per element and element-wise maxima the two took 163 us).  It writes 2.4 million sectors where 1.8 hold the
// bytes, since a warp's scales lie in four tiles.  read uses 0.67 of the slots; a thread's 32 bytes go out as two stores that fill
// half a sector each, twice the write requests that the bytes need.
#pragma once

#include "cache_format.cuh"

namespace samb200 {

struct KvStrides {
    int64_t row, token, head;   // elements
};

constexpr int kIoThreads = 256, kIoBlocks = 2;   // 16-channel blocks of a thread: both loads are under way together

// Block number g of a row -> token and block of the token.  A CTA starts at a 64-bit number and goes on in 32 bits; magic =
// ceil(2^32 / per_token) divides numbers below 2^16 exactly (per_token is 4 or 8 a head, so the multiplier fits 32 bits).
struct IoPlace {
    int64_t token0;
    int rest0;
    __device__ __forceinline__ IoPlace(int64_t begin, int per_token) : token0(begin / per_token), rest0(static_cast<int>(begin - token0 * per_token)) {}
    __device__ __forceinline__ void at(int i, int per_token, uint32_t magic, int64_t& token, int& block) const {
        const uint32_t g = rest0 + i, q = __umulhi(g, magic);
        token = token0 + q;
        block = g - q * per_token;
    }
};

// Sixteen elements, as 16-byte loads where everything is aligned for them.
template <typename T>
__device__ __forceinline__ void load_block(const T* p, bool wide, uint32_t (&x)[8]) {
    if (wide) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = h[2 * i] | static_cast<uint32_t>(h[2 * i + 1]) << 16;
    }
}

// Pairs of 16-bit elements.
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static __device__ __forceinline__ float lo(uint32_t x) { return __uint_as_float(x << 16); }
    static __device__ __forceinline__ float hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t max_nan(uint32_t x, uint32_t y) {
        uint32_t z;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
        return z;
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t z;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(z) : "f"(hi), "f"(lo));
        return z;
    }
};
template <> struct Pair<__half> {
    static __device__ __forceinline__ float lo(uint32_t x) { return __low2float(*reinterpret_cast<__half2*>(&x)); }
    static __device__ __forceinline__ float hi(uint32_t x) { return __high2float(*reinterpret_cast<__half2*>(&x)); }
    static __device__ __forceinline__ uint32_t max_nan(uint32_t x, uint32_t y) {
        uint32_t z;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
        return z;
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t z;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(z) : "f"(hi), "f"(lo));
        return z;
    }
};

// Sixteen values -> eight bytes of codes and a scale byte.  The definition rounds x / scale.  With an element of at most 11
// significant bits and a scale of at most 4, the quotient either is a tie between two codes or lies 2^-11 of itself or more
// away from every tie; so x times the reciprocal, rounded to 16 bits, falls on the same side, and on the tie where it is one.
template <typename T>
__device__ __forceinline__ uint2 quantise_block(const uint32_t (&x)[8], int exp, uint8_t* scale) {
    uint32_t big = x[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 8; ++i) big = Pair<T>::max_nan(big, x[i] & 0x7fff7fffu);
    const float amax = fmaxf(Pair<T>::lo(big), Pair<T>::hi(big));
    const bool nan = Pair<T>::lo(big) != Pair<T>::lo(big) || Pair<T>::hi(big) != Pair<T>::hi(big);
    const float down = pow2(-exp);
    const uint8_t s8 = nan ? 0x7f : float_to_e4m3(__fdiv_rn(amax * down, 6.f));
    *scale = s8;
    if (nan || s8 == 0) return make_uint2(0, 0);
    const float r = __frcp_rn(e4m3_to_float(s8)) * down;
    auto rounded = [&](float y) { return __uint_as_float((__float_as_uint(y * r) + 0x80u) & 0xffffff00u); };
    uint32_t byte[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) byte[i] = float2_to_e2m1(rounded(Pair<T>::lo(x[i])), rounded(Pair<T>::hi(x[i])));
    return make_uint2(byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24, byte[4] | byte[5] << 8 | byte[6] << 16 | byte[7] << 24);
}

// Grid: (blocks of a row, rows, keys / values).
template <typename T>
__global__ void __launch_bounds__(kIoThreads) append_kernel(CacheView c, int layer, const T* k, const T* v, KvStrides st, bool wide,
                                                            int Q, uint32_t magic, const int32_t* streams, const int32_t* n_new) {
    const int b = blockIdx.y;
    const bool is_v = blockIdx.z;
    const int s = c.stream_of(streams, b);
    if (s < 0) return;
    const int n = n_new ? min(n_new[b], Q) : Q;
    const int log_blocks = c.D == 128 ? 3 : 2, per_token = c.n_kv << log_blocks;
    const IoPlace place(static_cast<int64_t>(blockIdx.x) * (kIoThreads * kIoBlocks), per_token);
    if (place.token0 >= n) return;
    const int len = c.length_of(s), exp = is_v ? c.v_exp : c.k_exp;
    const T* src = (is_v ? v : k) + b * st.row;
    uint32_t x[kIoBlocks][8];
    uint8_t* tile[kIoBlocks];
    int where[kIoBlocks], block[kIoBlocks];   // token of the tile; block of the token's head
#pragma unroll
    for (int u = 0; u < kIoBlocks; ++u) {
        int64_t i;
        int r;
        place.at(u * kIoThreads + threadIdx.x, per_token, magic, i, r);
        const int64_t pos = len + i;
        tile[u] = nullptr;
        if (i >= n || pos >= c.capacity()) continue;
        const int page = c.page_at(s, static_cast<int>(pos >> c.log_p));
        if (page < 0) continue;
        const int head = r >> log_blocks, slot = static_cast<int>(pos) & (c.page_tokens() - 1);
        block[u] = r & ((1 << log_blocks) - 1);
        where[u] = slot & 15;
        tile[u] = c.tile(page, layer, head, slot);
        load_block(src + i * st.token + head * st.head + block[u] * 16, wide, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kIoBlocks; ++u) {
        if (!tile[u]) continue;
        uint8_t scale;
        const uint2 codes = quantise_block<T>(x[u], exp, &scale);
        *reinterpret_cast<uint2*>(tile[u] + (is_v ? 8 * c.D : 0) + where[u] * (c.D >> 1) + block[u] * 8) = codes;
        tile[u][(is_v ? 17 : 16) * c.D + (where[u] << log_blocks) + block[u]] = scale;
    }
}

template <typename T>
__global__ void __launch_bounds__(kIoThreads) read_kernel(CacheView c, int layer, int Q, uint32_t magic, const int32_t* streams, const int32_t* first,
                                                          const int32_t* n_read, T* k_out, T* v_out) {
    const int b = blockIdx.y;
    const bool is_v = blockIdx.z;
    const int s = c.stream_of(streams, b);
    const int n = s < 0 ? 0 : n_read ? min(n_read[b], Q) : Q;
    const int log_blocks = c.D == 128 ? 3 : 2, per_token = c.n_kv << log_blocks;
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * (kIoThreads * kIoBlocks), all = static_cast<int64_t>(Q) * per_token;
    const IoPlace place(begin, per_token);
    const int64_t at0 = first ? first[b] : 0;
    const float up = pow2(is_v ? c.v_exp : c.k_exp);
    uint2 codes[kIoBlocks];
    uint32_t scale[kIoBlocks];
#pragma unroll
    for (int u = 0; u < kIoBlocks; ++u) {
        int64_t i;
        int r;
        place.at(u * kIoThreads + threadIdx.x, per_token, magic, i, r);
        const int64_t pos = at0 + i;
        codes[u] = make_uint2(0, 0);
        scale[u] = 0;
        if (i >= n || pos < 0 || pos >= c.capacity()) continue;
        const int page = c.page_at(s, static_cast<int>(pos >> c.log_p));
        if (page < 0) continue;
        const int head = r >> log_blocks, block = r & ((1 << log_blocks) - 1), slot = static_cast<int>(pos) & (c.page_tokens() - 1);
        const uint8_t* tile = c.tile(page, layer, head, slot);
        codes[u] = *reinterpret_cast<const uint2*>(tile + (is_v ? 8 * c.D : 0) + (slot & 15) * (c.D >> 1) + block * 8);
        scale[u] = tile[(is_v ? 17 : 16) * c.D + ((slot & 15) << log_blocks) + block];
    }
    T* out = (is_v ? v_out : k_out) + b * all * 16;
#pragma unroll
    for (int u = 0; u < kIoBlocks; ++u) {
        const int64_t e = begin + u * kIoThreads + threadIdx.x;
        if (e >= all) continue;
        const float f = e4m3_to_float(static_cast<uint8_t>(scale[u])) * up;
        uint32_t y[8];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t h[4];
            e2m1x8_to_half2(w ? codes[u].y : codes[u].x, h);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float2 p = __half22float2(*reinterpret_cast<__half2*>(&h[q]));
                y[w * 4 + q] = Pair<T>::pack(p.x * f, p.y * f);
            }
        }
        uint4* o = reinterpret_cast<uint4*>(out + e * 16);
        o[0] = make_uint4(y[0], y[1], y[2], y[3]);
        o[1] = make_uint4(y[4], y[5], y[6], y[7]);
    }
}

}  // namespace samb200
