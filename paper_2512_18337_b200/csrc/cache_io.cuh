// Keys and values into the 4-bit cache (append) and back (read): one thread per 16-channel block.
#pragma once

#include "cache_format.cuh"

namespace samb200 {

struct KvStrides {
    int64_t row, token, head;   // elements
};

// Sixteen elements at p, as 16-byte loads where everything is aligned for them.
template <typename T>
__device__ __forceinline__ void load_block(const T* p, bool wide, float (&x)[16]) {
    alignas(16) T e[16];
    if (wide) {
        reinterpret_cast<uint4*>(e)[0] = __ldg(reinterpret_cast<const uint4*>(p));
        reinterpret_cast<uint4*>(e)[1] = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = Elem<T>::to_float(e[i]);
}

// Sixteen values -> eight bytes of codes and a scale byte.  amax / 6 and x / scale are correctly rounded divisions of
// 16-bit inputs by numbers of at most four bits, so a tie of the definition is a tie here and nothing else is one.
__device__ __forceinline__ uint2 quantise_block(const float (&x)[16], float inv_exp, uint8_t* scale) {
    float amax = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        amax = fmaxf(amax, fabsf(x[i]));
        nan |= x[i] != x[i];
    }
    const uint8_t s8 = nan ? 0x7f : float_to_e4m3(__fdiv_rn(amax * inv_exp, 6.f));
    *scale = s8;
    uint2 codes = make_uint2(0, 0);
    if (nan || s8 == 0) return codes;
    const float s = e4m3_to_float(s8);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const uint32_t b = float2_to_e2m1(__fdiv_rn(x[i] * inv_exp, s), __fdiv_rn(x[i + 1] * inv_exp, s));
        if (i < 8) codes.x |= b << (4 * i);
        else codes.y |= b << (4 * (i - 8));
    }
    return codes;
}

template <typename T>
__global__ void __launch_bounds__(256) append_kernel(CacheView c, int layer, const T* k, const T* v, KvStrides st, bool wide,
                                                     int Q, const int32_t* streams, const int32_t* n_new) {
    const int b = blockIdx.y;
    const int s = c.stream_of(streams, b);
    if (s < 0) return;
    const int n = n_new ? min(n_new[b], Q) : Q;
    const int blocks = c.D >> 4, per_token = c.n_kv * blocks;
    const int64_t total = static_cast<int64_t>(max(n, 0)) * per_token * 2;
    const int len = c.length_of(s);
    for (int64_t e = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; e < total; e += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t half = total >> 1;
        const bool is_v = e >= half;
        const int64_t f = is_v ? e - half : e;
        const int i = static_cast<int>(f / per_token), r = static_cast<int>(f % per_token);
        const int head = r / blocks, blk = r % blocks;
        const int64_t pos = static_cast<int64_t>(len) + i;
        if (pos >= c.capacity()) continue;
        const int page = c.page_at(s, static_cast<int>(pos >> c.log_p));
        if (page < 0) continue;
        float x[16];
        load_block((is_v ? v : k) + b * st.row + i * st.token + head * st.head + blk * 16, wide, x);
        const int slot = static_cast<int>(pos) & (c.page_tokens() - 1), t = slot & 15;
        uint8_t* tile = c.tile(page, layer, head, slot);
        uint8_t scale;
        const uint2 codes = quantise_block(x, pow2(-(is_v ? c.v_exp : c.k_exp)), &scale);
        *reinterpret_cast<uint2*>(tile + (is_v ? 8 * c.D : 0) + t * (c.D >> 1) + blk * 8) = codes;
        tile[(is_v ? 17 : 16) * c.D + t * blocks + blk] = scale;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) read_kernel(CacheView c, int layer, int Q, const int32_t* streams, const int32_t* first,
                                                   const int32_t* n_read, T* k_out, T* v_out) {
    const int b = blockIdx.y;
    const int s = c.stream_of(streams, b);
    const int n = s < 0 ? 0 : n_read ? min(n_read[b], Q) : Q;
    const int blocks = c.D >> 4, per_token = c.n_kv * blocks;
    const int64_t half = static_cast<int64_t>(Q) * per_token;
    const int64_t at0 = first ? first[b] : 0;
    for (int64_t e = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; e < 2 * half; e += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const bool is_v = e >= half;
        const int64_t f = is_v ? e - half : e;
        const int i = static_cast<int>(f / per_token), r = static_cast<int>(f % per_token);
        const int head = r / blocks, blk = r % blocks;
        const int64_t pos = at0 + i;
        int page = -1;
        if (i < n && pos >= 0 && pos < c.capacity()) page = c.page_at(s, static_cast<int>(pos >> c.log_p));
        alignas(16) T y[16];
        if (page < 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = Elem<T>::from_float(0.f);
        } else {
            const int slot = static_cast<int>(pos) & (c.page_tokens() - 1), t = slot & 15;
            const uint8_t* tile = c.tile(page, layer, head, slot);
            const uint2 codes = *reinterpret_cast<const uint2*>(tile + (is_v ? 8 * c.D : 0) + t * (c.D >> 1) + blk * 8);
            const float sc = e4m3_to_float(tile[(is_v ? 17 : 16) * c.D + t * blocks + blk]) * pow2(is_v ? c.v_exp : c.k_exp);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t h[4];
                e2m1x8_to_half2(w ? codes.y : codes.x, h);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 p = __half22float2(*reinterpret_cast<__half2*>(&h[j]));
                    y[w * 8 + 2 * j] = Elem<T>::from_float(p.x * sc);
                    y[w * 8 + 2 * j + 1] = Elem<T>::from_float(p.y * sc);
                }
            }
        }
        T* o = (is_v ? v_out : k_out) + (b * half + f) * 16;
        reinterpret_cast<uint4*>(o)[0] = reinterpret_cast<const uint4*>(y)[0];
        reinterpret_cast<uint4*>(o)[1] = reinterpret_cast<const uint4*>(y)[1];
    }
}

}  // namespace samb200
