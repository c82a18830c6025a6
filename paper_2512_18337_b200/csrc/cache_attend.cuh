// Attention over the 4-bit cache.
#pragma once

#include "cache_format.cuh"

namespace samb200 {

struct AttendArgs {
    CacheView c;
    const void* q;
    void* out;
    float* lse;
    const int32_t* streams;
    const int32_t* n_new;
    int64_t q_row, q_token, q_head, o_row, o_token, o_head;   // strides in elements
    int32_t layer, B, Q, H, window;
    float scale;
};

// One warp per query row; a lane holds D/32 neighbouring channels, the softmax runs token by token.
template <typename T, int D>
__global__ void __launch_bounds__(128) attend_rows_kernel(AttendArgs a) {
    constexpr int C = D / 32;
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 31;
    const int64_t w = blockIdx.x * 4ll + (threadIdx.x >> 5);
    if (w >= static_cast<int64_t>(a.B) * a.Q * a.H) return;
    const int h = static_cast<int>(w % a.H), i = static_cast<int>(w / a.H % a.Q), b = static_cast<int>(w / a.H / a.Q);
    const int s = c.stream_of(a.streams, b);
    const int n = s < 0 ? 0 : a.n_new ? min(a.n_new[b], a.Q) : a.Q;
    const int head = h / (a.H / c.n_kv);
    const T* q = static_cast<const T*>(a.q) + b * a.q_row + i * a.q_token + h * a.q_head;
    T* out = static_cast<T*>(a.out) + b * a.o_row + i * a.o_token + h * a.o_head;
    float qv[C], o[C], m = -INFINITY, l = 0.f;
    for (int j = 0; j < C; ++j) {
        qv[j] = Elem<T>::to_float(q[lane * C + j]) * a.scale;
        o[j] = 0.f;
    }
    if (i < n) {
        const int64_t p = static_cast<int64_t>(c.length_of(s)) + i;
        const int64_t end = min(p + 1, static_cast<int64_t>(c.capacity()));
        const int64_t begin = a.window > 0 ? max(p - a.window + 1, int64_t(0)) : 0;
        for (int64_t j = begin; j < end; ++j) {
            const int page = c.page_at(s, static_cast<int>(j >> c.log_p));
            if (page < 0) continue;
            const int slot = static_cast<int>(j) & (c.page_tokens() - 1), t = slot & 15;
            const uint8_t* tile = c.tile(page, a.layer, head, slot);
            float kv[2][C];
            for (int v = 0; v < 2; ++v) {
                const uint8_t* codes = tile + v * 8 * D + t * (D / 2) + lane * (C / 2);
                const float sc = e4m3_to_float(tile[(16 + v) * D + t * (D / 16) + lane * C / 16]) * pow2(v ? c.v_exp : c.k_exp);
                for (int k = 0; k < C; k += 2) {
                    const float2 f = e2m1x2_to_float2(codes[k / 2]);
                    kv[v][k] = f.x * sc;
                    kv[v][k + 1] = f.y * sc;
                }
            }
            float dot = 0.f;
            for (int k = 0; k < C; ++k) dot += qv[k] * kv[0][k];
            for (int d = 16; d; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
            const float mn = fmaxf(m, dot), keep = __expf(m - mn), e = __expf(dot - mn);
            l = l * keep + e;
            for (int k = 0; k < C; ++k) o[k] = o[k] * keep + e * kv[1][k];
            m = mn;
        }
    }
    for (int k = 0; k < C; ++k) out[lane * C + k] = Elem<T>::from_float(l > 0.f ? o[k] / l : l == 0.f ? 0.f : l);
    if (a.lse && lane == 0) a.lse[(static_cast<int64_t>(b) * a.Q + i) * a.H + h] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace samb200
