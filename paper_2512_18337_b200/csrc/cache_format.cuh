// Paged 4-bit key/value cache: geometry of the pool, the bit format, and 16-bit element types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

namespace samb200 {

// What the kernels need of a sam_cache, by value.
struct CacheView {
    uint8_t* pages;
    int32_t* table;
    int32_t* seq_len;
    int32_t* ref;
    int32_t* free_list;
    int32_t* meta;          // n_free, status
    int32_t* scratch;
    int64_t page_bytes;     // all layers
    int32_t n_pages, n_streams, max_pages, n_layers, n_kv, D;
    int32_t log_p;          // log2(page_tokens)
    int32_t k_exp, v_exp;

    __device__ __forceinline__ int page_tokens() const { return 1 << log_p; }
    __device__ __forceinline__ int capacity() const { return max_pages << log_p; }
    __device__ __forceinline__ int tile_bytes() const { return 18 * D; }
    // Stream of row b, -1 if its id is out of range.
    __device__ __forceinline__ int stream_of(const int32_t* streams, int b) const {
        const int s = streams ? streams[b] : b;
        return static_cast<unsigned>(s) < static_cast<unsigned>(n_streams) ? s : -1;
    }
    __device__ __forceinline__ int length_of(int s) const { return min(max(seq_len[s], 0), capacity()); }
    __device__ __forceinline__ int32_t* row(int s) const { return table + static_cast<int64_t>(s) * max_pages; }
    // Page of a table entry, -1 if there is none (or its id is out of range).
    __device__ __forceinline__ int page_at(int s, int i) const {
        const int p = row(s)[i];
        return static_cast<unsigned>(p) < static_cast<unsigned>(n_pages) ? p : -1;
    }
    // First byte of the tiles of one layer and head in a page.
    __device__ __forceinline__ uint8_t* head_tiles(int page, int layer, int head) const {
        return pages + page * page_bytes +
               (static_cast<int64_t>(layer * n_kv + head) << (log_p - 4)) * tile_bytes();
    }
    __device__ __forceinline__ uint8_t* tile(int page, int layer, int head, int slot) const {
        return head_tiles(page, layer, head) + (slot >> 4) * tile_bytes();
    }
};

// Eight e2m1 codes -> four pairs of fp16 (exact); pair i holds codes 2i, 2i+1.  One conversion per pair, 56 pairs per
// clock and SM together with a multiplication each on B200; the two shifts and masks per pair that do the same on the
// integer pipe reach 24.  All four pairs have to be used: ptxas 12.9 reads the wrong byte when some are dead.
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t codes, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
}

// Two e4m3 bytes -> a pair of fp16 (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
    return h;
}

__device__ __forceinline__ float e4m3_to_float(uint8_t b) {
    return __half2float(__ushort_as_half(static_cast<unsigned short>(e4m3x2_to_half2(b) & 0xffff)));
}

__device__ __forceinline__ uint8_t float_to_e4m3(float x) {   // nearest, ties to even, saturating
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
    return static_cast<uint8_t>(r);
}

// Two floats -> a byte of two e2m1 codes (lo in the low nibble), nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t float2_to_e2m1(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tmov.b32 %0, {a, 0, 0, 0};\n\t}"
        : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}

template <typename T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
};

// 2^e for |e| <= 126, exactly.
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }

}  // namespace samb200
