// C ABI of the paged 4-bit cache: argument checks and kernel launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "sam.h"
#include "sam_common.h"
#include "attend_stream.cuh"
#include "attend_wide.cuh"
#include "cache_attend.cuh"
#include "cache_format.cuh"
#include "cache_io.cuh"
#include "cache_pages.cuh"

using namespace samb200;

namespace {

bool geometry_ok(int32_t page_tokens, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim) {
    return page_tokens >= 16 && page_tokens <= 1024 && (page_tokens & (page_tokens - 1)) == 0 && n_layers >= 1 && n_layers <= 65536 &&
           n_kv_heads >= 1 && n_kv_heads <= 1024 && (head_dim == 64 || head_dim == 128);
}

constexpr int64_t kLargest = int64_t(1) << 30;   // positions of a stream, entries of the table, query rows of a stream

int check_cache(const sam_cache* c) {
    if (!c || !geometry_ok(c->page_tokens, c->n_layers, c->n_kv_heads, c->head_dim)) return SAM_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->n_streams < 1 || c->max_pages < 1) return SAM_ERR_INVALID_ARG;
    // positions of new tokens, sums of pages over rows and their tags are 32-bit numbers in the kernels
    if (static_cast<int64_t>(c->max_pages) * c->page_tokens > kLargest || static_cast<int64_t>(c->max_pages) * c->n_streams > kLargest)
        return SAM_ERR_INVALID_ARG;
    if (c->k_exp < -24 || c->k_exp > 24 || c->v_exp < -24 || c->v_exp > 24) return SAM_ERR_INVALID_ARG;
    if (!c->page_table || !c->seq_len) return SAM_ERR_INVALID_ARG;
    return SAM_OK;
}

int check_pages(const sam_cache* c) {
    return c->pages && aligned(c->pages, 128) ? SAM_OK : SAM_ERR_INVALID_ARG;
}

// The calls that keep the books need all of them, and scratch.
int check_books(const sam_cache* c) {
    if (int e = check_cache(c)) return e;
    if (!c->ref_count || !c->free_list || !c->meta || !c->scratch || !aligned(c->scratch, 16)) return SAM_ERR_INVALID_ARG;
    return c->scratch_bytes < sam_cache_scratch_bytes(c->n_streams, c->n_pages) ? SAM_ERR_TOO_SMALL : SAM_OK;
}

CacheView view(const sam_cache* c) {
    CacheView v;
    v.pages = static_cast<uint8_t*>(c->pages);
    v.table = c->page_table;
    v.seq_len = c->seq_len;
    v.ref = c->ref_count;
    v.free_list = c->free_list;
    v.meta = c->meta;
    v.scratch = static_cast<int32_t*>(c->scratch);
    v.page_bytes = sam_cache_page_bytes(c->page_tokens, c->n_layers, c->n_kv_heads, c->head_dim);
    v.n_pages = c->n_pages;
    v.n_streams = c->n_streams;
    v.max_pages = c->max_pages;
    v.n_layers = c->n_layers;
    v.n_kv = c->n_kv_heads;
    v.D = c->head_dim;
    v.log_p = 0;
    while ((1 << v.log_p) < c->page_tokens) ++v.log_p;
    v.k_exp = c->k_exp;
    v.v_exp = c->v_exp;
    return v;
}

int launched() {
    SAM_CUDA(cudaGetLastError());
    ++g_launches;
    return SAM_OK;
}

int copy_grid(int64_t pages, int64_t page_bytes, int* grid) {
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    *grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(pages * ((page_bytes + kCopyPiece - 1) / kCopyPiece), di.sms * 8)));
    return SAM_OK;
}

// Grid of append and read, and the multiplier that divides by the blocks of a token.
dim3 io_grid(const CacheView& v, int32_t B, int32_t Q, uint32_t* magic) {
    const int64_t per_token = static_cast<int64_t>(v.n_kv) * (v.D / 16);
    *magic = static_cast<uint32_t>(((int64_t(1) << 32) + per_token - 1) / per_token);
    const int64_t blocks = (Q * per_token + kIoThreads * kIoBlocks - 1) / (kIoThreads * kIoBlocks);
    return dim3(static_cast<unsigned>(blocks), B, 2);
}

template <typename T>
int launch_append(const CacheView& v, int32_t layer, const void* k, const void* vv, KvStrides st, int32_t B, int32_t Q,
                  const int32_t* streams, const int32_t* n_new, cudaStream_t s) {
    const bool wide = aligned(k, 16) && aligned(vv, 16) && st.row % 8 == 0 && st.token % 8 == 0 && st.head % 8 == 0;
    uint32_t magic;
    const dim3 grid = io_grid(v, B, Q, &magic);
    append_kernel<T><<<grid, kIoThreads, 0, s>>>(v, layer, static_cast<const T*>(k), static_cast<const T*>(vv), st, wide, Q, magic, streams, n_new);
    return launched();
}

template <typename T>
int launch_read(const CacheView& v, int32_t layer, int32_t B, int32_t Q, const int32_t* streams, const int32_t* first,
                const int32_t* n, void* k, void* vv, cudaStream_t s) {
    uint32_t magic;
    const dim3 grid = io_grid(v, B, Q, &magic);
    read_kernel<T><<<grid, kIoThreads, 0, s>>>(v, layer, Q, magic, streams, first, n, static_cast<T*>(k), static_cast<T*>(vv));
    return launched();
}

// Workspace of sam_cache_attend: arrival counters (zero between calls), then partial results of up to kMaxCtas CTAs.
constexpr int kMaxCtas = 512;
constexpr int64_t kCounterBytes = kMaxCtas * 4;
constexpr int64_t kNarrowRows = 32;   // query rows per key/value head up to which the streaming kernel is used

template <int D>
int64_t partial_bytes(int64_t rows) {
    if (rows <= kNarrowRows) return 2ll * kMaxCtas * 4 * StreamPlan<D, 2>::kPiece;
    return 2ll * kWideMaxCtas * 4 * WidePlan<D>::kPart;
}

// Dynamic shared memory above the default has to be asked for once per kernel and device.
template <typename K>
int allow_shared(K* kernel, int bytes, uint64_t* asked) {   // asked: the kernel's own, one bit per device
    int dev = 0;
    SAM_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (*asked & bit) return SAM_OK;
    SAM_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    *asked |= bit;
    return SAM_OK;
}

template <typename T, int D, int NT>
int launch_stream(const AttendArgs& a, int sms, cudaStream_t s) {
    using Plan = StreamPlan<D, NT>;
    static thread_local uint64_t asked = 0;
    if (int e = allow_shared(attend_stream_kernel<T, D, NT>, Plan::kSmem, &asked)) return e;
    attend_stream_kernel<T, D, NT><<<std::min(sms * Plan::kCtasPerSm, kMaxCtas), kStreamThreads, Plan::kSmem, s>>>(a);
    return launched();
}

template <typename T, int D>
int launch_wide(const AttendArgs& a, int sms, cudaStream_t s) {
    using Plan = WidePlan<D>;
    static thread_local uint64_t asked = 0;
    if (int e = allow_shared(attend_wide_kernel<T, D>, Plan::kSmem, &asked)) return e;
    attend_wide_kernel<T, D><<<std::min(sms, kWideMaxCtas), kWideThreads, Plan::kSmem, s>>>(a);
    return launched();
}

template <typename T, int D>
int launch_attend(const AttendArgs& a, cudaStream_t s) {
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    const int64_t rows = static_cast<int64_t>(a.Q) * a.group;
    if (rows <= 8) return launch_stream<T, D, 1>(a, di.sms, s);
    if (rows <= kNarrowRows) return launch_stream<T, D, 2>(a, di.sms, s);
    return launch_wide<T, D>(a, di.sms, s);
}

}  // namespace

extern "C" {

int64_t sam_cache_page_bytes(int32_t page_tokens, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim) {
    if (!geometry_ok(page_tokens, n_layers, n_kv_heads, head_dim)) return SAM_ERR_INVALID_ARG;
    return static_cast<int64_t>(n_layers) * n_kv_heads * (page_tokens / 16) * 18 * head_dim;
}

int64_t sam_cache_scratch_bytes(int32_t n_streams, int32_t n_pages) {
    if (n_streams < 1 || n_pages < 1) return SAM_ERR_INVALID_ARG;
    return page_scratch_ints(n_streams, n_pages) * 4;
}

int sam_cache_init(const sam_cache* c, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    cache_init_kernel<<<512, 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(view(c));
    return launched();
}

int sam_cache_status(const sam_cache* c, int32_t* n_free, int32_t* status, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int32_t both[2];
    SAM_CUDA(cudaMemcpyAsync(both, c->meta, sizeof(both), cudaMemcpyDeviceToHost, s));
    SAM_CUDA(cudaStreamSynchronize(s));
    if (n_free) *n_free = both[0];
    if (status) *status = both[1];
    return SAM_OK;
}

int sam_cache_reserve(const sam_cache* c, int32_t B, const int32_t* streams, const int32_t* n_new, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    if (int e = check_pages(c)) return e;
    if (B < 0) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B) return SAM_ERR_TOO_LARGE;
    if (B == 0) return SAM_OK;
    if (B > c->n_streams || !n_new) return SAM_ERR_INVALID_ARG;
    const CacheView v = view(c);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int grid;
    if (int e = copy_grid(B, v.page_bytes, &grid)) return e;
    reserve_kernel<<<1, kPageThreads, 0, s>>>(v, B, streams, n_new);
    if (int e = launched()) return e;
    const int64_t list = std::max(v.n_streams, v.n_pages);
    const int32_t* from = v.scratch + kScratchHead + 3ll * v.n_streams;
    copy_pages_kernel<<<grid, kCopyThreads, 0, s>>>(v.pages, v.pages, v.page_bytes, v.n_pages, v.n_pages, v.scratch, 0, from, from + list);
    return launched();
}

int sam_cache_commit(const sam_cache* c, int32_t B, const int32_t* streams, const int32_t* n_keep, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    if (B < 0) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B) return SAM_ERR_TOO_LARGE;
    if (B == 0) return SAM_OK;
    if (B > c->n_streams || !n_keep) return SAM_ERR_INVALID_ARG;
    commit_kernel<<<1, kPageThreads, (B + 1) * 4, static_cast<cudaStream_t>(cuda_stream)>>>(view(c), B, streams, n_keep);
    return launched();
}

int sam_cache_fork(const sam_cache* c, int32_t n, const int32_t* src, const int32_t* dst, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    if (n < 0) return SAM_ERR_INVALID_ARG;
    if (n == 0) return SAM_OK;
    if (n > c->n_streams || !src || !dst) return SAM_ERR_INVALID_ARG;
    fork_kernel<<<n, 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(view(c), src, dst);
    return launched();
}

int sam_cache_compact(const sam_cache* c, void* cuda_stream) {
    if (int e = check_books(c)) return e;
    if (int e = check_pages(c)) return e;
    const CacheView v = view(c);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int grid;
    if (int e = copy_grid(v.n_pages, v.page_bytes, &grid)) return e;
    compact_plan_kernel<<<1, kPageThreads, 0, s>>>(v);
    if (int e = launched()) return e;
    const int64_t list = std::max(v.n_streams, v.n_pages);
    const int32_t* from = v.scratch + kScratchHead + 3ll * v.n_streams;
    copy_pages_kernel<<<grid, kCopyThreads, 0, s>>>(v.pages, v.pages, v.page_bytes, v.n_pages, v.n_pages, v.scratch, 0, from, from + list);
    if (int e = launched()) return e;
    compact_tables_kernel<<<512, 256, 0, s>>>(v);
    return launched();
}

int sam_cache_copy_pages(const sam_cache* src, const sam_cache* dst, int32_t n, const int32_t* from, const int32_t* to, void* cuda_stream) {
    if (int e = check_cache(src)) return e;
    if (int e = check_cache(dst)) return e;
    if (int e = check_pages(src)) return e;
    if (int e = check_pages(dst)) return e;
    if (src->page_tokens != dst->page_tokens || src->n_layers != dst->n_layers || src->n_kv_heads != dst->n_kv_heads ||
        src->head_dim != dst->head_dim || src->k_exp != dst->k_exp || src->v_exp != dst->v_exp || n < 0)
        return SAM_ERR_INVALID_ARG;
    if (n == 0) return SAM_OK;
    if (!from || !to) return SAM_ERR_INVALID_ARG;
    const CacheView v = view(src);
    int grid;
    if (int e = copy_grid(n, v.page_bytes, &grid)) return e;
    copy_pages_kernel<<<grid, kCopyThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        v.pages, static_cast<uint8_t*>(dst->pages), v.page_bytes, src->n_pages, dst->n_pages, nullptr, n, from, to);
    return launched();
}

int sam_cache_append(const sam_cache* c, int32_t layer, const void* k, const void* v, int32_t dtype, int64_t row_stride,
                     int64_t token_stride, int64_t head_stride, int32_t B, int32_t Q, const int32_t* streams,
                     const int32_t* n_new, void* cuda_stream) {
    if (int e = check_cache(c)) return e;
    if (int e = check_pages(c)) return e;
    if (layer < 0 || layer >= c->n_layers || B < 0 || Q < 0 || (dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16)) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B) return SAM_ERR_TOO_LARGE;
    if (B == 0 || Q == 0) return SAM_OK;
    if (static_cast<int64_t>(Q) * c->n_kv_heads >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
    if (!k || !v || !aligned(k, 2) || !aligned(v, 2) || (!streams && B > c->n_streams)) return SAM_ERR_INVALID_ARG;
    const KvStrides st{row_stride, token_stride, head_stride};
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SAM_CACHE_BF16 ? launch_append<__nv_bfloat16>(view(c), layer, k, v, st, B, Q, streams, n_new, s)
                                   : launch_append<__half>(view(c), layer, k, v, st, B, Q, streams, n_new, s);
}

int sam_cache_read(const sam_cache* c, int32_t layer, int32_t B, int32_t Q, const int32_t* streams, const int32_t* first,
                   const int32_t* n, void* k_out, void* v_out, int32_t dtype, void* cuda_stream) {
    if (int e = check_cache(c)) return e;
    if (int e = check_pages(c)) return e;
    if (layer < 0 || layer >= c->n_layers || B < 0 || Q < 0 || (dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16)) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B) return SAM_ERR_TOO_LARGE;
    if (B == 0 || Q == 0) return SAM_OK;
    if (static_cast<int64_t>(Q) * c->n_kv_heads >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || (!streams && B > c->n_streams)) return SAM_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SAM_CACHE_BF16 ? launch_read<__nv_bfloat16>(view(c), layer, B, Q, streams, first, n, k_out, v_out, s)
                                   : launch_read<__half>(view(c), layer, B, Q, streams, first, n, k_out, v_out, s);
}

int64_t sam_cache_attend_workspace_bytes(const sam_cache* c, int32_t B, int32_t Q, int32_t H) {
    if (int e = check_cache(c)) return e;
    if (B < 0 || Q < 0 || H < 1 || H % c->n_kv_heads) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B) return SAM_ERR_TOO_LARGE;
    const int64_t rows = static_cast<int64_t>(Q) * (H / c->n_kv_heads);
    return kCounterBytes + (c->head_dim == 64 ? partial_bytes<64>(rows) : partial_bytes<128>(rows));
}

int sam_cache_attend(const sam_cache* c, int32_t layer, const void* q, int32_t dtype, int64_t q_row_stride, int64_t q_token_stride,
                     int64_t q_head_stride, int32_t B, int32_t Q, int32_t H, const int32_t* streams, const int32_t* n_new, float scale,
                     int32_t window, void* out, int64_t out_row_stride, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                     void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (int e = check_cache(c)) return e;
    if (int e = check_pages(c)) return e;
    if (layer < 0 || layer >= c->n_layers || window < 0 || !std::isfinite(scale) || (dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16)) return SAM_ERR_INVALID_ARG;
    const int64_t need = sam_cache_attend_workspace_bytes(c, B, Q, H);
    if (need < 0) return static_cast<int>(need);
    if (B == 0 || Q == 0) return SAM_OK;
    if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4) || !workspace || !aligned(workspace, 256) || (!streams && B > c->n_streams))
        return SAM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SAM_ERR_TOO_SMALL;
    if (Q > kLargest || static_cast<int64_t>(B) * Q * H >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
    AttendArgs a;
    a.c = view(c);
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.streams = streams;
    a.n_new = n_new;
    a.q_row = q_row_stride;
    a.q_token = q_token_stride;
    a.q_head = q_head_stride;
    a.o_row = out_row_stride;
    a.o_token = out_token_stride;
    a.o_head = out_head_stride;
    a.layer = layer;
    a.B = B;
    a.Q = Q;
    a.H = H;
    a.window = window;
    a.group = H / c->n_kv_heads;
    a.scale = scale;
    a.q_wide = aligned(q, 16) && (q_row_stride | q_token_stride | q_head_stride) % 8 == 0;
    a.o_wide = aligned(out, 16) && (out_row_stride | out_token_stride | out_head_stride) % 8 == 0;
    a.counters = static_cast<int32_t*>(workspace);
    a.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = dtype == SAM_CACHE_BF16;
    if (c->head_dim == 64) return bf16 ? launch_attend<__nv_bfloat16, 64>(a, s) : launch_attend<__half, 64>(a, s);
    return bf16 ? launch_attend<__nv_bfloat16, 128>(a, s) : launch_attend<__half, 128>(a, s);
}

}  // extern "C"
