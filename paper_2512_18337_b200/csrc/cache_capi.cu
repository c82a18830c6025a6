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
#include "cache_rotate.cuh"
#include "cache_select.cuh"

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
constexpr int64_t kSplitRows = 8;     // with many lists also for up to so many behind the wide kernel's last full tile

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

template <typename T, int D, int NT, bool kListed>
int launch_stream(const AttendArgs& a, int sms, cudaStream_t s, bool behind_wide = false) {
    using Plan = StreamPlan<D, NT>;
    static thread_local uint64_t asked = 0;
    if (int e = allow_shared(attend_stream_kernel<T, D, NT, kListed>, Plan::kSmem, &asked)) return e;
    const int grid = std::min(sms * Plan::kCtasPerSm, kMaxCtas);
    if (behind_wide) return launch_behind(attend_stream_kernel<T, D, NT, kListed>, grid, kStreamThreads, Plan::kSmem, s, a);
    attend_stream_kernel<T, D, NT, kListed><<<grid, kStreamThreads, Plan::kSmem, s>>>(a);
    return launched();
}

template <typename T, int D, bool kListed>
int launch_wide(const AttendArgs& a, int sms, cudaStream_t s) {
    using Plan = WidePlan<D>;
    static thread_local uint64_t asked = 0;
    if (int e = allow_shared(attend_wide_kernel<T, D, kListed>, Plan::kSmem, &asked)) return e;
    attend_wide_kernel<T, D, kListed><<<std::min(sms, kWideMaxCtas), kWideThreads, Plan::kSmem, s>>>(a);
    return launched();
}

template <typename T, int D>
int launch_attend(const AttendArgs& a, cudaStream_t s) {
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    const int64_t rows = static_cast<int64_t>(a.Q) * a.group;
    if (rows <= 8) return launch_stream<T, D, 1, false>(a, di.sms, s);
    if (rows <= kNarrowRows) return launch_stream<T, D, 2, false>(a, di.sms, s);
    return launch_wide<T, D, false>(a, di.sms, s);
}

template <typename T, int D>
int launch_attend_blocks(AttendArgs a, cudaStream_t s) {
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    // What a row tile of the wide kernel costs does not depend on how full it is; up to eight rows behind the last full one take
    // the streaming kernel less, which is placed while the other one ends, once there is more than one list and head for every two SMs: with fewer
    // the tile runs beside the full ones on SMs that would idle.  (Proposals of 17, 64/8 heads, lists of 2,048 positions: 48 streams 155 against 182
    // us, 24 101 against 105, 16 81 against 79, 8 65 against 52; of 256 positions: 48 streams 63 against 67, 12 31 against 33, 8 31 against 24.  Proposals of 33, which
    // have three tiles: 48 streams 232 against 252, 8 74 against 67.  Sixteen rows behind the tile, 48 streams: 168 against 184, and 149 against 144 with 12 to 17 tokens a stream.)
    const int64_t rows = static_cast<int64_t>(a.share) * a.group, rest = rows % kWideRows;
    a.row0 = 0;
    a.row1 = static_cast<int32_t>(rows);
    if (rows > kNarrowRows) {
        if (rest <= kSplitRows && 2 * static_cast<int64_t>(a.runs) * a.c.n_kv > di.sms) a.row1 -= static_cast<int32_t>(rest);
        if (int e = launch_wide<T, D, true>(a, di.sms, s)) return e;
        if (a.row1 == rows) return SAM_OK;
        a.row0 = a.row1;
        a.row1 = static_cast<int32_t>(rows);
    }
    const bool behind_wide = a.row0 > 0;
    return a.row1 - a.row0 <= 8 ? launch_stream<T, D, 1, true>(a, di.sms, s, behind_wide) : launch_stream<T, D, 2, true>(a, di.sms, s, behind_wide);
}

template <int kTeam, int kKeys>
int launch_pick(const SelectArgs& a, int64_t rows, cudaStream_t s) {
    constexpr int kLists = kPickThreads / kTeam;
    return launch_behind(select_pick_kernel<kTeam, kKeys>, static_cast<unsigned>((rows + kLists - 1) / kLists), kPickThreads, 0, s, a, rows);
}

int64_t key_stride(const sam_cache* c) { return (static_cast<int64_t>(c->max_pages) + 3) & ~int64_t(3); }
constexpr int64_t kKeyBytes = int64_t(128) << 20;   // of the keys that are in flight at a time, where there are as many

// Most lists of a row that are scored together: their keys are there together.
int64_t most_team(const sam_cache* c, int64_t lists) {
    return std::max<int64_t>(std::min({lists, int64_t(kScoreTeam), kKeyBytes / (c->n_kv_heads * key_stride(c) * 4)}), 1);
}

// Lists of a row that one block scores: as many as fit its columns; one where the rows of a single list are few and lists are, too.
int32_t select_team(const sam_cache* c, int64_t lists, int64_t rows) {
    return static_cast<int32_t>(std::min<int64_t>(std::max<int64_t>(kScoreColumns / ((rows + 7) / 8 * 8), 1), most_team(c, lists)));
}

template <typename T, int D>
int launch_score(const SelectArgs& a, int64_t n, int sms, cudaStream_t s) {
    const int64_t padded = (static_cast<int64_t>(a.share) * a.group + 7) / 8 * 8, heads = n * a.c.n_kv;
    auto shares = [&](int pages, int blocks) {            // of the pages: so that there are about so many blocks an SM
        return static_cast<unsigned>(std::max<int64_t>(std::min<int64_t>((a.c.max_pages + pages - 1) / pages, (static_cast<int64_t>(sms) * blocks + heads / 2) / heads), 1));
    };
    if (a.team == 1 && padded <= kFewColumns) {
        // streams differ in length, and a block begins quickly
        return launch_behind(select_score_few_kernel<T, D>, dim3(shares(kFewThreads / 2, 8), a.c.n_kv, static_cast<unsigned>(n)), kFewThreads, 0, s, a);
    }
    // A block takes 7 us for its queries before it begins: about as many of them as run at a time, to the nearest share.  (Rounded down, so that they all do: 48 proposals
    // of 17, 28/4 heads, contexts of 6,000 to 12,000 34.5 -> 32.9 us, but of 1,200 to 12,000, which more blocks even out, 39.2 -> 41.0; 176 list teams and heads 55.8 -> 58.8.)
    const dim3 grid(shares(kScorePages, 2), a.c.n_kv, static_cast<unsigned>(n));
    static thread_local uint64_t asked = 0;
    if (int e = allow_shared(select_score_kernel<T, D>, score_smem<D>(kScoreColumns), &asked)) return e;
    const int columns = static_cast<int>((std::min<int64_t>(a.team * padded, kScoreColumns) + 15) / 16 * 16);
    return launch_behind(select_score_kernel<T, D>, grid, kScoreThreads, score_smem<D>(columns), s, a);
}

// Scores and picks for all lists, as many at a time as the keys have room for.
template <typename T>
int launch_select(SelectArgs a, int64_t key_bytes, int sms, cudaStream_t s) {
    const int64_t all = static_cast<int64_t>(a.B) * a.teams, each = a.team * a.c.n_kv * a.key_stride * 4;   // bytes of a team's keys
    const int64_t most = std::min<int64_t>(std::max<int64_t>(key_bytes / each, 1), 65535);
    for (int64_t at = 0; at < all; at += most) {
        const int64_t n = std::min(all - at, most);
        a.first_team = at;
        if (int e = a.c.D == 64 ? launch_score<T, 64>(a, n, sms, s) : launch_score<T, 128>(a, n, sms, s)) return e;
        const int64_t rows = n * a.team * a.c.n_kv;
        // a warp a list where there are many short ones; a block a list takes less time for each
        const bool many = rows > sms * 8;
        const int e = many && a.c.max_pages <= 512    ? launch_pick<32, 16>(a, rows, s)
                      : many && a.c.max_pages <= 1024 ? launch_pick<32, 32>(a, rows, s)
                      : a.c.max_pages <= 1024         ? launch_pick<256, 4>(a, rows, s)
                      : a.c.max_pages <= 4096         ? launch_pick<256, 16>(a, rows, s)
                      : a.c.max_pages <= 16384        ? launch_pick<256, 64>(a, rows, s)
                                                      : launch_pick<256, 0>(a, rows, s);
        if (e) return e;
    }
    return SAM_OK;
}

int check_layer_call(const sam_cache* c, int32_t layer, int32_t B, int32_t Q, const int32_t* streams) {
    if (int e = check_cache(c)) return e;
    if (int e = check_pages(c)) return e;
    if (layer < 0 || layer >= c->n_layers || B < 0 || Q < 0) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B || Q > kLargest) return SAM_ERR_TOO_LARGE;
    return !streams && B > c->n_streams ? SAM_ERR_INVALID_ARG : SAM_OK;
}

int check_bounds(const int8_t* codes, const int8_t* exps) { return codes && exps && aligned(codes, 16) ? SAM_OK : SAM_ERR_INVALID_ARG; }

// f / 2 pi modulo 1 in units of 2^-64, to nearest; |f| < 2^20.  f is m 2^e with a whole number m below 2^53, 1 / 2 pi stands here in 192 bits: their
// product is a whole number below 2^243, of which the lowest 128 - e bits lie behind the unit.
uint64_t turns_of(double f) {
    constexpr uint64_t kInverse[3] = {0x36d8a5664f10e410u, 0x7f09d5f47d4d3770u, 0x28be60db9391054au};   // lowest first
    int exponent;
    const uint64_t m = static_cast<uint64_t>(std::ldexp(std::frexp(std::fabs(f), &exponent), 53));
    const int behind = 128 - (exponent - 53);              // 161 or more
    if (behind > 255) return 0;                            // less than half a unit
    uint64_t product[5] = {0, 0, 0, 0, 0};
    unsigned __int128 carry = 0;
    for (int i = 0; i < 3; ++i) {
        carry += static_cast<unsigned __int128>(m) * kInverse[i];
        product[i] = static_cast<uint64_t>(carry);
        carry >>= 64;
    }
    product[3] = static_cast<uint64_t>(carry);
    carry = uint64_t(1) << ((behind - 1) & 63);            // half a unit
    for (int i = (behind - 1) >> 6; i < 4; ++i) {
        carry += product[i];
        product[i] = static_cast<uint64_t>(carry);
        carry >>= 64;
    }
    const int word = behind >> 6, bit = behind & 63;       // the product stays below 2^256: product[4] is zero
    const uint64_t turns = product[word] >> bit | (bit ? product[word + 1] << (64 - bit) : 0);
    return f < 0 ? 0 - turns : turns;
}

template <typename T>
int launch_turn(const TurnArgs& a, cudaStream_t s) {
    const dim3 grid((a.Q + a.tokens - 1) / a.tokens, a.B);
    if (a.c.D == 64) append_rotated_kernel<T, 64><<<grid, kTurnThreads, 0, s>>>(a);
    else append_rotated_kernel<T, 128><<<grid, kTurnThreads, 0, s>>>(a);
    return launched();
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
    a.blocks = nullptr;
    a.runs = B;
    a.lists = 1;
    a.share = Q;
    a.n_blocks = a.row0 = a.row1 = 0;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = dtype == SAM_CACHE_BF16;
    if (c->head_dim == 64) return bf16 ? launch_attend<__nv_bfloat16, 64>(a, s) : launch_attend<__half, 64>(a, s);
    return bf16 ? launch_attend<__nv_bfloat16, 128>(a, s) : launch_attend<__half, 128>(a, s);
}

int64_t sam_cache_attend_blocks_workspace_bytes(const sam_cache* c, int32_t B, int32_t Q, int32_t H, int32_t share) {
    return share < 1 ? SAM_ERR_INVALID_ARG : sam_cache_attend_workspace_bytes(c, B, std::min(Q, share), H);
}

int sam_cache_attend_blocks(const sam_cache* c, int32_t layer, const void* q, int32_t dtype, int64_t q_row_stride, int64_t q_token_stride,
                            int64_t q_head_stride, int32_t B, int32_t Q, int32_t H, const int32_t* streams, const int32_t* n_new,
                            const int32_t* blocks, int32_t n_blocks, int32_t share, float scale, void* out, int64_t out_row_stride,
                            int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    if (int e = check_layer_call(c, layer, B, Q, streams)) return e;
    if (n_blocks < 1 || !std::isfinite(scale) || (dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16)) return SAM_ERR_INVALID_ARG;
    const int64_t need = sam_cache_attend_blocks_workspace_bytes(c, B, Q, H, share);
    if (need < 0) return static_cast<int>(need);
    if (B == 0 || Q == 0) return SAM_OK;
    if (!q || !out || !blocks || !aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4) || !aligned(blocks, 4) || !workspace || !aligned(workspace, 256))
        return SAM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SAM_ERR_TOO_SMALL;
    if (static_cast<int64_t>(B) * Q * H >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
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
    a.window = 0;
    a.group = H / c->n_kv_heads;
    a.scale = scale;
    a.q_wide = aligned(q, 16) && (q_row_stride | q_token_stride | q_head_stride) % 8 == 0;
    a.o_wide = aligned(out, 16) && (out_row_stride | out_token_stride | out_head_stride) % 8 == 0;
    a.counters = static_cast<int32_t*>(workspace);
    a.partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
    a.blocks = blocks;
    a.share = std::min(share, Q);
    a.lists = (Q - 1) / a.share + 1;
    a.runs = B * a.lists;
    a.n_blocks = n_blocks;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = dtype == SAM_CACHE_BF16;
    if (c->head_dim == 64) return bf16 ? launch_attend_blocks<__nv_bfloat16, 64>(a, s) : launch_attend_blocks<__half, 64>(a, s);
    return bf16 ? launch_attend_blocks<__nv_bfloat16, 128>(a, s) : launch_attend_blocks<__half, 128>(a, s);
}

int sam_rope_turns(const double* inv_freq, int32_t n, uint64_t* turns) {
    if (n < 1 || n > 64 || !inv_freq || !turns) return SAM_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (!std::isfinite(inv_freq[i]) || std::fabs(inv_freq[i]) > 1e6) return SAM_ERR_INVALID_ARG;
        turns[i] = turns_of(inv_freq[i]);
    }
    return SAM_OK;
}

int sam_cache_append_rotated(const sam_cache* c, int32_t layer, const void* q, int64_t q_row_stride, int64_t q_token_stride, int64_t q_head_stride,
                             const void* k, const void* v, int64_t row_stride, int64_t token_stride, int64_t head_stride, void* q_out,
                             int64_t out_row_stride, int64_t out_token_stride, int64_t out_head_stride, int32_t dtype, const sam_rope* rope, int32_t B,
                             int32_t Q, int32_t H, const int32_t* streams, const int32_t* n_new, const int32_t* positions, void* cuda_stream) {
    if (int e = check_layer_call(c, layer, B, Q, streams)) return e;
    if (dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16) return SAM_ERR_INVALID_ARG;
    if (!rope || !rope->turns || !aligned(rope->turns, 8) || rope->rotary_dim < 32 || rope->rotary_dim > c->head_dim || rope->rotary_dim % 32 ||
        !std::isfinite(rope->factor) || H < 0)
        return SAM_ERR_INVALID_ARG;
    if (H > 16384 || static_cast<int64_t>(Q) * B >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
    if (B == 0 || Q == 0) return SAM_OK;
    if (!k || !v || !aligned(k, 2) || !aligned(v, 2) || (H > 0 && (!q || !q_out || !aligned(q, 2) || !aligned(q_out, 2))) || !aligned(positions, 4))
        return SAM_ERR_INVALID_ARG;
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    TurnArgs a;
    a.c = view(c);
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.qs = KvStrides{q_row_stride, q_token_stride, q_head_stride};
    a.ks = KvStrides{row_stride, token_stride, head_stride};
    a.os = KvStrides{out_row_stride, out_token_stride, out_head_stride};
    a.turns = rope->turns;
    a.positions = positions;
    a.streams = streams;
    a.n_new = n_new;
    a.factor = rope->factor;
    a.layer = layer;
    a.B = B;
    a.Q = Q;
    a.H = H;
    a.rotary = rope->rotary_dim;
    a.interleaved = rope->interleaved != 0;
    // more tokens share a CTA once there are enough CTAs; unit numbers stay below 2^16, where the multiplier divides exactly
    const int32_t heads = H + 2 * c->n_kv_heads;
    a.tokens = static_cast<int32_t>(std::min<int64_t>({int64_t(kTurnTokens), std::max<int64_t>(1, static_cast<int64_t>(B) * Q / (di.sms * 32)), 65535 / heads}));
    a.magic = static_cast<uint32_t>(((int64_t(1) << 32) + heads - 1) / heads);
    auto wide = [](const void* p, const KvStrides& t) { return aligned(p, 16) && (t.row | t.token | t.head) % 8 == 0; };
    a.q_wide = wide(q, a.qs);
    a.k_wide = wide(k, a.ks) && aligned(v, 16);
    a.o_wide = wide(q_out, a.os);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SAM_CACHE_BF16 ? launch_turn<__nv_bfloat16>(a, s) : launch_turn<__half>(a, s);
}

int sam_cache_bounds_update(const sam_cache* c, int32_t layer, int8_t* codes, int8_t* exps, int32_t B, int32_t Q, const int32_t* streams,
                            const int32_t* n_new, void* cuda_stream) {
    if (int e = check_layer_call(c, layer, B, Q, streams)) return e;
    if (int e = check_bounds(codes, exps)) return e;
    if (B == 0 || Q == 0) return SAM_OK;
    const CacheView v = view(c);
    const unsigned pages = static_cast<unsigned>(std::min<int64_t>(Q / c->page_tokens + 1, 1024));
    bounds_update_kernel<<<dim3(c->n_kv_heads, B, pages), kBoundThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(v, BoundsView{codes, exps}, layer, Q, streams, n_new);
    return launched();
}

int sam_cache_bounds_rebuild(const sam_cache* c, int8_t* codes, int8_t* exps, int32_t n, const int32_t* pages, void* cuda_stream) {
    if (int e = check_cache(c)) return e;
    if (int e = check_pages(c)) return e;
    if (int e = check_bounds(codes, exps)) return e;
    if (n < 0 || (!pages && n > c->n_pages)) return SAM_ERR_INVALID_ARG;
    if (n == 0) return SAM_OK;
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    const int64_t all = static_cast<int64_t>(n) * c->n_layers * c->n_kv_heads;
    bounds_rebuild_kernel<<<static_cast<unsigned>(std::min<int64_t>(all, di.sms * 16)), kBoundThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        view(c), BoundsView{codes, exps}, n, pages);
    return launched();
}

int64_t sam_cache_select_workspace_bytes(const sam_cache* c, int32_t B, int32_t Q, int32_t share) {
    if (int e = check_cache(c)) return e;
    if (B < 0 || Q < 0 || share < 1) return SAM_ERR_INVALID_ARG;
    if (B > SAM_CACHE_MAX_B || Q > kLargest) return SAM_ERR_TOO_LARGE;
    // the last team of a row may be short of lists
    const int64_t each = static_cast<int64_t>(c->n_kv_heads) * key_stride(c) * 4, lists = (static_cast<int64_t>(Q) + share - 1) / share;
    return std::max<int64_t>(std::min(B * (lists + most_team(c, lists) - 1) * each, kKeyBytes), each);
}

int sam_cache_select(const sam_cache* c, int32_t layer, const int8_t* codes, const int8_t* exps, const void* q, int32_t dtype, int64_t q_row_stride,
                     int64_t q_token_stride, int64_t q_head_stride, int32_t B, int32_t Q, int32_t H, const int32_t* streams, const int32_t* n_new,
                     int32_t share, int32_t n_sink, int32_t n_recent, int32_t* blocks, int32_t n_blocks, void* workspace, int64_t workspace_bytes,
                     void* cuda_stream) {
    if (int e = check_layer_call(c, layer, B, Q, streams)) return e;
    if (int e = check_bounds(codes, exps)) return e;
    if ((dtype != SAM_CACHE_BF16 && dtype != SAM_CACHE_FP16) || H < 1 || H % c->n_kv_heads || share < 1 || n_sink < 0 || n_recent < 1 || n_blocks < 1)
        return SAM_ERR_INVALID_ARG;
    if (B == 0 || Q == 0) return SAM_OK;
    share = std::min(share, Q);
    // what is listed whatever its score has to fit: a run of `share` tokens lies in up to (share - 2) / page_tokens + 2 blocks
    const int64_t own = share == 1 ? 1 : (static_cast<int64_t>(share) - 2) / c->page_tokens + 2;
    if (static_cast<int64_t>(n_sink) + n_recent - 1 + own > n_blocks) return SAM_ERR_INVALID_ARG;
    const int64_t need = sam_cache_select_workspace_bytes(c, B, Q, share), lists = (static_cast<int64_t>(Q) - 1) / share + 1;
    if (!q || !aligned(q, 2) || !blocks || !aligned(blocks, 4) || !workspace || !aligned(workspace, 256)) return SAM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SAM_ERR_TOO_SMALL;
    if (static_cast<int64_t>(B) * Q * H >= (int64_t(1) << 31)) return SAM_ERR_TOO_LARGE;
    SelectArgs a;
    a.c = view(c);
    a.o = BoundsView{const_cast<int8_t*>(codes), const_cast<int8_t*>(exps)};
    a.q = q;
    a.streams = streams;
    a.n_new = n_new;
    a.q_row = q_row_stride;
    a.q_token = q_token_stride;
    a.q_head = q_head_stride;
    a.layer = layer;
    a.B = B;
    a.Q = Q;
    a.H = H;
    a.group = H / c->n_kv_heads;
    a.lists = static_cast<int32_t>(lists);
    a.share = share;
    a.n_blocks = n_blocks;
    a.n_sink = n_sink;
    a.n_recent = n_recent;
    DeviceInfo di;
    if (int e = device_info(&di)) return e;
    a.team = select_team(c, lists, static_cast<int64_t>(share) * a.group);
    a.teams = static_cast<int32_t>((lists + a.team - 1) / a.team);
    a.key_stride = key_stride(c);
    a.keys = static_cast<uint32_t*>(workspace);
    a.out = blocks;
    a.q_wide = aligned(q, 16) && (q_row_stride | q_token_stride | q_head_stride) % 8 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SAM_CACHE_BF16 ? launch_select<__nv_bfloat16>(a, workspace_bytes, di.sms, s) : launch_select<__half>(a, workspace_bytes, di.sms, s);
}

}  // extern "C"
