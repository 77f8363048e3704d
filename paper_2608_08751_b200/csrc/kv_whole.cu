// Host side of the operators on whole paged caches: attention over all of a request's pages, and the pages' life (fork, compact,
// copy).  Argument checks before any CUDA call, then the launches.
#include "../../include/ivf_b200.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <limits>
#include <type_traits>
#include <utility>

#include "kv_chunk.cuh"
#include "kv_chunk_tile.cuh"
#include "kv_host.cuh"
#include "kv_pages.cuh"

namespace {

using namespace ivf;

int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return kv_host_fail(code, buf);
}

#define CUDA_TRY(expr)                                                                         \
    do {                                                                                       \
        cudaError_t e__ = (expr);                                                              \
        if (e__ != cudaSuccess)                                                                \
            return fail(IVF_ERR_CUDA, "%s failed: %s (%s:%d)", #expr, cudaGetErrorString(e__), \
                        __FILE__, __LINE__);                                                   \
    } while (0)

}  // namespace

#include "kv_check.cuh"

namespace {

constexpr int kMaxDevices = 64;
constexpr int64_t kMaxCount = 0x7FFFFFFF;

// A launch; `after`: it may start while the kernel before it in the stream ends (that kernel lets it, and it waits by itself before it
// touches memory).
template <typename... KArgs, typename... Args>
int launch(bool after, void (*kernel)(KArgs...), dim3 grid, int block, int smem, cudaStream_t stream, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 1 : 0;
    kv_host_launched();
    CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...));
    return IVF_OK;
}
// Allows a kernel the most dynamic shared memory that any call of it takes, once for a device.  `seen` belongs to one kernel.
struct SmemSeen {
    std::atomic<bool> device[kMaxDevices];
};
template <typename K>
int allow_smem(K kernel, int most, const KvHostCtx& ctx, SmemSeen& seen) {
    std::atomic<bool>& known = seen.device[ctx.index];
    if (known.load(std::memory_order_acquire)) return IVF_OK;
    CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    known.store(true, std::memory_order_release);
    return IVF_OK;
}

// ------------------------------------------------------------------ attention over whole caches
std::atomic<int> g_kv_chunk{0};  // test hook (ivf_debug_set_kv_chunk): 0 = by the sizes, 1 = rows kernel only, 2 = tile kernel wherever it can run

struct ChunkShape {
    int streams;  // of 128 rows; 0: the kernel of 16 rows
    int part_heads, parts, tile_tokens, ctas;
    int rows;  // of a slot: an even number, so that slots and their rows of sums start at multiples of 16 bytes
};
ChunkShape chunk_shape(int group, int dim, bool tile) {
    ChunkShape s;
    s.streams = !tile ? 0 : dim > 128 ? 1 : 2;
    const int rows = tile ? 128 : 16;
    s.part_heads = std::min(group, rows);
    s.parts = (group + rows - 1) / rows;
    s.tile_tokens = (group > rows ? 1 : rows / group) * std::max(s.streams, 1);
    s.rows = (s.tile_tokens * s.part_heads + 1) / 2 * 2;
    s.ctas = (tile || dim > 128 ? 1 : dim > 64 ? 2 : 3) * kChunkMaxSms;
    return s;
}
void chunk_settings(ChunkParams& p, const ChunkShape& s) {
    p.tile_tokens = s.tile_tokens, p.part_heads = s.part_heads, p.parts = s.parts, p.rows = s.rows;
    p.item_cost = s.streams ? 384 : 160;
    p.least = s.streams ? 1024 : 160;
    p.grain = s.streams ? 128 : 64;
}
int chunk_ctas(const ChunkShape& s, int num_sms) { return s.ctas / kChunkMaxSms * std::min(num_sms, kChunkMaxSms); }
int64_t chunk_bytes(const ChunkShape& s, int dim) {
    return s.ctas * (static_cast<int64_t>(sizeof(ChunkDesc)) + 2ll * s.rows * (dim + 2) * sizeof(float));
}
// Small tiles read the keys once for 16 rows, large ones for up to 256, at some cost of starting.  By rows (new tokens by the heads of a
// group) to a request, small / large tiles in us: one request of 65,536 tokens by 8 heads of 128 in groups of 4: 16 rows 63 / 69, 32 rows 94 / 69, 128
// rows 282 / 79; 64 requests of 8,192: 16 rows 223 / 248, 32 rows 422 / 253.  Heads of 64: 16 rows 129 / 230, 32 rows 235 / 241.  Heads
// wider than 128 leave the small tiles one CTA on an SM: 64 requests of 8,192 by 4 heads of 256, 2 rows 384 / 232.  Those are of requests alike.  The host
// knows no request's tokens, only their sum and the table's rows, so rows without new tokens, or with one, count against a prompt beside
// them: 2,048 tokens of one request of 32,768, 8 heads of 128 in groups of 4, in a table of 1 or 64 rows 950 us by large tiles, of 512 rows 7,830 by
// small ones (955 by large); 512 tokens of 8,192 beside 255 single ones of 4,000 1,069 / 1,068.
bool chunk_tiles_pay(int64_t n_tokens, int n_req, int group, int dim) {
    const int kernel = g_kv_chunk.load();
    if (kernel == 1 || dim < 64) return false;
    return kernel == 2 || dim > 128 || n_tokens * group > (dim > 64 ? 16ll : 32ll) * std::max(n_req, 1);
}
int64_t chunk_workspace(int64_t n_tokens, int n_req, int group, int dim) {
    int64_t bytes = chunk_bytes(chunk_shape(group, dim, false), dim);
    if (chunk_tiles_pay(n_tokens, n_req, group, dim)) bytes = std::max(bytes, chunk_bytes(chunk_shape(group, dim, true), dim));
    return bytes;
}

template <typename T, int DP>
int launch_chunk_rows(const ChunkParams& p, int ctas, const KvHostCtx& ctx, cudaStream_t stream) {
    static SmemSeen seen;
    if (int rc = allow_smem(kv_chunk_rows_kernel<T, DP>, RowsShape<DP>::kSmem, ctx, seen)) return rc;
    return launch(false, kv_chunk_rows_kernel<T, DP>, dim3(ctas), kRowsThreads, RowsShape<DP>::kSmem, stream, p);
}
template <typename T, int DB, bool CAP, bool BIAS>
int launch_chunk_tile(const ChunkParams& p, const CUtensorMap& mk, const CUtensorMap& mv, int ctas, const KvHostCtx& ctx, cudaStream_t stream) {
    static SmemSeen seen;
    if (int rc = allow_smem(kv_chunk_tile_kernel<T, DB, CAP, BIAS>, chunk_tile_smem<DB>(), ctx, seen)) return rc;
    return launch(false, kv_chunk_tile_kernel<T, DB, CAP, BIAS>, dim3(ctas), ChunkTileShape<DB>::kThreads, chunk_tile_smem<DB>(), stream, mk, mv, p);
}
template <typename T, int DB>
int launch_chunk_tile(const ChunkParams& p, const CUtensorMap& mk, const CUtensorMap& mv, int ctas, const KvHostCtx& ctx, cudaStream_t stream) {
    if (p.slopes)
        return p.cap_out == 0.0f ? launch_chunk_tile<T, DB, false, true>(p, mk, mv, ctas, ctx, stream) : launch_chunk_tile<T, DB, true, true>(p, mk, mv, ctas, ctx, stream);
    return p.cap_out == 0.0f ? launch_chunk_tile<T, DB, false, false>(p, mk, mv, ctas, ctx, stream) : launch_chunk_tile<T, DB, true, false>(p, mk, mv, ctas, ctx, stream);
}
template <typename T>
int launch_chunk(ChunkParams& p, void* workspace, const KvHostCtx& ctx, cudaStream_t stream) {
    CUtensorMap mk, mv;
    const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    const int page = 1 << p.page_shift;
    // (an expanded cache has no tensor map: small tiles)
    const bool tile = chunk_tiles_pay(p.n_tokens, p.n_req, p.group, p.dim) && p.num_pages > 0 &&
                      kv_host_map(&mk, p.kc, p.dim, page, p.n_kv_heads, p.num_pages, bf16) && kv_host_map(&mv, p.vc, p.dim, page, p.n_kv_heads, p.num_pages, bf16);
    const ChunkShape s = chunk_shape(p.group, p.dim, tile);
    const int ctas = chunk_ctas(s, ctx.num_sms);
    chunk_settings(p, s);
    p.desc = static_cast<ChunkDesc*>(workspace);
    p.slots = reinterpret_cast<float*>(p.desc + s.ctas);
    int rc;
    if (tile)
        rc = p.dim <= 64 ? launch_chunk_tile<T, 1>(p, mk, mv, ctas, ctx, stream) : p.dim <= 128 ? launch_chunk_tile<T, 2>(p, mk, mv, ctas, ctx, stream)
                                                                                              : launch_chunk_tile<T, 4>(p, mk, mv, ctas, ctx, stream);
    else
        rc = p.dim <= 64 ? launch_chunk_rows<T, 64>(p, ctas, ctx, stream) : p.dim <= 128 ? launch_chunk_rows<T, 128>(p, ctas, ctx, stream)
                                                                                         : launch_chunk_rows<T, 256>(p, ctas, ctx, stream);
    if (rc != IVF_OK) return rc;
    // Several warps to a row where items have many parts: one token over 131,072 (37 parts) 93 us, with one warp 99; 37 requests in
    // windows (2 parts) 29, with one warp 27: the more blocks of threads there are to start.
    const bool many = !tile && ctas >= 8ll * std::max(p.n_req, 1) * p.n_kv_heads * p.parts;
    const dim3 grid(ctas, many ? p.rows : (p.rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32));
    return launch(true, many ? kv_chunk_join_kernel<T, kJoinThreads / 32> : kv_chunk_join_kernel<T, 1>, grid, kJoinThreads, 0, stream, p);
}

// Whether `out` has an element of `q`'s memory.  Views with the same strides (two parts of one buffer, its axes in any order) are told apart by
// the distance of their starts, rows of one buffer in turn (the same token stride) by their place in the turn, other tensors by their ranges.
bool out_over_q(const void* q, const int64_t* q_stride, const void* out, const int64_t* out_stride, int64_t n, int64_t heads, int dim) {
    const int64_t q_row = (heads - 1) * q_stride[1] + dim, o_row = (heads - 1) * out_stride[1] + dim, step = q_stride[0];
    const int64_t q0 = static_cast<int64_t>(reinterpret_cast<uintptr_t>(q)) / 2, o0 = static_cast<int64_t>(reinterpret_cast<uintptr_t>(out)) / 2;
    if (q0 + (n - 1) * step + q_row <= o0 || o0 + (n - 1) * out_stride[0] + o_row <= q0) return false;
    if ((n == 1 || step == out_stride[0]) && (heads == 1 || q_stride[1] == out_stride[1])) {
        // output (t', h') and query (t, h) lie o0 - q0 + (t' - t) step + (h' - h) q_stride[1] apart
        for (int64_t h = 1 - heads; h < heads; ++h) {
            const int64_t apart = o0 - q0 + h * q_stride[1];
            const int64_t t = n == 1 ? 0 : -apart / step;  // the nearest (a written tensor's stride is not 0), or one from it
            for (int64_t i = t - 1; i <= t + 1; ++i)
                if (i > -n && i < n && std::abs(apart + i * step) < dim) return true;
        }
        return false;
    }
    if (step == 0 || step != out_stride[0]) return true;
    const int64_t after = ((o0 - q0) % step + step) % step;  // of an output row behind the start of a query row
    return after < q_row || after + o_row > step;
}

// ------------------------------------------------------------------ pages
struct PagesPlace {
    int64_t words, before, claim, wish, bytes;  // offsets into the workspace
};
PagesPlace pages_place(int n_new, int64_t num_pages) {
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    PagesPlace w;
    w.words = (num_pages + 31) / 32;
    w.before = up(w.words * 4);
    w.claim = w.before + up((w.words + 1) * 4);
    w.wish = w.claim + up(num_pages * 4);
    w.bytes = w.wish + up(8ll * n_new);
    return w;
}
// One CTA does it all where its launch costs less than the three or four of the other way.
bool pages_small(int n_new, int max_blocks, int64_t num_pages) {
    return n_new <= kPageScan && num_pages <= 32768 && static_cast<int64_t>(n_new) * max_blocks <= 32768;
}
constexpr int kSmallSmem = (2 * 32768 / 32 + 5 * kPageScan) * 4;

int check_pages(const char* op, const int32_t* table, int64_t table_stride, const int32_t* lens, int n_old, int n_new, int max_blocks, int64_t num_pages,
                int page_size, const int32_t* out, int64_t out_stride) {
    if (n_old < 0 || n_new < 0) return fail(IVF_ERR_INVALID_ARG, "%s: negative row count", op);
    if (n_old > kPageMaxRows || n_new > kPageMaxRows) return fail(IVF_ERR_UNSUPPORTED, "%s: at most %d rows", op, kPageMaxRows);
    if (int rc = kv_check_page(page_size)) return rc;
    if (num_pages < 0 || num_pages > kMaxCount) return fail(IVF_ERR_INVALID_ARG, "num_pages = %lld", (long long)num_pages);
    if (max_blocks < 1 || (n_old > 1 && table_stride < max_blocks) || (n_new > 1 && out_stride < max_blocks))
        return fail(IVF_ERR_INVALID_ARG, "block table: max_blocks = %d, strides %lld and %lld", max_blocks, (long long)table_stride, (long long)out_stride);
    if ((n_old > 0 && (!table || !lens)) || (n_new > 0 && !out)) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    return IVF_OK;
}

// Where the outputs and inputs are, as rows of bytes.
struct Span {
    const void* p;
    int64_t row, step, n;
};
bool spans_meet(const Span& a, const Span& b) {
    if (!a.p || !b.p || a.n < 1 || b.n < 1 || a.row < 1 || b.row < 1) return false;
    auto end = [](const Span& s) { return static_cast<const char*>(s.p) + (s.n - 1) * s.step + s.row; };
    if (end(a) <= static_cast<const char*>(b.p) || end(b) <= static_cast<const char*>(a.p)) return false;
    const Span &many = a.n >= b.n ? a : b, &few = a.n >= b.n ? b : a;
    for (int64_t i = 0; i < few.n; ++i)
        if (kv_over_rows(static_cast<const char*>(few.p) + i * few.step, few.row, many.p, many.row, std::max<int64_t>(many.step, 1), many.n)) return true;
    return false;
}

}  // namespace

extern "C" {

int ivf_kv_attend_chunk_workspace(int64_t n_tokens, int n_heads, const ivf_kv_cache* cache, int n_req, int64_t* bytes) {
    if (!cache || !bytes) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if (n_tokens < 0 || n_req < 0) return fail(IVF_ERR_INVALID_ARG, "negative size: n_tokens = %lld, n_req = %d", (long long)n_tokens, n_req);
    int rc = kv_check_dim(cache->head_dim);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, cache->n_kv_heads);
    if (rc != IVF_OK) return rc;
    *bytes = n_tokens == 0 ? 0 : chunk_workspace(n_tokens, n_req, n_heads / cache->n_kv_heads, cache->head_dim);
    return IVF_OK;
}

int ivf_kv_attend_chunk(const void* q, const int64_t q_stride[2], int64_t n_tokens, int n_heads, const ivf_kv_cache* cache,
                        const int32_t* table, int64_t table_stride, int n_req, int max_blocks, const int32_t* token_start,
                        const int32_t* kv_lens, float scale, float cap, const float* slopes, int window, const int32_t* prefix, void* out,
                        const int64_t out_stride[2], float* out_lse, void* workspace, int64_t workspace_bytes, void* stream_) {
    if (n_tokens < 0 || n_req < 0) return fail(IVF_ERR_INVALID_ARG, "negative size: n_tokens = %lld, n_req = %d", (long long)n_tokens, n_req);
    if (n_tokens > kMaxCount / 8) return fail(IVF_ERR_UNSUPPORTED, "at most 2^28 - 1 tokens");
    if (n_req > kPageMaxRows) return fail(IVF_ERR_UNSUPPORTED, "n_req = %d: at most %d requests", n_req, kPageMaxRows);
    int rc = kv_check_cache(cache, n_tokens > 0, n_tokens > 0);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, cache->n_kv_heads);
    if (rc != IVF_OK) return rc;
    if (!(scale - scale == 0.0f)) return fail(IVF_ERR_INVALID_ARG, "scale must be finite");
    if (!(cap >= 0.0f && cap - cap == 0.0f)) return fail(IVF_ERR_INVALID_ARG, "cap must be finite and not negative (0: none)");
    const float log2e = 1.4426950408889634f, scale_log2 = scale * log2e, cap_in = cap > 0.0f ? scale / cap : 0.0f, cap_out = cap * log2e;
    if (!(scale_log2 - scale_log2 == 0.0f && cap_in - cap_in == 0.0f && cap_out - cap_out == 0.0f) ||
        (cap > 0.0f && scale != 0.0f && std::fabs(cap_in) < std::numeric_limits<float>::min()))
        return fail(IVF_ERR_INVALID_ARG, "scale = %g, cap = %g: scale * log2(e), cap * log2(e) and scale / cap must be finite, and scale / cap not below the normal numbers", scale, cap);
    if (window < 0) return fail(IVF_ERR_INVALID_ARG, "window = %d: must not be negative (0: none)", window);
    if (n_tokens == 0) return IVF_OK;
    if (max_blocks < 1 || (n_req > 1 && table_stride < max_blocks))
        return fail(IVF_ERR_INVALID_ARG, "block table: n_req = %d, max_blocks = %d, stride %lld", n_req, max_blocks, (long long)table_stride);
    if (!token_start || (n_req > 0 && (!table || !kv_lens))) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if ((rc = kv_check_rows("q", q, q_stride, 2)) != IVF_OK || (rc = kv_check_rows("out", out, out_stride, 2)) != IVF_OK ||
        (rc = kv_check_apart("out", out_stride, {n_tokens, n_heads}, cache->head_dim)) != IVF_OK)
        return rc;
    if (out_over_q(q, q_stride, out, out_stride, n_tokens, n_heads, cache->head_dim))
        return fail(IVF_ERR_INVALID_ARG, "out must not share memory with q: rows are read again by other blocks of threads");
    const int64_t need = chunk_workspace(n_tokens, n_req, n_heads / cache->n_kv_heads, cache->head_dim);
    if (!workspace || workspace_bytes < need || kv_misaligned(workspace, 16))
        return fail(IVF_ERR_INVALID_ARG, "workspace: %lld bytes, 16-byte aligned, are needed (ivf_kv_attend_chunk_workspace)", (long long)need);
    KvHostCtx ctx;
    if ((rc = kv_host_ctx(&ctx)) != IVF_OK) return rc;
    ChunkParams p;
    p.q = q, p.q_stride[0] = q_stride[0], p.q_stride[1] = q_stride[1], p.n_tokens = n_tokens;
    p.group = n_heads / cache->n_kv_heads, p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim;
    p.kc = KvPlane{cache->k, cache->k_stride[0], cache->k_stride[1], cache->k_stride[2]};
    p.vc = KvPlane{cache->v, cache->v_stride[0], cache->v_stride[1], cache->v_stride[2]};
    p.num_pages = cache->num_pages;
    p.table = table, p.table_stride = table_stride, p.n_req = n_req, p.max_blocks = max_blocks, p.page_shift = kv_shift(cache->page_size);
    p.token_start = token_start, p.kv_lens = kv_lens, p.prefix = prefix, p.window = window;
    p.scale_log2 = scale_log2, p.cap_in = cap_in, p.cap_out = cap_out;
    p.slopes = slopes, p.out = out, p.out_stride[0] = out_stride[0], p.out_stride[1] = out_stride[1], p.lse = out_lse, p.status = ctx.status;
    p.limit_ns = ctx.limit_ns;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return cache->dtype == IVF_F16 ? launch_chunk<__half>(p, workspace, ctx, stream) : launch_chunk<__nv_bfloat16>(p, workspace, ctx, stream);
}

int ivf_debug_set_kv_chunk(int kernel) {
    if (kernel < 0 || kernel > 2) return fail(IVF_ERR_INVALID_ARG, "kernel = %d", kernel);
    g_kv_chunk = kernel;
    return IVF_OK;
}

int ivf_debug_kv_chunk_spans(int64_t n_tokens, int n_heads, const ivf_kv_cache* cache, int n_req, int max_blocks, const int32_t* token_start,
                             const int32_t* kv_lens, int window, const int32_t* prefix, int tiles, int num_sms, int64_t* items, int64_t max_items,
                             int64_t info[4]) {
    if (!cache || !token_start || !kv_lens || !info || (max_items > 0 && !items)) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    int rc = kv_check_page(cache->page_size);
    if (rc == IVF_OK) rc = kv_check_dim(cache->head_dim);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, cache->n_kv_heads);
    if (rc != IVF_OK) return rc;
    if (n_tokens < 0 || n_req < 0 || max_blocks < 1 || window < 0 || num_sms < 1 || max_items < 0) return fail(IVF_ERR_INVALID_ARG, "negative size");
    const ChunkShape s = chunk_shape(n_heads / cache->n_kv_heads, cache->head_dim, tiles != 0);
    ChunkParams p = {};
    p.n_tokens = n_tokens, p.group = n_heads / cache->n_kv_heads, p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim;
    p.n_req = n_req, p.max_blocks = max_blocks, p.page_shift = kv_shift(cache->page_size);
    p.token_start = token_start, p.kv_lens = kv_lens, p.prefix = prefix, p.window = window;
    chunk_settings(p, s);
    int64_t total = 0, n = 0;
    for (int b = 0, taken = 0; b < n_req; ++b) {
        const ChunkReq r = chunk_req(p, b, taken, false);
        taken = r.start;
        total += p.n_kv_heads * p.parts * chunk_before(p, r, r.tiles);
    }
    ChunkSpans spans;
    chunk_spans(p, total, chunk_ctas(s, num_sms), spans);
    for (int c = 0; c < spans.ctas; ++c) {
        ChunkCursor at = {}, kept = {};
        at.left = spans.begin(c + 1) - spans.begin(c);
        if (at.left > 0) chunk_locate(p, 0, n_req, 0, spans.begin(c), at);
        bool keeps = tiles && chunk_keep(p, at, kept);
        while (true) {
            if (at.left <= 0 && keeps) {
                at = kept;
                keeps = false;
            }
            if (at.left <= 0) break;
            const ChunkItem it = chunk_item(p, at);
            if (n < max_items) {
                const int64_t row[11] = {c, at.b, it.hv, it.token, it.tokens, it.pos, it.k0, it.k1, it.first, it.last,
                                         it.first && !it.last ? chunk_parts(spans, c, it.rest) : 0};
                std::copy(row, row + 11, items + 11 * n);
            }
            ++n;
            chunk_next(p, at);
        }
    }
    info[0] = n, info[1] = spans.ctas, info[2] = s.tile_tokens, info[3] = total;
    return IVF_OK;
}

int ivf_kv_pages_workspace(int n_new, int max_blocks, int64_t num_pages, int64_t* bytes) {
    if (!bytes) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if (n_new < 0 || max_blocks < 1 || num_pages < 0 || num_pages > kMaxCount)
        return fail(IVF_ERR_INVALID_ARG, "n_new = %d, max_blocks = %d, num_pages = %lld", n_new, max_blocks, (long long)num_pages);
    *bytes = pages_small(n_new, max_blocks, num_pages) ? 0 : pages_place(n_new, num_pages).bytes;
    return IVF_OK;
}

int ivf_kv_fork(const int32_t* table, int64_t table_stride, const int32_t* kv_lens, int n_old, int max_blocks, const int32_t* parent,
                const int32_t* keep, int n_new, int64_t num_pages, int page_size, int32_t* out_table, int64_t out_stride, int32_t* out_lens,
                int32_t* copy_from, int32_t* copy_to, int32_t* copy_fill, int32_t* free_pages, int32_t* n_free, void* workspace,
                int64_t workspace_bytes, void* stream_) {
    int rc = check_pages("ivf_kv_fork", table, table_stride, kv_lens, n_old, n_new, max_blocks, num_pages, page_size, out_table, out_stride);
    if (rc != IVF_OK) return rc;
    if ((n_new > 0 && (!parent || !out_lens || !copy_from || !copy_to || !copy_fill)) || (num_pages > 0 && !free_pages) || !n_free)
        return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    const int64_t row = 4ll * max_blocks, flat = 4ll * n_new;
    const Span in[] = {{table, row, n_old > 1 ? 4 * table_stride : row, n_old}, {kv_lens, 4ll * n_old, 0, 1}, {parent, flat, 0, 1}, {keep, flat, 0, 1}};
    const Span outs[] = {{out_table, row, n_new > 1 ? 4 * out_stride : row, n_new}, {out_lens, flat, 0, 1}, {copy_from, flat, 0, 1}, {copy_to, flat, 0, 1},
                         {copy_fill, flat, 0, 1}, {free_pages, 4 * num_pages, 0, 1}, {n_free, 4, 0, 1}};
    for (const Span& i : in)
        for (const Span& o : outs)
            if (spans_meet(i, o)) return fail(IVF_ERR_INVALID_ARG, "the outputs must not lie over the table, kv_lens, parent or keep");
    for (const Span& a : outs)
        for (const Span& b : outs)
            if (&a != &b && spans_meet(a, b)) return fail(IVF_ERR_INVALID_ARG, "the outputs must not lie over each other");
    const bool small = pages_small(n_new, max_blocks, num_pages);
    const PagesPlace w = pages_place(n_new, num_pages);
    if (!small && (!workspace || workspace_bytes < w.bytes || kv_misaligned(workspace, 16)))
        return fail(IVF_ERR_INVALID_ARG, "workspace: %lld bytes, 16-byte aligned, are needed (ivf_kv_pages_workspace)", (long long)w.bytes);
    KvHostCtx ctx;
    if ((rc = kv_host_ctx(&ctx)) != IVF_OK) return rc;
    KvPagesParams p = {};
    p.table = table, p.lens = kv_lens, p.parent = parent, p.keep = keep, p.table_stride = table_stride, p.out_stride = out_stride;
    p.n_old = n_old, p.n_new = n_new, p.max_blocks = max_blocks, p.page_shift = kv_shift(page_size), p.num_pages = num_pages;
    p.out = out_table, p.out_lens = out_lens, p.copy_from = copy_from, p.copy_to = copy_to, p.copy_fill = copy_fill;
    p.free_pages = free_pages, p.count = n_free, p.words = w.words, p.status = ctx.status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (small) {
        static SmemSeen seen;
        if ((rc = allow_smem(kv_fork_small_kernel, kSmallSmem, ctx, seen)) != IVF_OK) return rc;
        return launch(false, kv_fork_small_kernel, dim3(1), kPageScan, static_cast<int>((w.words + 5 * n_new) * 4), stream, p);
    }
    char* ws = static_cast<char*>(workspace);
    p.bits = reinterpret_cast<uint32_t*>(ws), p.claim = reinterpret_cast<int32_t*>(ws + w.claim), p.wish = reinterpret_cast<int32_t*>(ws + w.wish);
    static SmemSeen seen;
    if ((rc = allow_smem(kv_fork_place_kernel, 2 * kPageMaxRows * 4, ctx, seen)) != IVF_OK) return rc;
    auto ctas = [&](int64_t items, int per, int most) { return dim3(static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((items + per - 1) / per, most)))); };
    const int64_t pieces = (max_blocks + 32ll * kMarkBatch - 1) / (32 * kMarkBatch);
    if ((rc = launch(false, kv_pages_clear_kernel, ctas(w.words / 4 + n_new, kPageThreads, 2 * ctx.num_sms), kPageThreads, 0, stream, p)) != IVF_OK ||
        (rc = launch(true, kv_pages_mark_kernel, ctas(n_new * pieces, kPageThreads / 32, 8 * ctx.num_sms), kPageThreads, 0, stream, p)) != IVF_OK ||
        (rc = launch(true, kv_fork_own_kernel, ctas(n_new, kPageThreads, kMaxCount), kPageThreads, 0, stream, p)) != IVF_OK)
        return rc;
    return launch(true, kv_fork_place_kernel, ctas(w.words, kPageScan / 8, ctx.num_sms), kPageScan, 8 * n_new, stream, p);
}

int ivf_kv_compact(const int32_t* table, int64_t table_stride, const int32_t* kv_lens, int n_req, int max_blocks, int64_t num_pages,
                   int page_size, int32_t* out_table, int64_t out_stride, int32_t* copy_from, int32_t* copy_to, int64_t max_moves,
                   int32_t* n_held, void* workspace, int64_t workspace_bytes, void* stream_) {
    int rc = check_pages("ivf_kv_compact", table, table_stride, kv_lens, n_req, n_req, max_blocks, num_pages, page_size, out_table, out_stride);
    if (rc != IVF_OK) return rc;
    if (max_moves < 0 || max_moves > kMaxCount) return fail(IVF_ERR_INVALID_ARG, "max_moves = %lld", (long long)max_moves);
    if ((max_moves > 0 && (!copy_from || !copy_to)) || !n_held) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    const int64_t row = 4ll * max_blocks;
    const Span t = {table, row, n_req > 1 ? 4 * table_stride : row, n_req}, o = {out_table, row, n_req > 1 ? 4 * out_stride : row, n_req}, l = {kv_lens, 4ll * n_req, 0, 1};
    const Span lists[] = {{copy_from, 4 * max_moves, 0, 1}, {copy_to, 4 * max_moves, 0, 1}, {n_held, 4, 0, 1}};
    bool over = spans_meet(l, o) || (spans_meet(t, o) && (table != out_table || (n_req > 1 && table_stride != out_stride)));
    for (const Span& s : lists) {
        over |= spans_meet(s, t) || spans_meet(s, l) || spans_meet(s, o);
        for (const Span& x : lists) over |= &s != &x && spans_meet(s, x);
    }
    if (over) return fail(IVF_ERR_INVALID_ARG, "the outputs must not lie over the table (unless out is the table itself), kv_lens or each other");
    const bool small = pages_small(n_req, max_blocks, num_pages);
    const PagesPlace w = pages_place(n_req, num_pages);
    if (!small && (!workspace || workspace_bytes < w.bytes || kv_misaligned(workspace, 16)))
        return fail(IVF_ERR_INVALID_ARG, "workspace: %lld bytes, 16-byte aligned, are needed (ivf_kv_pages_workspace)", (long long)w.bytes);
    KvHostCtx ctx;
    if ((rc = kv_host_ctx(&ctx)) != IVF_OK) return rc;
    KvPagesParams p = {};
    p.table = table, p.lens = kv_lens, p.table_stride = table_stride, p.out_stride = out_stride;
    p.n_old = p.n_new = n_req, p.max_blocks = max_blocks, p.page_shift = kv_shift(page_size), p.num_pages = num_pages;
    p.out = out_table, p.copy_from = copy_from, p.copy_to = copy_to, p.max_moves = max_moves, p.count = n_held, p.words = w.words, p.status = ctx.status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (small) {
        static SmemSeen seen;
        if ((rc = allow_smem(kv_compact_small_kernel, kSmallSmem, ctx, seen)) != IVF_OK) return rc;
        return launch(false, kv_compact_small_kernel, dim3(1), kPageScan, static_cast<int>(2 * w.words * 4), stream, p);
    }
    char* ws = static_cast<char*>(workspace);
    p.bits = reinterpret_cast<uint32_t*>(ws), p.before = reinterpret_cast<int32_t*>(ws + w.before);
    auto ctas = [&](int64_t items, int per, int most) { return dim3(static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((items + per - 1) / per, most)))); };
    const int64_t pieces = (max_blocks + 32ll * kMarkBatch - 1) / (32 * kMarkBatch);
    if ((rc = launch(false, kv_pages_clear_kernel, ctas(w.words / 4, kPageThreads, 2 * ctx.num_sms), kPageThreads, 0, stream, p)) != IVF_OK ||
        (rc = launch(true, kv_pages_mark_kernel, ctas(n_req * pieces, kPageThreads / 32, 8 * ctx.num_sms), kPageThreads, 0, stream, p)) != IVF_OK ||
        (rc = launch(true, kv_compact_place_kernel, ctas(w.words, kPageScan / 8, ctx.num_sms), kPageScan, 0, stream, p)) != IVF_OK)
        return rc;
    return launch(true, kv_compact_rename_kernel, ctas(n_req * pieces, kPageThreads / 32, 8 * ctx.num_sms), kPageThreads, 0, stream, p);
}

int ivf_kv_copy(const ivf_kv_cache* cache, const int32_t* copy_from, const int32_t* copy_to, const int32_t* copy_fill, int64_t n, int8_t* codes,
                float* scales, void* stream_) {
    if (n < 0) return fail(IVF_ERR_INVALID_ARG, "negative page count %lld", (long long)n);
    if (n > kMaxCount) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 pages");
    int rc = kv_check_cache(cache, n > 0, n > 0);
    if (rc == IVF_OK) rc = kv_check_heads(cache->n_kv_heads, cache->n_kv_heads);
    if (rc != IVF_OK || n == 0) return rc;
    if (!copy_from || !copy_to || (codes == nullptr) != (scales == nullptr))
        return fail(IVF_ERR_INVALID_ARG, "null pointer argument (codes and scales: both or neither)");
    if (kv_misaligned(codes, 16)) return fail(IVF_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    if ((rc = kv_check_apart("key cache", cache->k_stride, {cache->num_pages, cache->n_kv_heads, cache->page_size}, cache->head_dim)) != IVF_OK ||
        (rc = kv_check_apart("value cache", cache->v_stride, {cache->num_pages, cache->n_kv_heads, cache->page_size}, cache->head_dim)) != IVF_OK)
        return rc;
    KvHostCtx ctx;
    if ((rc = kv_host_ctx(&ctx)) != IVF_OK) return rc;
    KvCopyParams p;
    p.kc = KvPlane{cache->k, cache->k_stride[0], cache->k_stride[1], cache->k_stride[2]};
    p.vc = KvPlane{cache->v, cache->v_stride[0], cache->v_stride[1], cache->v_stride[2]};
    p.num_pages = cache->num_pages, p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim, p.page_size = cache->page_size;
    p.from = copy_from, p.to = copy_to, p.fill = copy_fill, p.n = n, p.codes = codes, p.scales = scales, p.status = ctx.status;
    return launch(false, kv_copy_kernel, dim3(static_cast<unsigned>(n), p.n_kv_heads, 2), kCopyThreads, 0, static_cast<cudaStream_t>(stream_), p);
}

}  // extern "C"
