// Host side of the block-cache operators: argument checks (before any CUDA call) and launches.
// Included by ivf_api.cu, whose error text, device context and launch counter it uses.
#pragma once

namespace {

inline bool kv_page_ok(int page_size) { return page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128; }
inline int kv_shift(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }
inline bool kv_misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

int kv_check_page(int page_size) {
    if (!kv_page_ok(page_size)) return fail(IVF_ERR_UNSUPPORTED, "page_size = %d: must be 16, 32, 64 or 128", page_size);
    return IVF_OK;
}
int kv_check_dim(int dim) {
    if (dim < 16 || dim > kKvMaxDim || dim % 16 != 0)
        return fail(IVF_ERR_UNSUPPORTED, "head_dim = %d: must be a multiple of 16 in [16, %d]", dim, kKvMaxDim);
    return IVF_OK;
}
int kv_check_heads(int n_heads, int n_kv_heads) {
    if (n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads != 0)
        return fail(IVF_ERR_INVALID_ARG, "%d query heads, %d kv heads: the second must divide the first", n_heads, n_kv_heads);
    if (n_heads / n_kv_heads > kKvMaxGroup || n_kv_heads > 1024)
        return fail(IVF_ERR_UNSUPPORTED, "%d query heads, %d kv heads: at most %d to a group and 1024 groups", n_heads, n_kv_heads, kKvMaxGroup);
    return IVF_OK;
}
int kv_check_rows(const char* what, const void* p, const int64_t* stride, int n) {
    if (!p || !stride) return fail(IVF_ERR_INVALID_ARG, "%s: null pointer argument", what);
    if (kv_misaligned(p, 16)) return fail(IVF_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
    for (int i = 0; i < n; ++i)
        if (stride[i] < 0 || stride[i] % 8 != 0)
            return fail(IVF_ERR_INVALID_ARG, "%s: stride %lld must be a non-negative multiple of 8 elements", what, (long long)stride[i]);
    return IVF_OK;
}
// A tensor that is written: no two elements in one place.  Axes of one element do not count, the others lie within each other.
int kv_check_apart(const char* what, const int64_t* stride, std::initializer_list<int64_t> size, int dim) {
    std::pair<int64_t, int64_t> axis[3];
    int n = 0, i = 0;
    for (int64_t s : size) {
        if (s > 1) axis[n++] = {stride[i], s};
        ++i;
    }
    std::sort(axis, axis + n);
    int64_t span = dim;
    for (i = 0; i < n; ++i) {
        if (axis[i].first < span)
            return fail(IVF_ERR_INVALID_ARG, "%s is written: its stride of %lld elements must not be below %lld", what, (long long)axis[i].first, (long long)span);
        span += (axis[i].second - 1) * axis[i].first;
    }
    return IVF_OK;
}
int kv_check_cache(const ivf_kv_cache* c, bool keys, bool values) {
    if (!c) return fail(IVF_ERR_INVALID_ARG, "null cache descriptor");
    if (c->dtype != IVF_F16 && c->dtype != IVF_BF16)
        return fail(IVF_ERR_INVALID_ARG, "element type %d: caches are IVF_F16 or IVF_BF16", static_cast<int>(c->dtype));
    int rc = kv_check_page(c->page_size);
    if (rc == IVF_OK) rc = kv_check_dim(c->head_dim);
    if (rc != IVF_OK) return rc;
    if (c->num_pages < 0 || c->num_pages > 0x7FFFFFFF)
        return fail(IVF_ERR_INVALID_ARG, "num_pages = %lld", (long long)c->num_pages);
    if (keys && (rc = kv_check_rows("key cache", c->k, c->k_stride, 3)) != IVF_OK) return rc;
    if (values && (rc = kv_check_rows("value cache", c->v, c->v_stride, 3)) != IVF_OK) return rc;
    return IVF_OK;
}
// Whether `bytes` at `p` share memory with one of `n` rows of `row` bytes, `step` apart.
bool kv_over_rows(const void* p, int64_t bytes, const void* rows, int64_t row, int64_t step, int64_t n) {
    const int64_t at = static_cast<int64_t>(reinterpret_cast<uintptr_t>(p)) - static_cast<int64_t>(reinterpret_cast<uintptr_t>(rows));
    if (bytes <= 0 || row <= 0 || n < 1 || at + bytes <= 0 || at >= (n - 1) * step + row) return false;
    if (at < 0) return true;
    const int64_t k = at / step;
    return at - k * step < row || (k + 1 < n && at + bytes > (k + 1) * step);
}
KvPlane kv_plane(void* base, const int64_t* s) { return KvPlane{base, s[0], s[1], s[2]}; }

// The table and the tokens' request and position, as select and attend take them.
int kv_check_tokens(const int32_t* table, int64_t table_stride, int n_req, int max_blocks, const int32_t* token_req,
                    const int32_t* token_pos) {
    if (n_req < 1 || max_blocks < 1 || table_stride < max_blocks)
        return fail(IVF_ERR_INVALID_ARG, "block table: n_req = %d, max_blocks = %d, stride %lld", n_req, max_blocks, (long long)table_stride);
    if (!table || !token_req || !token_pos) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    return IVF_OK;
}

// Allows a kernel the most dynamic shared memory that any call of it takes, once for a device (asking each time costs a call
// half a microsecond).  The same number from every thread: the limit can also be lowered, and with each call's own size the
// smaller of two first calls could undo the larger.  `seen` belongs to one kernel.
struct KvSmemSeen {
    std::atomic<bool> device[kMaxDevices];
};
template <typename K>
int kv_allow_smem(K kernel, int most, const DeviceCtx& ctx, KvSmemSeen& seen) {
    std::atomic<bool>& known = seen.device[&ctx - g_ctx];
    if (known.load(std::memory_order_acquire)) return IVF_OK;
    CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    known.store(true, std::memory_order_release);
    return IVF_OK;
}

template <typename T, int LG>
int kv_launch_append(const KvAppendParams& p, int num_sms, cudaStream_t stream) {
    constexpr int kGroups = kAppThreads / LG;
    // few tokens: the rows of one token are shared out over several CTAs
    const int parts = (p.n_heads + kGroups - 1) / kGroups + 2 * ((p.n_kv_heads + kGroups - 1) / kGroups);
    const dim3 grid(static_cast<unsigned>(p.n_tokens), p.n_tokens < 4 * num_sms ? parts : 1);
    if (p.interleaved) kv_append_kernel<T, LG, true><<<grid, kAppThreads, 0, stream>>>(p);
    else kv_append_kernel<T, LG, false><<<grid, kAppThreads, 0, stream>>>(p);
    LAUNCH_CHECK();
    return IVF_OK;
}
template <typename T>
int kv_launch_append(const KvAppendParams& p, int num_sms, cudaStream_t stream) {
    if (p.dim <= 16) return kv_launch_append<T, 2>(p, num_sms, stream);
    if (p.dim <= 32) return kv_launch_append<T, 4>(p, num_sms, stream);
    if (p.dim <= 64) return kv_launch_append<T, 8>(p, num_sms, stream);
    if (p.dim <= 128) return kv_launch_append<T, 16>(p, num_sms, stream);
    return kv_launch_append<T, 32>(p, num_sms, stream);
}

template <typename T, int LG, int DEEP>
int kv_launch_summary(const KvSummaryParams& p, int64_t n, cudaStream_t stream) {
    kv_summary_kernel<T, LG, DEEP><<<dim3(static_cast<unsigned>(n), p.n_kv_heads), kSumThreads, 0, stream>>>(p);
    LAUNCH_CHECK();
    return IVF_OK;
}
template <typename T, int LG>
int kv_launch_summary(const KvSummaryParams& p, int64_t n, cudaStream_t stream) {
    constexpr int kRows = kSumThreads / LG;  // token rows side by side
    switch (p.page_size) {
        case 16: return kv_launch_summary<T, LG, (16 + kRows - 1) / kRows>(p, n, stream);
        case 32: return kv_launch_summary<T, LG, (32 + kRows - 1) / kRows>(p, n, stream);
        case 64: return kv_launch_summary<T, LG, (64 + kRows - 1) / kRows>(p, n, stream);
        default: return kv_launch_summary<T, LG, (128 + kRows - 1) / kRows>(p, n, stream);
    }
}
template <typename T>
int kv_launch_summary(const KvSummaryParams& p, int64_t n, cudaStream_t stream) {
    if (p.dim <= 16) return kv_launch_summary<T, 2>(p, n, stream);
    if (p.dim <= 32) return kv_launch_summary<T, 4>(p, n, stream);
    if (p.dim <= 64) return kv_launch_summary<T, 8>(p, n, stream);
    if (p.dim <= 128) return kv_launch_summary<T, 16>(p, n, stream);
    return kv_launch_summary<T, 32>(p, n, stream);
}

int g_kv_select = 0;  // test hook (ivf_debug_set_kv_select): 0 = by the sizes, 1 = rows kernel, 2 = windows kernel wherever it can run

template <typename T, int L, int NP>
int kv_launch_select_rows(const KvSelectParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    auto kernel = kv_select_rows_kernel<T, L, NP>;
    const int smem = p.max_blocks * 4;
    static KvSmemSeen seen;
    if (int rc = kv_allow_smem(kernel, kSelMaxBlocks * 4, ctx, seen)) return rc;
    // CTAs to a row: as many as live on the card at a time, as long as each still has 64 blocks
    const int64_t rows = p.n_tokens * p.n_kv_heads;
    const unsigned ranks = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>({8, kSelRowCtas * ctx.num_sms / rows, p.max_blocks / 64})));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.n_tokens) * ranks, p.n_kv_heads);
    cfg.blockDim = kSelRowThreads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    g_launches.fetch_add(1);
    CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
    return IVF_OK;
}
template <typename T, int K>
int kv_launch_select_windows(const KvSelectParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    auto kernel = kv_select_windows_kernel<T, K>;
    const int smem = static_cast<int>(sel_window_smem(p.max_blocks));
    static KvSmemSeen seen;
    if (int rc = kv_allow_smem(kernel, static_cast<int>(sel_window_smem(kSelWindowBlocks)), ctx, seen)) return rc;
    const dim3 grid(static_cast<unsigned>((p.n_tokens + kSelWindow - 1) / kSelWindow), p.n_kv_heads);
    kernel<<<grid, kSelThreads, smem, stream>>>(p, (p.max_blocks + 63) / 64 * 64);
    LAUNCH_CHECK();
    return IVF_OK;
}
template <typename T>
int kv_launch_select(const KvSelectParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    bool windows = g_kv_select != 1 && p.max_blocks <= kSelWindowBlocks;
    // Single tokens read a row's codes once for each token, windows once for 16; a window starts slower, and takes the requests
    // in it one after the other.  (Heads wider than 192 spill there and still win: 4,096 tokens by 4 heads of 512 blocks, d = 256,
    // windows 100 us, rows 299; d = 224 117 and 326; d = 128 66 and 242.)  256 blocks of d = 128, rows / windows: 16 tokens by 8 heads 13 / 19 us, 256 by 4
    // heads 23 / 19, 256 by 8 heads 33 / 19, 512 by 8 heads of 32 requests 54 / 21, but 64 by 8 heads of 32 requests 15 / 47.
    if (g_kv_select == 0)
        windows = windows && p.n_tokens * p.n_kv_heads >= 6 * ctx.num_sms && p.n_tokens >= 2 * static_cast<int64_t>(p.n_req);
    if (windows) {
        switch ((p.dim + 31) / 32) {
            case 1: return kv_launch_select_windows<T, 1>(p, ctx, stream);
            case 2: return kv_launch_select_windows<T, 2>(p, ctx, stream);
            case 3: return kv_launch_select_windows<T, 3>(p, ctx, stream);
            case 4: return kv_launch_select_windows<T, 4>(p, ctx, stream);
            case 5: return kv_launch_select_windows<T, 5>(p, ctx, stream);
            case 6: return kv_launch_select_windows<T, 6>(p, ctx, stream);
            case 7: return kv_launch_select_windows<T, 7>(p, ctx, stream);
            default: return kv_launch_select_windows<T, 8>(p, ctx, stream);
        }
    }
    if (p.dim <= 64) return kv_launch_select_rows<T, 4, 1>(p, ctx, stream);
    if (p.dim <= 128) return kv_launch_select_rows<T, 4, 2>(p, ctx, stream);
    return kv_launch_select_rows<T, 8, 2>(p, ctx, stream);
}

int g_kv_attend = 0;  // test hook (ivf_debug_set_kv_attend): 0 = by the sizes, 1 = rows kernel only, 2 = tile kernel wherever it can run

template <typename T, int DP, bool SPLIT>
int kv_launch_rows(const KvAttendParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    auto kernel = kv_attend_rows_kernel<T, DP, SPLIT>;
    static KvSmemSeen seen;
    if (int rc = kv_allow_smem(kernel, RowsShape<DP>::kSmem, ctx, seen)) return rc;
    const int z = (p.group + 15) / 16;
    unsigned ranks = 1, x = static_cast<unsigned>(p.n_tokens);
    if (p.window) {  // what the tile kernel left: a few CTAs look for it
        x = static_cast<unsigned>(std::min<int64_t>(p.n_tokens, std::max(1, 2 * ctx.num_sms / p.n_kv_heads)));
    } else {
        // CTAs to a token: until the card has two for each SM, as long as each warp still has a piece.  (More of them than
        // that costs: 64 tokens by 8 heads take 121 us with 4 CTAs to a token, 92 us with one.)
        const int pieces = p.n_select << (p.page_shift - 4);
        while (ranks < 8 && p.n_tokens * p.n_kv_heads * z * ranks < 2 * ctx.num_sms && pieces >= static_cast<int>(ranks) * 2 * kRowsWarps) ranks *= 2;
        x *= ranks;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(x, p.n_kv_heads, z);
    cfg.blockDim = kRowsThreads;
    cfg.dynamicSmemBytes = RowsShape<DP>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    g_launches.fetch_add(1);
    CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
    return IVF_OK;
}
template <typename T, bool SPLIT>
int kv_launch_rows(const KvAttendParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    if (p.dim <= 64) return kv_launch_rows<T, 64, SPLIT>(p, ctx, stream);
    if (p.dim <= 128) return kv_launch_rows<T, 128, SPLIT>(p, ctx, stream);
    return kv_launch_rows<T, 256, SPLIT>(p, ctx, stream);
}
template <typename T>
int kv_launch_rows(const KvAttendParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    return p.group <= 8 ? kv_launch_rows<T, true>(p, ctx, stream) : kv_launch_rows<T, false>(p, ctx, stream);
}

// A page of one head (64 tokens of it at most), 64 columns wide, with the 128-byte swizzle.
bool kv_make_map(CUtensorMap* map, const KvPlane& c, const KvAttendParams& p, bool bf16) {
    const int64_t page = 1 << p.page_shift;
    const int64_t size[4] = {p.dim, page, p.n_kv_heads, p.num_pages};
    const int64_t stride[3] = {c.token_stride, c.head_stride, c.page_stride};
    cuuint64_t dims[4], strides[3];
    for (int i = 0; i < 4; ++i) dims[i] = static_cast<cuuint64_t>(size[i]);
    for (int i = 0; i < 3; ++i) {
        if (stride[i] == 0 && size[i + 1] > 1) return false;  // an expanded axis: the map has no zero strides
        strides[i] = static_cast<cuuint64_t>(stride[i] == 0 ? p.dim : stride[i]) * 2;
        if (strides[i] >= (cuuint64_t(1) << 40)) return false;
    }
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(std::min<int64_t>(page, 64)), 1, 1}, step[4] = {1, 1, 1, 1};
    return g_encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, c.base, dims, strides, box, step,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DB>
int kv_launch_tile(const KvAttendParams& p, const CUtensorMap& mk, const CUtensorMap& mv, const DeviceCtx& ctx, cudaStream_t stream) {
    static KvSmemSeen seen;
    if (int rc = kv_allow_smem(kv_attend_tile_kernel<T, DB>, tile_smem<DB>(), ctx, seen)) return rc;
    const dim3 grid(static_cast<unsigned>((p.n_tokens + p.window - 1) / p.window), p.n_kv_heads);
    kv_attend_tile_kernel<T, DB><<<grid, TileShape<DB>::kThreads, tile_smem<DB>(), stream>>>(mk, mv, p);
    LAUNCH_CHECK();
    return IVF_OK;
}

// Whether `out` has an element of `q`'s memory.  Rows of one buffer in turn (the same token stride) are told apart, other
// tensors by their ranges.
bool kv_out_over_q(const KvAttendParams& p) {
    const int64_t heads = static_cast<int64_t>(p.group) * p.n_kv_heads;
    const int64_t q_row = (heads - 1) * p.q_stride[1] + p.dim, o_row = (heads - 1) * p.out_stride[1] + p.dim;
    const int64_t q0 = static_cast<int64_t>(reinterpret_cast<uintptr_t>(p.q)) / 2, o0 = static_cast<int64_t>(reinterpret_cast<uintptr_t>(p.out)) / 2;
    if (q0 + (p.n_tokens - 1) * p.q_stride[0] + q_row <= o0 || o0 + (p.n_tokens - 1) * p.out_stride[0] + o_row <= q0) return false;
    const int64_t step = p.q_stride[0];
    if (step == 0 || step != p.out_stride[0]) return true;
    const int64_t after = ((o0 - q0) % step + step) % step;  // of an output row behind the start of a query row
    return after < q_row || after + o_row > step;
}

template <typename T>
int kv_launch_attend(KvAttendParams& p, const DeviceCtx& ctx, cudaStream_t stream) {
    const int window = 128 / p.group;
    p.window = 0;
    p.limit_ns = g_wait_limit_ns.load();
    CUtensorMap mk, mv;
    const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    bool tile = g_kv_attend != 1 && p.dim >= 64 && p.num_pages > 0;
    // Windows pay where there is work for the whole card and tokens enough beyond one to a request to fill some; what they do
    // not take is left to the rows.  16 blocks of 64 keys, d = 128, rows / windows: 64 tokens by 4 heads of a group of 8
    // 31 / 43 us, 256 tokens 86 / 43, 512 tokens of 32 requests 152 / 43; by 8 heads without groups (128 tokens to a
    // window) 128 tokens of 8 requests 85 / 307, 256 tokens of one 146 / 107.
    const int64_t parts = (p.group + 15) / 16;
    // A window may be taken twice, and the second time needs its queries: an output in their place goes by the rows alone, which
    // read a row before they write it.
    tile = tile && !kv_out_over_q(p);
    if (g_kv_attend == 0) tile = tile && p.n_tokens * p.n_kv_heads * parts >= 4 * ctx.num_sms && p.n_tokens - p.n_req + 1 >= 2 * window;
    if (tile) {
        if (int rc = get_encode()) return rc;
        tile = kv_make_map(&mk, p.kc, p, bf16) && kv_make_map(&mv, p.vc, p, bf16);
    }
    if (!tile) return kv_launch_rows<T>(p, ctx, stream);
    p.window = window;
    const int rc = p.dim <= 64 ? kv_launch_tile<T, 1>(p, mk, mv, ctx, stream) : p.dim <= 128 ? kv_launch_tile<T, 2>(p, mk, mv, ctx, stream)
                                                                                       : kv_launch_tile<T, 4>(p, mk, mv, ctx, stream);
    return rc != IVF_OK ? rc : kv_launch_rows<T>(p, ctx, stream);
}

constexpr int64_t kKvMaxTokens = 0x7FFFFFFF;

}  // namespace

extern "C" {

int ivf_kv_tables(const int32_t* cached, const int32_t* fresh, int n_req, int page_size, const int32_t* free_pages, int n_free,
                  int32_t* table, int64_t table_stride, int max_blocks, int32_t* kv_lens, int32_t* token_start,
                  int32_t* token_req, int32_t* token_pos, int64_t* token_slot, int64_t max_tokens, int32_t* touched_page,
                  int32_t* touched_fill, int64_t max_touched, int32_t* used, void* stream_) {
    if (n_req < 0 || n_free < 0 || max_tokens < 0 || max_touched < 0)
        return fail(IVF_ERR_INVALID_ARG, "negative size: n_req = %d, n_free = %d, max_tokens = %lld, max_touched = %lld", n_req, n_free,
                    (long long)max_tokens, (long long)max_touched);
    if (int rc = kv_check_page(page_size)) return rc;
    if (n_req > kTabMaxReq) return fail(IVF_ERR_UNSUPPORTED, "n_req = %d: at most %d requests", n_req, kTabMaxReq);
    if (max_tokens > kKvMaxTokens || max_touched > kKvMaxTokens) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 tokens and touched blocks");
    if (n_req == 0) return IVF_OK;
    if (max_blocks < 1 || table_stride < max_blocks)
        return fail(IVF_ERR_INVALID_ARG, "block table: max_blocks = %d, stride %lld", max_blocks, (long long)table_stride);
    if (!cached || !fresh || !table || !kv_lens || !token_start || !used || (n_free > 0 && !free_pages) ||
        (max_tokens > 0 && (!token_req || !token_pos || !token_slot)) || (max_touched > 0 && (!touched_page || !touched_fill)))
        return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    // Every block of threads reads the lengths and the free list throughout, so nothing may be written over them: a plan's
    // kv_lens cannot be the `cached` of a call that fills the same plan.
    struct { const void* p; int64_t bytes; } out[] = {
        {kv_lens, 4ll * n_req}, {token_start, 4ll * n_req + 4}, {token_req, 4 * max_tokens}, {token_pos, 4 * max_tokens}, {token_slot, 8 * max_tokens},
        {touched_page, 4 * max_touched}, {touched_fill, 4 * max_touched}, {used, 4}}, in[] = {{cached, 4ll * n_req}, {fresh, 4ll * n_req}, {free_pages, 4ll * n_free}};
    for (const auto& i : in) {
        bool over = kv_over_rows(i.p, i.bytes, table, 4ll * max_blocks, 4 * table_stride, n_req);
        for (const auto& o : out) over |= kv_over_rows(i.p, i.bytes, o.p, o.bytes, o.bytes, 1);
        if (over) return fail(IVF_ERR_INVALID_ARG, "the table and the plan must not lie over cached, fresh or free_pages");
    }
    DeviceCtx* pctx = nullptr;
    if (int rc = get_ctx(&pctx)) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    KvTablesParams p;
    p.cached = cached, p.fresh = fresh, p.free_pages = free_pages;
    p.n_req = n_req, p.page_shift = kv_shift(page_size), p.n_free = n_free, p.max_blocks = max_blocks;
    p.table = table, p.table_stride = table_stride;
    p.kv_lens = kv_lens, p.token_start = token_start, p.token_req = token_req, p.token_pos = token_pos, p.token_slot = token_slot;
    p.max_tokens = max_tokens, p.touched_page = touched_page, p.touched_fill = touched_fill, p.max_touched = max_touched;
    p.used = used, p.status = pctx->status;
    auto smem_of = [](int requests) { return 3 * (requests + 1) * static_cast<int>(sizeof(int)); };
    const int smem = smem_of(n_req);
    static KvSmemSeen seen;
    if (int rc = kv_allow_smem(kv_tables_kernel, smem_of(kTabMaxReq), *pctx, seen)) return rc;
    const int64_t items = (static_cast<int64_t>(n_req) * max_blocks) / 8 + max_tokens + max_touched;
    // (the lengths and counts are written even where there is room for nothing else)
    const int64_t grid = std::max<int64_t>(1, std::min<int64_t>((items + kTabThreads - 1) / kTabThreads, pctx->num_sms));
    kv_tables_kernel<<<static_cast<unsigned>(grid), kTabThreads, smem, stream>>>(p);
    LAUNCH_CHECK();
    return IVF_OK;
}

int ivf_kv_append(const void* q, const int64_t q_stride[2], const void* k, const int64_t k_stride[2], const void* v,
                  const int64_t v_stride[2], int64_t n_tokens, int n_heads, const ivf_kv_cache* cache, const int32_t* token_pos,
                  const int64_t* token_slot, const float* rotary, int n_pos, int rot_dim, int interleaved, const float* q_weight,
                  const float* k_weight, float eps, void* q_out, const int64_t q_out_stride[2], void* stream_) {
    if (n_tokens < 0) return fail(IVF_ERR_INVALID_ARG, "negative token count %lld", (long long)n_tokens);
    if (n_tokens > kKvMaxTokens) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 tokens");
    int rc = kv_check_cache(cache, n_tokens > 0, n_tokens > 0);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, cache->n_kv_heads);
    if (rc != IVF_OK) return rc;
    if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16 != 0)
        return fail(IVF_ERR_UNSUPPORTED, "rot_dim = %d: must be a multiple of 16 in [0, head_dim = %d]", rot_dim, cache->head_dim);
    if (rot_dim > 0 && n_pos < 1) return fail(IVF_ERR_INVALID_ARG, "n_pos = %d rows of angles", n_pos);
    if (!(eps >= 0.0f)) return fail(IVF_ERR_INVALID_ARG, "eps must not be negative");
    if (n_tokens == 0) return IVF_OK;
    if ((rc = kv_check_rows("q", q, q_stride, 2)) != IVF_OK || (rc = kv_check_rows("k", k, k_stride, 2)) != IVF_OK ||
        (rc = kv_check_rows("v", v, v_stride, 2)) != IVF_OK || (rc = kv_check_rows("q_out", q_out, q_out_stride, 2)) != IVF_OK ||
        (rc = kv_check_apart("q_out", q_out_stride, {n_tokens, n_heads}, cache->head_dim)) != IVF_OK ||
        (rc = kv_check_apart("key cache", cache->k_stride, {cache->num_pages, cache->n_kv_heads, cache->page_size}, cache->head_dim)) != IVF_OK ||
        (rc = kv_check_apart("value cache", cache->v_stride, {cache->num_pages, cache->n_kv_heads, cache->page_size}, cache->head_dim)) != IVF_OK)
        return rc;
    if (!token_pos || !token_slot || (rot_dim > 0 && !rotary)) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if (kv_misaligned(rotary, 16) || kv_misaligned(q_weight, 16) || kv_misaligned(k_weight, 16))
        return fail(IVF_ERR_INVALID_ARG, "rotary, q_weight and k_weight must be 16-byte aligned");
    DeviceCtx* pctx = nullptr;
    if ((rc = get_ctx(&pctx)) != IVF_OK) return rc;
    KvAppendParams p;
    p.q = q, p.k = k, p.v = v, p.q_out = q_out;
    for (int i = 0; i < 2; ++i)
        p.q_stride[i] = q_stride[i], p.k_stride[i] = k_stride[i], p.v_stride[i] = v_stride[i], p.qo_stride[i] = q_out_stride[i];
    p.n_tokens = n_tokens, p.n_heads = n_heads, p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim;
    p.page_shift = kv_shift(cache->page_size), p.num_pages = cache->num_pages;
    p.kc = kv_plane(cache->k, cache->k_stride), p.vc = kv_plane(cache->v, cache->v_stride);
    p.token_pos = token_pos, p.token_slot = token_slot, p.rotary = rotary, p.n_pos = n_pos, p.rot_dim = rot_dim;
    p.interleaved = interleaved, p.q_weight = q_weight, p.k_weight = k_weight, p.eps = eps, p.status = pctx->status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return cache->dtype == IVF_F16 ? kv_launch_append<__half>(p, pctx->num_sms, stream)
                                   : kv_launch_append<__nv_bfloat16>(p, pctx->num_sms, stream);
}

int ivf_kv_summarize(const ivf_kv_cache* cache, const int32_t* pages, const int32_t* fills, int64_t n, int8_t* codes,
                     float* scales, void* stream_) {
    if (n < 0) return fail(IVF_ERR_INVALID_ARG, "negative page count %lld", (long long)n);
    if (n > kKvMaxTokens) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 pages");
    int rc = kv_check_cache(cache, n > 0, false);
    if (rc == IVF_OK) rc = kv_check_heads(cache->n_kv_heads, cache->n_kv_heads);
    if (rc != IVF_OK || n == 0) return rc;
    if (!pages || !fills || !codes || !scales) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if (kv_misaligned(codes, 16)) return fail(IVF_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    DeviceCtx* pctx = nullptr;
    if ((rc = get_ctx(&pctx)) != IVF_OK) return rc;
    KvSummaryParams p;
    p.kc = kv_plane(cache->k, cache->k_stride), p.num_pages = cache->num_pages;
    p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim, p.page_size = cache->page_size;
    p.pages = pages, p.fills = fills, p.codes = codes, p.scales = scales, p.status = pctx->status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return cache->dtype == IVF_F16 ? kv_launch_summary<__half>(p, n, stream) : kv_launch_summary<__nv_bfloat16>(p, n, stream);
}

int ivf_kv_select(const void* q, const int64_t q_stride[2], ivf_dtype dtype, int64_t n_tokens, int n_heads, int n_kv_heads,
                  int head_dim, const int8_t* codes, const float* scales, int64_t num_pages, const int32_t* table,
                  int64_t table_stride, int n_req, int max_blocks, int page_size, const int32_t* token_req,
                  const int32_t* token_pos, int n_select, int n_first, int n_last, int32_t* out, void* stream_) {
    if (n_tokens < 0) return fail(IVF_ERR_INVALID_ARG, "negative token count %lld", (long long)n_tokens);
    if (n_tokens > kKvMaxTokens) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 tokens");
    if (dtype != IVF_F16 && dtype != IVF_BF16) return fail(IVF_ERR_INVALID_ARG, "element type %d: queries are IVF_F16 or IVF_BF16", static_cast<int>(dtype));
    int rc = kv_check_page(page_size);
    if (rc == IVF_OK) rc = kv_check_dim(head_dim);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, n_kv_heads);
    if (rc != IVF_OK) return rc;
    if (n_select < 1 || n_select > kKvMaxSelect) return fail(IVF_ERR_UNSUPPORTED, "n_select = %d: must be in [1, %d]", n_select, kKvMaxSelect);
    if (n_first < 0 || n_last < 1 || n_first > n_select || n_last > n_select - n_first)
        return fail(IVF_ERR_INVALID_ARG, "n_first = %d, n_last = %d: n_last must be at least 1 and both fit n_select = %d", n_first, n_last, n_select);
    if (num_pages < 0 || num_pages > 0x7FFFFFFF) return fail(IVF_ERR_INVALID_ARG, "num_pages = %lld", (long long)num_pages);
    if (n_tokens > kKvMaxTokens / 8) return fail(IVF_ERR_UNSUPPORTED, "at most 2^28 - 1 tokens");
    if (n_tokens == 0) return IVF_OK;
    if ((rc = kv_check_tokens(table, table_stride, n_req, max_blocks, token_req, token_pos)) != IVF_OK) return rc;
    if (max_blocks > kSelMaxBlocks) return fail(IVF_ERR_UNSUPPORTED, "max_blocks = %d: at most %d blocks of one request", max_blocks, kSelMaxBlocks);
    if ((rc = kv_check_rows("q", q, q_stride, 2)) != IVF_OK) return rc;
    if (!codes || !scales || !out) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    if (kv_misaligned(codes, 16)) return fail(IVF_ERR_INVALID_ARG, "codes must be 16-byte aligned");
    DeviceCtx* pctx = nullptr;
    if ((rc = get_ctx(&pctx)) != IVF_OK) return rc;
    KvSelectParams p;
    p.q = q, p.q_stride[0] = q_stride[0], p.q_stride[1] = q_stride[1], p.n_tokens = n_tokens;
    p.group = n_heads / n_kv_heads, p.n_kv_heads = n_kv_heads, p.dim = head_dim;
    p.codes = codes, p.scales = scales, p.num_pages = num_pages;
    p.table = table, p.table_stride = table_stride, p.n_req = n_req, p.max_blocks = max_blocks, p.page_shift = kv_shift(page_size);
    p.token_req = token_req, p.token_pos = token_pos, p.n_select = n_select, p.n_first = n_first, p.n_last = n_last;
    p.out = out, p.status = pctx->status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return dtype == IVF_F16 ? kv_launch_select<__half>(p, *pctx, stream) : kv_launch_select<__nv_bfloat16>(p, *pctx, stream);
}

int ivf_kv_attend(const void* q, const int64_t q_stride[2], int64_t n_tokens, int n_heads, const ivf_kv_cache* cache,
                  const int32_t* table, int64_t table_stride, int n_req, int max_blocks, const int32_t* token_req,
                  const int32_t* token_pos, const int32_t* selected, int n_select, float scale, void* out,
                  const int64_t out_stride[2], float* out_lse, void* stream_) {
    if (n_tokens < 0) return fail(IVF_ERR_INVALID_ARG, "negative token count %lld", (long long)n_tokens);
    if (n_tokens > kKvMaxTokens) return fail(IVF_ERR_UNSUPPORTED, "at most 2^31 - 1 tokens");
    int rc = kv_check_cache(cache, n_tokens > 0, n_tokens > 0);
    if (rc == IVF_OK) rc = kv_check_heads(n_heads, cache->n_kv_heads);
    if (rc != IVF_OK) return rc;
    if (n_select < 1 || n_select > kKvMaxSelect) return fail(IVF_ERR_UNSUPPORTED, "n_select = %d: must be in [1, %d]", n_select, kKvMaxSelect);
    if (!(scale - scale == 0.0f)) return fail(IVF_ERR_INVALID_ARG, "scale must be finite");
    if (n_tokens == 0) return IVF_OK;
    if ((rc = kv_check_tokens(table, table_stride, n_req, max_blocks, token_req, token_pos)) != IVF_OK) return rc;
    if ((rc = kv_check_rows("q", q, q_stride, 2)) != IVF_OK || (rc = kv_check_rows("out", out, out_stride, 2)) != IVF_OK ||
        (rc = kv_check_apart("out", out_stride, {n_tokens, n_heads}, cache->head_dim)) != IVF_OK)
        return rc;
    if (n_tokens > kKvMaxTokens / 8) return fail(IVF_ERR_UNSUPPORTED, "at most 2^28 - 1 tokens");
    if (!selected) return fail(IVF_ERR_INVALID_ARG, "null pointer argument");
    DeviceCtx* pctx = nullptr;
    if ((rc = get_ctx(&pctx)) != IVF_OK) return rc;
    KvAttendParams p;
    p.q = q, p.q_stride[0] = q_stride[0], p.q_stride[1] = q_stride[1], p.n_tokens = n_tokens;
    p.group = n_heads / cache->n_kv_heads, p.n_kv_heads = cache->n_kv_heads, p.dim = cache->head_dim;
    p.kc = kv_plane(cache->k, cache->k_stride), p.vc = kv_plane(cache->v, cache->v_stride), p.num_pages = cache->num_pages;
    p.table = table, p.table_stride = table_stride, p.n_req = n_req, p.max_blocks = max_blocks, p.page_shift = kv_shift(cache->page_size);
    p.token_req = token_req, p.token_pos = token_pos, p.selected = selected, p.n_select = n_select;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = out, p.out_stride[0] = out_stride[0], p.out_stride[1] = out_stride[1], p.lse = out_lse, p.status = pctx->status;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return cache->dtype == IVF_F16 ? kv_launch_attend<__half>(p, *pctx, stream) : kv_launch_attend<__nv_bfloat16>(p, *pctx, stream);
}

int ivf_debug_set_kv_select(int kernel) {
    if (kernel < 0 || kernel > 2) return fail(IVF_ERR_INVALID_ARG, "kernel = %d", kernel);
    g_kv_select = kernel;
    return IVF_OK;
}

int ivf_debug_set_kv_attend(int kernel) {
    if (kernel < 0 || kernel > 2) return fail(IVF_ERR_INVALID_ARG, "kernel = %d", kernel);
    g_kv_attend = kernel;
    return IVF_OK;
}

}  // extern "C"
