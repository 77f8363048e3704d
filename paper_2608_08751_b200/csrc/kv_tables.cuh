// Block tables and slot maps from request lengths.
//
// Request b holds cached_b tokens in old_b = ceil(cached_b / p) pages and gets fresh_b more; it then needs
// now_b = ceil((cached_b + fresh_b) / p) pages.  With exclusive prefix sums over the requests of the new
// tokens, of the new pages now_b - old_b and of the touched blocks, every output element follows by itself:
// table[b][j] = free[pages_before_b + j - old_b] for old_b <= j < now_b, and for new token i of request b
// pos = cached_b + i, slot = page(pos / p) * p + pos % p.  The sums are taken in 64 bits and held at 2^31 - 1 where they are
// stored: no list is as long, so what lies behind such a sum has no place in any.
//
// One launch, no workspace, no atomics: every CTA scans all lengths itself (they are 8 bytes a request and
// come from L2) and keeps the three prefix sums in shared memory; then the CTAs share out the table rows,
// the tokens and the touched blocks.  A token in a page that was there before reads the table's old entry,
// which no CTA writes; one in a new page reads the free list, so no CTA waits for another.  A small step is one launch's
// latency (32 requests: 4.6 us); 2,048 requests with a table of 4,096 columns, of which 7 MB are written, take 12 us.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kTabThreads = 512;
constexpr int kTabMaxReq = 16384;  // three ints each in shared memory

struct KvTablesParams {
    const int32_t *cached, *fresh, *free_pages;
    int n_req, page_shift, n_free, max_blocks;
    int32_t* table;
    int64_t table_stride;
    int32_t *kv_lens, *token_start, *token_req, *token_pos;
    int64_t* token_slot;
    int64_t max_tokens;
    int32_t *touched_page, *touched_fill;
    int64_t max_touched;
    int32_t* used;
    int* status;
};

struct TabLengths {
    int cached, fresh, old_blocks, now_blocks;
    bool bad;
};

__device__ __forceinline__ TabLengths tab_lengths(const KvTablesParams& p, int b) {
    TabLengths l;
    const int c = p.cached[b], f = p.fresh[b];
    l.bad = c < 0 || f < 0 || static_cast<int64_t>(c) + f > 0x7FFFFFFFll - (1 << p.page_shift);
    l.cached = l.bad ? 0 : c;
    l.fresh = l.bad ? 0 : f;
    l.old_blocks = (l.cached + (1 << p.page_shift) - 1) >> p.page_shift;
    l.now_blocks = (l.cached + l.fresh + (1 << p.page_shift) - 1) >> p.page_shift;
    return l;
}

// Blocks that hold new tokens of a request.
__device__ __forceinline__ int tab_touched(const KvTablesParams& p, const TabLengths& l) {
    return l.fresh > 0 ? l.now_blocks - (l.cached >> p.page_shift) : 0;
}

__device__ __forceinline__ int tab_held(int64_t sum) { return static_cast<int>(min(sum, static_cast<int64_t>(0x7FFFFFFF))); }

// Last index i in [0, n) with start[i] <= x (start ascends, start[0] == 0): skips entries of empty requests.
__device__ __forceinline__ int tab_find(const int* start, int n, int x) {
    int lo = 0, hi = n;  // start[lo] <= x < start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The page of block j of request b, whichever of the two lists holds it; -1 where there is none.
__device__ __forceinline__ int tab_page(const KvTablesParams& p, int b, int j, int old_blocks, int first) {
    if (j >= p.max_blocks) return -1;
    if (j < old_blocks) return p.table[b * p.table_stride + j];
    const int64_t at = static_cast<int64_t>(first) + (j - old_blocks);
    return at < p.n_free ? p.free_pages[at] : -1;
}

__global__ void __launch_bounds__(kTabThreads) kv_tables_kernel(KvTablesParams p) {
    extern __shared__ int tab_smem[];
    int* s_tok = tab_smem;                // [n_req + 1] first token of each request
    int* s_page = s_tok + p.n_req + 1;    // [n_req + 1] new pages before it
    int* s_touch = s_page + p.n_req + 1;  // [n_req + 1] touched blocks before it
    __shared__ int64_t s_warp[3][kTabThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    // ---- prefix sums: each thread owns a contiguous run of requests
    const int per = (p.n_req + kTabThreads - 1) / kTabThreads;
    const int b0 = min(tid * per, p.n_req), b1 = min(b0 + per, p.n_req);
    int64_t sum[3] = {0, 0, 0};
    bool bad = false, cramped = false;
    for (int b = b0; b < b1; ++b) {
        const TabLengths l = tab_lengths(p, b);
        sum[0] += l.fresh;
        sum[1] += l.now_blocks - l.old_blocks;
        sum[2] += tab_touched(p, l);
        bad |= l.bad;
        cramped |= l.now_blocks > p.max_blocks;
        if (blockIdx.x == 0) p.kv_lens[b] = l.cached + l.fresh;
    }
    int64_t incl[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        incl[k] = sum[k];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t v = __shfl_up_sync(0xFFFFFFFFu, incl[k], off);
            if (lane >= off) incl[k] += v;
        }
        if (lane == 31) s_warp[k][warp] = incl[k];
    }
    __syncthreads();
    int64_t base[3], total[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        base[k] = incl[k] - sum[k];
        total[k] = 0;
        for (int w = 0; w < kTabThreads / 32; ++w) {
            const int64_t v = s_warp[k][w];
            if (w < warp) base[k] += v;
            total[k] += v;
        }
    }
    for (int b = b0; b < b1; ++b) {
        const TabLengths l = tab_lengths(p, b);
        s_tok[b] = tab_held(base[0]);
        s_page[b] = tab_held(base[1]);
        s_touch[b] = tab_held(base[2]);
        if (blockIdx.x == 0) p.token_start[b] = s_tok[b];
        base[0] += l.fresh;
        base[1] += l.now_blocks - l.old_blocks;
        base[2] += tab_touched(p, l);
    }
    if (tid == 0) {
        s_tok[p.n_req] = tab_held(total[0]);
        s_page[p.n_req] = tab_held(total[1]);
        s_touch[p.n_req] = tab_held(total[2]);
        if (blockIdx.x == 0) {
            p.token_start[p.n_req] = s_tok[p.n_req];
            *p.used = s_page[p.n_req];
            if (total[1] > p.n_free || total[0] > p.max_tokens || total[2] > p.max_touched)
                kv_report(p.status, kKvStatusNoPages, KV_SITE_TABLES);
        }
    }
    if (blockIdx.x == 0) {
        if (bad) kv_report(p.status, kKvStatusBadId, KV_SITE_TABLES);
        if (cramped) kv_report(p.status, kKvStatusNoPages, KV_SITE_TABLES);
    }
    __syncthreads();

    const int64_t threads = static_cast<int64_t>(gridDim.x) * kTabThreads;
    const int64_t me = static_cast<int64_t>(blockIdx.x) * kTabThreads + tid;

    // ---- tokens
    for (int64_t t = me; t < p.max_tokens; t += threads) {
        int req = -1, pos = -1;
        int64_t slot = -1;
        if (t < total[0]) {
            req = tab_find(s_tok, p.n_req, static_cast<int>(t));
            const TabLengths l = tab_lengths(p, req);
            pos = l.cached + (static_cast<int>(t) - s_tok[req]);
            const int page = tab_page(p, req, pos >> p.page_shift, l.old_blocks, s_page[req]);
            if (page >= 0) slot = (static_cast<int64_t>(page) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        }
        p.token_req[t] = req;
        p.token_pos[t] = pos;
        p.token_slot[t] = slot;
    }
    // ---- blocks that hold new tokens
    for (int64_t w = me; w < p.max_touched; w += threads) {
        int page = -1, fill = 0;
        if (w < total[2]) {
            const int b = tab_find(s_touch, p.n_req, static_cast<int>(w));
            const TabLengths l = tab_lengths(p, b);
            const int j = (l.cached >> p.page_shift) + (static_cast<int>(w) - s_touch[b]);
            page = tab_page(p, b, j, l.old_blocks, s_page[b]);
            fill = page >= 0 ? min(1 << p.page_shift, l.cached + l.fresh - (j << p.page_shift)) : 0;
        }
        p.touched_page[w] = page;
        p.touched_fill[w] = fill;
    }
    // ---- table rows, a warp per row: entries from old_blocks on
    const int64_t warps = threads / 32;
    for (int64_t b = me / 32; b < p.n_req; b += warps) {
        const TabLengths l = tab_lengths(p, static_cast<int>(b));
        int32_t* row = p.table + b * p.table_stride;
        for (int j = l.old_blocks + lane; j < p.max_blocks; j += 32)
            row[j] = j < l.now_blocks ? tab_page(p, static_cast<int>(b), j, l.old_blocks, s_page[b]) : -1;
    }
}

}  // namespace ivf
