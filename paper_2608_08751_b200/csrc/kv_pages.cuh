// The life of a cache's pages: tables that fork, pages that move, and the copies that both ask for.
//
// Nothing is counted from step to step.  What holds a page is the table, so the pages that nobody holds follow from the table
// and the lengths alone: a bit for each page, set by whoever holds it, and ranks from sums over the words of bits.
//
// ivf_kv_fork: new row i holds the first keep_i tokens of old row parent_i.  Blocks that those tokens fill are shared.  A block
// that they fill in part gets tokens appended, so one holder may keep the page and the others take copies: the lowest row keeps it,
// if no row shares it as a filled block.  Copies go to the lowest pages that nobody holds, in row order.
// ivf_kv_compact: with n pages held, the held pages from number n on move to the holes below n, the highest into the lowest hole.
//
// Four launches, since each step wants all bits of the one before: bits and claims are cleared; the table is read, bits set; owners of partly
// filled blocks are settled; ranks are taken and lists written (compaction: ranks and lists, then the table is renamed).  Every CTA that takes ranks adds up
// the words before its own itself, from L2.  1,024 rows of up to 2,048 blocks, 1.3 million pages held: 35 us, 16 of them the bits' 1.3 million
// atomic operations at random places; compaction of 512 such rows 25 us.  Small tables go by one CTA: 32 beams 9.3 us, 64 rows 8.6 us, of which 8 are the
// host's.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kPageThreads = 256;
constexpr int kPageScan = 1024;     // threads of the kernels that take ranks
constexpr int kPageMaxRows = 16384;

struct KvPagesParams {
    const int32_t *table, *lens, *parent, *keep;  // parent null: compaction
    int64_t table_stride, out_stride;
    int n_old, n_new, max_blocks, page_shift;
    int64_t num_pages;
    int32_t *out, *out_lens, *copy_from, *copy_to, *copy_fill, *free_pages, *count;
    int64_t max_moves;
    uint32_t* bits;   // [words]: pages held as filled blocks; compaction: all held ones
    int32_t* claim;   // [num_pages]: lowest row that holds the page as a partly filled block; only claimed pages' are set
    int32_t* before;  // [words + 1] compaction: held pages before the word
    int32_t* wish;    // [2 * n_new] page that a row wants a copy of, or -1; then the row's filled blocks
    int64_t words;
    int* status;
};

struct ForkRow {
    int parent, keep;  // keep = 0: an empty row
    int full, rest;    // filled blocks, tokens in the block behind them
};
__device__ __forceinline__ ForkRow fork_row(const KvPagesParams& p, int i, bool report) {
    ForkRow f;
    f.parent = p.parent[i];
    bool bad = f.parent >= p.n_old;
    f.keep = 0;
    if (f.parent >= 0 && !bad) {
        const int len = p.lens[f.parent];
        f.keep = p.keep ? p.keep[i] : len;
        bad = len < 0 || f.keep < 0 || f.keep > len || f.keep > static_cast<int64_t>(p.max_blocks) << p.page_shift;
        if (bad) f.keep = 0;
    }
    if (bad && report) kv_report(p.status, kKvStatusBadId, KV_SITE_FORK);
    f.full = f.keep >> p.page_shift;
    f.rest = f.keep & ((1 << p.page_shift) - 1);
    return f;
}
// An entry that a row holds: a page of the cache, or -1.
__device__ __forceinline__ int held_page(const KvPagesParams& p, int page, int site) {
    if (page >= p.num_pages) {
        kv_report(p.status, kKvStatusBadId, site);
        return -1;
    }
    return page < 0 ? -1 : page;
}
__device__ __forceinline__ int compact_blocks(const KvPagesParams& p, int b, bool report) {
    const int len = p.lens[b];
    const bool bad = len < 0 || len > static_cast<int64_t>(p.max_blocks) << p.page_shift;
    if (bad && report) kv_report(p.status, kKvStatusBadId, KV_SITE_COMPACT);
    if (len < 0) return 0;
    return static_cast<int>(min((static_cast<int64_t>(len) + (1 << p.page_shift) - 1) >> p.page_shift, static_cast<int64_t>(p.max_blocks)));
}

__global__ void __launch_bounds__(kPageThreads) kv_pages_clear_kernel(const KvPagesParams p) {
    pdl_trigger();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kPageThreads, me = static_cast<int64_t>(blockIdx.x) * kPageThreads + threadIdx.x;
    for (int64_t w = me; w < (p.words + 3) / 4; w += step) reinterpret_cast<uint4*>(p.bits)[w] = make_uint4(0, 0, 0, 0);
    if (p.parent)
        for (int64_t i = me; i < p.n_new; i += step) {
            const ForkRow f = fork_row(p, static_cast<int>(i), true);
            if (!f.rest) continue;
            const int page = held_page(p, p.table[f.parent * p.table_stride + f.full], KV_SITE_FORK);
            if (page >= 0) p.claim[page] = 0x7FFFFFFF;
        }
}

// A warp to 32 * kBatch entries of a row.
constexpr int kMarkBatch = 4;
__global__ void __launch_bounds__(kPageThreads) kv_pages_mark_kernel(const KvPagesParams p) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int pieces = (p.max_blocks + 32 * kMarkBatch - 1) / (32 * kMarkBatch);
    const int64_t items = static_cast<int64_t>(p.n_new) * pieces, step = static_cast<int64_t>(gridDim.x) * (kPageThreads / 32);
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * (kPageThreads / 32) + (threadIdx.x >> 5); w < items; w += step) {
        const int i = static_cast<int>(w / pieces), j0 = static_cast<int>(w % pieces) * 32 * kMarkBatch + lane;
        int row = i, full, rest = 0;
        if (p.parent) {
            const ForkRow f = fork_row(p, i, false);
            row = f.keep > 0 ? f.parent : 0;
            full = f.full;
            rest = f.rest;
            if (j0 == 0) p.out_lens[i] = f.keep;
        } else {
            full = compact_blocks(p, i, j0 == 0);
        }
        const int32_t* src = p.table + row * p.table_stride;
        int page[kMarkBatch];
#pragma unroll
        for (int k = 0; k < kMarkBatch; ++k) {
            const int j = j0 + 32 * k;
            page[k] = j < full + (rest > 0) ? src[j] : -1;
        }
#pragma unroll
        for (int k = 0; k < kMarkBatch; ++k) {
            const int j = j0 + 32 * k;
            page[k] = held_page(p, page[k], p.parent ? KV_SITE_FORK : KV_SITE_COMPACT);
            if (page[k] >= 0) {
                if (j < full) atomicOr(&p.bits[page[k] >> 5], 1u << (page[k] & 31));
                else atomicMin(&p.claim[page[k]], i);
            }
            // the block that is partly filled is entered later
            if (p.parent && j < p.max_blocks && !(rest > 0 && j == full)) p.out[i * p.out_stride + j] = j < full ? page[k] : -1;
        }
    }
}

// Sum over the CTA; every thread gets the sum of the threads before it, and the total.
__device__ __forceinline__ int page_scan(int v, int* warp_sum, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += x;
    }
    __syncthreads();  // (the words of a scan before)
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        const int mine = warp_sum[lane];
        int all = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xFFFFFFFFu, all, o);
            if (lane >= o) all += x;
        }
        warp_sum[lane] = all;
    }
    __syncthreads();
    total = warp_sum[31];
    return upto - v + (warp > 0 ? warp_sum[warp - 1] : 0);
}
// Held pages in words [0, w0) and in all words, by the whole CTA; words come by four (their number is rounded up to that, the last ones 0).
__device__ __forceinline__ void page_sums(const KvPagesParams& p, int64_t w0, int* warp_sum, int& before, int& all) {
    const uint4* bits = reinterpret_cast<const uint4*>(p.bits);
    int mine = 0, front = 0;
#pragma unroll 4
    for (int64_t w = threadIdx.x; w < (p.words + 3) / 4; w += kPageScan) {
        const uint4 v = bits[w];
        const int n = __popc(v.x) + __popc(v.y) + __popc(v.z) + __popc(v.w);
        mine += n;
        front += w * 4 < w0 ? n : 0;
    }
    page_scan(mine, warp_sum, all);
    page_scan(front, warp_sum, before);
}
// The words of a CTA: a multiple of four.
__device__ __forceinline__ void page_share(const KvPagesParams& p, int64_t& w0, int64_t& w1) {
    const int64_t per = ((p.words + gridDim.x - 1) / gridDim.x + 3) / 4 * 4;
    w0 = min(per * blockIdx.x, p.words);
    w1 = min(w0 + per, p.words);
}
// Bits of pages that exist in a word.
__device__ __forceinline__ uint32_t word_mask(const KvPagesParams& p, int64_t w) {
    const int64_t left = p.num_pages - w * 32;
    return left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1;
}

// Owners of partly filled blocks set their page's bit too, so that the bits are all held pages.  A page's own bit is what its lowest claim
// looks at, and no other row sets it here.
__global__ void __launch_bounds__(kPageThreads) kv_fork_own_kernel(const KvPagesParams p) {
    pdl_wait();
    pdl_trigger();
    const int i = blockIdx.x * kPageThreads + threadIdx.x;
    if (i >= p.n_new) return;
    const ForkRow f = fork_row(p, i, false);
    int from = -1;
    if (f.rest) {
        const int page = held_page(p, p.table[f.parent * p.table_stride + f.full], KV_SITE_FORK);
        int entry = -1;
        if (page >= 0) {
            const uint32_t bit = 1u << (page & 31);
            if (p.claim[page] == i && !(*reinterpret_cast<volatile uint32_t*>(&p.bits[page >> 5]) & bit)) {
                entry = page;
                atomicOr(&p.bits[page >> 5], bit);
            } else {
                from = page;
            }
        }
        p.out[i * p.out_stride + f.full] = entry;
    }
    p.wish[i] = from;
    p.wish[p.n_new + i] = f.full;
    p.copy_from[i] = from;
    p.copy_to[i] = -1;
    p.copy_fill[i] = from >= 0 ? f.rest : 0;
}

// The page that a row's copy goes to, its block `full`; page < 0: there is none left.
__device__ __forceinline__ void fork_copy(const KvPagesParams& p, int i, int full, int page) {
    if (page >= 0) {
        p.out[i * p.out_stride + full] = page;
        p.copy_to[i] = page;
    } else {
        p.copy_from[i] = -1;
        p.copy_fill[i] = 0;
        kv_report(p.status, kKvStatusNoPages, KV_SITE_FORK);
    }
}
// Words of bits by the whole CTA: f(word's number, its bits, pages counted before it) is called by every warp for words of its own, a lane to a
// page.  `count` says which pages of a word count, `some` whether f wants the word at all; both are called once for a word.
struct PageWords {
    uint32_t bits[kPageScan];
    int before[kPageScan];
    int warp_sum[32];
};
template <typename B, typename C, typename S, typename F>
__device__ __forceinline__ void each_word(int64_t w0, int64_t w1, int before, PageWords& s, B&& bits_of, C&& count, S&& some, F&& f) {
    for (int64_t base = w0; base < w1; base += kPageScan) {
        const int64_t w = base + threadIdx.x;
        const uint32_t bits = w < w1 ? bits_of(w) : 0;
        int total;
        const int first = before + page_scan(w < w1 ? __popc(count(w, bits)) : 0, s.warp_sum, total);  // (its barriers part the rounds)
        before += total;
        s.bits[threadIdx.x] = bits;
        s.before[threadIdx.x] = first;
        __syncthreads();
        const int n = static_cast<int>(min(w1 - base, static_cast<int64_t>(kPageScan)));
        for (int x = threadIdx.x >> 5; x < n; x += kPageScan / 32)
            if (some(base + x, s.bits[x])) f(base + x, s.bits[x], s.before[x]);
    }
}
// Free pages of words [w0, w1), `before` of them in earlier words: the first `copies` of all go to the rows that want copies (by rank, with their
// filled blocks), the others into the list.  Every thread of the CTA calls it.
template <typename F>
__device__ __forceinline__ void fork_list(const KvPagesParams& p, int64_t w0, int64_t w1, int before, int copies, const int* row_of, const int* full_of, PageWords& s, F&& bits_of) {
    const int lane = threadIdx.x & 31;
    auto free_of = [&](int64_t w, uint32_t bits) { return ~bits & word_mask(p, w); };
    each_word(w0, w1, before, s, bits_of, free_of, [&](int64_t w, uint32_t bits) { return free_of(w, bits) != 0; }, [&](int64_t w, uint32_t bits, int first) {
        const uint32_t free = free_of(w, bits);
        if (!(free >> lane & 1)) return;
        const int rank = first + __popc(free & ((1u << lane) - 1)), page = static_cast<int>(w * 32) + lane;
        if (rank < copies) fork_copy(p, row_of[rank], full_of[rank], page);
        else p.free_pages[rank - copies] = page;
    });
}

// Ranks of the rows that want copies and of the free pages.  A CTA takes a run of words.
__global__ void __launch_bounds__(kPageScan) kv_fork_place_kernel(const KvPagesParams p) {
    extern __shared__ int page_rows[];  // [2 * n_new] rows that want copies, by rank, and their filled blocks
    int* page_full = page_rows + p.n_new;
    __shared__ PageWords words;
    int* warp_sum = words.warp_sum;
    pdl_wait();
    int64_t w0, w1;
    int before, all;
    page_share(p, w0, w1);
    page_sums(p, w0, warp_sum, before, all);
    before = static_cast<int>(min(w0 * 32, p.num_pages)) - before;  // free ones from here on
    all = static_cast<int>(p.num_pages) - all;
    int copies = 0;
    for (int base = 0; base < p.n_new; base += kPageScan) {
        const int i = base + threadIdx.x;
        const bool wants = i < p.n_new && p.wish[i] >= 0;
        int total;
        const int rank = copies + page_scan(wants, warp_sum, total);
        if (wants) page_rows[rank] = i, page_full[rank] = p.wish[p.n_new + i];
        copies += total;
    }
    __syncthreads();
    fork_list(p, w0, w1, before, copies, page_rows, page_full, words, [&](int64_t w) { return p.bits[w]; });
    const int left = max(all - copies, 0);
    for (int64_t k = left + static_cast<int64_t>(blockIdx.x) * kPageScan + threadIdx.x; k < p.num_pages; k += static_cast<int64_t>(gridDim.x) * kPageScan)
        p.free_pages[k] = -1;
    if (blockIdx.x == 0) {
        for (int k = all + threadIdx.x; k < copies; k += kPageScan) fork_copy(p, page_rows[k], page_full[k], -1);
        if (threadIdx.x == 0) *p.count = left;
    }
}

// The whole of it in one CTA: small tables, where the launches would take longer than the work.  A row's thread keeps what it read of it.
__global__ void __launch_bounds__(kPageScan) kv_fork_small_kernel(const KvPagesParams p) {
    extern __shared__ __align__(16) int page_smem[];
    uint32_t* bits = reinterpret_cast<uint32_t*>(page_smem);  // [words]
    int* rows = page_smem + p.words;                          // [n_new] rows that want copies, by rank
    int* last = rows + p.n_new;                               // [n_new] page of the partly filled block, or -1
    int* source = last + p.n_new;                             // [n_new] the old row
    int* full = source + p.n_new;                             // [n_new] filled blocks
    int* wants_full = full + p.n_new;                         // [n_new] those of `rows`
    __shared__ PageWords words;
    int* warp_sum = words.warp_sum;
    const int tid = threadIdx.x;
    ForkRow mine = {-1, 0, 0, 0};  // of row `tid` (there are at most as many rows as threads)
    if (tid < p.n_new) {
        mine = fork_row(p, tid, true);
        source[tid] = mine.keep > 0 ? mine.parent : 0;
        full[tid] = mine.full;
        p.out_lens[tid] = mine.keep;
    }
    for (int w = tid; w < p.words; w += kPageScan) bits[w] = 0;
    __syncthreads();
    // (asked for before the rows are read, looked at behind them)
    const int partly = mine.rest ? p.table[mine.parent * p.table_stride + mine.full] : -1;
    // a thread to entries kPageScan apart of all rows together, four at a time
    const int entries = p.n_new * p.max_blocks;  // (32,768 at most)
    for (int e0 = tid; e0 < entries; e0 += 4 * kPageScan) {
        int row[4], j[4], page[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = e0 + k * kPageScan;
            row[k] = e / p.max_blocks;
            j[k] = e - row[k] * p.max_blocks;
            page[k] = e < entries && j[k] < full[row[k]] ? p.table[source[row[k]] * p.table_stride + j[k]] : -1;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (e0 + k * kPageScan >= entries) continue;
            page[k] = held_page(p, page[k], KV_SITE_FORK);
            if (page[k] >= 0) atomicOr(&bits[page[k] >> 5], 1u << (page[k] & 31));
            p.out[row[k] * p.out_stride + j[k]] = page[k];
        }
    }
    const int page = mine.rest ? held_page(p, partly, KV_SITE_FORK) : -1;
    if (tid < p.n_new) last[tid] = page;
    __syncthreads();
    bool own = false;
    if (page >= 0) {
        own = !(bits[page >> 5] >> (page & 31) & 1);
        for (int j = 0; own && j < tid; ++j) own = last[j] != page;
    }
    const bool wants = page >= 0 && !own;
    __syncthreads();
    if (own) {
        atomicOr(&bits[page >> 5], 1u << (page & 31));
        p.out[tid * p.out_stride + mine.full] = page;
    }
    if (tid < p.n_new) {
        p.copy_from[tid] = wants ? page : -1;
        p.copy_to[tid] = -1;
        p.copy_fill[tid] = wants ? mine.rest : 0;
    }
    int copies;
    const int rank = page_scan(wants, warp_sum, copies);
    if (wants) rows[rank] = tid, wants_full[rank] = mine.full;
    __syncthreads();  // (the bits, too)
    int held = 0, all;
    for (int w = tid; w < p.words; w += kPageScan) held += __popc(bits[w]);
    page_scan(held, warp_sum, all);
    all = static_cast<int>(p.num_pages) - all;
    fork_list(p, 0, p.words, 0, copies, rows, wants_full, words, [&](int64_t w) { return bits[w]; });
    const int left = max(all - copies, 0);
    for (int64_t k = left + tid; k < p.num_pages; k += kPageScan) p.free_pages[k] = -1;
    for (int k = all + tid; k < copies; k += kPageScan) fork_copy(p, rows[k], wants_full[k], -1);
    if (tid == 0) *p.count = left;
}

// ---------------------------------------------------------------------------------------------- compaction
// Moves of a run of words: `before` held pages lie in earlier ones.  held: of all; moves: how many are made.
template <typename F>
__device__ __forceinline__ void compact_list(const KvPagesParams& p, int64_t w0, int64_t w1, int before, int held, int64_t moves, PageWords& s, int32_t* before_of, F&& bits_of) {
    const int lane = threadIdx.x & 31;
    each_word(w0, w1, before, s, bits_of, [](int64_t, uint32_t bits) { return bits; },
              [&](int64_t, uint32_t) { return true; },
              [&](int64_t w, uint32_t bits, int upto) {
        if (lane == 0) before_of[w] = upto;
        // holes below `held`, from the lowest; pages from `held` on, from the highest
        const int below = upto + __popc(bits & ((1u << lane) - 1));
        const int64_t page = w * 32 + lane;
        const bool is = bits >> lane & 1;
        if (page < held ? is : !is) return;
        const int64_t rank = page < held ? page - below : static_cast<int64_t>(held) - 1 - below;
        if (rank < moves) (page < held ? p.copy_to : p.copy_from)[rank] = static_cast<int>(page);
    });
}
// Held pages among the first n pages, of bits in global memory (four words at a time) or in shared memory.
__device__ __forceinline__ int held_below(const uint32_t* bits, int n, int* warp_sum) {
    int v = 0;
    const int words = n / 32;
#pragma unroll 4
    for (int w = threadIdx.x; w < words / 4; w += kPageScan) {
        const uint4 u = reinterpret_cast<const uint4*>(bits)[w];
        v += __popc(u.x) + __popc(u.y) + __popc(u.z) + __popc(u.w);
    }
    const int w = words / 4 * 4 + threadIdx.x;  // up to three words, and a part of one
    if (w < words) v += __popc(bits[w]);
    else if (w == words && n % 32) v += __popc(bits[w] & ((1u << n % 32) - 1));
    int total;
    page_scan(v, warp_sum, total);
    return total;
}
// The number that a held page has afterwards.
template <typename F>
__device__ __forceinline__ int renamed(const KvPagesParams& p, int page, int held, int64_t moves, const int32_t* before_of, F&& bits_of) {
    if (page < held) return page;
    const uint32_t below = bits_of(page >> 5) & ((1u << (page & 31)) - 1);
    const int64_t rank = static_cast<int64_t>(held) - 1 - (before_of[page >> 5] + __popc(below));
    return rank < moves ? p.copy_to[rank] : page;
}

__global__ void __launch_bounds__(kPageScan) kv_compact_place_kernel(const KvPagesParams p) {
    __shared__ PageWords words;
    int* warp_sum = words.warp_sum;
    pdl_wait();
    pdl_trigger();
    int64_t w0, w1;
    int before, held;
    page_share(p, w0, w1);
    page_sums(p, w0, warp_sum, before, held);
    auto bits_of = [&](int64_t w) { return p.bits[w]; };
    const int64_t moves = min(static_cast<int64_t>(held - held_below(p.bits, held, warp_sum)), p.max_moves);
    compact_list(p, w0, w1, before, held, moves, words, p.before, bits_of);
    for (int64_t k = moves + static_cast<int64_t>(blockIdx.x) * kPageScan + threadIdx.x; k < p.max_moves; k += static_cast<int64_t>(gridDim.x) * kPageScan)
        p.copy_from[k] = p.copy_to[k] = -1;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *p.count = held;
        p.before[p.words] = static_cast<int>(moves);
    }
}

// A warp to 32 * kMarkBatch entries of a row.
__global__ void __launch_bounds__(kPageThreads) kv_compact_rename_kernel(const KvPagesParams p) {
    pdl_wait();
    const int lane = threadIdx.x & 31, held = *p.count;
    const int64_t moves = p.before[p.words];
    const int pieces = (p.max_blocks + 32 * kMarkBatch - 1) / (32 * kMarkBatch);
    const int64_t items = static_cast<int64_t>(p.n_new) * pieces, step = static_cast<int64_t>(gridDim.x) * (kPageThreads / 32);
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * (kPageThreads / 32) + (threadIdx.x >> 5); w < items; w += step) {
        const int i = static_cast<int>(w / pieces), j0 = static_cast<int>(w % pieces) * 32 * kMarkBatch + lane;
        const int blocks = compact_blocks(p, i, false);
        int page[kMarkBatch];
#pragma unroll
        for (int k = 0; k < kMarkBatch; ++k) {
            const int j = j0 + 32 * k;
            page[k] = j < blocks ? held_page(p, p.table[i * p.table_stride + j], KV_SITE_COMPACT) : -1;
        }
#pragma unroll
        for (int k = 0; k < kMarkBatch; ++k)
            if (page[k] >= 0) page[k] = renamed(p, page[k], held, moves, p.before, [&](int64_t x) { return p.bits[x]; });
#pragma unroll
        for (int k = 0; k < kMarkBatch; ++k)
            if (j0 + 32 * k < p.max_blocks) p.out[i * p.out_stride + j0 + 32 * k] = page[k];
    }
}

__global__ void __launch_bounds__(kPageScan) kv_compact_small_kernel(const KvPagesParams p) {
    extern __shared__ __align__(16) int page_smem[];
    uint32_t* bits = reinterpret_cast<uint32_t*>(page_smem);  // [words]
    int32_t* before_of = page_smem + p.words;                 // [words] (the bits by four: at a multiple of 16 bytes)
    __shared__ PageWords words;
    int* warp_sum = words.warp_sum;
    const int tid = threadIdx.x, lane = tid & 31;
    for (int w = tid; w < p.words; w += kPageScan) bits[w] = 0;
    __syncthreads();
    for (int i = tid >> 5; i < p.n_new; i += kPageScan / 32) {
        const int blocks = compact_blocks(p, i, lane == 0);
#pragma unroll 4
        for (int j = lane; j < blocks; j += 32) {
            const int page = held_page(p, p.table[i * p.table_stride + j], KV_SITE_COMPACT);
            if (page >= 0) atomicOr(&bits[page >> 5], 1u << (page & 31));
        }
    }
    __syncthreads();
    auto bits_of = [&](int64_t w) { return bits[w]; };
    int held = 0;
    for (int w = tid; w < p.words; w += kPageScan) held += __popc(bits[w]);
    page_scan(held, warp_sum, held);
    const int64_t moves = min(static_cast<int64_t>(held - held_below(bits, held, warp_sum)), p.max_moves);
    compact_list(p, 0, p.words, 0, held, moves, words, before_of, bits_of);
    for (int64_t k = moves + tid; k < p.max_moves; k += kPageScan) p.copy_from[k] = p.copy_to[k] = -1;
    if (tid == 0) *p.count = held;
    __syncthreads();  // the list of places, and the words' sums
    for (int i = tid >> 5; i < p.n_new; i += kPageScan / 32) {
        const int blocks = compact_blocks(p, i, false);
#pragma unroll 4
        for (int j = lane; j < p.max_blocks; j += 32) {
            const int page = j < blocks ? held_page(p, p.table[i * p.table_stride + j], KV_SITE_COMPACT) : -1;
            p.out[i * p.out_stride + j] = page >= 0 ? renamed(p, page, held, moves, before_of, bits_of) : -1;
        }
    }
}

// ---------------------------------------------------------------------------------------------- copies
// The first fill tokens (null: all) of page from[i] onto page to[i], for every kv head of keys and values, and the page's summary.  Bound
// by memory: each number is read once and written once (4,096 pages of 8 heads, 64 tokens and 128 columns, 2.1 GB: 333 us, 6.45 TB/s).
struct KvCopyParams {
    KvPlane kc, vc;
    int64_t num_pages;
    int n_kv_heads, dim, page_size;
    const int32_t *from, *to, *fill;
    int64_t n;
    int8_t* codes;  // [num_pages][n_kv_heads][dim] or null
    float* scales;  // [num_pages][n_kv_heads]
    int* status;
};
constexpr int kCopyThreads = 256;
constexpr int kCopyBatch = 4;  // pieces of 16 bytes in flight for each thread

__global__ void __launch_bounds__(kCopyThreads) kv_copy_kernel(const KvCopyParams p) {
    const int64_t i = blockIdx.x;
    const int h = blockIdx.y;
    const int from = p.from[i], to = p.to[i];
    int fill = p.fill ? p.fill[i] : p.page_size;
    const bool bad = from >= p.num_pages || to >= p.num_pages || fill > p.page_size;
    if (bad && threadIdx.x == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_COPY);
    if (from < 0 || to < 0 || from == to || bad || fill <= 0) return;
    const KvPlane& c = blockIdx.z ? p.vc : p.kc;
    const uint16_t* src = static_cast<const uint16_t*>(c.base) + from * c.page_stride + h * c.head_stride;
    uint16_t* dst = static_cast<uint16_t*>(c.base) + to * c.page_stride + h * c.head_stride;
    const int pieces = p.dim / 8, all = fill * pieces;
    for (int x0 = threadIdx.x; x0 < all; x0 += kCopyThreads * kCopyBatch) {
        uint4 v[kCopyBatch];
        int64_t at[kCopyBatch];
#pragma unroll
        for (int k = 0; k < kCopyBatch; ++k) {
            const int x = x0 + k * kCopyThreads, tok = x / pieces;
            at[k] = tok * c.token_stride + (x - tok * pieces) * 8;
            if (x < all) v[k] = *reinterpret_cast<const uint4*>(src + at[k]);
        }
#pragma unroll
        for (int k = 0; k < kCopyBatch; ++k)
            if (x0 + k * kCopyThreads < all) *reinterpret_cast<uint4*>(dst + at[k]) = v[k];
    }
    if (p.codes && blockIdx.z == 0) {
        const int64_t a = static_cast<int64_t>(from) * p.n_kv_heads + h, b = static_cast<int64_t>(to) * p.n_kv_heads + h;
        for (int x = threadIdx.x; x < p.dim / 16; x += kCopyThreads)
            *reinterpret_cast<uint4*>(p.codes + b * p.dim + x * 16) = *reinterpret_cast<const uint4*>(p.codes + a * p.dim + x * 16);
        if (threadIdx.x == 0) p.scales[b] = p.scales[a];
    }
}

}  // namespace ivf
