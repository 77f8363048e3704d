// Selection of cache blocks for each new token and kv head by a cheap score.
//
// The query of a kv head is the sum u of its group's query heads, coded in 8 bits; block b scores
// fl(int(u^ . code_b) * scale_b).  The dot product is a whole number, so scores, order and ids are the same
// on every launch; ties go to the lower block.  Blocks 0 .. pos / page_size are visible; the first n_first
// and the last n_last of them are always taken, the best of the others fill up to n_select.  Ids come out
// ascending, -1 after the last.
//
// Scores become 32-bit keys in shared memory (larger score, larger key) and never reach global memory.  The largest keys
// of parts of a row give a lower bound of its n_select-th largest key; what reaches it, a few more keys than are wanted,
// goes on a short list in block order, and among those the threshold is found bit by bit.  (Bit by bit over
// the whole row took 4,700 instructions of a warp for a row of 512 blocks.)
//
//   rows     (single and drafted tokens) a cluster of CTAs shares the blocks of one (token, kv head), 4-byte dot products
//            straight from the loads; the keys meet in the first CTA's shared memory.  32 requests of up to 4,096 blocks by 8
//            heads: 89 MB of codes in 37 us from call to call (14 at a copy's rate).  Stamps in the kernel: all CTAs run after
//            1.7 us, the last query is coded at 6.8, the scores are there at 19 on average and at 27 for the longest
//            rows (contexts are ragged, each row has the same three CTAs), the short list takes 4 more and the ids 2; the rest is
//            the change of kernels.  2,048 blocks of one request 11 us.
//   windows  (prompts) 16 tokens by one kv head to a CTA, scores by the integer matrix instruction, a warp selects a row.
//            Bound by the selection's instructions (about 2,500 of a warp for a row of 512 blocks): 16,384 rows in 57 us.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelMaxBlocks = 49152;  // keys of one row in shared memory
constexpr int kSelWindow = 16;        // tokens of a window: rows of the matrix instruction
// A row's short list.  What does not fit goes bit by bit over the whole row.  4,096 tokens by 4 heads of 512 random blocks,
// windows / rows kernel: 16 blocks a token 66 / 242 us, 48 70 / 250, 64 (of which the bound lets 227 through) 127 / 254, 256
// 117 / 299.
constexpr int kSelWindowList = 192;
// Blocks that a window's keys, pages and scales have room for in shared memory: not where the kernels cross.  Windows / rows
// kernel by blocks of a request (16 a token): 512 66 / 244 us, 1,024 139 / 348, 2,048 297 / 582, 2,688 358 / 735.
// The room is taken by the table's columns, not by the blocks in use: 512 blocks in a table of 1,024 columns 92 us, of 2,688 137.
constexpr int kSelWindowBlocks = 2688;

struct KvSelectParams {
    const void* q;
    int64_t q_stride[2];
    int64_t n_tokens;
    int group, n_kv_heads, dim;
    const int8_t* codes;
    const float* scales;
    int64_t num_pages;
    const int32_t* table;
    int64_t table_stride;
    int n_req, max_blocks, page_shift;
    const int32_t *token_req, *token_pos;
    int n_select, n_first, n_last;
    int32_t* out;
    int* status;
};

// Larger scores get larger keys; 0 is kept for blocks that cannot be taken, all ones for those always taken.
constexpr uint32_t kSelAlways = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t sel_key(int dot, float scale) {
    const uint32_t u = __float_as_uint(__fmul_rn(static_cast<float>(dot), scale) + 0.0f);  // -0 counts as 0
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return min(max(k, 1u), kSelAlways - 1);
}

// Sum of x(o), x(o + S), x(o + 2S) ... below P by halving: the same additions as halving_sum, without an array.
template <int P, int S, typename F>
__device__ __forceinline__ void sel_halving(float (&r)[8], int o, F&& load) {
    if constexpr (S >= P) {
        load(o, r);
    } else {
        float b[8];
        sel_halving<P, 2 * S>(r, o, load);
        sel_halving<P, 2 * S>(b, o + S, load);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = __fadd_rn(r[i], b[i]);
    }
}

// The coded query of (token t, kv head h) by one warp: 8 elements to a lane.  P: group rounded up to a power of two.
template <typename T, int P>
__device__ __forceinline__ uint2 sel_code_warp(const KvSelectParams& p, int64_t t, int h) {
    const int e0 = (threadIdx.x & 31) * 8;
    const T* src = static_cast<const T*>(p.q) + t * p.q_stride[0] + static_cast<int64_t>(h) * p.group * p.q_stride[1] + e0;
    float u[8];
    sel_halving<P, 1>(u, 0, [&](int g, float (&x)[8]) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (g < p.group && e0 < p.dim) v = *reinterpret_cast<const uint4*>(src + g * p.q_stride[1]);
        unpack8<T>(v, x);
    });
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max_magnitude(amax, u[i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
    const float scale = code_scale(amax);
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[k] |= static_cast<uint32_t>(code_of(u[4 * k + i], scale) & 255) << (8 * i);
    }
    return make_uint2(w[0], w[1]);
}
template <typename T>
__device__ __noinline__ uint2 sel_code(const KvSelectParams& p, int64_t t, int h) {
    if (p.group <= 1) return sel_code_warp<T, 1>(p, t, h);
    if (p.group <= 2) return sel_code_warp<T, 2>(p, t, h);
    if (p.group <= 4) return sel_code_warp<T, 4>(p, t, h);
    if (p.group <= 8) return sel_code_warp<T, 8>(p, t, h);
    if (p.group <= 16) return sel_code_warp<T, 16>(p, t, h);
    return sel_code_warp<T, 64>(p, t, h);
}

// ---------------------------------------------------------------------------------------------- from keys to ids, by a warp
// The k-th largest of the 64 numbers that the lanes hold two of each, rounded down to its upper 16 bits; 0 if there are
// fewer than k above 0.
__device__ __forceinline__ uint32_t sel_kth_of_64(uint32_t a, uint32_t b, int k) {
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t cand = t | (1u << bit);
        if (__popc(__ballot_sync(0xFFFFFFFFu, a >= cand)) + __popc(__ballot_sync(0xFFFFFFFFu, b >= cand)) >= k) t = cand;
    }
    return t;
}

// The largest scored keys of key[b0 .. b1), of even and of odd groups of 32.
__device__ __forceinline__ void sel_two_largest(const uint32_t* key, int b0, int b1, uint32_t& a, uint32_t& b) {
    a = b = 0;
    for (int i = b0 + (threadIdx.x & 31); i < b1; i += 64) {
        const uint32_t x = key[i], y = i + 32 < b1 ? key[i + 32] : 0u;
        if (x != kSelAlways) a = max(a, x);
        if (y != kSelAlways) b = max(b, y);
    }
}

// Writes the ids of the n_select largest of m keys in their order (all of them where there are fewer), -1 after the last.  Keys
// of 0 do not count, those always taken come first; equal keys go to the earlier.  id: the keys' blocks, null: 0, 1, 2 ...
__device__ __forceinline__ void sel_finish(const uint32_t* key, const int* id, int m, int n_select, int32_t* out) {
    const int lane = threadIdx.x & 31;
    constexpr int kHeld = 8;
    uint32_t held[kHeld];  // short lists stay in registers
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = i * 32 + lane < m ? key[i * 32 + lane] : 0u;
    const bool in_regs = m <= kHeld * 32;
    const int used = (m + 31) / 32;  // a list is mostly much shorter than what there is room for
    int always = 0, valid = 0;
    uint32_t all_or = 0, all_and = 0xFFFFFFFFu;
    auto look = [&](uint32_t k) {
        always += k == kSelAlways;
        valid += k != 0;
        if (k != 0 && k != kSelAlways) {
            all_or |= k;
            all_and &= k;
        }
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        if (i >= used) break;
        look(held[i]);
    }
    for (int b = kHeld * 32 + lane; b < m; b += 32) look(key[b]);
    always = __reduce_add_sync(0xFFFFFFFFu, always);
    valid = __reduce_add_sync(0xFFFFFFFFu, valid);
    const int take = min(n_select, valid), want = take - always;
    uint32_t thr = 1;  // larger keys are taken, and of those equal to it the first `spare`
    int spare = 0x7FFFFFFF;
    if (valid > n_select) {
        int at_least = valid - always;
        if (want <= 0) {
            thr = kSelAlways;
            at_least = always;
        } else {
            all_or = __reduce_or_sync(0xFFFFFFFFu, all_or);
            all_and = __reduce_and_sync(0xFFFFFFFFu, all_and);
            const int top = 31 - __clz((all_or ^ all_and) | 1u);
            thr = all_and & ~((2u << top) - 1);
            for (int bit = top; bit >= 0 && at_least != want; --bit) {
                const uint32_t cand = thr | (1u << bit);
                int cnt = 0;
                if (in_regs) {
#pragma unroll
                    for (int i = 0; i < kHeld; ++i) {
                        if (i >= used) break;
                        cnt += held[i] >= cand;
                    }
                } else {
                    for (int b = lane; b < m; b += 32) cnt += key[b] >= cand;
                }
                cnt = __reduce_add_sync(0xFFFFFFFFu, cnt) - always;
                if (cnt >= want) {
                    thr = cand;
                    at_least = cnt;
                }
            }
        }
        const int surplus = at_least - (want <= 0 ? take : want);
        if (surplus > 0) {
            int eq = 0;
            for (int b = lane; b < m; b += 32) eq += key[b] == thr;
            spare = __reduce_add_sync(0xFFFFFFFFu, eq) - surplus;
        }
    }
    int gt_before = 0, eq_before = 0;
    for (int b0 = 0; b0 < m; b0 += 32) {
        const int b = b0 + lane;
        const uint32_t k = b < m ? key[b] : 0u;
        const unsigned mg = __ballot_sync(0xFFFFFFFFu, k > thr), me = __ballot_sync(0xFFFFFFFFu, k == thr);
        const unsigned below = (1u << lane) - 1;
        const int g = gt_before + __popc(mg & below), e = eq_before + __popc(me & below);
        if (k > thr || (k == thr && e < spare)) out[g + min(e, spare)] = id ? id[b] : b;
        gt_before += __popc(mg);
        eq_before += __popc(me);
    }
    for (int i = take + lane; i < n_select; i += 32) out[i] = -1;
}

// ---------------------------------------------------------------------------------------------- rows
constexpr int kSelRowThreads = 128, kSelRowWarps = kSelRowThreads / 32;
constexpr int kSelRowCtas = 6;  // on an SM
// A row's short list.  Above 256 blocks a token there is no bound, and rows longer than the list go bit by bit: 32 requests by 8 heads
// of 2,048 blocks, 64 blocks a token 37 us, 128 39, 256 and 512 55.  (A table of more columns than 8,192 costs CTAs on an SM:
// 512 blocks in 2,048 columns 21 us, in 16,384 31, in 49,152 66.)
constexpr int kSelList = 1024;

// L lanes to a block's codes, NP pieces of 16 bytes each (16 L NP >= dim); four blocks of a lane group are in flight, their
// pages are fetched a step ahead.  Few lanes to a block: what is not a load is paid once for a block and lane.
template <typename T, int L, int NP>
__global__ void __launch_bounds__(kSelRowThreads, kSelRowCtas) kv_select_rows_kernel(KvSelectParams p) {
    extern __shared__ uint32_t sel_keys[];  // of the first CTA of the cluster: one key per visible block
    __shared__ __align__(16) int8_t s_code[kKvMaxDim];
    __shared__ uint32_t s_bound[kSelRowWarps];
    __shared__ int s_count[kSelRowWarps];
    __shared__ uint32_t s_key[kSelList];
    __shared__ int s_id[kSelList];
    constexpr int kDeep = 4;
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    const int64_t t = blockIdx.x / ranks;
    const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* out = p.out + (t * p.n_kv_heads + h) * p.n_select;
    if (warp == 0) {  // first of all: behind the codes its loads would wait for them
        const uint2 w = sel_code<T>(p, t, h);
        if (lane * 8 < p.dim) *reinterpret_cast<uint2*>(s_code + lane * 8) = w;
    }
    const int req = p.token_req[t], pos = p.token_pos[t];
    const bool padded = req < 0 || pos < 0;
    const bool bad = req >= p.n_req || (!padded && (pos >> p.page_shift) >= p.max_blocks);
    if (padded || bad) {  // the whole cluster
        if (rank == 0) {
            if (bad && tid == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
            for (int i = tid; i < p.n_select; i += kSelRowThreads) out[i] = -1;
        }
        return;
    }
    if (ranks > 1) cluster_arrive();
    const int n = (pos >> p.page_shift) + 1;
    const int32_t* row = p.table + req * p.table_stride;
    const uint32_t keys0 = cluster_addr(sel_keys, 0);

    // lane group g of the cluster takes blocks g, g + step, ...; kDeep of them at a time
    constexpr int kGroups = kSelRowThreads / L;
    const int sub = tid % L;
    const int step = kGroups * static_cast<int>(ranks);
    static_assert(kDeep == 4 && L >= kDeep, "a lane of the group finishes a block");
    int4 code[kDeep][NP];
    int page[kDeep], ahead[kDeep];
    auto pages_of = [&](int b0, int (&to)[kDeep]) {
#pragma unroll
        for (int i = 0; i < kDeep; ++i) to[i] = b0 + i * step < n ? row[b0 + i * step] : -1;
    };
    const int8_t* codes = p.codes + static_cast<int64_t>(h) * p.dim + sub * 16;
    const int64_t page_bytes = static_cast<int64_t>(p.n_kv_heads) * p.dim;
    auto codes_of = [&]() {
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const bool ok = page[i] >= 0 && page[i] < p.num_pages;
            const int8_t* src = codes + (ok ? page[i] * page_bytes : 0);
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                code[i][k] = make_int4(0, 0, 0, 0);
                if (ok && (sub + k * L) * 16 < p.dim) code[i][k] = *reinterpret_cast<const int4*>(src + k * L * 16);
            }
        }
    };
    const int first = static_cast<int>(rank) * kGroups + tid / L;
    pages_of(first, page);
    pages_of(first + kDeep * step, ahead);
    codes_of();
    __syncthreads();
    int4 u[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        u[k] = make_int4(0, 0, 0, 0);
        if ((sub + k * L) * 16 < p.dim) u[k] = *reinterpret_cast<const int4*>(s_code + (sub + k * L) * 16);
    }
    if (ranks > 1) cluster_wait();  // the first CTA runs, so its shared memory may be written
    for (int b0 = first; b0 - tid / L < n; b0 += kDeep * step) {
        // lane `sub` of the group finishes block `sub` of the four
        const int mine = sub == 0 ? page[0] : sub == 1 ? page[1] : sub == 2 ? page[2] : page[3];
        const bool there = sub < kDeep && mine >= 0 && mine < p.num_pages;
        const float scale = there ? p.scales[static_cast<int64_t>(mine) * p.n_kv_heads + h] : 0.0f;
        int dot[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            dot[i] = 0;
#pragma unroll
            for (int k = 0; k < NP; ++k)
                dot[i] = __dp4a(code[i][k].w, u[k].w, __dp4a(code[i][k].z, u[k].z, __dp4a(code[i][k].y, u[k].y, __dp4a(code[i][k].x, u[k].x, dot[i]))));
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) page[i] = ahead[i];
        codes_of();
        pages_of(b0 + 2 * kDeep * step, ahead);
        // sums over the group, each lane keeping its own block's: lanes apart by 1 exchange odd and even blocks, by 2 the pairs
        const int e0 = sub & 1 ? dot[0] : dot[1], e1 = sub & 1 ? dot[2] : dot[3];
        int k0 = (sub & 1 ? dot[1] : dot[0]) + __shfl_xor_sync(0xFFFFFFFFu, e0, 1), k1 = (sub & 1 ? dot[3] : dot[2]) + __shfl_xor_sync(0xFFFFFFFFu, e1, 1);
        int sum = (sub & 2 ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, sub & 2 ? k0 : k1, 2);
#pragma unroll
        for (int off = 4; off < L; off <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
        const int b = b0 + sub * step;
        if (sub < kDeep && b < n) {
            uint32_t key = 0;
            if (there) key = b < p.n_first || b >= n - p.n_last ? kSelAlways : sel_key(sum, scale);
            else if (mine >= p.num_pages) kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
            cluster_store(keys0 + b * 4, key);
        }
    }
    if (ranks > 1) cluster_sync();
    else __syncthreads();
    if (rank != 0) return;

    // ---- the short list: every warp takes a part of the row.  At least ceil(n_select / 4) scored keys of each part reach
    // the smallest of the parts' bounds, so at least n_select of the row do
    const int per = (n + kSelRowThreads - 1) / kSelRowThreads * 32;
    const int w0 = min(warp * per, n), w1 = min(w0 + per, n);
    uint32_t a, b;
    sel_two_largest(sel_keys, w0, w1, a, b);
    const uint32_t bound_w = sel_kth_of_64(a, b, (p.n_select + kSelRowWarps - 1) / kSelRowWarps);
    if (lane == 0) s_bound[warp] = bound_w;
    __syncthreads();
    uint32_t bound = s_bound[0];
#pragma unroll
    for (int w = 1; w < kSelRowWarps; ++w) bound = min(bound, s_bound[w]);
    bound = max(bound, 1u);
    int count = 0;
    for (int i = w0 + lane; i < w1; i += 32) count += sel_keys[i] >= bound;
    count = __reduce_add_sync(0xFFFFFFFFu, count);
    if (lane == 0) s_count[warp] = count;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kSelRowWarps; ++w) {
        if (w < warp) before += s_count[w];
        total += s_count[w];
    }
    if (total <= kSelList) {
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < w1 ? sel_keys[i] : 0u;
            const unsigned m = __ballot_sync(0xFFFFFFFFu, k >= bound);
            if (k >= bound) {
                const int at = before + __popc(m & ((1u << lane) - 1));
                s_key[at] = k;
                s_id[at] = i;
            }
            before += __popc(m);
        }
    }
    __syncthreads();
    if (warp == 0) {
        if (total <= kSelList) sel_finish(s_key, s_id, total, p.n_select, out);
        else sel_finish(sel_keys, nullptr, n, p.n_select, out);
    }
}

// ---------------------------------------------------------------------------------------------- windows
__device__ __forceinline__ void mma_s8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

inline size_t sel_window_smem(int blocks) {
    const int padded = (blocks + 63) / 64 * 64;
    return static_cast<size_t>(kSelWindow + 2) * padded * 4;
}

// K: steps of 32 elements (32 * K >= dim).  A dot product may take its elements in any order: lane q of a block's four lanes
// takes elements 8 K q .. 8 K (q + 1), so that its loads are contiguous, and the query's fragments do the same.
template <typename T, int K>
__global__ void __launch_bounds__(kSelThreads, 4) kv_select_windows_kernel(KvSelectParams p, int padded) {
    extern __shared__ uint32_t sel_smem[];
    uint32_t* keys = sel_smem;                                        // [16][padded]
    int* s_page = reinterpret_cast<int*>(keys + kSelWindow * padded);  // [padded]
    float* s_scale = reinterpret_cast<float*>(s_page + padded);        // [padded]
    __shared__ __align__(16) int8_t s_code[kSelWindow][32 * K];
    __shared__ int s_req[kSelWindow], s_pos[kSelWindow];
    __shared__ uint32_t s_key[kSelWarps][kSelWindowList];
    __shared__ int s_id[kSelWarps][kSelWindowList];
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kSelWindow;
    const int tokens = static_cast<int>(min(static_cast<int64_t>(kSelWindow), p.n_tokens - t0));
    const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid < kSelWindow) {
        int req = -1, pos = -1;
        if (tid < tokens) {
            req = p.token_req[t0 + tid];
            pos = p.token_pos[t0 + tid];
            if (req >= p.n_req || (req >= 0 && pos >= 0 && (pos >> p.page_shift) >= p.max_blocks)) {
                kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
                req = -1;
            }
            if (pos < 0) req = -1;
        }
        s_req[tid] = req;
        s_pos[tid] = pos;
    }
    for (int r = warp; r < kSelWindow; r += kSelWarps) {
        if (r < tokens) {
            const uint2 w = sel_code<T>(p, t0 + r, h);
            if (lane * 8 < 32 * K) *reinterpret_cast<uint2*>(&s_code[r][lane * 8]) = lane * 8 < p.dim ? w : make_uint2(0, 0);
        } else if (lane * 8 < 32 * K) {
            *reinterpret_cast<uint2*>(&s_code[r][lane * 8]) = make_uint2(0, 0);
        }
    }
    __syncthreads();
    const int q = lane & 3, nb = lane >> 2;
    uint32_t a[K][4];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        a[k][0] = *reinterpret_cast<const uint32_t*>(&s_code[nb][q * 8 * K + k * 8]);
        a[k][1] = *reinterpret_cast<const uint32_t*>(&s_code[nb + 8][q * 8 * K + k * 8]);
        a[k][2] = *reinterpret_cast<const uint32_t*>(&s_code[nb][q * 8 * K + k * 8 + 4]);
        a[k][3] = *reinterpret_cast<const uint32_t*>(&s_code[nb + 8][q * 8 * K + k * 8 + 4]);
    }
    // one request after the other: mostly there is one
    for (int r0 = 0; r0 < tokens;) {
        const int req = s_req[r0];
        int r1 = r0, last = -1;
        while (r1 < tokens && s_req[r1] == req) last = max(last, s_pos[r1++]);
        const int n = req < 0 ? 0 : (last >> p.page_shift) + 1;
        bool gaps = false;  // blocks without a page
        for (int b = tid; b < n; b += kSelThreads) {
            int page = p.table[req * p.table_stride + b];
            float scale = 0.0f;
            if (page >= p.num_pages) {
                kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
                page = -1;
            }
            if (page >= 0) scale = p.scales[static_cast<int64_t>(page) * p.n_kv_heads + h];
            gaps |= page < 0;
            s_page[b] = page;
            s_scale[b] = scale;
        }
        gaps = __syncthreads_or(gaps);
        const bool keep[2] = {nb >= r0 && nb < r1, nb + 8 >= r0 && nb + 8 < r1};
        // two tiles of 8 blocks to a warp at a time; their codes are fetched a step ahead
        uint32_t code[2][2 * K];
        auto fetch = [&](int b0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int b = b0 + i * 8 + nb;
                const int page = b < n ? s_page[b] : -1;
                const int8_t* src = p.codes + (page >= 0 ? static_cast<int64_t>(page) * p.n_kv_heads + h : 0) * p.dim;
                const int e0 = q * 8 * K;
                if constexpr (K % 2 == 0) {
#pragma unroll
                    for (int k = 0; k < K; k += 2) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (page >= 0 && e0 + k * 8 < p.dim) v = *reinterpret_cast<const uint4*>(src + e0 + k * 8);
                        code[i][2 * k] = v.x, code[i][2 * k + 1] = v.y, code[i][2 * k + 2] = v.z, code[i][2 * k + 3] = v.w;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        uint2 v = make_uint2(0, 0);
                        if (page >= 0 && e0 + k * 8 < p.dim) v = *reinterpret_cast<const uint2*>(src + e0 + k * 8);
                        code[i][2 * k] = v.x, code[i][2 * k + 1] = v.y;
                    }
                }
            }
        };
        fetch(warp * 16);
        for (int b0 = warp * 16; b0 < n; b0 += kSelWarps * 16) {
            int c[2][4] = {};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                mma_s8(c[0], a[k], code[0][2 * k], code[0][2 * k + 1]);
                mma_s8(c[1], a[k], code[1][2 * k], code[1][2 * k + 1]);
            }
            fetch(b0 + kSelWarps * 16);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int b = b0 + i * 8 + 2 * q + y;
                    if (b < n) {
                        const float scale = s_scale[b];
                        uint32_t lo = sel_key(c[i][y], scale), hi = sel_key(c[i][y + 2], scale);
                        if (gaps && s_page[b] < 0) lo = hi = 0;
                        if (keep[0]) keys[nb * padded + b] = lo;
                        if (keep[1]) keys[(nb + 8) * padded + b] = hi;
                    }
                }
            }
        }
        __syncthreads();
        // a warp selects a row
        for (int r = r0 + warp; r < r1; r += kSelWarps) {
            int32_t* out = p.out + ((t0 + r) * p.n_kv_heads + h) * p.n_select;
            uint32_t* key = keys + r * padded;
            const int m = req < 0 ? 0 : (s_pos[r] >> p.page_shift) + 1;
            for (int i = lane; i < p.n_first + p.n_last; i += 32) {  // those always taken, as far as they are there
                const int b = i < p.n_first ? i : m - 1 - (i - p.n_first);
                if (b >= 0 && b < m && key[b] != 0) key[b] = kSelAlways;
            }
            __syncwarp();
            uint32_t x = 0, y = 0, bound;
            int total = 0;
            auto enlist = [&](uint32_t k, int b) {
                const unsigned in = __ballot_sync(0xFFFFFFFFu, k >= bound);
                if (k >= bound) {
                    const int at = total + __popc(in & ((1u << lane) - 1));
                    s_key[warp][at] = k;
                    s_id[warp][at] = b;
                }
                total += __popc(in);
            };
            constexpr int kHeld = 16;  // a row of up to 512 keys stays in registers between the bound and the list
            if (m <= kHeld * 32) {
                uint32_t held[kHeld];
#pragma unroll
                for (int i = 0; i < kHeld; ++i) {
                    held[i] = i * 32 + lane < m ? key[i * 32 + lane] : 0u;
                    const uint32_t k = held[i] == kSelAlways ? 0u : held[i];
                    if (i & 1) y = max(y, k);
                    else x = max(x, k);
                }
                bound = max(sel_kth_of_64(x, y, p.n_select), 1u);
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (i * 32 < m && total <= kSelWindowList - 32) enlist(held[i], i * 32 + lane);
            } else {
                sel_two_largest(key, 0, m, x, y);
                bound = max(sel_kth_of_64(x, y, p.n_select), 1u);
                for (int b0 = 0; b0 < m && total <= kSelWindowList - 32; b0 += 32) enlist(b0 + lane < m ? key[b0 + lane] : 0u, b0 + lane);
            }
            __syncwarp();
            if (total <= kSelWindowList - 32) sel_finish(s_key[warp], s_id[warp], total, p.n_select, out);
            else sel_finish(key, nullptr, m, p.n_select, out);
            __syncwarp();
        }
        __syncthreads();
        r0 = r1;
    }
}

}  // namespace ivf
