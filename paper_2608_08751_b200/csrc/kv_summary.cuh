// Summaries of cache blocks: the mean of a page's first `fill` keys for each kv head, coded in 8 bits.
//
// m = (1 / fill) * sum of the keys (32 bits; the tokens of the page, those past `fill` as zeros, are added by
// halving: token i + n/2 onto token i), scale = max|m| / 127, code = round(m / scale).  The order of the
// additions and the correctly rounded divisions make the codes the same whole numbers on every launch.
//
// Bound by memory: fill * D keys are read once, D + 4 bytes written.  One CTA per (page, head): D / 8 lanes
// span a token row with 16-byte loads, all loads of a thread are independent, and ten CTAs an SM keep enough of them
// under way (8,192 pages of 64 tokens by 8 heads of 128: 1.08 GB in 195 us, 5.5 TB/s; with room for 128 tokens in
// every thread's registers 260 us).  Wide heads with pages of 128 tokens do not fit the registers and spill: the same bytes by
// heads of 256 at 3.5 TB/s, of 192 at 3.1; with pages of 64 at 5.2.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kSumThreads = 128;

struct KvSummaryParams {
    KvPlane kc;
    int64_t num_pages;
    int n_kv_heads, dim, page_size;
    const int32_t *pages, *fills;
    int8_t* codes;  // [num_pages][n_kv_heads][dim]
    float* scales;  // [num_pages][n_kv_heads]
    int* status;
};

// LG lanes span a row (a power of two, LG * 8 >= D); kSumThreads / LG token rows are read at a time, DEEP of them by a
// thread: a page, no more, so that registers are left for many CTAs.
template <typename T, int LG, int DEEP>
__global__ void __launch_bounds__(kSumThreads, DEEP <= 8 ? 10 : 5) kv_summary_kernel(KvSummaryParams p) {
    constexpr int kRows = kSumThreads / LG;  // rows (tokens) side by side, a power of two
    constexpr int kDeep = DEEP;              // tokens of one thread
    __shared__ float s_part[kRows][LG * 8];
    __shared__ float s_max[kSumThreads / 32];
    const int item = blockIdx.x, h = blockIdx.y;
    const int page = p.pages[item];
    int fill = p.fills[item];
    if (page < 0 || fill == 0) {
        if ((page < -1 || fill < 0) && threadIdx.x == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_SUMMARIZE);
        return;  // padding of a touched list
    }
    if (page >= p.num_pages || fill < 0 || fill > p.page_size) {
        if (threadIdx.x == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_SUMMARIZE);
        return;
    }
    const int gl = threadIdx.x % LG, row = threadIdx.x / LG;
    const int e0 = gl * 8;
    const T* src = static_cast<const T*>(p.kc.base) + page * p.kc.page_stride + h * p.kc.head_stride + e0;
    // thread rows hold tokens row, row + kRows, ...: the halvings at distances >= kRows stay in registers
    float acc[8];
    {
        uint4 raw[kDeep];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int tok = row + j * kRows;
            raw[j] = make_uint4(0, 0, 0, 0);
            if (tok < fill && e0 < p.dim) raw[j] = *reinterpret_cast<const uint4*>(src + tok * p.kc.token_stride);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x[kDeep];
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                const uint32_t w = i / 2 == 0 ? raw[j].x : i / 2 == 1 ? raw[j].y : i / 2 == 2 ? raw[j].z : raw[j].w;
                const float2 v = Pair16<T>::unpack(w);
                x[j] = (i & 1) ? v.y : v.x;
            }
            acc[i] = halving_sum<kDeep>(x);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s_part[row][e0 + i] = acc[i];
    __syncthreads();
    const int live_rows = p.page_size < kRows ? p.page_size : kRows;  // rows past the page hold zeros
    float mean[(LG * 8 + kSumThreads - 1) / kSumThreads];
    float amax = 0.0f;
#pragma unroll
    for (int c = 0; c < (LG * 8 + kSumThreads - 1) / kSumThreads; ++c) {
        const int e = threadIdx.x + c * kSumThreads;
        mean[c] = 0.0f;
        if (e < p.dim) {
            float x[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r) x[r] = r < live_rows ? s_part[r][e] : 0.0f;
            mean[c] = __fdiv_rn(halving_sum<kRows>(x), static_cast<float>(fill));
            amax = max_magnitude(amax, mean[c]);
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = max_magnitude(max_magnitude(s_max[0], s_max[1]), max_magnitude(s_max[2], s_max[3]));
    const float scale = code_scale(amax);
    const int64_t at = static_cast<int64_t>(page) * p.n_kv_heads + h;
#pragma unroll
    for (int c = 0; c < (LG * 8 + kSumThreads - 1) / kSumThreads; ++c) {
        const int e = threadIdx.x + c * kSumThreads;
        if (e < p.dim) p.codes[at * p.dim + e] = static_cast<int8_t>(code_of(mean[c], scale));
    }
    if (threadIdx.x == 0) p.scales[at] = scale;
}

}  // namespace ivf
