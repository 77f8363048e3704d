// Selection of cache blocks for each new token and kv head by a cheap score.
//
// The query of a kv head is the sum u of its group's query heads, coded in 8 bits; block b scores
// fl(int(u^ . code_b) * scale_b).  The dot product is a whole number, so scores, order and ids are the same
// on every launch; ties go to the lower block.  Blocks 0 .. pos / page_size are visible; the first n_first
// and the last n_last of them are always taken, the best of the others fill up to n_select.  Ids come out
// ascending, -1 after the last.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kSelThreads = 256;
constexpr int kSelMaxBlocks = 49152;  // keys of one row in shared memory

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
__device__ __forceinline__ uint32_t sel_key(float score) {
    const uint32_t u = __float_as_uint(score + 0.0f);  // -0 counts as 0
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return min(max(k, 1u), 0xFFFFFFFEu);
}

// The group's coded query, dim bytes into s_code.  P: group rounded up to a power of two.
template <typename T, int P>
__device__ __forceinline__ void sel_query(const KvSelectParams& p, int64_t t, int h, int8_t* s_code, float* s_red) {
    const int e = threadIdx.x;
    float u = 0.0f;
    if (e < p.dim) {
        const T* src = static_cast<const T*>(p.q) + t * p.q_stride[0] + static_cast<int64_t>(h) * p.group * p.q_stride[1] + e;
        float x[P];
#pragma unroll
        for (int g = 0; g < P; ++g) x[g] = g < p.group ? static_cast<float>(src[g * p.q_stride[1]]) : 0.0f;
        u = halving_sum<P>(x);
    }
    float amax = fabsf(u);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, off));
    if ((e & 31) == 0) s_red[e >> 5] = amax;
    __syncthreads();
    amax = 0.0f;
    for (int w = 0; w < kSelThreads / 32; ++w) amax = fmaxf(amax, s_red[w]);
    if (e < p.dim) s_code[e] = static_cast<int8_t>(code_of(u, code_scale(amax)));
    __syncthreads();
}

__device__ __forceinline__ int sel_block_sum(int v, int* s_red) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = v;
    __syncthreads();
    int s = 0;
    for (int w = 0; w < kSelThreads / 32; ++w) s += s_red[w];
    return s;
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(KvSelectParams p) {
    extern __shared__ uint32_t sel_keys[];
    __shared__ __align__(16) int8_t s_code[kKvMaxDim];
    __shared__ float s_redf[kSelThreads / 32];
    __shared__ int s_red[kSelThreads / 32];
    const int64_t t = blockIdx.x;
    const int h = blockIdx.y, tid = threadIdx.x;
    int32_t* out = p.out + (t * p.n_kv_heads + h) * p.n_select;
    const int req = p.token_req[t], pos = p.token_pos[t];
    const bool padded = req < 0 || pos < 0;
    const bool bad = req >= p.n_req || (!padded && (pos >> p.page_shift) >= p.max_blocks);
    if (padded || bad) {
        if (bad && tid == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
        for (int i = tid; i < p.n_select; i += kSelThreads) out[i] = -1;
        return;
    }
    if (p.group <= 1) sel_query<T, 1>(p, t, h, s_code, s_redf);
    else if (p.group <= 2) sel_query<T, 2>(p, t, h, s_code, s_redf);
    else if (p.group <= 4) sel_query<T, 4>(p, t, h, s_code, s_redf);
    else if (p.group <= 8) sel_query<T, 8>(p, t, h, s_code, s_redf);
    else if (p.group <= 16) sel_query<T, 16>(p, t, h, s_code, s_redf);
    else sel_query<T, 64>(p, t, h, s_code, s_redf);

    const int n = (pos >> p.page_shift) + 1;
    const int32_t* row = p.table + req * p.table_stride;
    int valid = 0;
    for (int b = tid; b < n; b += kSelThreads) {
        const int page = row[b];
        uint32_t key = 0;
        if (page >= 0 && page < p.num_pages) {
            ++valid;
            if (b < p.n_first || b >= n - p.n_last) {
                key = 0xFFFFFFFFu;
            } else {
                const int64_t at = static_cast<int64_t>(page) * p.n_kv_heads + h;
                const int4* c = reinterpret_cast<const int4*>(p.codes + at * p.dim);
                int dot = 0;
                for (int i = 0; i < p.dim / 16; ++i) {
                    const int4 a = c[i], u = reinterpret_cast<const int4*>(s_code)[i];
                    dot = __dp4a(a.x, u.x, dot);
                    dot = __dp4a(a.y, u.y, dot);
                    dot = __dp4a(a.z, u.z, dot);
                    dot = __dp4a(a.w, u.w, dot);
                }
                key = sel_key(__fmul_rn(static_cast<float>(dot), p.scales[at]));
            }
        } else if (page >= p.num_pages) {
            kv_report(p.status, kKvStatusBadId, KV_SITE_SELECT);
        }
        sel_keys[b] = key;
    }
    const int total = sel_block_sum(valid, s_red);
    const int take = min(p.n_select, total);
    // the take-th largest key: bit by bit the largest threshold that at least `take` keys reach
    uint32_t thr = 1;
    if (total > p.n_select) {
        thr = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t cand = thr | (1u << bit);
            int c = 0;
            for (int b = tid; b < n; b += kSelThreads) c += sel_keys[b] >= cand;
            if (sel_block_sum(c, s_red) >= take) thr = cand;
        }
    }
    int above = 0;
    for (int b = tid; b < n; b += kSelThreads) above += sel_keys[b] > thr;
    const int equals = take - sel_block_sum(above, s_red);  // of the keys at the threshold, the lowest blocks
    // ascending ids: each thread owns a contiguous run of blocks
    const int per = (n + kSelThreads - 1) / kSelThreads;
    const int b0 = min(tid * per, n), b1 = min(b0 + per, n);
    int gt = 0, eq = 0;
    for (int b = b0; b < b1; ++b) gt += sel_keys[b] > thr, eq += sel_keys[b] == thr && thr > 0;
    __shared__ int s_scan[2][kSelThreads];
    s_scan[0][tid] = gt;
    s_scan[1][tid] = eq;
    __syncthreads();
    if (tid == 0) {
        int a = 0, c = 0;
        for (int i = 0; i < kSelThreads; ++i) {
            const int x = s_scan[0][i], y = s_scan[1][i];
            s_scan[0][i] = a;
            s_scan[1][i] = c;
            a += x;
            c += y;
        }
    }
    __syncthreads();
    int ngt = s_scan[0][tid], neq = s_scan[1][tid];
    for (int b = b0; b < b1; ++b) {
        const uint32_t k = sel_keys[b];
        if (k > thr) out[ngt++ + min(neq, equals)] = b;
        else if (k == thr && k > 0) {
            if (neq < equals) out[ngt + neq] = b;
            ++neq;
        }
    }
    for (int i = take + tid; i < p.n_select; i += kSelThreads) out[i] = -1;
}

}  // namespace ivf
