// Norm of queries and keys for each head, position rotation, and the write into the paged cache.
//
// For a head row x of D numbers with weight w:  y = x * rsqrt(mean(x^2) + eps) * w, then the first R entries
// are rotated in pairs (a, b) -> (a cos - b sin, a sin + b cos) by the angles of the token's position; a pair
// is (i, i + R/2), or (2i, 2i + 1) when interleaved.  All of it is in 32 bits and rounded once.  Queries go to
// q_out, keys and values to the cache slot of the token.
//
// Bound by memory: every row is read once and written once.  A row lies across D / 8 lanes, 16 bytes each;
// the sum of squares is a butterfly over those lanes and the halves of a pair meet by shuffle.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kAppThreads = 256;

struct KvAppendParams {
    const void *q, *k, *v;
    int64_t q_stride[2], k_stride[2], v_stride[2];  // token, head
    void* q_out;
    int64_t qo_stride[2];
    int64_t n_tokens;
    int n_heads, n_kv_heads, dim, page_shift;
    int64_t num_pages;
    KvPlane kc, vc;
    const int32_t* token_pos;
    const int64_t* token_slot;
    const float* rotary;  // [n_pos][rot_dim]: cosines, then sines
    int n_pos, rot_dim, interleaved;
    const float *q_weight, *k_weight;
    float eps;
    int* status;
};

// LG: lanes of a row (a power of two, LG * 8 >= D).
template <typename T, int LG>
__global__ void __launch_bounds__(kAppThreads) kv_append_kernel(KvAppendParams p) {
    constexpr int kGroups = kAppThreads / LG;
    const int64_t t = blockIdx.x;
    const int gl = threadIdx.x % LG, group = threadIdx.x / LG;
    const int e0 = gl * 8;
    const bool live = e0 < p.dim;
    const int pos = p.token_pos[t];
    const int64_t slot = p.token_slot ? p.token_slot[t] : -1;
    const bool bad_pos = p.rot_dim > 0 && pos >= p.n_pos;
    const bool bad_slot = slot >= (p.num_pages << p.page_shift);
    if (threadIdx.x == 0 && blockIdx.y == 0 && (bad_pos || bad_slot)) kv_report(p.status, kKvStatusBadId, KV_SITE_APPEND);
    const bool padded = pos < 0 || bad_pos;
    const bool store = !padded && slot >= 0 && !bad_slot;

    // the token's angles: entry e of the rotated part uses angle e (mod R/2), or e / 2 when interleaved
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
    const int half = p.rot_dim >> 1;
    const bool turned = live && e0 < p.rot_dim;
    if (turned && !padded) {
        const float* row = p.rotary + static_cast<int64_t>(pos) * p.rot_dim;
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cs[2 * i] = cs[2 * i + 1] = row[e0 / 2 + i];
                sn[2 * i] = sn[2 * i + 1] = row[half + e0 / 2 + i];
            }
        } else {
            const int a0 = e0 < half ? e0 : e0 - half;
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = row[a0 + i], sn[i] = row[half + a0 + i];
        }
    }
    const int partner = e0 < half ? gl + half / 8 : gl - half / 8;

    const int rows = p.n_heads + 2 * p.n_kv_heads;
    for (int r0 = blockIdx.y * kGroups; r0 < rows; r0 += gridDim.y * kGroups) {
        const int r = r0 + group;
        const bool is_q = r < p.n_heads, is_k = !is_q && r < p.n_heads + p.n_kv_heads;
        const bool is_v = !is_q && !is_k && r < rows;
        const int h = is_q ? r : is_k ? r - p.n_heads : r - p.n_heads - p.n_kv_heads;
        const T* src = is_q ? static_cast<const T*>(p.q) + t * p.q_stride[0] + h * p.q_stride[1]
                     : is_k ? static_cast<const T*>(p.k) + t * p.k_stride[0] + h * p.k_stride[1]
                            : static_cast<const T*>(p.v) + t * p.v_stride[0] + h * p.v_stride[1];
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (live && r < rows && !padded) raw = *reinterpret_cast<const uint4*>(src + e0);
        const int64_t page = store ? slot >> p.page_shift : 0, off = store ? slot & ((1 << p.page_shift) - 1) : 0;
        if (is_v) {
            if (store && live)
                *reinterpret_cast<uint4*>(static_cast<T*>(p.vc.base) + page * p.vc.page_stride + h * p.vc.head_stride +
                                          off * p.vc.token_stride + e0) = raw;
        }
        float x[8];
        unpack8<T>(raw, x);
        const float* w = is_q ? p.q_weight : p.k_weight;
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int off2 = LG / 2; off2 > 0; off2 >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, off2, LG);
        if (w != nullptr && live && !padded) {
            const float rn = rsqrtf(ss / static_cast<float>(p.dim) + p.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * rn * w[e0 + i];
        }
        float y[8];
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                y[i] = x[i] * cs[i] - x[i + 1] * sn[i];
                y[i + 1] = x[i] * sn[i] + x[i + 1] * cs[i];
            }
        } else {
            const float sign = e0 < half ? -1.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float o = __shfl_sync(0xFFFFFFFFu, x[i], turned ? partner : gl, LG);
                y[i] = x[i] * cs[i] + sign * o * sn[i];
            }
        }
        if (!turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i];  // past the rotated part: untouched, infinities too
        }
        if (!live) continue;
        if (is_q)
            *reinterpret_cast<uint4*>(static_cast<T*>(p.q_out) + t * p.qo_stride[0] + h * p.qo_stride[1] + e0) = pack8<T>(y);
        else if (is_k && store)
            *reinterpret_cast<uint4*>(static_cast<T*>(p.kc.base) + page * p.kc.page_stride + h * p.kc.head_stride +
                                      off * p.kc.token_stride + e0) = pack8<T>(y);
    }
}

}  // namespace ivf
