// Norm of queries and keys for each head, position rotation, and the write into the paged cache.
//
// For a head row x of D numbers with weight w:  y = x * rsqrt(mean(x^2) + eps) * w, then the first R entries
// are rotated in pairs (a, b) -> (a cos - b sin, a sin + b cos) by the angles of the token's position; a pair
// is (i, i + R/2), or (2i, 2i + 1) when interleaved.  All of it is in 32 bits and rounded once.  Queries go to
// q_out, keys and values to the cache slot of the token.
//
// Bound by memory: every row is read once and written once.  A row lies across D / 8 lanes; a lane of the rotated part
// holds four elements and their four partners (with 16-byte pieces the partners met by eight shuffles a row), so the
// only exchange is the butterfly of the sum of squares.  411 MB of 16,384 tokens move in 84 us (4.9 TB/s); 37 tokens take 2.4 us.
#pragma once
#include "kv_common.cuh"

namespace ivf {

constexpr int kAppThreads = 64;

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

__device__ __forceinline__ void app_load4(const float* p, float (&f)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
}

// LG: lanes of a row (a power of two, LG * 8 >= D).  PAIRS: neighbours are rotated, not halves.  A CTA takes one token; its lane
// groups take the token's query heads, then its keys, then its values (of few tokens each CTA takes a part of them:
// gridDim.y > 1).  Weights, cosines and sines of a lane are multiplied once for all rows: (a, b) -> rn (a A - b B, a C + b D).
// Small CTAs: the wait for a token's angles and rows is filled by other tokens (16,384 tokens of 48 rows of 128:
// 149 us with 256 threads, 97 us with 128, 91 us with 64).
template <typename T, int LG, bool PAIRS>
__global__ void __launch_bounds__(kAppThreads, 12) kv_append_kernel(KvAppendParams p) {
    constexpr int kGroups = kAppThreads / LG, kDeep = 4;
    const int64_t t = blockIdx.x;
    const int gl = threadIdx.x % LG;
    const int group = threadIdx.x / LG;
    // which rows: all of the token's, or one part
    const int q_parts = (p.n_heads + kGroups - 1) / kGroups, kv_parts = (p.n_kv_heads + kGroups - 1) / kGroups;
    const bool whole = gridDim.y == 1;
    const int part = blockIdx.y;
    const bool do_q = whole || part < q_parts, do_k = whole || (part >= q_parts && part < q_parts + kv_parts), do_v = whole || part >= q_parts + kv_parts;
    const int first = group + (whole ? 0 : (part < q_parts ? part : part < q_parts + kv_parts ? part - q_parts : part - q_parts - kv_parts) * kGroups);
    const int stride = whole ? kGroups : 1 << 20;  // a part has one row to a group
    const bool live = gl * 8 < p.dim;
    // two pieces of four elements: i and i + R/2 where halves are rotated, neighbours elsewhere
    const int half = p.rot_dim >> 1;
    const bool in_turn = live && gl * 8 < p.rot_dim;
    const bool split = in_turn && !PAIRS;
    const int e0 = split ? gl * 4 : gl * 8, e1 = split ? half + gl * 4 : gl * 8 + 4;
    const int pos = p.token_pos[t];
    const int64_t slot = p.token_slot[t];

    // rows first, first + stride, ... of a tensor's `count`: kDeep loads in flight
    uint2 raw[kDeep][2];
    auto fetch = [&](const void* base, const int64_t* st, int r, int count) {
        const T* src = static_cast<const T*>(base) + t * st[0] + r * st[1];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            raw[i][0] = raw[i][1] = make_uint2(0, 0);
            if (live && r + i * stride < count) {
                raw[i][0] = *reinterpret_cast<const uint2*>(src + e0);
                raw[i][1] = *reinterpret_cast<const uint2*>(src + e1);
            }
            src += stride * st[1];
        }
    };
    // (of a padded token too: its rows are there)
    if (do_q) fetch(p.q, p.q_stride, first, p.n_heads);
    else if (do_k) fetch(p.k, p.k_stride, first, p.n_kv_heads);
    uint4 v_row[2];
    const T* v_src = static_cast<const T*>(p.v) + t * p.v_stride[0] + gl * 8;
    if (do_v && live) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (first + i * stride < p.n_kv_heads) v_row[i] = *reinterpret_cast<const uint4*>(v_src + (first + i * stride) * p.v_stride[1]);
    }

    const bool bad_pos = p.rot_dim > 0 && pos >= p.n_pos;
    const bool bad_slot = slot >= (p.num_pages << p.page_shift);
    const bool padded = pos < 0 || bad_pos;
    const bool store = !padded && slot >= 0 && !bad_slot;
    if (threadIdx.x == 0 && blockIdx.y == 0 && (bad_pos || bad_slot)) kv_report(p.status, kKvStatusBadId, KV_SITE_APPEND);
    const bool turned = in_turn && !padded;
    float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {};
    if (turned) {
        const float* row = p.rotary + static_cast<int64_t>(pos) * p.rot_dim + gl * 4;
        app_load4(row, cs);
        app_load4(row + half, sn);
    }
    const float inv_dim = 1.0f / static_cast<float>(p.dim);

    // norm and rotation of `count` rows, to dst + row * dst_stride
    auto turn = [&](const void* base, const int64_t* st, int count, const float* weight, T* dst, int64_t dst_stride) {
        float A[4], B[4], C[4], D[4];
        {
            float wx[4] = {1.f, 1.f, 1.f, 1.f}, wy[4] = {1.f, 1.f, 1.f, 1.f};
            if (weight != nullptr && live) {
                app_load4(weight + e0, wx);
                app_load4(weight + e1, wy);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float wa = PAIRS ? (j < 2 ? wx[2 * j] : wy[2 * j - 4]) : wx[j], wb = PAIRS ? (j < 2 ? wx[2 * j + 1] : wy[2 * j - 3]) : wy[j];
                A[j] = wa * cs[j], B[j] = wb * sn[j], C[j] = wa * sn[j], D[j] = wb * cs[j];
            }
        }
        T* to = dst + first * dst_stride;
        for (int r = first; r - group < count; r += kDeep * stride) {
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                if (r + i * stride - group >= count) break;  // the same for the whole CTA
                const float2 f0 = Pair16<T>::unpack(raw[i][0].x), f1 = Pair16<T>::unpack(raw[i][0].y);
                const float2 f2 = Pair16<T>::unpack(raw[i][1].x), f3 = Pair16<T>::unpack(raw[i][1].y);
                float a[4], b[4];
                if (PAIRS) a[0] = f0.x, b[0] = f0.y, a[1] = f1.x, b[1] = f1.y, a[2] = f2.x, b[2] = f2.y, a[3] = f3.x, b[3] = f3.y;
                else a[0] = f0.x, a[1] = f0.y, a[2] = f1.x, a[3] = f1.y, b[0] = f2.x, b[1] = f2.y, b[2] = f3.x, b[3] = f3.y;
                float rn = 1.0f;
                if (weight != nullptr) {
                    float ss = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
#pragma unroll
                    for (int d = LG / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, d, LG);
                    rn = rsqrtf(fmaf(ss, inv_dim, p.eps));
                }
                float x[4], y[4];
                if (in_turn) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[j] = rn * (a[j] * A[j] - b[j] * B[j]);
                        y[j] = rn * (a[j] * C[j] + b[j] * D[j]);
                    }
                } else {  // past the rotated part: infinities stay where they are
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = rn * (a[j] * A[j]), y[j] = rn * (b[j] * D[j]);
                }
                uint2 o0, o1;
                if (PAIRS) {
                    o0 = make_uint2(Pair16<T>::pack(x[0], y[0]), Pair16<T>::pack(x[1], y[1]));
                    o1 = make_uint2(Pair16<T>::pack(x[2], y[2]), Pair16<T>::pack(x[3], y[3]));
                } else {
                    o0 = make_uint2(Pair16<T>::pack(x[0], x[1]), Pair16<T>::pack(x[2], x[3]));
                    o1 = make_uint2(Pair16<T>::pack(y[0], y[1]), Pair16<T>::pack(y[2], y[3]));
                }
                if (padded) o0 = o1 = make_uint2(0, 0);
                if (live && r + i * stride < count) {
                    *reinterpret_cast<uint2*>(to + e0) = o0;
                    *reinterpret_cast<uint2*>(to + e1) = o1;
                }
                to += stride * dst_stride;
            }
            if (r - group + kDeep * stride < count) fetch(base, st, r + kDeep * stride, count);
        }
    };
    if (do_q) {
        turn(p.q, p.q_stride, p.n_heads, p.q_weight, static_cast<T*>(p.q_out) + t * p.qo_stride[0], p.qo_stride[1]);
        if (do_k) fetch(p.k, p.k_stride, first, p.n_kv_heads);
    }
    if (!store) return;  // (the whole CTA)
    const int64_t page = slot >> p.page_shift, off = slot & ((1 << p.page_shift) - 1);
    if (do_v && live) {
        T* dst = static_cast<T*>(p.vc.base) + page * p.vc.page_stride + off * p.vc.token_stride + gl * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (first + i * stride < p.n_kv_heads) *reinterpret_cast<uint4*>(dst + (first + i * stride) * p.vc.head_stride) = v_row[i];
        for (int r = first + 2 * stride; r < p.n_kv_heads; r += stride)
            *reinterpret_cast<uint4*>(dst + r * p.vc.head_stride) = *reinterpret_cast<const uint4*>(v_src + r * p.v_stride[1]);
    }
    if (do_k)
        turn(p.k, p.k_stride, p.n_kv_heads, p.k_weight, static_cast<T*>(p.kc.base) + page * p.kc.page_stride + off * p.kc.token_stride,
             p.kc.head_stride);
}

}  // namespace ivf
