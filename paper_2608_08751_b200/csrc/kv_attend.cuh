// Attention of each new token over the cache blocks selected for it.
//
// out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), s_j = scale * q . k_j, over the tokens j of the selected
// blocks at positions <= pos; lse = m + log(sum).  One pass over the keys with a running maximum and sum, both
// in 32 bits.  As operands of the second product the exponentials take the cache's 16-bit type, since the matrix instruction
// wants one type for both: each is off by up to 2^-8 (bfloat16) or 2^-11 (float16) of itself, an output by as much of the
// weighted mean of |v|.  Where it costs nothing, in the rows kernel for up to 8 query heads to a kv head, they are carried in two
// parts, rounding and rest (2^-16, 2^-22).
#pragma once
#include "kv_common.cuh"

namespace ivf {

struct KvAttendParams {
    const void* q;
    int64_t q_stride[2];
    int64_t n_tokens;
    int group, n_kv_heads, dim;
    KvPlane kc, vc;
    int64_t num_pages;
    const int32_t* table;
    int64_t table_stride;
    int n_req, max_blocks, page_shift;
    const int32_t *token_req, *token_pos, *selected;
    int n_select;
    float scale_log2;  // scale * log2(e)
    void* out;
    int64_t out_stride[2];
    float* lse;  // [n_tokens][n_heads] or null
    int* status;
    int window;          // tokens of a window of the tile kernel; 0 where the rows kernel runs alone
    uint64_t limit_ns;
};

// What the tile kernel leaves to the rows kernel it marks in the output itself: the first four bytes of a token's row, one mark
// for each kv head and 16 query heads of its group.  No finished row can hold it: both halves are NaN in either type, and a
// finished window is finite.  (No memory of the library's own: calls of several streams and captured graphs share nothing.)
constexpr uint32_t kKvLeft = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t* kv_mark(const KvAttendParams& p, int64_t t, int h, int part) {
    return reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + t * p.out_stride[0] +
                                       (static_cast<int64_t>(h) * p.group + part * 16) * p.out_stride[1]);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ bool is_finite(float x) { return x - x == 0.0f; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {
    const int n = ok ? 16 : 0;  // the rest is filled with zeros
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------------------------- rows
// A cluster of CTAs per (token, kv head, 16 query heads of its group).  The group's heads are the 16 rows of the matrix
// product, the keys come in pieces of 16 tokens.  Each warp takes pieces of its own through a ring of its own
// and keeps its own running maximum, sum and output; the warps meet once, at the end, and then the cluster's CTAs,
// through each other's shared memory.  Bound by the selected pages' bytes: 64 tokens by 8 heads of 32 pages, 537 MB, in
// 92 us (5.8 TB/s, 0.90 of a copy's rate); one token by 4 heads of 96, 3 MB, in 9.1 us, a chain of waits: request, block,
// page, keys, and two meetings.
constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = kRowsWarps * 32;

template <int DP>
struct RowsShape {
    static constexpr int kStages = DP == 64 ? 4 : 3;  // two CTAs on an SM (one for wide heads)
    static constexpr int kPlaneBytes = 16 * DP * 2;         // 16 tokens
    static constexpr int kStageBytes = 2 * kPlaneBytes;     // keys and values
    static constexpr int kRing = kRowsWarps * kStages * kStageBytes;
    static constexpr int kQBytes = 16 * DP * 2;
    static constexpr int kMergeBytes = kRowsWarps * 16 * (DP + 8) * 4;  // over the ring, after the loop
    static constexpr int kSmem = (kRing > kMergeBytes ? kRing : kMergeBytes) + kQBytes;
};

// Address of 16-byte piece c of row r in a tile of DP-wide 16-bit rows: pieces are exchanged by the row's low
// bits, so that the eight rows of a matrix load lie in different banks.
template <int DP>
__device__ __forceinline__ uint32_t rows_addr(uint32_t base, int r, int c) {
    return base + r * (DP * 2) + ((c ^ (r & 7)) << 4);
}

//
// SPLIT: at most 8 query heads.  The product's other 8 rows then take the second parts of the weights, and their sums are added at
// the end.  (With rows of their own the second parts are a second product: 64 tokens by 8 heads of a group of 16 took
// 121 us with it, next to the first or apart from it, 110 without; so larger groups go without.)
template <typename T, int DP, bool SPLIT>
__device__ __forceinline__ void attend_rows(const KvAttendParams& p, const int64_t t, const int rank, const int ranks, uint8_t* rows_smem, int* s_page, int* s_first, int& s_n) {
    using S = RowsShape<DP>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = blockIdx.y, g0 = blockIdx.z * 16;
    const int rows = min(16, p.group - g0);
    const int n_heads = p.group * p.n_kv_heads;
    const int head0 = h * p.group + g0;
    const int req = p.token_req[t], pos = p.token_pos[t];
    const bool live = req >= 0 && req < p.n_req && pos >= 0;
    if (req >= p.n_req && tid == 0) kv_report(p.status, kKvStatusBadId, KV_SITE_ATTEND);

    // the pages to read, in the order given
    if (tid == 0) s_n = 0;
    __syncthreads();
    if (warp == 0 && live) {
        const int32_t* sel = p.selected + (t * p.n_kv_heads + h) * p.n_select;
        int n = 0;
        for (int i0 = 0; i0 < p.n_select; i0 += 32) {
            const int i = i0 + lane;
            const int b = i < p.n_select ? sel[i] : -1;
            int page = -1;
            const bool want = b >= 0 && b <= (pos >> p.page_shift);
            if (want && b < p.max_blocks) page = p.table[req * p.table_stride + b];
            if (want && (b >= p.max_blocks || page >= p.num_pages)) {
                kv_report(p.status, kKvStatusBadId, KV_SITE_ATTEND);
                page = -1;
            }
            const unsigned m = __ballot_sync(0xFFFFFFFFu, page >= 0);
            if (page >= 0) {
                const int at = n + __popc(m & ((1u << lane) - 1));
                s_page[at] = page;
                s_first[at] = b << p.page_shift;
            }
            n += __popc(m);
        }
        if (lane == 0) s_n = n;
    }
    // queries: 16 rows, zeros past the group and past dim
    const uint32_t smem0 = smem_u32(rows_smem);
    const uint32_t s_q = smem0 + S::kSmem - S::kQBytes;
    for (int i = tid; i < 16 * (DP / 8); i += kRowsThreads) {
        const int r = i / (DP / 8), c = i % (DP / 8);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rows && c * 8 < p.dim)
            v = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + t * p.q_stride[0] + (head0 + r) * p.q_stride[1] + c * 8);
        *reinterpret_cast<uint4*>(rows_smem + (rows_addr<DP>(s_q, r, c) - smem0)) = v;
    }
    __syncthreads();
    const int per = 1 << (p.page_shift - 4);  // pieces of 16 tokens in a page
    const int pieces = s_n * per;
    const uint32_t ring = smem0 + warp * (S::kStages * S::kStageBytes);
    const int ksteps = p.dim >> 4;
    const int first = rank * kRowsWarps + warp, stride = ranks * kRowsWarps;  // this warp's pieces

    auto fetch = [&](int piece, int stage) {
        if (piece < pieces) {
            const int e = piece / per, part = piece % per;
            const int64_t page = s_page[e];
            const int tok0 = part * 16;
            const int seen = pos - s_first[e] - tok0;  // tokens 0 .. seen of the piece count
            const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + S::kPlaneBytes;
            const T* ks = static_cast<const T*>(p.kc.base) + page * p.kc.page_stride + h * p.kc.head_stride;
            const T* vs = static_cast<const T*>(p.vc.base) + page * p.vc.page_stride + h * p.vc.head_stride;
            if (seen >= 0) {
                // a lane keeps its column, its rows follow at a fixed distance
                constexpr int kLanes = DP / 8 < 32 ? DP / 8 : 32, kRowsAtOnce = 32 / kLanes;
                const int c = lane % kLanes, r0 = lane / kLanes;
                const T* kp = ks + (tok0 + r0) * p.kc.token_stride + c * 8;
                const T* vp = vs + (tok0 + r0) * p.vc.token_stride + c * 8;
                if (c * 8 < p.dim) {
#pragma unroll
                    for (int r = r0; r < 16; r += kRowsAtOnce) {
                        const bool ok = r <= seen;  // what lies past the token is never read: it may hold anything
                        cp_async16(rows_addr<DP>(kb, r, c), ok ? kp : ks, ok);
                        cp_async16(rows_addr<DP>(vb, r, c), ok ? vp : vs, ok);
                        kp += kRowsAtOnce * p.kc.token_stride;
                        vp += kRowsAtOnce * p.vc.token_stride;
                    }
                }
            }
        }
        cp_async_commit();
    };

    uint32_t qf[DP / 16][4];
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) ldsm4(qf[k], rows_addr<DP>(s_q, lane & 15, 2 * k + (lane >> 4)));
    float o[DP / 8][4];
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) fetch(first + s * stride, s);
    int stage = 0;
    for (int piece = first; piece < pieces; piece += stride) {
        cp_async_wait<S::kStages - 2>();
        __syncwarp();
        fetch(piece + (S::kStages - 1) * stride, stage == 0 ? S::kStages - 1 : stage - 1);
        const int e = piece / per;
        const int seen = pos - s_first[e] - (piece % per) * 16;
        const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + S::kPlaneBytes;
        if (++stage == S::kStages) stage = 0;
        if (seen < 0) continue;
        float sc[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[0][i] = sc[1][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            if (k < ksteps) {
                uint32_t b[4];  // tokens 0-7 and 8-15, columns 16k .. 16k + 15
                ldsm4(b, rows_addr<DP>(kb, (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)));
                mma16816<T>(sc[0], qf[k], b[0], b[1]);
                mma16816<T>(sc[1], qf[k], b[2], b[3]);
            }
        }
        // row lane / 4 (and + 8): tokens 2 (lane % 4), + 1, + 8, + 9
        constexpr int kR = SPLIT ? 1 : 2;
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i = 0; i < 2 * kR; ++i) {
                const int tok = n * 8 + (lane & 3) * 2 + (i & 1);
                sc[n][i] = tok <= seen ? sc[n][i] * p.scale_log2 : -INFINITY;
                top[i >> 1] = fmaxf(top[i >> 1], sc[n][i]);
            }
        }
        float fix[2], base[2];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], 2));
            const float mn = fmaxf(m[r], top[r]);
            base[r] = mn == -INFINITY ? 0.0f : mn;
            fix[r] = exp2_fast(m[r] - base[r]);
            m[r] = mn;
        }
        float add[2] = {0.0f, 0.0f};
        uint32_t pf[4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                const float w0 = exp2_fast(sc[n][2 * r] - base[r]), w1 = exp2_fast(sc[n][2 * r + 1] - base[r]);
                add[r] += w0 + w1;
                pf[2 * n + r] = Pair16<T>::pack(w0, w1);
                if (SPLIT) {
                    const float2 first = Pair16<T>::unpack(pf[2 * n]);
                    pf[2 * n + 1] = Pair16<T>::pack(w0 - first.x, w1 - first.y);
                }
            }
        }
        if (SPLIT) fix[1] = fix[0];
#pragma unroll
        for (int r = 0; r < kR; ++r) l[r] = l[r] * fix[r] + add[r];
        if (__any_sync(0xFFFFFFFFu, fix[0] != 1.0f || fix[1] != 1.0f)) {
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                o[i][0] *= fix[0];
                o[i][1] *= fix[0];
                o[i][2] *= fix[1];
                o[i][3] *= fix[1];
            }
        }
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
            if (n < ksteps) {
                uint32_t b[4];
                ldsm4_t(b, rows_addr<DP>(vb, lane & 15, 2 * n + (lane >> 4)));
                mma16816<T>(o[2 * n], pf, b[0], b[1]);
                mma16816<T>(o[2 * n + 1], pf, b[2], b[3]);
            }
        }
    }
    if (SPLIT) {
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {  // an infinite value is infinite with the first parts; with the second ones it may be 0 * inf
            o[i][0] += is_finite(o[i][0]) ? o[i][2] : 0.0f;
            o[i][1] += is_finite(o[i][1]) ? o[i][3] : 0.0f;
        }
    }
    cp_async_wait<0>();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 1);
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 2);
    }
    // the warps meet: rows of DP + 8 floats, the last ones maximum and sum
    __syncthreads();
    float* s_o = reinterpret_cast<float*>(rows_smem);
    constexpr int kRow = DP + 8;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float* dst = s_o + (warp * 16 + (lane >> 2) + r * 8) * kRow;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i)
            *reinterpret_cast<float2*>(dst + i * 8 + (lane & 3) * 2) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
        if ((lane & 3) == 0) {
            dst[DP] = m[r];
            dst[DP + 1] = l[r];
        }
    }
    __syncthreads();
    // the CTA's sum over its warps: into the first warp's rows, or to the end where the CTA is alone
    const bool alone = ranks == 1;
    for (int i = tid; i < rows * (DP / 8); i += kRowsThreads) {
        const int r = i / (DP / 8), c = i % (DP / 8);
        if (c * 8 >= p.dim) continue;
        float top = -INFINITY, sum = 0.0f, acc[8] = {};
#pragma unroll
        for (int k = 0; k < kRowsWarps; ++k) top = fmaxf(top, s_o[(k * 16 + r) * kRow + DP]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int k = 0; k < kRowsWarps; ++k) {
            const float* src = s_o + (k * 16 + r) * kRow;
            const float w = exp2_fast(src[DP] - base);
            sum += w * src[DP + 1];
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += w * src[c * 8 + j];
        }
        if (alone) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;  // nothing seen: zeros
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] *= inv;
            *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + t * p.out_stride[0] + (head0 + r) * p.out_stride[1] + c * 8) = pack8<T>(acc);
            if (c == 0 && p.lse) p.lse[t * n_heads + head0 + r] = sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994531f;
        } else {
            float* dst = s_o + r * kRow + c * 8;
            *reinterpret_cast<float4*>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
            if (c == 0) *reinterpret_cast<float2*>(s_o + r * kRow + DP + 4) = make_float2(top, sum);  // (apart from the warps' own)
        }
    }
    if (!alone) {
        // the CTAs share out the rows and read each other's
        cluster_sync();
        const int pieces_all = rows * (DP / 8);
        for (int i = rank * kRowsThreads + tid; i < pieces_all; i += ranks * kRowsThreads) {
            const int r = i / (DP / 8), c = i % (DP / 8);
            if (c * 8 >= p.dim) continue;
            float2 ml[8];
            float top = -INFINITY, sum = 0.0f, acc[8] = {};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                ml[k] = make_float2(-INFINITY, 0.0f);
                if (k < ranks) ml[k] = cluster_load2(cluster_addr(s_o + r * kRow + DP + 4, k));
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k < ranks) {
                    const uint32_t src = cluster_addr(s_o + r * kRow + c * 8, k);
                    const float4 lo = cluster_load4(src), hi = cluster_load4(src + 16);
                    const float w = exp2_fast(ml[k].x - base);
                    sum += w * ml[k].y;
                    acc[0] += w * lo.x, acc[1] += w * lo.y, acc[2] += w * lo.z, acc[3] += w * lo.w;
                    acc[4] += w * hi.x, acc[5] += w * hi.y, acc[6] += w * hi.z, acc[7] += w * hi.w;
                }
            }
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] *= inv;
            *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + t * p.out_stride[0] + (head0 + r) * p.out_stride[1] + c * 8) = pack8<T>(acc);
            if (c == 0 && p.lse) p.lse[t * n_heads + head0 + r] = sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994531f;
        }
        cluster_sync();  // nobody leaves while its rows are read
    }
    __syncthreads();  // the next token's lists and ring lie over this one's
}

template <typename T, int DP, bool SPLIT>
__global__ void __launch_bounds__(kRowsThreads) kv_attend_rows_kernel(KvAttendParams p) {
    extern __shared__ __align__(128) uint8_t rows_smem[];
    __shared__ int s_page[kKvMaxSelect], s_first[kKvMaxSelect];
    __shared__ int s_n;
    if (p.window == 0) {
        const int ranks = static_cast<int>(cluster_size());
        attend_rows<T, DP, SPLIT>(p, blockIdx.x / ranks, static_cast<int>(cluster_rank()), ranks, rows_smem, s_page, s_first, s_n);
        return;
    }
    // what the tile kernel left: each thread looks at one token of the CTA's (its own CTA alone writes that token's row, behind
    // the barrier)
    __shared__ unsigned s_left[kRowsWarps];
    for (int64_t t0 = blockIdx.x; t0 < p.n_tokens; t0 += static_cast<int64_t>(gridDim.x) * kRowsThreads) {
        const int64_t mine = t0 + static_cast<int64_t>(threadIdx.x) * gridDim.x;
        const unsigned left = __ballot_sync(0xFFFFFFFFu, mine < p.n_tokens && *kv_mark(p, mine, blockIdx.y, blockIdx.z) == kKvLeft);
        if ((threadIdx.x & 31) == 0) s_left[threadIdx.x >> 5] = left;
        if (!__syncthreads_or(left != 0)) continue;
        for (int w = 0; w < kRowsWarps; ++w)
            for (unsigned rest = s_left[w]; rest; rest &= rest - 1)
                attend_rows<T, DP, SPLIT>(p, t0 + static_cast<int64_t>(w * 32 + __ffs(rest) - 1) * gridDim.x, 0, 1, rows_smem, s_page, s_first, s_n);
        __syncthreads();  // the next round's words lie over these
    }
}

}  // namespace ivf
