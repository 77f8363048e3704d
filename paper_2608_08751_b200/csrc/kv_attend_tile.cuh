// Attention over selected blocks for prompt chunks: 5th-generation tensor cores, keys and values by TMA.
//
// Neighbouring tokens of a prompt select much the same blocks.  A CTA takes a window of consecutive tokens and one kv
// head; its 128 rows are (token, query head of the group), and it walks the union of the blocks that any token of the
// window selected, each block fetched once for all rows.  A row that did not select a block sees it masked.
//
//   before the loop all warps build the plan: a bitmap of the blocks that the window's tokens selected, its prefix
//                   sums give every block its place, and every (token, block) sets the token's bit there.  (A
//                   warp that merged the tokens' lists tile by tile needed 2,600 cycles for a tile and held all
//                   the others up.)
//   issuer          one thread serves in whatever order their inputs come: S = Q K^T into TMEM, O += P V with P read
//                   from TMEM, and the copies of keys and values (TMA)
//   softmax warps   one thread per row: S out of TMEM, maximum and sum in registers, P into TMEM.  O is rescaled
//                   only when the maximum has grown by more than 2^8 past the reference of the exponentials; the
//                   reference cancels in the final division.
//
// A tile is 64 keys.  There is one S and there are two P: S(j + 1) is computed as soon as the rows of S(j) are in
// registers, so the softmax warps never wait for a product.  (With P over S, S(j + 2) had to wait for P(j) V.)  Two
// CTAs live on an SM (one for heads wider than 128).
//
// 4,096 tokens of two requests by 4 heads of a group of 8, d = 128, 16 of up to 512 blocks of 64: 160 us, 430 TFLOP/s of
// useful products.  The 16 tokens of a window select 23 blocks between them, so 1.45 times the useful work is done.  A
// tile takes a CTA 1.24 us, nearly all of it one softmax warp's dependent instructions (2,300 cycles; the products take 350 of
// them, and no unit is full: issue slots 34 %, tensor pipe 32 %, exponentials 28 %).  5 us of a CTA's 37 go
// into queries and plan, 3 into the output, partly under the other CTA's work.  (Weights in two parts, as the rows kernel has
// them, were right and took 219 us in place of 163: the parts are made in the same warps.)
//
// What a page holds past the window's last token may be anything: those value rows are zeroed in shared memory.  A
// value that is not finite at a token that only some rows see turns the other rows' sums into NaN (0 * NaN);
// such a window, one whose tokens belong to many requests and one whose plan is too long is left to the rows
// kernel by marks in its output rows.
#pragma once
#include "kv_attend.cuh"

namespace ivf {

// DB: 64-element blocks of a head (1, 2, 4).
template <int DB>
struct TileShape {
    static constexpr int kCtas = DB == 4 ? 1 : 2;       // on an SM
    static constexpr int kKeys = 64;                    // keys of a tile
    static constexpr int kStages = 2;
    static constexpr int kBlockBytes = kKeys * 128;     // 64 columns of all keys
    static constexpr int kPlaneBytes = DB * kBlockBytes;
    static constexpr int kStageBytes = 2 * kPlaneBytes;
    static constexpr int kQBytes = DB * 128 * 128;
    // Of a plan: as many as fit beside two CTAs' tiles on an SM.  Windows win where they fit (2,048 tokens of one request by 4 heads
    // of a group of 8, windows / rows kernel): 64 blocks of 64 keys a token, 90 to a window 263 / 1,958 us; 16 blocks a
    // token that hardly agree, 170 to a window 402 / 567.  What does not fit costs the plan on top of the rows: 537 blocks to
    // a window 1,973 / 1,976, 256 blocks of 16 keys a token, 346 to a window 2,178 / 2,078.
    static constexpr int kBoxes = 320;
    static constexpr int kMapWords = 1024;              // bitmap of 32,768 blocks at a time, in the ring before the loop
    static constexpr int kRows = 128;
    static constexpr int kWarps = 5;                    // softmax 0-3, issuer 4
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kPCol = kKeys, kOCol = 2 * kKeys;  // TMEM columns: S, P twice (16-bit: half as wide), O
    static constexpr int kCols = DB == 4 ? 512 : 256;
};

template <int DB>
struct TileControl {
    uint64_t k_full[2], v_full[2], k_empty[2], v_empty[2];
    // by the tile's parity: a waiter may be one tile late, not two
    uint64_t s_free, s_full[2], p_ready[2], pv_done[2], drain;
    // the plan, a box being a page or a half of a page of 128
    struct alignas(16) Box {
        int first;         // position of its first token
        int dead;          // tokens from here on lie past the window's last: value rows to be zeroed
        int page;
        uint32_t members;  // tokens 0-31 of the window that selected it
    } box[TileShape<DB>::kBoxes];
    uint32_t more[TileShape<DB>::kBoxes][3];  // tokens 32-127
    int req[TileShape<DB>::kRows], pos[TileShape<DB>::kRows], seg[TileShape<DB>::kRows];
    int seg_last[TileShape<DB>::kRows];          // last position that a token of the segment sees
    int warp_sum[TileShape<DB>::kWarps];
    uint32_t tmem;
    int abort_flag, bad;
};

template <int DB>
constexpr int tile_smem() {
    using S = TileShape<DB>;
    return 1024 + S::kQBytes + S::kStages * S::kStageBytes + static_cast<int>(sizeof(TileControl<DB>));
}

// True in one lane of the warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A holds two 16-bit numbers to a column.
__device__ __forceinline__ void umma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 16 columns, the wait included.
__device__ __forceinline__ void tmem_ld_32x32b_x16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two 32-bit numbers in one 64-bit register pair: sm_100 multiplies and adds them in one instruction.
__device__ __forceinline__ uint64_t pair32(float a, float b) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float lo32(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float hi32(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float max3f(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max3f(uint32_t a, uint32_t b, uint32_t c) {
    return max3f(__uint_as_float(a), __uint_as_float(b), __uint_as_float(c));
}

// row / group for row < 128: `inv` = 65536 / group + 1
__device__ __forceinline__ int token_of(int row, uint32_t inv) { return static_cast<int>((static_cast<uint32_t>(row) * inv) >> 16); }

// A wait of a whole warp: its lanes give up together, since they meet in warp-wide instructions later.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const WaitCtl& ctl, int where) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, ctl, where));
}

template <typename T>
struct UmmaType;
template <>
struct UmmaType<__half> { static constexpr uint32_t kFormat = 0; };
template <>
struct UmmaType<__nv_bfloat16> { static constexpr uint32_t kFormat = 1; };

// Instruction descriptor: 16-bit A and B of one type, fp32 accumulator, M = 128.  b_mn: B lies with its N axis contiguous.
template <typename T>
__device__ __forceinline__ uint32_t tile_idesc(int n, bool b_mn) {
    return (1u << 4) | (UmmaType<T>::kFormat << 7) | (UmmaType<T>::kFormat << 10) | (b_mn ? 1u << 16 : 0u) |
           (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}

template <typename T, int DB>
__global__ void __launch_bounds__(TileShape<DB>::kThreads, TileShape<DB>::kCtas)
kv_attend_tile_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const KvAttendParams p) {
    using S = TileShape<DB>;
    extern __shared__ uint8_t tile_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tile_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* ring = smem + S::kQBytes;
    TileControl<DB>& c = *reinterpret_cast<TileControl<DB>*>(ring + S::kStages * S::kStageBytes);
    const int tid = threadIdx.x, lane = tid & 31;
    // (broadcast, so that the compiler knows it to be the same for the warp: the products' descriptors then live in uniform
    // registers and an issue takes 48 cycles instead of 79)
    const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const int h = blockIdx.y;
    const int64_t w0 = static_cast<int64_t>(blockIdx.x) * p.window;
    const int tokens = static_cast<int>(min(static_cast<int64_t>(p.window), p.n_tokens - w0));
    auto leave = [&]() {  // to the rows kernel
        const int parts = (p.group + 15) / 16;
        for (int i = tid; i < tokens * parts; i += S::kThreads) *kv_mark(p, w0 + i / parts, h, i % parts) = kKvLeft;
    };

    // ---- queries: rows of 128 bytes to a 64-column block, 16-byte pieces exchanged by the row's low bits; they come
    // while the plan is built
    const uint32_t inv_group = 65536u / p.group + 1;
    {
        constexpr int kPieces = DB * 8, kStep = S::kThreads / kPieces;  // rows at a time
        const int piece = tid % kPieces, row0 = tid / kPieces;
        const bool in = tid < kStep * kPieces && piece * 8 < p.dim;
        const T* q0 = static_cast<const T*>(p.q) + w0 * p.q_stride[0] + static_cast<int64_t>(h) * p.group * p.q_stride[1] + piece * 8;
        const uint32_t to = smem_u32(smem) + (piece >> 3) * (128 * 128);
#pragma unroll
        for (int row = row0; row < S::kRows; row += kStep) {
            const int tok = token_of(row, inv_group);
            const bool ok = in && tok < tokens;
            const T* src = ok ? q0 + tok * p.q_stride[0] + (row - tok * p.group) * p.q_stride[1] : static_cast<const T*>(p.q);
            if (tid < kStep * kPieces) cp_async16(to + row * 128 + (((piece & 7) ^ (row & 7)) << 4), src, ok);
        }
    }
    cp_async_commit();

    // ---- the window's tokens; one of many requests is left to the rows kernel: below 8 tokens to a request the
    // union is hardly shared
    int change = 0;
    if (tid < S::kRows) {
        int req = -1, pos = -1;
        if (tid < tokens) {
            req = p.token_req[w0 + tid];
            pos = p.token_pos[w0 + tid];
            change = tid > 0 && req != p.token_req[w0 + tid - 1];
            if (req >= p.n_req) {
                kv_report(p.status, kKvStatusBadId, KV_SITE_ATTEND);
                req = -1;
            }
            if (pos < 0) req = -1;
        }
        c.req[tid] = req;
        c.pos[tid] = pos;
        c.seg_last[tid] = -1;
    }
    const int segments = __syncthreads_count(change) + 1;
    if (segments > 1 && segments * 8 > tokens) {
        cp_async_wait<0>();
        leave();
        return;
    }

    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(&c.k_full[i], 1);
            mbar_init(&c.v_full[i], 1);
            mbar_init(&c.k_empty[i], 1);
            mbar_init(&c.v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&c.s_full[i], 1);
            mbar_init(&c.p_ready[i], 128);
            mbar_init(&c.pv_done[i], 1);
        }
        mbar_init(&c.s_free, 128);
        mbar_init(&c.drain, 1);
        c.abort_flag = 0;
        c.bad = 0;
        fence_mbar_init();
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    // ---- the plan
    const int box_shift = min(p.page_shift, 6), box = 1 << box_shift;  // a page of 128 tokens is two boxes of 64
    const int halves = 1 << (p.page_shift - box_shift);
    const int per_tile = S::kKeys >> box_shift;
    uint32_t* map = reinterpret_cast<uint32_t*>(ring);
    int* rank = reinterpret_cast<int*>(map + S::kMapWords);  // selected blocks before a word of the map
    for (int i = tid; i < S::kBoxes; i += S::kThreads) {
        c.box[i].members = 0;
        if (tokens > 32) c.more[i][0] = c.more[i][1] = c.more[i][2] = 0;
    }
    if (segments == 1) {
        if (tid < S::kRows) c.seg[tid] = 0;
    } else if (tid < 32) {
        int before = 0;
        for (int t0 = 0; t0 < tokens; t0 += 32) {
            const int t = t0 + lane;
            // the requests as given, as they were counted: a token that is padding by its position stays inside its segment
            const unsigned m = __ballot_sync(0xFFFFFFFFu, t > 0 && t < tokens && p.token_req[w0 + t] != p.token_req[w0 + t - 1]);
            c.seg[t] = before + __popc(m & (0xFFFFFFFFu >> (31 - lane)));
            before += __popc(m);
        }
    }
    __syncthreads();
    if (segments == 1) {
        if (tid < 32) {  // one request: its token of the largest position
            int far = -1;
            for (int t = lane; t < tokens; t += 32) far = max(far, c.req[t] >= 0 ? c.pos[t] : -1);
            far = __reduce_max_sync(0xFFFFFFFFu, far);
            if (lane == 0) c.seg_last[0] = far;
        }
    } else if (tid < tokens && c.req[tid] >= 0) {
        atomicMax(&c.seg_last[c.seg[tid]], c.pos[tid]);
    }
    __syncthreads();
    int boxes = 0;
    for (int s = 0; s < segments && boxes >= 0; ++s) {
        const int last_pos = c.seg_last[s], last_block = last_pos >> p.page_shift;  // -1: nobody sees anything
        for (int base = 0; base <= last_block; base += S::kMapWords * 32) {
            const int words = min((last_block - base) / 32 + 1, S::kMapWords);
            for (int i = tid; i < words; i += S::kThreads) map[i] = 0;
            __syncthreads();
            // entries (token, block) of this segment and range: once to fill the map, once to set the members
            auto each = [&](auto&& f) {
                constexpr int kAtOnce = 4;
                for (int e0 = tid; e0 < tokens * p.n_select; e0 += S::kThreads * kAtOnce) {
                    int tok[kAtOnce], b[kAtOnce];
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) {
                        const int e = e0 + k * S::kThreads;
                        tok[k] = e / p.n_select;
                        b[k] = tok[k] < tokens ? p.selected[((w0 + tok[k]) * p.n_kv_heads + h) * p.n_select + e - tok[k] * p.n_select] : -1;
                    }
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k)
                        if (tok[k] < tokens && c.seg[tok[k]] == s && c.req[tok[k]] >= 0 && b[k] >= base && b[k] <= (c.pos[tok[k]] >> p.page_shift) &&
                            b[k] - base < words * 32)
                            f(tok[k], b[k] - base);
                }
            };
            each([&](int, int b) { atomicOr(&map[b >> 5], 1u << (b & 31)); });
            __syncthreads();
            constexpr int kPer = (S::kMapWords + S::kThreads - 1) / S::kThreads;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (tid * kPer + i < words) mine += __popc(map[tid * kPer + i]);
            int upto = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int v = __shfl_up_sync(0xFFFFFFFFu, upto, off);
                if (lane >= off) upto += v;
            }
            if (lane == 31) c.warp_sum[warp] = upto;
            __syncthreads();
            int before = upto - mine, found = 0;
#pragma unroll
            for (int w = 0; w < S::kWarps; ++w) {
                if (w < warp) before += c.warp_sum[w];
                found += c.warp_sum[w];
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (tid * kPer + i < words) {
                    rank[tid * kPer + i] = before;
                    before += __popc(map[tid * kPer + i]);
                }
            }
            __syncthreads();
            if (boxes + found * halves > S::kBoxes) {
                boxes = -1;
                break;
            }
            each([&](int tok, int b) {
                const uint32_t word = map[b >> 5];
                const int at = boxes + (rank[b >> 5] + __popc(word & ((1u << (b & 31)) - 1))) * halves;
                const int first = (base + b) << p.page_shift;
                for (int half = 0; half < halves; ++half) {
                    atomicOr(tok < 32 ? &c.box[at + half].members : &c.more[at + half][(tok >> 5) - 1], 1u << (tok & 31));
                    c.box[at + half].first = first + half * 64;
                    c.box[at + half].dead = max(0, min(box - 1, last_pos - first - half * 64) + 1);
                    c.box[at + half].page = c.req[tok];  // whose page: looked up below
                }
            });
            boxes += found * halves;
            // (of this request's own boxes: one that found none must leave the last box of the request before it)
            if (halves == 2 && found > 0 && base + S::kMapWords * 32 > last_block) {
                __syncthreads();
                if (c.box[boxes - 1].first > last_pos) {  // the last block's second half is empty: the next request gets its place
                    --boxes;
                    __syncthreads();
                    if (tid == 0) c.box[boxes].members = c.more[boxes][0] = c.more[boxes][1] = c.more[boxes][2] = 0;
                }
            }
            __syncthreads();
        }
    }
    if (boxes < 0) {  // more than the plan holds: a tile would serve a few of its rows only
        cp_async_wait<0>();
        leave();
        return;
    }
    for (int b = tid; b < boxes; b += S::kThreads) {
        const int block = c.box[b].first >> p.page_shift;
        int page = -1;
        if (block < p.max_blocks) page = p.table[c.box[b].page * p.table_stride + block];
        if (block >= p.max_blocks || page >= p.num_pages) {
            kv_report(p.status, kKvStatusBadId, KV_SITE_ATTEND);
            page = -1;
        }
        if (page < 0) {
            page = 0;  // a stand-in, all of it zeroed and unseen
            c.box[b].dead = 0;
            c.box[b].members = c.more[b][0] = c.more[b][1] = c.more[b][2] = 0;
        }
        c.box[b].page = page;
    }
    const int tiles = (boxes + per_tile - 1) / per_tile;
    if (warp == S::kWarps - 1) {
        tmem_alloc(&c.tmem, S::kCols);
        tmem_relinquish();
    }
    cp_async_wait<0>();
    fence_proxy_async_smem();  // the queries; and the map's words, before copies land on them
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = c.tmem;
    WaitCtl ctl;
    ctl.abort_flag = &c.abort_flag;
    ctl.status = p.status;
    ctl.limit_ns = p.limit_ns;
    const uint32_t ring0 = smem_u32(ring);
    auto keys_of = [&](int j) { return min(per_tile, boxes - j * per_tile) << box_shift; };
    if (warp == S::kWarps - 1) {
        // ------------------------------------------------------------ issuer
        if (elect_one()) {
            const uint32_t t_o = tmem + S::kOCol;
            const uint32_t q_lo = umma_desc_lo(smem_u32(smem));
            const uint32_t idesc_o = tile_idesc<T>(p.dim, true);
            const uint32_t negate = p.scale_log2 < 0.0f ? 1u << 13 : 0u;  // a negative scale is a positive one of negated queries
            const int ksteps = p.dim >> 4;
            auto copy = [&](int j, const CUtensorMap* from, uint64_t* full, uint32_t to) {
                const int b0 = j * per_tile, n = min(per_tile, boxes - b0);
                mbar_arrive_expect_tx(full, n * DB * box * 128);
                for (int i = 0; i < n; ++i) {
                    const int row = halves == 2 ? c.box[b0 + i].first & 64 : 0, page = c.box[b0 + i].page;
#pragma unroll
                    for (int d = 0; d < DB; ++d) tma_load_4d(to + i * box * 128 + d * S::kBlockBytes, from, full, d * 64, row, h, page);
                }
            };
            auto is_free = [&](uint64_t* empty, int j) {
                return j < S::kStages || mbar_test_wait(&empty[j % S::kStages], (j / S::kStages - 1) & 1);
            };
            int k = 0, v = 0;        // next keys and values to copy
            int sj = 0, pj = 0;  // next S and P V
            uint64_t since = 0;
            uint32_t idle = 0;
            while (pj < tiles) {
                bool moved = false;
                if (sj < k && mbar_test_wait(&c.k_full[sj % S::kStages], (sj / S::kStages) & 1) &&
                    (sj == 0 || mbar_test_wait(&c.s_free, (sj - 1) & 1))) {
                    tc_fence_after_sync();
                    const uint32_t k_lo = umma_desc_lo(ring0 + (sj % S::kStages) * S::kStageBytes);
                    const uint32_t idesc = tile_idesc<T>(keys_of(sj), false) | negate;
#pragma unroll
                    for (int k = 0; k < DB * 4; ++k) {
                        if (k < ksteps)
                            umma_f16(tmem, umma_desc_join(q_lo + (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2, kDescHiSw128),
                                     umma_desc_join(k_lo + (k >> 2) * (S::kBlockBytes >> 4) + (k & 3) * 2, kDescHiSw128), idesc, k > 0);
                    }
                    umma_commit(&c.s_full[sj & 1]);
                    umma_commit(&c.k_empty[sj % S::kStages]);
                    ++sj;
                    moved = true;
                }
                if (pj < sj && pj < v && mbar_test_wait(&c.p_ready[pj & 1], (pj >> 1) & 1) &&
                    mbar_test_wait(&c.v_full[pj % S::kStages], (pj / S::kStages) & 1)) {
                    tc_fence_after_sync();
                    // values: N (the head's columns) contiguous; blocks of 64 columns kBlockBytes apart, 8 keys 1024 bytes
                    const uint32_t v_addr = ring0 + (pj % S::kStages) * S::kStageBytes + S::kPlaneBytes;
                    const uint32_t v_lo = ((v_addr & 0x3FFFFu) >> 4) | (static_cast<uint32_t>(S::kBlockBytes >> 4) << 16);
                    const uint32_t t_p = tmem + S::kPCol + (pj & 1) * (S::kKeys / 2);
                    const int steps = keys_of(pj) >> 4;
#pragma unroll
                    for (int k = 0; k < S::kKeys / 16; ++k)
                        if (k < steps)
                            umma_f16_ts(t_o, t_p + k * 8, umma_desc_join(v_lo + k * (2048 >> 4), kDescHiSw128), idesc_o, (pj > 0 || k > 0) ? 1u : 0u);
                    umma_commit(&c.pv_done[pj & 1]);
                    umma_commit(&c.v_empty[pj % S::kStages]);
                    ++pj;
                    moved = true;
                }
                if (k < tiles && is_free(c.k_empty, k)) {
                    copy(k, &map_k, &c.k_full[k % S::kStages], ring0 + (k % S::kStages) * S::kStageBytes);
                    ++k;
                    moved = true;
                }
                if (v < k && is_free(c.v_empty, v)) {
                    copy(v, &map_v, &c.v_full[v % S::kStages], ring0 + (v % S::kStages) * S::kStageBytes + S::kPlaneBytes);
                    ++v;
                    moved = true;
                }
                if (moved) {
                    idle = 0;
                } else if ((++idle & 255u) == 0u) {
                    const uint64_t t = global_timer_ns();
                    if (idle == 256u) since = t;
                    if (t - since > ctl.limit_ns) report_timeout(ctl, 202);
                    if (*ctl.abort_flag) break;
                }
            }
            // Copies and products already issued end before the CTA and its TMEM go (bounded), whoever gave up: this thread may have issued
            // its last ones and left its loop in good order before a softmax warp's wait ran out.
            umma_commit(&c.drain);
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(&c.drain, 0) && global_timer_ns() - t0 < 2000000000ull) {
            }
            for (int i = max(0, k - S::kStages); i < k; ++i)
                while (!mbar_try_wait(&c.k_full[i % S::kStages], (i / S::kStages) & 1) && global_timer_ns() - t0 < 2000000000ull) {
                }
            for (int i = max(0, v - S::kStages); i < v; ++i)
                while (!mbar_try_wait(&c.v_full[i % S::kStages], (i / S::kStages) & 1) && global_timer_ns() - t0 < 2000000000ull) {
                }
        }
    } else {
        // ------------------------------------------------------------ softmax: thread = row = TMEM lane
        const int r = tid;
        const int tok = token_of(r, inv_group);
        const bool row_live = tok < tokens;
        const int pos = row_live && c.req[tok] >= 0 ? c.pos[tok] : -1;
        const int word = row_live ? tok >> 5 : 0;
        const uint32_t bit = row_live && pos >= 0 ? 1u << (tok & 31) : 0u;
        const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
        const uint32_t t_rows = tmem + lanes, t_o = t_rows + S::kOCol;
        const float scale = fmaxf(fabsf(p.scale_log2), 1.2e-38f);  // zero would turn masked logits into NaN
        const float slack = 8.0f / scale;
        float m = -INFINITY, l = 0.0f;  // reference of the exponentials (in logits before scaling), sum
        bool ok = true;
        const uint64_t scale2 = pair32(scale, scale);
        auto members_of = [&](int b, uint32_t low) { return word == 0 ? low : c.more[b][word - 1]; };
        auto ahead = c.box[0];  // the next tile's first box, fetched under this tile's exponentials
        for (int j = 0; j < tiles; ++j) {
            const int b0 = j * per_tile, n_boxes = min(per_tile, boxes - b0);
            const uint32_t t_p = t_rows + S::kPCol + (j & 1) * (S::kKeys / 2);
            // groups of 16 keys that the row sees: whole ones, and one whose first `rem` keys it sees (a position may be
            // 2^31 - 1: one is added after the minimum)
            int seen = (members_of(b0, ahead.members) & bit) ? max(min(pos - ahead.first, box - 1) + 1, 0) : 0;
            uint32_t full = (1u << (seen >> 4)) - 1, part = seen & 15 ? 1u << (seen >> 4) : 0u;
            int rem = seen & 15;
            bool tail = ahead.dead < box;
            for (int i = 1; i < n_boxes; ++i) {
                seen = (members_of(b0 + i, c.box[b0 + i].members) & bit) ? max(min(pos - c.box[b0 + i].first, box - 1) + 1, 0) : 0;
                const int g0 = (i << box_shift) >> 4;
                full |= ((1u << (seen >> 4)) - 1) << g0;
                if (seen & 15) {
                    part |= 1u << (g0 + (seen >> 4));
                    rem = seen & 15;
                }
                tail |= c.box[b0 + i].dead < box;
            }
            const uint32_t mine = full | part;
            const bool some = __any_sync(0xFFFFFFFFu, mine != 0);
            // keys that only part of a group's rows see, and columns that hold no key of the request
            const bool cut = __any_sync(0xFFFFFFFFu, part != 0) || tail || n_boxes < per_tile;
            if (!(ok = warp_wait(&c.s_full[j & 1], (j >> 1) & 1, ctl, 208))) break;
            tc_fence_after_sync();
            uint32_t s[S::kKeys];
            constexpr int kGroups = S::kKeys / 16;
            if (some) {
                tmem_ld_32x32b_x64(t_rows, s);
                tmem_wait_ld_regs(s);
            }
            tc_fence_before_sync();
            mbar_arrive(&c.s_free);
            float top = -INFINITY;
            if (some) {
                if (cut) {
#pragma unroll
                    for (int g = 0; g < kGroups; ++g) {
                        const int see = full >> g & 1 ? 16 : part >> g & 1 ? rem : 0;
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            if (x >= see) s[g * 16 + x] = 0xFF800000u;
                    }
                }
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const uint32_t* v = &s[g * 16];
                    const float a = max3f(v[0], v[1], v[2]), b = max3f(v[3], v[4], v[5]), d = max3f(v[6], v[7], v[8]), f = max3f(v[9], v[10], v[11]);
                    const float t = fmaxf(max3f(max3f(a, b, d), f, max3f(v[12], v[13], v[14])), __uint_as_float(v[15]));
                    top = fmaxf(top, mine >> g & 1 ? t : -INFINITY);
                }
            }
            if (j > 1) {  // the weights of tile j - 2 have been used
                if (!(ok = warp_wait(&c.pv_done[j & 1], ((j >> 1) - 1) & 1, ctl, 215))) break;
                tc_fence_after_sync();
            }
            if (tail) {  // value rows that no token of the window sees (their stage is known to be one copy behind at most, too)
                if (!(ok = warp_wait(&c.v_full[j % S::kStages], (j / S::kStages) & 1, ctl, 207))) break;
                for (int i = 0; i < n_boxes; ++i) {
                    const int dead = c.box[b0 + i].dead;
                    uint8_t* base = ring + (j % S::kStages) * S::kStageBytes + S::kPlaneBytes + (i * box + dead) * 128;
                    for (int x = r; x < (box - dead) * 8 * DB; x += 128) {
                        const int piece = x & 7, rest = x >> 3;
                        *reinterpret_cast<uint4*>(base + (rest % DB) * S::kBlockBytes + (rest / DB) * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
                    }
                }
                fence_proxy_async_smem();
            }
            const bool grow = top > m + slack || (m == -INFINITY && top > m);
            if (__any_sync(0xFFFFFFFFu, grow)) {
                const float fix = grow && l > 0.0f ? exp2_fast((m - top) * scale) : 1.0f;
                if (grow) m = top;
                if (__any_sync(0xFFFFFFFFu, fix != 1.0f)) {  // (a sum that is not zero: j > 0)
                    if (!(ok = warp_wait(&c.pv_done[(j - 1) & 1], ((j - 1) >> 1) & 1, ctl, 211))) break;
                    tc_fence_after_sync();
                    l *= fix;
                    for (int q = 0; q < p.dim >> 4; ++q) {  // 16 columns at a time: the logits stay in registers
                        uint32_t o[16];
                        tmem_ld_32x32b_x16(t_o + q * 16, o);
#pragma unroll
                        for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * fix);
                        tmem_st_32x32b_x16(t_o + q * 16, o);
                    }
                }
            }
            if (j + 1 < tiles) ahead = c.box[b0 + per_tile];
            if (some) {
                const float base = m == -INFINITY ? 0.0f : m * scale;
                uint64_t sum[2] = {0, 0};  // of two 32-bit sums each
#pragma unroll
                for (int q = 0; q < S::kKeys / 32; ++q) {
                    uint32_t out[16];
#pragma unroll
                    for (int x = 0; x < 32; x += 2) {
                        const int i = q * 32 + x;
                        const float off = mine >> (i / 16) & 1 ? -base : -INFINITY;  // a group that the row does not see: all weights 0
                        const uint64_t z = fma2(pair32(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), scale2, pair32(off, off));
                        const float a = exp2_fast(lo32(z)), b = exp2_fast(hi32(z));
                        sum[x / 2 & 1] = add2(sum[x / 2 & 1], pair32(a, b));
                        out[x / 2] = Pair16<T>::pack(a, b);
                    }
                    tmem_st_32x32b_x16(t_p + q * 16, out);
                }
                const uint64_t both = add2(sum[0], sum[1]);
                l += lo32(both) + hi32(both);
            } else {  // no row of the warp selected any of it
                const uint32_t none[16] = {};
#pragma unroll
                for (int q = 0; q < S::kKeys / 32; ++q) tmem_st_32x32b_x16(t_p + q * 16, none);
            }
            tmem_wait_st();
            tc_fence_before_sync();
            mbar_arrive(&c.p_ready[j & 1]);
        }
        if (ok && tiles > 0 && (ok = warp_wait(&c.pv_done[(tiles - 1) & 1], ((tiles - 1) >> 1) & 1, ctl, 209))) tc_fence_after_sync();
        if (ok) {
            // through the query tile, which the products have left: a warp's 32 rows go out with whole
            // rows side by side
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            uint8_t* stash = smem + warp * (32 * DB * 128);
            bool bad = false;
            for (int q = 0; q < (p.dim + 31) / 32; ++q) {
                uint32_t o[32];
                if (tiles > 0) {
                    tmem_ld_32x32b_x32(t_o + q * 32, o);
                    tmem_wait_ld_regs(o);
                }
#pragma unroll
                for (int x = 0; x < 32; x += 8) {
                    if (q * 32 + x < p.dim) {
                        float f[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            f[i] = l == 0.0f ? 0.0f : __uint_as_float(o[x + i]) * inv;
                            bad |= row_live && !(fabsf(f[i]) <= 3.4e38f);
                        }
                        *reinterpret_cast<uint4*>(stash + lane * (DB * 128) + (((q * 4 + x / 8) ^ (lane & 7)) << 4)) = pack8<T>(f);
                    }
                }
            }
            __syncwarp();
            const int pieces = p.dim >> 3;
            constexpr int kAtOnce = 32 / (DB * 8) > 0 ? 32 / (DB * 8) : 1;  // rows of a store
            for (int row0 = 0; row0 < 32; row0 += kAtOnce) {
                const int row = row0 + lane / (DB * 8 < 32 ? DB * 8 : 32), piece = lane % (DB * 8 < 32 ? DB * 8 : 32);
                const int out_row = warp * 32 + row, tk = token_of(out_row, inv_group);
                if (tk < tokens && piece < pieces) {
                    const uint4 v = *reinterpret_cast<const uint4*>(stash + row * (DB * 128) + ((piece ^ (row & 7)) << 4));
                    *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + (w0 + tk) * p.out_stride[0] +
                                              (static_cast<int64_t>(h) * p.group + out_row - tk * p.group) * p.out_stride[1] + piece * 8) = v;
                }
            }
            if (row_live && p.lse)
                p.lse[(w0 + tok) * p.group * p.n_kv_heads + static_cast<int64_t>(h) * p.group + r - tok * p.group] =
                    l == 0.0f ? -INFINITY : (m * scale + log2f(l)) * 0.69314718055994531f;
            if (bad) c.bad = 1;
        }
    }
    // ------------------------------------------------------------ teardown (also the abort path)
    tc_fence_before_sync();
    __syncthreads();
    if (warp == S::kWarps - 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, S::kCols);
    }
    if (c.bad) leave();  // (over what other threads wrote before the barrier)
}

}  // namespace ivf
