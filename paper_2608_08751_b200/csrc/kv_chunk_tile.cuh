// Attention over whole caches for prompt chunks: 5th-generation tensor cores, keys and values by TMA.
//
// An item's rows are one or two streams of 128 (tokens by query heads of a kv head's group).  Both streams go over the same keys, each
// fetched once, a tile of keys at a time:
//
//   softmax warps   a thread per row: S out of TMEM, maximum and sum in registers, P over S in TMEM.  O is rescaled only when the maximum has
//                   grown by more than 2^8 past the reference of the exponentials; the reference cancels in the final division
//   issuers         a thread to a stream: S = Q K^T into TMEM, O += P V with P from TMEM
//   copier          the tiles' pages, looked up a tile ahead, by TMA
//   planner         walks the CTA's span and leaves a record of each item for the other warps, whose loops need the registers; and cleans: value
//                   rows that no row of the item may look at become zeros, and in tiles that not all rows see values that are not
//                   finite are taken out
//
// The keys are taken from the last to the first: near ones weigh most where a bias falls with the distance, so the maximum is found at once
// (taken from the first it grew with every tile, and O was rescaled: 3,104 against 1,719 us).
//
// A tile is 64 keys.  A stream has two S, P lies over its S, and S(j + 1) is issued before P(j) V: the softmax warps find the next
// logits ready.  TMEM holds it exactly: two streams of two S (256 columns) and of O (256).  Heads wider than 128 take all of the second half
// for one stream's O; it has two threads to a row then, 32 keys each, which tell each other their maxima through shared memory.
//
// 4,096 tokens of two requests of 32,768 by 4 heads of a group of 8, d = 128 (1.67 TFLOP of useful products): 1.45 ms in short runs, 1.68 to 1.73 ms under the
// power limit, 1,150 and 980 TFLOP/s.  A tile of the two streams takes 1,850 cycles: its products alone 1,500 (with 64 keys to an
// instruction S waits for the queries' tile in shared memory, 48 cycles for 32), its softmax alone 1,650 (1,024 of them the special function unit's
// 16 exponentials a cycle), its copies alone 950.  What was tried: 128 keys to a tile with one S (1.74 ms where 64
// keys with two took 2.00; not again since then), two threads to a row here too (1.97), a quarter or an eighth of the exponentials by polynomial (1.62, 1.45), taking turns at the exponentials (1.73).
#pragma once
#include "kv_chunk.cuh"
#include "kv_attend_tile.cuh"

namespace ivf {

// DB: 64-element blocks of a head (1, 2, 4).
template <int DB>
struct ChunkTileShape {
    static constexpr int kStreams = DB == 4 ? 1 : 2;
    static constexpr int kHalves = DB == 4 ? 2 : 1;  // threads of a row
    static constexpr int kKeys = 64;
    static constexpr int kMine = kKeys / kHalves;    // keys of a softmax thread
    static constexpr int kStages = DB == 4 ? 2 : 4;  // of keys, and of values
    static constexpr int kBlockBytes = kKeys * 128;  // 64 columns of all keys
    static constexpr int kPlaneBytes = DB * kBlockBytes;
    static constexpr int kQBytes = DB * 128 * 128;   // of a stream
    static constexpr int kSoftWarps = 8;
    static constexpr int kRowThreads = 128 * kHalves;  // of a stream
    static constexpr int kWarps = kSoftWarps + 4;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kOCol = 256, kCols = 512;   // of TMEM; S lies at 0
    static constexpr int kPCol = DB == 4 ? 128 : -1; // -1: P lies over its S
    static constexpr int kPStep = DB == 4 ? kKeys / 2 : kKeys;
    static constexpr int kHoles = 16;                // tiles whose missing pages are remembered
    static constexpr int kItems = 4;                 // items that are planned ahead
};

// What the warps have to know of an item, or of the part of it that the span has.
struct ChunkTileItem {
    int tokens;            // 0: the span has ended
    int b, h, head0, heads;
    int token, pos;        // of its first token
    int lo, hi, k0, k1;
    int last, count;       // tiles of the part: its i-th is tile last - i
    int from[2], to[2];    // of them (i from .. to - 1) those that a stream has rows for
    int all_lo, all_hi;    // keys that every row of the item sees
    bool whole;
    int slot;
    ChunkReq r;
};

template <int DB>
struct ChunkTileControl {
    using S = ChunkTileShape<DB>;
    ChunkTileItem item[S::kItems];
    uint64_t item_full[S::kItems], item_empty[S::kItems];
    uint64_t k_full[S::kStages], v_full[S::kStages], k_empty[S::kStages], v_empty[S::kStages], v_clean[S::kStages];
    uint64_t q_full[S::kStreams], s_full[S::kStreams * 2], p_ready[S::kStreams * 2], pv_done[S::kStreams], o_full[S::kStreams], o_free[S::kStreams];
    uint64_t halves[S::kStreams * 4], drain[S::kStreams];
    float told[S::kStreams * 4][2][2][32];  // by warp pair, turn and half: maxima of a tile, at last the sums
    ChunkPlan<S::kThreads> plan;
    uint32_t holes[S::kHoles];  // by tile: groups of 16 keys without a page
    int odd[4];                 // by item: a value that is not finite was taken out
    uint32_t tmem;
    int abort_flag;
};

template <int DB>
constexpr int chunk_tile_smem() {
    using S = ChunkTileShape<DB>;
    return 1024 + S::kStreams * S::kQBytes + 2 * S::kStages * S::kPlaneBytes + static_cast<int>(sizeof(ChunkTileControl<DB>));
}

template <int STREAMS, int KEYS>
__device__ __forceinline__ void chunk_record(const ChunkParams& p, const ChunkCursor& at, const ChunkItem& it, ChunkTileItem& t) {
    t.b = at.b;
    t.h = it.hv / p.parts;
    const int g0 = it.hv % p.parts * p.part_heads;
    t.head0 = t.h * p.group + g0;
    t.heads = min(p.part_heads, p.group - g0);
    t.tokens = it.tokens, t.token = it.token, t.pos = it.pos;
    t.lo = it.lo, t.hi = it.hi, t.k0 = it.k0, t.k1 = it.k1;
    t.whole = it.first && it.last;
    t.slot = 2 * blockIdx.x + (it.first ? 1 : 0);
    t.r = at.r;
    const int first = it.k0 / KEYS, end = it.k1 > it.k0 ? (it.k1 + KEYS - 1) / KEYS : first;
    t.last = end - 1;
    t.count = end - first;
    const int per = p.tile_tokens / STREAMS;
    int skip;
    for (int s = 0; s < STREAMS; ++s) {
        const int n = min(per, it.tokens - s * per);
        int lo, hi;
        chunk_sees(p, at.r, it.pos + s * per, true, lo, skip);
        chunk_sees(p, at.r, it.pos + s * per + n - 1, true, skip, hi);
        lo = max(lo, it.k0);
        hi = min(hi, it.k1);
        const bool some = n > 0 && hi > lo;
        t.from[s] = some ? end - (hi + KEYS - 1) / KEYS : 0;
        t.to[s] = some ? end - lo / KEYS : 0;
    }
    chunk_sees(p, at.r, it.pos, true, skip, t.all_hi);
    chunk_sees(p, at.r, it.pos + it.tokens - 1, true, t.all_lo, skip);
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// CAP, BIAS: whether there is one.
template <typename T, int DB, bool CAP, bool BIAS>
__global__ void __launch_bounds__(ChunkTileShape<DB>::kThreads, 1)
kv_chunk_tile_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ ChunkParams p) {
    using S = ChunkTileShape<DB>;
    constexpr int kKeys = S::kKeys, kStreams = S::kStreams, kStages = S::kStages;
    extern __shared__ uint8_t tile_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tile_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* k_ring = smem + kStreams * S::kQBytes;
    uint8_t* v_ring = k_ring + kStages * S::kPlaneBytes;
    ChunkTileControl<DB>& c = *reinterpret_cast<ChunkTileControl<DB>*>(v_ring + kStages * S::kPlaneBytes);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);  // the same for the warp, as the compiler can see
    pdl_trigger();
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&c.k_full[i], 1);
            mbar_init(&c.v_full[i], 1);
            mbar_init(&c.k_empty[i], kStreams);
            mbar_init(&c.v_empty[i], kStreams);
            mbar_init(&c.v_clean[i], 1);
        }
        for (int i = 0; i < kStreams; ++i) {
            mbar_init(&c.q_full[i], 4 * S::kHalves);
            mbar_init(&c.pv_done[i], 1);
            mbar_init(&c.o_full[i], 1);
            mbar_init(&c.drain[i], 1);
            mbar_init(&c.o_free[i], 4 * S::kHalves);
        }
        for (int i = 0; i < kStreams * 2; ++i) {
            mbar_init(&c.s_full[i], 1);
            mbar_init(&c.p_ready[i], 4 * S::kHalves);
        }
        for (int i = 0; i < S::kItems; ++i) {
            mbar_init(&c.item_full[i], 1);
            mbar_init(&c.item_empty[i], S::kSoftWarps + kStreams + 1);
        }
        for (int i = 0; i < kStreams * 4; ++i) mbar_init(&c.halves[i], 2);
        c.abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    if (warp == S::kSoftWarps) {
        tmem_alloc(&c.tmem, S::kCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    ChunkSpans spans;
    ChunkCursor at = chunk_plan<S::kThreads>(p, c.plan, spans);  // (its barriers order the above, too)
    tc_fence_after_sync();
    chunk_padding<T>(p, spans, S::kThreads);
    const uint32_t tmem = c.tmem;
    WaitCtl ctl;
    ctl.abort_flag = &c.abort_flag;
    ctl.status = p.status;
    ctl.limit_ns = p.limit_ns;
    const int per = p.tile_tokens / kStreams;  // tokens of a stream
    bool ok = true;
    if (warp >= S::kSoftWarps && warp < S::kSoftWarps + kStreams) {
        // ------------------------------------------------------------ issuers: one to a stream
        if (elect_one()) {
            const int s = warp - S::kSoftWarps;
            const uint32_t negate = p.scale_log2 < 0.0f ? 1u << 13 : 0u;  // a negative scale is a positive one of negated queries
            const uint32_t idesc_s = tile_idesc<T>(kKeys, false) | negate, idesc_o = tile_idesc<T>(p.dim, true);
            const int ksteps = p.dim >> 4;
            const uint32_t k0_lo = umma_desc_lo(smem_u32(k_ring)), q_lo = umma_desc_lo(smem_u32(smem)) + s * (S::kQBytes >> 4);
            // values: N (the head's columns) contiguous; blocks of 64 columns kBlockBytes apart, 8 keys 1024 bytes
            const uint32_t v0_lo = ((smem_u32(v_ring) & 0x3FFFFu) >> 4) | (static_cast<uint32_t>(S::kBlockBytes >> 4) << 16);
            const uint32_t t_s = tmem + s * 2 * kKeys, t_p = S::kPCol >= 0 ? tmem + S::kPCol : t_s, t_o = tmem + S::kOCol + s * (DB * 64);
            int tiles = 0;  // copied tiles before this item
            int done = 0;   // tiles of the stream before it
            int items = 0;  // items with tiles of the stream
            for (int seq = 0;; ++seq) {
                if (!(ok = mbar_wait(&c.item_full[seq % S::kItems], (seq / S::kItems) & 1, ctl, 240))) break;
                const ChunkTileItem& t = c.item[seq % S::kItems];
                if (t.tokens == 0) break;
                // (in registers: read from shared memory at each use they cost more than the products)
                const int count = t.count, from = t.from[s], to = t.to[s];
                // S(i + 1) goes where P(i - 1) was, whose product was issued before it: a thread's products run in order
                for (int i = -1; ok && i < count; ++i) {
                    const int next = i + 1;
                    if (next < count) {
                        const int n = tiles + next, d = done + next - from;
                        if (!(ok = mbar_wait(&c.k_full[n % kStages], (n / kStages) & 1, ctl, 241))) break;
                        if (next >= from && next < to) {
                            if (next == from && !(ok = mbar_wait(&c.q_full[s], items & 1, ctl, 242))) break;
                            tc_fence_after_sync();
                            const uint32_t k_lo = k0_lo + (n % kStages) * (S::kPlaneBytes >> 4);
#pragma unroll
                            for (int k = 0; k < DB * 4; ++k)
                                if (k < ksteps)
                                    umma_f16(t_s + (d & 1) * kKeys, umma_desc_join(q_lo + (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2, kDescHiSw128),
                                             umma_desc_join(k_lo + (k >> 2) * (S::kBlockBytes >> 4) + (k & 3) * 2, kDescHiSw128), idesc_s, k > 0);
                            umma_commit(&c.s_full[s * 2 + (d & 1)]);
                            umma_commit(&c.k_empty[n % kStages]);
                        } else {
                            mbar_arrive(&c.k_empty[n % kStages]);
                        }
                    }
                    if (i >= 0) {
                        const int n = tiles + i, d = done + i - from;
                        if (!(ok = mbar_wait(&c.v_clean[n % kStages], (n / kStages) & 1, ctl, 243))) break;
                        if (i >= from && i < to) {
                            if (i == from && items > 0 && !(ok = mbar_wait(&c.o_free[s], (items - 1) & 1, ctl, 244))) break;
                            if (!(ok = mbar_wait(&c.p_ready[s * 2 + (d & 1)], (d >> 1) & 1, ctl, 245))) break;
                            tc_fence_after_sync();
                            const uint32_t v_lo = v0_lo + (n % kStages) * (S::kPlaneBytes >> 4);
#pragma unroll
                            for (int k = 0; k < kKeys / 16; ++k)
                                umma_f16_ts(t_o, t_p + (d & 1) * S::kPStep + k * 8, umma_desc_join(v_lo + k * (2048 >> 4), kDescHiSw128), idesc_o, (i > from || k > 0) ? 1u : 0u);
                            umma_commit(&c.pv_done[s]);
                            umma_commit(&c.v_empty[n % kStages]);
                            if (i == to - 1) umma_commit(&c.o_full[s]);
                        } else {
                            mbar_arrive(&c.v_empty[n % kStages]);
                        }
                    }
                }
                if (!ok) break;
                tiles += count;
                done += to - from;
                items += to > from;
                mbar_arrive(&c.item_empty[seq % S::kItems]);
            }
            // Products already issued end before the CTA and its TMEM go (bounded), whoever gave up: this thread may have issued its
            // last ones and left its loop in good order before another warp's wait ran out.
            umma_commit(&c.drain[s]);
            const uint64_t t0 = global_timer_ns();
            while (!mbar_try_wait(&c.drain[s], 0) && global_timer_ns() - t0 < 2000000000ull) {
            }
        }
    } else if (warp == S::kSoftWarps + 2) {
        // ------------------------------------------------------------ copier
        const int box_shift = min(p.page_shift, 6), box = 1 << box_shift;  // a page of 128 tokens is two boxes of 64
        const int boxes = kKeys >> box_shift;
        const uint32_t k_at = smem_u32(k_ring), v_at = smem_u32(v_ring);
        int n = 0, n_v = 0;  // tiles whose keys, whose values have been asked for
        for (int seq = 0; ok; ++seq) {
            if (!(ok = warp_wait(&c.item_full[seq % S::kItems], (seq / S::kItems) & 1, ctl, 240))) break;
            const ChunkTileItem& t = c.item[seq % S::kItems];
            if (t.tokens == 0) break;
            const int h = t.h, last = t.last, count = t.count, k0 = t.k0, k1 = t.k1;
            const int32_t* pages = p.table + t.b * p.table_stride;
            // each lane knows the page of one of 32 boxes, and has asked for that of the box 32 further on: the table answers while
            // those are copied (asked for a tile ahead and looked at at once, it held every tile up by its latency)
            auto entry = [&](int i) {  // of the part's i-th box
                const int key = (last - i / boxes) * kKeys + ((i & (boxes - 1)) << box_shift);
                return i < count * boxes && key < k1 && key + box > k0 ? pages[key >> p.page_shift] : -1;
            };
            auto checked = [&](int page) {
                if (page >= p.num_pages) {
                    kv_report(p.status, kKvStatusBadId, KV_SITE_CHUNK);
                    page = -1;
                }
                return max(page, -1);
            };
            int page = checked(entry(lane)), ahead = entry(32 + lane);
            int at_box = 0;  // the tile's first box, among the 32
            for (int i = 0; i < count; ++i, at_box += boxes) {
                if (at_box == 32) {
                    page = checked(ahead);
                    ahead = entry(i * boxes + 32 + lane);
                    at_box = 0;
                }
                const int stage = n % kStages;
                const unsigned none = __ballot_sync(0xFFFFFFFFu, page < 0) >> at_box;
                // a lane to each copy of 64 columns of a box: one after the other from one lane they took the warp 110 cycles each, and a tile of
                // four pages of 16 tokens is 16 of them
                const int b = lane / DB, d = lane % DB;
                const int pg = __shfl_sync(0xFFFFFFFFu, page, at_box + b);  // (page -1 lies outside the map: zeros)
                const int row = (((last - i) * boxes + b) << box_shift) & ((1 << p.page_shift) - 1);
                const uint32_t place = stage * S::kPlaneBytes + b * box * 128 + d * S::kBlockBytes;
                if (n >= kStages && !(ok = warp_wait(&c.k_empty[stage], (n / kStages - 1) & 1, ctl, 246))) break;
                if (lane == 0) {
                    uint32_t holes = 0;
                    if (none & ((1u << boxes) - 1))
                        for (int x = 0; x < boxes; ++x)
                            if (none >> x & 1) holes |= ((1u << (box / 16)) - 1) << (x * (box / 16));
                    *reinterpret_cast<volatile uint32_t*>(&c.holes[n % S::kHoles]) = holes;
                    mbar_arrive_expect_tx(&c.k_full[stage], S::kPlaneBytes);
                }
                __syncwarp();
                if (b < boxes) tma_load_4d(k_at + place, &map_k, &c.k_full[stage], d * 64, row, h, pg);
                ++n;
                if (n_v >= kStages && !(ok = warp_wait(&c.v_empty[stage], (n_v / kStages - 1) & 1, ctl, 246))) break;
                if (lane == 0) mbar_arrive_expect_tx(&c.v_full[stage], S::kPlaneBytes);
                __syncwarp();
                if (b < boxes) tma_load_4d(v_at + place, &map_v, &c.v_full[stage], d * 64, row, h, pg);
                ++n_v;
            }
            if (!ok) break;  // (a tile's values were not asked for, its keys may have been)
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.item_empty[seq % S::kItems]);
        }
        // Copies in flight land before the CTA goes (bounded), whoever gave up; those of a place before its last ones have (the place was
        // free again).
        const uint64_t t0 = global_timer_ns();
        for (int i = max(0, n - kStages); i < n; ++i)
            while (!mbar_try_wait(&c.k_full[i % kStages], (i / kStages) & 1) && global_timer_ns() - t0 < 2000000000ull) {
            }
        for (int i = max(0, n_v - kStages); i < n_v; ++i)
            while (!mbar_try_wait(&c.v_full[i % kStages], (i / kStages) & 1) && global_timer_ns() - t0 < 2000000000ull) {
            }
    } else if (warp == S::kSoftWarps + 3) {
        // ------------------------------------------------------------ planner and cleaner
        ChunkDesc tail = {0, 0, 0, 0};
        WaitCtl patient = ctl;  // for an item's time, not a tile's; the others' waits raise the flag that ends this one, too
        patient.limit_ns = 16 * ctl.limit_ns;
        int planned = 0, n = 0, items = 0;
        bool end = false;
        // A span that begins inside an item takes the end of that one last: then all CTAs of a head begin at the same keys and go over them
        // together, and the keys come from L2 more often.  Groups of 4 or 2, heads of 128, with it / without: 8 requests of 65,536 by 512 tokens
        // 4,107 / 4,271 us, 4 of 32,768 by 1,024 2,073 / 2,150, 16 of 8,192 by 1,024 2,158 / 2,170; no difference for 4,096 tokens of two requests of
        // 32,768 by 4 heads; 512 tokens of two requests of 131,072 by heads of 256 4,768 / 4,679.
        ChunkCursor kept;
        bool keeps = chunk_keep(p, at, kept);
        for (int seq = 0; ok; ++seq) {
            // two items ahead: their places are free when the item two before this one has ended
            for (; !end && planned <= seq + 2; ++planned) {
                ChunkTileItem& t = c.item[planned % S::kItems];
                if (planned >= S::kItems && !(ok = warp_wait(&c.item_empty[planned % S::kItems], (planned / S::kItems - 1) & 1, patient, 239))) break;
                if (at.left <= 0 && keeps) {
                    at = kept;
                    keeps = false;
                }
                end = at.left <= 0;
                if (lane == 0) {
                    if (end) {
                        t.tokens = 0;
                    } else {
                        const ChunkItem it = chunk_item(p, at);
                        chunk_record<kStreams, kKeys>(p, at, it, t);
                        if (it.first && !it.last) tail = ChunkDesc{chunk_parts(spans, blockIdx.x, it.rest), it.token, it.tokens, it.hv};
                    }
                    mbar_arrive(&c.item_full[planned % S::kItems]);
                }
                if (!end) chunk_next(p, at);
            }
            __syncwarp();
            if (!ok) break;
            const ChunkTileItem& t = c.item[seq % S::kItems];
            if (*reinterpret_cast<const volatile int*>(&t.tokens) == 0) break;
            const int last = t.last, count = t.count, item_lo = t.lo, item_hi = t.hi, all_lo = t.all_lo, all_hi = t.all_hi;
            if (lane == 0 && count > 0) c.odd[items & 3] = 0;
            __syncwarp();
            for (int i = 0; i < count; ++i, ++n) {
                const int stage = n % kStages, key0 = (last - i) * kKeys;
                if (!(ok = warp_wait(&c.v_full[stage], (n / kStages) & 1, ctl, 247))) break;
                const int dead0 = max(item_lo - key0, 0), dead1 = min(item_hi - key0, kKeys);  // rows before and from which on nobody may look
                const bool cut = key0 < all_lo || key0 + kKeys > all_hi;
                if (dead0 > 0 || dead1 < kKeys || cut) {
                    uint8_t* base = v_ring + stage * S::kPlaneBytes;
                    bool odd = false;
#pragma unroll 4
                    for (int x = lane; x < kKeys * 8 * DB; x += 32) {
                        const int row = (x >> 3) % kKeys;  // (16-byte pieces change places within a row only)
                        uint4* piece = reinterpret_cast<uint4*>(base + x * 16);
                        uint4 v = *piece;
                        if (row < dead0 || row >= dead1) {
                            *piece = make_uint4(0, 0, 0, 0);
                        } else if (cut && take_out_odd<T>(v)) {
                            *piece = v;
                            odd = true;
                        }
                    }
                    if (odd) c.odd[items & 3] = 1;
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&c.v_clean[stage]);
            }
            items += count > 0;
        }
        if (lane == 0) p.desc[blockIdx.x] = tail;
    } else if (warp < S::kSoftWarps) {
        // ------------------------------------------------------------ softmax: thread = row = TMEM lane
        const int s = S::kHalves == 2 ? 0 : warp >> 2, half = S::kHalves == 2 ? warp >> 2 : 0, r = tid & 127, pair = s * 4 + (warp & 3);
        const uint32_t inv_heads = 65536u / p.part_heads + 1;
        const int tok = token_of(r, inv_heads), head = r - tok * p.part_heads;
        const uint32_t t_rows = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16), t_o = t_rows + S::kOCol + s * (DB * 64);
        const uint32_t t_p = S::kPCol >= 0 ? t_rows + S::kPCol : t_rows + s * 2 * kKeys;
        const float scale = CAP || BIAS ? 1.0f : fmaxf(fabsf(p.scale_log2), 1.2e-38f);  // zero would turn masked logits into NaN
        const float slack = fminf(8.0f / scale, 3e38f);  // (finite: added to a reference of -infinity it stays that)
        const float factor = fabsf(CAP ? p.cap_in : p.scale_log2);  // of a product, where there is a cap or a bias
        const uint64_t scale2 = pair32(scale, scale);
        constexpr int kMine = S::kMine;
        auto arrive = [&](uint64_t* bar) {  // once for the warp: 128 threads' arrivals at one address took as long as a third of a tile
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        int turn = 0;  // of what the halves tell each other
        auto tell = [&](float v) {  // the other half's number (whatever it is where the wait failed and ok is false)
            c.told[pair][turn & 1][half][lane] = v;
            __syncwarp();
            if (lane == 0) mbar_arrive(&c.halves[pair]);
            ok = warp_wait(&c.halves[pair], turn & 1, ctl, 251);
            const float other = *reinterpret_cast<volatile float*>(&c.told[pair][turn & 1][half ^ 1][lane]);
            ++turn;
            return other;
        };
        int n = 0, items = 0, all_items = 0, tiles = 0;  // tiles and items of this stream; items with tiles; copied tiles
        for (int seq = 0; ok; ++seq) {
            if (!(ok = warp_wait(&c.item_full[seq % S::kItems], (seq / S::kItems) & 1, ctl, 240))) break;
            const ChunkTileItem& t = c.item[seq % S::kItems];
            if (t.tokens == 0) break;
            const int my_tok = s * per + tok, pos = t.pos + my_tok;
            const bool live = tok < per && my_tok < t.tokens && head < t.heads;
            const int from = t.from[s], to = t.to[s];
            float m = -INFINITY, l = 0.0f;  // reference of the exponentials (in logits before scaling), sum over this half's keys
            int lo = 0, hi = 0x7FFFFFFF;    // rows that are nobody's look at everything: no tile is cut for them
            if (live) chunk_sees(p, t.r, pos, true, lo, hi);
            const int warp_lo = __reduce_max_sync(0xFFFFFFFFu, lo), warp_hi = __reduce_min_sync(0xFFFFFFFFu, hi);
            if (to > from) {
                // queries: rows of 128 bytes to a 64-column block, 16-byte pieces exchanged by the row's low bits
                constexpr int kPieces = DB * 8, kStep = S::kRowThreads / kPieces;
                const int piece = r % kPieces;
                const uint32_t dst = smem_u32(smem) + s * S::kQBytes + (piece >> 3) * (128 * 128);
                const T* q0 = static_cast<const T*>(p.q) + static_cast<int64_t>(t.token + s * per) * p.q_stride[0] + static_cast<int64_t>(t.head0) * p.q_stride[1] + piece * 8;
#pragma unroll 4
                for (int row = (half * 128 + r) / kPieces; row < 128; row += kStep) {
                    const int tk = token_of(row, inv_heads), hd = row - tk * p.part_heads;
                    const bool in = piece * 8 < p.dim && tk < per && s * per + tk < t.tokens && hd < t.heads;
                    cp_async16(dst + row * 128 + (((piece & 7) ^ (row & 7)) << 4), in ? q0 + tk * p.q_stride[0] + hd * p.q_stride[1] : static_cast<const T*>(p.q), in);
                }
                cp_async_commit();
                cp_async_wait<0>();
                fence_proxy_async_smem();
                arrive(&c.q_full[s]);
            }
            const int last = t.last;
            float slope = 0.0f;
            if (BIAS && live) slope = p.slopes[t.head0 + head] * 1.4426950408889634f;

            for (int i = from; i < to; ++i, ++n) {
                const int key0 = (last - i) * kKeys + half * kMine;
                const int buffer = s * 2 + (n & 1);
                const uint32_t t_s = t_rows + buffer * kKeys;
                if (!(ok = warp_wait(&c.s_full[buffer], (n >> 1) & 1, ctl, 248))) break;
                tc_fence_after_sync();
                uint32_t x[kMine];
                if constexpr (kMine == 64) tmem_ld_32x32b_x64(t_s + half * kMine, x);
                else tmem_ld_32x32b_x32(t_s + half * kMine, x);
                const uint32_t holes = *reinterpret_cast<volatile uint32_t*>(&c.holes[(tiles + i) % S::kHoles]) >> (half * (kMine / 16));
                tmem_wait_ld_regs(x);
                if (CAP) {
                    float most = 0.0f;
                    const uint64_t f2 = pair32(factor, factor);
#pragma unroll
                    for (int i = 0; i < kMine; i += 2) {
                        const uint64_t y = mul2(pair32(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), f2);
                        x[i] = static_cast<uint32_t>(y);
                        x[i + 1] = static_cast<uint32_t>(y >> 32);
                        most = max3f(most, fabsf(lo32(y)), fabsf(hi32(y)));
                    }
                    const uint64_t cap2 = pair32(p.cap_out, p.cap_out);
                    auto near = [&](uint64_t y) {  // cap * tanh of a pair within [-1, 1]
                        const uint64_t u = mul2(y, y);
                        uint64_t t = pair32(tanh_term(6), tanh_term(6));
#pragma unroll
                        for (int k = 5; k >= 0; --k) t = fma2(t, u, pair32(tanh_term(k), tanh_term(k)));
                        return mul2(t, mul2(y, cap2));
                    };
                    if (!__any_sync(0xFFFFFFFFu, most > 1.0f)) {  // as a rule, for caps that keep logits within reason
#pragma unroll
                        for (int i = 0; i < kMine; i += 2) {
                            const uint64_t t = near(pair32(__uint_as_float(x[i]), __uint_as_float(x[i + 1])));
                            x[i] = static_cast<uint32_t>(t);
                            x[i + 1] = static_cast<uint32_t>(t >> 32);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kMine; i += 2) {
                            const float a = __uint_as_float(x[i]), b = __uint_as_float(x[i + 1]);
                            const uint64_t t = near(pair32(a, b)), far = mul2(pair32(tanh_far(a), tanh_far(b)), cap2);
                            x[i] = fabsf(a) > 1.0f ? static_cast<uint32_t>(far) : static_cast<uint32_t>(t);
                            x[i + 1] = fabsf(b) > 1.0f ? static_cast<uint32_t>(far >> 32) : static_cast<uint32_t>(t >> 32);
                        }
                    }
                }
                if (BIAS) {  // less slope times the distance; keys in front of the row's token, nearly all of them, lie on one line
                    const float near = static_cast<float>(key0 - pos);
                    const uint64_t line = pair32(slope, slope), f2 = pair32(factor, factor);
                    if (__all_sync(0xFFFFFFFFu, key0 + kMine - 1 <= pos)) {
#pragma unroll
                        for (int i = 0; i < kMine; i += 2) {
                            const uint64_t y = pair32(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), d = add2(pair32(near, near), pair32(i, i + 1));
                            const uint64_t z = fma2(line, d, CAP ? y : mul2(y, f2));
                            x[i] = static_cast<uint32_t>(z);
                            x[i + 1] = static_cast<uint32_t>(z >> 32);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < kMine; ++i) {
                            const float y = __uint_as_float(x[i]);
                            x[i] = __float_as_uint(fmaf(-slope, fabsf(near + i), CAP ? y : y * factor));
                        }
                    }
                }
                if (key0 < warp_lo || key0 + kMine > warp_hi || holes) {  // not all rows of the warp see all of it
                    const int a = lo - key0, b = hi - key0;
#pragma unroll
                    for (int i = 0; i < kMine; ++i)
                        if (i < a || i >= b || (holes >> (i / 16) & 1)) x[i] = 0xFF800000u;
                }
                // The exponentials are taken against the reference as it is, the maximum beside them (the special function unit leaves room for
                // it); where it turns out to be too far above, which is rare but for a row's first tile, they are taken again.
                uint64_t sum[2];
                while (true) {
                    const float base = m == -INFINITY ? 0.0f : m * scale;
                    const uint64_t off = pair32(-base, -base);
                    float part[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    sum[0] = sum[1] = 0;  // of two 32-bit sums each
#pragma unroll
                    for (int q = 0; q < kMine / 32; ++q) {
                        uint32_t out[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float a = __uint_as_float(x[q * 32 + i]), b = __uint_as_float(x[q * 32 + i + 1]);
                            part[i / 2 & 3] = max3f(part[i / 2 & 3], a, b);
                            const uint64_t z = fma2(pair32(a, b), scale2, off);
                            const uint64_t w = pair32(exp2_fast(lo32(z)), exp2_fast(hi32(z)));
                            sum[i / 2 & 1] = add2(sum[i / 2 & 1], w);
                            out[i / 2] = Pair16<T>::pack(lo32(w), hi32(w));
                        }
                        tmem_st_32x32b_x16(t_p + (n & 1) * S::kPStep + half * (kMine / 2) + q * 16, out);
                    }
                    float top = fmaxf(max3f(part[0], part[1], part[2]), part[3]);
                    if (S::kHalves == 2) {
                        top = fmaxf(top, tell(top));
                        if (!ok) break;
                    }
                    const bool grow = top > m + slack;
                    if (!__any_sync(0xFFFFFFFFu, grow)) break;
                    const float fix = grow && m > -INFINITY ? exp2_fast((m - top) * scale) : 1.0f;
                    if (grow) m = top;
                    if (__any_sync(0xFFFFFFFFu, fix != 1.0f)) {  // (something was seen before: i > from)
                        if (!(ok = warp_wait(&c.pv_done[s], (n - 1) & 1, ctl, 249))) break;
                        tc_fence_after_sync();
                        l *= fix;
                        const int q1 = p.dim >> 4;  // the first half takes the first columns, 16 at a time: the logits stay in registers
                        for (int q = half * ((q1 + 1) / 2); q < (S::kHalves == 2 && !half ? (q1 + 1) / 2 : q1); ++q) {
                            uint32_t o[16];
                            tmem_ld_32x32b_x16(t_o + q * 16, o);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fix);
                            tmem_st_32x32b_x16(t_o + q * 16, o);
                        }
                    }
                }
                if (!ok) break;
                const uint64_t both = add2(sum[0], sum[1]);
                l += lo32(both) + hi32(both);
                tmem_wait_st();
                tc_fence_before_sync();
                arrive(&c.p_ready[buffer]);
            }
            if (!ok) break;
            if (to > from) {
                if (S::kHalves == 2) l += tell(l);
                if (!ok || !(ok = warp_wait(&c.o_full[s], items & 1, ctl, 250))) break;
                tc_fence_after_sync();
                ++items;
            }
            const bool whole = t.whole;
            const bool odd = t.count > 0 && *reinterpret_cast<volatile int*>(&c.odd[all_items & 3]) != 0;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int row = my_tok * p.part_heads + head;
            float* slot = p.slots + static_cast<int64_t>(t.slot) * p.rows * (p.dim + 2);
            T* out = static_cast<T*>(p.out) + static_cast<int64_t>(t.token + my_tok) * p.out_stride[0] + static_cast<int64_t>(t.head0 + head) * p.out_stride[1];
            const int q1 = (p.dim + 31) / 32;
            for (int q = half * ((q1 + 1) / 2); q < (S::kHalves == 2 && !half ? (q1 + 1) / 2 : q1); ++q) {
                uint32_t o[32];
                if (to > from) {
                    tmem_ld_32x32b_x32(t_o + q * 32, o);
                    tmem_wait_ld_regs(o);
                }
                if (!live) continue;
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    if (q * 32 + i >= p.dim) continue;
                    float f[8];
#pragma unroll
                    for (int y = 0; y < 8; ++y) f[y] = l == 0.0f ? 0.0f : __uint_as_float(o[i + y]);
                    if (odd) add_odd<T>(p, t.b, t.h, lo, hi, t.k0, t.k1, (t.all_lo + kKeys - 1) & -kKeys, t.all_hi & -kKeys, q * 32 + i, f);
                    if (whole) {
#pragma unroll
                        for (int y = 0; y < 8; ++y) f[y] *= inv;
                        *reinterpret_cast<uint4*>(out + q * 32 + i) = pack8<T>(f);
                    } else {
                        float4* dst = reinterpret_cast<float4*>(slot + static_cast<int64_t>(row) * p.dim + q * 32 + i);
                        dst[0] = make_float4(f[0], f[1], f[2], f[3]);
                        dst[1] = make_float4(f[4], f[5], f[6], f[7]);
                    }
                }
            }
            if (to > from) {
                tc_fence_before_sync();
                arrive(&c.o_free[s]);
            }
            if (live && half == 0) {
                const float best = m * scale;
                if (whole) {
                    if (p.lse)
                        p.lse[static_cast<int64_t>(t.token + my_tok) * p.group * p.n_kv_heads + t.head0 + head] =
                            l == 0.0f ? -INFINITY : (best + log2f(l)) * 0.69314718055994531f;
                } else {
                    slot[p.rows * p.dim + row] = l == 0.0f ? -INFINITY : best;
                    slot[p.rows * (p.dim + 1) + row] = l;
                }
            }
            tiles += t.count;
            all_items += t.count > 0;
            arrive(&c.item_empty[seq % S::kItems]);
        }
        __syncwarp();
        tmem_wait_st();  // (a wait that ran out may have left stores behind it)
    }
    // ------------------------------------------------------------ teardown (also the abort path)
    tc_fence_before_sync();
    __syncthreads();
    if (warp == S::kSoftWarps) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, S::kCols);
    }
}

}  // namespace ivf
