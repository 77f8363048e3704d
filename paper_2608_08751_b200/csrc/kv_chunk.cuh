// Attention of each request's new tokens over its whole cache.
//
// out = sum_k exp(z_k - m) v_k / sum_k exp(z_k - m) over the keys k that a token at position p of its request sees:
//   z_k = scale * q . k,  with a cap  z_k = cap * tanh(scale * q . k / cap),  with a bias  z_k - slope_head * |p - k|
//   seen: k < the request's length, k <= p or k < its prefix, and p - k < the window.  Always an interval [lo, hi).
// One pass over the keys with a running maximum and sum, both in 32 bits; the exponentials take the cache's 16-bit type as
// operands of the second product (off by up to 2^-8 or 2^-11 of themselves; in two parts, 2^-16 or 2^-22, where a tile of 16 rows has 8 of them at
// most), the sum that divides them is of the unrounded ones.
//
// How the work is shared out.  An item is a tile of new tokens of one request and one kv head: the tile's tokens by the
// head's group of query heads are the rows of one matrix product.  Only the device knows the lengths, and they are ragged,
// so the grid is as many CTAs as live on the card and each takes an equal, contiguous span of the line of all items, an item
// being as long as the keys it reads and a constant for its start and end.  Lengths, prefixes and windows make hi and lo
// of a request's tiles piecewise linear, so every place on the line follows from sums in closed form and one scan over the
// requests, which each CTA does for itself.  Where a span begins or ends inside an item its CTA leaves the rows' sums in
// the workspace (two items at most), and a second kernel joins them.  Every order is fixed: a call gives the same bits each time.
//
// A value that is not finite at a key that only some rows of a tile see would reach the others as 0 * inf.  In pieces that not
// all rows see such values are looked for, taken out of the product, and added at the end to the rows that do see them.
#pragma once
#include "kv_attend.cuh"

namespace ivf {

constexpr int kChunkMaxSms = 148;  // CTAs that a call may use: on each of so many SMs three, two or one of small tiles (heads of up to 64, 128, 256), one of large ones

struct ChunkDesc {  // of the item that a CTA's span ends in
    int parts;      // CTAs that have a part of it; 0: the span ends with an item
    int token, tokens, hv;
};

struct ChunkParams {
    const void* q;
    int64_t q_stride[2];
    int64_t n_tokens;
    int group, n_kv_heads, dim;
    KvPlane kc, vc;
    int64_t num_pages;
    const int32_t* table;
    int64_t table_stride;
    int n_req, max_blocks, page_shift;
    const int32_t *token_start, *kv_lens, *prefix;  // prefix may be null
    int window;            // 0: none
    float scale_log2;      // scale * log2(e)
    float cap_in, cap_out; // with a cap: z in base 2 = cap_out * tanh(cap_in * (q . k)); cap_out 0: none
    const float* slopes;   // [n_heads] or null
    void* out;
    int64_t out_stride[2];
    float* lse;  // [n_tokens][n_heads] or null
    int* status;
    int tile_tokens;       // tokens of a tile
    int part_heads, parts; // query heads of a tile's rows, and how many such parts a group has
    int item_cost;         // of an item's start and end, in keys
    int least;             // keys of a span, at least
    int grain;             // items are cut at multiples of this many keys (a power of two)
    int rows;              // of a slot: tile_tokens * part_heads, and one more if that is odd
    ChunkDesc* desc;       // [CTAs]
    float* slots;          // [2 * CTAs][rows * (dim + 2)]: sums, then maxima, then totals; row = token of the tile * part_heads + head
    uint64_t limit_ns;
};

// ------------------------------------------------------------------ the line of items
// (also compiled for the host, where ivf_debug_kv_chunk_span walks it)
struct ChunkReq {
    int start, fresh;  // its first row, its rows in this call
    int base;          // position of the first
    int len, far;      // tokens in the cache; keys that the table has columns for
    int prefix, tiles;
    bool blind;        // its lengths make no sense: its tokens see nothing
    int64_t j_hi, j_lo;  // tiles before these end at the prefix, begin at key 0
};

// `taken`: rows before it are an earlier request's, or nobody's.  That is the start of the request before (where token_start descends, which is an
// error, the largest so far), so every row has one request.
__host__ __device__ __forceinline__ ChunkReq chunk_req(const ChunkParams& p, int b, int taken, bool report) {
    ChunkReq r;
    const int s0 = p.token_start[b], s1 = p.token_start[b + 1], len = p.kv_lens[b];
    const int64_t given = max(static_cast<int64_t>(s1) - s0, static_cast<int64_t>(0));
    r.blind = len < given;
    r.start = max(s0, taken);
    const int64_t room = static_cast<int64_t>(p.max_blocks) << p.page_shift;
#ifdef __CUDA_ARCH__
    if (report && (s0 < 0 || s1 < s0 || r.blind || len > room)) kv_report(p.status, kKvStatusBadId, KV_SITE_CHUNK);
#endif
    r.fresh = static_cast<int>(max(min(static_cast<int64_t>(s1), p.n_tokens) - r.start, static_cast<int64_t>(0)));
    r.len = r.blind ? 0 : len;
    r.base = r.blind ? 0 : static_cast<int>(len - given + min(static_cast<int64_t>(r.start) - s0, given));
    r.far = static_cast<int>(min(static_cast<int64_t>(r.len), room));
    r.prefix = p.prefix ? max(0, min(p.prefix[b], r.len)) : 0;
    r.tiles = (r.fresh + p.tile_tokens - 1) / p.tile_tokens;
    // tile j ends at max(base + (j + 1) T, prefix) and begins at max(base + j T - window + 1, 0)
    const unsigned T = p.tile_tokens;
    const int a = r.prefix - r.base, c = p.window - 1 - r.base;
    r.j_hi = a <= 0 ? 0 : (static_cast<unsigned>(a) - 1) / T;
    r.j_lo = p.window <= 0 ? r.tiles : c < 0 ? 0 : static_cast<unsigned>(c) / T + 1;
    return r;
}
__host__ __device__ __forceinline__ int chunk_hi(const ChunkParams& p, const ChunkReq& r, int j) {  // one past the last key that the tile sees
    const int last = min((j + 1) * p.tile_tokens, r.fresh);
    return r.blind ? 0 : max(r.base + last, r.prefix);
}
__host__ __device__ __forceinline__ int chunk_lo(const ChunkParams& p, const ChunkReq& r, int j) {
    return r.blind || p.window <= 0 ? 0 : max(r.base + j * p.tile_tokens - p.window + 1, 0);
}
__host__ __device__ __forceinline__ int64_t chunk_weight(const ChunkParams& p, const ChunkReq& r, int j) {
    return static_cast<int64_t>(chunk_hi(p, r, j)) - chunk_lo(p, r, j) + p.item_cost;
}
// Weights of the tiles before tile i of one head.
__host__ __device__ __forceinline__ int64_t chunk_before(const ChunkParams& p, const ChunkReq& r, int64_t i) {
    const int64_t cost = i * p.item_cost;
    if (r.blind || i == 0) return cost;
    const int64_t n = i == r.tiles ? i - 1 : i, T = p.tile_tokens;  // the last tile may be short
    const int64_t a = min(r.j_hi, n);
    int64_t sum = a * r.prefix + (n - a) * r.base + T * ((n * (n + 1) - a * (a + 1)) / 2);
    if (n < i) sum += chunk_hi(p, r, static_cast<int>(n));
    const int64_t c = min(r.j_lo, i);
    sum -= (i - c) * (static_cast<int64_t>(r.base) - p.window + 1) + T * ((i * (i - 1) - c * (c - 1)) / 2);
    return sum + cost;
}

// A CTA's place on the line.
struct ChunkCursor {
    int b, hv, tile;
    int64_t off;   // inside the item
    int64_t left;  // of the span
    ChunkReq r;    // of request b
};
template <int THREADS>
struct ChunkPlan {
    int64_t warp_sum[THREADS / 32];
    ChunkCursor at;
};
// Where the spans begin: the line in `ctas` parts of `whole` and a share of what is left over.
struct ChunkSpans {
    int ctas, over;
    int64_t whole;
    int end;  // rows from here on are no request's
    __host__ __device__ __forceinline__ int64_t begin(int c) const { return whole * c + static_cast<unsigned>(over * c) / static_cast<unsigned>(ctas); }
};
// (a 64-bit division takes a hundred instructions, and nearly every line is shorter)
__host__ __device__ __forceinline__ int64_t chunk_div(int64_t a, int64_t b) {
    return (a | b) >> 32 ? a / b : static_cast<int64_t>(static_cast<unsigned>(a) / static_cast<unsigned>(b));
}

// Where a weight `rest` behind the start of request b0 lies, before request b1.
__host__ __device__ __forceinline__ void chunk_locate(const ChunkParams& p, int b0, int b1, int taken, int64_t rest, ChunkCursor& at) {
    const int hvs = p.n_kv_heads * p.parts;
    for (int b = b0; b < b1; ++b) {
        const ChunkReq r = chunk_req(p, b, taken, false);
        taken = r.start;
        const int64_t one = chunk_before(p, r, r.tiles);
        if (rest >= one * hvs) {
            rest -= one * hvs;
            continue;
        }
        at.b = b;
        at.hv = static_cast<int>(chunk_div(rest, one));
        rest -= at.hv * one;
        int lo = 0, hi = r.tiles;  // before(lo) <= rest < before(hi)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (chunk_before(p, r, mid) <= rest) lo = mid;
            else hi = mid;
        }
        at.tile = lo;
        at.off = rest - chunk_before(p, r, lo);
        at.r = r;
        return;
    }
}
// The line in spans of at least p.least keys, as many as `most` at the most.
__host__ __device__ __forceinline__ void chunk_spans(const ChunkParams& p, int64_t total, int most, ChunkSpans& spans) {
    spans.ctas = static_cast<int>(max(min(chunk_div(total, p.least), static_cast<int64_t>(most)), static_cast<int64_t>(1)));
    spans.whole = chunk_div(total, spans.ctas);
    spans.over = static_cast<int>(total - spans.whole * spans.ctas);
}

// All threads: the CTA's cursor (left = 0: nothing to do) and where the spans lie.
template <int THREADS>
__device__ __forceinline__ ChunkCursor chunk_plan(const ChunkParams& p, ChunkPlan<THREADS>& s, ChunkSpans& spans) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.n_req + THREADS - 1) / THREADS;
    const int b0 = min(tid * per, p.n_req), b1 = min(b0 + per, p.n_req);
    const int hvs = p.n_kv_heads * p.parts;
    int64_t mine, upto;
    int taken = 0;
    auto add_up = [&](bool report) {  // whether token_start descends among the thread's requests
        bool down = false;
        mine = 0;
        int t = taken;
        for (int b = b0; b < b1; ++b) {
            const ChunkReq r = chunk_req(p, b, t, report);
            t = r.start;
            down |= p.token_start[b + 1] < t;
            mine += hvs * chunk_before(p, r, r.tiles);
        }
        upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) s.warp_sum[warp] = upto;
        return down;
    };
    const bool down = add_up(blockIdx.x == 0);
    if (tid == 0) s.at.left = 0;
    spans.end = p.token_start[p.n_req];
    if (__syncthreads_or(down)) {  // an error: once more, with what all requests before the thread's have taken
        for (int b = 0; b < b0; ++b) taken = max(taken, p.token_start[b]);
        for (int b = 0; b < p.n_req; ++b) spans.end = max(spans.end, p.token_start[b]);
        add_up(false);
        __syncthreads();
    }
    int64_t total = 0;
    upto -= mine;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) upto += s.warp_sum[w];
        total += s.warp_sum[w];
    }
    chunk_spans(p, total, gridDim.x, spans);
    const int c = blockIdx.x;
    if (c < spans.ctas) {
        const int64_t u0 = spans.begin(c), u1 = spans.begin(c + 1);
        if (u0 >= upto && u0 < upto + mine) {
            chunk_locate(p, b0, b1, taken, u0 - upto, s.at);
            s.at.left = u1 - u0;
        }
    }
    __syncthreads();
    return s.at;
}

// One item, or the part of it that a span has.
struct ChunkItem {
    int hv, token, tokens;  // first token of the tile, and how many
    int pos;                // position of the first
    int lo, hi;             // keys that some row sees
    int k0, k1;             // of them this part's
    bool first, last;       // the part begins, ends the item
    int64_t rest;           // of the item behind the part
};
__host__ __device__ __forceinline__ ChunkItem chunk_item(const ChunkParams& p, const ChunkCursor& at) {
    ChunkItem it;
    const ChunkReq& r = at.r;
    const int64_t w = chunk_weight(p, r, at.tile), take = min(at.left, w - at.off);
    it.hv = at.hv;
    it.token = r.start + at.tile * p.tile_tokens;
    it.tokens = min(p.tile_tokens, r.fresh - at.tile * p.tile_tokens);
    it.pos = r.base + at.tile * p.tile_tokens;
    it.lo = chunk_lo(p, r, at.tile);
    it.hi = min(chunk_hi(p, r, at.tile), r.far);
    it.lo = min(it.lo, it.hi);
    it.first = at.off == 0;
    it.last = at.off + take == w;
    it.rest = w - at.off - take;
    auto cut = [&](int64_t off) {  // a place in the item as a key
        const int64_t k = (it.lo + max(off - p.item_cost, static_cast<int64_t>(0))) & -static_cast<int64_t>(p.grain);
        return static_cast<int>(max(static_cast<int64_t>(it.lo), min(k, static_cast<int64_t>(it.hi))));
    };
    it.k0 = it.first ? it.lo : cut(at.off);
    it.k1 = it.last ? it.hi : cut(at.off + take);
    return it;
}
__host__ __device__ __forceinline__ void chunk_next(const ChunkParams& p, ChunkCursor& at) {
    const int64_t take = min(at.left, chunk_weight(p, at.r, at.tile) - at.off);
    at.left -= take;
    at.off = 0;
    if (++at.tile < at.r.tiles) return;
    at.tile = 0;
    if (++at.hv < p.n_kv_heads * p.parts) return;
    at.hv = 0;
    if (at.left > 0)  // (weights left: there is a request with tokens)
        do at.r = chunk_req(p, ++at.b, at.r.start, false);
        while (at.r.tiles == 0 && at.b < p.n_req - 1);
}
// A span that begins inside an item and goes on behind it: `at` moves on to the next item, `kept` is the end of the first one, to be taken last.
__host__ __device__ __forceinline__ bool chunk_keep(const ChunkParams& p, ChunkCursor& at, ChunkCursor& kept) {
    if (at.left <= 0 || at.off == 0) return false;
    const int64_t w = chunk_weight(p, at.r, at.tile) - at.off;
    if (at.left <= w) return false;
    kept = at;
    kept.left = w;
    chunk_next(p, at);
    return true;
}
// The CTAs that take part in an item whose rest lies behind this CTA's span.
__host__ __device__ __forceinline__ int chunk_parts(const ChunkSpans& spans, int c, int64_t rest) {
    const int64_t end = spans.begin(c + 1) + rest;  // of the item
    int past = min(c + 1 + static_cast<int>(chunk_div(rest, spans.whole + 1)), spans.ctas);  // no span is longer: none before it ends the item
    while (past < spans.ctas && spans.begin(past) < end) ++past;
    return past - c;
}

// Keys that a token at position pos sees.
__host__ __device__ __forceinline__ void chunk_sees(const ChunkParams& p, const ChunkReq& r, int pos, bool live, int& lo, int& hi) {
    live = live && !r.blind;
    lo = live && p.window > 0 ? max(pos - p.window + 1, 0) : 0;
    hi = live ? min(max(pos + 1, r.prefix), r.far) : 0;
}

// Tokens that belong to no request: zeros.
template <typename T>
__device__ __forceinline__ void chunk_padding(const ChunkParams& p, const ChunkSpans& spans, int threads) {
    const int n_heads = p.group * p.n_kv_heads;
    const int64_t before = max(static_cast<int64_t>(0), min(static_cast<int64_t>(p.token_start[0]), p.n_tokens));
    const int64_t from = max(before, min(static_cast<int64_t>(spans.end), p.n_tokens));
    const int64_t pad = before + p.n_tokens - from;
    if (pad == 0) return;
    const int pieces = p.dim / 8;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * threads + threadIdx.x; i < pad * n_heads * pieces; i += static_cast<int64_t>(gridDim.x) * threads) {
        const int c = static_cast<int>(i % pieces);
        const int64_t row = i / pieces, at = row / n_heads, t = at < before ? at : from + at - before;
        const int head = static_cast<int>(row % n_heads);
        *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + t * p.out_stride[0] + head * p.out_stride[1] + c * 8) = make_uint4(0, 0, 0, 0);
        if (c == 0 && p.lse) p.lse[t * n_heads + head] = -INFINITY;
    }
}

__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// tanh(x) for |x| <= 1 is x P(x^2), P of degree 6 (Remez exchange on the relative error; 1.6e-7 in 32 bits).  As 1 - 2 / (1 + exp(2 x)), which
// is what is left for larger ones, a small logit would keep no more digits than the cap has.
__host__ __device__ constexpr float tanh_term(int k) {
    constexpr float term[7] = {0.9999999403953552f, -0.33332839608192444f, 0.13325203955173492f, -0.05345702916383743f, 0.020289979875087738f,
                               -0.006203379016369581f, 0.0010410225950181484f};
    return term[k];
}
__device__ __forceinline__ float tanh_far(float x) {
    return copysignf(fmaf(-2.0f, rcp_fast(1.0f + exp2_fast(2.885390043258667f * fabsf(x))), 1.0f), x);
}
// A product as a logit in base 2, before the bias.
__device__ __forceinline__ float chunk_logit(const ChunkParams& p, float s) {
    if (p.cap_out == 0.0f) return s * p.scale_log2;
    const float x = s * p.cap_in, u = x * x;
    float y = tanh_term(6);
#pragma unroll
    for (int i = 5; i >= 0; --i) y = fmaf(y, u, tanh_term(i));
    float t = x * y;
    if (fabsf(x) > 1.0f) t = tanh_far(x);
    return p.cap_out * t;
}

// The numbers of `v` (two 16-bit ones to a word) that are not finite; `clean` gets zeros in their places.
template <typename T>
__device__ __forceinline__ bool odd_pair(uint32_t v, uint32_t& clean) {
    constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    const bool lo = (v & kExp) == kExp, hi = (v >> 16 & kExp) == kExp;
    clean = (lo ? 0u : v & 0xFFFFu) | (hi ? 0u : v & 0xFFFF0000u);
    return lo || hi;
}
template <typename T>
__device__ __forceinline__ bool take_out_odd(uint4& v) {
    const bool a = odd_pair<T>(v.x, v.x), b = odd_pair<T>(v.y, v.y), c = odd_pair<T>(v.z, v.z), d = odd_pair<T>(v.w, v.w);
    return a || b || c || d;
}
// What was taken out of the products, for eight columns of a row that sees keys [lo, hi): added to its sums.  Keys [k0, k1) were this
// part's; those of [clear0, clear1) stayed in the products.
template <typename T>
__device__ __noinline__ void add_odd(const ChunkParams& p, int b, int h, int lo, int hi, int k0, int k1, int clear0, int clear1, int column, float (&acc)[8]) {
    for (int k = max(lo, k0); k < min(hi, k1); ++k) {
        if (k >= clear0 && k < clear1) {
            k = clear1 - 1;
            continue;
        }
        const int page = p.table[b * p.table_stride + (k >> p.page_shift)];
        if (page < 0 || page >= p.num_pages) continue;
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.vc.base) + page * p.vc.page_stride + h * p.vc.head_stride +
                                                        (k & ((1 << p.page_shift) - 1)) * p.vc.token_stride + column);
        float f[8];
        unpack8<T>(v, f);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!is_finite(f[i])) acc[i] += f[i];
    }
}

// ---------------------------------------------------------------------------------------------- rows
// Tiles of 16 rows: single and drafted tokens.  As in ivf_kv_attend's kernel of that name each of four warps takes pieces of 16 keys
// through a ring of its own and the warps meet at an item's end.  Bound by the keys' bytes: one token over 131,072 by 8 heads of 128 takes 93 us
// (537 MB, 5.8 TB/s with the joining of 37 parts to an item), 64 requests of 4,000 tokens 113 us (5.9 TB/s, 0.90 of a copy's rate), drafted tokens by 16 heads
// of 64 184 to 205 us (5.1 to 5.6 TB/s; three CTAs on an SM, with two 232).  A small call is a chain of waits: lengths, place, table, keys, warps,
// join: 10 us.
template <int DP>
struct ChunkRowsControl {
    ChunkPlan<kRowsThreads> plan;
    int odd;
};

template <typename T, int DP>
__global__ void __launch_bounds__(kRowsThreads, DP == 64 ? 3 : DP == 128 ? 2 : 1) kv_chunk_rows_kernel(const __grid_constant__ ChunkParams p) {
    using S = RowsShape<DP>;
    extern __shared__ __align__(128) uint8_t rows_smem[];
    __shared__ ChunkRowsControl<DP> c;
    pdl_trigger();  // (the kernel that joins the parts waits for this one's end by itself)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ChunkSpans spans;
    chunk_plan<kRowsThreads>(p, c.plan, spans);
    const ChunkCursor& at = c.plan.at;  // (in shared memory: the loop wants the registers)
    chunk_padding<T>(p, spans, kRowsThreads);
    const uint32_t smem0 = smem_u32(rows_smem);
    const uint32_t s_q = smem0 + S::kSmem - S::kQBytes;
    const uint32_t ring = smem0 + warp * (S::kStages * S::kStageBytes);
    const int ksteps = p.dim >> 4;
    const int n_heads = p.group * p.n_kv_heads;
    ChunkDesc tail = {0, 0, 0, 0};

    while (at.left > 0) {
        const ChunkItem it = chunk_item(p, at);
        const int h = it.hv / p.parts, g0 = it.hv % p.parts * p.part_heads;
        const int heads = min(p.part_heads, p.group - g0);
        const int head0 = h * p.group + g0;
        const int32_t* pages = p.table + at.b * p.table_stride;
        // At most 8 rows: as in ivf_kv_attend's kernel the product's other rows take the second parts of the weights, what their rounding to 16
        // bits leaves over (2^-16 or 2^-22 of themselves then)
        const bool split = it.tokens * p.part_heads <= 8;
        auto row_token = [&](int r) { return r / p.part_heads; };
        auto row_live = [&](int r) { return row_token(r) < it.tokens && r % p.part_heads < heads; };

        // keys that all rows see: those of the first and of the last token
        int all_lo, all_hi, skip;
        chunk_sees(p, at.r, it.pos, true, skip, all_hi);
        chunk_sees(p, at.r, it.pos + it.tokens - 1, true, all_lo, skip);
        const int piece0 = it.k0 >> 4, pieces = it.k1 > it.k0 ? ((it.k1 + 15) >> 4) - piece0 : 0;
        const int mine = pieces > warp ? (pieces - warp + kRowsWarps - 1) / kRowsWarps : 0;
        // the warp's j-th piece, the last ones first: where a bias falls with the distance the maximum is found at once
        auto key_of = [&](int j) { return (piece0 + warp + (mine - 1 - j) * kRowsWarps) << 4; };
        auto page_of = [&](int j) { return j < mine ? pages[key_of(j) >> p.page_shift] : -1; };
        auto checked = [&](int page) {
            if (page >= p.num_pages) {
                kv_report(p.status, kKvStatusBadId, KV_SITE_CHUNK);
                page = -1;
            }
            return page;
        };
        int page_now = page_of(lane), page_next = page_of(32 + lane);
        uint32_t there = 0;  // by stage: the piece has a page
        // the queries, behind the table's entries that are asked for above and in front of the first keys: one wait for all three
        if (tid == 0) c.odd = 0;
        for (int i = tid; i < 16 * (DP / 8); i += kRowsThreads) {
            const int r = i / (DP / 8), col = i % (DP / 8);
            const bool ok = row_live(r) && col * 8 < p.dim;
            cp_async16(rows_addr<DP>(s_q, r, col), ok ? static_cast<const T*>(p.q) + static_cast<int64_t>(it.token + row_token(r)) * p.q_stride[0] +
                                                            static_cast<int64_t>(head0 + r % p.part_heads) * p.q_stride[1] + col * 8 : static_cast<const T*>(p.q), ok);
        }
        cp_async_commit();
        page_now = checked(page_now);

        auto fetch = [&](int j, int stage) {
            if (j > 0 && (j & 31) == 0) {
                page_now = checked(page_next);
                page_next = page_of(j + 32 + lane);
            }
            const int64_t page = __shfl_sync(0xFFFFFFFFu, page_now, j & 31);
            there = page >= 0 ? there | 1u << stage : there & ~(1u << stage);
            if (page >= 0) {
                const int key0 = key_of(j);
                const int tok0 = key0 & ((1 << p.page_shift) - 1);
                const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + S::kPlaneBytes;
                const T* ks = static_cast<const T*>(p.kc.base) + page * p.kc.page_stride + h * p.kc.head_stride;
                const T* vs = static_cast<const T*>(p.vc.base) + page * p.vc.page_stride + h * p.vc.head_stride;
                constexpr int kLanes = DP / 8 < 32 ? DP / 8 : 32, kRowsAtOnce = 32 / kLanes;
                const int col = lane % kLanes, r0 = lane / kLanes;
                const T* kp = ks + (tok0 + r0) * p.kc.token_stride + col * 8;
                const T* vp = vs + (tok0 + r0) * p.vc.token_stride + col * 8;
                if (col * 8 < p.dim) {
#pragma unroll
                    for (int r = r0; r < 16; r += kRowsAtOnce) {
                        const bool ok = key0 + r >= it.k0 && key0 + r < it.k1;  // what no row sees is never read: it may hold anything
                        cp_async16(rows_addr<DP>(kb, r, col), ok ? kp : ks, ok);
                        cp_async16(rows_addr<DP>(vb, r, col), ok ? vp : vs, ok);
                        kp += kRowsAtOnce * p.kc.token_stride;
                        vp += kRowsAtOnce * p.vc.token_stride;
                    }
                }
            }
            cp_async_commit();
        };

#pragma unroll
        for (int s = 0; s < S::kStages - 1; ++s) fetch(s, s);
        cp_async_wait<S::kStages - 1>();  // the queries
        __syncthreads();
        uint32_t qf[DP / 16][4];
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) ldsm4(qf[k], rows_addr<DP>(s_q, lane & 15, 2 * k + (lane >> 4)));
        float o[DP / 8][4];
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        int lo[2], hi[2], pos[2];
        float slope[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = (lane >> 2) + r * 8;
            pos[r] = it.pos + row_token(row);
            chunk_sees(p, at.r, pos[r], row_live(row), lo[r], hi[r]);
            slope[r] = p.slopes && row_live(row) ? p.slopes[head0 + row % p.part_heads] * 1.4426950408889634f : 0.0f;
        }

        int stage = 0;
        for (int j = 0; j < mine; ++j) {
            cp_async_wait<S::kStages - 2>();
            __syncwarp();
            fetch(j + S::kStages - 1, stage == 0 ? S::kStages - 1 : stage - 1);
            const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + S::kPlaneBytes;
            const bool has = there >> stage & 1;
            if (++stage == S::kStages) stage = 0;
            if (!has) continue;
            const int key0 = key_of(j);
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
            if (it.tokens > 1 && (key0 < all_lo || key0 + 16 > all_hi)) {  // not all rows see all of it
                bool odd = false;
                for (int i = lane; i < 16 * (DP / 8); i += 32) {
                    const int r = i / (DP / 8), col = i % (DP / 8);
                    uint4* at_v = reinterpret_cast<uint4*>(rows_smem + (rows_addr<DP>(vb, r, col) - smem0));
                    uint4 v = *at_v;
                    if (col * 8 < p.dim && take_out_odd<T>(v)) {
                        *at_v = v;
                        odd = true;
                    }
                }
                if (odd) c.odd = 1;
                __syncwarp();
            }
            // row lane / 4 (and + 8): keys 2 (lane % 4), + 1, + 8, + 9
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = i >> 1, key = key0 + n * 8 + (lane & 3) * 2 + (i & 1);
                    float z = chunk_logit(p, sc[n][i]);
                    if (p.slopes) z = fmaf(-slope[r], fabsf(static_cast<float>(pos[r] - key)), z);
                    z = key >= lo[r] && key < hi[r] && key >= it.k0 && key < it.k1 ? z : -INFINITY;
                    sc[n][i] = z;
                    top[r] = fmaxf(top[r], z);
                }
            }
            float fix[2], base[2], add[2] = {0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = fmaxf(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], 1));
                top[r] = fmaxf(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], 2));
                const float mn = fmaxf(m[r], top[r]);
                base[r] = mn == -INFINITY ? 0.0f : mn;
                fix[r] = exp2_fast(m[r] - base[r]);
                m[r] = mn;
            }
            uint32_t pf[4];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int r = 1; r >= 0; --r) {
                    const float w0 = exp2_fast(sc[n][2 * r] - base[r]), w1 = exp2_fast(sc[n][2 * r + 1] - base[r]);
                    add[r] += w0 + w1;
                    pf[2 * n + r] = Pair16<T>::pack(w0, w1);
                    if (r == 0 && split) {
                        const float2 first = Pair16<T>::unpack(pf[2 * n]);
                        pf[2 * n + 1] = Pair16<T>::pack(w0 - first.x, w1 - first.y);
                    }
                }
            }
            if (split) fix[1] = fix[0];
#pragma unroll
            for (int r = 0; r < 2; ++r) l[r] = l[r] * fix[r] + add[r];
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
        if (split) {
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
        const bool whole = it.first && it.last;
        float* slot = p.slots + static_cast<int64_t>(2 * blockIdx.x + (it.first ? 1 : 0)) * p.rows * (p.dim + 2);
        for (int i = tid; i < 16 * (DP / 8); i += kRowsThreads) {
            const int r = i / (DP / 8), col = i % (DP / 8);
            if (col * 8 >= p.dim || !row_live(r)) continue;
            float best = -INFINITY, sum = 0.0f, acc[8] = {};
#pragma unroll
            for (int k = 0; k < kRowsWarps; ++k) best = fmaxf(best, s_o[(k * 16 + r) * kRow + DP]);
            const float base = best == -INFINITY ? 0.0f : best;
#pragma unroll
            for (int k = 0; k < kRowsWarps; ++k) {
                const float* src = s_o + (k * 16 + r) * kRow;
                const float w = exp2_fast(src[DP] - base);
                sum += w * src[DP + 1];
#pragma unroll
                for (int x = 0; x < 8; ++x) acc[x] += w * src[col * 8 + x];
            }
            if (c.odd) {
                int from, to;
                chunk_sees(p, at.r, it.pos + row_token(r), true, from, to);
                add_odd<T>(p, at.b, h, from, to, it.k0, it.k1, (all_lo + 15) & ~15, all_hi & ~15, col * 8, acc);
            }
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;  // nothing seen: zeros
#pragma unroll
                for (int x = 0; x < 8; ++x) acc[x] *= inv;
                const int64_t t = it.token + row_token(r);
                const int head = head0 + r % p.part_heads;
                *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + t * p.out_stride[0] + head * p.out_stride[1] + col * 8) = pack8<T>(acc);
                if (col == 0 && p.lse) p.lse[t * n_heads + head] = sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.69314718055994531f;
            } else {
                float* dst = slot + r * p.dim + col * 8;
                *reinterpret_cast<float4*>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                *reinterpret_cast<float4*>(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (col == 0) {
                    slot[p.rows * p.dim + r] = best;
                    slot[p.rows * (p.dim + 1) + r] = sum;
                }
            }
        }
        if (it.first && !it.last && tid == 0)
            tail = ChunkDesc{chunk_parts(spans, blockIdx.x, it.rest), it.token, it.tokens, it.hv};
        __syncthreads();  // the next item's queries and ring lie over this one's
        if (tid == 0) chunk_next(p, c.plan.at);
        __syncthreads();
    }
    if (tid == 0) p.desc[blockIdx.x] = tail;
}

// Joins the parts of the items that spans have cut: blockIdx.x is the CTA that the item began in.  WARPS warps to a row, each with its
// share of the parts, eight at a time: sums, maxima and totals of those are asked for together.  (A thread to four columns that went over the parts twice by
// itself took 30 us for 37 parts, a third of the attention; one warp to a row 10 us, four 4 us.)
constexpr int kJoinThreads = 128;
template <typename T, int WARPS>
__global__ void __launch_bounds__(kJoinThreads) kv_chunk_join_kernel(const ChunkParams p) {
    constexpr int kRows = kJoinThreads / 32 / WARPS, kAtOnce = 8;
    __shared__ float4 s_acc[WARPS > 1 ? WARPS : 1][64];
    __shared__ float2 s_ml[WARPS];
    pdl_wait();
    const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = warp % WARPS;
    const ChunkDesc d = p.desc[c];
    const int r = blockIdx.y * kRows + warp / WARPS;
    if (d.parts == 0 || r >= d.tokens * p.part_heads) return;  // (with several warps to a row the whole CTA)
    const int h = d.hv / p.parts, g0 = d.hv % p.parts * p.part_heads;
    if (r % p.part_heads >= min(p.part_heads, p.group - g0)) return;
    const int n_heads = p.group * p.n_kv_heads, quads = p.dim / 4;
    const int64_t step = static_cast<int64_t>(p.rows) * (p.dim + 2);
    auto part = [&](int k) { return p.slots + (k == 0 ? 2 * c + 1 : 2 * (c + k)) * step; };
    float m = -INFINITY, sum = 0.0f;
    float4 acc[2] = {};
    for (int k0 = share; k0 < d.parts; k0 += WARPS * kAtOnce) {
        float4 v[kAtOnce][2];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at = k0 + k * WARPS;
                v[k][i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (at < d.parts && lane + 32 * i < quads) v[k][i] = *reinterpret_cast<const float4*>(part(at) + static_cast<int64_t>(r) * p.dim + (lane + 32 * i) * 4);
            }
        float mine = -INFINITY, total = 0.0f;  // of part k0 + lane * WARPS
        if (lane < kAtOnce && k0 + lane * WARPS < d.parts) {
            const float* src = part(k0 + lane * WARPS) + p.rows * p.dim + r;
            mine = src[0];
            total = src[p.rows];
        }
        float top = mine;
#pragma unroll
        for (int o = kAtOnce / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        top = fmaxf(m, __shfl_sync(0xFFFFFFFFu, top, 0));
        const float base = top == -INFINITY ? 0.0f : top, fix = exp2_fast(m - base), w = exp2_fast(mine - base);
        m = top;
        sum = sum * fix + w * total;
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[i].x *= fix, acc[i].y *= fix, acc[i].z *= fix, acc[i].w *= fix;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float f = __shfl_sync(0xFFFFFFFFu, w, k);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                acc[i].x += f * v[k][i].x, acc[i].y += f * v[k][i].y, acc[i].z += f * v[k][i].z, acc[i].w += f * v[k][i].w;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (WARPS > 1) {
        if (lane == 0) s_ml[share] = make_float2(m, sum);
#pragma unroll
        for (int i = 0; i < 2; ++i) s_acc[share][lane + 32 * i] = acc[i];
        __syncthreads();
        if (share > 0) return;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_ml[w].x);
        m = top;
        sum = 0.0f;
        acc[0] = acc[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = exp2_fast(s_ml[w].x - (top == -INFINITY ? 0.0f : top));
            sum += f * s_ml[w].y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 v = s_acc[w][lane + 32 * i];
                acc[i].x += f * v.x, acc[i].y += f * v.y, acc[i].z += f * v.z, acc[i].w += f * v.w;
            }
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t t = d.token + r / p.part_heads;
    const int head = h * p.group + g0 + r % p.part_heads;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (lane + 32 * i >= quads) continue;
        const uint2 v = make_uint2(Pair16<T>::pack(acc[i].x * inv, acc[i].y * inv), Pair16<T>::pack(acc[i].z * inv, acc[i].w * inv));
        *reinterpret_cast<uint2*>(static_cast<T*>(p.out) + t * p.out_stride[0] + head * p.out_stride[1] + (lane + 32 * i) * 4) = v;
    }
    if (lane == 0 && p.lse) p.lse[t * n_heads + head] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.69314718055994531f;
}

}  // namespace ivf
