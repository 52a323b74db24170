// Attention for a tree of drafted tokens over the paged cache.
//
// Token i of request r (its node i, cached at position prior + i) attends the request's whole context, keys 0 .. prior - 1, and the
// tree tokens that its mask row names, bit j for node j:
//     out[i, h] = sum_k softmax_k(q[i, h] . K[k, g] / sqrt(d)) V[k, g],   lse[i, h] = log sum_k exp(q . K[k, g] / sqrt(d)).
// All nodes of a tree read the same context, so with few nodes the kernel is bound by the bytes of K and V (4 d nodes G
// operations for 4 d bytes of a token and kv head: 148 SMs' tensor cores and HBM meet at some 250 (node, head) rows).  It streams
// every K and V tile once and runs both products on the 5th-generation tensor cores, whose 128 rows are the (node, head) pairs that
// share a kv head.
//
// Work: an item is one (request, kv head, group of up to 256 rows).  Its keys are tiles of 128, and all items' tiles, with
// some more an item for its start and end, make one line that is cut into equal shares, a CTA each, wherever the cuts fall
// (stream-K); few and short items are a CTA each.  So one request on a long context, or a ragged batch, fills all SMs, and a CTA has at most two pieces of an item:
// partial rows go to fixed places of the workspace and tree_merge_kernel joins them in the order of their keys.  The shares
// follow from the batch's lengths, which travel as kernel parameters: there is no work list to upload and nothing to
// initialise.
//
//   warps 0-3, 4-7  softmax of streams 0 and 1; thread t owns row t (TMEM lane t).  A step is 64 keys of 128 rows.  With two q tiles each
//                   stream has one and takes both halves of every key tile; with one q tile the streams take a half of every key
//                   tile each, with a running maximum, sum and accumulator of their own, joined when the item ends.  Results go out
//                   through the Q tile's place, so that global stores cover whole sectors of a row.
//   warp 8          K and V tiles: pool blocks gathered by tensor map into one ring, in the order of use K0 K1 V0 K2 V1 ...
//   warps 9, 10     MMA issue of streams 0 and 1: S = Q K^T (operands in shared memory) two steps ahead, into two buffers in turn,
//                   O += P V (P as bf16 in the columns that S had), whichever's operands are there first
//   warp 11         Q tiles; and V tiles that hold tree tokens or the sequence's end: rows behind the end become zero, and rows with
//                   infinities or NaN (FP8: or a scale over 255) too, because 0 * inf would reach nodes that do not see them; their weights are added by
//                   the rows that do when the item ends.
//
// FP8 cache (E4M3 codes, a scale per token and kv head): half the bytes a key, so the conversion of the codes is what costs.  K's are
// multiplied as they lie in the page: q 2^e (e of its row, the largest element in (224, 448]) is the sum of two E4M3 numbers, exactly
// where an element has at least 2^-2 and within 2^-10 elsewhere, so S = Q1 K^T + Q2 K^T on the 8-bit tensor pipe, at the price
// of one 16-bit product.  K's scales multiply the scores in fp32.  V becomes f16, code times half the scale (11 of at most 12 significant
// bits; half, so that scales up to 255 stay in range; as code / 256, exactly, times 128 scales, so that a scale's 8 bits lie in f16's normal range
// down to 2^-21), and the weights are rounded to f16.  Warp 11 converts Q, warps 12-15 V,
// in a ring of its own behind the copies'.
//
// Measured, with the merge kernel (32 q and 8 kv heads; floors, all of bytes, at 6.56 TB/s), in calls one after the other for 15 ms / for more than a second, when
// 128 dimensions run at the power cap: 32 trees of 11-32 nodes on 512-4096 tokens, 352 MB, 70 / 79 us (5.0 / 4.5 TB/s; floor 54; 1.96 / 1.55 GHz); FP8, 64 of 7-32,
// 352 MB, 152 / 161 us (floor 54); 8 heads of 64 without grouping, 24 of 20-61 on 300-5000, 128 MB, 43 us (floor 20); 64 of 48-64 on 4096-12288, 2.48 GB,
// 640 / 746 us (floor 378; operations 327; 1.45 GHz); one of 8 nodes on 700, 13 us.  Within an item bf16 of 128 dimensions runs at HBM's rate.  The others are
// bound by the chain of a step: 1850 cycles (FP8 3200) for 64 keys of 128 rows, 1100 of them on exponentials, two warps a scheduler, the rest tensor-memory loads
// and stores, fences and barriers.  (With at most 64 rows both streams' rows lie in the same 64 lanes, so two of the four schedulers have all of them; and the FP8
// form's 16 warps have 128 registers each, of which the softmax spills 29 words.)  An item's start and end cost some 8500 cycles (64 dimensions 5400, FP8 15000),
// in which the loads get no further than the ring.
//
// Roundings: scores, maxima, sums and accumulators are fp32.  The weights that multiply V are rounded to V's type, bf16 or f16, because both operands of one
// product have the same; the sums are of the unrounded ones.  An output's largest error against 64 bits, relative to its row's largest element, is 0.0023 (FP8
// cache 0.0017), of which the result's own rounding to bf16 makes 0.0017.
//
// Every wait is bounded; on expiry the CTA flags the pool and drains.
#include <cuda_fp16.h>

#include "tcgen05.cuh"

namespace ps {

namespace {

constexpr int kLoadWarp = 8, kMmaWarp = 9, kQWarp = 11, kConvertWarp = 12;  // (MMA: 9 and 10)
constexpr int kTileKeys = 128, kRows = 128;
constexpr int kGroupRows = 2 * kRows;      // rows of an item
constexpr int kMaxNodes = 256;
constexpr float kRescaleThreshold = 8.f;   // log2 units

template <int D, bool FP8>
struct Cfg {
    static constexpr int kThreads = FP8 ? 512 : 384;         // (of three warps a scheduler each may have 168 registers)
    // What an item's start and end cost, in key tiles.  Measured with 1 / 3 / 4 / 6 / 9: 32 trees of 11-32 nodes on 500-4000 tokens, 128 dimensions 76.0 /
    // 71.7 / 71.7 / 71.2 / 73.4 us; 24 of 20-61 on 300-5000, 64 dimensions 48.6 / 44.0 / 44.7 / 46.0 / 47.5; FP8, 64 of 7-32 on 500-4000 183 / 167 / 160 / 152 / 155.
    static constexpr int kItemUnits = FP8 ? 7 : D == 128 ? 5 : 3;
    // Few and short items stay whole, a CTA each, where cutting would save fewer steps than joining the pieces costs; and a share has at least kLeastShare units.
    // Measured, one tree of 8 nodes on 250 / 500 / 1000 / 1500 / 3000 tokens, whole and cut (32 q and 8 kv heads of 128): 7.7 / 9.8 / 13.6 / 17.4 /
    // 29.4 and 11.4 / 12.6 / 13.9 / 14.3 / 17.4 us; FP8 17.6 / 20.2 / 26.1 / 32.3 / 50.9 and 18.4 / 23.0 / 24.0 / 24.8 / 27.9; 8 heads of 64 without grouping 6.6 /
    // 8.5 / 12.1 / 15.7 / 26.9 and 11.2 / 13.5 / 14.3 / 15.5 / 19.3; of 64 nodes, two q tiles of 128, 13.8 / 17.9 / 25.4 / 32.8 / 54.7 and 18.1 / 19.9 / 21.2 / 21.9 / 26.2.
    // (Shares of two units: 19.7 instead of 17.4 at 3000, 64 dimensions 25.8, of three 21.0, instead of 19.3.)
    static constexpr int kMergeSteps = FP8 ? 3 : D == 128 ? 5 : 8, kLeastShare = D == 128 ? 3 : 4;
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = kTileKeys * 128;
    static constexpr int kTileBytes = kHalves * kHalfBytes;  // a tile of Q, K or V in 16 bits
    static constexpr int kCodeBytes = kTileKeys * D;         // of codes
    // K and V tiles in flight: one ring in the order of their use; FP8: rings of K (codes), V (codes) and V (f16)
    static constexpr int kSlots = FP8 ? 3 : D == 128 ? 5 : 10;
    static constexpr int kRaw = FP8 ? 2 : kSlots / 2 + 2;    // V tiles on their way through warp 11 (more than the ring holds) or 12-15
    static constexpr int kConv = FP8 ? 2 : 0;
    // Tiles whose rows taken out of V are kept: an item's last three, and as many as are begun before the slower stream has written it out.
    // (One stream may be one item ahead of the other, PV then stops, and the ring holds kSlots / 2 + 1 V tiles more.)
    static constexpr int kFlagTiles = !FP8 && D == 64 ? 16 : 8;
    // Tiles whose scales are kept: while the softmax works on one, K is loaded for at most four behind it.
    static constexpr int kScaleTiles = 6, kScaleBytes = kTileKeys / kPage * 128;
    static constexpr int kOffQ = 0;                          // two tiles
    static constexpr int kOffKV = 2 * kTileBytes;
    static constexpr int kOffRaw = kOffKV + kSlots * (FP8 ? kCodeBytes : kTileBytes);
    static constexpr int kOffConv = kOffRaw + (FP8 ? kRaw * kCodeBytes : 0);
    static constexpr int kOffScale = kOffConv + kConv * kTileBytes;
    static constexpr int kOffQScale = kOffScale + (FP8 ? kScaleTiles * kScaleBytes : 0);
    static constexpr int kOffRawScale = kOffQScale + (FP8 ? 2 * kRows * 4 : 0);  // with V's codes
    static constexpr int kOffPieces = kOffRawScale + (FP8 ? kRaw * kScaleBytes : 0);  // [softmax warp][2]
    static constexpr int kOffBar = kOffPieces + (FP8 ? 8 * 2 * 48 : 0);
    // barrier block
    static constexpr int full = 0, empty = full + 8 * kSlots, raw = empty + 8 * kSlots, raw_empty = raw + 8 * kRaw, conv_full = raw_empty + (FP8 ? 8 * kRaw : 0),
                         conv_empty = conv_full + 8 * kConv, q_ready = conv_empty + 8 * kConv;
    // [stream][its step & 1]: scores there, weights there, product with V done
    static constexpr int s_full = q_ready + (FP8 ? 16 : 0), p_ready = s_full + 32, pv_done = p_ready + 32;
    static constexpr int q_full = pv_done + 32, q_empty = q_full + 16, ex_full = q_empty + 16, ex_free = ex_full + 8, mma_drained = ex_free + 8, n_bars = (mma_drained + 8) / 8;
    static constexpr int tmem_slot = 8 * n_bars, abort_slot = tmem_slot + 4, limit_slot = abort_slot + 4, armed = limit_slot + 4;  // slots, Q tiles, raw V tiles
    static constexpr int flagged = armed + 4 * (kSlots + 2 + kRaw);           // [tile % kFlagTiles][4]: rows taken out of V
    static constexpr int exchange = (flagged + kFlagTiles * 16 + 7) / 8 * 8;  // [stream][row] (maximum, sum of the weights)
    static constexpr int bar_bytes = exchange + 2 * kRows * 8;
    static constexpr int kSmemBytes = kOffBar + bar_bytes;
    static_assert(kSmemBytes <= 232448, "shared memory");
};
// Where tile n of K, and of V as the products read it, lies: its barriers, their phase, its place.  16 bits: one ring in the order
// K0 K1 V0 K2 V1 ...
struct Slot {
    uint32_t full, empty, par, at;
};
template <class C, bool FP8>
__device__ __forceinline__ Slot ring_slot(uint32_t e) {
    const uint32_t s = e % C::kSlots;
    return Slot{C::full + 8 * s, C::empty + 8 * s, (e / C::kSlots) & 1, C::kOffKV + s * (FP8 ? C::kCodeBytes : C::kTileBytes)};
}
template <class C, bool FP8>
__device__ __forceinline__ Slot k_slot(uint32_t n) { return ring_slot<C, FP8>(FP8 ? n : n == 0 ? 0 : 2 * n - 1); }
template <class C, bool FP8>
__device__ __forceinline__ Slot v_slot(uint32_t n) {
    if (FP8) return Slot{C::conv_full + 8 * (n & 1), C::conv_empty + 8 * (n & 1), (n >> 1) & 1, C::kOffConv + (n & 1) * C::kTileBytes};
    return ring_slot<C, FP8>(2 * n + 2);
}

// the lengths of a batch
template <int N>
struct TreeRows {
    int32_t q_start[N + 1], unit_start[N + 1], prior[N];
};
constexpr int kTreeRowsMax = 2600;  // 31 KB of kernel parameters

struct TreeParams {
    const __nv_bfloat16* q;
    const int32_t* block_table;
    const uint32_t* mask;   // 2 * mask_words 32-bit words a token
    const char* pool;
    __nv_bfloat16* out;
    float* lse;
    float2* part_ml;        // [2 CTAs][256 rows]: maximum (log2 units), sum of the weights
    float* part_o;
    int* flag;
    int64_t num_pages;
    uint32_t wait_limit_ns;
    int32_t max_pages, mask_words, n, Hq, Hkv, G;
    int32_t item_units;     // of an item beside its tiles; negative: -item_units in all, of every item, and a share is an item
    int32_t share, longer;  // a share's units; the first `longer` shares have one more
};

// pieces of items in a CTA's share of the line
struct Piece {
    int r, head, q_tok, n_tok, nodes, prior, kv_len;  // (the group's tokens)
    int tile0, tile1, tiles;
    __device__ __forceinline__ int n_x(int G) const { return n_tok * G > kRows ? 2 : 1; }
    __device__ __forceinline__ bool whole() const { return tile0 == 0 && tile1 == tiles; }
    // first tile with tree tokens or the sequence's end in it
    __device__ __forceinline__ int tree_tile() const { return prior / kTileKeys; }
};
__device__ __forceinline__ int share_begin(const TreeParams& p, int c) { return c * p.share + min(c, p.longer); }

// (What is common to the roles is short: their code shares the SM's instruction cache, which all of it together overflows.)
template <class Rows>
struct PieceIter {
    const Rows& rows;
    const TreeParams& p;
    const int G, Hkv;  // (kept: read from the parameters at each use, FP8 takes 167 us instead of 151)
    int left, r, head, group, w0;  // units left of the share; where it goes on: request, kv head, group, units into the item
    __device__ __forceinline__ int tiles() const { return (rows.prior[r] + rows.q_start[r + 1] - rows.q_start[r] + kTileKeys - 1) / kTileKeys; }
    __device__ __forceinline__ int beside(int tiles) const { return p.item_units >= 0 ? p.item_units : -p.item_units - tiles; }
    __device__ __forceinline__ int groups(int nodes) const {
        const int shift = 31 - __clz(kGroupRows / G);  // (G is a power of two)
        return (nodes + (1 << shift) - 1) >> shift;
    }
    __device__ __forceinline__ PieceIter(const Rows& rows_, const TreeParams& p_, int u, int end) : rows(rows_), p(p_), G(p_.G), Hkv(p_.Hkv), left(end - u) {
        int lo = 0, hi = p.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (rows.unit_start[mid] <= u) lo = mid; else hi = mid - 1;
        }
        r = lo;
        const int per = tiles() + beside(tiles()), o = u - rows.unit_start[r], item = o / per, gr = groups(rows.q_start[r + 1] - rows.q_start[r]);
        w0 = o - item * per;
        head = item / gr;
        group = item - head * gr;
    }
    __device__ __forceinline__ bool next(Piece& x) {
        while (left > 0) {
            x.r = r;
            x.prior = rows.prior[r];
            x.q_tok = rows.q_start[r];
            x.nodes = rows.q_start[r + 1] - x.q_tok;
            x.kv_len = x.prior + x.nodes;
            x.tiles = tiles();
            x.head = head;
            const int extra = beside(x.tiles);
            x.tile0 = max(0, w0 - extra);
            x.tile1 = max(0, min(x.tiles + extra, w0 + left) - extra);
            left -= x.tiles + extra - w0;
            w0 = 0;
            const int tok0 = group * (kGroupRows / G);
            x.n_tok = min(kGroupRows / G, x.nodes - tok0);
            x.q_tok += tok0;
            if (tok0 + x.n_tok == x.nodes) {
                group = 0;
                if (++head == Hkv) head = 0, ++r;
            } else {
                ++group;
            }
            if (x.tile1 > x.tile0) return true;
        }
        return false;
    }
};

// Word w of a row's mask without the bits behind the last node
__device__ __forceinline__ uint32_t up_to(uint32_t x, int w, int nodes) {
    const int left = nodes - 32 * w;
    return left >= 32 ? x : left <= 0 ? 0u : x & ((1u << left) - 1u);
}
__device__ __forceinline__ uint32_t mask_word(const uint32_t* row, int w, int nodes) { return 32 * w < nodes ? up_to(__ldg(row + w), w, nodes) : 0u; }
// 32 bits of a row's mask from node `at` on; nodes before the tree are context and visible, behind its end there is nothing (w0, w1: the first two
// words as they stand)
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* row, uint32_t w0, uint32_t w1, int at, int nodes) {
    if (at <= -32) return 0xffffffffu;
    if (at < 0) return ((1u << -at) - 1u) | up_to(w0, 0, nodes) << -at;
    auto word = [&](int w) { return w < 2 ? up_to(w == 0 ? w0 : w1, w, nodes) : mask_word(row, w, nodes); };
    const int w = at >> 5, s = at & 31;
    const uint32_t lo = word(w);
    return s == 0 ? lo : __funnelshift_r(lo, word(w + 1), s);
}

// A warp's 32 rows of BYTES each, a row a lane, through its stage, so that stores cover BYTES of a row: dst(row) is where a row goes, or null.
// (Units of 16 bytes change places row by row against bank conflicts.)
template <int BYTES, class F>
__device__ __forceinline__ void store_rows(char* stage, int lane, const uint32_t* v, const F& dst) {
    constexpr int U = BYTES / 16;  // units of a row
    auto place = [&](int row, int u) { return stage + row * BYTES + ((u ^ (U == 8 ? row & 7 : row >> 1 & 3)) << 4); };
#pragma unroll
    for (int u = 0; u < U; ++u) *reinterpret_cast<uint4*>(place(lane, u)) = make_uint4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
    __syncwarp();
    // (all loads first: the compiler cannot tell that the stores go elsewhere)
    uint4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = *reinterpret_cast<const uint4*>(place(k * (32 / U) + lane / U, lane % U));
#pragma unroll
    for (int k = 0; k < U; ++k) {
        char* const to = dst(k * (32 / U) + lane / U);
        if (to) *reinterpret_cast<uint4*>(to + 16 * (lane % U)) = x[k];
    }
    __syncwarp();
}

// Element e of the K (kv = 0) or V vector of a slot of a page's block
template <int D, bool FP8>
__device__ __forceinline__ float pool_value(const char* blk, int kv, int slot, int e) {
    if (FP8) {
        const uint8_t code = *reinterpret_cast<const uint8_t*>(blk + kv * kPage * D + slot * D + (((e >> 4) ^ (slot & 7)) << 4) + (e & 15));
        uint32_t two;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"((uint16_t)code));
        return __half2float(__ushort_as_half((unsigned short)two)) * reinterpret_cast<const float*>(blk + 2 * kPage * D)[kv * kPage + slot];
    }
    return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(blk + kv * block_bytes(D) + unit_offset(slot, e) + 2 * (e & 7)));
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ bool any_not_finite(const uint4& x) {
    auto bad = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
    return bad(x.x) || bad(x.y) || bad(x.z) || bad(x.w);
}

template <int D, bool FP8, class Rows>
__global__ void __launch_bounds__(Cfg<D, FP8>::kThreads, 1) tree_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap q_map,
                                                                         const __grid_constant__ CUtensorMap pool_map, const __grid_constant__ CUtensorMap scale_map,
                                                                         const __grid_constant__ Rows rows) {
    using C = Cfg<D, FP8>;
    extern __shared__ __align__(1024) char smem[];  // (the 128-byte swizzle wants tiles on 1024 bytes)
    const uint32_t sbase = smem_u32(smem), bars = sbase + C::kOffBar;
    volatile int* const s_abort = reinterpret_cast<volatile int*>(smem + C::kOffBar + C::abort_slot);
    volatile int* const s_armed = reinterpret_cast<volatile int*>(smem + C::kOffBar + C::armed);  // (-1: never; read only after an abort)
    volatile uint32_t* const s_flagged = reinterpret_cast<volatile uint32_t*>(smem + C::kOffBar + C::flagged);
    float2* const exchange = reinterpret_cast<float2*>(smem + C::kOffBar + C::exchange);
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kSlots; ++s) {
            mbar_init(bars + C::full + 8 * s, 1);
            mbar_init(bars + C::empty + 8 * s, 2);
        }
        for (int s = 0; s < C::kRaw; ++s) mbar_init(bars + C::raw + 8 * s, 1);
        if (FP8) {
            for (int s = 0; s < C::kRaw; ++s) mbar_init(bars + C::raw_empty + 8 * s, 4);
            for (int s = 0; s < 2; ++s) {
                mbar_init(bars + C::conv_full + 8 * s, 4);
                mbar_init(bars + C::conv_empty + 8 * s, 2);
                mbar_init(bars + C::q_ready + 8 * s, 1);
            }
        }
        for (int k = 0; k < 4; ++k) {
            mbar_init(bars + C::s_full + 8 * k, 1);
            mbar_init(bars + C::p_ready + 8 * k, 4);
            mbar_init(bars + C::pv_done + 8 * k, 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(bars + C::q_full + 8 * x, 1);
            mbar_init(bars + C::q_empty + 8 * x, 8);
        }
        mbar_init(bars + C::ex_full, 8);
        mbar_init(bars + C::ex_free, 8);
        mbar_init(bars + C::mma_drained, 2);
        mbar_fence_init();
        s_abort[0] = 0;
        s_abort[1] = (int)p.wait_limit_ns;
        for (int s = 0; s < C::kSlots + 2 + C::kRaw; ++s) s_armed[s] = -1;
    }
    if (warp == 0) {
        tmem_alloc(bars + C::tmem_slot, 512);
        tmem_relinquish();
    }
    pdl_trigger();
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + C::kOffBar + C::tmem_slot);
    auto wait_all = [](uint32_t bar, uint32_t parity, volatile int* abort_flag) { return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_flag)); };

    // f() until it is not 0, polled for at most about the wait limit; 0 then.  (Sleep between polls only where the answer is not urgent: a sleep of
    // 20 ns puts the MMA warps some 700 cycles behind.)
    auto poll = [&](uint32_t sleep_ns, auto f) -> int {
        uint32_t t0 = 0;
        for (uint32_t i = 1;; ++i) {
            const int got = f();
            if (got) return got;
            if (sleep_ns) __nanosleep(sleep_ns);
            const uint32_t limit_ns = (uint32_t)s_abort[1];
            if ((i & 15) == 0 || limit_ns == 0) {
                const uint32_t now = global_timer_lo() | 1u;
                if (t0 == 0) t0 = now;
                if (__any_sync(0xffffffffu, *s_abort || limit_ns == 0 || now - t0 > limit_ns)) break;
            }
        }
        *s_abort = 1;
        return 0;
    };
    auto complete = [](uint32_t bar, uint32_t par) { return (bool)__all_sync(0xffffffffu, mbar_test_wait(bar, par)); };
    // which of two phases is complete first: 1, 2, or 0
    auto either = [&](uint32_t sleep_ns, uint32_t bar1, uint32_t par1, uint32_t bar2, uint32_t par2) {
        return poll(sleep_ns, [&]() { return complete(bar1, par1) ? 1 : complete(bar2, par2) ? 2 : 0; });
    };

    constexpr uint32_t kColO = 256;
    PieceIter<Rows> iter(rows, p, share_begin(p, blockIdx.x), share_begin(p, blockIdx.x + 1));
    Piece it;
    const int tile_tok = kRows / p.G, g_shift = 31 - __clz(p.G);

    if (warp < 8) {
        // ====================================================================
        // softmax
        // ====================================================================
        const int x = warp >> 2, t = threadIdx.x & 127;
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        constexpr float kScaleLog2 = scale_log2(D);
        uint32_t steps = 0, q_tiles = 0, tiles = 0, n_ex = 0;  // of this stream; q and key tiles of the items before; exchanges
        bool ok = true, must_wait_free = false;
        // FP8: the pieces wait in shared memory, for want of registers beside a step's scores
        Piece ahead;
        bool more = iter.next(ahead);
        uint32_t n_piece = 0;
        int* const kept = reinterpret_cast<int*>(smem + C::kOffPieces + warp * 96);
        auto keep = [&](uint32_t n, const Piece& a) {
            if (FP8 && lane == 0) {
                int* const to = kept + (n & 1) * 12;
                to[0] = a.r, to[1] = a.head, to[2] = a.q_tok, to[3] = a.n_tok, to[4] = a.nodes, to[5] = a.prior, to[6] = a.kv_len, to[7] = a.tile0, to[8] = a.tile1, to[9] = a.tiles;
            }
            __syncwarp();
        };
        auto kept_piece = [&](uint32_t n) {
            const volatile int* const from = kept + (n & 1) * 12;
            Piece a;
            a.r = from[0], a.head = from[1], a.q_tok = from[2], a.n_tok = from[3], a.nodes = from[4], a.prior = from[5], a.kv_len = from[6], a.tile0 = from[7], a.tile1 = from[8], a.tiles = from[9];
            return a;
        };
        if (more) keep(0, ahead);
        while (ok && more) {
            if (FP8) it = kept_piece(n_piece);
            else it = ahead;
            const int n_x = it.n_x(p.G), n_tiles = it.tile1 - it.tile0;
            const int q_tile = n_x == 2 ? x : 0;
            const int row_tok = q_tile * tile_tok + (t >> g_shift);  // token of this row within the item
            const bool valid = row_tok < it.n_tok;
            const bool warp_valid = q_tile * tile_tok + ((t & ~31) >> g_shift) < it.n_tok;  // any row of this warp
            const int64_t token = it.q_tok + row_tok;
            const uint32_t* const mask_row = p.mask + token * 2 * p.mask_words;
            // (the first 64 nodes' are wanted soon enough to ask for them now)
            const uint32_t mask0 = valid ? __ldg(mask_row) : 0u, mask1 = valid ? __ldg(mask_row + 1) : 0u;
            float row_scale = kScaleLog2;            // of the scores, to log2 units
            float m = -INFINITY, l = 0.f;            // running maximum (log2 units), sum of the weights
            for (int k = 0; k < n_tiles * n_x; ++k) {
                const int tile = n_x == 2 ? k >> 1 : k, half = n_x == 2 ? k & 1 : x;
                const uint32_t buf = steps & 1;
                ok = wait_all(bars + C::s_full + 16 * x + 8 * buf, (steps >> 1) & 1, s_abort);
                if (!ok) break;
                tc_fence_after();
                if (FP8 && k == 0) row_scale = kScaleLog2 * *reinterpret_cast<const float*>(smem + C::kOffQScale + (((q_tiles + q_tile) & 1) * kRows + t) * 4);
                if (warp_valid) {
                    const uint32_t s_addr = tmem + lane_addr + x * 128 + buf * 64;
                    const int key0 = (it.tile0 + tile) * kTileKeys + half * 64;
                    const bool masked = key0 + 64 > it.prior;
                    const uint64_t sc2 = pack2(row_scale, row_scale);
                    // FP8: times the keys' scales, 16 of K and 16 of V a page
                    const float* const scales = reinterpret_cast<const float*>(smem + C::kOffScale + (tiles + tile) % C::kScaleTiles * C::kScaleBytes) + half * 128;
                    auto scaled = [&](uint32_t (&sv)[32], int q) {
                        if constexpr (FP8) {
#pragma unroll
                            for (int c = 0; c < 32; c += 4) {
                                const float4 ks = *reinterpret_cast<const float4*>(scales + (q * 2 + (c >> 4)) * 32 + (c & 15));
                                float a0, a1, a2, a3;
                                unpack2(mul2(pack2(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), pack2(ks.x, ks.y)), a0, a1);
                                unpack2(mul2(pack2(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), pack2(ks.z, ks.w)), a2, a3);
                                sv[c] = __float_as_uint(a0), sv[c + 1] = __float_as_uint(a1), sv[c + 2] = __float_as_uint(a2), sv[c + 3] = __float_as_uint(a3);
                            }
                        }
                    };
                    bool done = false;
                    if (!masked && k > 0) {
                        // Nearly every step leaves the running maximum as it is: weights and maximum at once, and again where one lies above.
                        // (The second half's scores come under the first's exponentials.)
                        uint32_t sa[32], sb[32], packed[32];
                        tmem_ld32(s_addr, sa);
                        tmem_wait_ld();
                        tmem_ld32(s_addr + 32, sb);
                        const float m_sub = m == -INFINITY ? 0.f : m;
                        const uint64_t nm2 = pack2(-m_sub, -m_sub);
                        uint64_t ls0 = 0ull, ls1 = 0ull;
                        float mx0 = -INFINITY, mx1 = -INFINITY;
                        auto weights = [&](uint32_t (&sv)[32], int q) {
                            scaled(sv, q);
#pragma unroll
                            for (int c = 0; c < 32; c += 2) {
                                const float s0 = __uint_as_float(sv[c]), s1 = __uint_as_float(sv[c + 1]);
                                float e0, e1;
                                unpack2(fma2(pack2(s0, s1), sc2, nm2), e0, e1);
                                e0 = fast_exp2(e0), e1 = fast_exp2(e1);
                                if (c & 2) {
                                    mx1 = max3(mx1, s0, s1);
                                    ls1 = add2(ls1, pack2(e0, e1));
                                } else {
                                    mx0 = max3(mx0, s0, s1);
                                    ls0 = add2(ls0, pack2(e0, e1));
                                }
                                packed[q * 16 + (c >> 1)] = FP8 ? pack_f16(e0, e1) : pack_bf16(e0, e1);
                            }
                        };
                        weights(sa, 0);
                        tmem_wait_ld();
                        weights(sb, 1);
                        if (!__any_sync(0xffffffffu, fmaxf(mx0, mx1) * row_scale > m + kRescaleThreshold)) {
                            tmem_st32(s_addr, packed);
                            float a0, a1, a2, a3;
                            unpack2(ls0, a0, a1);
                            unpack2(ls1, a2, a3);
                            l += (a0 + a2) + (a1 + a3);
                            done = true;
                        }
                    }
                    // (said to be rare, so that the compiler lays this code out of the loop's way: the instruction cache holds little more than the loop)
                    if (__builtin_expect(!done, 0)) {
                        uint32_t sv[2][32];
                        tmem_ld32(s_addr, sv[0]);
                        tmem_ld32(s_addr + 32, sv[1]);
                        tmem_wait_ld();
                        scaled(sv[0], 0);
                        scaled(sv[1], 1);
                        if (masked) {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const uint32_t vis = valid ? mask_bits(mask_row, mask0, mask1, key0 + 32 * q - it.prior, it.nodes) : 0u;
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (!(vis >> c & 1u)) sv[q][c] = 0xff800000u;
                            }
                        }
                        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int c = 0; c < 32; c += 8) {
                                mx0 = max3(mx0, __uint_as_float(sv[q][c]), __uint_as_float(sv[q][c + 1]));
                                mx1 = max3(mx1, __uint_as_float(sv[q][c + 2]), __uint_as_float(sv[q][c + 3]));
                                mx2 = max3(mx2, __uint_as_float(sv[q][c + 4]), __uint_as_float(sv[q][c + 5]));
                                mx3 = max3(mx3, __uint_as_float(sv[q][c + 6]), __uint_as_float(sv[q][c + 7]));
                            }
                        const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * row_scale;
                        const float m_new = mx > m + kRescaleThreshold ? mx : m;  // also the first finite maximum
                        const float alpha = m_new == m ? 1.f : fast_exp2(m - m_new);
                        if (k > 0 && __any_sync(0xffffffffu, m_new != m)) {
                            // the accumulator as of the step before (what came before that was complete when these scores were)
                            ok = wait_all(bars + C::pv_done + 16 * x + 8 * (buf ^ 1), ((steps - 1) >> 1) & 1, s_abort);
                            if (!ok) break;
                            tc_fence_after();
                            const uint32_t o_addr = tmem + lane_addr + kColO + x * D;
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 32) {
                                uint32_t v[32];
                                tmem_ld32(o_addr + c0, v);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * alpha);
                                tmem_st32(o_addr + c0, v);
                            }
                            tmem_wait_st();
                        }
                        l *= alpha;
                        m = m_new;
                        const float m_sub = m == -INFINITY ? 0.f : m;
                        const uint64_t nm2 = pack2(-m_sub, -m_sub);
                        // (masked scores are -inf, and their weights exp2(-inf) = 0)
                        uint64_t ls0 = 0ull, ls1 = 0ull;
                        uint32_t packed[32];
#pragma unroll
                        for (int q = 0; q < 2; ++q)
#pragma unroll
                            for (int c = 0; c < 32; c += 2) {
                                float e0, e1;
                                unpack2(fma2(pack2(__uint_as_float(sv[q][c]), __uint_as_float(sv[q][c + 1])), sc2, nm2), e0, e1);
                                e0 = fast_exp2(e0), e1 = fast_exp2(e1);
                                if (c & 2) ls1 = add2(ls1, pack2(e0, e1));
                                else ls0 = add2(ls0, pack2(e0, e1));
                                packed[q * 16 + (c >> 1)] = FP8 ? pack_f16(e0, e1) : pack_bf16(e0, e1);
                            }
                        tmem_st32(s_addr, packed);
                        float a0, a1, a2, a3;
                        unpack2(ls0, a0, a1);
                        unpack2(ls1, a2, a3);
                        l += (a0 + a2) + (a1 + a3);
                    }
                    tmem_wait_st();
                }
                ++steps;
                if (must_wait_free) {
                    // the other stream's warps have read this stream's last accumulator, which the product to come overwrites
                    ok = wait_all(bars + C::ex_free, (n_ex & 1) ^ 1, s_abort);
                    if (!ok) break;
                    must_wait_free = false;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bars + C::p_ready + 16 * x + 8 * buf);
            }
            if (!ok) break;
            // ---- the item's end ----
            float w0 = 1.f, w1 = 0.f;  // weights of the accumulators (streams 0 and 1 where both have a part of the row)
            int col0 = 0, col1 = D;
            uint32_t o0 = tmem + lane_addr + kColO + x * D, o1 = o0;
            if (n_x == 1) {
                exchange[x * kRows + t] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(bars + C::ex_full);
            }
            more = iter.next(ahead);  // (under the last PV)
            if (more) keep(n_piece + 1, ahead);
            if (FP8) it = kept_piece(n_piece);
            const uint32_t last = 8 * ((steps - 1) & 1), last_par = ((steps - 1) >> 1) & 1;
            ok = wait_all(bars + C::pv_done + 16 * x + last, last_par, s_abort);
            if (!ok) break;
            if (n_x == 1) {
                // rows of one q tile: join the streams, which have taken as many steps; each writes half of the columns.  (The other's PV before
                // its last was complete when it had the scores of its last.)
                ok = wait_all(bars + C::ex_full, n_ex & 1, s_abort);
                if (ok) ok = wait_all(bars + C::pv_done + 16 * (x ^ 1) + last, last_par, s_abort);
                if (!ok) break;
                const float2 a = exchange[t], b = exchange[kRows + t];
                ++n_ex;
                must_wait_free = true;
                m = fmaxf(a.x, b.x);
                const float m_sub = m == -INFINITY ? 0.f : m;
                w0 = fast_exp2(a.x - m_sub);
                w1 = fast_exp2(b.x - m_sub);
                l = a.y * w0 + b.y * w1;
                o0 = tmem + lane_addr + kColO;
                o1 = o0 + D;
                col0 = x * (D / 2);
                col1 = col0 + D / 2;
            }
            tc_fence_after();
            if (warp_valid) {
                const bool whole = it.whole();
                const float inv = !whole ? 1.f : l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (l NaN: a score was)
                const int head = it.head * p.G + (t & (p.G - 1));
                char* const stage = smem + C::kOffQ + ((q_tiles + q_tile) & 1) * C::kTileBytes + (n_x == 2 ? (warp & 3) * 2 : warp) * (C::kTileBytes / 8);
                const int slot_row = (2 * (int)blockIdx.x + (it.tile0 > 0 ? 0 : 1)) * kGroupRows + q_tile * kRows + t;
                uint32_t flags = 0;
                for (int j = max(it.tile0, it.tree_tile()); j < it.tile1; ++j) {
                    const volatile uint32_t* const f = s_flagged + (tiles + j - it.tile0) % C::kFlagTiles * 4;
                    flags |= f[0] | f[1] | f[2] | f[3];
                }
#pragma unroll 1
                for (int c0 = col0; c0 < col1; c0 += 32) {
                    uint32_t v[32];
                    tmem_ld32(o0 + c0, v);
                    if (n_x == 1) {
                        uint32_t u[32];
                        tmem_ld32(o1 + c0, u);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(fmaf(__uint_as_float(v[c]), w0, __uint_as_float(u[c]) * w1));
                    } else {
                        tmem_wait_ld();
                    }
                    if (FP8) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(2.f * __uint_as_float(v[c]));  // (V was halved)
                    }
                    if (__builtin_expect(flags != 0 && valid, 0)) {
                        // tree tokens whose V row was taken out of the products: their weight times that row
#pragma unroll 1
                        for (int w = 4 * max(it.tile0, it.tree_tile()); w < 4 * it.tile1; ++w) {  // 32 keys
                            uint32_t todo = s_flagged[(tiles + (w >> 2) - it.tile0) % C::kFlagTiles * 4 + (w & 3)] & mask_bits(mask_row, mask0, mask1, 32 * w - it.prior, it.nodes);
                            while (todo) {
                                const int pos = 32 * w + __ffs(todo) - 1;
                                todo &= todo - 1;
                                const int64_t page = __ldg(p.block_table + (int64_t)it.r * p.max_pages + pos / kPage);
                                const char* const blk = p.pool + (page * p.Hkv + it.head) * (int64_t)(FP8 ? fp8_page_head_bytes(D) : page_head_bytes(D));
                                const __nv_bfloat16* const qr = p.q + (token * p.Hq + head) * D;
                                float dot = 0.f;
#pragma unroll 1
                                for (int e = 0; e < D; ++e) dot = fmaf(__bfloat162float(qr[e]), pool_value<D, FP8>(blk, 0, pos % kPage, e), dot);
                                const float weight = fast_exp2(fmaf(dot, kScaleLog2, -m));
#pragma unroll
                                for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(fmaf(weight, pool_value<D, FP8>(blk, 1, pos % kPage, c0 + c), __uint_as_float(v[c])));
                            }
                        }
                    }
                    if (whole) {
                        uint32_t y[16];
#pragma unroll
                        for (int c = 0; c < 32; c += 2) y[c / 2] = pack_bf16(__uint_as_float(v[c]) * inv, __uint_as_float(v[c + 1]) * inv);
                        store_rows<64>(stage, lane, y, [&](int row) -> char* {
                            const int tt = (t & ~31) + row, tok = q_tile * tile_tok + (tt >> g_shift);
                            return tok < it.n_tok ? reinterpret_cast<char*>(p.out + (((int64_t)it.q_tok + tok) * p.Hq + it.head * p.G + (tt & (p.G - 1))) * D + c0) : nullptr;
                        });
                    } else {
                        auto to = [&](int row, int c) -> char* {
                            return q_tile * tile_tok + (((t & ~31) + row) >> g_shift) < it.n_tok ? reinterpret_cast<char*>(p.part_o + (int64_t)(slot_row - lane + row) * D + c0 + c) : nullptr;
                        };
                        if (D == 128) {
                            store_rows<128>(stage, lane, v, [&](int row) { return to(row, 0); });
                        } else {
                            store_rows<64>(stage, lane, v, [&](int row) { return to(row, 0); });
                            store_rows<64>(stage, lane, v + 16, [&](int row) { return to(row, 16); });
                        }
                    }
                }
                if (valid && col0 == 0) {
                    if (!whole) p.part_ml[slot_row] = make_float2(m, l);
                    else if (p.lse) p.lse[token * p.Hq + head] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : l == 0.f ? -INFINITY : l;
                }
            }
            tc_fence_before();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (n_x == 1) mbar_arrive(bars + C::ex_free);
                for (int k = 0; k < n_x; ++k) mbar_arrive(bars + C::q_empty + 8 * ((q_tiles + k) & 1));
            }
            q_tiles += n_x;
            tiles += n_tiles;
            ++n_piece;
        }
    } else {
        if (warp == kLoadWarp) {
            // ================================================================
            // K and V tiles, in the order of use; entry e of the ring lies in slot e % kSlots
            // ================================================================
            const uint64_t policy = l2_policy_evict_first();
            int j = 0, head = 0;
            const int32_t* bt = nullptr;
            it.tile1 = 0;
            bool have = true, ok = true;
            // pages of the next tile (lanes 0-7: as far as the sequence goes), requested a tile ahead of their use
            auto fetch = [&](int& page, bool& inside, int& kv_head, bool& tree) {
                if (j == it.tile1) {
                    have = iter.next(it);
                    if (!have) return;
                    j = it.tile0;
                    head = it.head;
                    bt = p.block_table + (int64_t)it.r * p.max_pages;
                }
                const int at = j * (kTileKeys / kPage) + lane;
                inside = lane < kTileKeys / kPage && at * kPage < it.kv_len;
                page = inside ? __ldg(bt + at) : -1;
                kv_head = head;
                tree = j >= it.tree_tile();
                ++j;
            };
            auto pool_row = [&](int page, bool inside, int kv_head) {
                const bool good = (uint32_t)page < (uint64_t)p.num_pages;
                if (!good && inside) atomicOr(p.flag, kStatusBounds);
                return good ? (page * p.Hkv + kv_head) * (FP8 ? 1 : 2 * C::kHalves) : -8;  // (rows outside the pool read as zero)
            };
            uint32_t n_raw = 0;
            // K (kv = 0) or V of tile n; raw: V that warp 11 looks over
            auto load = [&](int row, uint32_t n, int kv, bool raw) {
                int r[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) r[k] = __shfl_sync(0xffffffffu, row, k);
                if (FP8) {
                    const Slot at = k_slot<C, FP8>(n);
                    const uint32_t land = kv ? C::raw + 8 * (n % C::kRaw) : at.full, free_ = kv ? C::raw_empty + 8 * (n % C::kRaw) : at.empty;
                    const uint32_t par = kv ? (n / C::kRaw) & 1 : at.par, dst = sbase + (kv ? C::kOffRaw + n % C::kRaw * C::kCodeBytes : at.at);
                    if (!wait_all(bars + free_, par ^ 1, s_abort)) return false;
                    if (elect_one()) {
                        const uint32_t scales = sbase + (kv ? C::kOffRawScale + n % C::kRaw * C::kScaleBytes : C::kOffScale + n % C::kScaleTiles * C::kScaleBytes);
                        mbar_expect_tx(bars + land, C::kCodeBytes + C::kScaleBytes);
                        s_armed[kv ? C::kSlots + 2 + n % C::kRaw : n % C::kSlots] = (int)par;
#pragma unroll
                        for (int k = 0; k < 8; k += 4) {
                            gather4_at(dst + k * kPage * D, &pool_map, kv * (kPage * D / 8), r[k], r[k + 1], r[k + 2], r[k + 3], bars + land, policy);
                            gather4_at(scales + k * 128, &scale_map, 0, r[k], r[k + 1], r[k + 2], r[k + 3], bars + land, policy);
                        }
                    }
                } else {
                    const Slot at = kv ? v_slot<C, FP8>(n) : k_slot<C, FP8>(n);
                    if (!wait_all(bars + at.empty, at.par ^ 1, s_abort)) return false;
                    if (elect_one()) {
                        const uint32_t land = bars + (raw ? C::raw + 8 * (n_raw % C::kRaw) : at.full), dst = sbase + at.at;
                        mbar_expect_tx(land, C::kTileBytes);
                        if (raw) s_armed[C::kSlots + 2 + n_raw % C::kRaw] = (int)(n_raw / C::kRaw & 1);
                        else s_armed[(at.full - C::full) / 8] = (int)at.par;
#pragma unroll
                        for (int h = 0; h < C::kHalves; ++h) {
                            int b[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) b[k] = r[k] < 0 ? r[k] : r[k] + kv * C::kHalves + h;
                            gather4(dst + h * C::kHalfBytes, &pool_map, b[0], b[1], b[2], b[3], land, policy);
                            gather4(dst + h * C::kHalfBytes + 4 * kPoolBlock, &pool_map, b[4], b[5], b[6], b[7], land, policy);
                        }
                    }
                }
                __syncwarp();
                return true;
            };
            int page = -1, kv_head = 0;
            bool inside = false, tree = false;
            fetch(page, inside, kv_head, tree);
            // K of tile n, then V of the one before
            int row_k = -8, row_v = -8;
            bool tree_v = false, more = have;
            for (uint32_t n = 0; ok && (more || n > 0); ++n) {
                for (int kv = 0; kv < 2 && ok; ++kv) {
                    if (kv == 0) {
                        row_v = row_k;
                        if (!more) continue;
                        row_k = pool_row(page, inside, kv_head);
                    } else if (n == 0) {
                        continue;
                    }
                    const bool raw = kv && tree_v;
                    ok = load(kv ? row_v : row_k, n - kv, kv, raw);
                    if (raw) ++n_raw;
                }
                if (!more) break;
                tree_v = tree;
                fetch(page, inside, kv_head, tree);
                more = have;
            }
        } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            // ================================================================
            // MMA issue of stream x.  QK^T of a step goes to the buffer that the step before the last had, once the PV that reads its weights has
            // been issued: the tensor pipe runs a thread's MMAs in order.
            // ================================================================
            const uint32_t x = warp - kMmaWarp;
            constexpr uint32_t kQBar = FP8 ? C::q_ready : C::q_full;
            // (FP8: E4M3 x E4M3, and f16 x f16)
            constexpr uint32_t kTypes = (1u << 7) | (1u << 10);  // bf16 x bf16
            constexpr uint32_t kIdescQK = instr_desc(kRows, 64, false) & (FP8 ? ~kTypes : ~0u), kIdescPV = instr_desc(kRows, D, true) & (FP8 ? ~kTypes : ~0u);
            const uint64_t desc_kmajor = smem_desc(0, 16, 1024), desc_v = smem_desc(0, C::kHalfBytes, 1024);
            PieceIter<Rows> iter_v = iter;
            Piece iv;
            bool ok = true, have_k = true;
            uint32_t k_tile = 0, v_tile = 0;         // tiles that QK^T and PV have finished
            uint32_t k_steps = 0, v_steps = 0;       // steps that they have issued
            uint32_t q_tiles = 0;                    // q tiles of the items before QK^T's
            int sk = 0, nk = 0, xk = 1;              // QK^T's step within the item, the stream's number of them, the item's q tiles
            int sv = 0, nv = 0, xv = 1;              // the same of PV
            while (ok) {
                if (have_k && sk == nk) {
                    if (nk > 0) q_tiles += xk;
                    have_k = iter.next(it);
                    xk = it.n_x(p.G);
                    nk = have_k ? (it.tile1 - it.tile0) * xk : 0;
                    sk = 0;
                }
                if (v_steps == k_steps && !have_k) break;
                const Slot ks = k_slot<C, FP8>(k_tile);
                const uint32_t vb = v_steps & 1;
                const uint32_t qs = (q_tiles + (xk == 2 ? x : 0)) & 1;
                bool do_qk = have_k && k_steps - v_steps < 2;
                // (the item's Q tile may have to wait for the end of the one before, and that for its PVs)
                const uint32_t q0 = q_tiles & 1, q0_par = (q_tiles >> 1) & 1, q1_par = ((q_tiles + 1) >> 1) & 1;
                if (do_qk && sk == 0 && v_steps != k_steps) {
                    const bool there = mbar_test_wait(bars + kQBar + 8 * q0, q0_par) && (xk == 1 || mbar_test_wait(bars + kQBar + 8 * (q0 ^ 1), q1_par));
                    do_qk = __all_sync(0xffffffffu, there);
                }
                if (do_qk && (xk == 1 || (sk & 1) == 0)) {
                    if (v_steps == k_steps) {
                        ok = wait_all(bars + ks.full, ks.par, s_abort);
                    } else {
                        const int which = either(0, bars + ks.full, ks.par, bars + C::p_ready + 16 * x + 8 * vb, (v_steps >> 1) & 1);
                        ok = which != 0;
                        do_qk = which == 1;
                    }
                    if (!ok) break;
                }
                if (do_qk) {
                    const uint32_t half = xk == 2 ? sk & 1 : x;
                    if (sk == 0) {
                        // (both of two tiles, so that neither barrier is ever a phase behind)
                        ok = wait_all(bars + kQBar + 8 * q0, q0_par, s_abort);
                        if (ok && xk == 2) ok = wait_all(bars + kQBar + 8 * (q0 ^ 1), q1_par, s_abort);
                        if (!ok) break;
                    }
                    const bool tile_ends = xk == 1 || (sk & 1) == 1;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t qd = desc_kmajor + ((sbase + C::kOffQ + qs * C::kTileBytes) >> 4),
                                       kd = desc_kmajor + ((sbase + ks.at + half * (64 * 128)) >> 4);
                        const uint32_t d_tm = tmem + x * 128 + (k_steps & 1) * 64;
                        if (FP8) {
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)  // the two parts of q, 32 elements a product
                                tc_mma_f8_ss(d_tm, qd + (((kk >> 2) * C::kHalfBytes + (kk & 3) * 32) >> 4), kd + ((kk & 3) * 32 >> 4), kIdescQK, kk > 0);
                        } else {
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint32_t off = ((kk >> 2) * C::kHalfBytes + (kk & 3) * 32) >> 4;
                                tc_mma_ss(d_tm, qd + off, kd + off, kIdescQK, kk > 0);
                            }
                        }
                        tc_commit(bars + C::s_full + 16 * x + 8 * (k_steps & 1));
                        if (tile_ends) tc_commit(bars + ks.empty);
                    }
                    __syncwarp();
                    if (tile_ends) ++k_tile;
                    ++sk;
                    ++k_steps;
                    continue;
                }
                if (sv == nv) {
                    iter_v.next(iv);
                    xv = iv.n_x(p.G);
                    nv = (iv.tile1 - iv.tile0) * xv;
                    sv = 0;
                }
                const Slot vs = v_slot<C, FP8>(v_tile);
                const uint32_t half = xv == 2 ? sv & 1 : x;
                if (xv == 1 || (sv & 1) == 0) {
                    ok = wait_all(bars + vs.full, vs.par, s_abort);
                    if (!ok) break;
                }
                ok = wait_all(bars + C::p_ready + 16 * x + 8 * vb, (v_steps >> 1) & 1, s_abort);
                if (!ok) break;
                const bool tile_ends = xv == 1 || (sv & 1) == 1;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t vd = desc_v + ((sbase + vs.at + half * (64 * 128)) >> 4);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        tc_mma_ts(tmem + kColO + x * D, tmem + x * 128 + vb * 64 + kk * 8, vd + kk * (2048 >> 4), kIdescPV, (sv > 0 || kk > 0) ? 1u : 0u);
                    tc_commit(bars + C::pv_done + 16 * x + 8 * vb);
                    if (tile_ends) tc_commit(bars + vs.empty);
                }
                __syncwarp();
                if (tile_ends) ++v_tile;
                ++sv;
                ++v_steps;
            }
        } else if (FP8 && warp == kQWarp) {
            // ================================================================
            // Q tiles, and each into two E4M3 numbers an element in its place.  Eight lanes have a row, 16 elements each.
            // ================================================================
            const int u = lane & 7;
            uint32_t n = 0, n_split = 0, pending = 0;
            bool ok = true;
            auto split = [&](uint32_t qb) {
                        char* const tile = smem + C::kOffQ + qb * C::kTileBytes;
        #pragma unroll 1
                        for (int i = 0; i < kRows / 4; ++i) {
                            const int row = 4 * i + (lane >> 3);
                            const char* const src = tile + (u >> 2) * C::kHalfBytes + row * 128;
                            const uint4 a = *reinterpret_cast<const uint4*>(src + (((2 * u) ^ row) & 7) * 16), b = *reinterpret_cast<const uint4*>(src + (((2 * u + 1) ^ row) & 7) * 16);
                            const uint32_t raw[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                            float x[16], top = 0.f;
                            bool finite = true;
        #pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                x[2 * k] = bf16_lo(raw[k]), x[2 * k + 1] = bf16_hi(raw[k]);
                                top = fmaxf(top, fmaxf(fabsf(x[2 * k]), fabsf(x[2 * k + 1])));
                            }
                            finite = !any_not_finite(a) && !any_not_finite(b);
        #pragma unroll
                            for (int o = 4; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                            finite = (__ballot_sync(0xffffffffu, !finite) >> (lane & 24) & 0xffu) == 0;
                            // 2^e with the row's largest times it in (224, 448]
                            const int exponent = (int)(__float_as_uint(top) >> 23) - 127;  // (of a bf16 subnormal: -127)
                            const bool high = (__float_as_uint(top) & 0x7fffffu) > 0x600000u;
                            const int e = min(8 - exponent - (high ? 1 : 0), 120);
                            const float up = __uint_as_float((uint32_t)(127 + e) << 23);
                            uint32_t hi[4], lo[4];
        #pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                float y[4], rest[4];
                                uint32_t code = 0;
        #pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    y[2 * h] = x[4 * k + 2 * h] * up, y[2 * h + 1] = x[4 * k + 2 * h + 1] * up;
                                    uint16_t two;
                                    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(y[2 * h + 1]), "f"(y[2 * h]));
                                    code |= (uint32_t)two << (16 * h);
                                    uint32_t back;
                                    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(two));
                                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&back));
                                    rest[2 * h] = y[2 * h] - f.x, rest[2 * h + 1] = y[2 * h + 1] - f.y;
                                }
                                hi[k] = code;
                                uint16_t r0, r1;
                                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r0) : "f"(rest[1]), "f"(rest[0]));
                                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r1) : "f"(rest[3]), "f"(rest[2]));
                                lo[k] = (uint32_t)r0 | (uint32_t)r1 << 16;
                            }
                            __syncwarp();  // (the row's other lanes have read what is overwritten)
                            char* const dst = tile + row * 128 + (((u ^ row) & 7) << 4);
                            *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                            *reinterpret_cast<uint4*>(dst + C::kHalfBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                            if (u == 0) *reinterpret_cast<float*>(smem + C::kOffQScale + (qb * kRows + row) * 4) = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : __uint_as_float(0x7fffffffu);
                            __syncwarp();
                        }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bars + C::q_ready + 8 * qb);
            };
            // (a tile is asked for before the one before it is split)
            auto finish = [&]() {
                if (pending == 0) return;
                ok = wait_all(bars + C::q_full + 8 * (n_split & 1), (n_split >> 1) & 1, s_abort);
                if (ok) split(n_split & 1);
                ++n_split;
                --pending;
            };
            while (ok && iter.next(it)) {
                for (int x = 0; x < it.n_x(p.G) && ok; ++x, ++n) {
                    if (!complete(bars + C::q_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1)) {
                        finish();  // (what it waits for may need that tile)
                        if (ok) ok = wait_all(bars + C::q_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1, s_abort);
                        if (!ok) break;
                    }
                    if (elect_one()) {
                        mbar_expect_tx(bars + C::q_full + 8 * (n & 1), C::kTileBytes);
                        s_armed[C::kSlots + (n & 1)] = (int)((n >> 1) & 1);
#pragma unroll
                        for (int h = 0; h < C::kHalves; ++h)
                            tma_load_3d(sbase + C::kOffQ + (n & 1) * C::kTileBytes + h * C::kHalfBytes, &q_map, h * 64, it.head * p.G, it.q_tok + x * tile_tok, bars + C::q_full + 8 * (n & 1));
                    }
                    __syncwarp();
                    finish();
                    ++pending;
                }
            }
            if (ok) finish();
        } else if (warp == kQWarp) {
            // ================================================================
            // Q tiles: rows (token, head of the group) in token-major order, a box of [128 / G tokens][G heads][64 elements] per half; and V
            // rows that no product may read.  (Their tiles land on barriers of their own, and this warp's arrival takes the place of the
            // copy's on the slot's.)  An item's Q may have to wait for the end of the one before, and that for its V: whichever
            // can go on.
            // ================================================================
            PieceIter<Rows> iter_v = iter;
            Piece iv;
            uint32_t n = 0, v_tile = 0, n_raw = 0;
            int x = 0, n_x = 0;        // q tile of the item, of that many
            int j = 0;                 // key tile of the item whose V comes next
            bool ok = true, have_q = iter.next(it), have_v = iter_v.next(iv);
            n_x = it.n_x(p.G);
            auto begin_v = [&]() {     // to the item's first tile with tree tokens, past those that have none
                while (have_v) {
                    j = max(iv.tile0, iv.tree_tile());
                    if (j < iv.tile1) return;
                    v_tile += iv.tile1 - iv.tile0;
                    have_v = iter_v.next(iv);
                }
            };
            begin_v();
            while (ok && (have_q || have_v)) {
                const uint32_t bq = bars + C::q_empty + 8 * (n & 1), pq = ((n >> 1) & 1) ^ 1, bv = bars + C::raw + 8 * (n_raw % C::kRaw), pv = n_raw / C::kRaw & 1;
                const int which = have_q && have_v ? either(200, bq, pq, bv, pv) : wait_all(have_q ? bq : bv, have_q ? pq : pv, s_abort) ? (have_q ? 1 : 2) : 0;
                ok = which != 0;
                if (which == 1) {
                    if (elect_one()) {
                        mbar_expect_tx(bars + C::q_full + 8 * (n & 1), C::kTileBytes);
                        s_armed[C::kSlots + (n & 1)] = (int)((n >> 1) & 1);
#pragma unroll
                        for (int h = 0; h < C::kHalves; ++h)
                            tma_load_3d(sbase + C::kOffQ + (n & 1) * C::kTileBytes + h * C::kHalfBytes, &q_map, h * 64, it.head * p.G, it.q_tok + x * tile_tok, bars + C::q_full + 8 * (n & 1));
                    }
                    __syncwarp();
                    ++n;
                    if (++x == n_x) {
                        x = 0;
                        have_q = iter.next(it);
                        n_x = it.n_x(p.G);
                    }
                } else if (which == 2) {
                    ++n_raw;
                    const uint32_t n_v = v_tile + j - iv.tile0;
                    const Slot at = v_slot<C, FP8>(n_v);
                    // (pages behind the last have landed as zeros)
                    const int last = (iv.kv_len + kPage - 1) / kPage * kPage;
                    for (int q = 0; q < 4; ++q) {
                        const int row = 32 * q + lane, key = j * kTileKeys + row;
                        char* const vrow = smem + at.at + row * 128;
                        bool odd = false;
                        if (key >= iv.prior && key < iv.kv_len) {
#pragma unroll
                            for (int u = 0; u < 8 * C::kHalves; ++u)
                                odd = any_not_finite(*reinterpret_cast<const uint4*>(vrow + (u >> 3) * C::kHalfBytes + (((u ^ row) & 7) << 4))) || odd;
                        }
                        const uint32_t flags = __ballot_sync(0xffffffffu, odd);
                        if (lane == 0) s_flagged[n_v % C::kFlagTiles * 4 + q] = flags;
                        if (odd || (key >= iv.kv_len && key < last)) {
#pragma unroll
                            for (int u = 0; u < 8 * C::kHalves; ++u) *reinterpret_cast<uint4*>(vrow + (u >> 3) * C::kHalfBytes + ((u & 7) << 4)) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bars + at.full);
                    if (++j == iv.tile1) {
                        v_tile += iv.tile1 - iv.tile0;
                        have_v = iter_v.next(iv);
                        begin_v();
                    }
                }
            }
        }
    }

    if constexpr (FP8) if (warp >= kConvertWarp) {
        // ====================================================================
        // FP8: V's codes into f16; 32 rows of a tile a warp.  Eight lanes have a row, 16 elements each.
        // ====================================================================
        const int w = warp - kConvertWarp, u = lane & 7;
        uint32_t n_v = 0;
        bool ok = true;
        while (ok && iter.next(it)) {
            for (int j = it.tile0; j < it.tile1; ++j, ++n_v) {
                const uint32_t vb = n_v & 1, rb = n_v % C::kRaw;
                ok = wait_all(bars + C::raw + 8 * rb, (n_v / C::kRaw) & 1, s_abort);
                if (ok) ok = wait_all(bars + C::conv_empty + 8 * vb, ((n_v >> 1) & 1) ^ 1, s_abort);
                if (!ok) break;
                const bool tree = j >= it.tree_tile();
                const char* const src = smem + C::kOffRaw + rb * C::kCodeBytes;
                char* const dst = smem + C::kOffConv + vb * C::kTileBytes + (u >> 2) * C::kHalfBytes;
                uint32_t flags = 0;
                // (rolled, a row ahead of its loads: this code shares the instruction cache with four other roles')
                const char* from = src + (32 * w + (lane >> 3)) * 128;
                const float* scale_at = reinterpret_cast<const float*>(smem + C::kOffRawScale + rb * C::kScaleBytes) + 2 * w * 32 + 16 + (lane >> 3);
                uint4 next = *reinterpret_cast<const uint4*>(from + (((u ^ (lane >> 3)) & 7) << 4));
                float next_scale = *scale_at;
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const int row = 32 * w + 4 * i + (lane >> 3), key = j * kTileKeys + row;
                    uint4 code = next;
                    const float vs = next_scale;
                    if (i < 7) {
                        next = *reinterpret_cast<const uint4*>(from + (i + 1) * 512 + (((u ^ (row + 4)) & 7) << 4));
                        next_scale = scale_at[(i + 1 >> 2) * 32 + (i + 1 & 3) * 4];
                    }
                    bool gone = false;
                    if (tree) {
                        auto nan = [](uint32_t c) { return (((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; };
                        const bool odd = key >= it.prior && key < it.kv_len && (nan(code.x) || nan(code.y) || nan(code.z) || nan(code.w) || !(fabsf(vs) <= 255.f));
                        const uint32_t any = __ballot_sync(0xffffffffu, odd);
#pragma unroll
                        for (int k = 0; k < 4; ++k) flags |= (any >> (8 * k) & 0xffu ? 1u : 0u) << (4 * i + k);
                        gone = key >= it.kv_len || (any >> (lane & 24) & 0xffu);
                        if (gone) code = make_uint4(0, 0, 0, 0);
                    }
                    const __half2 by = __float2half2_rn(gone ? 0.f : 128.f * vs), part = __float2half2_rn(1.f / 256.f);
                    const uint32_t c[4] = {code.x, code.y, code.z, code.w};
                    uint32_t y[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[2 * k]) : "h"((uint16_t)c[k]));
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y[2 * k + 1]) : "h"((uint16_t)(c[k] >> 16)));
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const __half2 v = __hmul2(__hmul2(*reinterpret_cast<const __half2*>(&y[k]), part), by);
                        y[k] = *reinterpret_cast<const uint32_t*>(&v);
                    }
                    // (the halves' lanes begin at different units: no bank conflicts)
                    const bool swap = u & 4;
                    const int u0 = 2 * u + (swap ? 1 : 0), u1 = 2 * u + (swap ? 0 : 1);
                    *reinterpret_cast<uint4*>(dst + row * 128 + (((u0 ^ row) & 7) << 4)) = swap ? make_uint4(y[4], y[5], y[6], y[7]) : make_uint4(y[0], y[1], y[2], y[3]);
                    *reinterpret_cast<uint4*>(dst + row * 128 + (((u1 ^ row) & 7) << 4)) = swap ? make_uint4(y[0], y[1], y[2], y[3]) : make_uint4(y[4], y[5], y[6], y[7]);
                }
                if (tree && lane == 0) s_flagged[n_v % C::kFlagTiles * 4 + w] = flags;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bars + C::conv_full + 8 * vb);
                    mbar_arrive(bars + C::raw_empty + 8 * rb);
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();  // every role has left its loop
    if (*s_abort) {
        // A bounded wait ran out: the output is invalid and the pool is flagged.  Copies under way get a bounded time to land, the MMAs
        // issued so far to retire, before shared and tensor memory are given back.
        if (threadIdx.x == 0) atomicOr(p.flag, kStatusTimeout);
        if (warp == kLoadWarp) {
            for (int s = 0; s < C::kSlots; ++s)
                if (s_armed[s] >= 0) mbar_wait(bars + C::full + 8 * s, (uint32_t)s_armed[s], kDrainLimitNs);
            for (int k = 0; k < C::kRaw; ++k)
                if (s_armed[C::kSlots + 2 + k] >= 0) mbar_wait(bars + C::raw + 8 * k, (uint32_t)s_armed[C::kSlots + 2 + k], kDrainLimitNs);
            for (int x = 0; x < 2; ++x)
                if (s_armed[C::kSlots + x] >= 0) mbar_wait(bars + C::q_full + 8 * x, (uint32_t)s_armed[C::kSlots + x], kDrainLimitNs);
        }
        if (warp == kMmaWarp || warp == kMmaWarp + 1) {
            if (elect_one()) tc_commit(bars + C::mma_drained);
            __syncwarp();
            mbar_wait(bars + C::mma_drained, 0, kDrainLimitNs);
        }
        tc_fence_before();
        __syncthreads();
    }
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------------------
// Items that a share's border cuts: with M the largest of the pieces' maxima,
//     out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s,
// piece after piece in the order of their keys.  blockIdx.x + 1 is the share that begins inside the item and is the first to; a warp
// has four rows.  Bound by latency: the search of the item, then one read of each piece's rows (147 cuts of 256 rows, 39 MB at the most);
// behind a tree kernel it takes some 4 us.
// ---------------------------------------------------------------------------
constexpr int kMergeThreads = 256, kMergeRows = 4;  // rows of a warp

template <int D, class Rows>
__global__ void __launch_bounds__(kMergeThreads) tree_merge_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ Rows rows) {
    constexpr int V = D / 32;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = (int)blockIdx.x + 1, border = share_begin(p, c);
    int r;
    {
        int lo = 0, hi = p.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (rows.unit_start[mid] <= border) lo = mid; else hi = mid - 1;
        }
        r = lo;
    }
    const int prior = rows.prior[r], q_tok = rows.q_start[r], nodes = rows.q_start[r + 1] - q_tok;
    const int tiles = (prior + nodes + kTileKeys - 1) / kTileKeys, per = tiles + p.item_units;
    const int item = (border - rows.unit_start[r]) / per, begin = rows.unit_start[r] + item * per, end = begin + per;
    pdl_wait();
    // (a border at an item's begin cuts nothing, nor does one before its first tile; and the item is the first border's inside it)
    const int first_tile = begin + p.item_units;
    if (border <= first_tile || share_begin(p, c - 1) > first_tile) return;
    const int group_tok = kGroupRows / p.G, groups = (nodes + group_tok - 1) / group_tok;
    const int head = item / groups, tok0 = (item - head * groups) * group_tok, n_rows = min(group_tok, nodes - tok0) * p.G;
    const int row0 = ((int)blockIdx.y * (kMergeThreads / 32) + warp) * kMergeRows;
    if (row0 >= n_rows) return;
    // pieces: shares c - 1, c, ...: the first one's begins with the item, so it lies in its share's second place, the others' in the first
    int n_seg = 2;
    while (share_begin(p, c + n_seg - 1) < end) ++n_seg;
    auto place = [&](int s) { return (int64_t)(2 * (c - 1 + s) + (s == 0 ? 1 : 0)) * kGroupRows; };
    float M[kMergeRows], l[kMergeRows], acc[kMergeRows][V];
#pragma unroll
    for (int k = 0; k < kMergeRows; ++k) {
        M[k] = -INFINITY, l[k] = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) acc[k][v] = 0.f;
    }
    for (int s = 0; s < n_seg; ++s) {
        float2 ml[kMergeRows];
        float x[kMergeRows][V];
#pragma unroll
        for (int k = 0; k < kMergeRows; ++k) {
            const int64_t at = place(s) + min(row0 + k, n_rows - 1);
            ml[k] = p.part_ml[at];
            const float* const src = p.part_o + at * D + lane * V;
            if (V == 4) *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(src);
            else *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(src);
        }
#pragma unroll
        for (int k = 0; k < kMergeRows; ++k) {
            const float top = fmaxf(M[k], ml[k].x), base = top == -INFINITY ? 0.f : top;
            const float a = fast_exp2(M[k] - base), b = fast_exp2(ml[k].x - base);
            M[k] = top;
            l[k] = fmaf(l[k], a, ml[k].y * b);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[k][v] = fmaf(acc[k][v], a, x[k][v] * b);
        }
    }
#pragma unroll
    for (int k = 0; k < kMergeRows; ++k) {
        const int row = row0 + k;
        if (row >= n_rows) break;
        const float inv = l[k] > 0.f ? 1.f / l[k] : l[k] == 0.f ? 0.f : l[k];
        const int64_t at = (int64_t)(q_tok + tok0 + row / p.G) * p.Hq + head * p.G + row % p.G;
        uint32_t* const dst = reinterpret_cast<uint32_t*>(p.out + at * D + lane * V);
#pragma unroll
        for (int v = 0; v < V; v += 2) dst[v / 2] = pack_bf16(acc[k][v] * inv, acc[k][v + 1] * inv);
        if (p.lse && lane == 0) p.lse[at] = l[k] > 0.f ? (M[k] + log2f(l[k])) * 0.6931471805599453f : l[k] == 0.f ? -INFINITY : l[k];
    }
}

constexpr int kSms = 148;  // of the device that the library is built for: CTAs, and places in the workspace

size_t workspace_bytes(const ps_shape& s) { return 2 * (size_t)kSms * kGroupRows * (s.head_dim * sizeof(float) + sizeof(float2)); }

struct TreeCall {
    const KvPool* pool;
    const void* q;
    const int32_t* block_table;
    int32_t max_pages;
    const int64_t* mask;
    int32_t mask_words;
    const int32_t *prior, *n_nodes;
    int32_t n;
    void* out;
    float* lse;
    char* ws;
    cudaStream_t stream;
};

template <int D, bool FP8, int N>
ps_status launch_rows(const TreeCall& a) {
    const ps_shape& shape = a.pool->shape;
    const int Hq = shape.n_q_heads, Hkv = shape.n_kv_heads, G = Hq / Hkv, group_tok = kGroupRows / G;
    using Rows = TreeRows<N>;
    Rows rows;  // (entries past n are not read)
    auto tiles_of = [&](int r) { return ((int64_t)a.prior[r] + a.n_nodes[r] + kTileKeys - 1) / kTileKeys; };
    auto items_of = [&](int r) { return Hkv * ((a.n_nodes[r] + group_tok - 1) / group_tok); };
    int64_t units = 0, items = 0, longest = 0;
    for (int r = 0; r < a.n; ++r) {
        items += items_of(r);
        units += items_of(r) * (tiles_of(r) + Cfg<D, FP8>::kItemUnits);
        longest = tiles_of(r) > longest ? tiles_of(r) : longest;
        if (units > 0x3fffffff) return fail(PS_ERR_INVALID, "too many keys in one batch");
    }
    const int64_t fair = units / kSms > Cfg<D, FP8>::kLeastShare ? units / kSms : Cfg<D, FP8>::kLeastShare;
    bool whole = items <= kSms;
    for (int r = 0; whole && r < a.n; ++r) whole = (tiles_of(r) - fair) * (a.n_nodes[r] * G > kRows ? 2 : 1) <= Cfg<D, FP8>::kMergeSteps;
    int32_t tokens = 0, begin = 0;
    for (int r = 0; r < a.n; ++r) {
        rows.q_start[r] = tokens;
        rows.unit_start[r] = begin;
        rows.prior[r] = a.prior[r];
        tokens += a.n_nodes[r];
        begin += (int32_t)(items_of(r) * (whole ? longest : tiles_of(r) + Cfg<D, FP8>::kItemUnits));
    }
    rows.q_start[a.n] = tokens;
    rows.unit_start[a.n] = begin;

    static PerDeviceOnce configured;
    const ps_status cfg = once_per_device(configured, []() -> ps_status {
        PS_CUDA_TRY(cudaFuncSetAttribute(tree_kernel<D, FP8, Rows>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, FP8>::kSmemBytes));
        return PS_OK;
    });
    if (cfg != PS_OK) return cfg;
    RunArgs m{};
    m.shape = shape;
    m.pool = a.pool->base;
    m.num_pages = a.pool->num_pages;
    m.q = (const __nv_bfloat16*)a.q;
    m.total_q = tokens;
    CUtensorMap q_map, pool_map, scale_map;
    ps_status st = encode_q_map(m, &q_map);
    if (st == PS_OK) st = FP8 ? encode_fp8_pool_maps(m, &pool_map, &scale_map) : encode_pool_map(m, &pool_map);
    if (!FP8) scale_map = pool_map;  // (not used)
    if (st != PS_OK) return st;
    TreeParams p{};
    p.q = m.q;
    p.block_table = a.block_table;
    p.mask = (const uint32_t*)a.mask;
    p.pool = a.pool->base;
    p.out = (__nv_bfloat16*)a.out;
    p.lse = a.lse;
    p.part_ml = (float2*)a.ws;
    p.part_o = (float*)(a.ws + 2 * (size_t)kSms * kGroupRows * sizeof(float2));
    p.flag = a.pool->flag_dev;
    p.num_pages = a.pool->num_pages;
    p.wait_limit_ns = (uint32_t)a.pool->wait_limit_ns;
    p.max_pages = a.max_pages, p.mask_words = a.mask_words, p.n = a.n, p.Hq = Hq, p.Hkv = Hkv, p.G = G, p.item_units = whole ? -(int32_t)longest : Cfg<D, FP8>::kItemUnits;
    const int64_t cut = units / Cfg<D, FP8>::kLeastShare;
    const int grid = (int)(whole ? items : cut < kSms ? cut : kSms);
    p.share = begin / grid, p.longer = begin % grid;
    st = launch_kernel(tree_kernel<D, FP8, Rows>, grid, Cfg<D, FP8>::kThreads, Cfg<D, FP8>::kSmemBytes, a.stream, 1, true, p, q_map, pool_map, scale_map, rows);
    if (st != PS_OK || whole) return st;
    return launch_kernel(tree_merge_kernel<D, Rows>, dim3(grid - 1, kGroupRows / (kMergeThreads / 32 * kMergeRows)), kMergeThreads, 0, a.stream, 1, true, p, rows);
}

}  // namespace

}  // namespace ps

using namespace ps;

extern "C" {

ps_status ps_attn_tree_workspace(const ps_shape* shape, size_t* bytes_out) {
    const ps_status st = check_shape(shape);
    if (st != PS_OK) return st;
    if (!bytes_out) return fail(PS_ERR_INVALID, "null argument");
    *bytes_out = workspace_bytes(*shape);
    return PS_OK;
}

ps_status ps_attn_tree(const ps_kv* kv, const void* q_dev, const int32_t* block_table_dev, int32_t max_pages, const int64_t* mask_dev, int32_t mask_words,
                       const int32_t* prior_host, const int32_t* n_nodes_host, int32_t n, void* out_dev, float* lse_out_dev, void* workspace_dev,
                       size_t workspace_bytes_given, void* stream) {
    if (!kv || !q_dev || !block_table_dev || !mask_dev || !prior_host || !n_nodes_host || !out_dev || !workspace_dev) return fail(PS_ERR_INVALID, "null argument");
    if (n < 1 || max_pages < 1) return fail(PS_ERR_INVALID, "n=%d, max_pages=%d must be positive", n, max_pages);
    if (mask_words < 1 || mask_words > kMaxNodes / 64) return fail(PS_ERR_UNSUPPORTED, "mask_words=%d: masks of 1 to %d words are supported", mask_words, kMaxNodes / 64);
    const KvPool& pool = pool_of(kv);
    if (workspace_bytes_given < workspace_bytes(pool.shape))
        return fail(PS_ERR_WORKSPACE, "workspace has %zu bytes, tree attention needs %zu", workspace_bytes_given, workspace_bytes(pool.shape));
    if ((uintptr_t)workspace_dev % 256 != 0) return fail(PS_ERR_INVALID, "workspace must be 256-byte aligned");
    if (((uintptr_t)q_dev | (uintptr_t)out_dev) % 16 != 0) return fail(PS_ERR_INVALID, "q and out must be 16-byte aligned");
    int64_t T = 0;
    for (int r = 0; r < n; ++r) {
        if (prior_host[r] < 0 || n_nodes_host[r] < 1) return fail(PS_ERR_INVALID, "request %d: %d nodes behind %d tokens", r, n_nodes_host[r], prior_host[r]);
        if (n_nodes_host[r] > 64 * mask_words) return fail(PS_ERR_INVALID, "request %d: %d nodes in a mask of %d bits", r, n_nodes_host[r], 64 * mask_words);
        if ((int64_t)prior_host[r] + n_nodes_host[r] > (int64_t)max_pages * kPage) return fail(PS_ERR_INVALID, "request %d: its tokens exceed max_pages * page_size", r);
        if ((int64_t)prior_host[r] + n_nodes_host[r] > kMaxTokens) return fail(PS_ERR_INVALID, "request %d: more than %lld tokens", r, (long long)kMaxTokens);
        T += n_nodes_host[r];
        if (T > (1 << 24)) return fail(PS_ERR_INVALID, "more than 2^24 tokens in one batch");
    }
    const int64_t row = (int64_t)pool.shape.n_q_heads * pool.shape.head_dim;
    // Results are stored while inputs are still read: queries and masks by other CTAs, and again by rows that see a V row taken out of the products.
    const void* const read[3] = {q_dev, mask_dev, block_table_dev};
    const void* const written[3] = {out_dev, lse_out_dev, workspace_dev};
    const int64_t read_bytes[3] = {T * row * 2, T * mask_words * 8, (int64_t)n * max_pages * 4};
    const int64_t written_bytes[3] = {T * row * 2, lse_out_dev ? T * pool.shape.n_q_heads * 4 : 0, (int64_t)workspace_bytes(pool.shape)};
    for (int i = 0; i < 3; ++i)
        for (int k = 0; k < 3; ++k)
            if (overlap(written[i], written_bytes[i], read[k], read_bytes[k]) || (i < k && overlap(written[i], written_bytes[i], written[k], written_bytes[k])))
                return fail(PS_ERR_INVALID, "out, lse and the workspace must not overlap each other or an input");
    int64_t t0 = 0;
    for (int32_t r0 = 0; r0 < n; r0 += kTreeRowsMax) {  // (a slice's kernel waits for the one before, whose workspace it uses)
        const int32_t m = n - r0 < kTreeRowsMax ? n - r0 : kTreeRowsMax;
        const TreeCall a{&pool, (const char*)q_dev + t0 * row * 2, block_table_dev + (int64_t)r0 * max_pages, max_pages, mask_dev + t0 * mask_words, mask_words, prior_host + r0,
                         n_nodes_host + r0, m, (char*)out_dev + t0 * row * 2, lse_out_dev ? lse_out_dev + t0 * pool.shape.n_q_heads : nullptr, (char*)workspace_dev,
                         (cudaStream_t)stream};
        const ps_status st = pool.shape.dtype == 1        ? (m <= 64 ? launch_rows<128, true, 64>(a) : m <= 512 ? launch_rows<128, true, 512>(a) : launch_rows<128, true, kTreeRowsMax>(a))
                             : pool.shape.head_dim == 128 ? (m <= 64 ? launch_rows<128, false, 64>(a) : m <= 512 ? launch_rows<128, false, 512>(a) : launch_rows<128, false, kTreeRowsMax>(a))
                                                          : (m <= 64 ? launch_rows<64, false, 64>(a) : m <= 512 ? launch_rows<64, false, 512>(a) : launch_rows<64, false, kTreeRowsMax>(a));
        if (st != PS_OK) return st;
        for (int32_t r = r0; r < r0 + m; ++r) t0 += n_nodes_host[r];
    }
    return PS_OK;
}

ps_status ps_kv_set_wait_limit(ps_kv* kv, int64_t limit_ns) {
    if (!kv) return fail(PS_ERR_INVALID, "null argument");
    if (limit_ns < 0 || limit_ns > kMaxWaitLimitNs) return fail(PS_ERR_INVALID, "limit_ns=%lld outside 0 .. %lld", (long long)limit_ns, (long long)kMaxWaitLimitNs);
    const_cast<KvPool&>(pool_of(kv)).wait_limit_ns = limit_ns;
    return PS_OK;
}

}  // extern "C"
