// The paged cache's side of a speculative step: append with the norms of queries and keys and the position rotation in the
// same pass, moving an accepted path's tokens, and reading stretches of many sequences back as bf16.
#include <type_traits>

#include "kv_rows.cuh"
#include "tcgen05.cuh"

namespace ps {

namespace {

// ---------------------------------------------------------------------------
// Append with norms and rotation
//
//     y = x / sqrt(mean(x^2) + eps) * w            (q and k heads; where weights are given)
//     (a, b) -> (a cos - b sin, b cos + a sin)     (pairs of the first rot_dim elements)
//
// q goes to its output, k and v to their pages.  Everything between the load and the store is fp32: a key is rounded once, to bf16
// or, in an FP8 cache, to its code.  D / 8 lanes hold a head, 16 bytes each, so the norm is a sum over 8 or 16 lanes, a rotated pair's
// other half (half-split pairs) comes by shuffle from the lane rot_dim / 16 away, and a lane's angles and norm weights are the same for
// every head of their kind and are loaded once a token.  Bound by memory and, nearly as much, by instructions: some 60 a warp and pair of
// heads with two elements an instruction.  Measured: 6722 tokens of 32 + 8 + 8 heads of 128, 166 MB, in 36 us (4.6 TB/s; 50 us with a CTA a
// token); 2560 tokens of 64 + 8 + 8 into an FP8 cache, 99 MB, in 29 us.
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeAhead = 3;     // few tokens: heads of a lane whose loads are under way together
// Many tokens: four stages a CTA and two CTAs an SM.  (32 + 8 + 8 heads, bf16: 3000 tokens take 18.8 us with four stages and two teams of
// four warps, 17.8 with eight stages and four teams of two, but 6722 tokens 36 us against 39; one team of eight warps 23.1, a warp a token 28.)
constexpr int kRopeStages = 4, kRopeTeams = 2, kRopeTeamWarps = kRopeThreads / 32 / kRopeTeams;
// (Tokens of which four do not fit, from some 100 heads of 128 in all, take a CTA each at any count, at a price: 6000 tokens of 80 + 10 + 10 heads in stretches 60 us,
// 5.2 TB/s; of 96 + 12 + 12 a CTA each 133 us, 2.8 TB/s.)
constexpr int kRopeRingBytes = 108 * 1024, kRopeRingCtas = 2 * 148;
// Up to here a CTA a token is faster: all of them run at once and none waits for a stage.  (The same heads, a CTA a token and in
// stretches: 64 tokens 3.4 and 5.9 us, 256 4.1 and 6.6, 400 7.3 and 6.0, 900 12.5 and 8.8; FP8 256 4.7 and 8.1, 400 8.3 and 7.0.)
constexpr int kRopeFew = 2 * 148;

struct RopeParams {
    char* pool;
    int64_t num_pages;
    const __nv_bfloat16 *q, *k, *v;  // of the launch's first token
    int64_t q_stride, k_stride, v_stride;
    __nv_bfloat16* q_out;
    const __nv_bfloat16 *q_weight, *k_weight;
    const float* cos_sin;
    int64_t n_positions;
    const int32_t* positions;
    const int32_t* block_table;
    int* flag;
    float eps;
    uint32_t wait_limit_ns;
    int32_t rot_dim, interleaved, max_pages, n, Hq, Hkv, tokens, stage_bytes;
};

__device__ __forceinline__ uint64_t widened(uint32_t two) { return pack2(bf16_lo(two), bf16_hi(two)); }

// A lane's part of a head: y = x a + x' b over its 8 elements, x' the other elements of their pairs, a and b the angles times the norm's weights.
template <int D, bool FP8>
struct RopeLane {
    static constexpr int L = D / 8;  // lanes of a head
    const RopeParams& p;
    int l, e0, other;  // the lane within its head, its first element, the lane of its pairs' other elements
    bool turns;
    uint4 wq, wq_other, wk, wk_other;
    struct Kind {
        uint64_t a[4], b[4];  // of pairs of elements
    };

    __device__ __forceinline__ explicit RopeLane(const RopeParams& params) : p(params) {
        const int half = p.rot_dim >> 1;
        l = threadIdx.x % L, e0 = 8 * l;
        turns = e0 < p.rot_dim;
        other = !turns || p.interleaved ? l : e0 < half ? l + half / 8 : l - half / 8;
        wq = wq_other = wk = wk_other = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);  // ones
        if (p.q_weight) wq = __ldg(reinterpret_cast<const uint4*>(p.q_weight + e0)), wq_other = __ldg(reinterpret_cast<const uint4*>(p.q_weight + 8 * other));
        if (p.k_weight) wk = __ldg(reinterpret_cast<const uint4*>(p.k_weight + e0)), wk_other = __ldg(reinterpret_cast<const uint4*>(p.k_weight + 8 * other));
        if (p.interleaved) wq_other = swapped(wq), wk_other = swapped(wk);
    }
    static __device__ __forceinline__ uint4 swapped(const uint4& x) {  // the pairs themselves, turned round
        return make_uint4(__byte_perm(x.x, 0, 0x1032), __byte_perm(x.y, 0, 0x1032), __byte_perm(x.z, 0, 0x1032), __byte_perm(x.w, 0, 0x1032));
    }
    // cosines and, with the sign of the other element's part, sines of the lane's elements, from a row of the table
    __device__ __forceinline__ Kind angles(const float* row) const {
        Kind f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f.a[i] = pack2(1.f, 1.f), f.b[i] = 0ull;
        if (!turns) return f;
        const int half = p.rot_dim >> 1;
        if (p.interleaved) {
            const float4 c = *reinterpret_cast<const float4*>(row + e0 / 2), s = *reinterpret_cast<const float4*>(row + half + e0 / 2);
            f.a[0] = pack2(c.x, c.x), f.a[1] = pack2(c.y, c.y), f.a[2] = pack2(c.z, c.z), f.a[3] = pack2(c.w, c.w);
            f.b[0] = pack2(-s.x, s.x), f.b[1] = pack2(-s.y, s.y), f.b[2] = pack2(-s.z, s.z), f.b[3] = pack2(-s.w, s.w);
        } else {
            const float* const at = row + (e0 < half ? e0 : e0 - half);
            const float sign = e0 < half ? -1.f : 1.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 c = reinterpret_cast<const float4*>(at)[i], s = reinterpret_cast<const float4*>(at + half)[i];
                f.a[2 * i] = pack2(c.x, c.y), f.a[2 * i + 1] = pack2(c.z, c.w);
                f.b[2 * i] = pack2(sign * s.x, sign * s.y), f.b[2 * i + 1] = pack2(sign * s.z, sign * s.w);
            }
        }
        return f;
    }
    __device__ __forceinline__ static Kind weighted(const Kind& f, const uint4& w4, const uint4& wo4) {
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w}, wo[4] = {wo4.x, wo4.y, wo4.z, wo4.w};
        Kind g;
#pragma unroll
        for (int i = 0; i < 4; ++i) g.a[i] = mul2(f.a[i], widened(w[i])), g.b[i] = mul2(f.b[i], widened(wo[i]));
        return g;
    }
    // 1 / root mean square of the head, by all lanes of a warp
    __device__ __forceinline__ float inverse_rms(const uint64_t (&y)[4]) const {
        uint64_t ss2 = 0ull;
#pragma unroll
        for (int i = 0; i < 4; ++i) ss2 = fma2(y[i], y[i], ss2);
        float s0, s1;
        unpack2(ss2, s0, s1);
        float ss = s0 + s1;
#pragma unroll
        for (int o = L / 2; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        return rsqrtf(ss * (1.f / D) + p.eps);
    }
    // y: the lane's elements, x_other: the others of their pairs
    __device__ __forceinline__ void turn(uint64_t (&y)[4], const uint4& x_other, const Kind& f, bool normed, float rstd) const {
        const uint32_t xo[4] = {x_other.x, x_other.y, x_other.z, x_other.w};
        const uint64_t by = pack2(rstd, rstd);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint64_t z = widened(xo[i]);
            if (normed) y[i] = mul2(y[i], by), z = mul2(z, by);  // (first, so that no product with a weight overflows)
            y[i] = mul2(y[i], f.a[i]);
            if (turns) y[i] = fma2(z, f.b[i], y[i]);
        }
    }
    __device__ __forceinline__ void store16(char* dst, const uint64_t (&y)[4]) const {
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(y[i], f[2 * i], f[2 * i + 1]);
        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
    // the lane's part of a token in a bf16 page
    __device__ __forceinline__ char* place(int g, int which, int64_t page, int slot) const {
        return p.pool + (page * p.Hkv + g) * (int64_t)page_head_bytes(D) + which * block_bytes(D) + unit_offset(slot, e0);
    }
    // The lane's part of a key (which = 0) or value (1) of kv head g to its page; by all lanes of a warp, some of which store nothing.
    __device__ __forceinline__ void store_kv(const uint64_t (&y)[4], int g, int which, int64_t page, int slot, bool yes) const {
        if (!FP8) {
            if (yes) store16(place(g, which, page, slot), y);
            return;
        }
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(y[i], f[2 * i], f[2 * i + 1]);
        float amax = fmaxf(fabsf(f[0]), fabsf(f[1]));
#pragma unroll
        for (int i = 2; i < 8; i += 2) amax = max3(amax, fabsf(f[i]), fabsf(f[i + 1]));
#pragma unroll
        for (int o = L / 2; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        if (!yes) return;
        const float scale = fp8_scale(amax);
        char* const blk = p.pool + (page * p.Hkv + g) * (int64_t)fp8_page_head_bytes(D);
        *reinterpret_cast<uint2*>(blk + which * (kPage * D) + slot * D + (((l >> 1) ^ (slot & 7)) << 4) + 8 * (l & 1)) =
            make_uint2(quantise4(f[0], f[1], f[2], f[3], scale), quantise4(f[4], f[5], f[6], f[7], scale));
        if (l == 0) reinterpret_cast<float*>(blk + 2 * kPage * D)[which * kPage + slot] = scale;
    }
};

// Few tokens: a CTA has one.  Bound by latency: the lookup of the request, then the page and the heads together, then the angles.
template <int D, bool FP8, class Rows>
__global__ void __launch_bounds__(kRopeThreads) write_rope_kernel(const RopeParams p, const __grid_constant__ Rows rows) {
    constexpr int L = D / 8, kGroups = kRopeThreads / L;
    pdl_trigger();
    const int t = blockIdx.x, group = threadIdx.x / L;
    const int r = request_of(rows, p.n, t);
    const int pos = rows.prior(r) + (t - rows.q_start(r)), slot = pos % kPage;
    const int n_vec = p.Hq + 2 * p.Hkv;
    pdl_wait();
    const int64_t page = p.block_table[(int64_t)r * p.max_pages + pos / kPage];
    const int64_t angle = p.positions ? p.positions[t] : pos;
    const RopeLane<D, FP8> mine(p);
    const int other_lane = (threadIdx.x & 31) - mine.l + mine.other;
    const __nv_bfloat16 *const q_row = p.q + (int64_t)t * p.q_stride + mine.e0, *const k_row = p.k + (int64_t)t * p.k_stride + mine.e0,
                              *const v_row = p.v + (int64_t)t * p.v_stride + mine.e0;
    uint4 raw[kRopeAhead];
    auto load = [&](int v0) {
#pragma unroll
        for (int a = 0; a < kRopeAhead; ++a) {
            const int vec = v0 + a * kGroups;
            raw[a] = make_uint4(0, 0, 0, 0);
            if (vec < n_vec)
                raw[a] = *reinterpret_cast<const uint4*>(vec < p.Hq ? q_row + vec * D : vec < p.Hq + p.Hkv ? k_row + (vec - p.Hq) * D : v_row + (vec - p.Hq - p.Hkv) * D);
        }
    };
    load(group);
    if (page < 0 || page >= p.num_pages || (p.rot_dim > 0 && (angle < 0 || angle >= p.n_positions))) {
        if (threadIdx.x == 0) atomicOr(p.flag, kStatusBounds);
        return;
    }
    const auto f = mine.angles(p.cos_sin + angle * p.rot_dim);
#pragma unroll 1
    for (int v0 = group; v0 - group < n_vec; v0 += kGroups * kRopeAhead) {  // (the same number of steps in every lane of a warp: they shuffle)
        if (v0 != group) load(v0);
#pragma unroll
        for (int a = 0; a < kRopeAhead; ++a) {
            const int vec = v0 + a * kGroups;
            if (vec - group >= n_vec) continue;
            const bool is_q = vec < p.Hq, is_v = vec >= p.Hq + p.Hkv;
            const uint4 x = raw[a];
            uint64_t y[4] = {widened(x.x), widened(x.y), widened(x.z), widened(x.w)};
            if (!__all_sync(0xffffffffu, is_v)) {
                const bool normed = is_q ? p.q_weight != nullptr : p.k_weight != nullptr;
                const float rstd = mine.inverse_rms(y);
                uint4 xo;
                xo.x = __shfl_sync(0xffffffffu, x.x, other_lane), xo.y = __shfl_sync(0xffffffffu, x.y, other_lane);
                xo.z = __shfl_sync(0xffffffffu, x.z, other_lane), xo.w = __shfl_sync(0xffffffffu, x.w, other_lane);
                if (p.interleaved) xo = mine.swapped(x);
                if (!is_v) mine.turn(y, xo, is_q ? mine.weighted(f, mine.wq, mine.wq_other) : mine.weighted(f, mine.wk, mine.wk_other), normed, rstd);
            }
            if (is_q) mine.store16(reinterpret_cast<char*>(p.q_out + ((int64_t)t * p.Hq + vec) * D + mine.e0), y);
            if (!FP8 && is_v) {  // (as it came: through fp32 a NaN would lose its bits)
                if (vec < n_vec) *reinterpret_cast<uint4*>(mine.place(vec - p.Hq - p.Hkv, 1, page, slot)) = x;
            } else if (!FP8 || !__all_sync(0xffffffffu, is_q)) {
                mine.store_kv(y, vec - p.Hq - (is_v ? p.Hkv : 0), is_v, page, slot, !is_q && vec < n_vec);
            }
        }
    }
}

// Many tokens: a CTA has a stretch of them.  Its last warp looks the tokens up, 32 at a time, and sends a token's three rows and its angles to
// shared memory by bulk copies; the others work in two teams, a token each, so that what a token needs once (angles times weights) is
// worked out in four warps, and a team's next token is under way meanwhile.  A stage is always the same team's: both sides of its
// barriers see every phase.
template <int D, bool FP8, class Rows>
__global__ void __launch_bounds__(kRopeThreads + 32, 2) write_rope_ring_kernel(const RopeParams p, const __grid_constant__ Rows rows) {
    constexpr int L = D / 8, kWarps = kRopeThreads / 32;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint64_t s_bar[2 * kRopeStages];  // full, empty
    __shared__ int2 s_where[kRopeStages];        // page (-1: the token is passed over) and slot
    __shared__ int s_abort[2];
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t full = smem_u32(s_bar), empty = full + 8 * kRopeStages;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kRopeStages; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, kRopeTeamWarps);
        mbar_fence_init();
        s_abort[0] = 0, s_abort[1] = (int)p.wait_limit_ns;
    }
    __syncthreads();
    pdl_wait();
    const int t0 = (int)((int64_t)p.tokens * blockIdx.x / gridDim.x), n = (int)((int64_t)p.tokens * (blockIdx.x + 1) / gridDim.x) - t0;
    const uint32_t q_bytes = p.Hq * D * 2, kv_bytes = p.Hkv * D * 2, angle_bytes = p.rot_dim * 4;
    if (warp == kWarps) {
        const uint64_t policy = l2_policy_evict_first();
        int stage = 0, issued = 0;
        uint32_t par = 0;
        bool ok = true;
        for (int i0 = 0; ok && i0 < n; i0 += 32) {
            const int m = min(32, n - i0), t = t0 + i0 + min(lane, m - 1);
            const int r = request_of(rows, p.n, t);
            const int pos = rows.prior(r) + (t - rows.q_start(r));
            int page = p.block_table[(int64_t)r * p.max_pages + pos / kPage];
            const int angle = p.positions ? p.positions[t] : pos;
            if (page < 0 || page >= p.num_pages || (p.rot_dim > 0 && (angle < 0 || angle >= p.n_positions))) {
                atomicOr(p.flag, kStatusBounds);
                page = -1;
            }
            for (int i = 0; i < m; ++i) {
                ok = __all_sync(0xffffffffu, wait_or_abort(empty + 8 * stage, par ^ 1, s_abort));
                if (!ok) break;
                const int page_i = __shfl_sync(0xffffffffu, page, i), slot_i = __shfl_sync(0xffffffffu, pos % kPage, i);
                const int64_t angle_i = __shfl_sync(0xffffffffu, angle, i), t_i = t0 + i0 + i;
                if (lane == 0) {
                    s_where[stage] = make_int2(page_i, slot_i);
                    const uint32_t bar = full + 8 * stage, dst = smem_u32(smem) + stage * p.stage_bytes;
                    if (page_i < 0) {
                        mbar_arrive(bar);
                    } else {
                        mbar_expect_tx(bar, q_bytes + 2 * kv_bytes + angle_bytes);
                        bulk_g2s_hint(dst, p.q + t_i * p.q_stride, q_bytes, bar, policy);
                        bulk_g2s_hint(dst + q_bytes, p.k + t_i * p.k_stride, kv_bytes, bar, policy);
                        bulk_g2s_hint(dst + q_bytes + kv_bytes, p.v + t_i * p.v_stride, kv_bytes, bar, policy);
                        if (angle_bytes) bulk_g2s_hint(dst + q_bytes + 2 * kv_bytes, p.cos_sin + angle_i * p.rot_dim, angle_bytes, bar, policy);
                    }
                }
                __syncwarp();
                ++issued;
                if (++stage == kRopeStages) stage = 0, par ^= 1;
            }
        }
        __syncwarp();
        // what is under way lands before the block ends (as it does by itself where no wait ran out)
        for (int i = max(0, issued - kRopeStages); i < issued; ++i) mbar_wait(full + 8 * (i % kRopeStages), (i / kRopeStages) & 1, kDrainLimitNs);
        if (!ok && lane == 0) atomicOr(p.flag, kStatusAppendTimeout);
    } else {
        const RopeLane<D, FP8> mine(p);
        constexpr int kHeads = 32 / L;  // of a warp
        constexpr int kStep = kRopeTeamWarps * kHeads;
        const int team = warp / kRopeTeamWarps, first = warp % kRopeTeamWarps * kHeads, sub = lane / L;
        int stage = team;
        uint32_t par = 0;
        for (int i = team; i < n; i += kRopeTeams) {
            if (!__all_sync(0xffffffffu, wait_or_abort(full + 8 * stage, par, s_abort))) {
                if (lane == 0) atomicOr(p.flag, kStatusAppendTimeout);
                break;
            }
            const int2 where = s_where[stage];
            if (where.x >= 0) {
                const char* const src = smem + stage * p.stage_bytes;
                const float* const row = reinterpret_cast<const float*>(src + q_bytes + 2 * kv_bytes);
                const char* const mine_at = src + 2 * mine.e0;
                // a head's elements, normed and turned
                auto worked = [&](uint64_t (&y)[4], const char* at, const auto& f, bool normed) {
                    const uint4 x = *reinterpret_cast<const uint4*>(at);
                    y[0] = widened(x.x), y[1] = widened(x.y), y[2] = widened(x.z), y[3] = widened(x.w);
                    const float rstd = normed ? mine.inverse_rms(y) : 1.f;
                    mine.turn(y, p.interleaved ? mine.swapped(x) : *reinterpret_cast<const uint4*>(at + 16 * (mine.other - mine.l)), f, normed, rstd);
                };
                {
                    const auto f = mine.weighted(mine.angles(row), mine.wq, mine.wq_other);
                    const bool normed = p.q_weight != nullptr;
                    char* const out = reinterpret_cast<char*>(p.q_out + (int64_t)(t0 + i) * p.Hq * D + mine.e0);
#pragma unroll 2
                    for (int h0 = first; h0 < p.Hq; h0 += kStep) {
                        const int h = min(h0 + sub, p.Hq - 1);
                        uint64_t y[4];
                        worked(y, mine_at + h * (2 * D), f, normed);
                        if (h == h0 + sub) mine.store16(out + h * (2 * D), y);
                    }
                }
                const auto f = mine.weighted(mine.angles(row), mine.wk, mine.wk_other);
                const bool normed = p.k_weight != nullptr;
#pragma unroll 1
                for (int g0 = first; g0 < p.Hkv; g0 += kStep) {
                    const int g = min(g0 + sub, p.Hkv - 1);
                    uint64_t y[4];
                    worked(y, mine_at + q_bytes + g * (2 * D), f, normed);
                    mine.store_kv(y, g, 0, where.x, where.y, g == g0 + sub);
                }
#pragma unroll 1
                for (int g0 = first; g0 < p.Hkv; g0 += kStep) {
                    const int g = min(g0 + sub, p.Hkv - 1);
                    const uint4 x = *reinterpret_cast<const uint4*>(mine_at + q_bytes + kv_bytes + g * (2 * D));
                    if (FP8) {
                        const uint64_t y[4] = {widened(x.x), widened(x.y), widened(x.z), widened(x.w)};
                        mine.store_kv(y, g, 1, where.x, where.y, g == g0 + sub);
                    } else if (g == g0 + sub) {
                        *reinterpret_cast<uint4*>(mine.place(g, 1, where.x, where.y)) = x;
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * stage);
            if ((stage += kRopeTeams) >= kRopeStages) stage = team, par ^= 1;
        }
    }
}

// ---------------------------------------------------------------------------
// Accepted paths: slot prior + i of the sequence receives token prior + index[i], i < count, for an increasing path.
//
// A warp has one (request, kv head), a lane one 16-byte unit of K or V (and, FP8, a scale), the same unit of every token, so what a lane
// reads no other lane writes.  It reads a group of tokens before it stores any of them, and what it has stored
// lies below every later source: index[i] >= i.  Bound by the latency of a chain (path, pages, tokens), so the path's places and pages are
// looked up by 32 lanes at once and handed round; one lookup after the other for each token took 12.8 us where this takes 11.1 (256 requests,
// 8 kv heads, paths of up to 9 tokens in an FP8 cache, cold; 3 MB).
// ---------------------------------------------------------------------------
constexpr int kAcceptThreads = 128;
constexpr int kAcceptAhead = 8;

struct AcceptParams {
    char* pool;
    int64_t num_pages;
    const int32_t* block_table;
    const int32_t *index, *count;
    int* flag;
    int32_t index_stride, max_pages, n, Hkv;
};

template <int D, bool FP8, class Rows>
__global__ void __launch_bounds__(kAcceptThreads) accept_kernel(const AcceptParams p, const __grid_constant__ Rows rows) {
    constexpr int kUnits = FP8 ? D / 16 : D / 8;  // 16-byte units of a token's K, and of its V
    constexpr int kLanes = 2 * kUnits + (FP8 ? 2 : 0);
    static_assert(kLanes <= 32, "a lane per unit");
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t job = (int64_t)blockIdx.x * (kAcceptThreads / 32) + (threadIdx.x >> 5);
    const int r = (int)(job / p.Hkv), g = (int)(job % p.Hkv);
    pdl_wait();
    if (r >= p.n) return;
    const int nodes = rows.q_start(r + 1) - rows.q_start(r), prior = rows.prior(r);
    const int count = p.count[r];
    const int32_t* const index = p.index + (int64_t)r * p.index_stride;
    int node = lane < p.index_stride ? index[lane] : 0;  // (under way with the count)
    bool good = count >= 0 && count <= nodes && count <= p.index_stride;
    if (good) {
        for (int i = lane; i < count; i += 32) {
            const int at = i == lane ? node : index[i];
            good = good && at >= i && at < nodes && (i == 0 || at > index[i - 1]);
        }
    }
    if (!__all_sync(0xffffffffu, good)) {
        if (lane == 0) atomicOr(p.flag, kStatusBounds);
        return;
    }
    const int32_t* const table = p.block_table + (int64_t)r * p.max_pages;
    const int64_t head_bytes = FP8 ? fp8_page_head_bytes(D) : page_head_bytes(D);
    char* const pool = p.pool + g * head_bytes;
    auto part = [&](int32_t page, int slot) -> char* {  // this lane's part of a token
        char* const blk = pool + (int64_t)page * p.Hkv * head_bytes;
        if (FP8) {
            if (lane >= 2 * kUnits) return blk + 2 * kPage * D + ((lane - 2 * kUnits) * kPage + slot) * 4;
            return blk + (lane / kUnits) * (kPage * D) + slot * D + (((lane % kUnits) ^ (slot & 7)) << 4);
        }
        return blk + (lane / kUnits) * block_bytes(D) + unit_offset(slot, 8 * (lane % kUnits));
    };
    for (int c0 = 0; c0 < count; c0 += 32) {
        // lane a: where the path's token c0 + a is and where it goes
        const int mine = c0 + lane;
        if (c0 > 0 && mine < count) node = index[mine];
        int32_t from = 0, to = 0;
        bool moves = mine < count && node != mine;  // (else it is there already)
        if (moves) {
            from = table[(prior + node) / kPage], to = table[(prior + mine) / kPage];
            if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) {
                atomicOr(p.flag, kStatusBounds);
                moves = false;
            }
        }
        const uint32_t moving = __ballot_sync(0xffffffffu, moves);
        const int n = min(32, count - c0), from_slot = (prior + node) % kPage;
        for (int i0 = 0; i0 < n; i0 += kAcceptAhead) {
            uint4 x[kAcceptAhead];
            int32_t to_page[kAcceptAhead];
#pragma unroll
            for (int a = 0; a < kAcceptAhead; ++a) {
                const int i = i0 + a;
                const int32_t page = __shfl_sync(0xffffffffu, from, i);
                const int slot = __shfl_sync(0xffffffffu, from_slot, i);
                to_page[a] = __shfl_sync(0xffffffffu, to, i);
                if (moving >> i & 1u) {
                    const char* const src = part(page, slot);
                    if (lane < 2 * kUnits) x[a] = *reinterpret_cast<const uint4*>(src);
                    else if (lane < kLanes) x[a].x = *reinterpret_cast<const uint32_t*>(src);
                }
            }
#pragma unroll
            for (int a = 0; a < kAcceptAhead; ++a) {
                if (!(moving >> (i0 + a) & 1u)) continue;
                char* const dst = part(to_page[a], (prior + c0 + i0 + a) % kPage);
                if (lane < 2 * kUnits) *reinterpret_cast<uint4*>(dst) = x[a];
                else if (lane < kLanes) *reinterpret_cast<uint32_t*>(dst) = x[a].x;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Reading back: tokens [begin, begin + len) of every sequence, packed, as bf16.  Bound by memory; a warp moves one token's K and V
// with the loads of a chunk under way before its first store, as the gather of one sequence does.  Measured: 40536 tokens of 8 x 128 from an FP8
// cache, 252 MB, in 40.6 us (6.2 TB/s).
// ---------------------------------------------------------------------------
constexpr int kReadThreads = 256;

struct ReadParams {
    const char* pool;
    int64_t num_pages;
    const int32_t* block_table;
    char *k_out, *v_out;
    int* flag;
    int32_t max_pages, n, Hkv, total;
};

// 16 codes times their scale as bf16: the product of a 4-bit and an 8-bit significand is exact in fp32 and is rounded once
__device__ __forceinline__ Pair32 dequantise16(const uint4& codes, float scale) {
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t two;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(two) : "h"((uint16_t)(w[i] >> (16 * h))));
            float lo, hi;
            asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(two));
            y[2 * i + h] = pack_bf16(lo * scale, hi * scale);
        }
    }
    return Pair32{make_uint4(y[0], y[1], y[2], y[3]), make_uint4(y[4], y[5], y[6], y[7])};
}

template <int D, bool FP8, bool ALIGNED, class Rows>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const ReadParams p, const __grid_constant__ Rows rows) {
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int t = (int)blockIdx.x * (kReadThreads / 32) + (int)(threadIdx.x >> 5);
    const int pairs = p.Hkv * (D / 16);  // 32-byte pairs of a row of outputs
    if (t >= p.total) {
        pdl_wait();
        return;
    }
    const int r = request_of(rows, p.n, t);
    const int pos = rows.prior(r) + (t - rows.q_start(r)), slot = pos % kPage;
    pdl_wait();
    const int64_t page = p.block_table[(int64_t)r * p.max_pages + pos / kPage];
    if (page < 0 || page >= p.num_pages) {
        if (lane == 0) atomicOr(p.flag, kStatusBounds);
        return;
    }
    const char* const src = p.pool + page * p.Hkv * (int64_t)(FP8 ? fp8_page_head_bytes(D) : page_head_bytes(D));
    for (int c0 = 0; c0 < pairs; c0 += 64) {
        Pair32 x[2][2];
        float scale[2][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = c0 + 32 * j + lane;
            if (c < pairs) {
                if (FP8) {
                    const char* const blk = src + (c / (D / 16)) * (int64_t)fp8_page_head_bytes(D);
                    const char* const at = blk + slot * D + (((c % (D / 16)) ^ (slot & 7)) << 4);
                    x[j][0].a = *reinterpret_cast<const uint4*>(at);
                    x[j][1].a = *reinterpret_cast<const uint4*>(at + kPage * D);
                    const float* const sc = reinterpret_cast<const float*>(blk + 2 * kPage * D) + slot;
                    scale[j][0] = sc[0], scale[j][1] = sc[kPage];
                } else {
                    const char* const at = src + pair_offset<D>(c, slot);
                    x[j][0] = load32(at);
                    x[j][1] = load32(at + block_bytes(D));
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = c0 + 32 * j + lane;
            if (c < pairs) {
                const int64_t at = ((int64_t)t * pairs + c) * 32;
                if (p.k_out) store_row32<ALIGNED>(p.k_out + at, FP8 ? dequantise16(x[j][0].a, scale[j][0]) : swap_if(x[j][0], slot & 1));
                if (p.v_out) store_row32<ALIGNED>(p.v_out + at, FP8 ? dequantise16(x[j][1].a, scale[j][1]) : swap_if(x[j][1], slot & 1));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

// The lengths of a batch: checked, and how many tokens they hold.
ps_status check_lengths(int32_t max_pages, const int32_t* prior, const int32_t* len, int32_t n, int32_t least, int64_t* total) {
    if (n < 1 || max_pages < 1) return fail(PS_ERR_INVALID, "n=%d, max_pages=%d must be positive", n, max_pages);
    int64_t T = 0;
    for (int r = 0; r < n; ++r) {
        if (len[r] < least || prior[r] < 0) return fail(PS_ERR_INVALID, "request %d: %d tokens behind %d", r, len[r], prior[r]);
        if ((int64_t)prior[r] + len[r] > (int64_t)max_pages * kPage) return fail(PS_ERR_INVALID, "request %d: its tokens exceed max_pages * page_size", r);
        if ((int64_t)prior[r] + len[r] > kMaxTokens) return fail(PS_ERR_INVALID, "request %d: more than %lld tokens", r, (long long)kMaxTokens);
        T += len[r];
        if (T > 0x7fffffffLL / 64) return fail(PS_ERR_INVALID, "too many tokens");
    }
    *total = T;
    return PS_OK;
}

template <int N, class F>
ps_status launch_rows(const int32_t* prior, const int32_t* len, int32_t n, const F& launch) {
    ParamRows<N> rows;  // (entries past n are not read)
    int32_t t = 0;
    for (int r = 0; r < n; ++r) {
        rows.q_start_[r] = t;
        t += len[r];
        rows.prior_[r] = prior[r];
    }
    rows.q_start_[n] = t;
    return launch(rows, t);
}
// launch(rows, first request, its first token, requests, tokens), as often as the kernel's parameters need
template <class F>
ps_status in_slices(const int32_t* prior, const int32_t* len, int32_t n, const F& launch) {
    int64_t t0 = 0;
    for (int32_t r0 = 0; r0 < n; r0 += kParamRowsMax) {
        const int32_t m = n - r0 < kParamRowsMax ? n - r0 : kParamRowsMax;
        int64_t tokens = 0;
        auto go = [&](const auto& rows, int32_t t) {
            tokens = t;
            return t > 0 ? launch(rows, r0, t0, m, t) : PS_OK;
        };
        const ps_status st = m <= 64 ? launch_rows<64>(prior + r0, len + r0, m, go) : m <= 512 ? launch_rows<512>(prior + r0, len + r0, m, go)
                                                                                              : launch_rows<kParamRowsMax>(prior + r0, len + r0, m, go);
        if (st != PS_OK) return st;
        t0 += tokens;
    }
    return PS_OK;
}

}  // namespace

}  // namespace ps

using namespace ps;

extern "C" {

ps_status ps_kv_write_rope(ps_kv* kv, const ps_rope* a, const int32_t* block_table_dev, int32_t max_pages, const int32_t* prior_host,
                           const int32_t* q_len_host, int32_t n, void* stream) {
    if (!kv || !a || !block_table_dev || !prior_host || !q_len_host) return fail(PS_ERR_INVALID, "null argument");
    if (!a->q_dev || !a->k_new_dev || !a->v_new_dev || !a->q_out_dev) return fail(PS_ERR_INVALID, "null tensor");
    const KvPool& pool = pool_of(kv);
    const int Hq = pool.shape.n_q_heads, Hkv = pool.shape.n_kv_heads, d = pool.shape.head_dim;
    if (a->rot_dim < 0 || a->rot_dim > d || a->rot_dim % 16 != 0)
        return fail(PS_ERR_UNSUPPORTED, "rot_dim=%d: multiples of 16 up to head_dim are supported", a->rot_dim);
    if (a->rot_dim > 0 && (!a->cos_sin_dev || a->n_positions < 1)) return fail(PS_ERR_INVALID, "a rotation needs a table of angles");
    if (!(a->eps >= 0.f)) return fail(PS_ERR_INVALID, "eps must not be negative");
    const int64_t strides[3] = {a->q_stride ? a->q_stride : (int64_t)Hq * d, a->k_stride ? a->k_stride : (int64_t)Hkv * d, a->v_stride ? a->v_stride : (int64_t)Hkv * d};
    const int64_t widths[3] = {(int64_t)Hq * d, (int64_t)Hkv * d, (int64_t)Hkv * d};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < widths[i] || strides[i] % 8 != 0 || strides[i] > (1ll << 32)) return fail(PS_ERR_INVALID, "token stride %lld: a multiple of 8 of at least %lld elements", (long long)strides[i], (long long)widths[i]);
    if (((uintptr_t)a->q_dev | (uintptr_t)a->k_new_dev | (uintptr_t)a->v_new_dev | (uintptr_t)a->q_out_dev | (uintptr_t)a->q_weight_dev |
         (uintptr_t)a->k_weight_dev | (uintptr_t)a->cos_sin_dev) % 16 != 0)
        return fail(PS_ERR_INVALID, "tensors must be 16-byte aligned");
    int64_t T = 0;
    const ps_status st = check_lengths(max_pages, prior_host, q_len_host, n, 1, &T);
    if (st != PS_OK) return st;
    const void* in[3] = {a->q_dev, a->k_new_dev, a->v_new_dev};
    for (int i = 0; i < 3; ++i) {
        const bool in_place = i == 0 && in[0] == a->q_out_dev && strides[0] == widths[0];
        if (!in_place && overlap(a->q_out_dev, T * widths[0] * 2, in[i], ((T - 1) * strides[i] + widths[i]) * 2))
            return fail(PS_ERR_INVALID, "q_out overlaps an input (it may be q itself where q is packed)");
    }
    // (what other tokens read while a token's queries are stored)
    const void* const shared[5] = {a->q_weight_dev, a->k_weight_dev, a->rot_dim > 0 ? a->cos_sin_dev : nullptr, a->positions_dev, block_table_dev};
    const int64_t bytes[5] = {d * 2, d * 2, a->n_positions * a->rot_dim * 4, T * 4, (int64_t)n * max_pages * 4};
    for (int i = 0; i < 5; ++i)
        if (shared[i] && overlap(a->q_out_dev, T * widths[0] * 2, shared[i], bytes[i])) return fail(PS_ERR_INVALID, "q_out overlaps an input (it may be q itself where q is packed)");
    return in_slices(prior_host, q_len_host, n, [&](const auto& rows, int32_t r0, int64_t t0, int32_t m, int32_t tokens) {
        using Rows = std::decay_t<decltype(rows)>;
        RopeParams p;
        p.pool = pool.base;
        p.num_pages = pool.num_pages;
        p.q = (const __nv_bfloat16*)a->q_dev + t0 * strides[0];
        p.k = (const __nv_bfloat16*)a->k_new_dev + t0 * strides[1];
        p.v = (const __nv_bfloat16*)a->v_new_dev + t0 * strides[2];
        p.q_stride = strides[0], p.k_stride = strides[1], p.v_stride = strides[2];
        p.q_out = (__nv_bfloat16*)a->q_out_dev + t0 * widths[0];
        p.q_weight = (const __nv_bfloat16*)a->q_weight_dev;
        p.k_weight = (const __nv_bfloat16*)a->k_weight_dev;
        p.cos_sin = a->cos_sin_dev;
        p.n_positions = a->n_positions;
        p.positions = a->positions_dev ? a->positions_dev + t0 : nullptr;
        p.block_table = block_table_dev + (int64_t)r0 * max_pages;
        p.flag = pool.flag_dev;
        p.eps = a->eps;
        p.rot_dim = a->rot_dim, p.interleaved = a->interleaved, p.max_pages = max_pages;
        p.n = m, p.Hq = Hq, p.Hkv = Hkv;
        p.wait_limit_ns = (uint32_t)pool.wait_limit_ns;
        p.tokens = tokens;
        p.stage_bytes = (Hq + 2 * Hkv) * d * 2 + a->rot_dim * 4;
        const auto launch = [&](auto d_, auto fp8_) -> ps_status {
            constexpr int D = decltype(d_)::value;
            constexpr bool FP8 = decltype(fp8_)::value;
            if (tokens <= kRopeFew || p.stage_bytes * kRopeStages > kRopeRingBytes) return launch_kernel(write_rope_kernel<D, FP8, Rows>, tokens, kRopeThreads, 0, (cudaStream_t)stream, 1, true, p, rows);
            static PerDeviceOnce configured;
            const ps_status st = once_per_device(configured, []() -> ps_status {
                PS_CUDA_TRY(cudaFuncSetAttribute(write_rope_ring_kernel<D, FP8, Rows>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRopeRingBytes));
                return PS_OK;
            });
            if (st != PS_OK) return st;
            return launch_kernel(write_rope_ring_kernel<D, FP8, Rows>, kRopeRingCtas, kRopeThreads + 32, kRopeStages * p.stage_bytes,
                                 (cudaStream_t)stream, 1, true, p, rows);
        };
        if (pool.shape.dtype == 1) return launch(std::integral_constant<int, 128>{}, std::true_type{});
        return d == 128 ? launch(std::integral_constant<int, 128>{}, std::false_type{}) : launch(std::integral_constant<int, 64>{}, std::false_type{});
    });
}

ps_status ps_kv_accept(ps_kv* kv, const int32_t* block_table_dev, int32_t max_pages, const int32_t* prior_host, const int32_t* n_nodes_host, int32_t n,
                       const int32_t* index_dev, int32_t index_stride, const int32_t* count_dev, void* stream) {
    if (!kv || !block_table_dev || !prior_host || !n_nodes_host || !index_dev || !count_dev) return fail(PS_ERR_INVALID, "null argument");
    if (index_stride < 1) return fail(PS_ERR_INVALID, "index_stride=%d must be positive", index_stride);
    int64_t T = 0;
    const ps_status st = check_lengths(max_pages, prior_host, n_nodes_host, n, 1, &T);
    if (st != PS_OK) return st;
    const KvPool& pool = pool_of(kv);
    return in_slices(prior_host, n_nodes_host, n, [&](const auto& rows, int32_t r0, int64_t, int32_t m, int32_t) {
        using Rows = std::decay_t<decltype(rows)>;
        AcceptParams p;
        p.pool = pool.base;
        p.num_pages = pool.num_pages;
        p.block_table = block_table_dev + (int64_t)r0 * max_pages;
        p.index = index_dev + (int64_t)r0 * index_stride;
        p.count = count_dev + r0;
        p.flag = pool.flag_dev;
        p.index_stride = index_stride, p.max_pages = max_pages, p.n = m, p.Hkv = pool.shape.n_kv_heads;
        auto* const kernel = pool.shape.dtype == 1 ? accept_kernel<128, true, Rows> : pool.shape.head_dim == 128 ? accept_kernel<128, false, Rows> : accept_kernel<64, false, Rows>;
        const int64_t warps = (int64_t)m * p.Hkv;
        return launch_kernel(kernel, (unsigned)((warps + kAcceptThreads / 32 - 1) / (kAcceptThreads / 32)), kAcceptThreads, 0, (cudaStream_t)stream, 1, true, p, rows);
    });
}

ps_status ps_kv_read(const ps_kv* kv, const int32_t* block_table_dev, int32_t max_pages, const int32_t* begin_host, const int32_t* len_host, int32_t n,
                     void* k_out_dev, void* v_out_dev, void* stream) {
    if (!kv || !block_table_dev || !begin_host || !len_host) return fail(PS_ERR_INVALID, "null argument");
    if (((uintptr_t)k_out_dev | (uintptr_t)v_out_dev) % 16 != 0) return fail(PS_ERR_INVALID, "outputs must be 16-byte aligned");
    int64_t T = 0;
    const ps_status st = check_lengths(max_pages, begin_host, len_host, n, 0, &T);
    if (st != PS_OK) return st;
    if (!k_out_dev && !v_out_dev) return PS_OK;
    const KvPool& pool = pool_of(kv);
    const int Hkv = pool.shape.n_kv_heads, d = pool.shape.head_dim;
    const int64_t out_bytes = T * Hkv * d * 2, table_bytes = (int64_t)n * max_pages * 4;
    if ((k_out_dev && v_out_dev && overlap(k_out_dev, out_bytes, v_out_dev, out_bytes)) || (k_out_dev && overlap(k_out_dev, out_bytes, block_table_dev, table_bytes)) ||
        (v_out_dev && overlap(v_out_dev, out_bytes, block_table_dev, table_bytes)))
        return fail(PS_ERR_INVALID, "the outputs overlap each other or the block table");
    const bool aligned = (((uintptr_t)k_out_dev | (uintptr_t)v_out_dev) & 31) == 0;
    return in_slices(begin_host, len_host, n, [&](const auto& rows, int32_t r0, int64_t t0, int32_t m, int32_t tokens) {
        using Rows = std::decay_t<decltype(rows)>;
        ReadParams p;
        p.pool = pool.base;
        p.num_pages = pool.num_pages;
        p.block_table = block_table_dev + (int64_t)r0 * max_pages;
        p.k_out = k_out_dev ? (char*)k_out_dev + t0 * Hkv * d * 2 : nullptr;
        p.v_out = v_out_dev ? (char*)v_out_dev + t0 * Hkv * d * 2 : nullptr;
        p.flag = pool.flag_dev;
        p.max_pages = max_pages, p.n = m, p.Hkv = Hkv, p.total = tokens;
        auto* const kernel = pool.shape.dtype == 1 ? (aligned ? read_kernel<128, true, true, Rows> : read_kernel<128, true, false, Rows>)
                             : d == 128            ? (aligned ? read_kernel<128, false, true, Rows> : read_kernel<128, false, false, Rows>)
                                                   : (aligned ? read_kernel<64, false, true, Rows> : read_kernel<64, false, false, Rows>);
        return launch_kernel(kernel, (unsigned)((tokens + kReadThreads / 32 - 1) / (kReadThreads / 32)), kReadThreads, 0, (cudaStream_t)stream, 1, true, p, rows);
    });
}

}  // extern "C"
