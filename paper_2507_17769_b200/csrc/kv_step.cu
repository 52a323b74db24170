// The paged cache's side of a speculative step: append with the norms of queries and keys and the position rotation in the
// same pass, moving an accepted path's tokens, and reading stretches of many sequences back as bf16.
#include <type_traits>

#include "kv_rows.cuh"

namespace ps {

namespace {

// ---------------------------------------------------------------------------
// Append with norms and rotation
//
//     y = x / sqrt(mean(x^2) + eps) * w            (q and k heads; where weights are given)
//     (a, b) -> (a cos - b sin, b cos + a sin)     (pairs of the first rot_dim elements)
//
// q goes to its output, k and v to their pages.  Everything between the load and the store is fp32: a key is rounded once, to bf16
// or, in an FP8 cache, to its code.  A CTA has one token: D / 8 lanes hold a head, 16 bytes each, so the norm is a sum over 8 or
// 16 lanes, a rotated pair's other half (half-split pairs) comes by shuffle from the lane rot_dim / 16 away, and a lane's angles are the
// same for every head of the token and are loaded once.
// ---------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeAhead = 3;  // heads of a lane whose loads are under way together

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
    int32_t rot_dim, interleaved, max_pages, n, Hq, Hkv;
};

__device__ __forceinline__ void widen8(const uint4& x, float (&y)[8]) {
    y[0] = bf16_lo(x.x), y[1] = bf16_hi(x.x), y[2] = bf16_lo(x.y), y[3] = bf16_hi(x.y);
    y[4] = bf16_lo(x.z), y[5] = bf16_hi(x.z), y[6] = bf16_lo(x.w), y[7] = bf16_hi(x.w);
}
__device__ __forceinline__ uint4 narrow8(const float (&y)[8]) {
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

template <int D, bool FP8, class Rows>
__global__ void __launch_bounds__(kRopeThreads) write_rope_kernel(const RopeParams p, const __grid_constant__ Rows rows) {
    constexpr int L = D / 8;                      // lanes of a head
    constexpr int kGroups = kRopeThreads / L;
    pdl_trigger();
    const int t = blockIdx.x, lane = threadIdx.x & 31, l = threadIdx.x % L, group = threadIdx.x / L;
    const int r = request_of(rows, p.n, t);
    const int pos = rows.prior(r) + (t - rows.q_start(r)), slot = pos % kPage;
    pdl_wait();
    const int64_t page = p.block_table[(int64_t)r * p.max_pages + pos / kPage];
    const int64_t angle = p.positions ? p.positions[t] : pos;
    if (page < 0 || page >= p.num_pages || (p.rot_dim > 0 && (angle < 0 || angle >= p.n_positions))) {
        if (threadIdx.x == 0) atomicOr(p.flag, kStatusBounds);
        return;
    }
    const int half = p.rot_dim >> 1, e0 = 8 * l;
    const bool turns = e0 < p.rot_dim;
    // lane of the same head that holds the other elements of this lane's pairs, and the sign of their part
    const int other = !turns || p.interleaved ? l : e0 < half ? l + half / 8 : l - half / 8;
    const int other_lane = lane - l + other;
    float cosv[8], sinv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cosv[i] = 1.f, sinv[i] = 0.f;
    if (turns) {
        const float* const row = p.cos_sin + angle * p.rot_dim + (p.interleaved ? e0 / 2 : e0 < half ? e0 : e0 - half);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            if (!p.interleaved || i == 0) {
                const float4 c = *reinterpret_cast<const float4*>(row + i), s = *reinterpret_cast<const float4*>(row + half + i);
                cosv[i] = c.x, cosv[i + 1] = c.y, cosv[i + 2] = c.z, cosv[i + 3] = c.w;
                sinv[i] = s.x, sinv[i + 1] = s.y, sinv[i + 2] = s.z, sinv[i + 3] = s.w;
            }
        }
        if (!p.interleaved && e0 < half) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sinv[i] = -sinv[i];
        }
    }
    const int n_vec = p.Hq + 2 * p.Hkv;
    for (int v0 = group; v0 - group < n_vec; v0 += kGroups * kRopeAhead) {  // (the warp's lanes stay together: they shuffle)
        uint4 raw[kRopeAhead];
#pragma unroll
        for (int a = 0; a < kRopeAhead; ++a) {
            const int vec = v0 + a * kGroups;
            raw[a] = make_uint4(0, 0, 0, 0);
            if (vec < n_vec) {
                const __nv_bfloat16* src = vec < p.Hq          ? p.q + (int64_t)t * p.q_stride + vec * D
                                           : vec < p.Hq + p.Hkv ? p.k + (int64_t)t * p.k_stride + (vec - p.Hq) * D
                                                                : p.v + (int64_t)t * p.v_stride + (vec - p.Hq - p.Hkv) * D;
                raw[a] = *reinterpret_cast<const uint4*>(src + e0);
            }
        }
#pragma unroll
        for (int a = 0; a < kRopeAhead; ++a) {
            const int vec = v0 + a * kGroups;
            if (vec - group >= n_vec) break;  // (the same for the whole warp)
            const bool is_q = vec < p.Hq, is_v = vec >= p.Hq + p.Hkv;
            float x[8];
            widen8(raw[a], x);
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
            for (int o = L / 2; o >= 1; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            uint4 raw_other;
            raw_other.x = __shfl_sync(0xffffffffu, raw[a].x, other_lane);
            raw_other.y = __shfl_sync(0xffffffffu, raw[a].y, other_lane);
            raw_other.z = __shfl_sync(0xffffffffu, raw[a].z, other_lane);
            raw_other.w = __shfl_sync(0xffffffffu, raw[a].w, other_lane);
            float y[8];
            widen8(raw_other, y);
            const __nv_bfloat16* const weight = is_q ? p.q_weight : p.k_weight;
            if (!is_v) {
                if (weight) {
                    const float rstd = rsqrtf(ss * (1.f / D) + p.eps);
                    float w[8], wo[8];
                    widen8(__ldg(reinterpret_cast<const uint4*>(weight + e0)), w);
                    widen8(__ldg(reinterpret_cast<const uint4*>(weight + 8 * other)), wo);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] *= rstd * w[i], y[i] *= rstd * wo[i];
                }
                if (turns) {
                    if (p.interleaved) {
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float c = cosv[i >> 1], s = sinv[i >> 1], b = x[i + 1];
                            x[i + 1] = fmaf(b, c, x[i] * s);
                            x[i] = fmaf(x[i], c, -(b * s));
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], cosv[i], y[i] * sinv[i]);
                    }
                }
            }
            float scale = 1.f;
            if (FP8) {
                float amax = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
                for (int o = L / 2; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                scale = fp8_scale(amax);
            }
            if (vec >= n_vec) continue;
            if (is_q) {
                *reinterpret_cast<uint4*>(p.q_out + ((int64_t)t * p.Hq + vec) * D + e0) = narrow8(x);
            } else {
                const int g = vec - p.Hq - (is_v ? p.Hkv : 0);
                if (FP8) {
                    char* const blk = p.pool + (page * p.Hkv + g) * (int64_t)fp8_page_head_bytes(D);
                    *reinterpret_cast<uint2*>(blk + (is_v ? kPage * D : 0) + slot * D + (((l >> 1) ^ (slot & 7)) << 4) + 8 * (l & 1)) =
                        make_uint2(quantise4(x[0], x[1], x[2], x[3], scale), quantise4(x[4], x[5], x[6], x[7], scale));
                    if (l == 0) reinterpret_cast<float*>(blk + 2 * kPage * D)[(is_v ? kPage : 0) + slot] = scale;
                } else {
                    char* const blk = p.pool + (page * p.Hkv + g) * (int64_t)page_head_bytes(D) + (is_v ? block_bytes(D) : 0);
                    *reinterpret_cast<uint4*>(blk + unit_offset(slot, e0)) = narrow8(x);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Accepted paths: slot prior + i of the sequence receives token prior + index[i], i < count, for an increasing path.
//
// A warp has one (request, kv head), a lane one 16-byte unit of K or V (and, FP8, a scale), the same unit of every token, so what a lane
// reads no other lane writes.  It reads a group of tokens before it stores any of them, and what it has stored
// lies below every later source: index[i] >= i.
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
    bool good = count >= 0 && count <= nodes && count <= p.index_stride;
    if (good) {
        for (int i = lane; i < count; i += 32) {
            const int at = index[i];
            good = good && at >= i && at < nodes && (i == 0 || at > index[i - 1]);
        }
    }
    if (!__all_sync(0xffffffffu, good)) {
        if (lane == 0) atomicOr(p.flag, kStatusBounds);
        return;
    }
    const int32_t* const table = p.block_table + (int64_t)r * p.max_pages;
    const int64_t head_bytes = FP8 ? fp8_page_head_bytes(D) : page_head_bytes(D);
    auto place = [&](int node) -> char* {  // of this lane's part of a token; null: no such page
        const int pos = prior + node, slot = pos % kPage;
        const int64_t page = table[pos / kPage];
        if (page < 0 || page >= p.num_pages) return nullptr;
        char* const blk = p.pool + (page * p.Hkv + g) * head_bytes;
        if (FP8) {
            if (lane >= 2 * kUnits) return blk + 2 * kPage * D + ((lane - 2 * kUnits) * kPage + slot) * 4;
            return blk + (lane / kUnits) * (kPage * D) + slot * D + (((lane % kUnits) ^ (slot & 7)) << 4);
        }
        return blk + (lane / kUnits) * block_bytes(D) + unit_offset(slot, 8 * (lane % kUnits));
    };
    for (int i0 = 0; i0 < count; i0 += kAcceptAhead) {
        uint4 x[kAcceptAhead];
        char* dst[kAcceptAhead];
#pragma unroll
        for (int a = 0; a < kAcceptAhead; ++a) {
            const int i = i0 + a;
            dst[a] = nullptr;
            if (i < count) {
                const int at = index[i];
                if (at == i) continue;  // it is there already
                const char* const src = place(at);
                dst[a] = place(i);
                if (!src || !dst[a]) {
                    if (lane == 0) atomicOr(p.flag, kStatusBounds);
                    dst[a] = nullptr;
                } else if (lane < 2 * kUnits) {
                    x[a] = *reinterpret_cast<const uint4*>(src);
                } else if (lane < kLanes) {
                    x[a].x = *reinterpret_cast<const uint32_t*>(src);
                }
            }
        }
#pragma unroll
        for (int a = 0; a < kAcceptAhead; ++a) {
            if (!dst[a]) continue;
            if (lane < 2 * kUnits) *reinterpret_cast<uint4*>(dst[a]) = x[a];
            else if (lane < kLanes) *reinterpret_cast<uint32_t*>(dst[a]) = x[a].x;
        }
    }
}

// ---------------------------------------------------------------------------
// Reading back: tokens [begin, begin + len) of every sequence, packed, as bf16.  Bound by memory; a warp moves one token's K and V
// with the loads of a chunk under way before its first store, as the gather of one sequence does.
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

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    return (uintptr_t)a < (uintptr_t)b + (uintptr_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uintptr_t)a_bytes;
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
        auto* const kernel = pool.shape.dtype == 1 ? write_rope_kernel<128, true, Rows> : d == 128 ? write_rope_kernel<128, false, Rows> : write_rope_kernel<64, false, Rows>;
        return launch_kernel(kernel, tokens, kRopeThreads, 0, (cudaStream_t)stream, 1, true, p, rows);
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
