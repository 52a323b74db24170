// What the kernels that move tokens in and out of the paged cache share: the lengths of a batch as a kernel parameter, rows of
// a token in 32-byte pairs, and the FP8 quantiser.
#pragma once

#include "common.cuh"

namespace ps {

// Where the new tokens go: request r's are packed tokens q_start[r] .. q_start[r + 1] and follow prior[r] cached ones.  The
// lengths travel as a kernel parameter: copied to the device first they cost every append a small transfer that its stream
// has to wait for (about 6 us between two kernels, and 4 us of host time).  Batches of more than kParamRowsMax requests
// still take that way.
template <int N>
struct ParamRows {
    int32_t q_start_[N + 1], prior_[N];
    __device__ __forceinline__ int q_start(int r) const { return q_start_[r]; }
    __device__ __forceinline__ int prior(int r) const { return prior_[r]; }
};
struct DeviceRows {
    const int32_t *q_start_, *prior_;
    __device__ __forceinline__ int q_start(int r) const { return q_start_[r]; }
    __device__ __forceinline__ int prior(int r) const { return prior_[r]; }
};
constexpr int kParamRowsMax = 4000;  // 32 KB, as much as a kernel's parameters may be

// request of packed token t: last r with q_start(r) <= t (requests without tokens are passed over)
template <class Rows>
__device__ __forceinline__ int request_of(const Rows& rows, int n, int t) {
    // (up to the first request of several tokens, which in a serving batch come last, every request has one)
    if (t < n && rows.q_start(t) == t && rows.q_start(t + 1) > t) return t;
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (rows.q_start(mid) <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

struct Pair32 {
    uint4 a, b;
};
__device__ __forceinline__ Pair32 load32(const void* p) {
    Pair32 x;
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x.a.x), "=r"(x.a.y), "=r"(x.a.z), "=r"(x.a.w), "=r"(x.b.x), "=r"(x.b.y), "=r"(x.b.z), "=r"(x.b.w)
                 : "l"(p));
    return x;
}
__device__ __forceinline__ void store32(void* p, const Pair32& x) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x.a.x), "r"(x.a.y), "r"(x.a.z), "r"(x.a.w),
                 "r"(x.b.x), "r"(x.b.y), "r"(x.b.z), "r"(x.b.w)
                 : "memory");
}
// a token's row: 32-byte aligned where the caller's tensor is (ALIGNED), else 16
template <bool ALIGNED>
__device__ __forceinline__ Pair32 load_row32(const char* p) {
    if (ALIGNED) return load32(p);
    return Pair32{reinterpret_cast<const uint4*>(p)[0], reinterpret_cast<const uint4*>(p)[1]};
}
template <bool ALIGNED>
__device__ __forceinline__ void store_row32(char* p, const Pair32& x) {
    if (ALIGNED) {
        store32(p, x);
    } else {
        reinterpret_cast<uint4*>(p)[0] = x.a;
        reinterpret_cast<uint4*>(p)[1] = x.b;
    }
}
__device__ __forceinline__ Pair32 swap_if(const Pair32& x, bool odd) { return odd ? Pair32{x.b, x.a} : x; }
// 32-byte pair c of a token's row -> offset of its (page, kv head)'s pair in the K block, from the page's start
template <int D>
__device__ __forceinline__ uint32_t pair_offset(int c, int slot) {
    constexpr int kPairs = D / 16;
    return (uint32_t)(c / kPairs) * (uint32_t)page_head_bytes(D) + (unit_offset(slot, (c % kPairs) * 16) & ~16u);
}

// amax / 448 rounded up to 8 significant bits, 1 for a zero vector
__device__ __forceinline__ float fp8_scale(float amax) {
    uint32_t bits = __float_as_uint(amax > 0.f ? __fdiv_rn(amax, 448.f) : 1.f);
    if (bits & 0xffffu) bits = (bits | 0xffffu) + 1u;
    return __uint_as_float(bits);
}
__device__ __forceinline__ uint32_t quantise4(float x0, float x1, float x2, float x3, float scale) {
    uint16_t lo, hi;  // cvt packs its first operand into the upper byte
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fdiv_rn(x1, scale)), "f"(__fdiv_rn(x0, scale)));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fdiv_rn(x3, scale)), "f"(__fdiv_rn(x2, scale)));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}

}  // namespace ps
