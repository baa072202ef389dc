// The paged key/value cache and a batch over it, as the cache's kernels read them.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "zl_device.h"
#include "zl_ptx.cuh"

namespace zl {
namespace cache {

using namespace ptx;

// Everything a caller put into device memory is taken as it comes: ranges are cut to the tensors they index, a page number
// outside the cache is a page without keys.
struct SeqView {
    int32_t q0, q_len;  // rows of Q
    int32_t pos0;       // position of the first of them (negative: the sequence is shorter than its new rows)
    int32_t keys;       // keys that the page table can hold of it
    int32_t prefix;     // keys that every row sees
};

__device__ __forceinline__ SeqView load_seq(const CacheBatch& b, int page_shift, int s) {
    SeqView v;
    const int32_t total = b.total_q;
    v.q0 = min(max(__ldg(b.cu_q + s), 0), total);
    const int32_t q1 = min(max(__ldg(b.cu_q + s + 1), v.q0), total);
    v.q_len = q1 - v.q0;
    const int32_t len = max(__ldg(b.kv_len + s), 0);
    v.pos0 = len - v.q_len;
    v.keys = (int32_t)min((int64_t)len, (int64_t)b.max_pages << page_shift);
    v.prefix = b.prefix ? __ldg(b.prefix + s) : 0;
    return v;
}

// Keys [0, result) are seen by row i of the sequence.
__device__ __forceinline__ int32_t keys_seen(const SeqView& v, int32_t i) {
    return max(0, min(v.keys, max(v.pos0 + i + 1, v.prefix)));
}

// Page of a position (0 <= pos < keys), -1 for none.
__device__ __forceinline__ int32_t page_at(const CacheBatch& b, const CacheView& c, int s, int32_t pos) {
    const int32_t pg = __ldg(b.pages + (int64_t)s * b.max_pages + (pos >> c.page_shift));
    return (uint32_t)pg < (uint32_t)c.n_pages ? pg : -1;
}

// The same in two halves, for code that looks ahead: the entry of the table, whose use would wait for it, and what it means.
__device__ __forceinline__ int32_t page_entry(const CacheBatch& b, const CacheView& c, int s, int32_t pos) {
    return __ldg(b.pages + (int64_t)s * b.max_pages + (pos >> c.page_shift));
}
__device__ __forceinline__ int32_t valid_page(const CacheView& c, int32_t entry) {
    return (uint32_t)entry < (uint32_t)c.n_pages ? entry : -1;
}

// The sequence whose range [cu[s], cu[s + 1]) holds a row, -1 for none.
__device__ __forceinline__ int find_seq(const int32_t* cu, int n, int32_t row) {
    int lo = 0, hi = n;  // the last s with cu[s] <= row
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(cu + mid + 1) <= row) lo = mid + 1; else hi = mid;
    }
    return lo < n && __ldg(cu + lo) <= row ? lo : -1;
}

// a / b for numbers, not negative, that nearly always fit 32 bits.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// ------------------------------------------------------------------------------------------------ 8-bit codes
// Attention over 8-bit caches multiplies in fp16, which holds every code exactly and is reached in a third of the
// instructions: a whole number c goes through 0x64 in front of c + 128 (1152 + c, in steps of one), e4m3 through a conversion
// of its own (whose NaN codes stay NaN).  Four codes of a word, in pairs (0, 1), (2, 3) or (0, 2), (1, 3).
__device__ __forceinline__ uint32_t int8_half(uint32_t shifted, uint32_t sel) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(__byte_perm(shifted, 0x64646464u, sel)), "r"(0x64806480u));
    return r;
}
__device__ __forceinline__ void e4m3_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
}
template <int kFormat>
__device__ __forceinline__ void halves(uint32_t w, uint32_t& p01, uint32_t& p23) {
    if constexpr (kFormat == ZL_CACHE_INT8) {
        w ^= 0x80808080u;
        p01 = int8_half(w, 0x4140);
        p23 = int8_half(w, 0x4342);
    } else {
        e4m3_half(w, p01, p23);
    }
}
template <int kFormat>
__device__ __forceinline__ void halves_apart(uint32_t w, uint32_t& p02, uint32_t& p13) {
    if constexpr (kFormat == ZL_CACHE_INT8) {
        w ^= 0x80808080u;
        p02 = int8_half(w, 0x4240);
        p13 = int8_half(w, 0x4341);
    } else {
        e4m3_half(__byte_perm(w, 0u, 0x3120), p02, p13);
    }
}
// Queries, bf16, as fp16: times the power of two that brings the largest magnitude `big` to 2^14 .. 2^15 (below 2^-98: times 2^112).
// What is 2^-31 of it or more keeps its 8 bits above fp16's last step of 2^-24; the rest is off by half that step, 2^-39 of
// `big`.  `back`: the factor that undoes it.
__device__ __forceinline__ float half_factor(float big, float& back) {
    const int e = big > 0.f ? min(max((int)(__float_as_uint(big) >> 23) - 127 - 14, -112), 113) : 0;
    back = __uint_as_float((uint32_t)(127 + e) << 23);
    return __uint_as_float((uint32_t)(127 - e) << 23);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t bf16_pair_to_half(uint32_t w, float factor) {
    return pack_half(__uint_as_float(w << 16) * factor, __uint_as_float(w & 0xffff0000u) * factor);
}
// The weight of a value is its p times its scale.  Weights are held relative to a reference that follows the largest of
// THEM (not of the scores), so that fp16 gives a weight 11 bits down to 2^-14 of that reference and 2^-25 of it below,
// whatever the scales of other values are; the row's sum of p is kept relative to the same reference in fp32.  Scales below 2^-90
// count as 2^-90, which keeps the sum in range.
constexpr float kLeastScale = 0x1p-90f;

}  // namespace cache
}  // namespace zl
