// The paged key/value cache and a batch over it, as the cache's kernels read them.
#pragma once

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

// The sequence whose range [cu[s], cu[s + 1]) holds a row, -1 for none.
__device__ __forceinline__ int find_seq(const int32_t* cu, int n, int32_t row) {
    int lo = 0, hi = n;  // the last s with cu[s] <= row
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(cu + mid + 1) <= row) lo = mid + 1; else hi = mid;
    }
    return lo < n && __ldg(cu + lo) <= row ? lo : -1;
}

// ------------------------------------------------------------------------------------------------ 8-bit codes
// Two whole numbers in bytes I and J of `w` as a bf16 pair, exactly: 0x43 in front of the low seven bits is 128 + low bits
// (one unit in the last place is 1 there), and 128, or 256 for a negative number, is taken off again.
template <int I, int J>
__device__ __forceinline__ uint32_t int8_pair(uint32_t w) {
    const uint32_t x = __byte_perm(w, 0x43434343u, 0x4040u | (J << 8) | I);
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x & 0xff7fff7fu), "r"(x & 0xff80ff80u));
    return r;
}
// Two e4m3 numbers as a bf16 pair, exactly: sign, exponent and fraction moved to their places give the number times
// 2^-120, subnormal ones included, and a product with 2^120 puts the exponent right.
template <int I, int J>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w) {
    const uint32_t x = __byte_perm(w, 0u, 0x0404u | (J << 12) | (I << 4));
    return mul_bf16x2(((x >> 4) & 0x07f007f0u) | (x & 0x80008000u), 0x7b807b80u);
}
template <int kFormat, int I, int J>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    return kFormat == ZL_CACHE_INT8 ? int8_pair<I, J>(w) : e4m3_pair<I, J>(w);
}

}  // namespace cache
}  // namespace zl
