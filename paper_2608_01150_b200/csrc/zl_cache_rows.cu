// Rows into the paged cache and out of it (sm_100a): one pass over the data, bound by the bytes that it moves.
//
// A row (token, key head) of 64 or 128 elements belongs to four or eight lanes, sixteen elements each, keys and values together:
// the largest magnitude of a row is two or three shuffles away.  A lane has eight neighbours in either half of the row, so that
// every access of a warp covers whole sectors of 32 bytes (with its sixteen side by side, half sectors were stored: reading
// 37,920 tokens, 12 heads, d 128, from 8 bits took 71 us, now 56).  Where the row lies in the cache follows from the batch: a
// binary search in cu_q (or cu_kv), whose few entries stay in L1, and one entry of the page table.  When writing, the rows' own
// loads run ahead of that search.  Blocks of four warps: registers leave room for 36 warps that write, for 32 in blocks of eight
// (56 -> 52 us for 32,760 tokens); of two, the number of blocks becomes the limit (54).
// Measured, 12 heads, d 128: 32,760 tokens written in int8 51 us (6.0 TB/s; 56 in a run of seconds), in e4m3 50 (55), in bf16 63
// (6.4 TB/s); 37,920 tokens read from either 56 us (6.3 TB/s), from bf16 72 (6.5).
#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr int kThreads = 128;
constexpr int kEach = 16;  // elements of a lane
template <int D>
__device__ __forceinline__ uint32_t my_row() {
    return blockIdx.x * (kThreads / (D / kEach)) + threadIdx.x / (D / kEach);
}

__device__ __forceinline__ float lo_float(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_float(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Codes of sixteen elements, and the row's scale.  scale = largest magnitude / T and code = x / scale, both quotients rounded to
// fp32, then one rounding to the code's type (ties to even): a value read back is off by half a step of its code.
// Multiplying by a reciprocal instead would move values that lie between two codes.  Where nothing leaves the range of normal
// numbers, the quotient comes from the correctly rounded reciprocal y by Markstein's correction (IBM J. Res. Dev. 34, 1990):
// with q within a unit of x / s, the remainder x - q s is exact and q + (x - q s) y rounds to the rounded quotient.  q = x y is not
// always that near (6,987 of the 598,208 quotients of a bf16 number by a scale of bf16 numbers that can reach a code; the remainder is
// rounded in 841): that the result is the rounded quotient there too was found by going through all of them.  Three operations for two
// elements instead of a division's dozen for one, which were what bound this kernel (32,760 tokens, 12 heads, d 128, int8,
// written and read back: 161 -> 122 us).
template <int kFormat, int kLanes>
__device__ __forceinline__ uint4 quantise(const uint4 (&u)[2], float& scale) {
    constexpr float kTop = kFormat == ZL_CACHE_INT8 ? 127.f : 448.f;
    const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) big = max3_abs(big, lo_float(w[i]), hi_float(w[i]));
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
    scale = __fdiv_rn(big, kTop);
    uint32_t r[4] = {0, 0, 0, 0};
    if (scale >= 0x1p-80f && scale <= 0x1p80f) {
        const float y = __frcp_rn(scale);
        const float2 y2 = make_float2(y, y), less = make_float2(-scale, -scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2 q[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 x = make_float2(lo_float(w[2 * i + e]), hi_float(w[2 * i + e])), q0 = mul2(x, y2);
                q[e] = fma2(fma2(q0, less, x), y2, q0);
            }
            if constexpr (kFormat == ZL_CACHE_INT8) {
                // behind 1.5 * 2^23 a number ends in whole ones, two's complement: its low byte is the code
                uint32_t c[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float2 z = add2(q[e], make_float2(12582912.f, 12582912.f));
                    c[e] = __byte_perm(__float_as_uint(z.x), __float_as_uint(z.y), 0x0040);
                }
                r[i] = __byte_perm(c[0], c[1], 0x5410);
            } else {
                r[i] = (uint32_t)__nv_cvt_float2_to_fp8x2(q[0], __NV_SATFINITE, __NV_E4M3) |
                       ((uint32_t)__nv_cvt_float2_to_fp8x2(q[1], __NV_SATFINITE, __NV_E4M3) << 16);
            }
        }
    } else if (scale > 0.f) {  // (a row of zeros, or so small that its scale vanishes, has the codes of zero)
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            uint32_t v = w[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) v = i == e ? w[e] : v;
            const float a = fminf(fmaxf(__fdiv_rn(lo_float(v), scale), -kTop), kTop);
            const float b = fminf(fmaxf(__fdiv_rn(hi_float(v), scale), -kTop), kTop);
            uint32_t pair;
            if constexpr (kFormat == ZL_CACHE_INT8)
                pair = ((uint32_t)__float2int_rn(a) & 0xffu) | (((uint32_t)__float2int_rn(b) & 0xffu) << 8);
            else
                pair = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i >> 1 == e) r[e] |= pair << (16 * (i & 1));
        }
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads)
zl_cache_write_kernel(const CacheView c, const CacheBatch b, const __nv_bfloat16* k, const __nv_bfloat16* v, const int64_t row_stride) {
    constexpr int kLanes = D / kEach;
    grid_release();
    grid_wait();
    const uint32_t r = my_row<D>();
    const uint32_t token = r / (uint32_t)c.n_kv_heads, head = r - token * (uint32_t)c.n_kv_heads;
    const int lane = threadIdx.x % kLanes;
    uint4 xk[2], xv[2];
    xk[0] = xk[1] = xv[0] = xv[1] = make_uint4(0, 0, 0, 0);
    int64_t slot = -1;  // byte offset of the row in the cache
    int64_t at_scale = 0;
    if (token < (uint32_t)b.total_q) {
        const int64_t src = (int64_t)token * row_stride + (int64_t)head * D + lane * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            xk[i] = __ldg(reinterpret_cast<const uint4*>(k + src + i * (D / 2)));
            xv[i] = __ldg(reinterpret_cast<const uint4*>(v + src + i * (D / 2)));
        }
        const int s = find_seq(b.cu_q, b.n_seqs, (int32_t)token);
        if (s >= 0) {
            const SeqView sv = load_seq(b, c.page_shift, s);
            const int32_t i = (int32_t)token - sv.q0, pos = sv.pos0 + i;
            if (i >= 0 && i < sv.q_len && pos >= 0 && pos < sv.keys) {
                const int32_t pg = page_at(b, c, s, pos), in = pos & ((1 << c.page_shift) - 1);
                if (pg >= 0) {
                    slot = pg * c.page_stride + in * c.token_stride + head * c.head_stride;
                    at_scale = pg * c.scale_page + in * c.scale_token + head * c.scale_head;
                }
            }
        }
    }
    const bool live = slot >= 0;
    if constexpr (kFormat == ZL_CACHE_BF16) {
        if (live) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<uint4*>(c.k + slot + i * D + lane * 16) = xk[i];
                *reinterpret_cast<uint4*>(c.v + slot + i * D + lane * 16) = xv[i];
            }
        }
    } else {
        float sk, sv;
        const uint4 ck = quantise<kFormat, kLanes>(xk, sk), cv = quantise<kFormat, kLanes>(xv, sv);
        if (live) {
            *reinterpret_cast<uint2*>(c.k + slot + lane * 8) = make_uint2(ck.x, ck.y);
            *reinterpret_cast<uint2*>(c.k + slot + D / 2 + lane * 8) = make_uint2(ck.z, ck.w);
            *reinterpret_cast<uint2*>(c.v + slot + lane * 8) = make_uint2(cv.x, cv.y);
            *reinterpret_cast<uint2*>(c.v + slot + D / 2 + lane * 8) = make_uint2(cv.z, cv.w);
            if (lane == 0) c.k_scale[at_scale] = sk;
            if (lane == 1) c.v_scale[at_scale] = sv;
        }
    }
}

template <int kFormat>
__device__ __forceinline__ uint4 dequantise(uint32_t a, uint32_t b, float scale) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? a : b;
        float2 x;
        if constexpr (kFormat == ZL_CACHE_INT8) {
            // 0x4b0000 in front of c + 128 is 2^23 + 128 + c
            const uint32_t up = w ^ 0x80808080u;
            const uint32_t lo = __byte_perm(up, 0x4b000000u, 0x7650 + 2 * (i & 1)), hi = __byte_perm(up, 0x4b000000u, 0x7651 + 2 * (i & 1));
            x = add2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), make_float2(-8388736.f, -8388736.f));
        } else {
            uint32_t p[2];
            e4m3_half(w, p[0], p[1]);
            x = __half22float2(*reinterpret_cast<const __half2*>(&p[i & 1]));
        }
        x = mul2(x, make_float2(scale, scale));
        r[i] = pack_bf16(x.x, x.y);  // (the product is rounded to fp32, and that to bf16)
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads)
zl_cache_read_kernel(const CacheView c, const CacheBatch b, const CacheReadParams p) {
    constexpr int kLanes = D / kEach;
    grid_release();
    grid_wait();
    const uint32_t r = my_row<D>();
    const uint32_t row = r / (uint32_t)c.n_kv_heads, head = r - row * (uint32_t)c.n_kv_heads;
    const int lane = threadIdx.x % kLanes;
    if (row >= (uint32_t)p.total_kv) return;
    const int s = find_seq(p.cu_kv, b.n_seqs, (int32_t)row);
    if (s < 0) return;
    uint4 xk[2], xv[2];
    xk[0] = xk[1] = xv[0] = xv[1] = make_uint4(0, 0, 0, 0);
    const int64_t pos = (int64_t)(p.first ? __ldg(p.first + s) : 0) + ((int32_t)row - __ldg(p.cu_kv + s));
    if (pos >= 0 && pos < load_seq(b, c.page_shift, s).keys) {
        const int32_t pg = page_at(b, c, s, (int32_t)pos), in = (int32_t)pos & ((1 << c.page_shift) - 1);
        if (pg >= 0) {
            const int64_t slot = pg * c.page_stride + in * c.token_stride + head * c.head_stride;
            if constexpr (kFormat == ZL_CACHE_BF16) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xk[i] = *reinterpret_cast<const uint4*>(c.k + slot + i * D + lane * 16);
                    xv[i] = *reinterpret_cast<const uint4*>(c.v + slot + i * D + lane * 16);
                }
            } else {
                const int64_t at = pg * c.scale_page + in * c.scale_token + head * c.scale_head;
                uint2 ck[2], cv[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    ck[i] = *reinterpret_cast<const uint2*>(c.k + slot + i * (D / 2) + lane * 8);
                    cv[i] = *reinterpret_cast<const uint2*>(c.v + slot + i * (D / 2) + lane * 8);
                }
                const float sk = c.k_scale[at], sv = c.v_scale[at];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xk[i] = dequantise<kFormat>(ck[i].x, ck[i].y, sk);
                    xv[i] = dequantise<kFormat>(cv[i].x, cv[i].y, sv);
                }
            }
        }
    }
    const int64_t dst = ((int64_t)row * c.n_kv_heads + head) * D + lane * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        *reinterpret_cast<uint4*>(p.k + dst + i * (D / 2)) = xk[i];
        *reinterpret_cast<uint4*>(p.v + dst + i * (D / 2)) = xv[i];
    }
}

int blocks(int64_t rows, int head_dim) {
    const int per = kThreads / (head_dim / kEach);
    return (int)((rows + per - 1) / per);
}

}  // namespace

cudaError_t launch_cache_write(int head_dim, int format, const CacheView& c, const CacheBatch& b, const __nv_bfloat16* k,
                               const __nv_bfloat16* v, int64_t row_stride, cudaStream_t stream) {
    const int grid = blocks((int64_t)b.total_q * c.n_kv_heads, head_dim);
    auto go = [&](auto kernel) { return launch_dependent(kernel, grid, kThreads, 0, stream, true, c, b, k, v, row_stride); };
    if (head_dim == 128) {
        if (format == ZL_CACHE_BF16) return go(zl_cache_write_kernel<128, ZL_CACHE_BF16>);
        return format == ZL_CACHE_INT8 ? go(zl_cache_write_kernel<128, ZL_CACHE_INT8>) : go(zl_cache_write_kernel<128, ZL_CACHE_E4M3>);
    }
    if (format == ZL_CACHE_BF16) return go(zl_cache_write_kernel<64, ZL_CACHE_BF16>);
    return format == ZL_CACHE_INT8 ? go(zl_cache_write_kernel<64, ZL_CACHE_INT8>) : go(zl_cache_write_kernel<64, ZL_CACHE_E4M3>);
}

cudaError_t launch_cache_read(int head_dim, int format, const CacheView& c, const CacheBatch& b, const CacheReadParams& p,
                              cudaStream_t stream) {
    const int grid = blocks((int64_t)p.total_kv * c.n_kv_heads, head_dim);
    auto go = [&](auto kernel) { return launch_dependent(kernel, grid, kThreads, 0, stream, true, c, b, p); };
    if (head_dim == 128) {
        if (format == ZL_CACHE_BF16) return go(zl_cache_read_kernel<128, ZL_CACHE_BF16>);
        return format == ZL_CACHE_INT8 ? go(zl_cache_read_kernel<128, ZL_CACHE_INT8>) : go(zl_cache_read_kernel<128, ZL_CACHE_E4M3>);
    }
    if (format == ZL_CACHE_BF16) return go(zl_cache_read_kernel<64, ZL_CACHE_BF16>);
    return format == ZL_CACHE_INT8 ? go(zl_cache_read_kernel<64, ZL_CACHE_INT8>) : go(zl_cache_read_kernel<64, ZL_CACHE_E4M3>);
}

}  // namespace zl
