// Rows into the paged cache and out of it (sm_100a): one pass over the data, bound by the bytes that it moves.
//
// A row (token, key head) of 64 or 128 elements belongs to eight or sixteen lanes, eight elements (16 bytes of bf16) each,
// keys and values together, so that a warp's loads and stores cover whole rows and the largest magnitude of a row is three
// or four shuffles away.  Where the row lies in the cache follows from the batch: a binary search in cu_q (or cu_kv), whose
// few entries stay in L1, and one entry of the page table.
#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr int kThreads = 256;

struct Row {
    int32_t token, head;
};
template <int D>
__device__ __forceinline__ uint32_t my_row() {
    return blockIdx.x * (kThreads / (D / 8)) + threadIdx.x / (D / 8);
}

__device__ __forceinline__ void unpack(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// Codes of eight elements, and the row's scale.  scale = largest magnitude / T and code = x / scale, both quotients rounded to
// fp32, then one rounding to the code's type (ties to even): a value read back is off by half a step of its code.
// Multiplying by a reciprocal instead would move values that lie between two codes.
template <int kFormat, int kLanes>
__device__ __forceinline__ uint2 quantise(const uint4& u, float& scale) {
    constexpr float kTop = kFormat == ZL_CACHE_INT8 ? 127.f : 448.f;
    float x[8], big = 0.f;
    unpack(u, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(x[i]));
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
    scale = __fdiv_rn(big, kTop);
    uint32_t r[2] = {0, 0};
    if (scale > 0.f) {  // (a row of zeros, or so small that its scale vanishes, has the codes of zero)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = fminf(fmaxf(__fdiv_rn(x[2 * i], scale), -kTop), kTop);
            const float b = fminf(fmaxf(__fdiv_rn(x[2 * i + 1], scale), -kTop), kTop);
            uint32_t pair;
            if constexpr (kFormat == ZL_CACHE_INT8)
                pair = ((uint32_t)__float2int_rn(a) & 0xffu) | (((uint32_t)__float2int_rn(b) & 0xffu) << 8);
            else
                pair = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
            r[i >> 1] |= pair << (16 * (i & 1));
        }
    }
    return make_uint2(r[0], r[1]);
}

template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads)
zl_cache_write_kernel(const CacheView c, const CacheBatch b, const __nv_bfloat16* k, const __nv_bfloat16* v, const int64_t row_stride) {
    constexpr int kLanes = D / 8;
    grid_release();
    grid_wait();
    const uint32_t r = my_row<D>();
    const uint32_t token = r / (uint32_t)c.n_kv_heads, head = r - token * (uint32_t)c.n_kv_heads;
    const int lane = threadIdx.x % kLanes;
    int64_t slot = -1;  // byte offset of the row in the cache
    int64_t at_scale = 0;
    if (token < (uint32_t)b.total_q) {
        const int s = find_seq(b.cu_q, b.n_seqs, (int32_t)token);
        if (s >= 0) {
            const SeqView sv = load_seq(b, c.page_shift, s);
            const int32_t i = (int32_t)token - sv.q0, pos = sv.pos0 + i;
            if (i >= 0 && i < sv.q_len && pos >= 0 && pos < sv.keys) {
                const int32_t pg = page_at(b, c, s, pos), in = pos & ((1 << c.page_shift) - 1);
                if (pg >= 0) {
                    slot = pg * c.page_stride + in * c.token_stride + head * c.head_stride;
                    at_scale = (((int64_t)pg << c.page_shift) + in) * c.n_kv_heads + head;
                }
            }
        }
    }
    const bool live = slot >= 0;
    const int64_t src = (int64_t)token * row_stride + (int64_t)head * D + lane * 8;
    uint4 xk = make_uint4(0, 0, 0, 0), xv = xk;
    if (live) {
        xk = __ldg(reinterpret_cast<const uint4*>(k + src));
        xv = __ldg(reinterpret_cast<const uint4*>(v + src));
    }
    if constexpr (kFormat == ZL_CACHE_BF16) {
        if (live) {
            *reinterpret_cast<uint4*>(c.k + slot + lane * 16) = xk;
            *reinterpret_cast<uint4*>(c.v + slot + lane * 16) = xv;
        }
    } else {
        float sk, sv;
        const uint2 ck = quantise<kFormat, kLanes>(xk, sk), cv = quantise<kFormat, kLanes>(xv, sv);
        if (live) {
            *reinterpret_cast<uint2*>(c.k + slot + lane * 8) = ck;
            *reinterpret_cast<uint2*>(c.v + slot + lane * 8) = cv;
            if (lane == 0) c.k_scale[at_scale] = sk;
            if (lane == 1) c.v_scale[at_scale] = sv;
        }
    }
}

template <int kFormat>
__device__ __forceinline__ uint4 dequantise(const uint2& u, float scale) {
    const uint32_t w[4] = {code_pair<kFormat, 0, 1>(u.x), code_pair<kFormat, 2, 3>(u.x), code_pair<kFormat, 0, 1>(u.y),
                           code_pair<kFormat, 2, 3>(u.y)};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // one rounding, of the product
        r[i] = pack_bf16(__uint_as_float(w[i] << 16) * scale, __uint_as_float(w[i] & 0xffff0000u) * scale);
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads)
zl_cache_read_kernel(const CacheView c, const CacheBatch b, const CacheReadParams p) {
    constexpr int kLanes = D / 8;
    grid_release();
    grid_wait();
    const uint32_t r = my_row<D>();
    const uint32_t row = r / (uint32_t)c.n_kv_heads, head = r - row * (uint32_t)c.n_kv_heads;
    const int lane = threadIdx.x % kLanes;
    if (row >= (uint32_t)p.total_kv) return;
    const int s = find_seq(p.cu_kv, b.n_seqs, (int32_t)row);
    if (s < 0) return;
    uint4 xk = make_uint4(0, 0, 0, 0), xv = xk;
    const int64_t pos = (int64_t)(p.first ? __ldg(p.first + s) : 0) + ((int32_t)row - __ldg(p.cu_kv + s));
    if (pos >= 0 && pos < load_seq(b, c.page_shift, s).keys) {
        const int32_t pg = page_at(b, c, s, (int32_t)pos), in = (int32_t)pos & ((1 << c.page_shift) - 1);
        if (pg >= 0) {
            const int64_t slot = pg * c.page_stride + in * c.token_stride + head * c.head_stride;
            if constexpr (kFormat == ZL_CACHE_BF16) {
                xk = *reinterpret_cast<const uint4*>(c.k + slot + lane * 16);
                xv = *reinterpret_cast<const uint4*>(c.v + slot + lane * 16);
            } else {
                const int64_t at = (((int64_t)pg << c.page_shift) + in) * c.n_kv_heads + head;
                const uint2 ck = *reinterpret_cast<const uint2*>(c.k + slot + lane * 8);
                const uint2 cv = *reinterpret_cast<const uint2*>(c.v + slot + lane * 8);
                xk = dequantise<kFormat>(ck, c.k_scale[at]);
                xv = dequantise<kFormat>(cv, c.v_scale[at]);
            }
        }
    }
    const int64_t dst = ((int64_t)row * c.n_kv_heads + head) * D + lane * 8;
    *reinterpret_cast<uint4*>(p.k + dst) = xk;
    *reinterpret_cast<uint4*>(p.v + dst) = xv;
}

int blocks(int64_t rows, int head_dim) {
    const int per = kThreads / (head_dim / 8);
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
