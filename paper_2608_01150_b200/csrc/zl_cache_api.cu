// C-ABI layer of the paged cache: argument checks and launches.
#include <cmath>
#include <new>
#include <utility>

#include "zl_device.h"

using namespace zl;

struct zl_cached_attn {
    int32_t n_heads = 0, n_kv_heads = 0, head_dim = 0;
    int device = -1;  // -1: host-only handle (no CUDA device present)
    int n_sms = 0;
    int32_t* d_words = nullptr;  // [0, 2): status; from kCounters on one counter per SM
};

namespace {

constexpr int kCounters = 64;  // a line of its own for the status word

size_t tokens_bytes(const zl_cached_attn& a) { return align_up((size_t)a.n_sms * cached_tokens_part_bytes(a.head_dim), 256); }

size_t chunk_bytes(const zl_cached_attn& a) { return align_up((size_t)a.n_sms * cached_chunk_part_bytes(a.head_dim), 256); }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The cache and the batch as the kernels read them.  `tokens`: the call has rows of the batch's token space.
zl_status view(const zl_kv_cache* cache, const zl_cache_batch* batch, bool tokens, CacheView* c, CacheBatch* b) {
    if (!cache || !batch) return ZL_ERR_INVALID_ARG;
    const zl_kv_cache& x = *cache;
    if (x.head_dim != 64 && x.head_dim != 128) return ZL_ERR_UNSUPPORTED;
    if (x.format != ZL_CACHE_BF16 && x.format != ZL_CACHE_INT8 && x.format != ZL_CACHE_E4M3) return ZL_ERR_UNSUPPORTED;
    if (x.n_pages < 0 || x.n_kv_heads < 1 || x.page_size < 1) return ZL_ERR_INVALID_ARG;
    if (x.page_size < 8 || (x.page_size & (x.page_size - 1)) != 0 || x.page_size > (1 << 24)) return ZL_ERR_UNSUPPORTED;
    const int bytes = x.format == ZL_CACHE_BF16 ? 2 : 1;
    for (int64_t s : {x.page_stride, x.token_stride, x.head_stride})
        if (s < 0 || s >= (int64_t)1 << 35 || (s * bytes) % 16 != 0) return ZL_ERR_INVALID_ARG;  // (below 2^35, in units of 16 bytes they fit 32 bits)
    for (int64_t s : {x.scale_page_stride, x.scale_token_stride, x.scale_head_stride})
        if (s < 0 || s >= (int64_t)1 << 32) return ZL_ERR_INVALID_ARG;
    if (x.n_pages > 0) {
        if (!x.k || !x.v || !aligned16(x.k) || !aligned16(x.v)) return ZL_ERR_INVALID_ARG;
        if (x.format != ZL_CACHE_BF16) {
            if (!x.k_scale || !x.v_scale) return ZL_ERR_INVALID_ARG;
            if (x.scale_token_stride < 1 || (x.n_kv_heads > 1 && x.scale_head_stride < 1) || (x.n_pages > 1 && x.scale_page_stride < 1))
                return ZL_ERR_INVALID_ARG;
        }
        // rows of the cache may not lie over one another
        if (x.token_stride < x.head_dim || (x.n_kv_heads > 1 && x.head_stride < x.head_dim) || (x.n_pages > 1 && x.page_stride < x.head_dim))
            return ZL_ERR_INVALID_ARG;
    }
    if (x.format == ZL_CACHE_BF16 && (x.k_scale || x.v_scale)) return ZL_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(x.k_scale) | reinterpret_cast<uintptr_t>(x.v_scale)) & 3) != 0) return ZL_ERR_INVALID_ARG;
    if (batch->n_seqs < 0 || batch->max_pages < 0 || batch->total_q < 0 || batch->max_q < 0) return ZL_ERR_INVALID_ARG;
    if (batch->n_seqs > 0 && ((tokens && !batch->cu_q) || !batch->kv_len || (batch->max_pages > 0 && !batch->pages))) return ZL_ERR_INVALID_ARG;
    // positions are counted in 32 bits with room to spare
    if ((int64_t)batch->max_pages * x.page_size > (int64_t)1 << 30) return ZL_ERR_UNSUPPORTED;
    int shift = 0;
    while ((1 << shift) < x.page_size) ++shift;
    *c = CacheView{static_cast<uint8_t*>(x.k), static_cast<uint8_t*>(x.v), x.k_scale, x.v_scale,
                   x.page_stride * bytes, x.token_stride * bytes, x.head_stride * bytes, x.scale_page_stride, x.scale_token_stride, x.scale_head_stride,
                   (uint32_t)(x.page_stride * bytes / 16), (uint32_t)(x.token_stride * bytes / 16), (uint32_t)(x.head_stride * bytes / 16), x.n_pages, shift, x.n_kv_heads};
    *b = CacheBatch{batch->cu_q, batch->kv_len, batch->pages, batch->prefix, batch->n_seqs, x.n_pages > 0 ? batch->max_pages : 0, batch->total_q};
    return ZL_OK;
}

bool rows_fit(int64_t rows, int32_t heads) { return rows * heads < (int64_t)1 << 32; }

// Maps of the kernel for chunks.
bool make_maps(const zl_kv_cache& x, const CachedParams& p, CUtensorMap* tq, CUtensorMap* tk, CUtensorMap* tv) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    const cuuint64_t d = (cuuint64_t)x.head_dim;
    {
        const cuuint64_t dims[4] = {d, (cuuint64_t)p.group, (cuuint64_t)x.n_kv_heads, (cuuint64_t)p.b.total_q};
        const cuuint64_t strides[3] = {d * 2, d * 2 * p.group, (cuuint64_t)p.q_stride * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)p.group, 1, (cuuint32_t)(kTileQ / p.group)};
        if (fn(tq, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(p.q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    }
    const bool codes = x.format != ZL_CACHE_BF16;
    const cuuint32_t rows = (cuuint32_t)(x.page_size < kTileKV ? x.page_size : kTileKV);
    const cuuint64_t heads = (cuuint64_t)x.n_kv_heads, tokens = (cuuint64_t)x.page_size, pages = (cuuint64_t)x.n_pages;
    cuuint64_t dims[4] = {d, tokens, heads, pages}, strides[3] = {(cuuint64_t)p.c.token_stride, (cuuint64_t)p.c.head_stride, (cuuint64_t)p.c.page_stride};
    const cuuint64_t row = d * (codes ? 1 : 2);
    for (cuuint64_t& stride : strides) stride = stride ? stride : row;  // (of a dimension with one entry)
    cuuint32_t box[4] = {codes ? (cuuint32_t)d : 64u, rows, 1, 1};
    if (p.head_first) {
        std::swap(dims[1], dims[2]);
        std::swap(strides[0], strides[1]);
        std::swap(box[1], box[2]);
    }
    const CUtensorMapSwizzle swizzle = codes && x.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
    for (int i = 0; i < 2; ++i)
        if (fn(i == 0 ? tk : tv, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, i == 0 ? p.c.k : p.c.v, dims, strides, box, ones,
               CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
    return true;
}

// No device, or one that the kernels are not built for.
zl_status usable_device() {
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
        cudaGetLastError();
        return ZL_ERR_CUDA;
    }
    return major == 10 ? ZL_OK : ZL_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

zl_status zl_cache_write(const zl_kv_cache* cache, const zl_cache_batch* batch, const void* k, const void* v,
                         int64_t row_stride, void* stream) {
    CacheView c;
    CacheBatch b;
    if (const zl_status st = view(cache, batch, true, &c, &b)) return st;
    const int64_t row = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (b.total_q > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return ZL_ERR_INVALID_ARG;
    if (row_stride % 8 != 0 || row_stride < row) return ZL_ERR_INVALID_ARG;
    if (!rows_fit(b.total_q, c.n_kv_heads)) return ZL_ERR_UNSUPPORTED;
    if (const zl_status st = usable_device()) return st;
    if (b.total_q == 0 || b.n_seqs == 0 || b.max_pages == 0 || c.n_pages == 0) return ZL_OK;
    if (launch_cache_write(cache->head_dim, cache->format, c, b, static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v),
                           row_stride, static_cast<cudaStream_t>(stream)) != cudaSuccess)
        return ZL_ERR_CUDA;
    count_launch();
    return ZL_OK;
}

zl_status zl_cache_read(const zl_kv_cache* cache, const zl_cache_batch* batch, const int32_t* first, const int32_t* cu_kv,
                        int32_t total_kv, void* k, void* v, void* stream) {
    CacheView c;
    CacheBatch b;
    if (const zl_status st = view(cache, batch, false, &c, &b)) return st;
    if (total_kv < 0 || (b.n_seqs > 0 && !cu_kv)) return ZL_ERR_INVALID_ARG;
    if (total_kv > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return ZL_ERR_INVALID_ARG;
    if (!rows_fit(total_kv, c.n_kv_heads)) return ZL_ERR_UNSUPPORTED;
    if (const zl_status st = usable_device()) return st;
    if (total_kv == 0 || b.n_seqs == 0) return ZL_OK;
    b.cu_q = cu_kv;  // (the sequences' lengths are all that is read of the token space)
    const CacheReadParams p{first, cu_kv, total_kv, static_cast<__nv_bfloat16*>(k), static_cast<__nv_bfloat16*>(v)};
    if (launch_cache_read(cache->head_dim, cache->format, c, b, p, static_cast<cudaStream_t>(stream)) != cudaSuccess) return ZL_ERR_CUDA;
    count_launch();
    return ZL_OK;
}

zl_status zl_build_cached_attn(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void* stream, zl_cached_attn** out) {
    if (!out) return ZL_ERR_INVALID_ARG;
    *out = nullptr;
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0) return ZL_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return ZL_ERR_UNSUPPORTED;
    if (n_heads / n_kv_heads > 128) return ZL_ERR_UNSUPPORTED;
    zl_cached_attn* h = new (std::nothrow) zl_cached_attn();
    if (!h) return ZL_ERR_INVALID_ARG;
    h->n_heads = n_heads;
    h->n_kv_heads = n_kv_heads;
    h->head_dim = head_dim;
    int n_dev = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess || n_dev == 0) {
        cudaGetLastError();  // host-only handle: launches return ZL_ERR_CUDA
        *out = h;
        return ZL_OK;
    }
    int dev = 0, major = 0, n_sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        delete h;
        return ZL_ERR_CUDA;
    }
    if (major != 10) { delete h; return ZL_ERR_UNSUPPORTED; }
    const size_t bytes = (size_t)(kCounters + n_sms) * sizeof(int32_t);
    if (cudaMalloc(&h->d_words, bytes) != cudaSuccess) { delete h; return ZL_ERR_CUDA; }
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(h->d_words, 0, bytes, cs) != cudaSuccess || cudaStreamSynchronize(cs) != cudaSuccess) {
        cudaFree(h->d_words);
        delete h;
        return ZL_ERR_CUDA;
    }
    h->device = dev;
    h->n_sms = n_sms;
    *out = h;
    return ZL_OK;
}

void zl_free_cached_attn(zl_cached_attn* attn) {
    if (!attn) return;
    if (attn->d_words) cudaFree(attn->d_words);
    delete attn;
}

zl_status zl_cached_attn_workspace_bytes(const zl_cached_attn* attn, size_t* bytes) {
    if (!attn || !bytes) return ZL_ERR_INVALID_ARG;
    *bytes = tokens_bytes(*attn) + chunk_bytes(*attn) + align_up((size_t)attn->n_sms * cached_chunk_cut_bytes(), 256);
    return ZL_OK;
}

zl_status zl_cached_attn_device_status(const zl_cached_attn* attn, int32_t* code, int32_t* where) {
    if (!attn || !code || !where) return ZL_ERR_INVALID_ARG;
    *code = *where = 0;
    if (attn->device < 0) return ZL_ERR_CUDA;
    int prev = 0;
    if (cudaGetDevice(&prev) != cudaSuccess || cudaSetDevice(attn->device) != cudaSuccess) return ZL_ERR_CUDA;
    int32_t words[2] = {0, 0};
    zl_status st = ZL_OK;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(words, attn->d_words, sizeof(words), cudaMemcpyDeviceToHost) != cudaSuccess)
        st = ZL_ERR_CUDA;
    if (st == ZL_OK && words[0] != 0 && cudaMemset(attn->d_words, 0, (size_t)(kCounters + attn->n_sms) * sizeof(int32_t)) != cudaSuccess)
        st = ZL_ERR_CUDA;
    cudaSetDevice(prev);
    *code = words[0];
    *where = words[1];
    return st;
}

zl_status zl_cached_attn_fwd(const zl_cached_attn* attn, const zl_kv_cache* cache, const zl_cache_batch* batch, const void* q,
                             int64_t q_stride, float scale, void* o, float* lse, void* workspace, size_t workspace_bytes,
                             void* stream) {
    if (!attn) return ZL_ERR_INVALID_ARG;
    CachedParams p{};
    if (const zl_status st = view(cache, batch, true, &p.c, &p.b)) return st;
    if (cache->n_kv_heads != attn->n_kv_heads || cache->head_dim != attn->head_dim) return ZL_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f)) return ZL_ERR_INVALID_ARG;
    if (q_stride % 8 != 0 || q_stride < (int64_t)attn->n_heads * attn->head_dim) return ZL_ERR_INVALID_ARG;
    if (p.b.total_q > 0 && (!q || !o || !aligned16(q) || !aligned16(o))) return ZL_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(lse) & 3) != 0) return ZL_ERR_INVALID_ARG;
    if (!rows_fit(p.b.total_q, attn->n_heads)) return ZL_ERR_UNSUPPORTED;
    if (p.b.total_q > 0) {  // parts of an item read their queries while others write their output
        const char *q0 = static_cast<const char*>(q), *o0 = static_cast<const char*>(o);
        const int64_t row = (int64_t)attn->n_heads * attn->head_dim * 2;
        if (q0 < o0 + p.b.total_q * row && o0 < q0 + (p.b.total_q - 1) * q_stride * 2 + row) return ZL_ERR_INVALID_ARG;
    }
    if (attn->device < 0) return ZL_ERR_CUDA;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != attn->device) return ZL_ERR_INVALID_ARG;
    if (p.b.total_q == 0 || p.b.n_seqs == 0) return ZL_OK;
    size_t need = 0;
    zl_cached_attn_workspace_bytes(attn, &need);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return ZL_ERR_INVALID_ARG;
    if (workspace_bytes < need) return ZL_ERR_WORKSPACE;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.q_stride = q_stride;
    p.n_heads = attn->n_heads;
    p.group = attn->n_heads / attn->n_kv_heads;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.o = static_cast<__nv_bfloat16*>(o);
    p.lse = lse;
    p.part = static_cast<float*>(workspace);
    p.part_count = attn->d_words + kCounters;
    p.chunk_part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + tokens_bytes(*attn));
    p.chunk_cut = static_cast<uint8_t*>(workspace) + tokens_bytes(*attn) + chunk_bytes(*attn);
    p.status = attn->d_words;
    // Sequences of more than kTokenRows rows per key head are the chunk kernel's.  Where max_q says that there are none, or that
    // all are of that kind (as many rows as the longest times their number), the other kernel is not launched.  An item of the
    // tokens kernel has eight rows, or 16 where a single token, or the longest sequence, has more than eight.
    const int32_t max_q = batch->max_q;
    const bool few = max_q > 0 && (int64_t)max_q * p.group <= kTokenRows;
    p.token_rows = few ? (max_q * p.group <= 8 ? 8 : kTokenRows) : (p.group <= 8 ? 8 : kTokenRows);
    const bool all_long = !few && max_q > 0 && (int64_t)max_q * p.b.n_seqs == p.b.total_q;  // (if not so after all, it takes the rest too)
    // a cache without a page has no key, and nothing to describe to the copy engine
    const bool chunk = !few && p.c.n_pages > 0 && p.b.max_pages > 0;
    p.split = chunk && !all_long;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (chunk) {
        // dimensions in the order of their strides
        p.head_first = p.c.head_stride < p.c.token_stride;
        CUtensorMap tq, tk, tv;
        if (!make_maps(*cache, p, &tq, &tk, &tv)) return ZL_ERR_CUDA;
        if (launch_cached_chunk(attn->head_dim, cache->format, tq, tk, tv, p, attn->n_sms, cs) != cudaSuccess) return ZL_ERR_CUDA;
        count_launch();
    }
    if (!chunk || p.split) {  // (next behind the other: it starts before that has ended)
        if (launch_cached_tokens(attn->head_dim, cache->format, p, attn->n_sms, cs) != cudaSuccess) return ZL_ERR_CUDA;
        count_launch();
    }
    if (chunk) {
        if (launch_cached_join(attn->head_dim, p, attn->n_sms, cs) != cudaSuccess) return ZL_ERR_CUDA;
        count_launch();
    }
    return ZL_OK;
}

}  // extern "C"
