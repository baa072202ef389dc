// Kernel parameter blocks and launch entry points shared by the C-ABI layer and the kernels.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <utility>

#include "zl_internal.h"

namespace zl {

struct FwdParams {
    const Task* tasks;
    const WorkItem* items;
    int32_t n_items;
    int32_t n_heads;
    int32_t total_q;
    int32_t partial_rows;
    float scale_log2;  // scale * log2(e)
    __nv_bfloat16* o;
    float* lse;
    float* o_partial;
    float* lse_partial;
    int32_t* status;  // [0] = code, [1] = where
    const int32_t* lists;  // CTA c walks items [lists[c], lists[c + 1]); NULL: items c, c + grid, ... (scored kernels only)
    int32_t* part_count;  // [tasks, H] finished pieces of an item cut along the keys; zero between launches
};

struct MergeParams {
    const MergeGroup* groups;
    const int32_t* parts;       // partial slot row offsets
    const int32_t* row_prefix;  // n_groups + 1
    const int32_t* row_group;   // [row_prefix[n_groups]] group of every row; handles over a shared prefix only
    int32_t n_groups;
    int32_t n_heads;
    int32_t total_q;
    int32_t partial_rows;
    const float* o_partial;
    const float* lse_partial;
    __nv_bfloat16* o;
    float* lse;
};

struct BwdParams {
    const Task* tasks;
    const WorkItem* items;       // (kv group, head, first key row, rows)
    const KvGroup* kv_groups;
    const int32_t* kv_group_tasks;
    const QGroup* q_groups;
    int32_t n_items;
    int32_t n_q_groups;
    int32_t n_heads;
    int32_t total_q;
    int32_t q_pad_total;
    float scale;
    float scale_log2;
    const __nv_bfloat16* o;
    const __nv_bfloat16* d_o;
    const float* lse;
    __nv_bfloat16* dq;
    __nv_bfloat16* dk;
    __nv_bfloat16* dv;
    int64_t grad_row_stride;  // elements between token rows of dq, dk, dv (H*d, or 3*H*d when packed)
    int32_t dq_rows;  // rows of dq_acc that are converted
    float* dq_acc;  // [dq_acc_rows, H, d]
    uint8_t* aug;   // [H, q_pad_total / 128] tiles of 4 KB: bf16 splits of -lse/scale and -rowsum(dO o O)
    int32_t* status;
    float* lse_tiles;  // [H, q_pad_total] LSE * log2(e), 1e30 for rows without a key; NULL unless scores are capped
    const int32_t* lists;  // as in FwdParams
    bool zero_dq;      // the preprocess kernel clears dq_acc (its rows are the padded query rows)
    float* d_bucket_bias;      // [n_buckets, H] gradient of the bucket table, summed beside the dQ conversion; NULL: not wanted
    const float* bucket_part;  // [H, n_kv_tiles, kMaxBuckets] key tiles' shares of it
    int32_t n_buckets, n_kv_tiles;
};

// Scores beyond scale * q.k (zl_score), as the kernels read them.
struct ScoreParams {
    const TaskPos* pos;          // per task; NULL: every task starts at position 0 of its sequence
    const float* slopes;         // [H] or NULL
    const float* bucket_bias;    // [n_buckets, H] or NULL
    const int32_t* bucket_of;    // [2 * reach + 1] bucket of key position - query position, clamped to [-reach, reach]
    int32_t n_buckets, reach;    // reach 0 without buckets
    int32_t n_heads;
    int32_t masked;
    float cap_log2;              // cap * log2(e)
    float scale_over_cap;        // scale / cap
    float* bucket_part;          // backward, [H, n_kv_tiles, kMaxBuckets]: each key tile's share of the table's gradient
    int32_t n_kv_tiles;
};
enum ScoreKind { kScorePlain = 0, kScoreBias = 1, kScoreBiasGrad = 2 };  // what is added to the (capped) product

// Launches a kernel that calls ptx::grid_wait() before it touches memory that earlier work writes: it may start, and set
// itself up, while the grid before it in the stream drains (`early` false: an ordinary launch).
template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), int grid, int threads, int smem, cudaStream_t stream, bool early, A&&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}

cudaError_t launch_scored_fwd(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                              const CUtensorMap& tv, const CUtensorMap& to, const CUtensorMap& top, const FwdParams& p,
                              const ScoreParams& sp, int grid, cudaStream_t stream);
// Items of at most 128 query rows, plain or scored; `q_box_rows`: rows of the tq box, a multiple of 16 that covers every item.
cudaError_t launch_few_rows(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                            const CUtensorMap& tv, int q_box_rows, const FwdParams& p, const ScoreParams& sp, int grid,
                            cudaStream_t stream);
cudaError_t launch_scored_bwd(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                              const CUtensorMap& tv, const CUtensorMap& tdo, const CUtensorMap& tdq, const CUtensorMap& tdk,
                              const CUtensorMap& tdv, const BwdParams& p, const ScoreParams& sp, int grid, cudaStream_t stream);

cudaError_t launch_bwd_pre(int head_dim, const BwdParams& p, int n_sms, cudaStream_t stream);
cudaError_t launch_bwd_main(int head_dim, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                            const CUtensorMap& tdo, const CUtensorMap& tdq, const CUtensorMap& tdk,
                            const CUtensorMap& tdv, const BwdParams& p, int grid, cudaStream_t stream);
// CTA-pair form of the main kernel (head_dim 128): `p.items` is the pair item list, `tq64` / `tdo64` are maps
// with 64-row boxes, `taug` views the augmentation tiles as rows of 1 KB, `tdk32` / `tdv32` are the gradient maps
// with 32-row boxes (one warp's rows).
cudaError_t launch_bwd_pair(const CUtensorMap& tq, const CUtensorMap& tq64, const CUtensorMap& tk, const CUtensorMap& tv,
                            const CUtensorMap& tdo, const CUtensorMap& tdo64, const CUtensorMap& tdq,
                            const CUtensorMap& taug, const CUtensorMap& tdk32, const CUtensorMap& tdv32, const BwdParams& p,
                            int n_clusters, cudaStream_t stream);
cudaError_t launch_bwd_post(int head_dim, const BwdParams& p, int n_sms, cudaStream_t stream);

cudaError_t launch_fwd(int head_dim, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                       const CUtensorMap& to, const CUtensorMap& top, const FwdParams& p, int grid,
                       cudaStream_t stream);
// `max_parts`: the largest number of parts of any merge group (selects a register-resident variant).
cudaError_t launch_merge(int head_dim, const MergeParams& p, int max_parts, int n_sms, cudaStream_t stream);
// The same merge for a batch over a shared prefix: few rows, many parts each.
cudaError_t launch_merge_rows(int head_dim, const MergeParams& p, int64_t n_rows, cudaStream_t stream);
cudaError_t launch_wait_selftest(int32_t* status, uint64_t limit_ns, cudaStream_t stream);

// ------------------------------------------------------------------------------------------------ paged cache
// Keys and values in pages (zl_kv_cache); strides in bytes, a page has 1 << page_shift tokens.
struct CacheView {
    uint8_t* k;
    uint8_t* v;
    float* k_scale;  // one number a token and head; NULL where the cache holds bf16
    float* v_scale;
    int64_t page_stride, token_stride, head_stride;
    int64_t scale_page, scale_token, scale_head;  // strides of the scales, elements
    uint32_t page16, token16, head16;             // strides of the keys in 16 bytes
    int32_t n_pages, page_shift, n_kv_heads;
};
// A batch of sequences over it (zl_cache_batch).
struct CacheBatch {
    const int32_t* cu_q;
    const int32_t* kv_len;
    const int32_t* pages;
    const int32_t* prefix;
    int32_t n_seqs, max_pages, total_q;
};
struct CacheReadParams {
    const int32_t* first;
    const int32_t* cu_kv;
    int32_t total_kv;
    __nv_bfloat16* k;
    __nv_bfloat16* v;
};
constexpr int kTokenRows = 16;  // most rows (new tokens times query heads of a key head) for which mma.sync tiles do
// Attention of a batch's new tokens over the cache.
struct CachedParams {
    CacheView c;
    CacheBatch b;
    const __nv_bfloat16* q;
    int64_t q_stride;    // elements between token rows
    int32_t n_heads, group;  // query heads, query heads per key head
    float scale_log2;
    __nv_bfloat16* o;
    float* lse;          // may be NULL
    float* part;         // two partial results per CTA
    int32_t* part_count; // per CTA: finished parts of the item that is cut first in it; zero between launches
    float* chunk_part;   // the same of the kernel for chunks
    void* chunk_cut;     // per CTA of it: the item that is cut first in it
    int32_t split;       // both kernels run: sequences of at most kTokenRows rows per key head are the tokens kernel's
    int32_t token_rows;  // rows of an item of the tokens kernel: 8 or kTokenRows
    int32_t head_first;  // coordinates of the K and V maps are (column, head, token, page), else (column, token, head, page)
    int32_t* status;
};
cudaError_t launch_cache_write(int head_dim, int format, const CacheView& c, const CacheBatch& b, const __nv_bfloat16* k,
                               const __nv_bfloat16* v, int64_t row_stride, cudaStream_t stream);
cudaError_t launch_cache_read(int head_dim, int format, const CacheView& c, const CacheBatch& b, const CacheReadParams& p,
                              cudaStream_t stream);
cudaError_t launch_cached_tokens(int head_dim, int format, const CachedParams& p, int grid, cudaStream_t stream);
size_t cached_tokens_part_bytes(int head_dim);  // of a CTA's two partial results
// Maps: tq of [total_q, n_kv_heads, group, d], box 64 columns x group x 1 x whole tokens of 128 rows; tk and tv over the pages, box 64
// columns of bf16 or a row of codes, rows of one page, at most 128.
cudaError_t launch_cached_chunk(int head_dim, int format, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                                const CachedParams& p, int grid, cudaStream_t stream);
size_t cached_chunk_part_bytes(int head_dim);  // of a CTA's two partial results
size_t cached_chunk_cut_bytes();
// Joins the parts of items that the chunk kernel's CTAs share.
cudaError_t launch_cached_join(int head_dim, const CachedParams& p, int ctas, cudaStream_t stream);

// Of the C-ABI layer.
void count_launch();
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode_fn();

}  // namespace zl
