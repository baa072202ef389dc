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

}  // namespace zl
