// Internal definitions shared by the host scheduler and the kernels of libzellige.
#pragma once

#include <cstdint>
#include <vector>

#include "zellige.h"

#ifdef __CUDACC__
#define ZL_HOST_DEVICE __host__ __device__
#else
#define ZL_HOST_DEVICE
#endif

namespace zl {

constexpr int kTileQ = 128;   // query rows per MMA tile (TMEM lanes)
constexpr int kTileKV = 128;  // key rows per MMA tile
constexpr int kMaxBuckets = ZL_MAX_BUCKETS;
constexpr int kFwdBlockQ = 2 * kTileQ;  // query rows per forward work item: two tiles in flight per CTA

// One attention task on the device: whole sequence or shard.
struct alignas(32) Task {
    int32_t q_off, q_len, kv_off, kv_len;
    int32_t partial_slot;  // first row of the task's slot in o_partial, -1 for a whole sequence
    int32_t q_slot;        // first row of the task's query range in the padded backward scratch
    int32_t kv_group;      // -1 if kv_len == 0
    int32_t dq_slot;       // row of the dQ accumulator that belongs to q_off (q_slot, unless query ranges nest)
};

// Positions of a task's rows inside its sequence, for scores and masks that depend on them: query row r of the task
// has position q_pos + r, key row r position kv_pos + r; keys before `prefix` are seen by every query.
struct alignas(16) TaskPos {
    int32_t q_pos, kv_pos, prefix, pad_;
};

// Key rows (relative to the task) that query row `r` of the task sees under the prefix mask: [0, result).  Keys at
// positions before `prefix` and keys not after the query; positions never exceed INT32_MAX (checked when they are set).
ZL_HOST_DEVICE inline int32_t visible_keys(const TaskPos& tp, int32_t kv_len, int32_t r) {
    const int32_t by_prefix = tp.prefix - tp.kv_pos, by_order = tp.q_pos + r + 1 - tp.kv_pos;
    const int32_t n = by_prefix > by_order ? by_prefix : by_order;
    return n < 0 ? 0 : (n < kv_len ? n : kv_len);
}

// First query row (relative to the task) that sees key row `kr` of the task: rows [result, q_len) see it.  May be
// q_len or more: nobody does.
ZL_HOST_DEVICE inline int32_t first_query(const TaskPos& tp, int32_t kr) {
    if (tp.kv_pos + kr < tp.prefix) return 0;
    const int32_t r = tp.kv_pos + kr - tp.q_pos;
    return r < 0 ? 0 : r;
}

// (task | kv group, head, first row relative to the task's query range | group's key range, rows)
struct alignas(16) WorkItem {
    int32_t unit, head, row0, rows;
};

// Few query rows against long keys: the few-rows kernel takes an item in `parts` pieces along the keys.  Such an item has
// row0 = the piece and rows = parts << kPartsShift | rows.  Piece s leaves its partial result in rows s * q_len .. of the
// task's slot, which is padded to 128 rows; the piece that finishes last joins them into the first q_len.
constexpr int kPartsShift = 16;

// Shard tasks that share a query range and a head range; they are merged for heads
// [head_begin, head_begin + head_count) only.
struct alignas(32) MergeGroup {
    int32_t q_off, q_len;
    int32_t part_begin, n_parts;  // range in the merge part list (partial slot row offsets)
    int32_t head_begin, head_count;
    int32_t pad_[2];
};

// A distinct (query range, head range): rows [slot, slot + pad128(q_len)) of the backward scratch
// arrays, of which only the heads of the range are used.
struct alignas(32) QGroup {
    int32_t q_off, q_len, slot, pad;
    int32_t head_begin, head_count;
    int32_t pad_[2];
};

struct alignas(16) KvGroup {
    int32_t kv_off, kv_len;
    int32_t task_begin, n_tasks;  // range in the kv-group task list
    int32_t n_q_tiles;            // 128-row query tiles of all its tasks together
    int32_t tile_begin;           // number of 128-row key tiles of the groups before it
    int32_t first_q_len;          // query rows of its first task
    int32_t pad_;
};

// One attention problem of a placement as the builder receives it: a whole sequence (q range ==
// kv range, final after the forward launch) or a shard (one query chunk x one K/V chunk), over the
// heads [head_begin, head_begin + head_count).
struct InputTask {
    int32_t q_off, q_len, kv_off, kv_len, seq_id;
    int32_t head_begin, head_count;
    int32_t shard_idx;  // index into the caller's shard array, -1 for a whole sequence
};

// Work items dealt out to CTAs: CTA c walks items [begin[c], begin[c + 1]).
struct DealtList {
    std::vector<WorkItem> items;
    std::vector<int32_t> begin;
    bool few = false;   // forward: for the few-rows kernel (blocks of one query tile, or pieces along the keys)
    int32_t parts = 0;  // forward: pieces along the keys; 0: blocks and pieces not chosen yet
    int32_t ctas() const { return begin.empty() ? 0 : (int32_t)begin.size() - 1; }
};

// Everything zl_build_tasks derives from a placement, on the host.
struct Schedule {
    int32_t n_heads = 0, head_dim = 0, total_q = 0, total_kv = 0;
    std::vector<Task> tasks;
    std::vector<int32_t> task_head_begin, task_head_count;  // per task (host only: items carry their head)
    std::vector<int32_t> whole_to_task;     // per input whole sequence: task index or -1 (empty sequence)
    std::vector<int32_t> shard_to_task;     // per input shard: task index or -1 (q_len == 0)
    std::vector<int32_t> shard_kv_off, shard_kv_len;  // per input shard: its own key range (a fused task covers several)
    std::vector<int32_t> shard_slot_off;    // per input shard: slot row offset (or 0)
    std::vector<int32_t> shard_slot_rows;   // per input shard: padded slot rows (0 if skipped)
    std::vector<MergeGroup> merge_groups;
    std::vector<int32_t> merge_parts;       // slot row offsets, ascending shard order per group
    std::vector<int32_t> merge_row_group;   // group of every row (shared prefixes only)
    std::vector<int32_t> merge_row_prefix;  // n_merge_groups+1 prefix sums of q_len
    std::vector<QGroup> q_groups;
    int64_t q_pad_total = 0;                // rows of the padded backward scratch arrays
    int64_t dq_rows = 0;                    // rows of the dQ accumulator that are converted (q_pad_total, unless query ranges nest)
    int64_t dq_acc_rows = 0;                // rows of the dQ accumulator in the workspace
    int32_t n_kv_tiles = 0;                 // 128-row key tiles of all kv groups
    int32_t max_item_rows = 0;              // most query rows of a forward item
    bool all_heads = true;                  // every task covers all heads
    bool shared_prefix = false;             // built by build_prefix_schedule: query ranges nest
    // Lists of the scored kernels, dealt out to the CTAs: for calls without a mask (built with the handle, empty where
    // the plain lists are as even) and, with the positions (one entry per task, zl_set_positions), for masked ones.
    DealtList fwd_all, bwd_all, fwd_masked, bwd_masked;
    std::vector<TaskPos> task_pos;
    std::vector<KvGroup> kv_groups;
    std::vector<int32_t> kv_group_tasks;
    std::vector<WorkItem> fwd_items;
    std::vector<WorkItem> bwd_items;
    std::vector<WorkItem> bwd_pair_items;   // (kv group, head, first key row, rows <= 256): two key tiles per CTA pair
    // Launch phases: the work lists are grouped by phase and a phased launch walks one group.  Forward phases are
    // per task, backward phases per kv group; one phase (the whole list) until zl_set_fwd_phases / zl_set_bwd_phases.
    std::vector<int32_t> fwd_task_phase, bwd_group_phase;
    std::vector<int32_t> fwd_phase_begin, bwd_phase_begin, bwd_pair_phase_begin;  // n_phases + 1 offsets into the lists
    int64_t partial_rows = 0;
    int32_t n_fused_ranges = 0;             // shard query ranges lowered to one final task (chunk fusion)
    size_t bwd_workspace_bytes = 0;
    // byte offsets inside the backward workspace
    size_t ws_dq_acc_off = 0, ws_aug_off = 0;
};

// Validates the placement and fills `s`.  Pure host code, no CUDA.
// `in`: whole sequences first (in placement order), then shards (in the caller's order); `n_shards` is
// the size of the caller's shard array.  `flags`: ZL_BUILD_* bits of zl_build_tasks_ex.
zl_status build_schedule(const std::vector<InputTask>& in, int32_t n_shards, int32_t total_q, int32_t total_kv,
                         int32_t n_heads, int32_t head_dim, uint32_t flags, Schedule* s);

// A batch of sequences over one shared prefix of keys (zl_build_tasks_prefix).
zl_status build_prefix_schedule(const int32_t* cu_q, const int32_t* cu_kv, int32_t n_seqs, int32_t prefix_len,
                                int32_t total_q, int32_t total_kv, int32_t n_heads, int32_t head_dim, Schedule* s);

// Checks the positions and fills task_pos and the masked work lists of `s` (zl_set_positions), dealt out to `n_sms` CTAs.
zl_status set_positions(Schedule* s, const int32_t* whole_prefix, const zl_shard_pos* shard_pos, int32_t n_sms);

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace zl
