// Forward kernel of scored attention (sm_100a): scores capped by a tanh, biased by distance or by a learned bucket of
// the distance, and cut by a prefix mask, for the same work items, tensors and partial results as the plain forward.
//
//     s_ij = C(scale q_i.k_j) + b_h(pos(j) - pos(i)),   pairs beyond a row's visible keys left out
//     O_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij),      LSE_i = log sum_j exp(s_ij)
//
// Structure as in zl_fwd.cu: a persistent CTA holds two 128-row query tiles in flight, warp 0 feeds tiles by TMA, warp 1
// issues the MMAs, one warpgroup per tile runs the online softmax from TMEM.  What differs:
//   * The prefix mask leaves every row a leading stretch of keys, visible_keys() of them, and later rows never fewer.  So a
//     query tile walks the key tiles up to its last row's limit (tile A may stop before tile B), and one compare per
//     score against the row's limit masks the tiles at the border and the ragged end alike; full tiles compare nothing.
//   * The bias by distance needs no [Lq, Lk] matrix.  Where a 128 x 128 tile lies on one side of the diagonal and beyond the
//     buckets' reach it is linear in the column: a constant of the row, or one multiply-add more per score with slopes.
//     Near the diagonal a tile has only 255 different distances: the two warps without another role fetch them ahead
//     (table and bucket map are small and stay in L2) into a window in shared memory, of which a thread reads its row as
//     128 conflict-free words.
//   * The cap costs a tanh per score.  For a tile with |x / cap| <= 0.6 it is a polynomial of five packed multiply-adds,
//     run under the exponentials where the row needs no new reference; else two special-function operations (zl_score.cuh).
// Measured (B200, 12 heads, d 128): slopes over 9450 tokens 520-580 us (0.95-1.05 PFLOP/s of the pairs; the plain kernel 400-450),
// capped scores of the same tokens 600 us near zero and 1,000 us where they saturate, causal order 240 us.  No pipe is
// full (tensor, special-function and multiply-add 34-41 % each): what bounds it is the softmax chain of the two warps that
// an SM quarter has, and with short sequences the fill and drain of items of a few key tiles.
#include <cuda_runtime.h>

#include "zl_score.cuh"

namespace zl {

using namespace ptx;
using namespace score;

namespace {

constexpr int kFwdThreads = 384;

template <int D>
struct ScoredFwdSmem {
    static constexpr int kStages = (D == 128) ? 2 : 4;
    static constexpr int kTileBytes = kTileQ * D * 2;  // one 128-row tile of Q, K or V
    static constexpr int kBoxBytes = kTileQ * 128;     // one TMA box: 128 rows x 64 bf16
    static constexpr int kBoxes = D / 64;
    alignas(1024) uint8_t q[2][kTileBytes];
    alignas(1024) uint8_t k[kStages][kTileBytes];
    alignas(1024) uint8_t v[kStages][kTileBytes];
    alignas(1024) uint8_t o_stage[2][kBoxBytes];  // per softmax warpgroup: 128 rows x 128 bytes of O on their way out
    float window[2][kWindow];                      // per query tile: the biases of a near key tile
    alignas(8) uint64_t q_full[2], q_empty;
    uint64_t kv_full[kStages], kv_empty[kStages];  // K and V of a stage travel together
    uint64_t bias_full[2], bias_empty[2];
    uint64_t s_full[2], p_half[2][2], o_full[2];  // p_half[tile][half of the key columns]
    uint32_t tmem_base;
    volatile int32_t abort_flag;
};

// Wait used by a single elected thread.
#define ZL_WAIT(bar, parity, site)                                        \
    do {                                                                  \
        if (!wait((bar), (parity), &sm.abort_flag)) { \
            report(p.status, &sm.abort_flag, 3000 + (site));              \
            goto teardown;                                                \
        }                                                                 \
    } while (0)
// Wait used by all 32 lanes of a warp: the outcome is made warp-uniform and the warp
// reconverges before the .sync.aligned TMEM instructions that follow.
#define ZL_WAIT_WARP(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 3000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)
// The same from the warps that hold tiles in registers.
#define ZL_WAIT_REGS(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait_inline((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 3000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)

template <int D, bool kCap, bool kBias>
__global__ void __launch_bounds__(kFwdThreads, 1)
zl_scored_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
              const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
              const __grid_constant__ CUtensorMap tm_op, const FwdParams p, const ScoreParams sp) {
    using Smem = ScoredFwdSmem<D>;
    constexpr int kStages = Smem::kStages;
    constexpr int kBoxes = Smem::kBoxes;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    // TMEM columns: S_A [0,128), S_B [128,256), O_A [256,256+D), O_B [384,384+D).  P_x (bf16
    // pairs) overwrites the first 64 columns of S_x once the row has been read.
    constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;

    if ((smem_u32(smem_raw) & 1023u) != 0) {  // swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0 && atomicCAS(p.status, 0, (int)ZL_ERR_CUDA) == 0) p.status[1] = 3999;
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&sm.q_full[0], 1);
        mbar_init(&sm.q_full[1], 1);
        mbar_init(&sm.q_empty, 1);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.kv_full[s], 1);
            mbar_init(&sm.kv_empty[s], 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sm.s_full[x], 1);
            mbar_init(&sm.p_half[x][0], 128);
            mbar_init(&sm.p_half[x][1], 128);
            mbar_init(&sm.o_full[x], 1);
            mbar_init(&sm.bias_full[x], 1);
            mbar_init(&sm.bias_empty[x], 128);
        }
        sm.abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        prefetch_tmap(&tm_o);
        prefetch_tmap(&tm_op);
    }
    if (warp == 1) {
        tmem_alloc(&sm.tmem_base, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    grid_release();
    grid_wait();
    const Walk walk(p);

    if (warp < 4) {
        reg_dec<72>();
        if (warp == 0 && lane == 0) {
            // -------------------------------------------------------------- TMA producer
            uint32_t q_cnt = 0, qb_cnt = 0, kv_cnt = 0;
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const bool has_b = wi.rows > kTileQ;
                const int n_a = key_tiles(sp, t, wi.unit, wi.row0, min(wi.rows, kTileQ));
                const int n_b = key_tiles(sp, t, wi.unit, wi.row0 + kTileQ, wi.rows - kTileQ);
                const int n_kv = max(n_a, n_b);
                if (n_kv == 0) continue;
                ZL_WAIT(&sm.q_empty, (q_cnt & 1) ^ 1, 1);
                ++q_cnt;
                mbar_arrive_expect_tx(&sm.q_full[0], Smem::kTileBytes);
                for (int b = 0; b < kBoxes; ++b)
                    tma_load_3d(sm.q[0] + b * Smem::kBoxBytes, &tm_q, &sm.q_full[0], b * 64, wi.head, t.q_off + wi.row0);
                for (int j = 0; j < n_kv; ++j, ++kv_cnt) {
                    const int s = kv_cnt % kStages;
                    const uint32_t ph = (kv_cnt / kStages) & 1;
                    ZL_WAIT(&sm.kv_empty[s], ph ^ 1, 2);
                    mbar_arrive_expect_tx(&sm.kv_full[s], 2 * Smem::kTileBytes);
                    for (int b = 0; b < kBoxes; ++b)
                        tma_load_3d(sm.k[s] + b * Smem::kBoxBytes, &tm_k, &sm.kv_full[s], b * 64, wi.head,
                                    t.kv_off + j * kTileKV);
                    if (j == 0 && has_b) {  // second query tile right after the first K tile
                        mbar_arrive_expect_tx(&sm.q_full[1], Smem::kTileBytes);
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_3d(sm.q[1] + b * Smem::kBoxBytes, &tm_q, &sm.q_full[1], b * 64, wi.head,
                                        t.q_off + wi.row0 + kTileQ);
                        ++qb_cnt;
                    }
                    for (int b = 0; b < kBoxes; ++b)
                        tma_load_3d(sm.v[s] + b * Smem::kBoxBytes, &tm_v, &sm.kv_full[s], b * 64, wi.head,
                                    t.kv_off + j * kTileKV);
                }
            }
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMA issuer
            // The whole warp runs this loop converged and one elected lane issues, which keeps
            // descriptors and barrier addresses warp-uniform (cheaper commits and satisfied waits).
            const bool mma_lane = elect_one();
            constexpr uint32_t idesc_s = make_idesc_bf16(kTileQ, kTileKV, 0, 0);
            constexpr uint32_t idesc_o = make_idesc_bf16(kTileQ, D, 0, 1);
            const uint64_t dq0 = make_desc_sw128(smem_u32(sm.q[0]), 16, 1024);
            const uint64_t dk0 = make_desc_sw128(smem_u32(sm.k[0]), 16, 1024);
            const uint64_t dv0 = make_desc_sw128(smem_u32(sm.v[0]), Smem::kBoxBytes, 1024);  // V is the MN-major B operand
            constexpr uint32_t kTileStep = Smem::kTileBytes >> 4;
            // S_x = Q_x K^T
            auto issue_s = [&](int x, uint32_t stage) {
                const uint64_t dq = dq0 + x * kTileStep, dk = dk0 + stage * kTileStep;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = ((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4;
                    if (mma_lane) mma_ss(tmem + kColS + x * 128, dq + off, dk + off, idesc_s, ks > 0);
                }
                if (mma_lane) mma_commit(&sm.s_full[x]);
            };
            // O_x (+)= P_x V
            // (one half of the key columns: P arrives in two halves so that the first four K steps
            // run while the softmax warps still work on the second half)
            auto issue_pv = [&](int x, uint32_t stage, bool acc, int half) {
                const uint64_t dv = dv0 + stage * kTileStep + half * (kTileKV / 32) * (2048 >> 4);
                const uint32_t tp = tmem + kColS + x * 128 + half * (kTileKV / 32) * 8;
#pragma unroll
                for (int ks = 0; ks < kTileKV / 32; ++ks)
                    if (mma_lane) mma_ts(tmem + kColO + x * 128, tp + ks * 8, dv + ks * (2048 >> 4), idesc_o, acc || ks > 0);
            };
            uint32_t q_cnt = 0, qb_cnt = 0, kv_cnt = 0, p_cnt[2] = {0, 0};
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const bool has_b = wi.rows > kTileQ;
                const int n_a = key_tiles(sp, t, wi.unit, wi.row0, min(wi.rows, kTileQ));
                const int n_b = key_tiles(sp, t, wi.unit, wi.row0 + kTileQ, wi.rows - kTileQ);
                const int n_kv = max(n_a, n_b);
                if (n_kv == 0) continue;
                ZL_WAIT_WARP(&sm.q_full[0], q_cnt & 1, 11);
                ++q_cnt;
                // step j: P_A V(j), S_A(j + 1), P_B V(j), S_B(j + 1); one copy of each MMA group
#pragma unroll 1
                for (int j = -1; j < n_kv; ++j) {
                    const uint32_t s = (kv_cnt + j) % kStages, nk = kv_cnt + j + 1, sn = nk % kStages;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int n_x = x == 0 ? n_a : n_b;
                        if (j >= 0 && j < n_x) {
                            // P_x(j) is in TMEM (S_x(j) fully read, O_x rescaled if needed); K(j), V(j) were waited for
                            // when S(j) was issued
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                ZL_WAIT_WARP(&sm.p_half[x][half], p_cnt[x] & 1, 14);
                                tc_fence_after();
                                issue_pv(x, s, j > 0 || half > 0, half);
                            }
                            ++p_cnt[x];
                            if (j + 1 == n_x) if (mma_lane) mma_commit(&sm.o_full[x]);
                        }
                        if (x == 0) {
                            if (j + 1 < n_kv) ZL_WAIT_WARP(&sm.kv_full[sn], (nk / kStages) & 1, 16);
                        } else {
                            if (j >= 0) if (mma_lane) mma_commit(&sm.kv_empty[s]);  // S(j) and P(j) V of both tiles are the stage's last readers
                            if (j < 0 && has_b) {
                                ZL_WAIT_WARP(&sm.q_full[1], qb_cnt & 1, 13);
                                ++qb_cnt;
                            }
                        }
                        if (j + 1 < n_x) {
                            tc_fence_after();
                            issue_s(x, sn);  // overwrites P_x(j): ordered after P_x V on the tensor pipe
                        }
                    }
                    if (j + 2 == n_kv) if (mma_lane) mma_commit(&sm.q_empty);  // last S of the item issued
                }
                kv_cnt += n_kv;
            }
        } else if (kBias && warp >= 2) {  // (the other lanes of warp 0 have nothing to do)
            // -------------------------------------------------------------- biases of near tiles: warp 2 tile A, warp 3 tile B
            const int x = warp - 2;
            WindowFeed feed{&sm.bias_full[x], &sm.bias_empty[x], sm.window[x]};
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const TaskPos tp = task_pos(sp, wi.unit);
                const int row0 = wi.row0 + x * kTileQ;
                const int n_kv = key_tiles(sp, t, wi.unit, row0, min(kTileQ, wi.rows - x * kTileQ));
                HeadBias hb;
                hb.load(sp, wi.head);
                for (int j = 0; j < n_kv; ++j) {
                    const int lo = tp.kv_pos + j * kTileKV - (tp.q_pos + row0 + kTileQ - 1);
                    if (patch_side(sp, lo, lo + kTileQ + kTileKV - 2) != kNear) continue;
                    if (!feed.put(sp, hb, wi.head, lo, lane, &sm.abort_flag)) {
                        report(p.status, &sm.abort_flag, 3000 + 31);
                        goto teardown;
                    }
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax + epilogue
        reg_inc<216>();
        const int x = (warp - 4) >> 2;             // 0: tile A, 1: tile B
        const int quarter = warp & 3;              // TMEM lane quarter this warp may access
        const int row = quarter * 32 + lane;       // query row within the tile
        const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t col_s = kColS + x * 128, col_o = kColO + x * 128;
        uint32_t s_cnt = 0, o_cnt = 0;
        const bool store_leader = quarter == 0 && lane == 0;  // one thread per warpgroup issues its TMA stores
        bool store_pending = false;                            // this warpgroup's box may still be read by a store
        uint32_t bias_cnt = 0;
        for (int it = walk.first; it < walk.end; it += walk.step) {
            const WorkItem wi = p.items[it];
            const int tile_rows = min(kTileQ, wi.rows - x * kTileQ);  // rows of this warpgroup's tile
            if (tile_rows <= 0) continue;
            const Task t = p.tasks[wi.unit];
            const TaskPos tp = task_pos(sp, wi.unit);
            const int row0 = wi.row0 + x * kTileQ;  // first row of the tile, relative to the task
            const int n_kv = key_tiles(sp, t, wi.unit, row0, tile_rows);
            const int keys = sp.masked ? visible_keys(tp, t.kv_len, row0 + row) : t.kv_len;  // this row's
            HeadBias hb;
            if constexpr (kBias) hb.load(sp, wi.head);
            float m_ref = -INFINITY, l = 0.f;  // reference maximum (powers of two) and row sum
            for (int j = 0; j < n_kv; ++j) {
                const int dist_lo = tp.kv_pos + j * kTileKV - (tp.q_pos + row0 + kTileQ - 1);  // last row, first column
                const PatchSide side = kBias ? patch_side(sp, dist_lo, dist_lo + kTileQ + kTileKV - 2) : kNear;
                const bool ragged = __any_sync(0xffffffffu, keys - j * kTileKV < kTileKV);
                ZL_WAIT_REGS(&sm.s_full[x], s_cnt & 1, 21);
                ++s_cnt;
                if (kBias && side == kNear) {
                    ZL_WAIT_REGS(&sm.bias_full[x], bias_cnt & 1, 22);
                    ++bias_cnt;
                }
                tc_fence_after();
                float sv[kTileKV];
#pragma unroll
                for (int c = 0; c < kTileKV / 32; ++c) {
                    uint32_t r[32];
                    tmem_ld_x32(lane_addr + col_s + c * 32, r);
#pragma unroll
                    for (int i = 0; i < 32; ++i) sv[c * 32 + i] = __uint_as_float(r[i]);
                }
                tmem_wait_ld();
                softmax_tile<D, kCap, kBias>(sv, sp, hb, p.scale_log2, j == 0, side, sm.window[x] + kTileQ - 1 - row, &sm.bias_empty[x],
                                             dist_lo + kTileQ - 1 - row, keys - j * kTileKV, ragged, true, lane_addr + col_s, lane_addr + col_o,
                                             sm.p_half[x], m_ref, l);
            }
            // ---- epilogue
            const bool row_ok = row < tile_rows;
            const float inv_l = (l > 0.f) ? 1.f / l : 0.f;
            const float lse = (l > 0.f) ? (m_ref + log2f(l)) * 0.6931471805599453f : -INFINITY;
            if (n_kv > 0) {
                ZL_WAIT_REGS(&sm.o_full[x], o_cnt & 1, 23);
                ++o_cnt;
                tc_fence_after();
            }
            const int64_t grow0 = (int64_t)(t.partial_slot >= 0 ? t.partial_slot : t.q_off) + row0;
            const int64_t grow = grow0 + row;
            if (tile_rows == kTileQ && n_kv > 0) {
                // full tile: stage 128 bytes per row at a time in this warpgroup's box and write each box
                // with one TMA store -- coalesced, and the warpgroup is free for the next item while the
                // copy engine drains the box
                const uint32_t box_row = smem_u32(sm.o_stage[x]) + row * 128;
                if (t.partial_slot >= 0) {
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {  // 32 fp32 columns per box
                        if (c > 0 || store_pending) {
                            if (store_leader) bulk_wait_group_read<0>();
                            named_bar_sync(2 + x, 128);
                        }
                        uint32_t r[32];
                        tmem_ld_x32(lane_addr + col_o + c * 32, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int k4 = 0; k4 < 8; ++k4)
                            st_shared_v4(box_row + ((k4 ^ (row & 7)) << 4),
                                         __float_as_uint(__uint_as_float(r[k4 * 4]) * inv_l),
                                         __float_as_uint(__uint_as_float(r[k4 * 4 + 1]) * inv_l),
                                         __float_as_uint(__uint_as_float(r[k4 * 4 + 2]) * inv_l),
                                         __float_as_uint(__uint_as_float(r[k4 * 4 + 3]) * inv_l));
                        fence_proxy_async_smem();
                        named_bar_sync(2 + x, 128);
                        if (store_leader) {
                            tma_store_3d(&tm_op, sm.o_stage[x], c * 32, wi.head, (int32_t)grow0);
                            bulk_commit_group();
                        }
                    }
                    p.lse_partial[(int64_t)wi.head * p.partial_rows + grow] = lse;
                } else {
#pragma unroll 1
                    for (int b = 0; b < D / 64; ++b) {  // 64 bf16 columns per box
                        if (b > 0 || store_pending) {
                            if (store_leader) bulk_wait_group_read<0>();
                            named_bar_sync(2 + x, 128);
                        }
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            uint32_t r[32];
                            tmem_ld_x32(lane_addr + col_o + b * 64 + c * 32, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4) {
                                const int i = k4 * 8;
                                st_shared_v4(box_row + (((c * 4 + k4) ^ (row & 7)) << 4),
                                             pack_bf16(__uint_as_float(r[i]) * inv_l, __uint_as_float(r[i + 1]) * inv_l),
                                             pack_bf16(__uint_as_float(r[i + 2]) * inv_l, __uint_as_float(r[i + 3]) * inv_l),
                                             pack_bf16(__uint_as_float(r[i + 4]) * inv_l, __uint_as_float(r[i + 5]) * inv_l),
                                             pack_bf16(__uint_as_float(r[i + 6]) * inv_l, __uint_as_float(r[i + 7]) * inv_l));
                            }
                        }
                        fence_proxy_async_smem();
                        named_bar_sync(2 + x, 128);
                        if (store_leader) {
                            tma_store_3d(&tm_o, sm.o_stage[x], b * 64, wi.head, (int32_t)grow0);
                            bulk_commit_group();
                        }
                    }
                    p.lse[(int64_t)wi.head * p.total_q + grow] = lse;
                }
                store_pending = true;
            } else if (t.partial_slot >= 0) {
                float* dst = p.o_partial + (grow * p.n_heads + wi.head) * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t r[32];
                    if (n_kv > 0) {
                        tmem_ld_x32(lane_addr + col_o + c * 32, r);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0;
                    }
                    if (row_ok) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float4 o4 = make_float4(__uint_as_float(r[i]) * inv_l, __uint_as_float(r[i + 1]) * inv_l,
                                                    __uint_as_float(r[i + 2]) * inv_l, __uint_as_float(r[i + 3]) * inv_l);
                            *reinterpret_cast<float4*>(dst + c * 32 + i) = o4;
                        }
                    }
                }
                if (row_ok) p.lse_partial[(int64_t)wi.head * p.partial_rows + grow] = lse;
            } else {
                __nv_bfloat16* dst = p.o + (grow * p.n_heads + wi.head) * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t r[32];
                    if (n_kv > 0) {
                        tmem_ld_x32(lane_addr + col_o + c * 32, r);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0;
                    }
                    if (row_ok) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint4 o4;
                            o4.x = pack_bf16(__uint_as_float(r[i]) * inv_l, __uint_as_float(r[i + 1]) * inv_l);
                            o4.y = pack_bf16(__uint_as_float(r[i + 2]) * inv_l, __uint_as_float(r[i + 3]) * inv_l);
                            o4.z = pack_bf16(__uint_as_float(r[i + 4]) * inv_l, __uint_as_float(r[i + 5]) * inv_l);
                            o4.w = pack_bf16(__uint_as_float(r[i + 6]) * inv_l, __uint_as_float(r[i + 7]) * inv_l);
                            *reinterpret_cast<uint4*>(dst + c * 32 + i) = o4;
                        }
                    }
                }
                if (row_ok) p.lse[(int64_t)wi.head * p.total_q + grow] = lse;
            }
            tc_fence_before();
        }
        if (store_leader) bulk_wait_group<0>();  // the last O stores have left shared memory and landed
    }

teardown:
    // Also reached after an expired wait: bulk stores this thread has committed must have finished
    // reading shared memory before the CTA gives it up (a no-op on the normal path).
    bulk_wait_group<0>();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <int D, bool kCap, bool kBias>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& to,
                     const CUtensorMap& top, const FwdParams& p, const ScoreParams& sp, int grid, cudaStream_t stream) {
    constexpr int smem = sizeof(ScoredFwdSmem<D>);
    // the opt-in to large dynamic shared memory is a per-device attribute of the kernel
    constexpr int kMaxDevices = 64;
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_scored_fwd_kernel<D, kCap, kBias>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    return launch_dependent(zl_scored_fwd_kernel<D, kCap, kBias>, grid, kFwdThreads, smem, stream, true, tq, tk, tv, to, top, p, sp);
}

template <int D>
cudaError_t launch_d(bool capped, bool biased, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                     const CUtensorMap& to, const CUtensorMap& top, const FwdParams& p, const ScoreParams& sp, int grid,
                     cudaStream_t stream) {
    if (capped)
        return biased ? launch_t<D, true, true>(tq, tk, tv, to, top, p, sp, grid, stream)
                      : launch_t<D, true, false>(tq, tk, tv, to, top, p, sp, grid, stream);
    return biased ? launch_t<D, false, true>(tq, tk, tv, to, top, p, sp, grid, stream)
                  : launch_t<D, false, false>(tq, tk, tv, to, top, p, sp, grid, stream);
}

}  // namespace

cudaError_t launch_scored_fwd(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                              const CUtensorMap& tv, const CUtensorMap& to, const CUtensorMap& top, const FwdParams& p,
                              const ScoreParams& sp, int grid, cudaStream_t stream) {
    if (p.n_items == 0) return cudaSuccess;
    return head_dim == 128 ? launch_d<128>(capped, kind != kScorePlain, tq, tk, tv, to, top, p, sp, grid, stream)
                           : launch_d<64>(capped, kind != kScorePlain, tq, tk, tv, to, top, p, sp, grid, stream);
}

}  // namespace zl
