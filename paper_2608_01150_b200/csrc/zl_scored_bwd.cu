// Backward main kernel of scored attention (sm_100a).
//
//     P = exp(s - LSE),  G = P o (dO V^T - D),  dS = G C'(scale q.k)
//     dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K,  dtable[b][h] = sum of G over the pairs in bucket b
//
// Structure as zl_bwd_main_kernel (zl_bwd.cu), whose preprocess and dQ conversion it shares: a persistent CTA owns a
// 128-row key tile of one head, keeps K, V in shared memory and dK, dV in TMEM, and loops over the query tiles; S^T and
// dP^T come out of the tensor core with a key row per thread.  What differs:
//   * Under the prefix mask a key tile is seen by a trailing stretch of query tiles (first_query()), so the loop starts
//     there; a column below the thread's own first query is masked by one compare.
//   * Without a cap the product already holds -LSE / scale (the augmentation step), and the bias is added to it.  With
//     a cap the tanh needs the bare product: no augmentation step for S^T, the LSE comes from shared memory.
//   * G is formed in fp32 from the unrounded P and rounded once, as dS, on its way to the tensor core: the table's
//     gradient is a sum of large cancelling terms and is fp32 from end to end.
//   * The table's gradient needs the sums of G over diagonals.  A warp's patch of 32 keys x 64 queries either lies in the
//     constant part of the bias (one running sum per thread and side) or near the diagonal: there a register per lane
//     carries one diagonal's sum, moves one lane per column and is complete when it leaves lane 31, all of it while the
//     tensor core works on dS; the 95 sums are reduced by bucket (runs of equal buckets by shuffles) into registers
//     that hold two buckets per lane.  At the end of an item the eight warps' 64 sums are added in order and stored; the dQ
//     conversion's launch adds the key tiles in order.  No atomics: the same bits every time.
// Measured (B200): slopes over 9450 tokens, 12 heads, d 128: 1.31 ms of the whole backward's 1.34 (1.02 PFLOP/s, as the plain kernel
// of this form); 16 texts of up to 512 tokens, 12 heads, d 64: 83 us without and 107 us with the table's gradient.  Bound by the
// hand-overs between the MMA issuer and the P/dS warps as zl_bwd_main_kernel is, and with short sequences by the ends of items.
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "zl_score.cuh"

namespace zl {

using namespace ptx;
using namespace score;

namespace {

// Warp roles (16 warps): warp 0 TMA producer, warp 1 MMA issuer, warps 2-3 idle,
// warps 4-7 and 8-11 two P/dS warpgroups (query columns 0-63 and 64-127 of every tile, one key
// row per thread), warps 12-15 dQ warpgroup (one query row per thread).
constexpr int kBwdThreads = 512;

constexpr int kPatch = 96;  // distances of a patch of 32 keys x 64 queries: 32 + 64 - 1, rounded up

// Sums over the diagonals of a patch run in kChains stretches of columns side by side: a step of one stretch (a shuffle and an
// add, some 30 clocks one after the other) waits only for the step before it.  More stretches take more shared memory
// for their sums, which head_dim 128 does not have.
template <int D>
struct DiagSums {
    static constexpr int kChains = D == 64 ? 4 : 2;
    static constexpr int kCols = 64 / kChains;        // columns of a stretch
    static constexpr int kStride = 32 + kCols;        // its 31 + kCols diagonals, and one
    static constexpr int kFloats = kChains * kStride > kPatch ? kChains * kStride : kPatch;
};

template <int D, bool kCap>
struct ScoredBwdSmem {
    static constexpr int kTileBytes = 128 * D * 2;
    static constexpr int kBoxBytes = 128 * 128;
    static constexpr int kBoxes = D / 64;
    static constexpr int kDqChunkBytes = 128 * 32 * 4;  // 128 query rows x 32 fp32 columns
    alignas(1024) uint8_t k[kTileBytes];
    alignas(1024) uint8_t v[kTileBytes];
    alignas(1024) uint8_t q[2][kTileBytes];
    alignas(1024) uint8_t d_o[kTileBytes];
    alignas(1024) uint8_t ds[2 * kBoxBytes];            // dS^T tile: 128 key rows x 128 query columns, bf16
    alignas(1024) uint8_t dq_stage[kDqChunkBytes];      // one fp32 dQ chunk staged for the TMA reduce
    alignas(1024) uint8_t aug[2][4096];                 // per Q stage: bf16 pieces of -LSE/scale and -D
    alignas(1024) uint8_t ones[kCap ? 2 : 3][2048];     // [zeros][ones in elements 0..2] and, for the step of S^T, [zeros]
    alignas(16) float lse[kCap ? 2 : 1][kCap ? kTileQ : 4];  // per Q stage, capped scores: LSE * log2(e)
    float window[8][DiagSums<D>::kFloats];              // per P/dS warp: biases, then sums over diagonals
    alignas(8) uint64_t kv_full, kv_empty;
    uint64_t q_full[2], q_empty[2], do_full, do_empty;
    uint64_t sums_full, sums_empty;
    uint64_t s_full, dp_full, p_full, ds_full, ds_free, dq_full, dq_empty, acc_full;
    uint32_t tmem_base;
    volatile int32_t abort_flag;
};

#define ZL_WAIT(bar, parity, site)                                        \
    do {                                                                  \
        if (!wait((bar), (parity), &sm.abort_flag)) { \
            report(p.status, &sm.abort_flag, 4000 + (site));              \
            goto teardown;                                                \
        }                                                                 \
    } while (0)
#define ZL_WAIT_WARP(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 4000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)
// The same from the warps that hold tiles in registers.
#define ZL_WAIT_REGS(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait_inline((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 4000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)

// First query tile of `task` that sees any key of the tile at key row `row0`, at most the number of tiles.
__device__ __forceinline__ int first_tile(const ScoreParams& sp, const Task& t, int task, int row0) {
    const int n_q = (t.q_len + kTileQ - 1) / kTileQ;
    return sp.masked ? min(n_q, first_query(task_pos(sp, task), row0) / kTileQ) : 0;
}
// Number of 128-row query tiles a kv group's CTA iterates over.
__device__ __forceinline__ int count_q_tiles(const BwdParams& p, const ScoreParams& sp, const KvGroup& g, int row0) {
    int n = 0;
    for (int ti = 0; ti < g.n_tasks; ++ti) {
        const int task = p.kv_group_tasks[g.task_begin + ti];
        const Task t = p.tasks[task];
        n += (t.q_len + kTileQ - 1) / kTileQ - first_tile(sp, t, task, row0);
    }
    return n;
}

// Adds the sums v[i] of distances 32 i + lane (bucket b[i], -1 for none) to a table of kMaxBuckets sums in shared memory that
// only this warp uses.  Among 32 consecutive distances runs of equal buckets are summed by shuffles; where a bucket has
// several runs their sums are added one after the other, in lane order.  (One copy of the code: the instruction cache counts
// for more here than three chains side by side.)
__device__ __forceinline__ void add_by_bucket(float* sums, const float (&v)[kPatch / 32], const int (&b)[kPatch / 32], int lane) {
    static_assert(kPatch / 32 == 3, "");
#pragma unroll 1
    for (int i = 0; i < kPatch / 32; ++i) {
        float x = i == 0 ? v[0] : (i == 1 ? v[1] : v[2]);
        const int bucket = i == 0 ? b[0] : (i == 1 ? b[1] : b[2]);
        const int before = __shfl_up_sync(0xffffffffu, bucket, 1);
        const uint32_t heads = __ballot_sync(0xffffffffu, lane == 0 || bucket != before);
        const uint32_t later = heads & (0xfffffffeu << lane);  // run starts after this lane
        const int run = (later ? __ffs(later) - 1 : 32) - lane;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const float o = __shfl_down_sync(0xffffffffu, x, off);
            if (off < run) x += o;
        }
        const bool head = ((heads >> lane) & 1u) && bucket >= 0;
        const uint32_t same = __match_any_sync(0xffffffffu, head ? bucket : -1 - lane);
        const int rank = __popc(same & ((1u << lane) - 1u));
        const int rounds = __reduce_max_sync(0xffffffffu, head ? rank : 0);
#pragma unroll 1
        for (int r = 0; r <= rounds; ++r) {
            if (head && rank == r) sums[bucket] += x;
            __syncwarp();
        }
    }
}

template <int D, bool kCap, ScoreKind kKind>
__global__ void __launch_bounds__(kBwdThreads, 1)
zl_scored_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do,
                   const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                   const __grid_constant__ CUtensorMap tm_dv, const BwdParams p, const ScoreParams sp) {
    constexpr bool kBias = kKind != kScorePlain, kGrad = kKind == kScoreBiasGrad;
    using Smem = ScoredBwdSmem<D, kCap>;
    constexpr int kBoxes = Smem::kBoxes;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    // TMEM columns: S^T / P^T [0,128), dP^T / dQ [128,256), dV [256,256+D), dK [384,384+D)
    constexpr uint32_t kColS = 0, kColDP = 128, kColDV = 256, kColDK = 384, kTmemCols = 512;

    if ((smem_u32(smem_raw) & 1023u) != 0) {  // swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0 && atomicCAS(p.status, 0, (int)ZL_ERR_CUDA) == 0) p.status[1] = 4999;
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&sm.kv_full, 1);
        mbar_init(&sm.kv_empty, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm.q_full[s], 1);
            mbar_init(&sm.q_empty[s], 1);
        }
        mbar_init(&sm.do_full, 1);
        mbar_init(&sm.do_empty, 1);
        mbar_init(&sm.s_full, 1);
        mbar_init(&sm.dp_full, 1);
        mbar_init(&sm.p_full, 256);
        mbar_init(&sm.ds_full, 256);
        mbar_init(&sm.ds_free, 1);
        mbar_init(&sm.dq_full, 1);
        mbar_init(&sm.dq_empty, 128);
        mbar_init(&sm.acc_full, 1);
        mbar_init(&sm.sums_full, 256);
        mbar_init(&sm.sums_empty, 256);
        sm.abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        prefetch_tmap(&tm_do);
        prefetch_tmap(&tm_dq);
        prefetch_tmap(&tm_dk);
        prefetch_tmap(&tm_dv);
    }
    // constant A operand of the augmentation steps: 128 rows x 8 bf16 per block
    for (int i = threadIdx.x; i < (int)sizeof(sm.ones) / 4; i += kBwdThreads) {
        const int blk = i / 512, w = i % 4;  // w: 32-bit word inside the row's 16 bytes
        uint32_t val = 0;
        if (blk == 1) val = (w == 0) ? 0x3F803F80u : (w == 1 ? 0x00003F80u : 0u);
        reinterpret_cast<uint32_t*>(&sm.ones[0][0])[i] = val;
    }
    fence_proxy_async_smem();
    if (warp == 1) {
        tmem_alloc(&sm.tmem_base, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem_base;
    grid_wait();
    const Walk walk(p);

    if (warp < 4) {
        reg_dec<72>();
        if (warp == 0 && lane == 0) {
            // -------------------------------------------------------------- TMA producer
            uint32_t item_cnt = 0, it_cnt = 0;
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const KvGroup g = p.kv_groups[wi.unit];
                if (count_q_tiles(p, sp, g, wi.row0) == 0) continue;  // no query sees these keys
                ZL_WAIT(&sm.kv_empty, (item_cnt & 1) ^ 1, 1);
                mbar_arrive_expect_tx(&sm.kv_full, 2 * Smem::kTileBytes);
                for (int b = 0; b < kBoxes; ++b) {
                    tma_load_3d(sm.k + b * Smem::kBoxBytes, &tm_k, &sm.kv_full, b * 64, wi.head, g.kv_off + wi.row0);
                    tma_load_3d(sm.v + b * Smem::kBoxBytes, &tm_v, &sm.kv_full, b * 64, wi.head, g.kv_off + wi.row0);
                }
                ++item_cnt;
                for (int ti = 0; ti < g.n_tasks; ++ti) {
                    const int task = p.kv_group_tasks[g.task_begin + ti];
                    const Task t = p.tasks[task];
                    const int n_q = (t.q_len + kTileQ - 1) / kTileQ;
                    for (int qt = first_tile(sp, t, task, wi.row0); qt < n_q; ++qt, ++it_cnt) {
                        const int s = it_cnt & 1;
                        ZL_WAIT(&sm.q_empty[s], ((it_cnt >> 1) & 1) ^ 1, 2);
                        mbar_arrive_expect_tx(&sm.q_full[s], Smem::kTileBytes + 4096 + (kCap ? kTileQ * 4 : 0));
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_3d(sm.q[s] + b * Smem::kBoxBytes, &tm_q, &sm.q_full[s], b * 64, wi.head,
                                        t.q_off + qt * kTileQ);
                        const int64_t tile = (int64_t)wi.head * (p.q_pad_total / kTileQ) + t.q_slot / kTileQ + qt;
                        bulk_load_1d(sm.aug[s], p.aug + tile * 4096, 4096, &sm.q_full[s]);
                        if constexpr (kCap) bulk_load_1d(sm.lse[s], p.lse_tiles + tile * kTileQ, kTileQ * 4, &sm.q_full[s]);
                        ZL_WAIT(&sm.do_empty, (it_cnt & 1) ^ 1, 3);
                        mbar_arrive_expect_tx(&sm.do_full, Smem::kTileBytes);
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_3d(sm.d_o + b * Smem::kBoxBytes, &tm_do, &sm.do_full, b * 64, wi.head,
                                        t.q_off + qt * kTileQ);
                    }
                }
            }
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMA issuer
            // The whole warp runs this loop converged and one elected lane issues: descriptors
            // and barrier addresses then stay warp-uniform, which makes commits and satisfied
            // waits several times cheaper than from a single diverged thread.
            const bool mma_lane = elect_one();
            constexpr uint32_t idesc_s = make_idesc_bf16(128, 128, 0, 0);   // S^T, dP^T: K-major x K-major
            constexpr uint32_t idesc_dv = make_idesc_bf16(128, D, 0, 1);    // A in TMEM / K-major smem, B MN-major
            constexpr uint32_t idesc_dq = make_idesc_bf16(128, D, 1, 1);    // A MN-major smem, B MN-major
            // Descriptors are built once; stepping along K only adds a byte offset (>> 4) to the
            // start-address field, which cannot overflow for shared-memory addresses.
            const uint64_t dk_k = make_desc_sw128(smem_u32(sm.k), 16, 1024);                   // K tile, K-major
            const uint64_t dk_mn = make_desc_sw128(smem_u32(sm.k), Smem::kBoxBytes, 1024);     // K tile, MN-major
            const uint64_t dv_k = make_desc_sw128(smem_u32(sm.v), 16, 1024);
            const uint64_t ddo_k = make_desc_sw128(smem_u32(sm.d_o), 16, 1024);
            const uint64_t ddo_mn = make_desc_sw128(smem_u32(sm.d_o), Smem::kBoxBytes, 1024);
            const uint64_t dds_k = make_desc_sw128(smem_u32(sm.ds), 16, 1024);
            const uint64_t dds_mn = make_desc_sw128(smem_u32(sm.ds), Smem::kBoxBytes, 1024);
            const uint64_t dq_k0 = make_desc_sw128(smem_u32(sm.q[0]), 16, 1024);
            const uint64_t dq_mn0 = make_desc_sw128(smem_u32(sm.q[0]), Smem::kBoxBytes, 1024);
            const uint64_t daug0 = make_desc_noswizzle(smem_u32(sm.aug[0]), 2048, 128);
            const uint64_t dones_s = make_desc_noswizzle(smem_u32(&sm.ones[1][0]), 2048, 128);  // ones, then zeros
            const uint64_t dones_dp = make_desc_noswizzle(smem_u32(&sm.ones[0][0]), 2048, 128); // zeros, then ones
            constexpr uint32_t kQStageStep = Smem::kTileBytes >> 4, kAugStageStep = 4096 >> 4;
            // S^T = K Q^T, without a cap - LSE/scale: the last step multiplies the ones block with the LSE pieces
            auto issue_s = [&](uint32_t stage) {
                const uint64_t dq = dq_k0 + stage * kQStageStep;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = ((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4;
                    if (mma_lane) mma_ss(tmem + kColS, dk_k + off, dq + off, idesc_s, ks > 0);
                }
                if constexpr (!kCap)
                    if (mma_lane) mma_ss(tmem + kColS, dones_s, daug0 + stage * kAugStageStep, idesc_s, true);
                if (mma_lane) mma_commit(&sm.s_full);
            };
            // dP^T = V dO^T - D: the ones sit in the second K chunk, where the tile holds the D pieces
            auto issue_dp = [&](uint32_t stage) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = ((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4;
                    if (mma_lane) mma_ss(tmem + kColDP, dv_k + off, ddo_k + off, idesc_s, ks > 0);
                }
                if (mma_lane) mma_ss(tmem + kColDP, dones_dp, daug0 + stage * kAugStageStep, idesc_s, true);
                if (mma_lane) mma_commit(&sm.dp_full);
            };
            auto issue_dv = [&](bool acc) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)  // dV += P^T dO, K = 128 query rows
                    if (mma_lane) mma_ts(tmem + kColDV, tmem + kColS + (ks / 4) * 64 + (ks % 4) * 8, ddo_mn + ks * (2048 >> 4), idesc_dv,
                           acc || ks > 0);
                if (mma_lane) mma_commit(&sm.do_empty);
            };
            uint32_t item_cnt = 0, it_cnt = 0;
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const KvGroup g = p.kv_groups[wi.unit];
                const int n_it = count_q_tiles(p, sp, g, wi.row0);
                if (n_it == 0) continue;
                ZL_WAIT_WARP(&sm.kv_full, item_cnt & 1, 11);
                ++item_cnt;
                // prologue: S, dP, dV of the item's first query tile and S of the second.
                // Steady-state order on the tensor pipe: dQ(i) dK(i) dP(i+1) dV(i+1) S(i+2).
                ZL_WAIT_WARP(&sm.q_full[it_cnt & 1], (it_cnt >> 1) & 1, 12);
                tc_fence_after();
                issue_s(it_cnt & 1);
                ZL_WAIT_WARP(&sm.do_full, it_cnt & 1, 13);
                ZL_WAIT_WARP(&sm.dq_empty, (it_cnt & 1) ^ 1, 14);  // previous dQ tile drained from the dP columns
                tc_fence_after();
                issue_dp(it_cnt & 1);
                ZL_WAIT_WARP(&sm.p_full, it_cnt & 1, 15);
                tc_fence_after();
                issue_dv(false);
                if (n_it > 1) {
                    const uint32_t n1 = it_cnt + 1;
                    ZL_WAIT_WARP(&sm.q_full[n1 & 1], (n1 >> 1) & 1, 16);
                    tc_fence_after();
                    issue_s(n1 & 1);  // overwrites P^T: ordered after dV on the tensor pipe
                }
                for (int i = 0; i < n_it; ++i, ++it_cnt) {
                    const uint64_t dq_mn = dq_mn0 + (it_cnt & 1) * kQStageStep;
                    ZL_WAIT_WARP(&sm.ds_full, it_cnt & 1, 17);
                    tc_fence_after();
                    {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)  // dQ = dS K, K = 128 key rows; lands in the dP columns
                            if (mma_lane) mma_ss(tmem + kColDP, dds_mn + ks * (2048 >> 4), dk_mn + ks * (2048 >> 4), idesc_dq, ks > 0);
                        if (mma_lane) mma_commit(&sm.dq_full);  // dQ first: its drain from TMEM runs under the dK MMAs
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) {  // dK += dS^T Q, K = 128 query rows
                            const uint32_t off = ((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4;
                            if (mma_lane) mma_ss(tmem + kColDK, dds_k + off, dq_mn + ks * (2048 >> 4), idesc_dv, i > 0 || ks > 0);
                        }
                        if (mma_lane) mma_commit(&sm.q_empty[it_cnt & 1]);
                        if (mma_lane) mma_commit(&sm.ds_free);
                    }
                    if (i + 1 < n_it) {
                        const uint32_t n1 = it_cnt + 1, n2 = it_cnt + 2;
                        ZL_WAIT_WARP(&sm.do_full, n1 & 1, 18);
                        ZL_WAIT_WARP(&sm.dq_empty, it_cnt & 1, 19);
                        tc_fence_after();
                        issue_dp(n1 & 1);
                        ZL_WAIT_WARP(&sm.p_full, n1 & 1, 20);
                        tc_fence_after();
                        issue_dv(true);
                        if (i + 2 < n_it) {
                            ZL_WAIT_WARP(&sm.q_full[n2 & 1], (n2 >> 1) & 1, 16);
                            tc_fence_after();
                            issue_s(n2 & 1);
                        }
                    }
                }
                if (mma_lane) mma_commit(&sm.acc_full);
                if (mma_lane) mma_commit(&sm.kv_empty);
            }
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------------ P / dS warpgroups
        reg_inc<144>();
        const int wg = (warp - 4) >> 2;            // 0: query columns 0-63, 1: columns 64-127
        const int quarter = warp & 3;
        const int row = quarter * 32 + lane;       // key row within the tile
        const int col0 = wg * 64;
        const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t ds_row_addr = smem_u32(sm.ds) + row * 128;
        uint32_t item_cnt = 0, it_cnt = 0, sums_cnt = 0;
        const bool store_leader = (warp & 3) == 0 && lane == 0;  // one thread per warpgroup issues its TMA stores
        bool store_pending = false;
        float* const window = sm.window[warp - 4];
        for (int it = walk.first; it < walk.end; it += walk.step) {
            const WorkItem wi = p.items[it];
            const KvGroup g = p.kv_groups[wi.unit];
            const bool row_ok = row < wi.rows;
            HeadBias hb;
            if constexpr (kBias) hb.load(sp, wi.head);
            float far_sum[2] = {0.f, 0.f};             // this thread's G beyond the reach: distances <= -reach, >= reach
            float bucket_sum[2] = {0.f, 0.f};          // this warp's G by bucket: buckets lane and lane + 32
            const uint32_t it_first = it_cnt;
            for (int ti = 0; ti < g.n_tasks; ++ti) {
                const int task = p.kv_group_tasks[g.task_begin + ti];
                const Task t = p.tasks[task];
                const TaskPos tp = task_pos(sp, task);
                const int n_q = (t.q_len + kTileQ - 1) / kTileQ;
                const int first = sp.masked ? first_query(tp, wi.row0 + row) : 0;  // first query row that sees this key
                for (int qt = first_tile(sp, t, task, wi.row0); qt < n_q; ++qt, ++it_cnt) {
                    const int stage = it_cnt & 1;
                    // columns of this thread's 64 that count: [col_lo, col_hi)
                    const int col_lo = first - qt * kTileQ - col0;
                    const int col_hi = row_ok ? t.q_len - qt * kTileQ - col0 : 0;
                    const bool tile_full = __all_sync(0xffffffffu, col_lo <= 0 && col_hi >= 64);
                    const int dist_lo = tp.kv_pos + wi.row0 + quarter * 32 - (tp.q_pos + qt * kTileQ + col0 + 63);  // first row, last column
                    PatchSide side = kNear;
                    float near_bias[kPatch / 32];
                    int near_bucket[kPatch / 32];
                    if constexpr (kBias) {
                        side = patch_side(sp, dist_lo, dist_lo + 31 + 63);
                        if (side == kNear) {
#pragma unroll
                            for (int i = 0; i < kPatch / 32; ++i) {
                                const int d = dist_lo + i * 32 + lane;
                                near_bias[i] = hb.at(sp, wi.head, d);
                                if constexpr (kGrad) near_bucket[i] = i * 32 + lane < 95 ? bucket_at(sp, d) : -1;
                            }
                        }
                    }
                    ZL_WAIT_REGS(&sm.s_full, it_cnt & 1, 22);
                    if constexpr (kCap) ZL_WAIT_REGS(&sm.q_full[stage], (it_cnt >> 1) & 1, 26);  // the LSE came with Q: already complete
                    tc_fence_after();
                    float pr[64];        // P of this thread's key row, fp32
                    // C' of the capped scores, pairs of fp16: off by at most 2^-11 of the value down to 2^-14, by 2^-25 below.  There 1 - tanh^2 in
                    // fp32 holds no more: it carries twice the error of the tanh, some 2^-21 near 1
                    uint32_t slope[32];
                    {
                        uint32_t sr[2][32];
                        tmem_ld_x32(lane_addr + kColS + col0, sr[0]);
                        tmem_ld_x32(lane_addr + kColS + col0 + 32, sr[1]);
                        if constexpr (kBias) {
                            if (side == kNear) {
                                __syncwarp();  // what the window held has been read
#pragma unroll
                                for (int i = 0; i < kPatch / 32; ++i) window[i * 32 + lane] = near_bias[i];
                                __syncwarp();
                            }
                        }
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 64; ++c) pr[c] = __uint_as_float(sr[c >> 5][c & 31]);
                    }
                    float mul = p.scale_log2;
                    if constexpr (kCap) {
                        mul = 1.f;
                        if (!tile_full) {
                            // products with rows of other tasks, or of none: C' must not come from them (here finite rows give
                            // +-inf at most, hence a C' of 0, but nothing promises that an overflowing sum is never NaN)
#pragma unroll
                            for (int c = 0; c < 64; ++c)
                                if (c < col_lo || c >= col_hi) pr[c] = 0.f;
                        }
                        float big = 0.f;
#pragma unroll
                        for (int c = 0; c < 64; c += 2) big = max3_abs(big, pr[c], pr[c + 1]);
                        const float2 k1 = splat(sp.scale_over_cap), cl = splat(sp.cap_log2);
                        const float4* lse4 = reinterpret_cast<const float4*>(sm.lse[stage] + col0);
                        if (__all_sync(0xffffffffu, big * sp.scale_over_cap <= kTanhRange)) {
#pragma unroll
                            for (int c = 0; c < 64; c += 2) {
                                const float2 th = tanh_near(mul2(make_float2(pr[c], pr[c + 1]), k1));
                                pr[c] = th.x;
                                pr[c + 1] = th.y;
                            }
                        } else {  // each product in the form that fits it: a warp's may be small in one row and saturate in another
#pragma unroll
                            for (int c = 0; c < 64; c += 2) {
                                const float2 y = mul2(make_float2(pr[c], pr[c + 1]), k1);
                                const float2 th = tanh_near(y);
                                pr[c] = fabsf(y.x) <= kTanhRange ? th.x : tanh_far(y.x);
                                pr[c + 1] = fabsf(y.y) <= kTanhRange ? th.y : tanh_far(y.y);
                            }
                        }
#pragma unroll
                        for (int c = 0; c < 64; c += 4) {
                            const float4 ls = lse4[c / 4];
#pragma unroll
                            for (int e = 0; e < 4; e += 2) {
                                float2 th = make_float2(pr[c + e], pr[c + e + 1]);
                                const float2 cp = fma2(make_float2(-th.x, -th.y), th, splat(1.f));
                                const __half2 h2 = __floats2half2_rn(cp.x, cp.y);
                                slope[(c + e) / 2] = *reinterpret_cast<const uint32_t*>(&h2);
                                th = fma2(th, cl, e == 0 ? make_float2(-ls.x, -ls.y) : make_float2(-ls.z, -ls.w));
                                pr[c + e] = th.x;
                                pr[c + e + 1] = th.y;
                            }
                        }
                    }
                    if constexpr (kBias) {
                        if (side == kNear) {
                            const float* w = window + lane + 63;
#pragma unroll
                            for (int c = 0; c < 64; c += 2) {
                                const float2 v = fma2(make_float2(pr[c], pr[c + 1]), splat(mul), make_float2(w[-c], w[-c - 1]));
                                pr[c] = ex2(v.x);
                                pr[c + 1] = ex2(v.y);
                            }
                        } else {
                            const float step = side == kFarPos ? hb.slope : -hb.slope;  // per column: the distance shrinks
                            const float base = (side == kFarPos ? hb.far_pos : hb.far_neg) - step * (float)(dist_lo + lane + 63);
#pragma unroll
                            for (int c = 0; c < 64; c += 2) {
                                const float2 b = make_float2(fmaf(step, (float)c, base), fmaf(step, (float)(c + 1), base));
                                const float2 v = fma2(make_float2(pr[c], pr[c + 1]), splat(mul), b);
                                pr[c] = ex2(v.x);
                                pr[c + 1] = ex2(v.y);
                            }
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 64; ++c) pr[c] = ex2(pr[c] * mul);
                    }
                    if (!tile_full) {
#pragma unroll
                        for (int c = 0; c < 64; ++c)
                            if (c < col_lo || c >= col_hi) pr[c] = 0.f;  // select, never multiply
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) pk[i] = pack_bf16(pr[h * 32 + 2 * i], pr[h * 32 + 2 * i + 1]);
                        tmem_st_x16(lane_addr + kColS + col0 + h * 16, pk);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&sm.p_full);

                    ZL_WAIT_REGS(&sm.dp_full, it_cnt & 1, 23);
                    if (it_cnt > 0) ZL_WAIT_REGS(&sm.ds_free, (it_cnt - 1) & 1, 24);  // dS buffer consumed by dK/dQ
                    if (store_pending) {
                        // this warpgroup's box of the dS tile staged the previous item's dK / dV tile
                        if (store_leader) bulk_wait_group_read<0>();
                        named_bar_sync(2 + wg, 128);
                        store_pending = false;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t dr[32];
                        tmem_ld_x32(lane_addr + kColDP + col0 + c * 32, dr);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float d = __uint_as_float(dr[i]);
                            if (!tile_full) d = (c * 32 + i < col_lo || c * 32 + i >= col_hi) ? 0.f : d;  // P is zero there; keep 0 * inf out
                            pr[c * 32 + i] *= d;  // G
                        }
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4) {
                            uint32_t dd[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float2 ds = make_float2(pr[c * 32 + k4 * 8 + 2 * e], pr[c * 32 + k4 * 8 + 2 * e + 1]);
                                if constexpr (kCap)
                                    ds = mul2(ds, __half22float2(*reinterpret_cast<const __half2*>(&slope[c * 16 + k4 * 4 + e])));
                                dd[e] = pack_bf16(ds.x, ds.y);  // the one rounding between P, dP and the products with Q and K
                            }
                            const int c16 = (col0 >> 3) + c * 4 + k4;  // 16-byte chunk index along the query axis
                            const uint32_t addr = ds_row_addr + (c16 >> 3) * Smem::kBoxBytes + (((c16 & 7) ^ (row & 7)) << 4);
                            st_shared_v4(addr, dd[0], dd[1], dd[2], dd[3]);
                        }
                    }
                    tc_fence_before();
                    fence_proxy_async_smem();
                    mbar_arrive(&sm.ds_full);
                    if constexpr (kGrad) {  // while the tensor core works on dS
                        if (side == kNear) {
                            // Lane l, column t of a stretch: diagonal l - t + kCols - 1.  `diag` holds the sum of the lane's
                            // current diagonal; from one column to the next the diagonals move up by one lane, and the one
                            // that leaves lane 31 is complete.
                            using Sums = DiagSums<D>;
                            float diag[Sums::kChains];
                            __syncwarp();  // the biases have been read: the window takes the sums
#pragma unroll
                            for (int t = 0; t < Sums::kCols; ++t) {
#pragma unroll
                                for (int s = 0; s < Sums::kChains; ++s) {
                                    if (t == 0) {
                                        diag[s] = pr[s * Sums::kCols];
                                    } else {
                                        if (lane == 31) window[s * Sums::kStride + 31 + Sums::kCols - t] = diag[s];
                                        const float up = __shfl_up_sync(0xffffffffu, diag[s], 1);
                                        diag[s] = pr[s * Sums::kCols + t] + (lane == 0 ? 0.f : up);
                                    }
                                }
                            }
#pragma unroll
                            for (int s = 0; s < Sums::kChains; ++s) window[s * Sums::kStride + lane] = diag[s];
                            __syncwarp();
                            // stretch s holds the distance indexes from 64 - (s + 1) * kCols on
                            float v[kPatch / 32];
#pragma unroll
                            for (int i = 0; i < kPatch / 32; ++i) {
                                v[i] = 0.f;
#pragma unroll
                                for (int s = 0; s < Sums::kChains; ++s) {
                                    const int at = i * 32 + lane - (64 - (s + 1) * Sums::kCols);
                                    if (at >= 0 && at < Sums::kStride - 1) v[i] += window[s * Sums::kStride + at];
                                }
                            }
                            __syncwarp();
                            window[lane] = 0.f;
                            window[lane + 32] = 0.f;
                            __syncwarp();
                            add_by_bucket(window, v, near_bucket, lane);
                            bucket_sum[0] += window[lane];
                            bucket_sum[1] += window[lane + 32];
                        } else {
                            float2 s[4];
#pragma unroll
                            for (int c = 0; c < 4; ++c) s[c] = make_float2(pr[2 * c], pr[2 * c + 1]);
#pragma unroll
                            for (int c = 4; c < 32; ++c) s[c & 3] = add2(s[c & 3], make_float2(pr[2 * c], pr[2 * c + 1]));
                            s[0] = add2(add2(s[0], s[1]), add2(s[2], s[3]));
                            far_sum[side == kFarPos] += s[0].x + s[0].y;
                        }
                    }
                }
            }
            if constexpr (kGrad) {
                // the two far sums go to their buckets' lanes, the eight warps' sums are added in order
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float v = far_sum[e];
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
                    const int b = __ldg(sp.bucket_of + e * 2 * sp.reach);
                    if (b == lane) bucket_sum[0] += v;
                    if (b == lane + 32) bucket_sum[1] += v;
                }
                __syncwarp();
                window[lane] = bucket_sum[0];
                window[lane + 32] = bucket_sum[1];
                mbar_arrive(&sm.sums_full);
                ZL_WAIT_REGS(&sm.sums_full, sums_cnt & 1, 27);
                const int b = threadIdx.x - 128;  // 0 .. 255
                if (b < kMaxBuckets) {
                    float v = 0.f;
#pragma unroll
                    for (int w = 0; w < 8; ++w) v += sm.window[w][b];
                    sp.bucket_part[((int64_t)wi.head * sp.n_kv_tiles + g.tile_begin + wi.row0 / kTileKV) * kMaxBuckets + b] = v;
                }
                mbar_arrive(&sm.sums_empty);
                ZL_WAIT_REGS(&sm.sums_empty, sums_cnt & 1, 28);  // the windows are free again
                ++sums_cnt;
            }
            // ---- epilogue: warpgroup 0 stores dV, warpgroup 1 stores dK (scaled)
            const bool seen = it_cnt != it_first;  // else no query sees these keys: the gradients are zero
            if (seen) {
                ZL_WAIT_REGS(&sm.acc_full, item_cnt & 1, 25);
                ++item_cnt;
                tc_fence_after();
            }
            const float sc = (wg == 0) ? 1.f : p.scale;
            const uint32_t col_acc = (wg == 0) ? kColDV : kColDK;
            if (wi.rows == kTileKV && seen) {
                // full key tile: stage 64 columns at a time in this warpgroup's box of the (now idle) dS
                // tile and write them with one TMA store each -- coalesced, and the warpgroup moves on to
                // the next item while the copy engine drains the box
                const uint32_t box_addr = smem_u32(sm.ds) + wg * Smem::kBoxBytes + row * 128;
#pragma unroll 1
                for (int b = 0; b < kBoxes; ++b) {
                    if (b > 0) {
                        if (store_leader) bulk_wait_group_read<0>();
                        named_bar_sync(2 + wg, 128);
                    }
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        uint32_t r[32];
                        tmem_ld_x32(lane_addr + col_acc + b * 64 + c * 32, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4) {
                            const int i = k4 * 8;
                            st_shared_v4(box_addr + (((c * 4 + k4) ^ (row & 7)) << 4),
                                         pack_bf16(__uint_as_float(r[i]) * sc, __uint_as_float(r[i + 1]) * sc),
                                         pack_bf16(__uint_as_float(r[i + 2]) * sc, __uint_as_float(r[i + 3]) * sc),
                                         pack_bf16(__uint_as_float(r[i + 4]) * sc, __uint_as_float(r[i + 5]) * sc),
                                         pack_bf16(__uint_as_float(r[i + 6]) * sc, __uint_as_float(r[i + 7]) * sc));
                        }
                    }
                    fence_proxy_async_smem();
                    named_bar_sync(2 + wg, 128);
                    if (store_leader) {
                        tma_store_3d(wg == 0 ? &tm_dv : &tm_dk, sm.ds + wg * Smem::kBoxBytes, b * 64, wi.head,
                                     g.kv_off + wi.row0);
                        bulk_commit_group();
                    }
                }
                store_pending = true;
            } else {
                const int64_t grow = (int64_t)g.kv_off + wi.row0 + row;
                __nv_bfloat16* dst = (wg == 0 ? p.dv : p.dk) + grow * p.grad_row_stride + wi.head * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t r[32];
                    if (seen) {
                        tmem_ld_x32(lane_addr + col_acc + c * 32, r);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0;
                    }
                    if (row_ok) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint4 o4;
                            o4.x = pack_bf16(__uint_as_float(r[i]) * sc, __uint_as_float(r[i + 1]) * sc);
                            o4.y = pack_bf16(__uint_as_float(r[i + 2]) * sc, __uint_as_float(r[i + 3]) * sc);
                            o4.z = pack_bf16(__uint_as_float(r[i + 4]) * sc, __uint_as_float(r[i + 5]) * sc);
                            o4.w = pack_bf16(__uint_as_float(r[i + 6]) * sc, __uint_as_float(r[i + 7]) * sc);
                            *reinterpret_cast<uint4*>(dst + c * 32 + i) = o4;
                        }
                    }
                }
            }
            tc_fence_before();
        }
        if (store_leader) bulk_wait_group<0>();  // the last dK / dV stores have left shared memory and landed
    } else {
        // ------------------------------------------------------------------ dQ warpgroup (one query row per thread)
        reg_inc<152>();
        const int quarter = warp & 3;
        const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
        const bool leader = (lane == 0);  // per warp
        uint32_t it_cnt = 0, chunk_cnt = 0;
        for (int it = walk.first; it < walk.end; it += walk.step) {
            const WorkItem wi = p.items[it];
            const KvGroup g = p.kv_groups[wi.unit];
            for (int ti = 0; ti < g.n_tasks; ++ti) {
                const int task = p.kv_group_tasks[g.task_begin + ti];
                const Task t = p.tasks[task];
                const int n_q = (t.q_len + kTileQ - 1) / kTileQ;
                for (int qt = first_tile(sp, t, task, wi.row0); qt < n_q; ++qt, ++it_cnt) {
                    ZL_WAIT_REGS(&sm.dq_full, it_cnt & 1, 31);
                    tc_fence_after();
                    {
                        // read the whole tile (frees the TMEM columns for the next dP^T), then stage
                        // 32-column chunks in swizzled shared memory and add them with the TMA
                        uint32_t r[D];
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t tmp[32];
                            tmem_ld_x32(lane_addr + kColDP + c * 32, tmp);
#pragma unroll
                            for (int i = 0; i < 32; ++i) r[c * 32 + i] = tmp[i];
                        }
                        tmem_wait_ld();
                        tc_fence_before();
                        mbar_arrive(&sm.dq_empty);
#pragma unroll
                        for (int c = 0; c < D / 32; ++c, ++chunk_cnt) {
                            // each warp stages its own 32 rows and adds them with its own reduce: no
                            // warpgroup barrier, and the four streams overlap in the copy engine
                            uint8_t* buf = sm.dq_stage + quarter * 4096;
                            if (chunk_cnt >= 1) {
                                if (leader) bulk_wait_group_read<0>();  // the previous reduce has read the buffer
                                __syncwarp();
                            }
                            const uint32_t row_addr = smem_u32(buf) + lane * 128;
#pragma unroll
                            for (int k4 = 0; k4 < 8; ++k4)
                                st_shared_v4(row_addr + ((k4 ^ (lane & 7)) << 4), r[c * 32 + k4 * 4], r[c * 32 + k4 * 4 + 1],
                                             r[c * 32 + k4 * 4 + 2], r[c * 32 + k4 * 4 + 3]);
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (leader) {
                                tma_reduce_add_3d(&tm_dq, buf, c * 32, wi.head, t.dq_slot + qt * kTileQ + quarter * 32);
                                bulk_commit_group();
                            }
                        }
                    }
                }
            }
        }
        if (leader) bulk_wait_group<0>();
    }

teardown:
    // Also reached after an expired wait: bulk stores and reduces this thread has committed must have
    // finished reading shared memory before the CTA gives it up (a no-op on the normal path).
    bulk_wait_group<0>();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// The opt-in to large dynamic shared memory is a per-device attribute of the kernel.
constexpr int kMaxDevices = 64;

template <int D, bool kCap, ScoreKind kKind>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tdo,
                     const CUtensorMap& tdq, const CUtensorMap& tdk, const CUtensorMap& tdv, const BwdParams& p,
                     const ScoreParams& sp, int grid, cudaStream_t stream) {
    constexpr int smem = sizeof(ScoredBwdSmem<D, kCap>);
    static_assert(smem <= 232448, "shared memory of a CTA");
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_scored_bwd_kernel<D, kCap, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    // An early start hides the launch where a CTA has an item or two (128-row keys of three short sequences: 17.6 -> 16.8 us for
    // the whole backward); behind a full-size preprocess pass it gains nothing and costs up to 4 % (capped scores under a
    // prefix mask, 7 k tokens, 12 heads, d 128: 225 -> 235 us), as does releasing the next launch early from here.
    return launch_dependent(zl_scored_bwd_kernel<D, kCap, kKind>, grid, kBwdThreads, smem, stream, p.n_items <= 2 * grid,
                            tq, tk, tv, tdo, tdq, tdk, tdv, p, sp);
}

template <int D, bool kCap>
cudaError_t launch_k(ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                     const CUtensorMap& tdo, const CUtensorMap& tdq, const CUtensorMap& tdk, const CUtensorMap& tdv,
                     const BwdParams& p, const ScoreParams& sp, int grid, cudaStream_t stream) {
    switch (kind) {
        case kScorePlain: return launch_t<D, kCap, kScorePlain>(tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream);
        case kScoreBias: return launch_t<D, kCap, kScoreBias>(tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream);
        case kScoreBiasGrad: return launch_t<D, kCap, kScoreBiasGrad>(tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_scored_bwd(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                              const CUtensorMap& tv, const CUtensorMap& tdo, const CUtensorMap& tdq, const CUtensorMap& tdk,
                              const CUtensorMap& tdv, const BwdParams& p, const ScoreParams& sp, int grid, cudaStream_t stream) {
    if (p.n_items == 0) return cudaSuccess;
    if (head_dim == 128)
        return capped ? launch_k<128, true>(kind, tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream)
                      : launch_k<128, false>(kind, tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream);
    return capped ? launch_k<64, true>(kind, tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream)
                  : launch_k<64, false>(kind, tq, tk, tv, tdo, tdq, tdk, tdv, p, sp, grid, stream);
}

}  // namespace zl
