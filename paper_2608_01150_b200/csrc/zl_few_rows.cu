// Forward kernel for work items of at most 128 query rows (sm_100a): single tokens and short tails against long keys, and
// batches of a few rows over a shared prefix.  Plain or scored (zl_score.cuh).
//
// Such items are bound by the keys and values they read, not by the products: 128 keys of one head are 64 KB for at
// most 128 rows, and an SM's share of the memory bandwidth is one such tile every 2,800 clocks.  The two-tile kernels keep
// one tile of K and V per stage until its product with P is done, and with one query tile run S, softmax and P V one after
// the other (about 4,300 clocks a tile for one row).  Here
//   * the two softmax warpgroups take alternate KEY tiles of the same query tile, each with its own running maximum, sum
//     and accumulator (S_0, S_1, O_0, O_1 in TMEM), and join them at the end of the item: a warp of either warpgroup can
//     read both accumulators, which share its TMEM lanes, so only the maxima and sums pass through shared memory;
//   * K and V have rings of their own: a K tile is free again as soon as its S is done, a V tile when its P V is;
//   * Q takes only the rows it has (rounded up to 16) and two buffers, so that the loads of the next item run on under
//     the current one; rows of the MMA beyond them hold whatever the shared memory holds and never leave their row;
//   * warps without a valid row only take part in the barriers;
//   * where items are too few for the SMs they come in pieces along the keys (FewItem), and the piece that finishes last joins
//     them from the padding of the shard's slot.
// The same kernel takes the 128-row blocks of longer query ranges where 256-row blocks would leave SMs without work.
// Measured (B200, d 128): one token against 8 x 9450 keys, 40 heads 280-310 us with the merge (5.0-5.5 TB/s; 495 us with the
// two-tile kernel); against 9450 keys, 2 heads 19 us (95 us in one piece); 64 tokens over a shared prefix of 32,760 keys, 12
// heads 66 us (4.5 TB/s).  Registers and code size count: state that the join keeps alive across the tile loop, or loops
// unrolled further in it, cost 7-13 % of the first figure.
#include <cuda_runtime.h>

#include "zl_score.cuh"

namespace zl {

using namespace ptx;
using namespace score;

namespace {

constexpr int kThreads = 384;

template <int D, int kRows>
struct FewSmem {
    static constexpr int kTileBytes = kTileKV * D * 2;
    static constexpr int kBoxBytes = kTileKV * 128;  // 128 rows x 64 bf16
    static constexpr int kBoxes = D / 64;
    static constexpr int kStagesK = D == 64 ? 5 : (kRows == 64 ? 3 : 2);
    static constexpr int kStagesV = D == 64 ? 5 : 2;
    static constexpr int kQBoxBytes = kRows * 128;
    alignas(1024) uint8_t q[2][kRows * D * 2];  // followed by K: an MMA reads 128 rows from here on
    alignas(1024) uint8_t k[kStagesK][kTileBytes];
    alignas(1024) uint8_t v[kStagesV][kTileBytes];
    float window[2][kWindow];  // per warpgroup: the biases of a near key tile
    float2 stat[2][kTileQ];    // per warpgroup and row: reference maximum (powers of two) and sum
    alignas(8) uint64_t q_full[2], q_empty[2];
    uint64_t k_full[kStagesK], k_empty[kStagesK], v_full[kStagesV], v_empty[kStagesV];
    uint64_t bias_full[2], bias_empty[2];
    uint64_t s_full[2], p_half[2][2], o_full[2];
    uint64_t stat_full, join_done, part_bar;  // between the warpgroups at the end of an item
    int32_t ticket;
    uint32_t tmem_base;
    volatile int32_t abort_flag;
};

// An item as the roles walk it: `rows` query rows from row0 of the task over key tiles [tile0, tile0 + n_kv), piece `part` of `parts`.
struct FewItem {
    int row0, rows, part, parts, tile0, n_kv;
    __device__ __forceinline__ FewItem(const WorkItem& wi, const ScoreParams& sp, const Task& t) {
        parts = wi.rows >> kPartsShift;
        rows = wi.rows & ((1 << kPartsShift) - 1);
        part = parts > 1 ? wi.row0 : 0;
        row0 = parts > 1 ? 0 : wi.row0;
        const int tiles = key_tiles(sp, t, wi.unit, row0, rows);
        tile0 = parts > 1 ? tiles * part / parts : 0;
        n_kv = (parts > 1 ? tiles * (part + 1) / parts : tiles) - tile0;
    }
};

#define ZL_WAIT(bar, parity, site)                                        \
    do {                                                                  \
        if (!wait((bar), (parity), &sm.abort_flag)) { \
            report(p.status, &sm.abort_flag, 5000 + (site));              \
            goto teardown;                                                \
        }                                                                 \
    } while (0)
#define ZL_WAIT_WARP(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 5000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)
// The same from the warps that hold tiles in registers.
#define ZL_WAIT_REGS(bar, parity, site)                                              \
    do {                                                                             \
        const bool ok_ = wait_inline((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                         \
            report(p.status, &sm.abort_flag, 5000 + (site));                         \
            goto teardown;                                                           \
        }                                                                            \
    } while (0)

template <int D, int kRows, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1)
zl_few_rows_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                   const __grid_constant__ CUtensorMap tm_v, const int q_box_rows, const FwdParams p, const ScoreParams sp) {
    using Smem = FewSmem<D, kRows>;
    constexpr int kBoxes = Smem::kBoxes, kStagesK = Smem::kStagesK, kStagesV = Smem::kStagesV;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    // TMEM columns: S_0 [0,128), S_1 [128,256), O_0 [256,256+D), O_1 [384,384+D); P_x over the first half of S_x
    constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;

    if ((smem_u32(smem_raw) & 1023u) != 0) {  // swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0 && atomicCAS(p.status, 0, (int)ZL_ERR_CUDA) == 0) p.status[1] = 5999;
        return;
    }
    if (threadIdx.x == 0) {
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sm.q_full[x], 1);
            mbar_init(&sm.q_empty[x], 1);
            mbar_init(&sm.s_full[x], 1);
            mbar_init(&sm.p_half[x][0], 128);
            mbar_init(&sm.p_half[x][1], 128);
            mbar_init(&sm.o_full[x], 1);
            mbar_init(&sm.bias_full[x], 1);
            mbar_init(&sm.bias_empty[x], 128);
        }
        for (int s = 0; s < kStagesK; ++s) { mbar_init(&sm.k_full[s], 1); mbar_init(&sm.k_empty[s], 1); }
        for (int s = 0; s < kStagesV; ++s) { mbar_init(&sm.v_full[s], 1); mbar_init(&sm.v_empty[s], 1); }
        mbar_init(&sm.stat_full, 256);
        mbar_init(&sm.join_done, 256);
        mbar_init(&sm.part_bar, 256);
        sm.abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
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
            uint32_t item_cnt = 0, kv_cnt = 0;
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const FewItem fi(wi, sp, t);
                const int n_kv = fi.n_kv;
                if (n_kv == 0) continue;
                const int qb = item_cnt & 1;
                ZL_WAIT(&sm.q_empty[qb], ((item_cnt >> 1) & 1) ^ 1, 1);
                ++item_cnt;
                mbar_arrive_expect_tx(&sm.q_full[qb], q_box_rows * D * 2);
                for (int b = 0; b < kBoxes; ++b)
                    tma_load_3d(sm.q[qb] + b * Smem::kQBoxBytes, &tm_q, &sm.q_full[qb], b * 64, wi.head, t.q_off + fi.row0);
                for (int j = 0; j <= n_kv; ++j) {  // K runs one tile ahead of V: its slots free up first
                    if (j < n_kv) {
                        const uint32_t c = kv_cnt + j, ks = c % kStagesK;
                        ZL_WAIT(&sm.k_empty[ks], ((c / kStagesK) & 1) ^ 1, 2);
                        mbar_arrive_expect_tx(&sm.k_full[ks], Smem::kTileBytes);
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_3d(sm.k[ks] + b * Smem::kBoxBytes, &tm_k, &sm.k_full[ks], b * 64, wi.head, t.kv_off + (fi.tile0 + j) * kTileKV);
                    }
                    if (j > 0) {
                        const uint32_t c = kv_cnt + j - 1, vs = c % kStagesV;
                        ZL_WAIT(&sm.v_empty[vs], ((c / kStagesV) & 1) ^ 1, 3);
                        mbar_arrive_expect_tx(&sm.v_full[vs], Smem::kTileBytes);
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_3d(sm.v[vs] + b * Smem::kBoxBytes, &tm_v, &sm.v_full[vs], b * 64, wi.head, t.kv_off + (fi.tile0 + j - 1) * kTileKV);
                    }
                }
                kv_cnt += n_kv;
            }
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMA issuer (whole warp, one elected lane issues)
            const bool mma_lane = elect_one();
            constexpr uint32_t idesc_s = make_idesc_bf16(kTileQ, kTileKV, 0, 0);
            constexpr uint32_t idesc_o = make_idesc_bf16(kTileQ, D, 0, 1);
            const uint64_t dq0 = make_desc_sw128(smem_u32(sm.q[0]), 16, 1024);
            const uint64_t dk0 = make_desc_sw128(smem_u32(sm.k[0]), 16, 1024);
            const uint64_t dv0 = make_desc_sw128(smem_u32(sm.v[0]), Smem::kBoxBytes, 1024);  // V is the MN-major B operand
            constexpr uint32_t kTileStep = Smem::kTileBytes >> 4, kQStep = (uint32_t)sizeof(sm.q[0]) >> 4;
            uint32_t item_cnt = 0, kv_cnt = 0, pa_cnt = 0, pb_cnt = 0;
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const int n_kv = FewItem(wi, sp, t).n_kv;
                if (n_kv == 0) continue;
                const uint32_t qb = item_cnt & 1;
                ZL_WAIT_WARP(&sm.q_full[qb], (item_cnt >> 1) & 1, 11);
                ++item_cnt;
                // step j: S(j), two tiles ahead of P(j - 2) V(j - 2)
                for (int j = 0; j < n_kv + 2; ++j) {
                    if (j >= 2) {
                        const int x = j & 1;
                        const uint32_t c = kv_cnt + j - 2, vs = c % kStagesV;
                        ZL_WAIT_WARP(&sm.v_full[vs], (c / kStagesV) & 1, 12);
                        const uint64_t dv = dv0 + vs * kTileStep;
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            ZL_WAIT_WARP(&sm.p_half[x][half], (x == 0 ? pa_cnt : pb_cnt) & 1, 13);
                            tc_fence_after();
#pragma unroll
                            for (int ks = 0; ks < kTileKV / 32; ++ks) {
                                const int at = half * (kTileKV / 32) + ks;
                                if (mma_lane) mma_ts(tmem + kColO + x * 128, tmem + kColS + x * 128 + at * 8, dv + at * (2048 >> 4),
                                                     idesc_o, j > 3 || half > 0 || ks > 0);
                            }
                        }
                        if (x == 0) ++pa_cnt; else ++pb_cnt;
                        if (mma_lane) mma_commit(&sm.v_empty[vs]);
                        if (j >= n_kv) if (mma_lane) mma_commit(&sm.o_full[x]);  // the warpgroup's last tile
                    }
                    if (j < n_kv) {
                        const int x = j & 1;
                        const uint32_t c = kv_cnt + j, ks_ = c % kStagesK;
                        ZL_WAIT_WARP(&sm.k_full[ks_], (c / kStagesK) & 1, 15);
                        tc_fence_after();
                        const uint64_t dq = dq0 + qb * kQStep, dk = dk0 + ks_ * kTileStep;
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)  // over P_x(j - 2): ordered after P_x V on the tensor pipe
                            if (mma_lane) mma_ss(tmem + kColS + x * 128, dq + (((ks / 4) * Smem::kQBoxBytes + (ks % 4) * 32) >> 4),
                                                 dk + (((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4), idesc_s, ks > 0);
                        if (mma_lane) mma_commit(&sm.s_full[x]);
                        if (mma_lane) mma_commit(&sm.k_empty[ks_]);
                        if (j + 1 == n_kv) if (mma_lane) mma_commit(&sm.q_empty[qb]);
                    }
                }
                kv_cnt += n_kv;
            }
        } else if (kBias && warp >= 2) {  // (the other lanes of warp 0 have nothing to do)
            // -------------------------------------------------------------- biases of near tiles, one warp per warpgroup
            const int x = warp - 2;
            WindowFeed feed{&sm.bias_full[x], &sm.bias_empty[x], sm.window[x]};
            for (int it = walk.first; it < walk.end; it += walk.step) {
                const WorkItem wi = p.items[it];
                const Task t = p.tasks[wi.unit];
                const TaskPos tp = task_pos(sp, wi.unit);
                const FewItem fi(wi, sp, t);
                HeadBias hb;
                hb.load(sp, wi.head);
                for (int j = x; j < fi.n_kv; j += 2) {
                    const int lo = tp.kv_pos + (fi.tile0 + j) * kTileKV - (tp.q_pos + fi.row0 + kTileQ - 1);
                    if (patch_side(sp, lo, lo + kTileQ + kTileKV - 2) != kNear) continue;
                    if (!feed.put(sp, hb, wi.head, lo, lane, &sm.abort_flag)) {
                        report(p.status, &sm.abort_flag, 5000 + 31);
                        goto teardown;
                    }
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax, join and output
        reg_inc<216>();
        const int x = (warp - 4) >> 2;             // key tiles x, x + 2, ...
        const int quarter = warp & 3;              // TMEM lane quarter this warp may access
        const int row = quarter * 32 + lane;       // query row within the tile
        const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t col_s = kColS + x * 128, col_o = kColO + x * 128;
        uint32_t bias_cnt = 0;
        uint32_t s_cnt = 0, o_cnt[2] = {0, 0}, join_cnt = 0;
        for (int it = walk.first; it < walk.end; it += walk.step) {
            const WorkItem wi = p.items[it];
            const Task t = p.tasks[wi.unit];
            const TaskPos tp = task_pos(sp, wi.unit);
            const FewItem fi(wi, sp, t);
            const int n_kv = fi.n_kv;
            const int keys = (sp.masked ? visible_keys(tp, t.kv_len, fi.row0 + row) : t.kv_len) - fi.tile0 * kTileKV;  // this row's, from the piece on
            const bool busy = quarter * 32 < fi.rows;  // warp-uniform: the warp has a valid row
            const bool row_ok = row < fi.rows;
            HeadBias hb;
            if constexpr (kBias) hb.load(sp, wi.head);
            float m_ref = -INFINITY, l = 0.f;
            for (int j = x; j < n_kv; j += 2) {
                const int dist_lo = tp.kv_pos + (fi.tile0 + j) * kTileKV - (tp.q_pos + fi.row0 + kTileQ - 1);  // last row, first column
                const PatchSide side = kBias ? patch_side(sp, dist_lo, dist_lo + kTileQ + kTileKV - 2) : kNear;
                const bool ragged = __any_sync(0xffffffffu, keys - j * kTileKV < kTileKV);
                ZL_WAIT_REGS(&sm.s_full[x], s_cnt & 1, 21);
                ++s_cnt;
                if (!busy) {  // P of rows that do not exist is whatever S was
                    if (kBias && side == kNear) {
                        ZL_WAIT_REGS(&sm.bias_full[x], bias_cnt & 1, 25);
                        ++bias_cnt;
                        mbar_arrive(&sm.bias_empty[x]);
                    }
                    mbar_arrive(&sm.p_half[x][0]);
                    mbar_arrive(&sm.p_half[x][1]);
                    continue;
                }
                if (kBias && side == kNear) {
                    ZL_WAIT_REGS(&sm.bias_full[x], bias_cnt & 1, 26);
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
                softmax_tile<D, kCap, kBias>(sv, sp, hb, p.scale_log2, j == x, side, sm.window[x] + kTileQ - 1 - row, &sm.bias_empty[x],
                                             dist_lo + kTileQ - 1 - row, keys - j * kTileKV, ragged, row_ok, lane_addr + col_s, lane_addr + col_o,
                                             sm.p_half[x], m_ref, l);
            }
            // ---- join: O = (w_0 O_0 + w_1 O_1) / (w_0 l_0 + w_1 l_1), w_x = 2^(m_x - max); warpgroup x writes half of the columns
            float w[2] = {0.f, 0.f}, lse = -INFINITY;
            if (n_kv > 0) {
                for (int y = 0; y < 2; ++y)
                    if (n_kv > y) {
                        ZL_WAIT_REGS(&sm.o_full[y], o_cnt[y] & 1, 22 + y);
                        ++o_cnt[y];
                    }
                tc_fence_after();
                sm.stat[x][row] = make_float2(m_ref, l);
                mbar_arrive(&sm.stat_full);
                ZL_WAIT_REGS(&sm.stat_full, join_cnt & 1, 27);
                const float2 a = sm.stat[0][row], b = sm.stat[1][row];
                const float m = fmaxf(a.x, b.x);
                if (m > -INFINITY) {
                    const float wa = ex2(a.x - m), wb = ex2(b.x - m);
                    const float sum = wa * a.y + wb * b.y;
                    lse = (m + log2f(sum)) * 0.6931471805599453f;
                    w[0] = wa / sum;
                    w[1] = wb / sum;
                }
            }
            if (busy) {
                const int64_t grow = (int64_t)(t.partial_slot >= 0 ? t.partial_slot + fi.part * fi.rows : t.q_off) + fi.row0 + row;
                const int c0 = x * (D / 2);
#pragma unroll 1
                for (int c = 0; c < D / 64; ++c) {
                    float o[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0.f;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if (n_kv > y) {
                            uint32_t r[32];
                            tmem_ld_x32(lane_addr + kColO + y * 128 + c0 + c * 32, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = fmaf(w[y], __uint_as_float(r[i]), o[i]);
                        }
                    }
                    if (!row_ok) continue;
                    const int64_t at = (grow * p.n_heads + wi.head) * D + c0 + c * 32;
                    if (t.partial_slot >= 0) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4*>(p.o_partial + at + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint4 o4;
                            o4.x = pack_bf16(o[i], o[i + 1]);
                            o4.y = pack_bf16(o[i + 2], o[i + 3]);
                            o4.z = pack_bf16(o[i + 4], o[i + 5]);
                            o4.w = pack_bf16(o[i + 6], o[i + 7]);
                            *reinterpret_cast<uint4*>(p.o + at + i) = o4;
                        }
                    }
                }
                if (row_ok && x == 0) {
                    if (t.partial_slot >= 0) p.lse_partial[(int64_t)wi.head * p.partial_rows + grow] = lse;
                    else p.lse[(int64_t)wi.head * p.total_q + grow] = lse;
                }
            }
            tc_fence_before();
            if (n_kv > 0) {  // both accumulators and the statistics have been read
                mbar_arrive(&sm.join_done);
                ZL_WAIT_REGS(&sm.join_done, join_cnt & 1, 28);
                ++join_cnt;
            }
            // (the item is read again rather than kept: registers are short in the loop over tiles)
            const int4 again = __ldcg(reinterpret_cast<const int4*>(p.items + it));
            const int parts = again.w >> kPartsShift;
            if (parts > 1) {
                const int unit = again.x, head = again.y, rows = again.w & ((1 << kPartsShift) - 1);
                const int slot = __ldcg(&p.tasks[unit].partial_slot);
                // ---- the piece that finishes last joins all of them, in order (an even number of barrier phases either way):
                //      O = sum_s 2^(LSE_s - max) O_s / sum_s 2^(LSE_s - max)
                __threadfence();
                mbar_arrive(&sm.part_bar);
                ZL_WAIT_REGS(&sm.part_bar, 0, 29);  // this piece's rows are written and visible
                int32_t* count = p.part_count + (int64_t)unit * p.n_heads + head;
                const int tid = threadIdx.x - 128;  // 0 .. 255
                if (tid == 0) sm.ticket = atomicAdd(count, 1);
                mbar_arrive(&sm.part_bar);
                ZL_WAIT_REGS(&sm.part_bar, 1, 30);
                if (sm.ticket == parts - 1) {
                    __threadfence();
                    // all LSEs at once (they are contiguous in the slot), then four partial rows in flight per thread
                    const int n_lse = parts * rows;  // at most 128
                    float* lse_s = reinterpret_cast<float*>(&sm.stat[0][0]);
                    float* lse_p = p.lse_partial + (int64_t)head * p.partial_rows + slot;
                    if (tid < n_lse) lse_s[tid] = __ldcg(lse_p + tid);
                    mbar_arrive(&sm.part_bar);
                    ZL_WAIT_REGS(&sm.part_bar, 0, 31);
                    float4* o_p = reinterpret_cast<float4*>(p.o_partial + ((int64_t)slot * p.n_heads + head) * D);
                    const int64_t row4 = (int64_t)p.n_heads * D / 4;
#pragma unroll 1
                    for (int i = tid; i < rows * (D / 4); i += 256) {
                        const int r = i / (D / 4), c4 = i % (D / 4);
                        float m = -INFINITY, z = 0.f;
#pragma unroll 4
                        for (int s = r; s < n_lse; s += rows) m = fmaxf(m, lse_s[s]);
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                        for (int s0 = r; s0 < n_lse; s0 += 4 * rows) {
                            float4 o_s[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (s0 + e * rows < n_lse) o_s[e] = __ldcg(o_p + (s0 + e * rows) * row4 + c4);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (s0 + e * rows < n_lse) {
                                    const float w_s = m > -INFINITY ? ex2((lse_s[s0 + e * rows] - m) * kLog2e) : 0.f;
                                    z += w_s;
                                    acc.x = fmaf(w_s, o_s[e].x, acc.x); acc.y = fmaf(w_s, o_s[e].y, acc.y);
                                    acc.z = fmaf(w_s, o_s[e].z, acc.z); acc.w = fmaf(w_s, o_s[e].w, acc.w);
                                }
                        }
                        const float inv_z = z > 0.f ? 1.f / z : 0.f;
                        o_p[r * row4 + c4] = make_float4(acc.x * inv_z, acc.y * inv_z, acc.z * inv_z, acc.w * inv_z);
                        if (c4 == 0) lse_p[r] = m > -INFINITY ? m + logf(z) : -INFINITY;
                    }
                    if (tid == 0) *count = 0;  // for the next launch
                    mbar_arrive(&sm.part_bar);
                    ZL_WAIT_REGS(&sm.part_bar, 1, 32);  // the statistics' place is free again
                }
            }
        }
    }

teardown:
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

template <int D, int kRows, bool kCap, bool kBias>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, int q_box_rows, const FwdParams& p,
                     const ScoreParams& sp, int grid, cudaStream_t stream) {
    constexpr int smem = sizeof(FewSmem<D, kRows>);
    static_assert(smem <= 232448, "shared memory of a CTA");
    constexpr int kMaxDevices = 64;
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_few_rows_kernel<D, kRows, kCap, kBias>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    return launch_dependent(zl_few_rows_kernel<D, kRows, kCap, kBias>, grid, kThreads, smem, stream, true, tq, tk, tv, q_box_rows, p, sp);
}

template <int D, int kRows>
cudaError_t launch_s(bool capped, bool biased, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, int q_box_rows,
                     const FwdParams& p, const ScoreParams& sp, int grid, cudaStream_t stream) {
    if (capped)
        return biased ? launch_t<D, kRows, true, true>(tq, tk, tv, q_box_rows, p, sp, grid, stream)
                      : launch_t<D, kRows, true, false>(tq, tk, tv, q_box_rows, p, sp, grid, stream);
    return biased ? launch_t<D, kRows, false, true>(tq, tk, tv, q_box_rows, p, sp, grid, stream)
                  : launch_t<D, kRows, false, false>(tq, tk, tv, q_box_rows, p, sp, grid, stream);
}

}  // namespace

cudaError_t launch_few_rows(int head_dim, bool capped, ScoreKind kind, const CUtensorMap& tq, const CUtensorMap& tk,
                            const CUtensorMap& tv, int q_box_rows, const FwdParams& p, const ScoreParams& sp, int grid,
                            cudaStream_t stream) {
    if (p.n_items == 0) return cudaSuccess;
    const bool biased = kind != kScorePlain;
    if (head_dim == 128)
        return q_box_rows <= 64 ? launch_s<128, 64>(capped, biased, tq, tk, tv, q_box_rows, p, sp, grid, stream)
                                : launch_s<128, 128>(capped, biased, tq, tk, tv, q_box_rows, p, sp, grid, stream);
    return q_box_rows <= 64 ? launch_s<64, 64>(capped, biased, tq, tk, tv, q_box_rows, p, sp, grid, stream)
                            : launch_s<64, 128>(capped, biased, tq, tk, tv, q_box_rows, p, sp, grid, stream);
}

}  // namespace zl
