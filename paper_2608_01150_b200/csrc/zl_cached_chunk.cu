// Attention of chunks of new tokens over the paged cache (sm_100a): the products of many rows with every key, on the tensor cores.
//
// The rows of a key head are its sequence's new tokens times the query heads of its group; a tile takes as many whole tokens as
// fit 128 rows, so that one box of Q holds a tile.  An item is two such tiles (or the one that is left) of a sequence and key
// head.  All CTAs (one per SM) walk one line of work and each takes an equal stretch of it, wherever that cuts an item; the lengths
// are read when the kernel runs.  Stretches are found from sums in closed form: block b of a sequence sees
// min(keys, max(prefix, pos0 + (b + 1) tokens)) keys.
//   warp 0       TMA producer: Q once per item, K and V page by page through shared-memory rings
//   warp 2       walks the line and hands the items' descriptions to the others
//   warp 1       MMA issuer: S_x = Q K^T, O_x += P_x V (P read from TMEM), one step two ahead of the other
//   warps 4-11   softmax.  All of them work on the same scores, sixteen rows a warp, in turn on S_0 and S_1: those are two query tiles
//                against a key tile, or one query tile against two key tiles, whose accumulators are joined at the end.  While the
//                warps are at one, the tensor core has the other's P V and next S before it: a warpgroup with a tile of its own
//                stood still for those (1560 tokens over 9,750 bf16 keys 306 -> 300 us)
//   warps 12-15  (8-bit caches) codes become fp16, exactly, in their place (a tile of codes arrives in the second half of the tile it
//                becomes), and so do the queries of an item; the scale of a key multiplies its column of S, the scale of a value its
//                column of P, in fp32: the softmax takes s_j = S_j k_j + log2 v_j, so that its exponentials are the weights of the
//                values, and sums weight / v_j beside them.  (Values times their scale in fp16 would spare two of the three scales,
//                but lose the small ones beside a large one, and the two multiplications more kept these warps busy: 420 -> 572
//                us, 1560 tokens over 9,750 int8 keys.)
// An item that lies in several CTAs leaves its parts in the workspace, and a second launch joins them, in the order of the CTAs: a
// part is 133 KB, and one CTA alone took 20 us to join the six parts of 256 rows over 8,700 keys.
// Measured, d 128: 1560 tokens over 34,320 keys, 40 query heads over 8: bf16 1040 TFLOP/s (1662 is what products alone reach), e4m3
// 870, int8 860 (in a run of seconds, whose clocks fall under the power cap: 920, 820, 800); 512 tokens behind 8,190, 12 heads: bf16
// 45 us, 8 bits 57.  A step has 1,024 clocks of exponentials a tile and as many of products, but fills no pipe (special functions
// and tensor cores at 30 to 42 %): there are two warps to a scheduler, both at the same place, so that the load of S, the maximum,
// the scales, the store of P and its wait are all seen beside the exponentials.  (Part of the exponentials by multiply-adds: bf16 no faster, 8 bits 4 to 22 % slower; S of
// the next step asked for early: bf16 no faster, 8 bits without the registers for it.)
#include <type_traits>

#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr uint64_t kWaitLimitNs = 4000000000ull;
constexpr float kRescaleThresholdLog2 = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaskRing = 8;   // key tiles whose masks are kept: more than can be under way
// Units of work: a key tile under two query tiles takes 4,100 clocks (bf16; 8-bit codes 5,300), under one 2,900 (4,500).  With
// the second counted as half of the first, CTAs with single tiles finished a third later than the others.  An item's start and
// end (its queries, the first keys' way here, the last tile's output) count as three key tiles: half as many are 1 to 3 % slower.
constexpr int32_t kTwoCost = 8, kOneCost = 7;  // a key under two query tiles, under one
constexpr int32_t kItemCost = 3 * kTileKV * kTwoCost;
constexpr int64_t kLeastUnits = 4 * kTileKV * kTwoCost;  // least stretch of a CTA

// A CTA's part of an item, as warp 2 hands it to the other warps.
struct alignas(16) Item {
    int32_t s, head, tile0, tile1;       // sequence, key head, key tiles of this part (tile1 < 0: no more items)
    int32_t tok0, tokens, keys, two;     // new tokens, keys that they see, two query tiles
    int32_t q0, pos0, seq_keys, prefix;  // SeqView
    int32_t c_first, c_last;             // the CTAs that have parts of it
    int32_t place_first, pad_;           // the first of them keeps its part in place 1 (its stretch begins before) or 0
    __device__ __forceinline__ SeqView seq() const { return {q0, 0, pos0, seq_keys, prefix}; }
    __device__ __forceinline__ int32_t place(int32_t cta) const { return cta == c_first ? place_first : 0; }
};
constexpr int kItems = 4;  // descriptions under way

template <int D, int kFormat>
struct ChunkSmem {
    static constexpr bool kCodes = kFormat != ZL_CACHE_BF16;
    static constexpr int kTileBytes = kTileKV * D * 2;  // one 128-row tile of Q, K or V
    static constexpr int kBoxBytes = kTileKV * 128;     // 128 rows x 64 bf16
    static constexpr int kBoxes = D / 64;
    static constexpr int kStages = D == 128 ? 2 : 5;
    // A tile's K is prepared once V of the tile two before it has its place, which P V of kStages tiles earlier gave up: until
    // then masks and scales of a tile may be read.
    static constexpr int kScaleRing = D == 128 ? 4 : 8;
    static_assert(kScaleRing >= kStages + 2 || !kCodes, "scales of a tile are kept until its softmax is done");
    static_assert(kMaskRing >= kStages + 2, "masks of a tile are kept until its P V is done");
    alignas(1024) uint8_t q[2][kTileBytes];
    alignas(1024) uint8_t k[kStages][kTileBytes];
    alignas(1024) uint8_t v[kStages][kTileBytes];
    alignas(16) float key_scale[kCodes ? kScaleRing : 1][kTileKV];  // of the scores, in powers of two
    alignas(16) float value_log2[kCodes ? kScaleRing : 1][kTileKV], value_inv[kCodes ? kScaleRing : 1][kTileKV];  // log2 and inverse of its scale
    alignas(16) uint32_t mask[kMaskRing][4];            // keys of a tile that exist
    Item items[kItems];
    float2 stat[2][kTileQ];                             // per warpgroup and row: reference maximum (powers of two), sum
    float q_big[4];  // per converting warp: largest magnitude of its queries
    alignas(8) uint64_t q_full, q_empty, q_max, q_ready;
    uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t k_codes[kCodes ? kStages : 1], v_codes[kCodes ? kStages : 1], codes_read;
    uint64_t s_full[2], p_half[2][2], o_full[2], tile_full[kMaskRing];
    uint64_t stat_full, item_full[kItems], item_empty[kItems], drained;
    int64_t scan[16], start_base, total;
    int32_t start_seq;
    uint32_t q_loads, k_loads, v_loads;  // asked for so far (the producer's count)
    uint32_t tmem_base;
    volatile int32_t abort_flag;
};

template <int D>
constexpr int kPartTileFloats = kTileQ * (D + 2);  // maxima, sums, then the unnormalised output as [D / 4][row] of four

// ------------------------------------------------------------------------------------------------ the line of work
struct Geometry {
    int32_t tokens;  // whole tokens of a tile
    int32_t heads;
    int32_t rest_rows;  // sequences of at most as many rows are another kernel's
    __device__ __forceinline__ explicit Geometry(const CachedParams& p)
        : tokens(kTileQ / p.group), heads(p.c.n_kv_heads), rest_rows(p.split ? kTokenRows : 0) {}
};

struct SeqLine {
    SeqView v;
    int32_t blocks;
    int32_t by_prefix, by_prefix_until, by_order_until;  // keys that blocks before by_prefix_until see; blocks after by_order_until see all
    __device__ __forceinline__ SeqLine(const CachedParams& p, const Geometry& g, int s) : v(load_seq(p.b, p.c.page_shift, s)) {
        const uint32_t T = 2 * g.tokens;
        blocks = (int32_t)((uint32_t)v.q_len / T + ((uint32_t)v.q_len % T != 0));
        if ((int64_t)v.q_len * p.group <= g.rest_rows) blocks = 0;
        by_prefix = min(v.keys, max(v.prefix, 0));
        by_prefix_until = by_order_until = blocks;
        if (by_prefix < v.keys) {  // (differences of numbers of 31 bits and a sign: they fit 32 bits without one)
            by_prefix_until = by_prefix < v.pos0 ? 0 : (int32_t)min((uint32_t)blocks, ((uint32_t)by_prefix - (uint32_t)v.pos0) / T);
            by_order_until = v.keys < v.pos0 ? by_prefix_until
                                             : max(by_prefix_until, (int32_t)min((uint32_t)blocks, ((uint32_t)v.keys - (uint32_t)v.pos0) / T));
        }
    }
    __device__ __forceinline__ int32_t block_tokens(const Geometry& g, int b) const { return min(2 * g.tokens, v.q_len - b * 2 * g.tokens); }
    __device__ __forceinline__ int32_t block_keys(const Geometry& g, int b) const {
        return keys_seen(v, b * 2 * g.tokens + block_tokens(g, b) - 1);
    }
    __device__ __forceinline__ int64_t block_cost(const Geometry& g, int b) const {
        return kItemCost + (int64_t)block_keys(g, b) * (block_tokens(g, b) > g.tokens ? kTwoCost : kOneCost);
    }
    // Cost of blocks 0 .. b - 1 for one head, all of them full: kTwoCost times the sum of min(keys, max(prefix, pos0 + (i + 1) T)).
    __device__ __forceinline__ int64_t cost_before(const Geometry& g, int b) const {
        const int64_t T = 2 * g.tokens, i0 = min(b, by_prefix_until), i1 = min(b, by_order_until);
        const int64_t keys = i0 * by_prefix + (i1 - i0) * v.pos0 + (i1 * (i1 + 1) - i0 * (i0 + 1)) / 2 * T + (b - i1) * (int64_t)v.keys;
        return (int64_t)b * kItemCost + kTwoCost * keys;
    }
    __device__ __forceinline__ int64_t units(const Geometry& g) const {
        return blocks == 0 ? 0 : g.heads * (cost_before(g, blocks - 1) + block_cost(g, blocks - 1));
    }
};

// The items of a CTA's stretch [begin, end), in order.
struct ItemWalk {
    const CachedParams& p;
    const Geometry g;
    SeqLine line;
    int64_t base, at, end, per;
    int32_t s;

    __device__ __forceinline__ ItemWalk(const CachedParams& p_, int32_t s_, int64_t base_, int64_t per_, int64_t total)
        : p(p_), g(p_), line(p_, g, s_), base(base_), at(per_ * blockIdx.x), per(per_), s(s_) {
        end = min(at + per, total);
    }
    __device__ __forceinline__ bool next(Item& w) {
        while (at < end) {
            int64_t units = line.units(g);
            while (at >= base + units) {
                base += units;
                line = SeqLine(p, g, ++s);
                units = line.units(g);
            }
            int lo = 0, hi = line.blocks - 1;  // the last block that begins at or before `at`
            const int64_t in = at - base;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (g.heads * line.cost_before(g, mid) <= in) lo = mid; else hi = mid - 1;
            }
            const int64_t cost = line.block_cost(g, lo);
            const int64_t block0 = g.heads * line.cost_before(g, lo);
            const int32_t head = (int32_t)quotient(in - block0, cost);
            const int64_t item0 = base + block0 + head * cost;
            const int64_t stop = min(end, item0 + cost);
            const int32_t keys = line.block_keys(g, lo), tokens = line.block_tokens(g, lo);
            const bool two = tokens > g.tokens;
            const int32_t tiles = (keys + kTileKV - 1) / kTileKV;
            const int64_t step = kTileKV * (two ? kTwoCost : kOneCost), first = item0 + kItemCost;  // tile t lies where its first key does
            auto tiles_before = [&](int64_t u) { return u <= first ? 0 : (int32_t)min((int64_t)tiles, quotient(u - first + step - 1, step)); };
            const int32_t tile0 = tiles_before(at), tile1 = tiles_before(stop);
            const bool starts_here = at == item0;
            at = stop;
            if (tile1 <= tile0 && !(tiles == 0 && starts_here)) continue;  // only the start of an item whose tiles lie in later CTAs
            const int32_t c_first = tiles > 0 ? (int32_t)quotient(first, per) : 0;
            w = Item{s, head, tile0, tile1, lo * 2 * g.tokens, tokens, keys, two ? 1 : 0, line.v.q0, line.v.pos0, line.v.keys, line.v.prefix,
                     c_first, tiles > 0 ? (int32_t)quotient(first + (tiles - 1) * step, per) : 0, first > c_first * per ? 1 : 0, 0};
            return true;
        }
        return false;
    }
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); }

__device__ __forceinline__ void report(int32_t* status, volatile int32_t* abort_flag, int where) {
    *abort_flag = 1;
    if (atomicCAS(status, 0, (int)ZL_ERR_TIMEOUT) == 0) status[1] = where;
}
static __device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, const volatile int32_t* abort_flag) {
    return mbar_wait_slow(bar, parity, kWaitLimitNs, abort_flag);
}

// Behind an expired wait: at most a second more for what the CTA itself has under way.
static __device__ __noinline__ void wait_drained(uint64_t* bar, uint32_t parity) {
    const int32_t go_on = 0;
    mbar_wait(bar, parity, 1000000000ull, &go_on);
}

// A store of the lanes that have something to store, without a branch: the warp stays together for the collective instructions behind it.
__device__ __forceinline__ void store_if(bool live, void* to, const uint4& x) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\t}" ::"l"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w),
                 "r"((uint32_t)live)
                 : "memory");
}

// All lanes of a warp wait; the outcome is warp-uniform and the warp reconverges.
#define ZL_WAIT_WARP(bar, parity, site)                                                                       \
    do {                                                                                                      \
        const bool ok_ = mbar_try_wait((bar), (parity)) || wait_slow((bar), (parity), &sm.abort_flag);      \
        if (!__all_sync(0xffffffffu, ok_)) {                                                                  \
            report(p.status, &sm.abort_flag, 7000 + (site));                                                 \
            goto teardown;                                                                                    \
        }                                                                                                     \
    } while (0)
// The same from the warps that hold tiles in registers.
#define ZL_WAIT_REGS(bar, parity, site)                                            \
    do {                                                                           \
        const bool ok_ = mbar_wait((bar), (parity), kWaitLimitNs, &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                       \
            report(p.status, &sm.abort_flag, 7000 + (site));                      \
            goto teardown;                                                         \
        }                                                                          \
    } while (0)

// for (every item `w` of the CTA) { ... ZL_ITEM_DONE }
#define ZL_FOR_ITEMS(wait_, site)                                          \
    for (uint32_t it_ = 0;; ++it_) {                                       \
        const uint32_t slot_ = it_ % kItems;                               \
        wait_(&sm.item_full[slot_], (it_ / kItems) & 1, site);             \
        const Item& w = sm.items[slot_];                                   \
        if (w.tile1 < 0) break;                                            \
        const int n = w.tile1 - w.tile0;
#define ZL_ITEM_DONE                                                       \
        __syncwarp();                                                      \
        if (lane == 0) mbar_arrive(&sm.item_empty[slot_]);                 \
    }

template <int D, int kFormat>
__global__ void __launch_bounds__(kFormat == ZL_CACHE_BF16 ? 384 : 512, 1)
zl_cached_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const CachedParams p) {
    using Smem = ChunkSmem<D, kFormat>;
    constexpr bool kCodes = Smem::kCodes;
    constexpr int kBoxes = Smem::kBoxes, kStages = Smem::kStages;
    constexpr int kThreads = kCodes ? 512 : 384;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    // TMEM columns: S_0 [0,128), S_1 [128,256), O_0 [256,256+D), O_1 [384,384+D); P_x over the first half of S_x
    constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;

    if ((smem_u32(smem_raw) & 1023u) != 0) {  // swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0 && atomicCAS(p.status, 0, (int)ZL_ERR_CUDA) == 0) p.status[1] = 7999;
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&sm.q_full, 1);
        mbar_init(&sm.q_empty, 1);
        mbar_init(&sm.q_max, 128);
        mbar_init(&sm.q_ready, 128);
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sm.s_full[x], 1);
            mbar_init(&sm.p_half[x][0], 256);
            mbar_init(&sm.p_half[x][1], 256);
            mbar_init(&sm.o_full[x], 1);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.k_full[s], kCodes ? 128 : 1);
            mbar_init(&sm.k_empty[s], 1);
            mbar_init(&sm.v_full[s], kCodes ? 128 : 1);
            mbar_init(&sm.v_empty[s], 1);
        }
        if constexpr (kCodes) {
            for (int s = 0; s < kStages; ++s) {
                mbar_init(&sm.k_codes[s], 1);
                mbar_init(&sm.v_codes[s], 1);
            }
            mbar_init(&sm.codes_read, 128);
        }
        for (int s = 0; s < kMaskRing; ++s) mbar_init(&sm.tile_full[s], kCodes ? 128 : 1);
        mbar_init(&sm.stat_full, 256);
        mbar_init(&sm.drained, 1);
        for (int i = 0; i < kItems; ++i) {
            mbar_init(&sm.item_full[i], 1);
            mbar_init(&sm.item_empty[i], kCodes ? 14 : 10);  // warps that read it
        }
        sm.q_loads = sm.k_loads = sm.v_loads = 0;
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
    // (in this order: the tokens kernel behind it starts on the strength of what this grid has waited for)
    grid_wait();
    grid_release();
    if (threadIdx.x == 0) reinterpret_cast<Item*>(p.chunk_cut)[blockIdx.x].tile1 = -1;  // (what an earlier call left must not be joined)

    // ---- where this CTA's stretch begins
    {
        const Geometry g(p);
        const int tid = threadIdx.x, chunk = (p.b.n_seqs + kThreads - 1) / kThreads;
        const int s_end = min((tid + 1) * chunk, p.b.n_seqs);
        int64_t mine = 0;
        for (int s = tid * chunk; s < s_end; ++s) mine += SeqLine(p, g, s).units(g);
        int64_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) sm.scan[warp] = upto;
        __syncthreads();
        int64_t before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += sm.scan[w];
            total += sm.scan[w];
        }
        const int64_t per = max(quotient(total + gridDim.x - 1, gridDim.x), kLeastUnits);
        const int64_t begin = per * blockIdx.x;
        int64_t at = before + upto - mine;
        if (tid == 0) sm.total = total;
        if (at <= begin && begin < at + mine) {  // one thread
            int s = tid * chunk;
            while (true) {
                const int64_t n = SeqLine(p, g, s).units(g);
                if (begin < at + n) break;
                at += n;
                ++s;
            }
            sm.start_seq = s;
            sm.start_base = at;
        }
        __syncthreads();
    }
    const int64_t total = sm.total;
    const int64_t per = max(quotient(total + gridDim.x - 1, gridDim.x), kLeastUnits);
    if (per * blockIdx.x >= total) goto teardown;  // (nothing for this CTA)

    if (warp < 4) {
        if constexpr (kCodes) reg_dec<80>(); else reg_dec<136>();
        if (warp == 2) {
            // -------------------------------------------------------------- the line of work
            ItemWalk walk(p, sm.start_seq, sm.start_base, per, total);
            bool more = true;
            for (uint32_t it = 0; more; ++it) {
                Item w;
                more = walk.next(w);
                if (!more) w.tile1 = -1;
                // the item, if any, whose first part is the last of this CTA's stretch
                if (more && lane == 0 && w.c_first == (int32_t)blockIdx.x && w.c_last > w.c_first) reinterpret_cast<Item*>(p.chunk_cut)[blockIdx.x] = w;
                ZL_WAIT_WARP(&sm.item_empty[it % kItems], ((it / kItems) & 1) ^ 1, 9);
                if (lane == 0) {
                    sm.items[it % kItems] = w;
                    mbar_arrive(&sm.item_full[it % kItems]);
                }
            }
        } else if (warp == 0) {
            // -------------------------------------------------------------- TMA producer (a lane per page)
            const int32_t tile_tokens = kTileQ / p.group;
            const int page = 1 << p.c.page_shift;
            const int box = min(page, kTileKV);
            const int row = lane * box;          // this lane's rows of a tile: [row, row + box)
            const bool has_rows = row < kTileKV;
            uint32_t item_cnt = 0, kv_cnt = 0;
            // (entries of the table: what they mean is asked a tile later, when they are there)
            auto page_of = [&](const Item& w, int32_t pos) { return has_rows && pos < w.keys ? page_entry(p.b, p.c, w.s, pos) : -1; };
            auto load = [&](const Item& w, uint8_t* dst, const CUtensorMap* tm, uint64_t* bar, uint32_t* count, uint32_t c, int32_t pg, int32_t pos) {
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, pg >= 0));
                if (lane == 0) {
                    *count = c + 1;
                    mbar_arrive_expect_tx(bar, n * box * (kCodes ? D : D * 2));
                }
                __syncwarp();
                if (pg >= 0) {
                    const int32_t in = pos & (page - 1);
                    const int32_t c1 = p.head_first ? w.head : in, c2 = p.head_first ? in : w.head;
                    if constexpr (kCodes) {
                        tma_load_4d(dst + Smem::kTileBytes / 2 + row * D, tm, bar, 0, c1, c2, pg);
                    } else {
#pragma unroll
                        for (int b = 0; b < kBoxes; ++b) tma_load_4d(dst + b * Smem::kBoxBytes + row * 128, tm, bar, b * 64, c1, c2, pg);
                    }
                }
            };
            ZL_FOR_ITEMS(ZL_WAIT_WARP, 6)
                if (n > 0) {
                ZL_WAIT_WARP(&sm.q_empty, (item_cnt & 1) ^ 1, 1);
                ++item_cnt;
                if (lane == 0) {
                    const int q_tiles = w.two ? 2 : 1;
                    sm.q_loads = item_cnt;
                    mbar_arrive_expect_tx(&sm.q_full, q_tiles * tile_tokens * p.group * D * 2);
                    for (int x = 0; x < q_tiles; ++x)
                        for (int b = 0; b < kBoxes; ++b)
                            tma_load_4d(sm.q[x] + b * Smem::kBoxBytes, &tm_q, &sm.q_full, b * 64, 0, w.head, w.q0 + w.tok0 + x * tile_tokens);
                }
                {  // K runs one tile ahead of V
                    int32_t pg_k = valid_page(p.c, page_of(w, w.tile0 * kTileKV + row)), pg_v = -1;
                    for (int j = 0; j <= n; ++j) {
                        const int32_t key0 = (w.tile0 + j) * kTileKV;
                        const int32_t pg_next = j + 1 < n ? page_of(w, key0 + kTileKV + row) : -1;
                        if (j < n) {
                            const uint32_t c = kv_cnt + j, st = c % kStages;
                            ZL_WAIT_WARP(&sm.k_empty[st], ((c / kStages) & 1) ^ 1, 2);
                            if constexpr (!kCodes) {
                                const int32_t end_row = pg_k >= 0 ? row + min(box, w.keys - (key0 + row)) : 0;  // first row without a key
                                uint32_t word = 0;
    #pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint32_t all = __reduce_or_sync(0xffffffffu, pg_k >= 0 ? low_bits(end_row - 32 * i) & ~low_bits(row - 32 * i) : 0u);
                                    if (lane == i) word = all;
                                }
                                if (lane < 4) sm.mask[c % kMaskRing][lane] = word;
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&sm.tile_full[c % kMaskRing]);
                            }
                            load(w, sm.k[st], &tm_k, kCodes ? &sm.k_codes[st] : &sm.k_full[st], &sm.k_loads, c, pg_k, key0 + row);
                        }
                        if (j > 0) {
                            const uint32_t c = kv_cnt + j - 1, st = c % kStages;
                            ZL_WAIT_WARP(&sm.v_empty[st], ((c / kStages) & 1) ^ 1, 3);
                            load(w, sm.v[st], &tm_v, kCodes ? &sm.v_codes[st] : &sm.v_full[st], &sm.v_loads, c, pg_v, key0 - kTileKV + row);
                        }
                        pg_v = pg_k;
                        pg_k = valid_page(p.c, pg_next);
                    }
                    kv_cnt += n;
                }
                }
            ZL_ITEM_DONE
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMA issuer (whole warp, one elected lane issues)
            const bool mma_lane = elect_one();
            constexpr uint32_t idesc_s = make_idesc_f16(kCodes, kTileQ, kTileKV, 0, 0);
            constexpr uint32_t idesc_o = make_idesc_f16(kCodes, kTileQ, D, 0, 1);
            const uint64_t dq0 = make_desc_sw128(smem_u32(sm.q[0]), 16, 1024);
            const uint64_t dk0 = make_desc_sw128(smem_u32(sm.k[0]), 16, 1024);
            const uint64_t dv0 = make_desc_sw128(smem_u32(sm.v[0]), Smem::kBoxBytes, 1024);  // V is the MN-major B operand
            constexpr uint32_t kTileStep = Smem::kTileBytes >> 4;
            // Stages and phases are counted, not computed: this warp's own instructions lie on the way from P to the next scores.
            uint32_t item_cnt = 0, tile_cnt = 0, k_st = 0, k_ph = 0, v_st = 0, v_ph = 0, p_ph[2] = {0, 0};
            auto issue_s = [&](int x, int q) {  // S_x = Q_q K^T, over P_x of the step before: ordered after its P V on the tensor pipe
                const uint64_t dq = dq0 + q * kTileStep, dk = dk0 + k_st * kTileStep;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = ((ks / 4) * Smem::kBoxBytes + (ks % 4) * 32) >> 4;
                    if (mma_lane) mma_ss(tmem + kColS + x * 128, dq + off, dk + off, idesc_s, ks > 0);
                }
                if (mma_lane) mma_commit(&sm.s_full[x]);
            };
            auto issue_pv = [&](int x, int half, bool acc) {  // O_x (+)= P_x V over one half of the key columns
                const uint64_t dv = dv0 + v_st * kTileStep + half * (kTileKV / 32) * (2048 >> 4);
#pragma unroll
                for (int ks = 0; ks < kTileKV / 32; ++ks)
                    if (mma_lane)
                        mma_ts(tmem + kColO + x * 128, tmem + kColS + x * 128 + (half * (kTileKV / 32) + ks) * 8, dv + ks * (2048 >> 4), idesc_o, acc || ks > 0);
            };
            auto done_with_k = [&]() {
                if (mma_lane) mma_commit(&sm.k_empty[k_st]);
                if (++k_st == kStages) { k_st = 0; k_ph ^= 1; }
            };
            auto done_with_v = [&]() {
                if (mma_lane) mma_commit(&sm.v_empty[v_st]);
                if (++v_st == kStages) { v_st = 0; v_ph ^= 1; }
                ++tile_cnt;
            };
            // bf16: rows without a key may hold anything, NaN too: zeros, before they meet their weight of 0
            auto clean_v = [&]() {
                if constexpr (!kCodes) {
                    const uint4 m4 = *reinterpret_cast<const uint4*>(sm.mask[tile_cnt % kMaskRing]);
                    if ((m4.x & m4.y & m4.z & m4.w) != 0xffffffffu) {
                        const uint32_t words[4] = {m4.x, m4.y, m4.z, m4.w};
                        for (int i = 0; i < 4; ++i) {
                            if ((words[i] >> lane) & 1) continue;
                            const uint32_t at = smem_u32(sm.v[v_st]) + (i * 32 + lane) * 128;
#pragma unroll 1
                            for (int e = 0; e < 8 * kBoxes; ++e) st_shared_v4(at + (e >> 3) * Smem::kBoxBytes + (((e + lane) & 7) << 4), 0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                }
            };
#define ZL_PV(x_, acc_)                                                \
            do {                                                       \
                ZL_WAIT_WARP(&sm.p_half[x_][0], p_ph[x_], 13);         \
                tc_fence_after();                                      \
                issue_pv(x_, 0, acc_);                                 \
                ZL_WAIT_WARP(&sm.p_half[x_][1], p_ph[x_], 14);         \
                tc_fence_after();                                      \
                issue_pv(x_, 1, true);                                 \
                p_ph[x_] ^= 1;                                         \
            } while (0)
            ZL_FOR_ITEMS(ZL_WAIT_WARP, 7)
                if (n > 0) {
                    ZL_WAIT_WARP(kCodes ? &sm.q_ready : &sm.q_full, item_cnt & 1, 11);
                    ++item_cnt;
                    ZL_WAIT_WARP(&sm.k_full[k_st], k_ph, 15);
                    tc_fence_after();
                    issue_s(0, 0);
                    if (w.two) {
                        issue_s(1, 1);
                        done_with_k();
                        if (n == 1) if (mma_lane) mma_commit(&sm.q_empty);
                        for (int j = 0; j < n; ++j) {
                            const bool next = j + 1 < n;
                            ZL_WAIT_WARP(&sm.v_full[v_st], v_ph, 12);
                            clean_v();
                            ZL_PV(0, j > 0);
                            if (next) {
                                ZL_WAIT_WARP(&sm.k_full[k_st], k_ph, 16);
                                tc_fence_after();
                                issue_s(0, 0);
                            } else if (mma_lane) {
                                mma_commit(&sm.o_full[0]);
                            }
                            ZL_PV(1, j > 0);
                            done_with_v();
                            if (next) {
                                issue_s(1, 1);
                                done_with_k();
                                if (j + 2 == n) if (mma_lane) mma_commit(&sm.q_empty);  // the item's last S
                            } else if (mma_lane) {
                                mma_commit(&sm.o_full[1]);
                            }
                        }
                    } else {
                        // key tiles in turn to the two accumulators: S two tiles ahead of P V
                        done_with_k();
                        if (n > 1) {
                            ZL_WAIT_WARP(&sm.k_full[k_st], k_ph, 17);
                            tc_fence_after();
                            issue_s(1, 0);
                            done_with_k();
                        }
                        if (n <= 2) if (mma_lane) mma_commit(&sm.q_empty);
                        for (int j = 0; j < n; j += 2) {
                            ZL_WAIT_WARP(&sm.v_full[v_st], v_ph, 18);
                            clean_v();
                            ZL_PV(0, j > 0);
                            done_with_v();
                            if (j + 2 < n) {
                                ZL_WAIT_WARP(&sm.k_full[k_st], k_ph, 19);
                                tc_fence_after();
                                issue_s(0, 0);
                                done_with_k();
                                if (j + 3 == n) if (mma_lane) mma_commit(&sm.q_empty);
                            } else if (mma_lane) {
                                mma_commit(&sm.o_full[0]);
                            }
                            if (j + 1 == n) break;
                            ZL_WAIT_WARP(&sm.v_full[v_st], v_ph, 40);
                            clean_v();
                            ZL_PV(1, j > 0);
                            done_with_v();
                            if (j + 3 < n) {
                                ZL_WAIT_WARP(&sm.k_full[k_st], k_ph, 41);
                                tc_fence_after();
                                issue_s(1, 0);
                                done_with_k();
                                if (j + 4 == n) if (mma_lane) mma_commit(&sm.q_empty);
                            } else if (mma_lane) {
                                mma_commit(&sm.o_full[1]);
                            }
                        }
                    }
                }
            ZL_ITEM_DONE
        }
    } else if (kCodes && warp >= 12) {
        // ------------------------------------------------------------------ codes to fp16
        reg_dec<80>();
        if constexpr (kCodes) {
            const int t = threadIdx.x - 384;
            // This thread's 16-byte pieces of a tile of codes: piece `ch` of rows r, r + kRowStep, ... (a multiple of 8: the exchange
            // of pieces within a line is the same for all of them).  A piece of 16 codes becomes two of eight numbers; in the
            // second box the odd one goes first, so that eight lanes meet all banks.
            constexpr int kChunks = D / 16, kRowStep = 128 / kChunks, kPieces = kTileKV / kRowStep;
            const int r = t / kChunks, ch = t % kChunks;
            const bool swap = ch >= 4;
            const uint32_t from = Smem::kTileBytes / 2 + r * D + ((ch ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
            const uint32_t to = (ch >> 2) * Smem::kBoxBytes + r * 128;
            const uint32_t to0 = to + (((2 * (ch & 3) + (swap ? 1 : 0)) ^ (r & 7)) << 4), to1 = to0 ^ 16;
            uint32_t kv_cnt = 0, read_cnt = 0, item_cnt = 0;
            auto page_of = [&](const Item& w, int32_t key) { return key < w.keys ? page_entry(p.b, p.c, w.s, key) : -1; };
            // scales of this thread's key (key t of the tile), zeros without one
            auto scales_of = [&](const Item& w, int32_t key, int32_t pg) {
                float2 r = make_float2(0.f, 0.f);
                if (pg >= 0) {
                    const int64_t at = pg * p.c.scale_page + (key & ((1 << p.c.page_shift) - 1)) * p.c.scale_token + w.head * p.c.scale_head;
                    r = make_float2(__ldg(p.c.k_scale + at), __ldg(p.c.v_scale + at));
                }
                return r;
            };
            ZL_FOR_ITEMS(ZL_WAIT_WARP, 8)
                if (n > 0) {
                // ---- queries: a thread has row t of both tiles.  One factor for the item: the keys' scales take it back
                ZL_WAIT_WARP(&sm.q_full, item_cnt & 1, 30);
                float scores_by;
                {
                    const int q_tiles = w.two ? 2 : 1;
                    float big = 0.f;
                    const int32_t row_tok = t / p.group, tile_tokens = kTileQ / p.group;
                    for (int x = 0; x < q_tiles; ++x)
                        if (row_tok < tile_tokens && x * tile_tokens + row_tok < w.tokens)  // (other rows may hold anything)
#pragma unroll 4
                            for (int e = 0; e < 8 * kBoxes; ++e) {
                                const uint4 u = *reinterpret_cast<const uint4*>(sm.q[x] + (e >> 3) * Smem::kBoxBytes + t * 128 + (((e + t) & 7) << 4));
                                for (uint32_t v : {u.x, u.y, u.z, u.w}) big = max3_abs(big, __uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
                            }
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
                    if (lane == 0) sm.q_big[t >> 5] = big;
                    __syncwarp();
                    mbar_arrive(&sm.q_max);
                    ZL_WAIT_WARP(&sm.q_max, item_cnt & 1, 31);
                    float back;
                    const float factor = half_factor(fmaxf(fmaxf(sm.q_big[0], sm.q_big[1]), fmaxf(sm.q_big[2], sm.q_big[3])), back);
                    scores_by = back * p.scale_log2;
                    for (int x = 0; x < q_tiles; ++x)
#pragma unroll 4
                        for (int e = 0; e < 8 * kBoxes; ++e) {
                            uint4* const at = reinterpret_cast<uint4*>(sm.q[x] + (e >> 3) * Smem::kBoxBytes + t * 128 + (((e + t) & 7) << 4));
                            const uint4 u = *at;
                            *at = make_uint4(bf16_pair_to_half(u.x, factor), bf16_pair_to_half(u.y, factor), bf16_pair_to_half(u.z, factor),
                                             bf16_pair_to_half(u.w, factor));
                        }
                    fence_proxy_async_smem();
                    mbar_arrive(&sm.q_ready);
                    ++item_cnt;
                }
                // pages are looked up two tiles ahead, scales one: neither is waited for
                const int32_t key0 = w.tile0 * kTileKV + t;
                int32_t pg = valid_page(p.c, page_of(w, key0)), pg_next = page_of(w, key0 + kTileKV);
                float2 sc = scales_of(w, key0, pg);
                for (int j = 0; j <= n; ++j) {
                    for (int m = 0; m < 2; ++m) {
                        if (m == 0 ? j == n : j == 0) continue;
                        const uint32_t c = kv_cnt + j - m, st = c % kStages;
                        if (m == 0) {
                            const uint32_t word = __ballot_sync(0xffffffffu, pg >= 0);
                            const float v_scale = fmaxf(sc.y, kLeastScale);
                            sm.key_scale[c % Smem::kScaleRing][t] = sc.x * scores_by;
                            sm.value_log2[c % Smem::kScaleRing][t] = log2f(v_scale);
                            sm.value_inv[c % Smem::kScaleRing][t] = 1.f / v_scale;
                            if (lane == 0) sm.mask[c % kMaskRing][t >> 5] = word;
                            __syncwarp();
                            mbar_arrive(&sm.tile_full[c % kMaskRing]);
                            pg = valid_page(p.c, pg_next);
                            sc = scales_of(w, key0 + (j + 1) * kTileKV, pg);
                            pg_next = page_of(w, key0 + (j + 2) * kTileKV);
                        }
                        uint8_t* const tile = m == 0 ? sm.k[st] : sm.v[st];
                        ZL_WAIT_WARP(m == 0 ? &sm.k_codes[st] : &sm.v_codes[st], (c / kStages) & 1, 5);
                        uint4 code[kPieces];
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) code[i] = *reinterpret_cast<const uint4*>(tile + from + i * kRowStep * D);
                        // all codes have been read when the first of them is written over
                        mbar_arrive(&sm.codes_read);
                        // rows without a key may hold codes of NaN: zeros, before they meet their weight of 0
                        if (kFormat == ZL_CACHE_E4M3 && m == 1) {
                            ZL_WAIT_WARP(&sm.tile_full[c % kMaskRing], (c / kMaskRing) & 1, 32);
                            const uint4 there = *reinterpret_cast<const uint4*>(sm.mask[c % kMaskRing]);
                            if ((there.x & there.y & there.z & there.w) != ~0u) {
#pragma unroll
                                for (int i = 0; i < kPieces; ++i) {
                                    const int row = r + i * kRowStep;
                                    const uint32_t word = row < 64 ? (row < 32 ? there.x : there.y) : (row < 96 ? there.z : there.w);
                                    if (!((word >> (row & 31)) & 1)) code[i] = make_uint4(0, 0, 0, 0);
                                }
                            }
                        }
                        ZL_WAIT_WARP(&sm.codes_read, read_cnt & 1, 4);
                        ++read_cnt;
                        const uint32_t dst = smem_u32(tile);
#pragma unroll
                        for (int i = 0; i < kPieces; ++i) {
                            const uint32_t a = swap ? code[i].z : code[i].x, b = swap ? code[i].w : code[i].y;
                            const uint32_t c_ = swap ? code[i].x : code[i].z, d = swap ? code[i].y : code[i].w;
                            const uint32_t at = dst + i * kRowStep * 128;
                            uint32_t y[8];
                            halves<kFormat>(a, y[0], y[1]);
                            halves<kFormat>(b, y[2], y[3]);
                            halves<kFormat>(c_, y[4], y[5]);
                            halves<kFormat>(d, y[6], y[7]);
                            st_shared_v4(at + to0, y[0], y[1], y[2], y[3]);
                            st_shared_v4(at + to1, y[4], y[5], y[6], y[7]);
                        }
                        fence_proxy_async_smem();
                        mbar_arrive(m == 0 ? &sm.k_full[st] : &sm.v_full[st]);
                    }
                }
                kv_cnt += n;
                }
            ZL_ITEM_DONE
        }
    } else {
        // ------------------------------------------------------------------ softmax, join and output
        if constexpr (kCodes) reg_inc<176>(); else reg_inc<184>();
        const int x = (warp - 4) >> 2;             // half of the rows of a warp's TMEM quarter; tile or columns of the output
        const int quarter = warp & 3;              // TMEM lane quarter this warp may access
        const int row = quarter * 32 + lane;       // of the output
        const int quad = lane & 3;
        const uint32_t lane_addr = tmem + ((uint32_t)(quarter * 32) << 16), slab_addr = lane_addr + ((uint32_t)(x * 16) << 16);
        const float mul = kCodes ? 1.f : p.scale_log2;  // (of 8-bit caches the keys' scales have it)
        const int32_t tile_tokens = kTileQ / p.group;
        const int32_t row_tok = row / p.group, row_head = row - row_tok * p.group;
        const int32_t slab_row = quarter * 32 + x * 16 + (lane >> 2);  // this thread's rows of S: slab_row, slab_row + 8
        const int32_t slab_tok[2] = {slab_row / p.group, (slab_row + 8) / p.group};
        uint32_t kv_cnt = 0, s_ph[2] = {0, 0}, o_cnt[2] = {0, 0}, join_cnt = 0;
        ZL_FOR_ITEMS(ZL_WAIT_REGS, 28)
            const bool two = w.two != 0;
            // (rows that do not exist hold anything, and take no part in what a warp decides together)
            int32_t seen[2][2], seen_least[2];
            bool ok[2][2];
            float m2[2][2], l2[2][2];  // of S_0 and S_1: reference maximum in powers of two, sum
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int32_t tk = w.tok0 + (two ? y * tile_tokens : 0) + slab_tok[b];
                    ok[y][b] = slab_tok[b] < tile_tokens && tk < w.tok0 + w.tokens;
                    seen[y][b] = ok[y][b] ? keys_seen(w.seq(), tk) - w.tile0 * kTileKV : INT32_MAX;
                    m2[y][b] = -INFINITY;
                    l2[y][b] = 0.f;
                }
                seen_least[y] = __reduce_min_sync(0xffffffffu, min(seen[y][0], seen[y][1]));
            }
            // One step: P of accumulator Y against key tile j of this part.
            float2 by_key[kCodes ? 16 : 1], by_value[kCodes ? 16 : 1];  // 8-bit caches: of this thread's columns of key tile j
            auto step = [&](auto which, auto fetch, int j, bool first) -> bool {
                constexpr int Y = decltype(which)::value;
                const uint32_t c = kv_cnt + j;
                const bool okay = mbar_wait(&sm.tile_full[c % kMaskRing], (c / kMaskRing) & 1, kWaitLimitNs, &sm.abort_flag) &&
                                  mbar_wait(&sm.s_full[Y], s_ph[Y], kWaitLimitNs, &sm.abort_flag);
                if (!__all_sync(0xffffffffu, okay)) return false;
                s_ph[Y] ^= 1;
                tc_fence_after();
                // in the layout of an mma accumulator: 32 columns (8 k + 2 (lane % 4) + {0, 1}) of two rows
                float2 sv[2][16];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t r[32];
                    tmem_ld_16x64(slab_addr + kColS + Y * 128 + h * 64, r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        sv[0][h * 8 + k] = make_float2(__uint_as_float(r[4 * k]), __uint_as_float(r[4 * k + 1]));
                        sv[1][h * 8 + k] = make_float2(__uint_as_float(r[4 * k + 2]), __uint_as_float(r[4 * k + 3]));
                    }
                }
                if constexpr (kCodes && decltype(fetch)::value) {  // (fetched under the load of S; eight lanes share a column's)
                    const float2* ks = reinterpret_cast<const float2*>(sm.key_scale[c % Smem::kScaleRing]) + quad;
                    const float2* vl = reinterpret_cast<const float2*>(sm.value_log2[c % Smem::kScaleRing]) + quad;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        by_key[k] = ks[4 * k];
                        by_value[k] = vl[4 * k];
                    }
                }
                const uint4 m128 = *reinterpret_cast<const uint4*>(sm.mask[c % kMaskRing]);
                tmem_wait_ld();
                if constexpr (kCodes) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        sv[0][k] = fma2(sv[0][k], by_key[k], by_value[k]);
                        sv[1][k] = fma2(sv[1][k], by_key[k], by_value[k]);
                    }
                }
                if (seen_least[Y] - j * kTileKV < kTileKV || (m128.x & m128.y & m128.z & m128.w) != 0xffffffffu) {
                    const uint32_t words[4] = {m128.x, m128.y, m128.z, m128.w};
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int valid = ok[Y][b] ? seen[Y][b] - j * kTileKV : kTileKV;
#pragma unroll
                        for (int k = 0; k < 16; ++k) {  // select, never multiply
                            const uint32_t keep = (words[k >> 2] & low_bits(valid - 32 * (k >> 2))) >> (8 * (k & 3) + 2 * quad);
                            if (!(keep & 1)) sv[b][k].x = -INFINITY;
                            if (!(keep & 2)) sv[b][k].y = -INFINITY;
                        }
                    }
                }
                float mx[2];
                bool raise = false;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float u = max3(sv[b][0].x, sv[b][0].y, sv[b][1].x), v = max3(sv[b][1].y, sv[b][2].x, sv[b][2].y);
#pragma unroll
                    for (int k = 3; k < 15; k += 2) {
                        u = max3(u, sv[b][k].x, sv[b][k].y);
                        v = max3(v, sv[b][k + 1].x, sv[b][k + 1].y);
                    }
                    mx[b] = fmaxf(max3(u, sv[b][15].x, sv[b][15].y), v) * mul;
                    raise |= ok[Y][b] && mx[b] - m2[Y][b] > kRescaleThresholdLog2;
                }
                if (__any_sync(0xffffffffu, raise)) {
                    // all lanes of a row take its maximum as the new reference; O is rescaled (the step before this one is complete: S of
                    // this one was issued after it)
                    float alpha[2];
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        mx[b] = fmaxf(mx[b], __shfl_xor_sync(0xffffffffu, mx[b], 1));
                        mx[b] = fmaxf(mx[b], __shfl_xor_sync(0xffffffffu, mx[b], 2));
                        alpha[b] = 1.f;
                        if (ok[Y][b] && mx[b] > m2[Y][b]) {
                            alpha[b] = ex2(m2[Y][b] - mx[b]);
                            l2[Y][b] *= alpha[b];
                            m2[Y][b] = mx[b];
                        }
                    }
                    __syncwarp();  // (the choice above is a lane's own)
                    if (!first) {
#pragma unroll 1
                        for (int h = 0; h < D / 64; ++h) {
                            const uint32_t at = slab_addr + kColO + Y * 128 + h * 64;
                            uint32_t r[32];
                            tmem_ld_16x64(at, r);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * alpha[(k >> 1) & 1]);
                            tmem_st_16x64(at, r);
                        }
                    }
                }
                const float2* vi = reinterpret_cast<const float2*>(sm.value_inv[kCodes ? c % Smem::kScaleRing : 0]) + quad;
                float2 nm[2], sum[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const float ref = m2[Y][b], nmb = ref == -INFINITY ? 0.f : -ref;  // (a row may have seen no key yet)
                    nm[b] = make_float2(nmb, nmb);
                    sum[b] = make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // P, rounded once, goes to the MMA warp in two halves of 64 key columns
                    uint32_t pk[16];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 f = kCodes ? vi[4 * (8 * h + k)] : make_float2(1.f, 1.f);
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float2 e = kCodes ? add2(sv[b][8 * h + k], nm[b]) : fma2(sv[b][8 * h + k], make_float2(mul, mul), nm[b]);
                            e = make_float2(ex2(e.x), ex2(e.y));
                            sum[b] = kCodes ? fma2(e, f, sum[b]) : add2(sum[b], e);
                            pk[2 * k + b] = kCodes ? pack_half(e.x, e.y) : pack_bf16(e.x, e.y);
                        }
                    }
                    tmem_st_16x32(slab_addr + kColS + Y * 128 + h * 32, pk);
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&sm.p_half[Y][h]);
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) l2[Y][b] += sum[b].x + sum[b].y;
                return true;
            };
            bool okay = true;
            if (two) {
                for (int j = 0; j < n && okay; ++j)
                    okay = step(std::integral_constant<int, 0>(), std::true_type(), j, j == 0) &&
                           step(std::integral_constant<int, 1>(), std::false_type(), j, j == 0);
            } else {
                for (int j = 0; j < n && okay; j += 2) {
                    okay = step(std::integral_constant<int, 0>(), std::true_type(), j, j == 0);
                    if (j + 1 < n && okay) okay = step(std::integral_constant<int, 1>(), std::true_type(), j + 1, j == 0);
                }
            }
            if (!okay) {
                report(p.status, &sm.abort_flag, 7021);
                goto teardown;
            }
            // ---- the item's end.  P V of the last steps has seen every warp, so all are through with the item before: the statistics'
            // place is free.  From here on a row per thread; with two query tiles warpgroup x writes tile x, with one half of its columns
            if (n > 0) {
                for (int y = 0; y < 2; ++y)
                    if (two || n > y) {
                        ZL_WAIT_REGS(&sm.o_full[y], o_cnt[y] & 1, 22 + y);
                        ++o_cnt[y];
                    }
                tc_fence_after();
            }
            const int32_t tok = w.tok0 + (two ? x * tile_tokens : 0) + row_tok;  // of the sequence
            const bool row_ok = row_tok < tile_tokens && tok < w.tok0 + w.tokens;
            float m_ref = -INFINITY, l = 0.f, wt[2] = {two && x == 1 ? 0.f : 1.f, two && x == 1 ? 1.f : 0.f};  // weights of the accumulators
            if (n > 0) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        l2[y][b] += __shfl_xor_sync(0xffffffffu, l2[y][b], 1);
                        l2[y][b] += __shfl_xor_sync(0xffffffffu, l2[y][b], 2);
                        if (quad == 0) sm.stat[y][slab_row + 8 * b] = make_float2(m2[y][b], l2[y][b]);
                    }
                mbar_arrive(&sm.stat_full);
                ZL_WAIT_REGS(&sm.stat_full, join_cnt & 1, 24);
                ++join_cnt;
                const float2 s0 = sm.stat[0][row], s1 = sm.stat[1][row];
                if (two) {
                    m_ref = x == 0 ? s0.x : s1.x;
                    l = x == 0 ? s0.y : s1.y;
                } else {
                    m_ref = fmaxf(s0.x, s1.x);
                    wt[0] = m_ref == -INFINITY ? 0.f : ex2(s0.x - m_ref);
                    wt[1] = m_ref == -INFINITY ? 0.f : ex2(s1.x - m_ref);
                    l = wt[0] * s0.y + wt[1] * s1.y;
                }
            }
            const int c0 = two ? 0 : x * (D / 2), n_cols = two ? D : D / 2;
            const int32_t c_first = w.c_first, c_last = w.c_last;
            const bool whole = c_first == c_last;
            const int64_t grow = (int64_t)w.q0 + tok;
            const int32_t q_head = w.head * p.group + row_head;
            const bool has_lse = row_ok && (two || x == 0);  // one thread per row
            const int64_t o_at = (grow * p.n_heads + q_head) * D + c0;
            const int tile = two ? x : 0;
            auto part_of = [&](int32_t cta) { return p.chunk_part + (((int64_t)cta * 2 + w.place(cta)) * 2 + tile) * kPartTileFloats<D>; };
            const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll 1
            for (int q = 0; q < n_cols / 32; ++q) {
                float o[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0.f;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if (two ? y == x && n > 0 : n > y) {
                        uint32_t r[32];
                        tmem_ld_x32(lane_addr + kColO + y * 128 + c0 + q * 32, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = fmaf(wt[y], __uint_as_float(r[i]), o[i]);
                    }
                }
                if (whole) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint4 o4;
                        o4.x = pack_bf16(o[i] * inv, o[i + 1] * inv);
                        o4.y = pack_bf16(o[i + 2] * inv, o[i + 3] * inv);
                        o4.z = pack_bf16(o[i + 4] * inv, o[i + 5] * inv);
                        o4.w = pack_bf16(o[i + 6] * inv, o[i + 7] * inv);
                        store_if(row_ok, p.o + o_at + q * 32 + i, o4);
                    }
                } else {
                    float4* to = reinterpret_cast<float4*>(part_of(blockIdx.x) + 2 * kTileQ) + (c0 / 4 + q * 8) * kTileQ + row;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        store_if(row_ok, to + i * kTileQ,
                                 make_uint4(__float_as_uint(o[4 * i]), __float_as_uint(o[4 * i + 1]), __float_as_uint(o[4 * i + 2]), __float_as_uint(o[4 * i + 3])));
                }
            }
            if (has_lse) {
                if (whole) {
                    if (p.lse) p.lse[(int64_t)q_head * p.b.total_q + grow] = l > 0.f ? (m_ref + log2f(l)) * kLn2 : -INFINITY;
                } else {
                    float* to = part_of(blockIdx.x);
                    to[row] = m_ref;
                    to[kTileQ + row] = l;
                }
            }
            tc_fence_before();
            kv_cnt += n;
        ZL_ITEM_DONE
    }

teardown:
    tc_fence_before();
    __syncthreads();
    if (sm.abort_flag) {
        // A wait has expired: copies and products that are still under way have to end before shared memory and TMEM are given up.
        if (warp == 0) {
            const uint32_t q_loads = sm.q_loads, k_loads = sm.k_loads, v_loads = sm.v_loads;
            if (q_loads > 0) wait_drained(&sm.q_full, (q_loads - 1) & 1);
            for (uint32_t i = 0; i < kStages; ++i) {  // the last load into each stage
                if (k_loads > i) wait_drained(kCodes ? &sm.k_codes[(k_loads - 1 - i) % kStages] : &sm.k_full[(k_loads - 1 - i) % kStages], ((k_loads - 1 - i) / kStages) & 1);
                if (v_loads > i) wait_drained(kCodes ? &sm.v_codes[(v_loads - 1 - i) % kStages] : &sm.v_full[(v_loads - 1 - i) % kStages], ((v_loads - 1 - i) / kStages) & 1);
            }
        } else if (warp == 1) {
            if (elect_one()) mma_commit(&sm.drained);
            __syncwarp();
            wait_drained(&sm.drained, 0);
        }
        __syncthreads();
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// ------------------------------------------------------------------------------------------------ parts of cut items
// Block (c, i): rows 32 i .. of the item that is cut first in CTA c, a row per lane.
// O = sum_c 2^(m_c - max) O_c / sum_c 2^(m_c - max) l_c over its parts.
constexpr int kJoinThreads = 128, kJoinRows = 32;

template <int D>
__global__ void __launch_bounds__(kJoinThreads)
zl_cached_join_kernel(const CachedParams p) {
    __shared__ __align__(16) __nv_bfloat16 out[kJoinRows][D + 8];
    grid_release();
    grid_wait();
    const Item w = reinterpret_cast<const Item*>(p.chunk_cut)[blockIdx.x];
    if (w.tile1 < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = blockIdx.y * kJoinRows / kTileQ, row0 = blockIdx.y * kJoinRows % kTileQ, row = row0 + lane;
    const int32_t tile_tokens = kTileQ / p.group, tok0 = w.tok0 + tile * tile_tokens;
    if ((tile == 1 && !w.two) || row0 / p.group >= min(tile_tokens, w.tok0 + w.tokens - tok0)) return;
    const int32_t parts = w.c_last - w.c_first + 1;
    auto part_of = [&](int32_t i) {
        return p.chunk_part + (((int64_t)(w.c_first + i) * 2 + (i == 0 ? w.place_first : 0)) * 2 + tile) * kPartTileFloats<D>;
    };
    float m = -INFINITY, l = 0.f;
#pragma unroll 8
    for (int i = 0; i < parts; ++i) m = fmaxf(m, __ldcg(part_of(i) + row));
    constexpr int kEach = D / 4 / (kJoinThreads / 32);  // quadruples of columns of a warp
    float4 acc[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m > -INFINITY) {
#pragma unroll 2
        for (int i = 0; i < parts; ++i) {
            const float* part = part_of(i);
            const float f = ex2(__ldcg(part + row) - m);
            l = fmaf(f, __ldcg(part + kTileQ + row), l);
            const float4* from = reinterpret_cast<const float4*>(part + 2 * kTileQ) + (warp * kEach) * kTileQ + row;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const float4 x = __ldcg(from + e * kTileQ);
                acc[e].x = fmaf(f, x.x, acc[e].x); acc[e].y = fmaf(f, x.y, acc[e].y); acc[e].z = fmaf(f, x.z, acc[e].z); acc[e].w = fmaf(f, x.w, acc[e].w);
            }
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < kEach; ++e)
        *reinterpret_cast<uint2*>(&out[lane][(warp * kEach + e) * 4]) = make_uint2(pack_bf16(acc[e].x * inv, acc[e].y * inv), pack_bf16(acc[e].z * inv, acc[e].w * inv));
    __syncthreads();
    constexpr int kChunks = D / 8;
    for (int j = threadIdx.x; j < kJoinRows * kChunks; j += kJoinThreads) {
        const int r = j / kChunks, tok = (row0 + r) / p.group, head = w.head * p.group + (row0 + r) - tok * p.group;
        if (tok >= tile_tokens || tok0 + tok >= w.tok0 + w.tokens) continue;
        const int64_t grow = (int64_t)w.q0 + tok0 + tok;
        *reinterpret_cast<uint4*>(p.o + (grow * p.n_heads + head) * D + j % kChunks * 8) = *reinterpret_cast<const uint4*>(&out[r][j % kChunks * 8]);
    }
    if (warp == 0 && p.lse) {
        const int tok = row / p.group, head = w.head * p.group + row - tok * p.group;
        if (tok < tile_tokens && tok0 + tok < w.tok0 + w.tokens)
            p.lse[(int64_t)head * p.b.total_q + w.q0 + tok0 + tok] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
}

template <int D, int kFormat>
cudaError_t launch_t(const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CachedParams& p, int grid, cudaStream_t stream) {
    constexpr int smem = sizeof(ChunkSmem<D, kFormat>);
    static_assert(smem <= 232448, "shared memory of a CTA");
    constexpr int kMaxDevices = 64;
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_cached_chunk_kernel<D, kFormat>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    return launch_dependent(zl_cached_chunk_kernel<D, kFormat>, grid, kFormat == ZL_CACHE_BF16 ? 384 : 512, smem, stream, true, tq, tk, tv, p);
}

}  // namespace

size_t cached_chunk_part_bytes(int head_dim) {
    return 4 * sizeof(float) * (head_dim == 128 ? kPartTileFloats<128> : kPartTileFloats<64>);
}
size_t cached_chunk_cut_bytes() { return sizeof(Item); }

cudaError_t launch_cached_join(int head_dim, const CachedParams& p, int ctas, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas, 2 * kTileQ / kJoinRows);
    cfg.blockDim = dim3(kJoinThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, head_dim == 128 ? zl_cached_join_kernel<128> : zl_cached_join_kernel<64>, p);
}

cudaError_t launch_cached_chunk(int head_dim, int format, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv,
                                const CachedParams& p, int grid, cudaStream_t stream) {
    if (head_dim == 128) {
        if (format == ZL_CACHE_BF16) return launch_t<128, ZL_CACHE_BF16>(tq, tk, tv, p, grid, stream);
        return format == ZL_CACHE_INT8 ? launch_t<128, ZL_CACHE_INT8>(tq, tk, tv, p, grid, stream) : launch_t<128, ZL_CACHE_E4M3>(tq, tk, tv, p, grid, stream);
    }
    if (format == ZL_CACHE_BF16) return launch_t<64, ZL_CACHE_BF16>(tq, tk, tv, p, grid, stream);
    return format == ZL_CACHE_INT8 ? launch_t<64, ZL_CACHE_INT8>(tq, tk, tv, p, grid, stream) : launch_t<64, ZL_CACHE_E4M3>(tq, tk, tv, p, grid, stream);
}

}  // namespace zl
