// Attention of single new tokens, or a few, over the paged cache (sm_100a): O = softmax(scale q K^T) V and its log-sum-exp for
// the rows (token, query head of the group) of a sequence that share a key head.
//
// Bound by the keys and values, each of which is used for a handful of rows: at 6.4 TB/s an SM has 16 keys of 128 bf16
// columns every 185 clocks and needs some 50 KB in flight, all the time.  So
//   * one CTA per SM; all CTAs together walk one line of work, item after item (sequence, block of rows, key head), in tiles
//     of some hundred keys, and each takes an equal stretch of it, wherever that cuts an item.  The lengths are read from
//     device memory when the kernel runs: a captured call follows them, and nothing is planned on the host;
//   * a streaming warp fetches 16 keys and values (32 of 8 bits) at a time into its private ring (16-byte asynchronous copies, page by page)
//     and keeps its own running maximum, sum and accumulator: no barrier in the loop, and no pause between items;
//   * four helper warps do what items need beside that: they walk the line ahead of the stream, prepare an item's queries, and
//     join the streaming warps' results from shared memory while those are in the next item already.  (Done by all warps
//     between items, that took some 12,000 clocks an item, a quarter of the time of 64 sequences of up to 8192 8-bit keys.)
//   * products are mma.sync m16n8k16 with keys (S^T = K Q^T) and value columns (O^T = V^T P^T) as the 16 and eight query rows
//     as the 8: half the instructions, registers and exponentials of the other way round where a sequence has at most eight
//     rows; up to 16 rows take two such columns of tiles.  Products of so few rows are far from the tensor cores' rate with either kind
//     of instruction, and registers spare the way of S and P through tensor memory (about 2,000 clocks a tile for one row);
//   * codes of 8 bits become fp16 exactly, in registers (bf16 took three times the instructions); the scale of a key multiplies
//     its score and the scale of a value its weight, both in fp32.  Columns are summed, and come out, in the order in which
//     ldmatrix gives 8-bit codes;
//   * an item that lies in several CTAs is joined by the one that finishes last, in the order of the CTAs, so that results do
//     not depend on which that is.
// Measured, d 128: one token each of 64 sequences of up to 8192 keys, 40 query heads over 8: bf16 160 us (6.3 TB/s of 6.4), e4m3
// 103 (5.1; 112 in a run of seconds, whose clocks fall); one token over 75,600 int8 keys, 12 heads: 48 to 51 us (4.7 to 5.0 TB/s).
// With 8-bit codes the warps' own chains bound it (conversion, products, softmax; 1.5 of 4 instructions a clock with 14 warps,
// whose registers and rings fill the SM; nothing is above 55 %).
#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr int kJoin = 32;        // parts that are joined at a time
constexpr int kHelpers = 4;      // warps that do not stream
// Least units of a CTA's stretch, where items are that long: cutting an item costs its parts' way through memory, some
// 6,000 clocks, as much as six of its steps.
constexpr int64_t kLeastUnits = 6;
constexpr uint64_t kWaitLimitNs = 4000000000ull;
constexpr float kRescale = 8.f;  // powers of two by which a score may exceed the reference before sums are rescaled
constexpr float kLn2 = 0.6931471805599453f;

// A CTA's part of an item, as the helpers hand it to the streaming warps.
struct alignas(16) Item {
    int32_t s, head, tile0, tile1;      // sequence, key head, tiles of this part (tile1 < 0: no more items)
    int32_t keys, all_see, rows, row0;  // keys that any row sees, that all rows see; rows of the item, the first of them
    int32_t q0, c_first, c_last, place_first;  // first token row; the CTAs that have parts, and where the first of them keeps its own
};

// kCols: columns of eight query rows.
template <int D, int kFormat, int kCols>
struct TokenSmem {
    static constexpr bool kCodes = kFormat != ZL_CACHE_BF16;
    static constexpr int kRows = 8 * kCols;
    static constexpr int kWarps = kCodes ? (kCols == 1 ? (D == 128 ? 10 : 12) : 8) : (D == 64 ? (kCols == 1 ? 11 : 8) : (kCols == 1 ? 7 : 6));  // that stream
    static constexpr int kKeys = kCodes && kCols == 1 ? 32 : 16;  // of a warp's step: as many as amortise what a step costs beside them
    static constexpr int kRowBytes = D * (kCodes ? 1 : 2);
    static constexpr int kMatrixBytes = kKeys * kRowBytes;  // the keys or the values of a step
    static constexpr int kStageBytes = 2 * kMatrixBytes + (kCodes ? 2 * kKeys * 4 : 0);
    static constexpr int kStages = D == 128 ? (kKeys == 32 ? 2 : 3) : (kKeys == 32 ? 3 : (kCodes ? 6 : 4));
    // An item has a step at least, and a warp's copies are at most kStages - 1 steps ahead: with an item more than that
    // prepared, no warp waits for one that the helpers can only prepare after it has moved on.
    static constexpr int kItems = kStages + 1;
    static constexpr int kPitch = D + 4;    // floats between rows of an accumulator: the lanes of a store meet all banks
    static constexpr int kQPitch = D + 16;  // elements between rows of the queries, for the same reason
    alignas(1024) uint8_t ring[kWarps][kStages][kStageBytes];
    alignas(16) float o[kWarps][kRows][kPitch];  // the streaming warps' results of an item
    float m[kWarps][kRows], l[kWarps][kRows];
    uint32_t mask[kWarps][kStages];  // keys of a stage that exist
    Item items[kItems];
    alignas(16) uint16_t q[kItems][kRows][kQPitch];  // bf16; 8-bit caches: fp16
    float q_back[kItems][kRows];     // 8-bit caches: what scores have to be multiplied by beside the key's scale
    int32_t seen[kItems][kRows];     // keys that a row sees
    alignas(8) uint64_t item_full[kItems], q_full[kItems], item_done[kItems], o_free, helpers;
    int64_t scan[kWarps + kHelpers];
    int32_t longest[kWarps + kHelpers];
    float join_w[kJoin][kRows];      // weights and sums of parts that are joined
    float4 join_o[kHelpers * 32];
    float join_l[kHelpers * 32];
    int64_t start_base;
    int32_t start_seq, ticket;
    volatile int32_t abort_flag;
};

// A CTA's partial result of an item: maxima (powers of two) and sums of the rows, then their unnormalised outputs.
template <int D>
constexpr int kPartFloats = kTokenRows * (D + 2);

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {  // zeros if not live
    const int n = live ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool live) {
    const int n = live ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// An 8x8 matrix of 16-bit numbers, one row pair per lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// c += a b: 16 rows x 8 columns, 16 deep
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma16h(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a matrix: chunks are exchanged within lines of 128 bytes so that
// the eight rows of an 8x8 matrix lie on different banks.
template <int kRowBytes>
__device__ __forceinline__ uint32_t swizzled(int row, int chunk) {
    return row * kRowBytes + ((chunk ^ (kRowBytes == 64 ? (row >> 1) & 3 : row & 7)) << 4);
}

// The line of work: every sequence is `items` items of tiles + 1 units; unit 0 of an item stands for its start and end.
template <int kTile, int kRows>
struct SeqWork {
    int32_t items, tiles;
    __device__ __forceinline__ SeqWork(const CachedParams& p, const SeqView& v) {
        int32_t blocks = (int32_t)(((int64_t)v.q_len * p.group + kRows - 1) / kRows);
        if (p.split && (int64_t)v.q_len * p.group > kTokenRows) blocks = 0;  // the other kernel's
        items = blocks * p.c.n_kv_heads;
        tiles = v.q_len > 0 ? (keys_seen(v, v.q_len - 1) + kTile - 1) / kTile : 0;
    }
    __device__ __forceinline__ int64_t units() const { return (int64_t)items * (tiles + 1); }
};

__device__ __forceinline__ void report(int32_t* status, volatile int32_t* abort_flag, int where) {
    *abort_flag = 1;
    if (atomicCAS(status, 0, (int)ZL_ERR_TIMEOUT) == 0) status[1] = where;
}
static __device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, const volatile int32_t* abort_flag) {
    return mbar_wait_slow(bar, parity, kWaitLimitNs, abort_flag);
}
// All lanes of a warp wait; the outcome is warp-uniform and the warp reconverges.
#define ZL_WAIT_WARP(bar, parity, site)                                                                  \
    do {                                                                                                 \
        const bool ok_ = mbar_try_wait((bar), (parity)) || wait_slow((bar), (parity), &sm.abort_flag); \
        if (!__all_sync(0xffffffffu, ok_)) {                                                             \
            report(p.status, &sm.abort_flag, 8000 + (site));                                            \
            goto teardown;                                                                               \
        }                                                                                                \
    } while (0)

template <int D, int kFormat, int kCols>
__global__ void __launch_bounds__((TokenSmem<D, kFormat, kCols>::kWarps + kHelpers) * 32, 1)
zl_cached_tokens_kernel(const CachedParams p) {
    using Smem = TokenSmem<D, kFormat, kCols>;
    constexpr bool kCodes = Smem::kCodes;
    constexpr int kRowBytes = Smem::kRowBytes, kMatrixBytes = Smem::kMatrixBytes, kStages = Smem::kStages, kWarps = Smem::kWarps;
    constexpr int kThreads = (kWarps + kHelpers) * 32, kKeys = Smem::kKeys, kTile = kKeys * kWarps, kRows = Smem::kRows, kItems = Smem::kItems;
    using Work = SeqWork<kTile, kRows>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, quad = lane & 3;
    if (tid == 0) {
        for (int i = 0; i < kItems; ++i) {
            mbar_init(&sm.item_full[i], 1);
            mbar_init(&sm.q_full[i], kHelpers * 32);
            mbar_init(&sm.item_done[i], kWarps);
        }
        mbar_init(&sm.o_free, kHelpers * 32);
        mbar_init(&sm.helpers, kHelpers * 32);
        sm.abort_flag = 0;
        fence_mbar_init();
    }
    grid_release();
    // Behind the chunk kernel, whose CTAs release this grid when all that came before them has completed, it begins on SMs that have
    // no more chunks: neither reads what the other writes.  It waits at its end instead, so that its own end means that of both.
    const bool behind = p.split != 0;
    if (!behind) grid_wait();

    // ---- this CTA's stretch [begin, end) of the line, and the sequence that `begin` lies in
    int64_t begin, end, per;
    {
        const int chunk = (p.b.n_seqs + kThreads - 1) / kThreads;
        const int s_end = min((tid + 1) * chunk, p.b.n_seqs);
        int64_t mine = 0;
        int32_t longest = 0;
        for (int s = tid * chunk; s < s_end; ++s) {
            const Work x(p, load_seq(p.b, p.c.page_shift, s));
            mine += x.units();
            if (x.items > 0) longest = max(longest, x.tiles + 1);
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        int64_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) {
            sm.scan[warp] = upto;
            sm.longest[warp] = longest;
        }
        __syncthreads();
        int64_t before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < kWarps + kHelpers; ++w) {
            if (w < warp) before += sm.scan[w];
            total += sm.scan[w];
            longest = max(longest, sm.longest[w]);
        }
        per = max(quotient(total + gridDim.x - 1, gridDim.x), min((int64_t)longest, kLeastUnits));
        begin = per * blockIdx.x;
        end = min(begin + per, total);
        if (begin >= end) {
            if (behind) grid_wait();
            return;
        }
        int64_t at = before + upto - mine;
        if (at <= begin && begin < at + mine) {  // one thread
            int s = tid * chunk;
            while (true) {
                const int64_t n = Work(p, load_seq(p.b, p.c.page_shift, s)).units();
                if (begin < at + n) break;
                at += n;
                ++s;
            }
            sm.start_seq = s;
            sm.start_base = at;
        }
        __syncthreads();
    }

    if (warp >= kWarps) {
        // ------------------------------------------------------------------ helpers
        const int t = tid - kWarps * 32;
        int32_t s = sm.start_seq;
        int64_t base = sm.start_base, at = begin;
        SeqView sv = load_seq(p.b, p.c.page_shift, s);
        Work sw(p, sv);
        auto finish = [&](const Item& w, int r, int c4, float mm, float ll, const float4& acc) {
            const int32_t i = (w.row0 + r) / p.group, h = w.head * p.group + (w.row0 + r) - i * p.group;
            const float inv = ll > 0.f ? 1.f / ll : 0.f;
            uint2 x;
            x.x = pack_bf16(acc.x * inv, acc.y * inv);
            x.y = pack_bf16(acc.z * inv, acc.w * inv);
            const int64_t row = w.q0 + i;
            *reinterpret_cast<uint2*>(p.o + (row * p.n_heads + h) * D + c4 * 4) = x;
            if (c4 == 0 && p.lse) p.lse[(int64_t)h * p.b.total_q + row] = ll > 0.f ? (mm + log2f(ll)) * kLn2 : -INFINITY;
        };
        // The next item with tiles, or the end, into place `it`; items whose rows see no key are written at once.
        auto prepare = [&](uint32_t it) {
            Item w{};
            w.tile1 = -1;
            while (at < end) {
                while (at >= base + sw.units()) {
                    base += sw.units();
                    ++s;
                    sv = load_seq(p.b, p.c.page_shift, s);
                    sw = Work(p, sv);
                }
                const int32_t cost = sw.tiles + 1, item = (int32_t)quotient(at - base, cost);
                const int64_t item0 = base + (int64_t)item * cost, stop = min(end, item0 + cost);  // item0: unit 0 of the item
                const int32_t tile0 = (int32_t)max((int64_t)0, at - item0 - 1), tile1 = (int32_t)(stop - item0 - 1);
                const bool starts_here = at == item0;
                at = stop;
                if (tile1 <= tile0 && !(sw.tiles == 0 && starts_here)) continue;  // only the start of an item whose tiles lie in later CTAs
                const int32_t block = item / p.c.n_kv_heads;
                w.s = s;
                w.head = item - block * p.c.n_kv_heads;
                w.row0 = block * kRows;
                w.rows = (int32_t)min((int64_t)kRows, (int64_t)sv.q_len * p.group - w.row0);
                w.q0 = sv.q0;
                if (sw.tiles == 0) {
                    for (int j = t; j < w.rows * (D / 4); j += kHelpers * 32) finish(w, j / (D / 4), j % (D / 4), -INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f));
                    continue;
                }
                w.tile0 = tile0;
                w.tile1 = tile1;
                w.all_see = keys_seen(sv, w.row0 / p.group);  // (later rows see as many keys or more)
                w.keys = keys_seen(sv, (w.row0 + w.rows - 1) / p.group);
                w.c_first = (int32_t)quotient(item0 + 1, per);
                w.c_last = (int32_t)quotient(item0 + sw.tiles, per);
                w.place_first = item0 + 1 > w.c_first * per ? 1 : 0;
                break;
            }
            const uint32_t place = it % kItems;
            if (t == 0) {
                sm.items[place] = w;
                mbar_arrive(&sm.item_full[place]);
            }
            if (w.tile1 < 0) return false;
            // queries: sixteen threads a row
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
                const int row = 8 * n + (t >> 4), c = t & 15;
                constexpr int kEach = D / 16;  // elements
                const bool ok = row < w.rows;
                const int32_t r = w.row0 + (ok ? row : 0), i = r / p.group;
                const __nv_bfloat16* src = p.q + (int64_t)(sv.q0 + i) * p.q_stride + (int64_t)(w.head * p.group + r - i * p.group) * D + c * kEach;
                uint32_t x[kEach / 2];
#pragma unroll
                for (int e = 0; e < kEach / 2; e += 2) {
                    const uint2 u = ok ? __ldg(reinterpret_cast<const uint2*>(src + 2 * e)) : make_uint2(0, 0);
                    x[e] = u.x;
                    x[e + 1] = u.y;
                }
                if constexpr (kCodes) {
                    float big = 0.f, back;
#pragma unroll
                    for (int e = 0; e < kEach / 2; ++e) big = max3_abs(big, __uint_as_float(x[e] << 16), __uint_as_float(x[e] & 0xffff0000u));
#pragma unroll
                    for (int d = 8; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
                    const float factor = half_factor(big, back);
#pragma unroll
                    for (int e = 0; e < kEach / 2; ++e) x[e] = bf16_pair_to_half(x[e], factor);
                    if (c == 0) sm.q_back[place][row] = back * p.scale_log2;
                }
#pragma unroll
                for (int e = 0; e < kEach / 2; e += 2) *reinterpret_cast<uint2*>(&sm.q[place][row][c * kEach + 2 * e]) = make_uint2(x[e], x[e + 1]);
                if (c == 0) sm.seen[place][row] = ok ? keys_seen(sv, i) : 0;
            }
            mbar_arrive(&sm.q_full[place]);
            return true;
        };
        uint32_t n_items = 0;  // prepared so far
        bool more = true;
        while (more && n_items < kItems - 1) {
            more = prepare(n_items);
            if (more) ++n_items;
        }
        for (uint32_t it = 0; it < n_items; ++it) {
            ZL_WAIT_WARP(&sm.item_done[it % kItems], (it / kItems) & 1, 1);
            // By value: its place is prepared anew behind the next item, whose end is ordered behind this warp's o_free and behind
            // nothing that it does after that, while finish() needs the item to the end of its join.
            const Item w = sm.items[it % kItems];
            // ---- O = sum_w 2^(m_w - max) O_w over the streaming warps, and the same of the sums
            const bool whole = w.c_first == w.c_last;
            auto part_of = [&](int cta) { return p.part + ((int64_t)cta * 2 + (cta == w.c_first ? w.place_first : 0)) * kPartFloats<D>; };
            const int rows = w.rows;
            for (int j = t; j < rows * (D / 4); j += kHelpers * 32) {
                const int r = j / (D / 4), c4 = j % (D / 4);
                float mm = -INFINITY, ll = 0.f;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) mm = fmaxf(mm, sm.m[v][r]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                if (mm > -INFINITY) {
#pragma unroll
                    for (int v = 0; v < kWarps; ++v) {
                        const float f = ex2(sm.m[v][r] - mm);
                        const float4 x = *reinterpret_cast<const float4*>(&sm.o[v][r][c4 * 4]);
                        ll = fmaf(f, sm.l[v][r], ll);
                        acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                    }
                }
                if (whole) {
                    finish(w, r, c4, mm, ll, acc);
                } else {
                    float* to = part_of(blockIdx.x);
                    if (c4 == 0) {
                        to[r] = mm;
                        to[kTokenRows + r] = ll;
                    }
                    *reinterpret_cast<float4*>(to + 2 * kTokenRows + r * D + c4 * 4) = acc;
                }
            }
            mbar_arrive(&sm.o_free);
            if (!whole) {
                __threadfence();
                mbar_arrive(&sm.helpers);
                ZL_WAIT_WARP(&sm.helpers, 0, 2);
                if (t == 0) sm.ticket = atomicAdd(p.part_count + w.c_first, 1);
                mbar_arrive(&sm.helpers);
                ZL_WAIT_WARP(&sm.helpers, 1, 3);
                if (sm.ticket == w.c_last - w.c_first) {
                    __threadfence();
                    // Threads beyond a quadruple of columns each take every `groups`th part; weights are worked out once per part and
                    // row, kJoin parts at a time.  (An even number of barrier phases each time.)
                    const int quads = rows * (D / 4), parts = w.c_last - w.c_first + 1;
                    const int groups = quads >= kHelpers * 32 ? 1 : kHelpers * 32 / quads;
                    for (int j0 = 0; j0 < quads; j0 += kHelpers * 32) {
                        const int j = j0 + (groups > 1 ? t % quads : t), group = groups > 1 ? t / quads : 0;
                        const bool mine = j < quads && group < groups;
                        const int r = mine ? j / (D / 4) : 0, c4 = j % (D / 4);
                        float mm = -INFINITY, ll = 0.f;
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                        for (int p0 = 0; p0 < parts; p0 += kJoin) {
                            const int n = min(kJoin, parts - p0);
                            for (int i = t; i < n * rows; i += kHelpers * 32) sm.join_w[i / rows][i % rows] = __ldcg(part_of(w.c_first + p0 + i / rows) + i % rows);
                            mbar_arrive(&sm.helpers);
                            ZL_WAIT_WARP(&sm.helpers, 0, 4);
                            float up = mm;
                            for (int v = 0; v < n; ++v) up = fmaxf(up, sm.join_w[v][r]);
                            if (mine && up > -INFINITY) {
                                const float alpha = ex2(mm - up);
                                mm = up;
                                ll *= alpha;
                                acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
#pragma unroll 8
                                for (int v = group; v < n; v += groups) {
                                    const float* from = part_of(w.c_first + p0 + v);
                                    const float4 x = __ldcg(reinterpret_cast<const float4*>(from + 2 * kTokenRows + r * D + c4 * 4));
                                    const float lv = __ldcg(from + kTokenRows + r), f = ex2(sm.join_w[v][r] - mm);
                                    ll = fmaf(f, lv, ll);
                                    acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                                }
                            }
                            mbar_arrive(&sm.helpers);
                            ZL_WAIT_WARP(&sm.helpers, 1, 5);
                        }
                        if (groups > 1) {  // (all groups have the same maximum)
                            sm.join_o[t] = acc;
                            sm.join_l[t] = ll;
                            mbar_arrive(&sm.helpers);
                            ZL_WAIT_WARP(&sm.helpers, 0, 6);
                            if (mine && group == 0)
                                for (int g = 1; g < groups; ++g) {
                                    const float4 x = sm.join_o[g * quads + j];
                                    ll += sm.join_l[g * quads + j];
                                    acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
                                }
                            mbar_arrive(&sm.helpers);
                            ZL_WAIT_WARP(&sm.helpers, 1, 7);
                        }
                        if (mine && group == 0) finish(w, r, c4, mm, ll, acc);
                    }
                    if (t == 0) p.part_count[w.c_first] = 0;  // for the next launch
                }
            }
            if (more) {
                more = prepare(n_items);  // over the place of the item before this one
                if (more) ++n_items;
            }
        }
    } else {
        // ------------------------------------------------------------------ the stream of steps
        const uint32_t ring = smem_u32(sm.ring[warp]);
        // Offsets within a matrix: of this lane's piece of the rows it copies (rows 8 apart are alike), and of its row of ldmatrix,
        // whose chunks c, c + 2, ... are an exclusive or away.
        constexpr int kChunks = kRowBytes / 16, kRowsAtOnce = 32 / kChunks;
        uint32_t f_to[kRowsAtOnce < 8 ? 8 / kRowsAtOnce : 1];
#pragma unroll
        for (int i = 0; i < (kRowsAtOnce < 8 ? 8 / kRowsAtOnce : 1); ++i)
            f_to[i] = swizzled<kRowBytes>(i * kRowsAtOnce + lane / kChunks, lane % kChunks) - i * kRowsAtOnce * kRowBytes;
        const uint32_t k_at = swizzled<kRowBytes>(lane & 15, lane >> 4);
        const uint32_t v_at = kCodes ? k_at : swizzled<kRowBytes>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1);

        // ---- copies: this warp's kKeys keys of every tile of every item, kStages - 1 steps ahead of their use
        uint32_t f_item = 0, f_stage = 0;
        int32_t f_tile = 0, f_end = 0;  // the next step's tile, the item's last; f_end < 0: no more items
        int32_t f_page = -1;            // table entry of this lane's key (key lane % kKeys) of the next step, looked up a step ahead
        // the item's: keys, row of the page table, where its head lies in a token (16 bytes; elements of the scales)
        int32_t f_keys = 0;
        const int32_t* f_pages = nullptr;
        uint64_t f_head = 0, f_scale = 0;
        const int32_t in_page = (1 << p.c.page_shift) - 1;
        bool waited = true;
        auto fetch = [&]() {
            if (f_tile >= f_end && f_end >= 0) {
                const uint32_t place = f_item % kItems;
                const bool ok = mbar_try_wait(&sm.item_full[place], (f_item / kItems) & 1) ||
                                wait_slow(&sm.item_full[place], (f_item / kItems) & 1, &sm.abort_flag);
                waited = __all_sync(0xffffffffu, ok);
                f_tile = sm.items[place].tile0;
                f_end = waited ? sm.items[place].tile1 : -1;
                ++f_item;
                if (f_end >= 0) {
                    const Item& w = sm.items[place];
                    f_keys = w.keys;
                    f_pages = p.b.pages + (int64_t)w.s * p.b.max_pages;
                    f_head = (uint64_t)(uint32_t)w.head * p.c.head16;
                    f_scale = (uint64_t)(uint32_t)w.head * (uint32_t)p.c.scale_head;
                    const int32_t key = f_tile * kTile + warp * kKeys + (lane & (kKeys - 1));
                    f_page = key < f_keys ? __ldg(f_pages + (key >> p.c.page_shift)) : -1;
                }
            }
            if (f_end >= 0) {
                const int32_t key0 = f_tile * kTile + warp * kKeys;
                const uint32_t dst = ring + f_stage * Smem::kStageBytes;
                const int32_t key = key0 + (lane & (kKeys - 1));
                const int32_t pg = valid_page(p.c, f_page);
                const uint32_t exists = __ballot_sync(0xffffffffu, pg >= 0);
                if (++f_tile < f_end) f_page = key + kTile < f_keys ? __ldg(f_pages + ((key + kTile) >> p.c.page_shift)) : -1;
                if (lane == 0) sm.mask[warp][f_stage] = kKeys == 32 ? exists : exists & 0xffffu;
                // every lane works out its key's place; the copies of a row take it from there
                const uint32_t in = key & in_page;
                const uint64_t at16 = (uint64_t)(uint32_t)pg * p.c.page16 + ((uint64_t)in * p.c.token16 + f_head);
                const int64_t place = pg >= 0 ? (int64_t)(at16 << 4) : -1;
#pragma unroll
                for (int i = 0; i < kKeys / kRowsAtOnce; ++i) {
                    const int64_t from = __shfl_sync(0xffffffffu, place, i * kRowsAtOnce + lane / kChunks);
                    const bool live = from >= 0;
                    const uint32_t to = dst + f_to[(i * kRowsAtOnce % 8) / kRowsAtOnce] + i * kRowsAtOnce * kRowBytes;
                    const int64_t off = live ? from + lane % kChunks * 16 : 0;
                    cp16(to, p.c.k + off, live);
                    cp16(to + kMatrixBytes, p.c.v + off, live);
                }
                if constexpr (kCodes) {
                    const bool live = pg >= 0;
                    const uint64_t at = (uint64_t)(uint32_t)pg * (uint32_t)p.c.scale_page + ((uint64_t)in * (uint32_t)p.c.scale_token + f_scale);
                    const uint64_t off = live ? at : 0;
                    if constexpr (kKeys == 32) {
                        cp4(dst + 2 * kMatrixBytes + lane * 4, p.c.k_scale + off, live);
                        cp4(dst + 2 * kMatrixBytes + 128 + lane * 4, p.c.v_scale + off, live);
                    } else {
                        cp4(dst + 2 * kMatrixBytes + lane * 4, (lane < 16 ? p.c.k_scale : p.c.v_scale) + off, live);
                    }
                }
            }
            cp_commit();
            f_stage = f_stage + 1 == kStages ? 0 : f_stage + 1;
        };
#pragma unroll 1
        for (int i = 0; i < kStages - 1; ++i) fetch();

        uint32_t st = 0;  // stage of the next step
        for (uint32_t it = 0;; ++it) {
            const uint32_t place = it % kItems;
            ZL_WAIT_WARP(&sm.item_full[place], (it / kItems) & 1, 11);
            if (!waited) goto teardown;
            const int32_t tile1 = sm.items[place].tile1, all_see = sm.items[place].all_see;
            if (tile1 < 0) break;
            ZL_WAIT_WARP(&sm.q_full[place], (it / kItems) & 1, 12);
            // queries as B operands (row gid of every column); two columns of them are read from shared memory at every step
            uint32_t q[kCols == 1 ? D / 16 : 1][2];
            auto load_q = [&](int n, int ks, uint32_t& q0, uint32_t& q1) {
                const uint16_t* row = sm.q[place][8 * n + gid] + ks * 16;
                if constexpr (kCodes) {
                    const uint2 x = *reinterpret_cast<const uint2*>(row + quad * 4);
                    q0 = x.x;
                    q1 = x.y;
                } else {
                    q0 = *reinterpret_cast<const uint32_t*>(row + quad * 2);
                    q1 = *reinterpret_cast<const uint32_t*>(row + 8 + quad * 2);
                }
            };
            if constexpr (kCols == 1) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) load_q(0, ks, q[ks][0], q[ks][1]);
            }
            float by_row[kCols][2];  // 8-bit caches: what multiplies a score beside the key's scale
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) by_row[n][e] = kCodes ? sm.q_back[place][8 * n + 2 * quad + e] : p.scale_log2;

            float o[kCols][D / 16][4], m[kCols][2], l[kCols][2];
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
                m[n][0] = m[n][1] = -INFINITY;
                l[n][0] = l[n][1] = 0.f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[n][i][j] = 0.f;
            }
#pragma unroll 1
            for (int32_t tile = sm.items[place].tile0; tile < tile1; ++tile) {
                cp_wait<kStages - 2>();
                __syncwarp();
                fetch();  // into the stage of the step before this one
                const uint32_t k_addr = ring + st * Smem::kStageBytes + k_at, v_addr = ring + st * Smem::kStageBytes + kMatrixBytes + v_at;
                // ---- S^T: keys gid and gid + 8 of every sixteen, rows 2 quad and 2 quad + 1
                constexpr int kParts = kKeys / 16;
                float c[kParts][kCols][4];
#pragma unroll
                for (int g = 0; g < kParts; ++g) {
#pragma unroll
                    for (int n = 0; n < kCols; ++n) c[g][n][0] = c[g][n][1] = c[g][n][2] = c[g][n][3] = 0.f;
                    const uint32_t at = k_addr + g * 16 * kRowBytes;
                    if constexpr (kCodes) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ks += 2) {
                            uint32_t r[4];  // keys 0-7 and 8-15 of chunk ks, the same of chunk ks + 1
                            ldm4(r, at ^ (ks << 4));
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                uint32_t a0, a1, a2, a3;
                                halves<kFormat>(r[2 * e], a0, a2);
                                halves<kFormat>(r[2 * e + 1], a1, a3);
#pragma unroll
                                for (int n = 0; n < kCols; ++n) {
                                    uint32_t q0, q1;
                                    if constexpr (kCols == 1) { q0 = q[ks + e][0]; q1 = q[ks + e][1]; } else load_q(n, ks + e, q0, q1);
                                    mma16h(c[g][n], a0, a1, a2, a3, q0, q1);
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            uint32_t r[4];  // keys 0-7 and 8-15 of chunk 2 ks, the same of chunk 2 ks + 1
                            ldm4(r, at ^ (ks << 5));
#pragma unroll
                            for (int n = 0; n < kCols; ++n) {
                                uint32_t q0, q1;
                                if constexpr (kCols == 1) { q0 = q[ks][0]; q1 = q[ks][1]; } else load_q(n, ks, q0, q1);
                                mma16(c[g][n], r[0], r[1], r[2], r[3], q0, q1);
                            }
                        }
                    }
                }
                const int32_t key0 = tile * kTile + warp * kKeys;
                const uint32_t exists = sm.mask[warp][st];
                float key_scale[kParts][2], value_scale[kParts][2], value_log2[kParts][2];
                if constexpr (kCodes) {
                    const float* sc = reinterpret_cast<const float*>(sm.ring[warp][st] + 2 * kMatrixBytes);
#pragma unroll
                    for (int g = 0; g < kParts; ++g)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            key_scale[g][h] = sc[16 * g + 8 * h + gid];
                            value_scale[g][h] = fmaxf(sc[kKeys + 16 * g + 8 * h + gid], kLeastScale);
                            value_log2[g][h] = __log2f(value_scale[g][h]);
                        }
                }
                const bool cut = key0 + kKeys > all_see || exists != (kKeys == 32 ? 0xffffffffu : 0xffffu);
                uint32_t b[kParts][kCols][2];
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    float mx[2] = {-INFINITY, -INFINITY};  // what the reference has to follow: scores, or weights of 8-bit values
#pragma unroll
                    for (int g = 0; g < kParts; ++g) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) c[g][n][i] *= kCodes ? by_row[n][i & 1] * key_scale[g][i >> 1] : p.scale_log2;
                        if (cut) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int col = 16 * g + gid + 8 * (i >> 1);
                                if (key0 + col >= sm.seen[place][8 * n + 2 * quad + (i & 1)] || !((exists >> col) & 1)) c[g][n][i] = -INFINITY;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            mx[e] = kCodes ? max3(mx[e], c[g][n][e] + value_log2[g][0], c[g][n][2 + e] + value_log2[g][1])
                                           : max3(mx[e], c[g][n][e], c[g][n][2 + e]);
                    }
                    if (__any_sync(0xffffffffu, mx[0] > m[n][0] + kRescale || mx[1] > m[n][1] + kRescale)) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
#pragma unroll
                            for (int u = 4; u < 32; u <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], u));
                            const float up = fmaxf(m[n][e], mx[e]);
                            const float alpha = up == -INFINITY ? 1.f : ex2(m[n][e] - up);
                            m[n][e] = up;
                            l[n][e] *= alpha;
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) {
                                o[n][i][e] *= alpha;
                                o[n][i][2 + e] *= alpha;
                            }
                        }
                    }
                    // ---- P, rounded once for its product with V (bf16, or with the value's scale to fp16); the sums take it unrounded
                    const float ref[2] = {m[n][0] == -INFINITY ? 0.f : m[n][0], m[n][1] == -INFINITY ? 0.f : m[n][1]};
#pragma unroll
                    for (int g = 0; g < kParts; ++g)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float x = ex2(c[g][n][2 * h] - ref[0]), y = ex2(c[g][n][2 * h + 1] - ref[1]);
                            l[n][0] += x;
                            l[n][1] += y;
                            b[g][n][h] = transposed(kCodes ? pack_half(x * value_scale[g][h], y * value_scale[g][h]) : pack_bf16(x, y));
                        }
                }
                // ---- O^T += V^T P^T
#pragma unroll
                for (int g = 0; g < kParts; ++g) {
                    const uint32_t at = v_addr + g * 16 * kRowBytes;
                    if constexpr (kCodes) {
#pragma unroll
                        for (int ch = 0; ch < D / 16; ch += 2) {
                            uint32_t r[4];  // keys 0-7 and 8-15 of chunk ch, the same of chunk ch + 1
                            ldm4t(r, at ^ (ch << 4));
#pragma unroll
                            for (int e = 0; e < 2; ++e) {  // even columns of the chunk as rows 0-7, odd ones as rows 8-15
                                uint32_t a0, a1, a2, a3;
                                halves_apart<kFormat>(r[2 * e], a0, a1);
                                halves_apart<kFormat>(r[2 * e + 1], a2, a3);
#pragma unroll
                                for (int n = 0; n < kCols; ++n) mma16h(o[n][ch + e], a0, a1, a2, a3, b[g][n][0], b[g][n][1]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            uint32_t r[4];  // keys 0-7 of chunks 2 i and 2 i + 1, keys 8-15 of the same
                            ldm4t(r, at ^ (i << 5));
#pragma unroll
                            for (int n = 0; n < kCols; ++n) mma16(o[n][i], r[0], r[1], r[2], r[3], b[g][n][0], b[g][n][1]);
                        }
                    }
                }
                st = st + 1 == kStages ? 0 : st + 1;
            }
            // ---- this warp's result, once the helpers have read the one before
            if (it > 0) ZL_WAIT_WARP(&sm.o_free, (it - 1) & 1, 13);
#pragma unroll
            for (int n = 0; n < kCols; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                    const int row = 8 * n + 2 * quad + e;
                    if (gid == 0) {
                        sm.m[warp][row] = m[n][e];
                        sm.l[warp][row] = l[n][e];
                    }
                    float* to = sm.o[warp][row];
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        if constexpr (kCodes) {
                            *reinterpret_cast<float2*>(to + i * 16 + gid * 2) = make_float2(o[n][i][e], o[n][i][2 + e]);
                        } else {
                            to[i * 16 + gid] = o[n][i][e];
                            to[i * 16 + gid + 8] = o[n][i][2 + e];
                        }
                    }
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_done[place]);
        }
    }

teardown:
    cp_wait<0>();
    if (behind) grid_wait();
}

template <int D, int kFormat, int kCols>
cudaError_t launch_t(const CachedParams& p, int grid, cudaStream_t stream) {
    using Smem = TokenSmem<D, kFormat, kCols>;
    constexpr int smem = sizeof(Smem);
    static_assert(smem <= 232448, "shared memory of a CTA");
    constexpr int kMaxDevices = 64;
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_cached_tokens_kernel<D, kFormat, kCols>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    return launch_dependent(zl_cached_tokens_kernel<D, kFormat, kCols>, grid, (Smem::kWarps + kHelpers) * 32, smem, stream, true, p);
}

template <int D, int kCols>
cudaError_t launch_f(int format, const CachedParams& p, int grid, cudaStream_t stream) {
    if (format == ZL_CACHE_BF16) return launch_t<D, ZL_CACHE_BF16, kCols>(p, grid, stream);
    return format == ZL_CACHE_INT8 ? launch_t<D, ZL_CACHE_INT8, kCols>(p, grid, stream) : launch_t<D, ZL_CACHE_E4M3, kCols>(p, grid, stream);
}

}  // namespace

size_t cached_tokens_part_bytes(int head_dim) { return 2 * sizeof(float) * (head_dim == 128 ? kPartFloats<128> : kPartFloats<64>); }

cudaError_t launch_cached_tokens(int head_dim, int format, const CachedParams& p, int grid, cudaStream_t stream) {
    if (p.token_rows <= 8) return head_dim == 128 ? launch_f<128, 1>(format, p, grid, stream) : launch_f<64, 1>(format, p, grid, stream);
    return head_dim == 128 ? launch_f<128, 2>(format, p, grid, stream) : launch_f<64, 2>(format, p, grid, stream);
}

}  // namespace zl
