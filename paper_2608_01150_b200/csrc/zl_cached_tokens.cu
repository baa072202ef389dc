// Attention of single new tokens, or a few, over the paged cache (sm_100a): O = softmax(scale q K^T) V and its log-sum-exp for
// the rows (token, query head of the group) of a sequence that share a key head.
//
// Bound by the keys and values, each of which is used for a handful of rows: at 6.4 TB/s an SM has 16 keys of 128 bf16
// columns every 185 clocks and needs some 50 KB in flight.  So
//   * one CTA per SM; all CTAs together walk one line of work, item after item (sequence, block of rows, key head), in tiles
//     of some hundred keys, and each takes an equal stretch of it, wherever that cuts an item.  The lengths are read from
//     device memory when the kernel runs: a captured call follows them, and nothing is planned on the host;
//   * a warp is a stream of its own: it fetches 16 keys and values at a time into its private ring (16-byte asynchronous
//     copies, page by page), across the items of the stretch without a pause, and keeps its own running maximum, sum and
//     accumulator, without a barrier in the loop;
//   * products are mma.sync m16n8k16 with keys (S^T = K Q^T) and value columns (O^T = V^T P^T) as the 16 and eight query rows
//     as the 8: half the instructions, registers and exponentials of the other way round where a sequence has at most eight
//     rows; up to 16 rows take two such columns of tiles.  Products of so few rows are far from the tensor cores' rate with either kind
//     of instruction, and registers spare the way of S and P through tensor memory (about 2,000 clocks a tile for one row);
//   * codes of 8 bits become fp16 exactly, in registers (the integer pipe's half rate bounds that; bf16 took three times the
//     instructions); the scale of a key multiplies its score and the scale of a value its weight, both in fp32.  Columns are
//     summed, and come out, in the order in which ldmatrix gives 8-bit codes.  Twice the warps share that work;
//   * the warps of a CTA join at the end of a stretch of an item; an item that lies in several CTAs is joined by the one that
//     finishes last, in the order of the CTAs, so that results do not depend on which that is.
#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr int kKeys = 16;        // keys of a warp's step
constexpr float kRescale = 8.f;  // powers of two by which a score may exceed the reference before sums are rescaled
constexpr float kLn2 = 0.6931471805599453f;

// kCols: columns of eight query rows.
template <int D, int kFormat, int kCols>
struct TokenSmem {
    static constexpr bool kCodes = kFormat != ZL_CACHE_BF16;
    static constexpr int kWarps = kCodes && kCols == 1 ? 16 : 8;
    static constexpr int kRowBytes = D * (kCodes ? 1 : 2);
    static constexpr int kMatrixBytes = kKeys * kRowBytes;  // 16 keys or 16 values
    static constexpr int kStageBytes = 2 * kMatrixBytes + (kCodes ? 2 * kKeys * 4 : 0);
    static constexpr int kStages = !kCodes ? (D == 128 ? 3 : 6) : (D == 128 ? (kWarps == 16 ? 3 : 6) : (kWarps == 16 ? 6 : 8));
    // At the end of an item a warp leaves eight rows of its accumulator in the stage it has just read (the others hold the next
    // item's keys already); rows are D + 4 floats apart, so that the lanes of a store meet all banks.
    static constexpr int kPitch = D + 4;
    static_assert(kStageBytes >= 8 * kPitch * 4, "eight rows of a warp's accumulator fit a stage");
    alignas(1024) uint8_t ring[kWarps][kStages][kStageBytes];
    float m[kWarps][8], l[kWarps][8];
    uint32_t mask[kWarps][kStages];  // keys of a stage that exist
    int64_t scan[kWarps];
    int64_t start_base;
    int32_t start_seq, ticket;
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
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// c += a b: 16 rows x 8 columns, 16 deep
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma16h(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a 16-row matrix: chunks are exchanged within lines of 128 bytes so that
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
        if (p.split && blocks > 1) blocks = 0;  // the other kernel's
        items = blocks * p.c.n_kv_heads;
        tiles = v.q_len > 0 ? (keys_seen(v, v.q_len - 1) + kTile - 1) / kTile : 0;
    }
    __device__ __forceinline__ int64_t units() const { return (int64_t)items * (tiles + 1); }
};

// The parts of items in a stretch [at, end) of the line.
template <int kTile, int kRows>
struct Walk {
    int64_t base, at, end, item0;  // item0: unit 0 of the item
    int32_t s, head, row0, tile0, tile1;
    SeqView sv;
    SeqWork<kTile, kRows> sw;
    __device__ __forceinline__ Walk(const CachedParams& p, int32_t s_, int64_t base_, int64_t begin, int64_t end_)
        : base(base_), at(begin), end(end_), item0(0), s(s_), head(0), row0(0), tile0(0), tile1(0), sv(load_seq(p.b, p.c.page_shift, s_)),
          sw(p, sv) {}
    __device__ __forceinline__ bool next(const CachedParams& p) {
        while (at < end) {
            while (at >= base + sw.units()) {
                base += sw.units();
                ++s;
                sv = load_seq(p.b, p.c.page_shift, s);
                sw = SeqWork<kTile, kRows>(p, sv);
            }
            const int32_t cost = sw.tiles + 1, item = (int32_t)((at - base) / cost);
            item0 = base + (int64_t)item * cost;
            const int64_t stop = min(end, item0 + cost);
            tile0 = (int32_t)max((int64_t)0, at - item0 - 1);
            tile1 = (int32_t)(stop - item0 - 1);
            const bool starts_here = at == item0;
            at = stop;
            if (tile1 <= tile0 && !(sw.tiles == 0 && starts_here)) continue;  // only the start of an item whose tiles lie in later CTAs
            head = item % p.c.n_kv_heads;
            row0 = (item / p.c.n_kv_heads) * kRows;
            return true;
        }
        return false;
    }
    __device__ __forceinline__ int32_t rows(const CachedParams& p) const {
        return (int32_t)min((int64_t)kRows, (int64_t)sv.q_len * p.group - row0);
    }
};

template <int D, int kFormat, int kCols>
__global__ void __launch_bounds__(TokenSmem<D, kFormat, kCols>::kWarps * 32, 1)
zl_cached_tokens_kernel(const CachedParams p) {
    using Smem = TokenSmem<D, kFormat, kCols>;
    constexpr bool kCodes = Smem::kCodes;
    constexpr int kRowBytes = Smem::kRowBytes, kMatrixBytes = Smem::kMatrixBytes, kStages = Smem::kStages, kWarps = Smem::kWarps;
    constexpr int kThreads = kWarps * 32, kTile = kKeys * kWarps, kRows = 8 * kCols;
    using W = Walk<kTile, kRows>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, quad = lane & 3;
    grid_release();
    grid_wait();

    // ---- this CTA's stretch [begin, end) of the line, and the sequence that `begin` lies in
    int64_t begin, end, per;
    {
        const int chunk = (p.b.n_seqs + kThreads - 1) / kThreads;
        const int s_end = min((tid + 1) * chunk, p.b.n_seqs);
        int64_t mine = 0;
        for (int s = tid * chunk; s < s_end; ++s) mine += SeqWork<kTile, kRows>(p, load_seq(p.b, p.c.page_shift, s)).units();
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
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sm.scan[w];
            total += sm.scan[w];
        }
        per = (total + gridDim.x - 1) / gridDim.x;
        begin = per * blockIdx.x;
        end = min(begin + per, total);
        if (begin >= end) return;
        int64_t at = before + upto - mine;
        if (at <= begin && begin < at + mine) {  // one thread
            int s = tid * chunk;
            while (true) {
                const int64_t n = SeqWork<kTile, kRows>(p, load_seq(p.b, p.c.page_shift, s)).units();
                if (begin < at + n) break;
                at += n;
                ++s;
            }
            sm.start_seq = s;
            sm.start_base = at;
        }
        __syncthreads();
    }

    // ---- the stream of steps: this warp's 16 keys of every tile of every item, kStages - 1 steps ahead of their use
    const uint32_t ring = smem_u32(sm.ring[warp]);
    W ahead(p, sm.start_seq, sm.start_base, begin, end);
    int32_t f_tile = 0, f_keys = 0;  // the next step's tile; keys that the item's last row sees
    uint32_t f_stage = 0;
    // Offsets within a matrix: of this lane's piece of the rows it copies (rows 8 apart are alike), and of its row of ldmatrix,
    // whose chunks c, c + 2, ... are an exclusive or away.
    constexpr int kChunks = kRowBytes / 16, kRowsAtOnce = 32 / kChunks;
    uint32_t f_to[kRowsAtOnce < 8 ? 8 / kRowsAtOnce : 1];
#pragma unroll
    for (int i = 0; i < (kRowsAtOnce < 8 ? 8 / kRowsAtOnce : 1); ++i)
        f_to[i] = swizzled<kRowBytes>(i * kRowsAtOnce + lane / kChunks, lane % kChunks) - i * kRowsAtOnce * kRowBytes;
    const uint32_t k_at = swizzled<kRowBytes>(lane & 15, lane >> 4);
    const uint32_t v_at = kCodes ? k_at : swizzled<kRowBytes>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1);
    auto fetch = [&]() {
        while (f_tile >= ahead.tile1) {
            if (!ahead.next(p)) {
                f_tile = ahead.tile1 = INT32_MAX;  // (never reached by a step)
                break;
            }
            f_tile = ahead.tile0;
            f_keys = keys_seen(ahead.sv, (ahead.row0 + ahead.rows(p) - 1) / p.group);
        }
        if (f_tile != INT32_MAX) {
            const int32_t key0 = f_tile * kTile + warp * kKeys;
            const uint32_t dst = ring + f_stage * Smem::kStageBytes;
            const int32_t key = key0 + (lane & 15);
            const int32_t pg = key < f_keys ? page_at(p.b, p.c, ahead.s, key) : -1;
            const uint32_t exists = __ballot_sync(0xffffffffu, pg >= 0);
            if (lane == 0) sm.mask[warp][f_stage] = exists & 0xffffu;
            // every lane works out its key's place; the copies of a row take it from there
            const int32_t in = key & ((1 << p.c.page_shift) - 1);
            const int64_t place = pg >= 0 ? pg * p.c.page_stride + in * p.c.token_stride + ahead.head * p.c.head_stride : -1;
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
                const int64_t off = live ? (((int64_t)pg << p.c.page_shift) + in) * p.c.n_kv_heads + ahead.head : 0;
                cp4(dst + 2 * kMatrixBytes + lane * 4, (lane < 16 ? p.c.k_scale : p.c.v_scale) + off, live);
            }
            ++f_tile;
        }
        cp_commit();
        f_stage = f_stage + 1 == kStages ? 0 : f_stage + 1;
    };
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) fetch();

    W w(p, sm.start_seq, sm.start_base, begin, end);
    uint32_t st = 0;  // stage of the next step
    while (w.next(p)) {
        const int32_t rows = w.rows(p);
        const SeqView sv = w.sv;
        // ---- queries of the item as B operands (row gid of every column), and the keys that rows 2 quad, 2 quad + 1 see
        uint32_t q[kCols][D / 16][2];
        float by_row[kCols][2];  // 8-bit caches: what multiplies a score beside the key's scale
        int32_t seen[kCols][2], all_see = INT32_MAX;
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
            const bool ok = 8 * n + gid < rows;
            const int32_t r = w.row0 + (ok ? 8 * n + gid : 0), i = r / p.group;
            const __nv_bfloat16* src = p.q + (int64_t)(sv.q0 + i) * p.q_stride + (int64_t)(w.head * p.group + r - i * p.group) * D;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint2 x = make_uint2(0, 0);
                if (ok) {
                    if constexpr (kCodes) {
                        x = __ldg(reinterpret_cast<const uint2*>(src + ks * 16 + quad * 4));
                    } else {
                        x.x = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 16 + quad * 2));
                        x.y = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + quad * 2));
                    }
                }
                q[n][ks][0] = x.x;
                q[n][ks][1] = x.y;
            }
            if constexpr (kCodes) {  // to fp16, and the factor that undoes its scale, for the lane's columns of S^T
                float big = 0.f, back;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    const uint32_t x = q[n][i >> 1][i & 1];
                    big = max3_abs(big, __uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
                }
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const float factor = half_factor(big, back);
#pragma unroll
                for (int i = 0; i < D / 8; ++i) q[n][i >> 1][i & 1] = bf16_pair_to_half(q[n][i >> 1][i & 1], factor);
#pragma unroll
                for (int e = 0; e < 2; ++e) by_row[n][e] = __shfl_sync(0xffffffffu, back, (2 * quad + e) * 4) * p.scale_log2;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t row = 8 * n + 2 * quad + e;
                seen[n][e] = row < rows ? keys_seen(sv, (w.row0 + row) / p.group) : 0;
                if (row < rows) all_see = min(all_see, seen[n][e]);
            }
        }
        all_see = __reduce_min_sync(0xffffffffu, all_see);

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
        for (int32_t tile = w.tile0; tile < w.tile1; ++tile) {
            cp_wait<kStages - 2>();
            __syncwarp();
            fetch();  // into the stage of the step before this one
            const uint32_t k_addr = ring + st * Smem::kStageBytes + k_at, v_addr = ring + st * Smem::kStageBytes + kMatrixBytes + v_at;
            // ---- S^T: keys gid and gid + 8, rows 2 quad and 2 quad + 1
            float c[kCols][4];
#pragma unroll
            for (int n = 0; n < kCols; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
            if constexpr (kCodes) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ks += 2) {
                    uint32_t r[4];  // keys 0-7 and 8-15 of chunk ks, the same of chunk ks + 1
                    ldm4(r, k_addr ^ (ks << 4));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t a0, a1, a2, a3;
                        halves<kFormat>(r[2 * e], a0, a2);
                        halves<kFormat>(r[2 * e + 1], a1, a3);
#pragma unroll
                        for (int n = 0; n < kCols; ++n) mma16h(c[n], a0, a1, a2, a3, q[n][ks + e][0], q[n][ks + e][1]);
                    }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t r[4];  // keys 0-7 and 8-15 of chunk 2 ks, the same of chunk 2 ks + 1
                    ldm4(r, k_addr ^ (ks << 5));
#pragma unroll
                    for (int n = 0; n < kCols; ++n) mma16(c[n], r[0], r[1], r[2], r[3], q[n][ks][0], q[n][ks][1]);
                }
            }
            const int32_t key0 = tile * kTile + warp * kKeys;
            const uint32_t exists = sm.mask[warp][st];
            float key_scale[2], value_scale[2], value_log2[2];
            if constexpr (kCodes) {
                const float* sc = reinterpret_cast<const float*>(sm.ring[warp][st] + 2 * kMatrixBytes);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    key_scale[h] = sc[8 * h + gid];
                    value_scale[h] = fmaxf(sc[kKeys + 8 * h + gid], kLeastScale);
                    value_log2[h] = __log2f(value_scale[h]);
                }
            }
            const bool cut = key0 + kKeys > all_see || exists != 0xffffu;
            uint32_t b[kCols][2];
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) c[n][i] *= kCodes ? by_row[n][i & 1] * key_scale[i >> 1] : p.scale_log2;
                if (cut) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int col = gid + 8 * (i >> 1);
                        if (key0 + col >= seen[n][i & 1] || !((exists >> col) & 1)) c[n][i] = -INFINITY;
                    }
                }
                float mx[2];  // what the reference has to follow: scores, or weights of 8-bit values
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    mx[e] = kCodes ? fmaxf(c[n][e] + value_log2[0], c[n][2 + e] + value_log2[1]) : fmaxf(c[n][e], c[n][2 + e]);
                if (__any_sync(0xffffffffu, mx[0] > m[n][0] + kRescale || mx[1] > m[n][1] + kRescale)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], d));
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
                for (int h = 0; h < 2; ++h) {
                    const float x = ex2(c[n][2 * h] - ref[0]), y = ex2(c[n][2 * h + 1] - ref[1]);
                    l[n][0] += x;
                    l[n][1] += y;
                    b[n][h] = transposed(kCodes ? pack_half(x * value_scale[h], y * value_scale[h]) : pack_bf16(x, y));
                }
            }
            // ---- O^T += V^T P^T
            if constexpr (kCodes) {
#pragma unroll
                for (int ch = 0; ch < D / 16; ch += 2) {
                    uint32_t r[4];  // keys 0-7 and 8-15 of chunk ch, the same of chunk ch + 1
                    ldm4t(r, v_addr ^ (ch << 4));
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // even columns of the chunk as rows 0-7, odd ones as rows 8-15
                        uint32_t a0, a1, a2, a3;
                        halves_apart<kFormat>(r[2 * e], a0, a1);
                        halves_apart<kFormat>(r[2 * e + 1], a2, a3);
#pragma unroll
                        for (int n = 0; n < kCols; ++n) mma16h(o[n][ch + e], a0, a1, a2, a3, b[n][0], b[n][1]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    uint32_t r[4];  // keys 0-7 of chunks 2 i and 2 i + 1, keys 8-15 of the same
                    ldm4t(r, v_addr ^ (i << 5));
#pragma unroll
                    for (int n = 0; n < kCols; ++n) mma16(o[n][i], r[0], r[1], r[2], r[3], b[n][0], b[n][1]);
                }
            }
            st = st + 1 == kStages ? 0 : st + 1;
        }

        // ---- the warps' results side by side: O = sum_w 2^(m_w - max) O_w and the same of the sums
        const uint32_t last = st == 0 ? kStages - 1 : st - 1;  // the stage that was read last, free until the next step
        int32_t c_first = 0, c_last = 0;
        if (w.sw.tiles > 0) {
            c_first = (int32_t)((w.item0 + 1) / per);
            c_last = (int32_t)((w.item0 + w.sw.tiles) / per);
        }
        const bool whole = c_first == c_last;
        auto finish = [&](int r, int c4, float mm, float ll, const float4& acc) {
            const int32_t i = (w.row0 + r) / p.group, h = w.head * p.group + (w.row0 + r) - i * p.group;
            const float inv = ll > 0.f ? 1.f / ll : 0.f;
            uint2 x;
            x.x = pack_bf16(acc.x * inv, acc.y * inv);
            x.y = pack_bf16(acc.z * inv, acc.w * inv);
            const int64_t row = sv.q0 + i;
            *reinterpret_cast<uint2*>(p.o + (row * p.n_heads + h) * D + c4 * 4) = x;
            if (c4 == 0 && p.lse) p.lse[(int64_t)h * p.b.total_q + row] = ll > 0.f ? (mm + log2f(ll)) * kLn2 : -INFINITY;
        };
        auto part_of = [&](int cta) {  // the item's part that CTA `cta` wrote
            return p.part + ((int64_t)cta * 2 + (w.item0 + 1 > cta * per ? 1 : 0)) * kPartFloats<D>;
        };
        if (w.sw.tiles == 0) {  // nobody sees a key
            for (int j = tid; j < rows * (D / 4); j += kThreads) finish(j / (D / 4), j % (D / 4), -INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f));
            continue;
        }
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
            if (8 * n >= rows) break;
            float* mine = reinterpret_cast<float*>(sm.ring[warp][last]);
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                if (gid == 0) {
                    sm.m[warp][2 * quad + e] = m[n][e];
                    sm.l[warp][2 * quad + e] = l[n][e];
                }
                float* to = mine + (2 * quad + e) * Smem::kPitch;
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
            __syncthreads();
            for (int j = tid; j < min(8, rows - 8 * n) * (D / 4); j += kThreads) {
                const int r = j / (D / 4), c4 = j % (D / 4);
                float mm = -INFINITY, ll = 0.f;
#pragma unroll
                for (int v = 0; v < kWarps; ++v) mm = fmaxf(mm, sm.m[v][r]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                if (mm > -INFINITY) {
#pragma unroll
                    for (int v = 0; v < kWarps; ++v) {
                        const float f = ex2(sm.m[v][r] - mm);
                        const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(sm.ring[v][last]) + r * Smem::kPitch + c4 * 4);
                        ll = fmaf(f, sm.l[v][r], ll);
                        acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                    }
                }
                if (whole) {
                    finish(8 * n + r, c4, mm, ll, acc);
                } else {
                    float* to = part_of(blockIdx.x);
                    if (c4 == 0) {
                        to[8 * n + r] = mm;
                        to[kTokenRows + 8 * n + r] = ll;
                    }
                    *reinterpret_cast<float4*>(to + 2 * kTokenRows + (8 * n + r) * D + c4 * 4) = acc;
                }
            }
            if (!whole) __threadfence();
            __syncthreads();  // the stages are free again
        }
        if (!whole) {
            if (tid == 0) sm.ticket = atomicAdd(p.part_count + c_first, 1);
            __syncthreads();
            if (sm.ticket == c_last - c_first) {
                __threadfence();
                for (int j = tid; j < rows * (D / 4); j += kThreads) {
                    const int r = j / (D / 4), c4 = j % (D / 4);
                    float mm = -INFINITY, ll = 0.f;
                    for (int v = c_first; v <= c_last; ++v) mm = fmaxf(mm, __ldcg(part_of(v) + r));
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (mm > -INFINITY) {
#pragma unroll 4
                        for (int v = c_first; v <= c_last; ++v) {
                            const float* from = part_of(v);
                            const float f = ex2(__ldcg(from + r) - mm);
                            const float4 x = __ldcg(reinterpret_cast<const float4*>(from + 2 * kTokenRows + r * D + c4 * 4));
                            ll = fmaf(f, __ldcg(from + kTokenRows + r), ll);
                            acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                        }
                    }
                    finish(r, c4, mm, ll, acc);
                }
                if (tid == 0) p.part_count[c_first] = 0;  // for the next launch
            }
            __syncthreads();  // (the ticket's place is free again)
        }
    }
    cp_wait<0>();
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
    return launch_dependent(zl_cached_tokens_kernel<D, kFormat, kCols>, grid, Smem::kWarps * 32, smem, stream, true, p);
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
