// Attention of single new tokens, or a few, over the paged cache (sm_100a): O = softmax(scale q K^T) V and its log-sum-exp for
// the rows (token, query head of the group) of a sequence that share a key head.
//
// Bound by the keys and values, each of which is used for a handful of rows: at 6.4 TB/s an SM has 16 keys of 128 bf16
// columns every 185 clocks and needs some 50 KB in flight.  So
//   * one CTA per SM; all CTAs together walk one line of work, item after item (sequence, block of 16 rows, key head), in
//     tiles of 128 keys, and each takes an equal stretch of it, wherever that cuts an item.  The lengths are read from device
//     memory when the kernel runs: a captured call follows them, and nothing is planned on the host;
//   * a warp is a stream of its own: it fetches 16 keys and values at a time into its private ring (16-byte asynchronous
//     copies, page by page) and keeps its own running maximum, sum and accumulator, without a barrier in the loop;
//   * 16 rows and 16 keys are one tile of mma.sync m16n8k16: rows of queries, padded to 16, stay in registers, keys come
//     through ldmatrix.  Products of so few rows are far from the tensor cores' rate with either kind of instruction, and
//     registers spare the way of S and P through tensor memory (about 2,000 clocks a tile for one row);
//   * codes of 8 bits become bf16 exactly, in registers; the scale of a key multiplies its score and the scale of a value its
//     weight, both in fp32.  The columns of a product are summed in the order in which 8-bit codes come out of ldmatrix;
//   * the warps of a CTA join at the end of a stretch of an item; an item that lies in several CTAs is joined by the one that
//     finishes last, in the order of the CTAs, so that results do not depend on which that is.
#include "zl_cache.cuh"

namespace zl {

using namespace cache;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRows = kTokenRows;  // query rows of an item
constexpr int kKeys = 16;    // keys of a warp's step
constexpr int kTile = kKeys * kWarps;
constexpr float kRescale = 8.f;  // powers of two by which a score may exceed the reference before sums are rescaled
constexpr float kLn2 = 0.6931471805599453f;

template <int D, int kFormat>
struct TokenSmem {
    static constexpr bool kCodes = kFormat != ZL_CACHE_BF16;
    static constexpr int kRowBytes = D * (kCodes ? 1 : 2);
    static constexpr int kMatrixBytes = kKeys * kRowBytes;  // 16 keys or 16 values
    static constexpr int kStageBytes = 2 * kMatrixBytes + (kCodes ? 2 * kKeys * 4 : 0);
    static constexpr int kStages = (D == 128) ? (kCodes ? 6 : 3) : (kCodes ? 8 : 6);
    static constexpr int kOPitch = D + 8;  // floats between rows of a warp's accumulator: rows on different banks
    static constexpr int kRingBytes = kStages * kStageBytes;
    static_assert(kRingBytes >= kRows * kOPitch * 4, "a warp's accumulator takes the place of its ring");
    alignas(1024) uint8_t ring[kWarps][kRingBytes];
    float m[kWarps][kRows], l[kWarps][kRows];
    uint32_t mask[kWarps][kStages];  // keys of a stage that exist
    int64_t scan[kWarps + 1];
    int64_t start_base;
    int32_t start_seq, ticket;
};

// A CTA's partial result of an item: maxima (powers of two) and sums of the rows, then their unnormalised outputs.
template <int D>
constexpr int kPartFloats = kRows * (D + 2);

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
// c += a b: 16 rows x 8 columns, 16 deep
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a 16-row matrix: chunks are exchanged within lines of 128 bytes so that
// the eight rows of an 8x8 matrix lie on different banks.
template <int kRowBytes>
__device__ __forceinline__ uint32_t swizzled(int row, int chunk) {
    return row * kRowBytes + ((chunk ^ (kRowBytes == 64 ? (row >> 1) & 3 : row & 7)) << 4);
}

// The line of work: every sequence is `items` items of `cost` units; unit 0 of an item stands for its start and end, the
// others for its tiles.
struct SeqWork {
    int32_t items, tiles, blocks;
    __device__ __forceinline__ int64_t units() const { return (int64_t)items * (tiles + 1); }
};
__device__ __forceinline__ SeqWork seq_work(const CachedParams& p, const SeqView& v) {
    SeqWork w;
    w.blocks = (int32_t)(((int64_t)v.q_len * p.group + kRows - 1) / kRows);
    if (p.split && w.blocks > 1) w.blocks = 0;  // the other kernel's
    w.items = w.blocks * p.c.n_kv_heads;
    w.tiles = v.q_len > 0 ? (keys_seen(v, v.q_len - 1) + kTile - 1) / kTile : 0;
    return w;
}

template <int D, int kFormat>
__global__ void __launch_bounds__(kThreads, 1)
zl_cached_tokens_kernel(const CachedParams p) {
    using Smem = TokenSmem<D, kFormat>;
    constexpr bool kCodes = Smem::kCodes;
    constexpr int kRowBytes = Smem::kRowBytes, kMatrixBytes = Smem::kMatrixBytes, kStages = Smem::kStages;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, quad = lane & 3;
    grid_release();
    grid_wait();

    // ---- this CTA's stretch [begin, end) of the line, and the sequence that `begin` lies in
    int64_t begin, end, per;
    {
        const int chunk = (p.b.n_seqs + kThreads - 1) / kThreads;
        int64_t mine = 0;
        for (int s = tid * chunk; s < min((tid + 1) * chunk, p.b.n_seqs); ++s) mine += seq_work(p, load_seq(p.b, p.c.page_shift, s)).units();
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
                const int64_t n = seq_work(p, load_seq(p.b, p.c.page_shift, s)).units();
                if (begin < at + n) break;
                at += n;
                ++s;
            }
            sm.start_seq = s;
            sm.start_base = at;
        }
        __syncthreads();
    }
    int s = sm.start_seq;
    int64_t base = sm.start_base;
    SeqView sv = load_seq(p.b, p.c.page_shift, s);
    SeqWork sw = seq_work(p, sv);

    const uint32_t ring = smem_u32(sm.ring[warp]);
    for (int64_t at = begin; at < end;) {
        while (at >= base + sw.units()) {
            base += sw.units();
            ++s;
            sv = load_seq(p.b, p.c.page_shift, s);
            sw = seq_work(p, sv);
        }
        const int32_t cost = sw.tiles + 1;
        const int32_t item = (int32_t)((at - base) / cost);
        const int64_t item0 = base + (int64_t)item * cost;       // unit 0 of the item
        const int64_t stop = min(end, item0 + cost);
        const int32_t tile0 = (int32_t)max((int64_t)0, at - item0 - 1), tile1 = (int32_t)(stop - item0 - 1);
        const bool starts_here = at == item0;
        at = stop;
        if (tile1 <= tile0 && !(sw.tiles == 0 && starts_here)) continue;  // only the start of an item whose tiles lie in later CTAs
        const int32_t head = item % p.c.n_kv_heads, row0 = (item / p.c.n_kv_heads) * kRows;
        const int32_t rows = (int32_t)min((int64_t)kRows, (int64_t)sv.q_len * p.group - row0);

        // ---- queries of the item: rows gid and gid + 8 of an A operand, and the keys these rows see
        uint32_t q[D / 16][4];
        int32_t seen[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int32_t r = row0 + gid + 8 * e;
            const bool ok = gid + 8 * e < rows;
            const int32_t i = ok ? r / p.group : 0;
            const __nv_bfloat16* src = p.q + (int64_t)(sv.q0 + i) * p.q_stride + (int64_t)(head * p.group + (ok ? r - i * p.group : 0)) * D;
            seen[e] = ok ? keys_seen(sv, i) : 0;
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
                q[ks][e] = x.x;
                q[ks][2 + e] = x.y;
            }
        }
        const int32_t all_see = __reduce_min_sync(0xffffffffu, min(gid < rows ? seen[0] : INT32_MAX, gid + 8 < rows ? seen[1] : INT32_MAX));
        const int32_t any_sees = __reduce_max_sync(0xffffffffu, max(seen[0], seen[1]));

        // ---- this warp's steps: keys 16 * (tile * 8 + warp) ..
        const int32_t n_steps = tile1 - tile0;
        auto fetch = [&](int32_t step) {
            if (step < n_steps) {
                const int32_t key0 = (tile0 + step) * kTile + warp * kKeys;
                const int st = step % kStages;
                const uint32_t dst = ring + st * Smem::kStageBytes;
                const int32_t key = key0 + (lane & 15);
                const int32_t pg = key < any_sees ? page_at(p.b, p.c, s, key) : -1;
                const uint32_t exists = __ballot_sync(0xffffffffu, pg >= 0);
                if (lane == 0) sm.mask[warp][st] = exists & 0xffffu;
                const int32_t in_mask = (1 << p.c.page_shift) - 1;
                constexpr int kChunks = kRowBytes / 16, kRowsAtOnce = 32 / kChunks;
#pragma unroll
                for (int i = 0; i < kKeys / kRowsAtOnce; ++i) {
                    const int r = i * kRowsAtOnce + lane / kChunks, ch = lane % kChunks;
                    const int32_t page = __shfl_sync(0xffffffffu, pg, r);
                    const bool live = page >= 0;
                    const int64_t off = live ? page * p.c.page_stride + ((key0 + r) & in_mask) * p.c.token_stride + head * p.c.head_stride + ch * 16 : 0;
                    const uint32_t to = dst + swizzled<kRowBytes>(r, ch);
                    cp16(to, p.c.k + off, live);
                    cp16(to + kMatrixBytes, p.c.v + off, live);
                }
                if constexpr (kCodes) {
                    const bool live = pg >= 0;
                    const int64_t off = live ? (((int64_t)pg << p.c.page_shift) + (key & in_mask)) * p.c.n_kv_heads + head : 0;
                    cp4(dst + 2 * kMatrixBytes + lane * 4, (lane < 16 ? p.c.k_scale : p.c.v_scale) + off, live);
                }
            }
            cp_commit();
        };
        float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) fetch(i);
        for (int32_t step = 0; step < n_steps; ++step) {
            cp_wait<kStages - 2>();
            __syncwarp();
            fetch(step + kStages - 1);  // into the stage of the step before this one
            const int st = step % kStages;
            const uint32_t ks_addr = ring + st * Smem::kStageBytes, vs_addr = ks_addr + kMatrixBytes;
            // ---- S: columns 2 quad, 2 quad + 1 of both key halves, rows gid and gid + 8
            float c[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[0][i] = c[1][i] = 0.f;
            if constexpr (kCodes) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ks += 2) {
                    uint32_t r[4];  // keys 0-7 and 8-15 of chunk ks, the same of chunk ks + 1
                    ldm4(r, ks_addr + swizzled<kRowBytes>(lane & 15, ks + (lane >> 4)));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        mma16(c[e & 1], q[ks + (e >> 1)], code_pair<kFormat, 0, 1>(r[e]), code_pair<kFormat, 2, 3>(r[e]));
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t r[4];  // chunks 2 ks and 2 ks + 1 of keys 0-7, the same of keys 8-15
                    ldm4(r, ks_addr + swizzled<kRowBytes>((lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1)));
                    mma16(c[0], q[ks], r[0], r[1]);
                    mma16(c[1], q[ks], r[2], r[3]);
                }
            }
            float2 scale_v[2];
            const int32_t key0 = (tile0 + step) * kTile + warp * kKeys;
            const uint32_t exists = sm.mask[warp][st];
            if constexpr (kCodes) {
                const float2* sc = reinterpret_cast<const float2*>(sm.ring[warp] + st * Smem::kStageBytes + 2 * kMatrixBytes);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float2 k2 = sc[h * 4 + quad];
                    scale_v[h] = sc[8 + h * 4 + quad];
                    k2.x *= p.scale_log2;
                    k2.y *= p.scale_log2;
                    c[h][0] *= k2.x; c[h][1] *= k2.y; c[h][2] *= k2.x; c[h][3] *= k2.y;
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) c[h][i] *= p.scale_log2;
            }
            if (key0 + kKeys > all_see || exists != 0xffffu) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int col = h * 8 + quad * 2 + (i & 1);
                        if (key0 + col >= seen[i >> 1] || !((exists >> col) & 1)) c[h][i] = -INFINITY;
                    }
            }
            float mx[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) mx[e] = fmaxf(fmaxf(c[0][2 * e], c[0][2 * e + 1]), fmaxf(c[1][2 * e], c[1][2 * e + 1]));
            if (__any_sync(0xffffffffu, mx[0] > m[0] + kRescale || mx[1] > m[1] + kRescale)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
                    mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
                    const float up = fmaxf(m[e], mx[e]);
                    const float alpha = up == -INFINITY ? 1.f : ex2(m[e] - up);
                    m[e] = up;
                    l[e] *= alpha;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        o[i][2 * e] *= alpha;
                        o[i][2 * e + 1] *= alpha;
                    }
                }
            }
            // ---- P, rounded to bf16 for its product with V (the sums take it unrounded)
            const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
            uint32_t a[4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = ex2(c[h][2 * e] - ref[e]), y = ex2(c[h][2 * e + 1] - ref[e]);
                    l[e] += x + y;
                    if constexpr (kCodes) {
                        x *= scale_v[h].x;
                        y *= scale_v[h].y;
                    }
                    a[2 * h + e] = pack_bf16(x, y);
                }
            // ---- O += P V
#pragma unroll
            for (int ch = 0; ch < kRowBytes / 16; ch += 2) {
                uint32_t r[4];  // keys 0-7 and 8-15 of chunk ch, the same of chunk ch + 1
                ldm4t(r, vs_addr + swizzled<kRowBytes>(lane & 15, ch + (lane >> 4)));
                if constexpr (kCodes) {  // a chunk is 16 columns, even ones in bytes 0 and 2, odd ones in bytes 1 and 3
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        mma16(o[2 * (ch + e)], a, code_pair<kFormat, 0, 2>(r[2 * e]), code_pair<kFormat, 0, 2>(r[2 * e + 1]));
                        mma16(o[2 * (ch + e) + 1], a, code_pair<kFormat, 1, 3>(r[2 * e]), code_pair<kFormat, 1, 3>(r[2 * e + 1]));
                    }
                } else {
                    mma16(o[ch], a, r[0], r[1]);
                    mma16(o[ch + 1], a, r[2], r[3]);
                }
            }
        }
        cp_wait<0>();
        __syncwarp();

        // ---- the warps' results side by side: O = sum_w 2^(m_w - max) O_w and the same of the sums
        float* mine = reinterpret_cast<float*>(sm.ring[warp]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
            if (quad == 0) {
                sm.m[warp][gid + 8 * e] = m[e];
                sm.l[warp][gid + 8 * e] = l[e];
            }
            float* to = mine + (gid + 8 * e) * Smem::kOPitch;
            if constexpr (kCodes) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    *reinterpret_cast<float4*>(to + i * 16 + quad * 4) = make_float4(o[2 * i][2 * e], o[2 * i + 1][2 * e], o[2 * i][2 * e + 1], o[2 * i + 1][2 * e + 1]);
            } else {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2*>(to + i * 8 + quad * 2) = make_float2(o[i][2 * e], o[i][2 * e + 1]);
            }
        }
        __syncthreads();
        int32_t c_first = 0, c_last = 0;
        if (sw.tiles > 0) {
            c_first = (int32_t)((item0 + 1) / per);
            c_last = (int32_t)((item0 + sw.tiles) / per);
        }
        const bool whole = c_first == c_last;
        auto finish = [&](int r, int c4, float mm, float ll, const float4& acc) {
            const int32_t i = (row0 + r) / p.group, h = head * p.group + (row0 + r) % p.group;
            const float inv = ll > 0.f ? 1.f / ll : 0.f;
            uint2 w;
            w.x = pack_bf16(acc.x * inv, acc.y * inv);
            w.y = pack_bf16(acc.z * inv, acc.w * inv);
            const int64_t row = sv.q0 + i;
            *reinterpret_cast<uint2*>(p.o + (row * p.n_heads + h) * D + c4 * 4) = w;
            if (c4 == 0 && p.lse) p.lse[(int64_t)h * p.b.total_q + row] = ll > 0.f ? (mm + log2f(ll)) * kLn2 : -INFINITY;
        };
        auto part_of = [&](int cta) {  // the item's part that CTA `cta` wrote
            return p.part + ((int64_t)cta * 2 + (item0 + 1 > cta * per ? 1 : 0)) * kPartFloats<D>;
        };
        for (int j = tid; j < rows * (D / 4); j += kThreads) {
            const int r = j / (D / 4), c4 = j % (D / 4);
            float mm = -INFINITY, ll = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sm.m[w][r]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mm > -INFINITY) {
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float f = ex2(sm.m[w][r] - mm);
                    const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(sm.ring[w]) + r * Smem::kOPitch + c4 * 4);
                    ll = fmaf(f, sm.l[w][r], ll);
                    acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                }
            }
            if (whole) {
                finish(r, c4, mm, ll, acc);
            } else {
                float* to = part_of(blockIdx.x);
                if (c4 == 0) {
                    to[r] = mm;
                    to[kRows + r] = ll;
                }
                *reinterpret_cast<float4*>(to + 2 * kRows + r * D + c4 * 4) = acc;
            }
        }
        if (!whole) {
            __threadfence();
            __syncthreads();
            if (tid == 0) sm.ticket = atomicAdd(p.part_count + c_first, 1);
            __syncthreads();
            if (sm.ticket == c_last - c_first) {
                __threadfence();
                for (int j = tid; j < rows * (D / 4); j += kThreads) {
                    const int r = j / (D / 4), c4 = j % (D / 4);
                    float mm = -INFINITY, ll = 0.f;
                    for (int c = c_first; c <= c_last; ++c) mm = fmaxf(mm, __ldcg(part_of(c) + r));
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (mm > -INFINITY) {
#pragma unroll 4
                        for (int c = c_first; c <= c_last; ++c) {
                            const float* from = part_of(c);
                            const float f = ex2(__ldcg(from + r) - mm);
                            const float4 x = __ldcg(reinterpret_cast<const float4*>(from + 2 * kRows + r * D + c4 * 4));
                            ll = fmaf(f, __ldcg(from + kRows + r), ll);
                            acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
                        }
                    }
                    finish(r, c4, mm, ll, acc);
                }
                if (tid == 0) p.part_count[c_first] = 0;  // for the next launch
            }
        }
        __syncthreads();  // the rings are free again
    }
}

template <int D, int kFormat>
cudaError_t launch_t(const CachedParams& p, int grid, cudaStream_t stream) {
    constexpr int smem = sizeof(TokenSmem<D, kFormat>);
    static_assert(smem <= 232448, "shared memory of a CTA");
    constexpr int kMaxDevices = 64;
    static bool configured[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices || !configured[dev]) {
        e = cudaFuncSetAttribute(zl_cached_tokens_kernel<D, kFormat>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < kMaxDevices) configured[dev] = true;
    }
    return launch_dependent(zl_cached_tokens_kernel<D, kFormat>, grid, kThreads, smem, stream, true, p);
}

}  // namespace

size_t cached_tokens_part_bytes(int head_dim) { return 2 * sizeof(float) * (head_dim == 128 ? kPartFloats<128> : kPartFloats<64>); }

cudaError_t launch_cached_tokens(int head_dim, int format, const CachedParams& p, int grid, cudaStream_t stream) {
    if (head_dim == 128) {
        if (format == ZL_CACHE_BF16) return launch_t<128, ZL_CACHE_BF16>(p, grid, stream);
        return format == ZL_CACHE_INT8 ? launch_t<128, ZL_CACHE_INT8>(p, grid, stream) : launch_t<128, ZL_CACHE_E4M3>(p, grid, stream);
    }
    if (format == ZL_CACHE_BF16) return launch_t<64, ZL_CACHE_BF16>(p, grid, stream);
    return format == ZL_CACHE_INT8 ? launch_t<64, ZL_CACHE_INT8>(p, grid, stream) : launch_t<64, ZL_CACHE_E4M3>(p, grid, stream);
}

}  // namespace zl
