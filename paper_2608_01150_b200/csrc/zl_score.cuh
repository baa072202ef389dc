// Scores beyond scale * q.k, as the scored forward and backward kernels form them (both work in powers of two).
#pragma once

#include <type_traits>

#include "zl_device.h"
#include "zl_ptx.cuh"

namespace zl {
namespace score {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f;
// Bucket entries at or below this remove their pairs (score -inf), so that a table filled with the lowest value of its
// type cannot turn rows into sums of rounding errors.
constexpr float kRemoved = -1e30f;

// ------------------------------------------------------------------------------------------------ waits
// The timed loop of a bounded wait is out of line where registers allow a call (the producer and the MMA issuer): the kernels
// have dozens of wait sites and their loops should stay in the instruction cache.
constexpr uint64_t kWaitLimitNs = 4000000000ull;
static __device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, const volatile int32_t* abort_flag) {
    return mbar_wait_slow(bar, parity, kWaitLimitNs, abort_flag);
}
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, const volatile int32_t* abort_flag) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, abort_flag);
}
__device__ __forceinline__ bool wait_inline(uint64_t* bar, uint32_t parity, const volatile int32_t* abort_flag) {
    return mbar_wait(bar, parity, kWaitLimitNs, abort_flag);
}
__device__ __forceinline__ void report(int32_t* status, volatile int32_t* abort_flag, int where) {
    *abort_flag = 1;
    if (atomicCAS(status, 0, (int)ZL_ERR_TIMEOUT) == 0) status[1] = where;
}

// ------------------------------------------------------------------------------------------------ cap
// A capped score is off by at most 2^-20 of its own magnitude: 4e-7 of the tanh itself (below), and the roundings of the factors
// around it.  Two forms of the tanh:
// Near zero: tanh(y) / y as a polynomial in y^2 for |y| <= kTanhRange, fitted by iterated reweighted least squares on 4,000
// Chebyshev nodes, largest relative error 7e-8.  Five multiply-adds in packed fp32 and no special-function operation: that
// unit gives 16 results a clock and SM and already computes the softmax's exponentials (forward over 9450 tokens, 12
// heads, d 128: 600 us against 1,000 with exponential and reciprocal for every tanh).
constexpr float kTanhRange = 0.6f;
constexpr float kTanhC0 = 0.9999999307553031f, kTanhC1 = -0.3333234430833674f, kTanhC2 = 0.13310648814868545f,
                kTanhC3 = -0.052122548544318484f, kTanhC4 = 0.015504640407993653f;

__device__ __forceinline__ float2 splat(float x) { return make_float2(x, x); }

// tanh of both, |y| <= kTanhRange.
__device__ __forceinline__ float2 tanh_near(float2 y) {
    const float2 z = mul2(y, y);
    float2 r = fma2(z, splat(kTanhC4), splat(kTanhC3));
    r = fma2(z, r, splat(kTanhC2));
    r = fma2(z, r, splat(kTanhC1));
    r = fma2(z, r, splat(kTanhC0));
    return mul2(y, r);
}
// |y| > kTanhRange, for the backward, whose C' = 1 - tanh^2 wants small absolute errors near 1: 1 - 2 / (exp(2y) + 1), with
// exact limits at +-inf.
__device__ __forceinline__ float tanh_far(float y) {
    return 1.f - 2.f * rcp(ex2(y * (2.f * kLog2e)) + 1.f);
}
// Any y: tanh(y) / y = P(y^2) / Q(y^2) for |y| <= kTanhEnd, fitted the same way (largest relative error 1.5e-7, 4.3e-7 as
// evaluated); beyond, tanh is 1 to 2.3e-7.  1 - 2 / (exp(2y) + 1) would be right for large y only: near 0 its difference
// cancels, and a tile that saturates in one row may be small in the next.  One special-function operation per score instead
// of two: saturating scores of 1560 + 1560 + 3600 tokens 274 -> 261 us (12 heads, d 128).
constexpr float kTanhEnd = 8.f;
constexpr float kTanhP0 = 0.999999854f, kTanhP1 = 0.12925662f, kTanhP2 = 0.00295102275f, kTanhP3 = 1.14284123e-05f;
constexpr float kTanhQ1 = 0.462588777f, kTanhQ2 = 0.02381555f, kTanhQ3 = 0.000238669022f, kTanhQ4 = 2.45920737e-07f;
__device__ __forceinline__ float2 tanh_all(float2 y, float times) {  // times * tanh
    y = make_float2(clamp_abs(y.x, kTanhEnd), clamp_abs(y.y, kTanhEnd));
    const float2 z = mul2(y, y);
    float2 n = fma2(z, splat(kTanhP3), splat(kTanhP2));
    n = fma2(z, n, splat(kTanhP1));
    n = fma2(z, n, splat(kTanhP0));
    float2 q = fma2(z, splat(kTanhQ4), splat(kTanhQ3));
    q = fma2(z, q, splat(kTanhQ2));
    q = fma2(z, q, splat(kTanhQ1));
    q = fma2(z, q, splat(1.f));
    return mul2(mul2(y, n), mul2(make_float2(rcp(q.x), rcp(q.y)), splat(times)));  // (products with `times` ahead would stay in registers)
}

// ------------------------------------------------------------------------------------------------ bias by distance
// The bucket of a signed distance, -1 for none.
__device__ __forceinline__ int bucket_at(const ScoreParams& sp, int dist) {
    const int b = __ldg(sp.bucket_of + (min(max(dist, -sp.reach), sp.reach) + sp.reach));
    return (uint32_t)b < (uint32_t)sp.n_buckets ? b : -1;
}
// The bucket part for a signed distance, in powers of two.
__device__ __forceinline__ float bucket_bias_at(const ScoreParams& sp, int head, int dist) {
    if (!sp.bucket_bias) return 0.f;
    const int b = bucket_at(sp, dist);
    if (b < 0) return 0.f;
    const float v = __ldg(sp.bucket_bias + (int64_t)b * sp.n_heads + head);
    return v <= kRemoved ? -INFINITY : v * kLog2e;
}

// What a head adds: -slope |d| everywhere, and the bucket part, which is constant from the reach on.
struct HeadBias {
    float slope, far_neg, far_pos;  // powers of two; far_*: bucket part for distances <= -reach, >= reach
    __device__ __forceinline__ void load(const ScoreParams& sp, int head) {
        slope = sp.slopes ? __ldg(sp.slopes + head) * kLog2e : 0.f;
        far_neg = bucket_bias_at(sp, head, -sp.reach);
        far_pos = bucket_bias_at(sp, head, sp.reach);
    }
    __device__ __forceinline__ float at(const ScoreParams& sp, int head, int dist) const {
        return bucket_bias_at(sp, head, dist) - slope * fabsf((float)dist);
    }
};

// A patch of scores whose distances run from `lo` to `hi`: on one side of the query and beyond the reach (the bias is
// linear in the distance), or near it (the bias is looked up, one value per distance).
enum PatchSide { kNear = 0, kFarNeg = -1, kFarPos = 1 };
__device__ __forceinline__ PatchSide patch_side(const ScoreParams& sp, int lo, int hi) {
    return lo >= sp.reach ? kFarPos : (hi <= -sp.reach ? kFarNeg : kNear);
}

// The items of a CTA: for (int it = w.first; it < w.end; it += w.step).
struct Walk {
    int first, end, step;
    template <class Params>
    __device__ __forceinline__ explicit Walk(const Params& p) {
        first = p.lists ? __ldg(p.lists + blockIdx.x) : (int)blockIdx.x;
        end = p.lists ? __ldg(p.lists + blockIdx.x + 1) : p.n_items;
        step = p.lists ? 1 : (int)gridDim.x;
    }
};

__device__ __forceinline__ TaskPos task_pos(const ScoreParams& sp, int task) {
    return sp.pos ? sp.pos[task] : TaskPos{0, 0, 0, 0};
}

// ------------------------------------------------------------------------------------------------ a forward tile's row
// Key tiles that the query tile of an item starting at row `row0` with `rows` rows walks over.
__device__ __forceinline__ int key_tiles(const ScoreParams& sp, const Task& t, int task, int row0, int rows) {
    if (rows <= 0) return 0;
    const int keys = sp.masked ? visible_keys(task_pos(sp, task), t.kv_len, row0 + rows - 1) : t.kv_len;
    return (keys + kTileKV - 1) / kTileKV;
}

// Distances of a 128 x 128 tile: 255, and one more so that eight per lane cover them.
constexpr int kWindow = 256;

// Warps 2 and 3 of the forward kernels fetch the biases of near tiles, one distance each, ahead of the softmax warps: two
// dependent loads from L2 (bucket, then bias) would otherwise stand in front of every near tile.
struct WindowFeed {
    uint64_t *full, *empty;  // arrivals: the feeding warp; the 128 threads of the warpgroup that reads
    float* window;           // kWindow floats
    uint32_t count = 0;
    // Puts the biases of distances lo .. lo + 254 into the window; false: the bounded wait expired.
    __device__ __forceinline__ bool put(const ScoreParams& sp, const HeadBias& hb, int head, int lo, int lane,
                                        const volatile int32_t* abort_flag) {
        float v[kWindow / 32];
#pragma unroll
        for (int i = 0; i < kWindow / 32; ++i) v[i] = hb.at(sp, head, lo + i * 32 + lane);
        // up to a whole item of far tiles may lie between two near ones: a limit for the longest keys that fit the memory
        const bool ok = mbar_try_wait(empty, (count & 1) ^ 1) || mbar_wait_slow(empty, (count & 1) ^ 1, 16 * kWaitLimitNs, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) return false;
        ++count;
#pragma unroll
        for (int i = 0; i < kWindow / 32; ++i) window[i * 32 + lane] = v[i];
        __syncwarp();
        if (lane == 0) mbar_arrive(full);
        return true;
    }
};

// Largest of sv[c] * mul + base + step * c, or no more than a bound on it: with a slope, sixteen columns share the larger of
// their two edges' positions (sixteen independent chains of max either way).
constexpr int kMaxGroup = 16;
template <bool kBias>
__device__ __forceinline__ float row_bound(const float (&sv)[kTileKV], float mul, float base, float step) {
    float g[kTileKV / kMaxGroup];
#pragma unroll
    for (int i = 0; i < kTileKV / kMaxGroup; ++i) {
        const int c = i * kMaxGroup;
        g[i] = max3(sv[c], sv[c + 1], sv[c + 2]);
#pragma unroll
        for (int k = 3; k + 1 < kMaxGroup; k += 2) g[i] = max3(g[i], sv[c + k], sv[c + k + 1]);
    }
#pragma unroll
    for (int i = 0; i < kTileKV / kMaxGroup; ++i) {
        g[i] = fmaxf(g[i], sv[i * kMaxGroup + kMaxGroup - 1]);
        if constexpr (kBias) g[i] = fmaf(g[i], mul, fmaf(step, (float)(i * kMaxGroup), base));
    }
    const float m = fmaxf(max3(max3(g[0], g[1], g[2]), g[3], g[4]), max3(g[5], g[6], g[7]));
    return kBias ? m + fmaxf(0.f, step * (kMaxGroup - 1)) : m * mul;
}

// An upper bound of a row's scores serves as the softmax's reference as well as the maximum, so long as it is not far above:
// 2^-kSlack of the reference still leaves 2^60 to the smallest fp32 number, so nothing that counts is lost, and sums and
// LSE are exact relative to any reference.
constexpr float kSlack = 64.f;
// The reference of a row is only raised when a tile's maximum exceeds it by more than this many powers of two; until then
// exponentials stay below 2^8 and nothing is rescaled.
constexpr float kRescaleThresholdLog2 = 8.0f;

// One tile of the online softmax: a row of raw products `sv` becomes P (bf16, over S in TMEM, handed over in two halves of 64
// columns by `p_half`); the row's reference m_ref (powers of two) and sum l move on, O in TMEM is rescaled when the
// reference is raised.  Columns from `valid` on are invisible (`ragged`: for some row of the warp).  A near tile adds bias[c] (and releases the window), a far
// one a bias that is linear in the column, from distance `dist0` of column 0: that one stays in the exponential's
// multiply-add and costs nothing where it is constant.
template <int D, bool kCap, bool kBias>
__device__ __forceinline__ void softmax_tile(float (&sv)[kTileKV], const ScoreParams& sp, const HeadBias& hb, float scale_log2,
                                             bool first, PatchSide side, const float* bias, uint64_t* bias_empty, int dist0,
                                             int valid, bool ragged, bool row_ok, uint32_t s_addr, uint32_t o_addr, uint64_t (&p_half)[2],
                                             float& m_ref, float& l) {
    float mul = scale_log2, base = 0.f, step = 0.f;  // score(c) = sv[c] * mul + base + step * c, in powers of two
    float2 sum2 = make_float2(0.f, 0.f);
    // Half h of P is on its way to TMEM; the first half is handed over some way into the second, when its store has landed.
    constexpr int kLater = 16;  // columns of the second half
    auto hand_over = [&](int h) {
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&p_half[h]);
    };
    if constexpr (kCap) {
        mul = 1.f;
        float big = 0.f;
#pragma unroll
        for (int c = 0; c < kTileKV; c += 2) big = max3_abs(big, sv[c], sv[c + 1]);
        const bool near_zero = !row_ok || big * sp.scale_over_cap <= kTanhRange;  // rows that do not exist hold anything
        const float2 k1 = splat(sp.scale_over_cap);
        const float2 c0 = splat(kTanhC0 * sp.cap_log2), c1 = splat(kTanhC1 * sp.cap_log2), c2 = splat(kTanhC2 * sp.cap_log2),
                     c3 = splat(kTanhC3 * sp.cap_log2), c4 = splat(kTanhC4 * sp.cap_log2);
        if constexpr (!kBias) {
            // |C(x)| <= |x|, so the largest magnitude bounds the row's scores: where that does not ask for a higher
            // reference, cap and exponential run in one pass, the multiply-adds of one score under the exponential of another
            const bool easy = !row_ok || (near_zero && !ragged && big * scale_log2 - m_ref <= kRescaleThresholdLog2);
            if (__all_sync(0xffffffffu, easy)) {
                const float2 nm = splat(-m_ref);
                constexpr int kGroup = 8;  // pairs whose chains run side by side
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t pk[kTileKV / 4];
#pragma unroll
                    for (int g = 0; g < kTileKV / 4; g += kGroup) {
                        if (h == 1 && 2 * g == kLater) hand_over(0);
                        float2 y[kGroup], r[kGroup];
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) {
                            const int c = h * (kTileKV / 2) + 2 * (g + i);
                            y[i] = mul2(make_float2(sv[c], sv[c + 1]), k1);
                        }
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) r[i] = fma2(mul2(y[i], y[i]), c4, c3);
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) r[i] = fma2(mul2(y[i], y[i]), r[i], c2);
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) r[i] = fma2(mul2(y[i], y[i]), r[i], c1);
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) r[i] = fma2(mul2(y[i], y[i]), r[i], c0);
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) r[i] = fma2(y[i], r[i], nm);
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) {
                            const float p0 = ex2(r[i].x), p1 = ex2(r[i].y);
                            sum2 = add2(sum2, make_float2(p0, p1));
                            pk[g + i] = pack_bf16(p0, p1);
                        }
                    }
                    tmem_st_x32(s_addr + h * 32, pk);
                }
                hand_over(1);
                l += sum2.x + sum2.y;
                return;
            }
        }
        if (__all_sync(0xffffffffu, near_zero)) {
#pragma unroll
            for (int c = 0; c < kTileKV; c += 2) {
                const float2 y = mul2(make_float2(sv[c], sv[c + 1]), k1);
                const float2 z = mul2(y, y);
                const float2 v = mul2(y, fma2(z, fma2(z, fma2(z, fma2(z, c4, c3), c2), c1), c0));
                sv[c] = v.x;
                sv[c + 1] = v.y;
            }
        } else {
#pragma unroll
            for (int c = 0; c < kTileKV; c += 2) {
                const float2 v = tanh_all(mul2(make_float2(sv[c], sv[c + 1]), k1), sp.cap_log2);
                sv[c] = v.x;
                sv[c + 1] = v.y;
            }
        }
    }
    if constexpr (kBias) {
        if (side == kNear) {
#pragma unroll
            for (int c = 0; c < kTileKV; c += 2) {
                const float2 v = fma2(make_float2(sv[c], sv[c + 1]), splat(mul), make_float2(bias[c], bias[c + 1]));
                sv[c] = v.x;
                sv[c + 1] = v.y;
            }
            mbar_arrive(bias_empty);
            mul = 1.f;
        } else {
            step = side == kFarPos ? -hb.slope : hb.slope;
            base = (side == kFarPos ? hb.far_pos : hb.far_neg) + step * (float)dist0;
            if (fabsf(step) * (kMaxGroup - 1) > kSlack) {  // warp-uniform: steep slopes get their exact maximum
#pragma unroll
                for (int c = 0; c < kTileKV; ++c) sv[c] = fmaf(sv[c], mul, fmaf(step, (float)c, base));
                mul = 1.f;
                base = step = 0.f;
            }
        }
    }
    if (ragged) {
#pragma unroll
        for (int c = 0; c < kTileKV; ++c)
            if (c >= valid) sv[c] = -INFINITY;  // select, never multiply
    }
    const float mx = row_bound<kBias>(sv, mul, base, step);
    // lazy reference update: only when the tile maximum is far above the reference; a row that has seen no key yet has
    // reference -inf, and so long as it sees none (mx = -inf, the difference is NaN) keeps it
    const bool raise = row_ok && mx - m_ref > kRescaleThresholdLog2;
    if (__any_sync(0xffffffffu, raise && !first)) {
        // rescale O (the previous P V product is complete: this S was issued after it)
        const float alpha = raise ? ex2(m_ref - mx) : 1.f;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
            uint32_t r[32];
            tmem_ld_x32(o_addr + c * 32, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
            tmem_st_x32(o_addr + c * 32, r);
        }
        l *= alpha;
    }
    if (raise) {
        if (first) l = 0.f;
        m_ref = mx;
    }
    const float add = base - (m_ref > -INFINITY ? m_ref : 0.f);
    auto half_of_p = [&](int h, auto linear) {
        uint32_t pk[kTileKV / 4];
#pragma unroll
        for (int c = 0; c < kTileKV / 2; c += 2) {
            const int cc = h * (kTileKV / 2) + c;
            if (h == 1 && c == kLater) hand_over(0);
            const float2 b = decltype(linear)::value ? make_float2(fmaf(step, (float)cc, add), fmaf(step, (float)(cc + 1), add)) : splat(add);
            const float2 e = fma2(make_float2(sv[cc], sv[cc + 1]), splat(mul), b);
            const float p0 = ex2(e.x), p1 = ex2(e.y);
            sum2 = add2(sum2, make_float2(p0, p1));
            pk[c / 2] = pack_bf16(p0, p1);
        }
        tmem_st_x32(s_addr + h * 32, pk);
        if (h == 1) hand_over(1);
    };
    if (kBias && step != 0.f) {  // warp-uniform
        half_of_p(0, std::true_type());
        half_of_p(1, std::true_type());
    } else {
        half_of_p(0, std::false_type());
        half_of_p(1, std::false_type());
    }
    l += sum2.x + sum2.y;
}

}  // namespace score
}  // namespace zl
