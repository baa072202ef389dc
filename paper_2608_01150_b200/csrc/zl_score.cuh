// Scores beyond scale * q.k, as the scored forward and backward kernels form them (both work in powers of two).
#pragma once

#include "zl_device.h"
#include "zl_ptx.cuh"

namespace zl {
namespace score {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f;
// Bucket entries at or below this remove their pairs (score -inf), so that a table filled with the lowest value of its
// type cannot turn rows into sums of rounding errors.
constexpr float kRemoved = -1e30f;

// ------------------------------------------------------------------------------------------------ cap
// tanh(y) / y as a polynomial in y^2 for |y| <= kTanhRange: fitted by iterated reweighted least squares on 4,000
// Chebyshev nodes, largest relative error 7e-8.  Five multiply-adds in packed fp32 instead of two special-function
// operations (exponential and reciprocal) per score: the special-function unit gives 16 results a clock and SM and
// already computes the softmax's exponentials.
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
// tanh of any y, as 1 - 2 / (exp(2y) + 1): absolute error about 1e-7, exact limits at +-inf.
__device__ __forceinline__ float tanh_any(float y) {
    return 1.f - 2.f * rcp(ex2(y * (2.f * kLog2e)) + 1.f);
}

// ------------------------------------------------------------------------------------------------ bias by distance
// The bucket part for a signed distance, in powers of two.
__device__ __forceinline__ float bucket_bias_at(const ScoreParams& sp, int head, int dist) {
    if (!sp.bucket_bias) return 0.f;
    const int b = __ldg(sp.bucket_of + (min(max(dist, -sp.reach), sp.reach) + sp.reach));
    if ((uint32_t)b >= (uint32_t)sp.n_buckets) return 0.f;
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

// Distances of a 32 x 128 patch: 32 + 128 - 1, rounded up to a multiple of 32.
constexpr int kWindow = 160;

// Turns a row of raw products into scores: the cap, the bias, -inf from column `valid` on.  With a cap or a bias the
// result is in powers of two, else it stays the raw product (the exponential's multiply-add scales it).  `window` holds
// the biases of a near patch, `dist_lo` is the distance of the patch's last row to its first column.
template <bool kCap, bool kBias>
__device__ __forceinline__ void finish_scores(float (&sv)[kTileKV], const ScoreParams& sp, const HeadBias& hb, PatchSide side,
                                              const float* window, int dist_lo, float scale_log2, int valid, int lane) {
    if constexpr (kCap) {
        float big = 0.f;
#pragma unroll
        for (int c = 0; c < kTileKV; c += 2) big = max3_abs(big, sv[c], sv[c + 1]);
        const float2 k1 = splat(sp.scale_over_cap), cl = splat(sp.cap_log2);
        if (__all_sync(0xffffffffu, big * sp.scale_over_cap <= kTanhRange)) {
#pragma unroll
            for (int c = 0; c < kTileKV; c += 2) {
                const float2 v = mul2(tanh_near(mul2(make_float2(sv[c], sv[c + 1]), k1)), cl);
                sv[c] = v.x;
                sv[c + 1] = v.y;
            }
        } else {
#pragma unroll
            for (int c = 0; c < kTileKV; ++c) sv[c] = tanh_any(sv[c] * sp.scale_over_cap) * sp.cap_log2;
        }
    }
    if constexpr (kBias) {
        const float mul = kCap ? 1.f : scale_log2;
        if (side == kNear) {
            const float* w = window + 31 - lane;
#pragma unroll
            for (int c = 0; c < kTileKV; c += 2) {
                const float2 v = fma2(make_float2(sv[c], sv[c + 1]), splat(mul), make_float2(w[c], w[c + 1]));
                sv[c] = v.x;
                sv[c + 1] = v.y;
            }
        } else {
            const float step = side == kFarPos ? -hb.slope : hb.slope;
            const float base = (side == kFarPos ? hb.far_pos : hb.far_neg) + step * (float)(dist_lo + 31 - lane);
            if (step == 0.f) {  // warp-uniform
#pragma unroll
                for (int c = 0; c < kTileKV; c += 2) {
                    const float2 v = fma2(make_float2(sv[c], sv[c + 1]), splat(mul), splat(base));
                    sv[c] = v.x;
                    sv[c + 1] = v.y;
                }
            } else {
#pragma unroll
                for (int c = 0; c < kTileKV; c += 2) {
                    const float2 b = make_float2(fmaf(step, (float)c, base), fmaf(step, (float)(c + 1), base));
                    const float2 v = fma2(make_float2(sv[c], sv[c + 1]), splat(mul), b);
                    sv[c] = v.x;
                    sv[c + 1] = v.y;
                }
            }
        }
    }
    if (__any_sync(0xffffffffu, valid < kTileKV)) {
#pragma unroll
        for (int c = 0; c < kTileKV; ++c)
            if (c >= valid) sv[c] = -INFINITY;  // select, never multiply
    }
}

__device__ __forceinline__ float row_max(const float (&sv)[kTileKV]) {
    // four independent chains: a single running maximum is a 64-deep dependent chain
    float mx0 = max3(sv[0], sv[1], sv[2]), mx1 = max3(sv[3], sv[4], sv[5]);
    float mx2 = max3(sv[6], sv[7], sv[8]), mx3 = max3(sv[9], sv[10], sv[11]);
#pragma unroll
    for (int c = 12; c + 7 < kTileKV; c += 8) {
        mx0 = max3(mx0, sv[c], sv[c + 1]);
        mx1 = max3(mx1, sv[c + 2], sv[c + 3]);
        mx2 = max3(mx2, sv[c + 4], sv[c + 5]);
        mx3 = max3(mx3, sv[c + 6], sv[c + 7]);
    }
    // columns 124..127 remain (12 + 8 * 14 = 124)
    mx0 = max3(mx0, sv[kTileKV - 4], sv[kTileKV - 3]);
    mx1 = max3(mx1, sv[kTileKV - 2], sv[kTileKV - 1]);
    return fmaxf(max3(mx0, mx1, mx2), mx3);
}

}  // namespace score
}  // namespace zl
