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

}  // namespace score
}  // namespace zl
