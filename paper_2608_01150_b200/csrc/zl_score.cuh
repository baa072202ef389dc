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

// Distances of a 32 x 128 patch: 32 + 128 - 1, rounded up to a multiple of 32.  A warp's window holds their biases four
// times, copy s shifted by s: a thread's 128 consecutive biases start at 31 - lane, and in copy (31 - lane) % 4 that start
// is 16-byte aligned, so the row is 32 four-word loads instead of 128 single ones.  Copies lie 8 banks apart, which keeps
// the eight lanes of a load phase on different banks.
constexpr int kWindow = 160;
constexpr int kWindowStride = 168;
constexpr int kWindowFloats = 4 * kWindowStride;

__device__ __forceinline__ void fill_window(float* window, const float (&bias)[kWindow / 32], int lane) {
    __syncwarp();  // the previous patch has been read
#pragma unroll
    for (int i = 0; i < kWindow / 32; ++i) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (i * 32 + lane >= s) window[s * kWindowStride + i * 32 + lane - s] = bias[i];
    }
    __syncwarp();
}

// How the exponent of a tile's row follows from its values: score(c) = v[c] * mul + base + step * c, in powers of two.
struct RowScore {
    float mul, base, step;
    float max;  // of the row's scores, or an upper bound
};
// An upper bound serves as the softmax's reference so long as it is not far above: 2^-kSlack of the reference still leaves
// 2^60 to the smallest fp32 number, so nothing that counts is lost, and sums and LSE are exact relative to any reference.
constexpr float kSlack = 64.f;

__device__ __forceinline__ float row_max(const float (&sv)[kTileKV]);

// Turns a row of raw products into values with `mul`, `base` and `step`: the cap and near biases change the values, a far
// bias (linear in the column) only base and step; columns from `valid` on become -inf.  `window` holds the biases of a near
// patch, `dist_lo` is the distance of the patch's last row to its first column.
template <bool kCap, bool kBias>
__device__ __forceinline__ RowScore finish_scores(float (&sv)[kTileKV], const ScoreParams& sp, const HeadBias& hb, PatchSide side,
                                                  const float* window, int dist_lo, float scale_log2, int valid, int lane) {
    RowScore rs{scale_log2, 0.f, 0.f, 0.f};
    if constexpr (kCap) {
        rs.mul = 1.f;
        float big = 0.f;
#pragma unroll
        for (int c = 0; c < kTileKV; c += 2) big = max3_abs(big, sv[c], sv[c + 1]);
        if (__all_sync(0xffffffffu, big * sp.scale_over_cap <= kTanhRange)) {
            const float2 k1 = splat(sp.scale_over_cap);
            const float2 c0 = splat(kTanhC0 * sp.cap_log2), c1 = splat(kTanhC1 * sp.cap_log2), c2 = splat(kTanhC2 * sp.cap_log2),
                         c3 = splat(kTanhC3 * sp.cap_log2), c4 = splat(kTanhC4 * sp.cap_log2);
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
            for (int c = 0; c < kTileKV; ++c) sv[c] = tanh_any(sv[c] * sp.scale_over_cap) * sp.cap_log2;
        }
    }
    if constexpr (kBias) {
        if (side == kNear) {
            const int start = 31 - lane;
            const float4* w = reinterpret_cast<const float4*>(window + (start & 3) * kWindowStride + (start & ~3));
#pragma unroll
            for (int c = 0; c < kTileKV; c += 4) {
                const float4 b = w[c / 4];
                const float2 v0 = fma2(make_float2(sv[c], sv[c + 1]), splat(rs.mul), make_float2(b.x, b.y));
                const float2 v1 = fma2(make_float2(sv[c + 2], sv[c + 3]), splat(rs.mul), make_float2(b.z, b.w));
                sv[c] = v0.x;
                sv[c + 1] = v0.y;
                sv[c + 2] = v1.x;
                sv[c + 3] = v1.y;
            }
            rs.mul = 1.f;
        } else {
            rs.step = side == kFarPos ? -hb.slope : hb.slope;
            rs.base = (side == kFarPos ? hb.far_pos : hb.far_neg) + rs.step * (float)(dist_lo + 31 - lane);
            if (fabsf(rs.step) * (kTileKV - 1) > kSlack) {  // warp-uniform: steep slopes get their exact maximum
#pragma unroll
                for (int c = 0; c < kTileKV; ++c) sv[c] = fmaf(sv[c], rs.mul, fmaf(rs.step, (float)c, rs.base));
                rs = RowScore{1.f, 0.f, 0.f, 0.f};
            }
        }
    }
    if (__any_sync(0xffffffffu, valid < kTileKV)) {
#pragma unroll
        for (int c = 0; c < kTileKV; ++c)
            if (c >= valid) sv[c] = -INFINITY;  // select, never multiply
    }
    rs.max = fmaf(row_max(sv), rs.mul, rs.base + fmaxf(0.f, rs.step * (kTileKV - 1)));
    return rs;
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
