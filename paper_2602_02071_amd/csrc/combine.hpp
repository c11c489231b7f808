// Joins the parts of a row whose keys were split over workgroups: every part
// holds the unnormalised sum of P v over its keys, P relative to 2^m, and
// (m, sum of P); m = -inf for a part whose keys the row does not see.
#pragma once
#include "common.hpp"

namespace baps {

constexpr int kMaxSplits = 64;      // one lane of a wave per part

// One workgroup of 256 threads per row.  The lanes of a wave take the parts'
// maxima and weights at once; then 256 / (D/4) groups of D/4 threads add every
// so-manieth part, and the groups' sums meet in LDS in a fixed order: no load
// waits for the one before it (one thread per four elements over all parts in
// turn took 60 us for 64 parts).  Threads of group 0 get the row's four
// elements, normalised, in o and its log-sum-exp in lse (0 and -inf for a row
// without a key).  Returns whether the thread is one of them.
template <int D>
__device__ __forceinline__ bool combine_row(const float* part, const float* ml, int nsplit, long long rows, long long row,
                                            f32x4& o, float& lse)
{
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    __shared__ float weight[4][kMaxSplits];
    __shared__ f32x4 sums[kGroups - 1][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = tid / kLanes, d4 = tid % kLanes;
    const float ninf = -__builtin_huge_valf();
    // (every wave for itself: no barrier before the sums)
    float m = ninf, l = 0.0f;
    if (lane < nsplit) {
        const float* at = ml + 2 * (lane * rows + row);
        m = at[0];
        l = at[1];
    }
    const float top = wave_max_uniform(m);
    const float w = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    weight[wave][lane] = w;
    const float total = wave_sum(w * l);
    o = f32x4{};
#pragma unroll 4
    for (int k = g; k < nsplit; k += kGroups) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(part + (k * rows + row) * D + 4 * d4);
        const float wk = weight[wave][k];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += wk * x[e];
    }
    if (g > 0) sums[g - 1][d4] = o;
    __syncthreads();
    if (g > 0) return false;
#pragma unroll
    for (int k = 0; k < kGroups - 1; ++k) {
        const f32x4 x = sums[k][d4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[e];
    }
    const bool empty = top == ninf;
    const float inv = empty ? 0.0f : 1.0f / total;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    lse = empty ? ninf : 0.69314718055994531f * (top + log2f(total));
    return true;
}

// Up to kFewSplits parts: D/4 threads per row, d4 of 0 .. D/4 - 1, with all parts'
// loads in flight at once; several rows per workgroup, for a workgroup per row
// costs more to start than such a row takes (32768 rows of two parts, D = 128: 32
// -> 10 us).
constexpr int kFewSplits = 8;

template <int D>
__device__ __forceinline__ void combine_row_few(const float* part, const float* ml, int nsplit, long long rows, long long row,
                                                int d4, f32x4& o, float& lse)
{
    const float ninf = -__builtin_huge_valf();
    float m[kFewSplits], l[kFewSplits];
    f32x4 x[kFewSplits];
#pragma unroll
    for (int k = 0; k < kFewSplits; ++k) {
        m[k] = ninf;
        l[k] = 0.0f;
        x[k] = f32x4{};
        if (k < nsplit) {
            const long long at = k * rows + row;
            m[k] = ml[2 * at];
            l[k] = ml[2 * at + 1];
            x[k] = *reinterpret_cast<const f32x4*>(part + at * D + 4 * d4);
        }
    }
    float top = m[0];
#pragma unroll
    for (int k = 1; k < kFewSplits; ++k) top = fmaxf(top, m[k]);
    float total = 0.0f;
    o = f32x4{};
#pragma unroll
    for (int k = 0; k < kFewSplits; ++k) {
        const float w = m[k] == ninf ? 0.0f : __builtin_amdgcn_exp2f(m[k] - top);
        total += w * l[k];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += w * x[k][e];
    }
    const bool empty = top == ninf;
    const float inv = empty ? 0.0f : 1.0f / total;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    lse = empty ? ninf : 0.69314718055994531f * (top + log2f(total));
}

}  // namespace baps
