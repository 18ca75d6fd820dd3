// Device code that the head's losses share.
#pragma once

#include "head.h"

namespace tapout {

template <int DT> struct ElemOf { using T = float; };
template <> struct ElemOf<TAPOUT_BF16> { using T = __bf16; };

__device__ __forceinline__ bool row_counts(int t, int V, const float *lse, const float *row_weight, int n)
{
    if (counted_target(t, V) < 0) return false;
    const float l = lse[n];
    return fabsf(l) < INFINITY && (!row_weight || row_weight[n] != 0.f);
}

// lse of a row from its blocks' maxima and sums, in double, in every thread of a workgroup of 256.
__device__ __forceinline__ double join_lse(const float2 *p, int blocks, float *maxima, double *sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = -INFINITY;
    double s = 0.0;
    for (int x = threadIdx.x; x < blocks; x += 1024) {
        float2 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = x + k * 256 < blocks ? p[x + k * 256] : float2{-INFINITY, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float top = fmaxf(m, q[k].x), ref = top == -INFINITY ? 0.f : top;
            s = s * (double)__builtin_amdgcn_exp2f((fmaxf(m, -3.4e38f) - ref) * kLog2e) + (double)q[k].y * (double)__builtin_amdgcn_exp2f((fmaxf(q[k].x, -3.4e38f) - ref) * kLog2e);
            m = top;
        }
    }
    const float own = m;
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) maxima[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(maxima[0], maxima[1]), fmaxf(maxima[2], maxima[3]));
    const float ref = m == -INFINITY ? 0.f : m;
    s *= (double)__builtin_amdgcn_exp2f((fmaxf(own, -3.4e38f) - ref) * kLog2e);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    return (double)ref + log(((sums[0] + sums[1]) + sums[2]) + sums[3]);
}

}  // namespace tapout
