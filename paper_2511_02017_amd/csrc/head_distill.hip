// Distillation of the draft head from a teacher of which each row lists the largest logits.
//
//   t_k = exp(l_k - lse_T),  mass = sum_k t_k,  loss = sum_k t_k (ln t_k - z_(id_k) + lse)
//   g_v = row_weight (mass e^(z_v - lse) - sum over k with id_k = v of t_k),  dh = scale g W,  dW = scale g^T h
//
// lse_T is the teacher's own, or that of the list (then mass is 1).  The products are the cross entropy's: its loss kernel leaves lse, its gradient
// kernel the softmax times mass; what is added here are the listed tokens, a few hundred bytes a row beside its vocabulary.
#include "head_loss_device.h"

namespace tapout {
namespace {

// ---- the head's logits at the listed tokens ---------------------------------------------------------------
__device__ __forceinline__ float wave_sum_f(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
template <class E> __device__ __forceinline__ float dot16(u32x4 a, u32x4 b, float s)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(E) == 4) s = fmaf(__uint_as_float(a[k]), __uint_as_float(b[k]), s);
        else {
            s = fmaf(__uint_as_float(a[k] << 16), __uint_as_float(b[k] << 16), s);
            s = fmaf(__uint_as_float(a[k] & 0xffff0000u), __uint_as_float(b[k] & 0xffff0000u), s);
        }
    }
    return s;
}

// By a workgroup, a wavefront eight listed tokens at a time, whose weights it reads side by side.
template <class E> __device__ __forceinline__ void listed_logits(const LossArgs &a, int row)
{
    constexpr int U = 8, n = 16 / (int)sizeof(E);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const E *h = (const E *)((const char *)a.hidden.p + (int64_t)row * a.hidden.stride);
    const int32_t *ids = a.ids + (int64_t)row * a.T;
    for (int k0 = wave * U; k0 < a.T; k0 += 4 * U) {
        const E *w[U];
        bool real[U];
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id = k0 + u < a.T ? ids[k0 + u] : -1;
            real[u] = id >= 0 && id < a.V;
            w[u] = (const E *)((const char *)a.weight.p + (real[u] ? id : 0) * a.weight.stride);
            s[u] = 0.f;
        }
        for (int c = lane * n; c < a.D; c += 64 * n) {
            const u32x4 x = *(const u32x4 *)(h + c);
            u32x4 y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) y[u] = real[u] ? *(const u32x4 *)(w[u] + c) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < U; ++u) s[u] = real[u] ? dot16<E>(x, y[u], s[u]) : 0.f;
        }
        float mine = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float v = wave_sum_f(s[u]);
            if (lane == u) mine = v;
        }
        if (lane < U && k0 + lane < a.T) a.top[(int64_t)row * a.T + k0 + lane] = mine;
    }
}

// ---- a row's list ------------------------------------------------------------------------------------------
// What the teacher's side of a row says, in every lane of its wavefront.
struct Teacher {
    int listed;          // entries that count
    bool bad_token;      // an id behind the vocabulary
    double lse, mass;
    __device__ __forceinline__ Teacher(const int32_t *ids, const float *logits, const float *given, int T, int V)
    {
        const int lane = threadIdx.x & 63;
        float m = -INFINITY;
        bool bad = false, nan = false;
        int count = 0;
        for (int k = lane; k < T; k += 64) {
            const int id = ids[k];
            if (id < 0) continue;
            ++count;
            bad |= id >= V;
            nan |= !(logits[k] < INFINITY);
            m = fmaxf(m, logits[k]);
        }
        for (int d = 32; d; d >>= 1) { m = fmaxf(m, __shfl_xor(m, d)); count += __shfl_xor(count, d); }
        listed = count;
        bad_token = __any(bad);
        nan = __any(nan);
        const double ref = m > -INFINITY ? (double)m : 0.0;
        double s = 0.0;
        for (int k = lane; k < T; k += 64)
            if (ids[k] >= 0) s += exp((double)logits[k] - ref);
        for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
        lse = given ? (double)*given : ref + log(s);
        if (nan || !(fabs(lse) < (double)INFINITY)) lse = __longlong_as_double(0x7ff8000000000000ll);
        mass = given ? s * exp(ref - lse) : lse == lse ? 1.0 : lse;
    }
    __device__ __forceinline__ double log_t(float logit) const { return (double)logit - lse; }
    __device__ __forceinline__ bool counts() const { return listed > 0 && !bad_token && mass < (double)INFINITY; }
};

// A workgroup a row: the listed logits, lse from the blocks of the vocabulary, then its first wavefront the list.  Bound by what the caches deliver of the
// listed tokens' weights: 8192 rows of 64, dim = 2048, bfloat16, 260 us, 8.3 TB/s, a twelfth of the loss's product (with a launch of their own for the
// logits 293; 40 rows of 16, dim = 1024, binary32 10.1 us, with two launches 12.4 and the gap between them).
template <class E>
__global__ __launch_bounds__(256) void listed_join_kernel(LossArgs a, int blocks)
{
    __shared__ float maxima[4];
    __shared__ double sums[4];
    const int n = blockIdx.x;
    listed_logits<E>(a, n);                                    // in memory for the first wavefront behind the barriers of the sums
    const double lse = join_lse(a.part + (int64_t)n * blocks, blocks, maxima, sums);
    if (threadIdx.x >= 64) return;
    const int32_t *ids = a.ids + (int64_t)n * a.T;
    const float *logits = a.logits + (int64_t)n * a.T, *top = a.top + (int64_t)n * a.T;
    const Teacher t(ids, logits, a.teacher_lse ? a.teacher_lse + n : nullptr, a.T, a.V);
    double s = 0.0;
    for (int k = threadIdx.x; k < a.T; k += 64) {
        if (ids[k] < 0) continue;
        const double log_t = t.log_t(logits[k]), p = exp(log_t);
        if (p != 0.0) s += p * (log_t - (double)top[k] + lse);          // NaN too
    }
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (threadIdx.x) return;
    const bool bad = !(fabs(lse) < (double)INFINITY), no_teacher = t.listed && !(t.mass < (double)INFINITY);
    const float nan = __uint_as_float(0x7fc00000u);
    a.lse[n] = bad ? nan : (float)lse;
    a.loss[n] = !t.listed ? 0.f : t.bad_token || no_teacher || bad ? nan : (float)s;
    if (a.flags) {
        const uint32_t f = (t.listed && (bad || no_teacher) ? TAPOUT_FLAG_BAD_ROW : 0u) | (t.bad_token ? TAPOUT_FLAG_BAD_TOKEN : 0u);
        if (f) atomicOr(&a.flags[n / a.rows_per_seq], f);
    }
}

// ---- gradient ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void listed_rows_kernel(ListedArgs a)
{
    const int n = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (n >= a.N) return;
    const Teacher t(a.ids + (int64_t)n * a.T, a.logits + (int64_t)n * a.T, a.teacher_lse ? a.teacher_lse + n : nullptr, a.T, a.V);
    if (threadIdx.x & 63) return;
    const float w = a.row_weight ? a.row_weight[n] : 1.f;
    const bool counts = t.counts() && fabsf(a.lse[n]) < INFINITY && w != 0.f;
    a.state[n] = counts ? 0 : -1;
    a.factor[n] = counts ? (float)((double)w * t.mass) : 0.f;
}

// A wavefront a row.  A token listed more than once has the sum of its entries, in their order, from the lane of the first one.
// bfloat16: the element is made from the listed logit, since what is in the piece is rounded already.  binary32: the teacher's share is taken from the
// element that is there.  Its logit is summed like those in lse, so an error that a large one has is in both and mostly leaves the quotient: from the
// listed logit, which is nearer to the exact one, dW was off by 3.3e-6 of its norm (40 rows, V = 32000, dim = 1024), three times as far.
// Every entry is compared with all of its row's, and the list is gone through for each piece of the vocabulary: 8192 rows, V = 128256 in four pieces, 25 us a
// piece for 64 listed tokens, 1.44 ms for 1024 (with 3.9 ms for their logits in the loss 42 % of the 23.0 ms of loss and gradients, 256 listed: 14.6).
constexpr int kListCap = 1024;
template <class E>
__global__ __launch_bounds__(64) void listed_grad_kernel(ListedArgs a, GradArgs piece)
{
    __shared__ int32_t sh_id[kListCap];
    __shared__ float sh_t[kListCap];
    const int n = blockIdx.x, lane = threadIdx.x;
    if (a.state[n] < 0) return;
    const int32_t *ids = a.ids + (int64_t)n * a.T;
    const float *logits = a.logits + (int64_t)n * a.T, *top = a.top + (int64_t)n * a.T;
    const Teacher t(ids, logits, a.teacher_lse ? a.teacher_lse + n : nullptr, a.T, a.V);
    for (int k = lane; k < a.T; k += 64) {
        sh_id[k] = ids[k];
        sh_t[k] = ids[k] < 0 ? 0.f : (float)exp(t.log_t(logits[k]));
    }
    __syncthreads();
    const float lse = a.lse[n], w = a.row_weight ? a.row_weight[n] : 1.f;
    for (int k = lane; k < a.T; k += 64) {
        const int id = sh_id[k], v = id - piece.v0;
        if (id < 0 || v < 0 || v >= piece.n) continue;
        float sum = 0.f;
        bool again = false;
        for (int j = 0; j < a.T; ++j) {
            again |= j < k && sh_id[j] == id;
            sum += sh_id[j] == id ? sh_t[j] : 0.f;
        }
        if (again) continue;
        E *const to = (E *)piece.g + (int64_t)n * piece.g_stride + v;
        float g;
        if constexpr (sizeof(E) == 4) g = fmaf(-w, sum, *to);
        else g = w * ((float)t.mass * __builtin_amdgcn_exp2f((top[k] - lse) * kLog2e) - sum);
        *to = (E)g;
        ((E *)piece.gt)[(int64_t)v * piece.gt_stride + n] = (E)g;
    }
}

}  // namespace

hipError_t launch_listed_join(const LossArgs &a, int blocks, int dtype, hipStream_t st)
{
    if (dtype == TAPOUT_F32) listed_join_kernel<float><<<a.N, 256, 0, st>>>(a, blocks);
    else listed_join_kernel<__bf16><<<a.N, 256, 0, st>>>(a, blocks);
    return hipGetLastError();
}

hipError_t launch_listed_rows(const ListedArgs &a, hipStream_t st)
{
    listed_rows_kernel<<<up(a.N, 4), 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_listed_grad(const ListedArgs &a, const GradArgs &piece, int dtype, hipStream_t st)
{
    if (a.T > kListCap) return hipErrorInvalidValue;
    if (dtype == TAPOUT_F32) listed_grad_kernel<float><<<a.N, 64, 0, st>>>(a, piece);
    else listed_grad_kernel<__bf16><<<a.N, 64, 0, st>>>(a, piece);
    return hipGetLastError();
}

}  // namespace tapout
