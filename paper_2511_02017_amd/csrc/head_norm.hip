// Root-mean-square norm in front of the draft head, with the residual's addition, and its backward pass.
//
//   s = x + residual, rounded to the rows' type (the residual stream is kept in it, and the gradient is taken at what is kept)
//   r = 1 / sqrt(mean(s^2) + eps),  h = s r,  y = h w
//   u = g w,  ds = r (u - h mean(u h)) + g_sum,  dw = sum over rows of g h
//
// Squares are summed in binary64: binary32 squares of large states would overflow, and the sums cost nothing beside the memory's time.
#include "fp8_device.h"
#include "exp_device.h"

namespace tapout {
namespace {

template <class E> struct Vec {
    static constexpr int n = 16 / (int)sizeof(E), lanes_log = n == 8 ? 4 : 5;      // lanes whose vectors make 128 elements
    static __device__ __forceinline__ void unpack(const u32x4 &w, float (&x)[n])
    {
        if constexpr (n == 8) {
#pragma unroll
            for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(w[k]);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&x)[n])
    {
        E v[n];
#pragma unroll
        for (int k = 0; k < n; ++k) v[k] = (E)x[k];
        return *(const u32x4 *)v;
    }
};

template <class E> __device__ __forceinline__ const E *row_of(const Rows &m, int r, int K)
{
    const int b = K == 1 ? r : r / K;
    return (const E *)m.p + b * m.stride_b + (r - b * K) * m.stride_k;
}

// Sum over the threads of a row: a wavefront, or a workgroup of several (then every thread of it calls).
template <int TPR> __device__ __forceinline__ double row_sum(double v, double *sh)
{
    v = wave_sum_d(v);
    if constexpr (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int k = 0; k < TPR / 64; ++k) v += sh[k];
    }
    return v;
}

// A row for TPR threads, VPT 16-byte vectors a thread, all of them (of long rows, those of x) requested before the first is used.  A thread reads each of
// its places of a row before it writes there, and no other thread does either, so that the sum may take the place of x or of the residual.  Bound by
// memory: 8192 rows of 2048 bfloat16 with a residual 23.7 us, 5.7 TB/s; to 8 bits, 64 rows: 3.9 us, the launch.
template <class E, int TPR, int VPT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void head_norm_kernel(NormArgs a)
{
    using V = Vec<E>;
    constexpr int n = V::n;
    __shared__ double sh[TPR / 64];
    const int row = TPR == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x, t = threadIdx.x % TPR;
    if (row >= a.N) return;
    const E *x = row_of<E>(a.x, row, a.K), *res = a.residual.p ? row_of<E>(a.residual, row, a.K) : nullptr;
    u32x4 w[VPT], v[VPT], add[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = (t + i * TPR) * n;
        v[i] = add[i] = w[i] = u32x4{0, 0, 0, 0};
        if (c < a.D) {
            v[i] = *(const u32x4 *)(x + c);
            if (VPT <= 4 && res) add[i] = *(const u32x4 *)(res + c);
            if (VPT <= 4) w[i] = *(const u32x4 *)((const E *)a.weight + c);
        }
    }
    double squares = 0.0;
    E *sum = a.sum.p ? (E *)row_of<E>(a.sum, row, a.K) : nullptr;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float p[n], q[n];
        V::unpack(v[i], p);
        if (res) {
            if (VPT > 4 && (t + i * TPR) * n < a.D) add[i] = *(const u32x4 *)(res + (t + i * TPR) * n);
            V::unpack(add[i], q);
#pragma unroll
            for (int k = 0; k < n; ++k) p[k] += q[k];
            v[i] = V::pack(p);
            V::unpack(v[i], p);
        }
#pragma unroll
        for (int k = 0; k < n; ++k) squares = fma((double)p[k], (double)p[k], squares);
        if (sum && (t + i * TPR) * n < a.D) *(u32x4 *)(sum + (t + i * TPR) * n) = v[i];
    }
    const float r = (float)(1.0 / sqrt(row_sum<TPR>(squares, sh) / a.D + (double)a.eps));
    if (a.rstd && t == 0) a.rstd[row] = r;
    E *out = a.out.p ? (E *)row_of<E>(a.out, row, a.K) : nullptr;
    const int pad = (a.D + kFp8Block - 1) / kFp8Block * kFp8Block;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int c = (t + i * TPR) * n;
        if (VPT > 4 && c < a.D) w[i] = *(const u32x4 *)((const E *)a.weight + c);
        float y[n], q[n];
        V::unpack(v[i], y);
        V::unpack(VPT > 4 && c >= a.D ? u32x4{0, 0, 0, 0} : w[i], q);
#pragma unroll
        for (int k = 0; k < n; ++k) y[k] = y[k] * r * q[k];
        if (out && c < a.D) *(u32x4 *)(out + c) = V::pack(y);
        if (!a.codes) continue;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < n; ++k) {
            if (c >= a.D) y[k] = 0.f;                  // 0 times a row that is not finite
            top = max(top, __float_as_uint(y[k]) & 0x7fffffffu);
        }
        const float scale = fp8_scale(fp8_top<V::lanes_log>(top));
        if (c >= pad) continue;
        uint32_t *to = (uint32_t *)(a.codes + (int64_t)row * pad + c);
        if constexpr (n == 8) *(uint2 *)to = uint2{fp8_pack(y[0], y[1], y[2], y[3], scale), fp8_pack(y[4], y[5], y[6], y[7], scale)};
        else *to = fp8_pack(y[0], y[1], y[2], y[3], scale);
        if (c % kFp8Block == 0) a.scales[(int64_t)row * (pad / kFp8Block) + c / kFp8Block] = scale;
    }
}

// Workgroups take rows in turn, and each leaves the sum of g h over its own: columns stay with their threads.  A row that does not fit the registers
// beside these sums is read a second time.  Bound by memory: 8192 rows of 2048 bfloat16 19.6 us, 5.1 TB/s.
template <class E, int TPR, int VPT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void head_norm_grad_kernel(NormGradArgs a)
{
    using V = Vec<E>;
    constexpr int n = V::n, R = TPR < 256 ? 256 / TPR : 1;      // rows of a workgroup at a time
    constexpr bool keep = VPT <= 4;
    __shared__ double sh[TPR / 64];
    __shared__ float joined[R > 1 ? R * VPT * TPR * n : 1];
    const int group = TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, t = threadIdx.x % TPR;
    float dw[VPT][n];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int k = 0; k < n; ++k) dw[i][k] = 0.f;
    u32x4 w[keep ? VPT : 1];
    if constexpr (keep) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) w[i] = (t + i * TPR) * n < a.D ? *(const u32x4 *)((const E *)a.weight + (t + i * TPR) * n) : u32x4{0, 0, 0, 0};
    }
    for (int row = blockIdx.x * R + group; row < a.N; row += gridDim.x * R) {
        const E *g = row_of<E>(a.grad_out, row, a.K), *s = row_of<E>(a.sum, row, a.K), *more = a.grad_sum.p ? row_of<E>(a.grad_sum, row, a.K) : nullptr;
        E *to = (E *)row_of<E>(a.grad_x, row, a.K);
        const float r = a.rstd[row];
        u32x4 gv[keep ? VPT : 1], sv[keep ? VPT : 1];
        auto fetch = [&](int i, float (&gf)[n], float (&h)[n], float (&u)[n], bool first) {
            const int c = (t + i * TPR) * n;
            const bool in = c < a.D;
            const u32x4 zero = {0, 0, 0, 0};
            if (first || !keep) {
                const u32x4 p = in ? *(const u32x4 *)(g + c) : zero, q = in ? *(const u32x4 *)(s + c) : zero;
                if constexpr (keep) { gv[i] = p; sv[i] = q; }
                else {
                    const u32x4 ww = in ? *(const u32x4 *)((const E *)a.weight + c) : zero;
                    V::unpack(p, gf); V::unpack(q, h); V::unpack(ww, u);
                }
            }
            if constexpr (keep) { V::unpack(gv[i], gf); V::unpack(sv[i], h); V::unpack(w[i], u); }
#pragma unroll
            for (int k = 0; k < n; ++k) { h[k] *= r; u[k] *= gf[k]; }
        };
        float gf[n], h[n], u[n];
        double dot = 0.0;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            fetch(i, gf, h, u, true);
            if (keep || (t + i * TPR) * n < a.D) {
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    dot = fma((double)u[k], (double)h[k], dot);
                    dw[i][k] = fmaf(gf[k], h[k], dw[i][k]);
                }
            }
        }
        const float mean = (float)(row_sum<TPR>(dot, sh) / a.D);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (t + i * TPR) * n;
            if (c >= a.D) continue;
            fetch(i, gf, h, u, false);
#pragma unroll
            for (int k = 0; k < n; ++k) u[k] = r * fmaf(-h[k], mean, u[k]);
            if (more) {
                V::unpack(*(const u32x4 *)(more + c), gf);
#pragma unroll
                for (int k = 0; k < n; ++k) u[k] += gf[k];
            }
            *(u32x4 *)(to + c) = V::pack(u);
        }
    }
    float *part = a.part + (int64_t)blockIdx.x * a.D;
    if constexpr (R > 1) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int k = 0; k < n; ++k) joined[(group * VPT + i) * TPR * n + t * n + k] = dw[i][k];
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += 256) {
            float v = 0.f;
#pragma unroll
            for (int q = 0; q < R; ++q) v += joined[q * VPT * TPR * n + c];
            part[c] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int k = 0; k < n; ++k)
                if ((t + i * TPR) * n < a.D) part[(t + i * TPR) * n + k] = dw[i][k];
    }
}

// The workgroups' sums added in their order: 32 columns a workgroup, eight lanes of four columns, a 128th of the partial sums for each such lanes.
template <class E>
__global__ __launch_bounds__(1024) void head_norm_weight_kernel(NormGradArgs a, int parts)
{
    __shared__ f32x4 sh[128][8];
    const int lane = threadIdx.x & 7, run = threadIdx.x >> 3, c = blockIdx.x * 32 + lane * 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int p = run; p < parts; p += 128) s += *(const f32x4 *)(a.part + (int64_t)p * a.D + c);
    sh[run][lane] = s;
    __syncthreads();
    for (int half = 64; half; half >>= 1) {
        if (run < half) sh[run][lane] += sh[run + half][lane];
        __syncthreads();
    }
    if (run) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) ((E *)a.grad_weight)[c + k] = (E)sh[0][lane][k];
}

template <class E, int TPR, int VPT> hipError_t norm_with(const NormArgs &a, hipStream_t st)
{
    head_norm_kernel<E, TPR, VPT><<<TPR == 64 ? up(a.N, 4) : a.N, TPR < 256 ? 256 : TPR, 0, st>>>(a);
    return hipGetLastError();
}

template <class E, int TPR, int VPT> hipError_t grad_with(const NormGradArgs &a, hipStream_t st)
{
    constexpr int R = TPR < 256 ? 256 / TPR : 1;
    const int64_t room = a.part_cap / a.D;
    int parts = up(a.N, R);
    if (parts > 2 * kCUs) parts = 2 * kCUs;
    if (parts > room) parts = (int)room;
    if (parts < 1) return hipErrorInvalidValue;
    head_norm_grad_kernel<E, TPR, VPT><<<parts, TPR < 256 ? 256 : TPR, 0, st>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    head_norm_weight_kernel<E><<<a.D / 32, 1024, 0, st>>>(a, parts);
    return hipGetLastError();
}

// Threads and vectors for a row of so many vectors: a wavefront a row while two vectors a lane hold it, above that all threads of a workgroup, as few vectors
// each as hold it.  Four vectors a lane of one wavefront (MORE) only where the columns' sums are kept through many rows, which wavefronts of their own
// do without a barrier.  us for rows of 256 vectors (2048 bfloat16), one wavefront / 256 threads: 64 rows 4.9 / 3.8, 1024 rows 7.1 / 6.1, 8192 rows
// 24.8 / 23.4; the gradient's 7.2 / 6.2, 10.0 / 11.2, 24.5 / 27.8.  128 vectors: 8192 rows 12.6 / 15.3.  512 vectors, 256 threads x 2 / 1024 x 1:
// 64 rows 4.3 / 4.5, 8192 rows 47.0 / 58.8.  1024 vectors, 256 x 4 / 1024 x 1: 64 rows 5.2 / 4.8, 1024 rows 13.5 / 14.2, 8192 rows 104 / 103.
template <template <class, int, int> class F, bool MORE, class E, class A> hipError_t by_length(const A &a, hipStream_t st)
{
    const int vecs = a.D / Vec<E>::n;
    if (vecs <= 64) return F<E, 64, 1>::launch(a, st);
    if (vecs <= 128) return F<E, 64, 2>::launch(a, st);
    if (vecs <= 256) return F<E, MORE ? 64 : 256, MORE ? 4 : 1>::launch(a, st);
    if (vecs <= 512) return F<E, 256, 2>::launch(a, st);
    if (vecs <= 1024) return F<E, 256, 4>::launch(a, st);
    if (vecs <= 2048) return F<E, 1024, 2>::launch(a, st);
    if constexpr (!MORE || sizeof(E) == 4)                     // the gradient's bfloat16 rows do not fit the registers by four
        if (vecs <= 4096) return F<E, 1024, 4>::launch(a, st);
    if constexpr (sizeof(E) == 2) return F<E, 1024, 8>::launch(a, st);          // a row has 65536 elements at most
    else return F<E, 1024, 16>::launch(a, st);
}
template <class E, int TPR, int VPT> struct Norm { static hipError_t launch(const NormArgs &a, hipStream_t st) { return norm_with<E, TPR, VPT>(a, st); } };
template <class E, int TPR, int VPT> struct NormGrad { static hipError_t launch(const NormGradArgs &a, hipStream_t st) { return grad_with<E, TPR, VPT>(a, st); } };

}  // namespace

hipError_t launch_head_norm(const NormArgs &a, int dtype, hipStream_t st)
{
    return dtype == TAPOUT_F32 ? by_length<Norm, false, float>(a, st) : by_length<Norm, false, __bf16>(a, st);
}
hipError_t launch_head_norm_grad(const NormGradArgs &a, int dtype, hipStream_t st)
{
    return dtype == TAPOUT_F32 ? by_length<NormGrad, true, float>(a, st) : by_length<NormGrad, true, __bf16>(a, st);
}

}  // namespace tapout
