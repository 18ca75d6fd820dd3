// Cross entropy of the draft head's softmax over the whole vocabulary and its gradient.
//
//   z = h W^T,  lse = ln sum_v e^(z_v),  loss = lse - z_t
//   g = row_weight (e^(z - lse) - [v = t]),  dh = scale g W,  dW = scale g^T h
//
// The logits are never kept: the forward pass leaves a maximum and a sum for each tile of the vocabulary, and the backward
// pass forms the logits of one piece of the vocabulary again, turns them into g in the matrix instructions' accumulators and
// writes g, rounded to the operands' type, in both orientations, so that both products that follow read their operands along k.
#include "head.h"

namespace tapout {
namespace {

template <int DT> struct ElemOf { using T = float; };
template <> struct ElemOf<TAPOUT_BF16> { using T = __bf16; };

__device__ __forceinline__ bool row_counts(int t, int V, const float *lse, const float *row_weight, int n)
{
    if (counted_target(t, V) < 0) return false;
    const float l = lse[n];
    return fabsf(l) < INFINITY && (!row_weight || row_weight[n] != 0.f);
}

// ---- forward -----------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(T::threads) void head_loss_kernel(LossArgs a, int ni, int nj, int stages, int last_steps)
{
    extern __shared__ __align__(16) char lds[];
    const TileAt at = tile_at(blockIdx.x, ni, nj, 8);
    const int i0 = at.i * T::TI, j0 = at.j * T::TJ;
    if (blockIdx.x == 0 && a.flags)
        for (int b = threadIdx.x; b < a.B; b += T::threads) a.flags[b] = 0;
    typename T::Acc acc;
    T::run(a.weight, a.hidden, i0, j0, 0, stages, stages, last_steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / T::WJ, wj = wave % T::WJ;
    const int r16 = lane & 15, g = lane >> 4;
    const int iw = i0 + wi * T::MI * 16 + 4 * g, jw = wj * T::NJ * 16 + r16;
    float2 *red = (float2 *)lds;                       // [WI][TJ]
#pragma unroll
    for (int nj = 0; nj < T::NJ; ++nj) {
        const int j = j0 + jw + nj * 16;
        float m = -INFINITY;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (iw + mi * 16 + r < a.V) m = fmaxf(m, acc[mi][nj][r]);
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        const float ref = m == -INFINITY ? 0.f : m;
        float s = 0.f;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (iw + mi * 16 + r < a.V) s += __builtin_amdgcn_exp2f((acc[mi][nj][r] - ref) * kLog2e);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (g == 0) red[wi * T::TJ + jw + nj * 16] = float2{m, s};
        const int t = j < a.N ? a.target[j] : -1;
        if (t >= 0 && t < a.V) {
            const int d = t - iw;
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (d == mi * 16 + r) a.target_logit[j] = acc[mi][nj][r];
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < T::TJ; x += T::threads) {
        if (j0 + x >= a.N) continue;
        float m = -INFINITY, s = 0.f;
#pragma unroll
        for (int w = 0; w < T::WI; ++w) m = fmaxf(m, red[w * T::TJ + x].x);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < T::WI; ++w) {
            const float2 p = red[w * T::TJ + x];
            s += p.y * __builtin_amdgcn_exp2f(((p.x == -INFINITY ? 0.f : p.x) - ref) * kLog2e);
        }
        a.part[(int64_t)(j0 + x) * ni + at.i] = float2{m, s};
    }
}

// A wavefront a row: the tiles' maxima and sums to lse, in double.
__global__ __launch_bounds__(256) void head_loss_join_kernel(LossArgs a, int ni)
{
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (n >= a.N) return;
    const float2 *p = a.part + (int64_t)n * ni;
    float m = -INFINITY;
    for (int x = lane; x < ni; x += 64) m = fmaxf(m, p[x].x);
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float ref = m == -INFINITY ? 0.f : m;
    double s = 0.0;
    for (int x = lane; x < ni; x += 64) {
        const float2 q = p[x];
        s += (double)q.y * (double)__builtin_amdgcn_exp2f(((q.x == -INFINITY ? 0.f : q.x) - ref) * kLog2e);
    }
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane) return;
    const double lse = (double)ref + log(s);
    const int t = counted_target(a.target[n], a.V);
    const bool bad = !(fabs(lse) < (double)INFINITY);
    const float nan = __uint_as_float(0x7fc00000u);
    a.lse[n] = bad ? nan : (float)lse;
    a.loss[n] = t == -1 ? 0.f : t == -2 || bad ? nan : (float)(lse - (double)a.target_logit[n]);
    if (a.flags) {
        const uint32_t f = (t != -1 && bad ? TAPOUT_FLAG_BAD_ROW : 0u) | (t == -2 ? TAPOUT_FLAG_BAD_TOKEN : 0u);
        if (f) atomicOr(&a.flags[n / a.rows_per_seq], f);
    }
}

// ---- gradient by the logits of one piece ---------------------------------------------------------------
template <class T, class E>
__global__ __launch_bounds__(T::threads) void head_grad_kernel(GradArgs a, int ni, int nj, int stages, int last_steps, int n_pad, int N_pad)
{
    extern __shared__ __align__(16) char lds[];
    constexpr int V16 = 16 / sizeof(E), LI = T::TI + V16, LJ = T::TJ + V16;      // row lengths of the two tiles in LDS
    const TileAt at = tile_at(blockIdx.x, ni, nj, 8);
    const int i0 = at.i * T::TI, j0 = at.j * T::TJ;
    typename T::Acc acc;
    T::run(a.weight, a.hidden, i0, j0, 0, stages, stages, last_steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / T::WJ, wj = wave % T::WJ;
    const int r16 = lane & 15, g = lane >> 4;
    const int il = wi * T::MI * 16 + 4 * g, jl = wj * T::NJ * 16 + r16;
    E *tile = (E *)lds;
#pragma unroll
    for (int nj = 0; nj < T::NJ; ++nj) {
        const int j = j0 + jl + nj * 16;
        const int t = j < a.N ? a.target[j] : -1;
        const bool live = j < a.N && row_counts(t, a.V, a.lse, a.row_weight, j);
        const float lse = live ? a.lse[j] : 0.f, w = live && a.row_weight ? a.row_weight[j] : 1.f;
        const int d = t - a.v0 - i0 - il;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            E v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float p = __builtin_amdgcn_exp2f((acc[mi][nj][r] - lse) * kLog2e);
                p = (p - (d == mi * 16 + r ? 1.f : 0.f)) * w;
                p = live && i0 + il + mi * 16 + r < a.n ? p : 0.f;
                v[r] = (E)p;                              // to nearest: the matrix instructions take operands of one type
                acc[mi][nj][r] = p;
            }
            E *to = tile + (jl + nj * 16) * LI + il + mi * 16;
            to[0] = v[0]; to[1] = v[1]; to[2] = v[2]; to[3] = v[3];
        }
    }
    __syncthreads();
    constexpr int CI = T::TI / V16, CJ = T::TJ / V16;
    for (int x = threadIdx.x; x < T::TJ * CI; x += T::threads) {
        const int jr = x / CI, c = x % CI * V16;
        if (j0 + jr < a.N && i0 + c < n_pad) *(u32x4 *)((E *)a.g + (int64_t)(j0 + jr) * a.g_stride + i0 + c) = *(const u32x4 *)(tile + jr * LI + c);
    }
    __syncthreads();
#pragma unroll
    for (int nj = 0; nj < T::NJ; ++nj)
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int r = 0; r < 4; ++r) tile[(il + mi * 16 + r) * LJ + jl + nj * 16] = (E)acc[mi][nj][r];
    __syncthreads();
    for (int x = threadIdx.x; x < T::TI * CJ; x += T::threads) {
        const int ir = x / CJ, c = x % CJ * V16;
        if (i0 + ir < a.n && j0 + c < N_pad) *(u32x4 *)((E *)a.gt + (int64_t)(i0 + ir) * a.gt_stride + j0 + c) = *(const u32x4 *)(tile + ir * LJ + c);
    }
}

template <class E>
__global__ __launch_bounds__(256) void head_transpose_kernel(TransposeArgs a)
{
    constexpr int V16 = 16 / sizeof(E), S = 64, L = S + V16 / 2;
    __shared__ __align__(16) E tile[S * L];
    const int r0 = blockIdx.x * S, c0 = blockIdx.y * S;
    for (int x = threadIdx.x; x < S * (S / V16); x += 256) {
        const int r = x / (S / V16), c = x % (S / V16) * V16;
        E v[V16];
#pragma unroll
        for (int n = 0; n < V16; ++n) v[n] = (E)0.f;
        bool in = r0 + r < a.rows && c0 + c < a.cols;
        if (in && a.target) in = row_counts(a.target[r0 + r], a.V, a.lse, a.row_weight, r0 + r);
        if (in) *(u32x4 *)v = *(const u32x4 *)((const E *)a.src + (int64_t)(r0 + r) * a.src_stride + c0 + c);
#pragma unroll
        for (int n = 0; n < V16; ++n) tile[(c + n) * L + r] = v[n];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < S * (S / V16); x += 256) {
        const int c = x / (S / V16), r = x % (S / V16) * V16;
        if (c0 + c >= a.cols || r0 + r >= a.rows_pad) continue;
        E v[V16];
#pragma unroll
        for (int n = 0; n < V16; ++n) v[n] = tile[c * L + r + n];
        *(u32x4 *)((E *)a.dst + (int64_t)(c0 + c) * a.dst_stride + r0 + r) = *(const u32x4 *)v;
    }
}

// ---- products of the gradient ---------------------------------------------------------------------------
template <class T, class E>
__global__ __launch_bounds__(T::threads) void head_product_kernel(ProductArgs a, int ni, int nj, int stages, int last_steps, int per_split)
{
    extern __shared__ __align__(16) char lds[];
    const TileAt at = tile_at(blockIdx.x, ni, nj, 8);
    const int i0 = at.i * T::TI, j0 = at.j * T::TJ, split = blockIdx.y;
    const int first = split * per_split, n = max(0, min(per_split, stages - first));
    typename T::Acc acc;
    T::run(a.I, a.J, i0, j0, first, n, stages, last_steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / T::WJ, wj = wave % T::WJ;
    const int iw = i0 + wi * T::MI * 16 + 4 * (lane >> 4), jw = j0 + wj * T::NJ * 16 + (lane & 15);
    const float scale = a.part || !a.scale ? 1.f : *a.scale;
#pragma unroll
    for (int nj = 0; nj < T::NJ; ++nj) {
        const int j = jw + nj * 16;
        if (j >= a.nj) continue;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            const int i = iw + mi * 16;
            if (i >= a.ni) continue;
            if (a.part) {
                f32x4 *to = (f32x4 *)(a.part + ((int64_t)split * a.nj + j) * a.ni + i);
                *to = a.first ? acc[mi][nj] : *to + acc[mi][nj];
            } else {
                E v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = (E)(acc[mi][nj][r] * scale);
                E *to = (E *)a.out + (int64_t)j * a.out_stride + i;
                if constexpr (sizeof(E) == 4) *(u32x4 *)to = *(const u32x4 *)v;
                else *(uint2 *)to = *(const uint2 *)v;
            }
        }
    }
}

template <class E>
__global__ __launch_bounds__(256) void head_grad_hidden_kernel(GradHiddenArgs a)
{
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per = a.D / 4;
    const int n = (int)(x / per), d = (int)(x % per) * 4;
    if (n >= a.N) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (row_counts(a.target[n], a.V, a.lse, a.row_weight, n)) {
        for (int k = 0; k < a.splits; ++k) s += *(const f32x4 *)(a.part + ((int64_t)k * a.N + n) * a.D + d);
        if (a.scale) s *= *a.scale;
    }
    E v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (E)s[r];
    E *to = (E *)a.out + (n / a.K) * a.stride_b + (n % a.K) * a.stride_k + d;
    if constexpr (sizeof(E) == 4) *(u32x4 *)to = *(const u32x4 *)v;
    else *(uint2 *)to = *(const uint2 *)v;
}

template <class E>
__global__ __launch_bounds__(256) void head_pack_kernel(PackArgs a)
{
    constexpr int V16 = 16 / sizeof(E);
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per = a.cols_pad / V16;
    const int n = (int)(x / per), c = (int)(x % per) * V16;
    if (n >= a.N) return;
    u32x4 v = {0, 0, 0, 0};
    if (c < a.cols) v = *(const u32x4 *)((const E *)a.src + (n / a.K) * a.stride_b + (n % a.K) * a.stride_k + c);
    *(u32x4 *)((E *)a.dst + (int64_t)n * a.cols_pad + c) = v;
}

template <class T, class F> hipError_t with_lds(const void *kernel, int bytes, F launch)
{
    if (bytes > 65536) {
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    launch();
    return hipGetLastError();
}

inline int up(int a, int b) { return (a + b - 1) / b; }

template <class T> hipError_t loss_with(const LossArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int ni = up(a.V, T::TI), nj = up(a.N, T::TJ), steps = a.D / K::step_elems, stages = up(steps, K::steps);
    hipError_t e = with_lds<T>((const void *)head_loss_kernel<T>, T::lds_bytes, [&] {
        head_loss_kernel<T><<<ni * nj, T::threads, T::lds_bytes, st>>>(a, ni, nj, stages, steps - (stages - 1) * K::steps);
    });
    if (e != hipSuccess) return e;
    head_loss_join_kernel<<<up(a.N, 4), 256, 0, st>>>(a, ni);
    return hipGetLastError();
}

template <class T, class E> hipError_t grad_with(const GradArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    constexpr int V16 = 16 / sizeof(E);
    constexpr int t1 = T::TJ * (T::TI + V16) * (int)sizeof(E), t2 = T::TI * (T::TJ + V16) * (int)sizeof(E), tiles = t1 > t2 ? t1 : t2;
    constexpr int lds = T::lds_bytes > tiles ? T::lds_bytes : tiles;
    const int n_pad = up(a.n, 64) * 64, N_pad = up(a.N, 32) * 32;
    const int ni = up(n_pad, T::TI), nj = up(N_pad, T::TJ), steps = a.D / K::step_elems, stages = up(steps, K::steps);
    return with_lds<T>((const void *)head_grad_kernel<T, E>, lds, [&] {
        head_grad_kernel<T, E><<<ni * nj, T::threads, lds, st>>>(a, ni, nj, stages, steps - (stages - 1) * K::steps, n_pad, N_pad);
    });
}

template <class T, class E> hipError_t product_with(const ProductArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int ni = up(a.ni, T::TI), nj = up(a.nj, T::TJ), steps = a.k / K::step_elems, stages = up(steps, K::steps);
    return with_lds<T>((const void *)head_product_kernel<T, E>, T::lds_bytes, [&] {
        head_product_kernel<T, E><<<dim3(ni * nj, a.splits), T::threads, T::lds_bytes, st>>>(a, ni, nj, stages, steps - (stages - 1) * K::steps,
                                                                                             up(stages, a.splits));
    });
}

template <int KIND> using Small = Tile<KIND, 128, 32, 4, 1>;
template <int KIND> using Mid = Tile<KIND, 128, 128, 2, 2>;
#ifndef LARGE
#define LARGE 256, 256, 2, 4
#endif
template <int KIND> using Large = Tile<KIND, LARGE>;

}  // namespace

hipError_t launch_head_loss(const LossArgs &a, int dtype, hipStream_t st)
{
    if (dtype == TAPOUT_F32) return a.N <= 32 ? loss_with<Small<kTileF32>>(a, st) : loss_with<Mid<kTileF32>>(a, st);
    return a.N <= 32 ? loss_with<Small<kTileBf16>>(a, st) : a.N <= 256 ? loss_with<Mid<kTileBf16>>(a, st) : loss_with<Large<kTileBf16>>(a, st);
}

hipError_t launch_head_grad(const GradArgs &a, int dtype, hipStream_t st)
{
    if (dtype == TAPOUT_F32) return a.N <= 32 ? grad_with<Small<kTileF32>, float>(a, st) : grad_with<Mid<kTileF32>, float>(a, st);
    return a.N <= 32 ? grad_with<Small<kTileBf16>, __bf16>(a, st)
         : a.N <= 256 ? grad_with<Mid<kTileBf16>, __bf16>(a, st) : grad_with<Large<kTileBf16>, __bf16>(a, st);
}

int head_product_tiles(int ni, int nj, int dtype)
{
    if (nj <= 32) return up(ni, 128) * up(nj, 32);
    if (nj <= 256 || dtype == TAPOUT_F32) return up(ni, 128) * up(nj, 128);
    return up(ni, 256) * up(nj, 256);
}

hipError_t launch_head_product(const ProductArgs &a, int dtype, hipStream_t st)
{
    if (dtype == TAPOUT_F32) return a.nj <= 32 ? product_with<Small<kTileF32>, float>(a, st) : product_with<Mid<kTileF32>, float>(a, st);
    return a.nj <= 32 ? product_with<Small<kTileBf16>, __bf16>(a, st)
         : a.nj <= 256 ? product_with<Mid<kTileBf16>, __bf16>(a, st) : product_with<Large<kTileBf16>, __bf16>(a, st);
}

hipError_t launch_head_transpose(const TransposeArgs &a, int dtype, hipStream_t st)
{
    const dim3 grid(up(a.rows_pad, 64), up(a.cols, 64));
    if (dtype == TAPOUT_F32) head_transpose_kernel<float><<<grid, 256, 0, st>>>(a);
    else head_transpose_kernel<__bf16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_head_grad_hidden(const GradHiddenArgs &a, int dtype, hipStream_t st)
{
    const int64_t grid = ((int64_t)a.N * (a.D / 4) + 255) / 256;
    if (dtype == TAPOUT_F32) head_grad_hidden_kernel<float><<<grid, 256, 0, st>>>(a);
    else head_grad_hidden_kernel<__bf16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_head_pack(const PackArgs &a, int dtype, hipStream_t st)
{
    const int64_t grid = ((int64_t)a.N * (a.cols_pad / (dtype == TAPOUT_F32 ? 4 : 8)) + 255) / 256;
    if (dtype == TAPOUT_F32) head_pack_kernel<float><<<grid, 256, 0, st>>>(a);
    else head_pack_kernel<__bf16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace tapout
