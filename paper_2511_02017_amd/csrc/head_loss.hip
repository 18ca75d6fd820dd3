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

// Eight neighbouring results.
__device__ __forceinline__ void store8(float *to, f32x4 a, f32x4 b) { ((f32x4 *)to)[0] = a; ((f32x4 *)to)[1] = b; }
__device__ __forceinline__ void store8(__bf16 *to, f32x4 a, f32x4 b)
{
    *(bf16x8 *)to = bf16x8{(__bf16)a[0], (__bf16)a[1], (__bf16)a[2], (__bf16)a[3], (__bf16)b[0], (__bf16)b[1], (__bf16)b[2], (__bf16)b[3]};
}

__device__ __forceinline__ bool row_counts(int t, int V, const float *lse, const float *row_weight, int n)
{
    if (counted_target(t, V) < 0) return false;
    const float l = lse[n];
    return fabsf(l) < INFINITY && (!row_weight || row_weight[n] != 0.f);
}

// ---- forward -----------------------------------------------------------------------------------------
// Every wavefront leaves the maximum and sum of its own MI * 16 vocabulary rows for each of its tokens: 2 / (MI * 16) of the logits' bytes,
// joined by the next kernel.  Bound by the matrix unit from some 200 tokens on (V = 128256, dim = 2048, bfloat16: 512 rows 224 us, 1.20
// PFLOP/s; 8192 rows 3.14 ms, 1.37 PFLOP/s, where the clock gives way under the load and a library product of these sizes makes 1.41), by the
// weights' bytes below (32 rows 113 us, 4.6 TB/s).
template <class T>
__global__ __launch_bounds__(T::threads, T::per_simd) void head_loss_kernel(LossArgs a, int ni, int nj, int stages)
{
    extern __shared__ __align__(16) char lds[];
    if (blockIdx.x == 0 && a.flags)
        for (int b = threadIdx.x; b < a.B; b += T::threads) a.flags[b] = 0;
    int target[T::NJ];
    T::template work<0, true>(a.weight, a.hidden, Walk(ni, nj, 1), lds,
        [&](const Walk &t) { return Work{t.i() * T::TI, t.j() * T::TJ, 0, stages}; },
        [&](const Work &w) {
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                const int j = w.j0 + T::j_of(n);
                target[n] = j < a.N ? a.target[j] : -1;
            }
        },
        [&](const Work &w, typename T::Acc &acc) {
            const int left = a.V - w.i0;
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                const int j = w.j0 + T::j_of(n);
                if (left < T::TI) {
#pragma unroll
                    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (T::i_of(mi) + r >= left) acc[mi][n][r] = -INFINITY;
                }
                float m = -INFINITY;
#pragma unroll
                for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                    for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[mi][n][r]);
                m = fmaxf(m, __shfl_xor(m, 16));
                m = fmaxf(m, __shfl_xor(m, 32));
                const float ref = m == -INFINITY ? 0.f : m;
                float s = 0.f;
#pragma unroll
                for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f((acc[mi][n][r] - ref) * kLog2e);
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                if (j >= a.N) continue;
                if (T::lane() < 16) a.part[((int64_t)j * ni + w.i0 / T::TI) * T::WI + T::wave() / T::WJ] = float2{m, s};
                const int d = target[n] - w.i0;
                if (d >= 0 && d < min(left, T::TI)) {
#pragma unroll
                    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (d == T::i_of(mi) + r) a.target_logit[j] = acc[mi][n][r];
                }
            }
            return false;
        });
}

// A workgroup a row: the blocks' maxima and sums to lse, in double (bound by memory: 8192 rows of 1002 blocks 21 us, 3.1 TB/s).
__global__ __launch_bounds__(256) void head_loss_join_kernel(LossArgs a, int blocks)
{
    __shared__ float maxima[4];
    __shared__ double sums[4];
    const int n = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float2 *p = a.part + (int64_t)n * blocks;
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
    if (threadIdx.x) return;
    const double lse = (double)ref + log(((sums[0] + sums[1]) + sums[2]) + sums[3]);
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
// The loss's product once more, then e^(z - lse) and two stores of each g: rows of g as they are for dh, columns for dW.  The stores are what it
// takes longer for than the loss (8192 rows, V = 128256, dim = 2048: 3.95 ms against 3.14, matrix unit 55 % busy against 72 %).
template <class T, class E>
__global__ __launch_bounds__(T::threads, T::per_simd) void head_grad_kernel(GradArgs a, int ni, int nj, int stages, int n_pad, int N_pad)
{
    extern __shared__ __align__(16) char lds[];
    int target[T::NJ];                                        // -1: the row does not count
    float lse[T::NJ], weight[T::NJ];
    T::template work<0, true>(a.weight, a.hidden, Walk(ni, nj, 1), lds,
        [&](const Walk &t) { return Work{t.i() * T::TI, t.j() * T::TJ, 0, stages}; },
        [&](const Work &w) {
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                const int j = w.j0 + T::j_of(n);
                target[n] = j < a.N ? a.target[j] : -1;
                lse[n] = j < a.N ? a.lse[j] : 0.f;
                weight[n] = j < a.N && a.row_weight ? a.row_weight[j] : 1.f;
            }
        },
        [&](const Work &w, typename T::Acc &acc) {
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                const int j = w.j0 + T::j_of(n);
                const bool live = counted_target(target[n], a.V) >= 0 && fabsf(lse[n]) < INFINITY && weight[n] != 0.f;
                const int hot = target[n] - a.v0 - w.i0, end = live ? a.n - w.i0 : 0;
#pragma unroll
                for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = T::i_of(mi) + r;
                        const float p = __builtin_amdgcn_exp2f((acc[mi][n][r] - lse[n]) * kLog2e) - (i == hot ? 1.f : 0.f);
                        acc[mi][n][r] = i < end ? p * weight[n] : 0.f;
                    }
                // to nearest in the operands' type: the matrix instructions take both factors in one type
#pragma unroll
                for (int mi = 0; mi < T::MI; mi += 2)
                    if (j < a.N && w.i0 + T::i_of(mi) < n_pad) store8((E *)a.g + (int64_t)j * a.g_stride + w.i0 + T::i_of(mi), acc[mi][n], acc[mi + 1][n]);
            }
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = w.i0 + T::i_of(mi) + r, j = w.j0 + T::j_of(0);
                    if (i >= a.n || j >= N_pad) continue;
                    struct __align__(T::NJ * sizeof(E)) { E v[T::NJ]; } q;
#pragma unroll
                    for (int n = 0; n < T::NJ; ++n) q.v[n] = (E)acc[mi][n][r];
                    *(decltype(q) *)((E *)a.gt + (int64_t)i * a.gt_stride + j) = q;
                }
            return false;
        });
}

// 64 x 64 through LDS, 16 bytes a lane on either side (8192 x 2048 bfloat16: 17 us, 4.0 TB/s; two thirds of its LDS cycles are bank conflicts).
template <class E>
__global__ __launch_bounds__(256) void head_transpose_kernel(TransposeArgs a)
{
    constexpr int V16 = 16 / sizeof(E), S = 64, L = S + V16 / 2;
    __shared__ __align__(16) E tile[S * L];
    const int r0 = blockIdx.y * S, c0 = blockIdx.x * S;
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
// What a sum is multiplied by.  The mean over the rows that count, where none does, has an infinite factor: the sums, zeros, stay zeros.  The
// rows are looked through for that only where the factor is not finite.
__device__ __forceinline__ float sum_scale(const ProductArgs &a, float s)
{
    if (fabsf(s) < INFINITY) return s;
    for (int n0 = 0; n0 < a.rows; n0 += kWave) {
        const int n = n0 + (threadIdx.x & (kWave - 1));
        if (__any(n < a.rows && row_counts(a.target[n], a.V, a.lse, a.row_weight, n))) return s;
    }
    return 0.f;
}

// dh with the weights turned, its sums in binary32 over runs of the vocabulary; dW at once.  Bound by the matrix unit where rows are many
// (8192 rows, V = 128256, dim = 2048, bfloat16: dh 3.28 ms, 1.31 PFLOP/s, dW 2.83 ms, 1.52), by dW's stores where they are few (40 rows,
// 32000 x 1024 binary32: 45 us for 131 MB, 2.9 TB/s where a fill makes 6.8: a tile's two stages have its stores behind them, not beside).
// Partial sums of a later piece of the vocabulary are added block by block, a round trip each.
template <class T, class E>
__global__ __launch_bounds__(T::threads, T::per_simd) void head_product_kernel(ProductArgs a, int ni, int nj, int stages, int per_split, int splits)
{
    extern __shared__ __align__(16) char lds[];
    const float factor = T::turned || !a.scale ? 1.f : *a.scale;
    T::template work<0, false>(a.I, a.J, Walk(ni, nj, splits), lds,
        [&](const Walk &t) { return Work{t.i() * T::TI, t.j() * T::TJ, t.split * per_split, min(per_split, stages - t.split * per_split)}; },
        [&](const Work &) {},
        [&](const Work &w, typename T::Acc &acc) {
            const float scale = T::turned ? 1.f : sum_scale(a, factor);          // here: the first loads do not wait for the factor
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                const int j = w.j0 + T::j_of(n);
                if (j >= a.nj) continue;
                if constexpr (T::turned) {                        // partial sums
                    float *to = a.part + ((int64_t)(w.first / per_split) * a.nj + j) * a.ni + w.i0;
#pragma unroll
                    for (int mi = 0; mi < T::MI; ++mi) {
                        const int i = T::i_of(mi);
                        if (w.i0 + i < a.ni) *(f32x4 *)(to + i) = a.first ? acc[mi][n] : *(const f32x4 *)(to + i) + acc[mi][n];
                    }
                } else {
                    E *to = (E *)a.out + (int64_t)j * a.out_stride + w.i0;
#pragma unroll
                    for (int mi = 0; mi < T::MI; mi += 2) {
                        const int i = T::i_of(mi);
                        if (w.i0 + i < a.ni) store8(to + i, acc[mi][n] * scale, acc[mi + 1][n] * scale);
                    }
                }
            }
            return false;
        });
}

// The runs' sums added in their order, so that results do not change from call to call (8192 x 2048, one run: 26 us, 3.9 TB/s).
template <class E>
__global__ __launch_bounds__(256) void head_grad_hidden_kernel(GradHiddenArgs a)
{
    const RowColumn at((int64_t)blockIdx.x * 256, threadIdx.x, a.D / 4);
    const int n = at.r, d = at.c * 4;
    if (n >= a.N) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (row_counts(a.target[n], a.V, a.lse, a.row_weight, n)) {
        const float *p = a.part + (int64_t)n * a.D + d;
        const int64_t next = (int64_t)a.N * a.D;
        int k = 0;
        for (; k + 8 <= a.splits; k += 8) {                  // eight loads under way: with few rows this is a chain of round trips
            f32x4 v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = *(const f32x4 *)(p + (k + x) * next);
#pragma unroll
            for (int x = 0; x < 8; ++x) s += v[x];
        }
        for (; k < a.splits; ++k) s += *(const f32x4 *)(p + k * next);
        if (a.scale) s *= *a.scale;
    }
    E v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (E)s[r];
    E *to = (E *)a.out + (n / a.K) * a.stride_b + (n % a.K) * a.stride_k + d;
    if constexpr (sizeof(E) == 4) *(u32x4 *)to = *(const u32x4 *)v;
    else *(uint2 *)to = *(const uint2 *)v;
}

// Hidden states whose rows do not lie evenly, for loads that reach every row by one stride.
template <class E>
__global__ __launch_bounds__(256) void head_pack_kernel(PackArgs a)
{
    constexpr int V16 = 16 / sizeof(E);
    const RowColumn at((int64_t)blockIdx.x * 256, threadIdx.x, a.cols / V16);
    const int n = at.r, c = at.c * V16;
    if (n < a.N) *(u32x4 *)((E *)a.dst + (int64_t)n * a.cols + c) = *(const u32x4 *)((const E *)a.src + (n / a.K) * a.stride_b + (n % a.K) * a.stride_k + c);
}

template <class T> hipError_t loss_with(const LossArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int ni = up(a.V, T::TI), nj = up(a.N, T::TJ), stages = up(a.D, K::elems);
    if ((int64_t)a.N * ni * T::WI > a.part_cap) return hipErrorInvalidValue;
    hipError_t e = with_lds((const void *)head_loss_kernel<T>, T::ring_bytes, [&] {
        head_loss_kernel<T><<<grid_of<T>((int64_t)ni * nj), T::threads, T::ring_bytes, st>>>(a, ni, nj, stages);
    });
    if (e != hipSuccess) return e;
    head_loss_join_kernel<<<a.N, 256, 0, st>>>(a, ni * T::WI);
    return hipGetLastError();
}

template <class T, class E> hipError_t grad_with(const GradArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int n_pad = up(a.n, 64) * 64, N_pad = up(a.N, 32) * 32;
    const int ni = up(n_pad, T::TI), nj = up(N_pad, T::TJ), stages = up(a.D, K::elems);
    return with_lds((const void *)head_grad_kernel<T, E>, T::ring_bytes, [&] {
        head_grad_kernel<T, E><<<grid_of<T>((int64_t)ni * nj), T::threads, T::ring_bytes, st>>>(a, ni, nj, stages, n_pad, N_pad);
    });
}

template <class T, class E> hipError_t product_with(const ProductArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int ni = up(a.ni, T::TI), nj = up(a.nj, T::TJ), stages = up(a.k, K::elems);
    const int per_split = up(stages, a.splits), splits = up(stages, per_split);
    return with_lds((const void *)head_product_kernel<T, E>, T::ring_bytes, [&] {
        head_product_kernel<T, E><<<grid_of<T>((int64_t)ni * nj * splits), T::threads, T::ring_bytes, st>>>(a, ni, nj, stages,
                                                                                             per_split, splits);
    });
}

template <int KIND, bool TURNED = false> using Small = Tile<KIND, 128, 32, 4, 1, TURNED>;
template <int KIND, bool TURNED = false> using Mid = Tile<KIND, 128, 128, 2, 2, TURNED>;
template <int KIND, bool TURNED = false> using Large = Tile<KIND, 256, 256, 2, 4, TURNED>;

// Which tile for how many tokens.  A tile of 32 tokens while more would be empty, of 128 while the vocabulary rows' bytes are what
// takes the time anyway, else of 256, whose loads serve more products (cross entropy of V = 128256, dim = 2048, bfloat16, us with
// tiles of 32 / 128 / 256 tokens: 32 rows 113 / 116 / 125, 48 rows 122 / 117 / 125, 128 rows 188 / 117 / 126, 192 rows 244 / 165 / 129,
// 512 rows 560 / 328 / 220).
// binary32: products as they are while the tile is nearly empty, three bfloat16 each where the matrix unit sets the pace (V = 32000,
// dim = 1024, us with 32 native / 128 native / 128 split: 33 rows 44 / 81 / 65, 64 rows 45 / 81 / 65, 128 rows 82 / 85 / 72, 256 rows
// 159 / 148 / 103, 1000 rows - / 527 / 385, 3000 rows - / 1561 / 1046, which is 188 TFLOP/s of binary32).  By tokens alone: with a vocabulary
// shorter than these the largest tile leaves units empty.
template <template <class> class F, bool TURNED, class A> hipError_t by_tokens(A &&a, int tokens, int dtype, hipStream_t st)
{
    if (dtype == TAPOUT_F32) return tokens <= 64 ? F<Small<kTileF32, TURNED>>::launch(a, st) : F<Mid<kTileF32x3, TURNED>>::launch(a, st);
    return tokens <= 32 ? F<Small<kTileBf16, TURNED>>::launch(a, st)
         : tokens <= 128 ? F<Mid<kTileBf16, TURNED>>::launch(a, st) : F<Large<kTileBf16, TURNED>>::launch(a, st);
}

template <class T> struct Loss { static hipError_t launch(const LossArgs &a, hipStream_t st) { return loss_with<T>(a, st); } };
template <class T> struct Grad { static hipError_t launch(const GradArgs &a, hipStream_t st) { return grad_with<T, typename ElemOf<T::esz == 4 ? TAPOUT_F32 : TAPOUT_BF16>::T>(a, st); } };
template <class T> struct Product { static hipError_t launch(const ProductArgs &a, hipStream_t st) { return product_with<T, typename ElemOf<T::esz == 4 ? TAPOUT_F32 : TAPOUT_BF16>::T>(a, st); } };

}  // namespace

hipError_t launch_head_loss(const LossArgs &a, int dtype, hipStream_t st) { return by_tokens<Loss, false>(a, a.N, dtype, st); }
hipError_t launch_head_grad(const GradArgs &a, int dtype, hipStream_t st) { return by_tokens<Grad, false>(a, a.N, dtype, st); }
hipError_t launch_head_product(const ProductArgs &a, int dtype, hipStream_t st) { return a.part ? by_tokens<Product, true>(a, a.nj, dtype, st) : by_tokens<Product, false>(a, a.nj, dtype, st); }

template <class T> struct Slots { static hipError_t launch(int *out, hipStream_t) { *out = kCUs * T::per_cu; return hipSuccess; } };
template <class T> struct Sizes { static hipError_t launch(int *out, hipStream_t) { out[0] = T::TI; out[1] = T::TJ; return hipSuccess; } };
int head_product_slots(int nj, int dtype)
{
    int slots = 0;
    (void)by_tokens<Slots, true>(&slots, nj, dtype, nullptr);
    return slots;
}
int head_product_tiles(int ni, int nj, int dtype)
{
    int size[2] = {1, 1};
    (void)by_tokens<Sizes, true>(size, nj, dtype, nullptr);
    return up(ni, size[0]) * up(nj, size[1]);
}

hipError_t launch_head_transpose(const TransposeArgs &a, int dtype, hipStream_t st)
{
    const dim3 grid(up(a.cols, 64), up(a.rows_pad, 64));             // cols: up to 2^24, more than a grid's second axis holds
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
    const int64_t grid = ((int64_t)a.N * (a.cols / (dtype == TAPOUT_F32 ? 4 : 8)) + 255) / 256;
    if (dtype == TAPOUT_F32) head_pack_kernel<float><<<grid, 256, 0, st>>>(a);
    else head_pack_kernel<__bf16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace tapout
