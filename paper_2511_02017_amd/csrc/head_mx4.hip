// Microscaled 4-bit floating point for the draft head: quantisation, its inverse, and the logits of a head held that way.
//
// A block of 32 neighbouring elements of a row shares a scale 2^e, e = floor(log2 max|x|) - 2, held as the byte e + 127; an
// element is x / 2^e rounded to {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign (to nearest, ties to the even code, 6 from 5 on).
#include "head.h"

namespace tapout {
namespace {

inline int up(int a, int b) { return (a + b - 1) / b; }

__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
    for (int n = 0; n < 4; ++n) { x[n] = a[n]; x[n + 4] = b[n]; }
}
__device__ __forceinline__ void load8(const __bf16 *p, float (&x)[8])
{
    const u32x4 a = *(const u32x4 *)p;
#pragma unroll
    for (int n = 0; n < 4; ++n) { x[2 * n] = __uint_as_float(a[n] << 16); x[2 * n + 1] = __uint_as_float(a[n] & 0xffff0000u); }
}

// Eight elements a lane, four lanes a block.
template <class E>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(QuantArgs a, int per)      // per: groups of eight in a padded row
{
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int r = (int)(x / per), c = (int)(x % per);
    if (r >= a.rows) return;                           // whole blocks: per is a multiple of 4
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c * 8 < a.cols) load8((const E *)a.src + (r / a.K) * a.stride_b + (r % a.K) * a.stride_k + c * 8, v);
    uint32_t top = 0;                                  // of the magnitudes' bits, which order like the magnitudes; NaN on top
#pragma unroll
    for (int n = 0; n < 8; ++n) top = max(top, __float_as_uint(v[n]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const uint32_t e = top >> 23, byte = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
    const float inv = __uint_as_float((254u - min(byte, 252u)) << 23);                // 2^(127 - byte): the products are exact
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * inv, v[1] * inv, 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * inv, v[3] * inv, 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * inv, v[5] * inv, 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * inv, v[7] * inv, 1.f, 3);
    ((uint32_t *)a.codes)[x] = w;
    if ((c & 3) == 0) a.scales[x >> 2] = (uint8_t)byte;
}

template <class E>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(DequantArgs a, int per)
{
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int r = (int)(x / per), c = (int)(x % per);
    if (r >= a.rows || c * 8 >= a.cols) return;
    const uint32_t w = ((const uint32_t *)a.codes)[x];
    const float scale = scale_value(a.scales[x >> 2]);
    const u32x4 h = codes_to_bf16(w, scale);
    E *to = (E *)a.out + (int64_t)r * a.stride + c * 8;
    if constexpr (sizeof(E) == 2) *(u32x4 *)to = h;
    else {
        *(u32x4 *)to = u32x4{h[0] << 16, h[0] & 0xffff0000u, h[1] << 16, h[1] & 0xffff0000u};
        *(u32x4 *)(to + 4) = u32x4{h[2] << 16, h[2] & 0xffff0000u, h[3] << 16, h[3] & 0xffff0000u};
    }
}

// ---- logits -----------------------------------------------------------------------------------------------
template <class T, class E>
__global__ __launch_bounds__(T::threads) void head_logits_kernel(LogitsArgs a, int ni, int nj, int stages, int last_steps)
{
    extern __shared__ __align__(16) char lds[];
    const TileAt at = tile_at(blockIdx.x, ni, nj, 8);
    const int i0 = at.i * T::TI, j0 = at.j * T::TJ;
    typename T::Acc acc;
    T::run(a.weight, a.hidden, i0, j0, 0, stages, stages, last_steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / T::WJ, wj = wave % T::WJ;
    const int il = wi * T::MI * 16 + 4 * (lane >> 4), jl = wj * T::NJ * 16 + (lane & 15);
    auto row_of = [&](int j) -> E * {                  // NULL: not written
        if (j >= a.N) return nullptr;
        const int b = j / a.K, k = j % a.K;
        if (a.k_len && k >= a.k_len[b]) return nullptr;
        return (E *)a.out + b * a.stride_b + k * a.stride_k;
    };
    if constexpr (sizeof(E) == 4) {
        // four neighbours a lane
#pragma unroll
        for (int nj = 0; nj < T::NJ; ++nj) {
            E *row = row_of(j0 + jl + nj * 16);
            if (!row) continue;
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const int i = i0 + il + mi * 16;
                if (i + 4 <= a.V && ((uintptr_t)(row + i) & 15) == 0) *(f32x4 *)(row + i) = acc[mi][nj];
                else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i + r < a.V) row[i + r] = acc[mi][nj][r];
                }
            }
        }
    } else {
        // through LDS, so that a row of the tile leaves in whole 16-byte pieces; where the row starts between them, the pieces
        // are taken from LDS element by element
        constexpr int L = T::TI + 8, C = T::TI / 8 + 1;
        E *tile = (E *)lds;
#pragma unroll
        for (int nj = 0; nj < T::NJ; ++nj)
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const bf16x4 v = {(__bf16)acc[mi][nj][0], (__bf16)acc[mi][nj][1], (__bf16)acc[mi][nj][2], (__bf16)acc[mi][nj][3]};
                *(uint2 *)(tile + (jl + nj * 16) * L + il + mi * 16) = __builtin_bit_cast(uint2, v);
            }
        __syncthreads();
        const int n = min(T::TI, a.V - i0);
        for (int x = threadIdx.x; x < T::TJ * C; x += T::threads) {
            const int jr = x / C;
            E *row = row_of(j0 + jr);
            if (!row) continue;
            E *to = row + i0;
            const int mis = (int)(((uintptr_t)to >> 1) & 7), e = (x % C) * 8 - mis;
            const E *from = tile + jr * L;
            if (e >= 0 && e + 8 <= n) {
                u32x4 v;
                if (mis == 0) v = *(const u32x4 *)(from + e);
                else {
                    const uint16_t *h = (const uint16_t *)from + e;
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = (uint32_t)h[2 * q] | (uint32_t)h[2 * q + 1] << 16;
                }
                *(u32x4 *)(to + e) = v;
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (e + q >= 0 && e + q < n) to[e + q] = from[e + q];
            }
        }
    }
}

template <class T, class E> hipError_t logits_with(const LogitsArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    constexpr int tile = sizeof(E) == 2 ? T::TJ * (T::TI + 8) * 2 : 0, lds = T::lds_bytes > tile ? T::lds_bytes : tile;
    const int ni = up(a.V, T::TI), nj = up(a.N, T::TJ), steps = a.D / K::step_elems, stages = up(steps, K::steps);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void *)head_logits_kernel<T, E>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    head_logits_kernel<T, E><<<ni * nj, T::threads, lds, st>>>(a, ni, nj, stages, steps - (stages - 1) * K::steps);
    return hipGetLastError();
}

template <class E> hipError_t logits_of(const LogitsArgs &a, int kind, hipStream_t st)
{
    if (kind == kTileMx4)
        return a.N <= 32 ? logits_with<Tile<kTileMx4, 128, 32, 4, 1>, E>(a, st)
             : logits_with<Tile<kTileMx4, 128, 128, 2, 2>, E>(a, st);
    return a.N <= 32 ? logits_with<Tile<kTileMx4W, 128, 32, 4, 1>, E>(a, st)
         : a.N <= 64 ? logits_with<Tile<kTileMx4W, 128, 64, 4, 1>, E>(a, st) : logits_with<Tile<kTileMx4W, 128, 128, 2, 2>, E>(a, st);
}

}  // namespace

hipError_t launch_mx4_quantize(const QuantArgs &a, int dtype, hipStream_t st)
{
    const int per = (a.cols + kMx4Pad - 1) / kMx4Pad * kMx4Pad / 8;
    const int64_t grid = ((int64_t)a.rows * per + 255) / 256;
    if (dtype == TAPOUT_F32) mx4_quantize_kernel<float><<<grid, 256, 0, st>>>(a, per);
    else mx4_quantize_kernel<__bf16><<<grid, 256, 0, st>>>(a, per);
    return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const DequantArgs &a, int dtype, hipStream_t st)
{
    const int per = (a.cols + kMx4Pad - 1) / kMx4Pad * kMx4Pad / 8;
    const int64_t grid = ((int64_t)a.rows * per + 255) / 256;
    if (dtype == TAPOUT_F32) mx4_dequantize_kernel<float><<<grid, 256, 0, st>>>(a, per);
    else mx4_dequantize_kernel<__bf16><<<grid, 256, 0, st>>>(a, per);
    return hipGetLastError();
}

hipError_t launch_head_logits(const LogitsArgs &a, int kind, int dtype_out, hipStream_t st)
{
    return dtype_out == TAPOUT_F32 ? logits_of<float>(a, kind, st) : logits_of<__bf16>(a, kind, st);
}

}  // namespace tapout
