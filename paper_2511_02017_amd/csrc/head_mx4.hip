// Microscaled 4-bit floating point for the draft head: quantisation, its inverse, and the logits of a head held that way.
//
// A block of 32 neighbouring elements of a row shares a scale 2^e, e = floor(log2 max|x|) - 2, held as the byte e + 127; an
// element is x / 2^e rounded to {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign (to nearest, ties to the even code, 6 from 5 on).
#include "head.h"

namespace tapout {
namespace {

// Values are read and written once, past the caches' idea of what is used again (128256 x 2048 bfloat16, us with ordinary / nontemporal
// accesses: to 4 bits 144 / 110, back 124 / 90; binary32 50257 x 1120 to 4 bits 60 / 49).
__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const f32x4 a = __builtin_nontemporal_load((const f32x4 *)p), b = __builtin_nontemporal_load((const f32x4 *)(p + 4));
#pragma unroll
    for (int n = 0; n < 4; ++n) { x[n] = a[n]; x[n + 4] = b[n]; }
}
__device__ __forceinline__ void load8(const __bf16 *p, float (&x)[8])
{
    const u32x4 a = __builtin_nontemporal_load((const u32x4 *)p);
#pragma unroll
    for (int n = 0; n < 4; ++n) { x[2 * n] = __uint_as_float(a[n] << 16); x[2 * n + 1] = __uint_as_float(a[n] & 0xffff0000u); }
}

// The largest of four neighbouring lanes' values, in every one of them.
__device__ __forceinline__ uint32_t max_of_four(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));      // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));   // lanes 2 3 0 1
}

// Eight elements a lane, four lanes a block; U such groups, all requested first.  Bound by memory (128256 x 2048 bfloat16: 110 us, 6.0 TB/s).
template <class E, int U>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(QuantArgs a, int per, int64_t groups)      // per: groups of eight in a padded row
{
    const int64_t base = (int64_t)blockIdx.x * (256 * U);
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const RowColumn at(base, threadIdx.x + u * 256, per);
#pragma unroll
        for (int n = 0; n < 8; ++n) v[u][n] = 0.f;
        if (base + threadIdx.x + u * 256 < groups && at.c * 8 < a.cols) {
            const int b = a.K == 1 ? at.r : at.r / a.K, k = a.K == 1 ? 0 : at.r - b * a.K;
            load8((const E *)a.src + b * a.stride_b + k * a.stride_k + at.c * 8, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t x = base + threadIdx.x + u * 256;
        if (x >= groups) break;                        // whole blocks: per is a multiple of 4
        uint32_t top = 0;                              // of the magnitudes' bits, which order like the magnitudes; NaN on top
#pragma unroll
        for (int n = 0; n < 8; ++n) top = max(top, __float_as_uint(v[u][n]) & 0x7fffffffu);
        top = max_of_four(top);
        const uint32_t e = top >> 23, byte = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
        const float inv = __uint_as_float((254u - min(byte, 252u)) << 23);                // 2^(127 - byte): the products are exact
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][0] * inv, v[u][1] * inv, 1.f, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][2] * inv, v[u][3] * inv, 1.f, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][4] * inv, v[u][5] * inv, 1.f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][6] * inv, v[u][7] * inv, 1.f, 3);
        ((uint32_t *)a.codes)[x] = w;
        if ((threadIdx.x & 3) == 0) a.scales[x >> 2] = (uint8_t)byte;
    }
}

// Bound by memory (128256 x 2048 to bfloat16: 91 us, 7.3 TB/s of mostly writes).
template <class E>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(DequantArgs a, int per)
{
    const int64_t base = (int64_t)blockIdx.x * 256, x = base + threadIdx.x;
    const RowColumn at(base, threadIdx.x, per);
    const int r = at.r, c = at.c;
    if (r >= a.rows || c * 8 >= a.cols) return;
    const uint32_t w = ((const uint32_t *)a.codes)[x];
    const float scale = scale_value(a.scales[x >> 2]);
    const u32x4 h = codes_to_bf16(w, scale);
    E *to = (E *)a.out + (int64_t)r * a.stride + c * 8;
    if constexpr (sizeof(E) == 2) __builtin_nontemporal_store(h, (u32x4 *)to);
    else {
        // two stores to a line each: joined in the cache (nontemporal 78 us instead of 39)
        *(u32x4 *)to = u32x4{h[0] << 16, h[0] & 0xffff0000u, h[1] << 16, h[1] & 0xffff0000u};
        *(u32x4 *)(to + 4) = u32x4{h[2] << 16, h[2] & 0xffff0000u, h[3] << 16, h[3] & 0xffff0000u};
    }
}

// ---- logits -----------------------------------------------------------------------------------------------
// Eight neighbouring logits at any element-aligned address: the memory unit takes 16-byte stores there.
__device__ __forceinline__ void store8(float *to, f32x4 a, f32x4 b)
{
    struct __attribute__((packed, aligned(4))) Any { f32x4 v; };
    ((Any *)to)[0].v = a;
    ((Any *)to)[1].v = b;
}
__device__ __forceinline__ void store8(__bf16 *to, f32x4 a, f32x4 b)
{
    struct __attribute__((packed, aligned(2))) Any { bf16x8 v; };
    ((Any *)to)->v = bf16x8{(__bf16)a[0], (__bf16)a[1], (__bf16)a[2], (__bf16)a[3], (__bf16)b[0], (__bf16)b[1], (__bf16)b[2], (__bf16)b[3]};
}

// z = h W^T, rounded once.  Few rows: bound by the codes' and the results' bytes (64 rows, V = 128256, dim = 2048, 16-bit hidden states, bfloat16 results: 41 us,
// 3.9 TB/s).  Many: by the matrix unit and the conversion of codes beside it with 16-bit hidden states (512 rows 217 us, 1.24 PFLOP/s), with 4-bit ones by the
// results (512 rows 93 us; 4096 rows over V = 151936 902 us, 781 at the highest clock, 2.8 and 3.3 PFLOP/s, 620 without a store): they leave in bursts behind a tile.
template <class T, class E>
__global__ __launch_bounds__(T::threads) void head_logits_kernel(LogitsArgs a, int ni, int nj, int stages)
{
    extern __shared__ __align__(16) char lds[];
    const float k_inverse = 1.f / (float)a.K;
    T::template work<T::MI * T::NJ * (int)sizeof(E) / 4, false>(a.weight, a.hidden, Walk(ni, nj, 1), lds,
        [&](const Walk &t) { return Work{t.i() * T::TI, t.j() * T::TJ, 0, stages}; },
        [&](const Work &) {},
        [&](const Work &w, typename T::Acc &acc) {
            const int left = a.V - w.i0;
#pragma unroll
            for (int n = 0; n < T::NJ; ++n) {
                // j / K of at most 2^20 rows: the quotient in binary32 is off by less than one
                const int j = w.j0 + T::j_of(n);
                int b = (int)((float)j * k_inverse), k = j - b * a.K;
                if (k < 0) { --b; k += a.K; }
                if (k >= a.K) { ++b; k -= a.K; }
                if (j < a.N && (!a.k_len || k < a.k_len[b])) {
                    E *row = (E *)a.out + b * a.stride_b + k * a.stride_k + w.i0;
#pragma unroll
                    for (int mi = 0; mi < T::MI; mi += 2) {
                        const int i = T::i_of(mi);
                        if (i + 8 <= left) store8(row + i, acc[mi][n], acc[mi + 1][n]);
                        else {
#pragma unroll
                            for (int r = 0; r < 8; ++r)
                                if (i + r < left) row[i + r] = (E)acc[mi + r / 4][n][r % 4];
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            return left >= T::TI && w.j0 + T::TJ <= a.N && !a.k_len;
        });
}

template <class T, class E> hipError_t logits_with(const LogitsArgs &a, hipStream_t st)
{
    using K = Kind<T::kind>;
    const int ni = up(a.V, T::TI), nj = up(a.N, T::TJ), stages = up(a.D, K::elems);
    return with_lds((const void *)head_logits_kernel<T, E>, T::ring_bytes, [&] {
        head_logits_kernel<T, E><<<grid_of<T>((int64_t)ni * nj), T::threads, T::ring_bytes, st>>>(a, ni, nj, stages);
    });
}

template <class E> hipError_t logits_of(const LogitsArgs &a, int kind, hipStream_t st)
{
    // the smallest tile that holds the tokens, long in I where they are many; V = 128256, dim = 2048, us with tiles of 128 x 16 / 128 x 32 /
    // 128 x 64 / 256 x 128 / 256 x 256: 1 row 22 / 23 / 24 / 25 / 34, 32 rows 33 / 24 / 26 / 28 / 36, 64 rows 60 / 35 / 28 / 29 / 38,
    // 128 rows 109 / 62 / 42 / 35 / 40, 192 rows 153 / 90 / 62 / 55 / 44, 512 rows 403 / 229 / 157 / 119 / 96
    if (kind == kTileMx4)
        return a.N <= 16 ? logits_with<Tile<kTileMx4, 128, 16, 4, 1>, E>(a, st) : a.N <= 32 ? logits_with<Tile<kTileMx4, 128, 32, 4, 1>, E>(a, st)
             : a.N <= 64 ? logits_with<Tile<kTileMx4, 128, 64, 4, 1>, E>(a, st) : a.N <= 128 ? logits_with<Tile<kTileMx4, 256, 128, 4, 2>, E>(a, st)
             : logits_with<Tile<kTileMx4, 256, 256, 2, 4>, E>(a, st);
    // hidden states of 16 bits: they pass through LDS with the weights, four times their bytes for a row each, so tiles are long in I; V = 128256,
    // dim = 2048, us with tiles of 128 x 16 / 256 x 32 / 256 x 64 / 256 x 128: 1 row 27 / 28 / 36 / 55, 32 rows 45 / 30 / 36 / 52, 64 rows
    // 81 / 51 / 39 / 55, 128 rows 150 / 93 / 68 / 59, 512 rows 572 / 354 / 272 / 217 (128 x 128: 304)
    return a.N <= 16 ? logits_with<Tile<kTileMx4W, 128, 16, 4, 1>, E>(a, st) : a.N <= 32 ? logits_with<Tile<kTileMx4W, 256, 32, 8, 1>, E>(a, st)
         : a.N <= 64 ? logits_with<Tile<kTileMx4W, 256, 64, 8, 1>, E>(a, st) : logits_with<Tile<kTileMx4W, 256, 128, 4, 2>, E>(a, st);
}

}  // namespace

template <class E> static hipError_t quantize(const QuantArgs &a, hipStream_t st)
{
    const int per = mx4_cols(a.cols) / 8;
    const int64_t groups = (int64_t)a.rows * per;
    // four groups a lane where the values come from memory, not from the 256 MiB cache before it (one / four a lane, us, rows of 2048 bfloat16:
    // 64 rows 2.6 / 4.5, 4096 rows 6.3 / 7.2, 32768 rows 33.2 / 34.3, 65536 rows 64 / 60, 128256 rows 126 / 114; 50257 x 1120 binary32 48.2 / 49.4)
    if (groups * 8 * (int)sizeof(E) >= 1 << 28) mx4_quantize_kernel<E, 4><<<(groups + 1023) / 1024, 256, 0, st>>>(a, per, groups);
    else mx4_quantize_kernel<E, 1><<<(groups + 255) / 256, 256, 0, st>>>(a, per, groups);
    return hipGetLastError();
}

hipError_t launch_mx4_quantize(const QuantArgs &a, int dtype, hipStream_t st)
{
    return dtype == TAPOUT_F32 ? quantize<float>(a, st) : quantize<__bf16>(a, st);
}

hipError_t launch_mx4_dequantize(const DequantArgs &a, int dtype, hipStream_t st)
{
    const int per = mx4_cols(a.cols) / 8;
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
