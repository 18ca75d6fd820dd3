// 8-bit floating point with a binary32 scale for each block of 128: quantisation, its inverse, and the logits of a head held that way.
//
// A block is 128 neighbours of a row (hidden states) or of 128 rows (weights).  Its scale s is its largest magnitude times 1/448, an element's code
// x / s in E4M3, to nearest.
#include "fp8_device.h"

namespace tapout {
namespace {

// Eight neighbouring values from memory, and back.
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
__device__ __forceinline__ uint32_t top_of(const float (&x)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < 8; ++n) top = max(top, __float_as_uint(x[n]) & 0x7fffffffu);
    return top;
}
__device__ __forceinline__ uint2 pack8(const float (&x)[8], float scale) { return uint2{fp8_pack(x[0], x[1], x[2], x[3], scale), fp8_pack(x[4], x[5], x[6], x[7], scale)}; }

// Eight elements a lane, sixteen lanes a block.  64 rows of 2048 bfloat16 4.9 us, the launch; 128256 rows 200 us, 4.0 TB/s.
template <class E>
__global__ __launch_bounds__(256) void fp8_quantize_rows_kernel(Fp8QuantArgs a, int per, int64_t groups)      // per: groups of eight in a padded row
{
    const int64_t base = (int64_t)blockIdx.x * 256, x = base + threadIdx.x;
    const RowColumn at(base, threadIdx.x, per);
    float v[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) v[n] = 0.f;
    if (x < groups && at.c * 8 < a.cols) {
        const int b = a.K == 1 ? at.r : at.r / a.K, k = a.K == 1 ? 0 : at.r - b * a.K;
        load8((const E *)a.src + b * a.stride_b + k * a.stride_k + at.c * 8, v);
    }
    const float scale = fp8_scale(fp8_top<4>(top_of(v)));       // whole blocks: per is a multiple of 16
    if (x >= groups) return;
    ((uint2 *)a.codes)[x] = pack8(v, scale);
    if ((threadIdx.x & 15) == 0) a.scales[x >> 4] = scale;
}

// A workgroup a block of 128 x 128, which stays in its registers: sixteen lanes a row, sixteen rows at a time.  Bound by memory: 128256 x 2048
// bfloat16 154 us, 5.2 TB/s; 50257 x 1120 binary32 59 us, 4.8 TB/s.
template <class E>
__global__ __launch_bounds__(256) void fp8_quantize_blocks_kernel(Fp8QuantArgs a, int across)       // across: blocks in a row of blocks
{
    __shared__ uint32_t tops[4];
    const int br = blockIdx.x / across, bc = blockIdx.x - br * across, r0 = br * 128 + (threadIdx.x >> 4), c = bc * 128 + (threadIdx.x & 15) * 8;
    float v[8][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int n = 0; n < 8; ++n) v[i][n] = 0.f;
        if (r0 + i * 16 < a.rows && c < a.cols) load8((const E *)a.src + (r0 + i * 16) * a.stride_b + c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, top_of(v[i]));
    top = fp8_top<6>(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    const float scale = fp8_scale(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (r0 + i * 16 < a.rows) *(uint2 *)(a.codes + (int64_t)(r0 + i * 16) * (across * 128) + c) = pack8(v[i], scale);
    if (threadIdx.x == 0) a.scales[blockIdx.x] = scale;
}

// Eight elements a lane.  Bound by memory: 128256 x 2048 to bfloat16 139 us, 5.7 TB/s.
template <class E>
__global__ __launch_bounds__(256) void fp8_dequantize_kernel(Fp8DequantArgs a, int per)
{
    const int64_t base = (int64_t)blockIdx.x * 256, x = base + threadIdx.x;
    const RowColumn at(base, threadIdx.x, per);
    if (at.r >= a.rows || at.c * 8 >= a.cols) return;
    const uint2 w = ((const uint2 *)a.codes)[x];
    const float s = a.scales[(int64_t)(at.r / a.block_rows) * (per / 16) + at.c / 16];
    E *to = (E *)a.out + (int64_t)at.r * a.stride + at.c * 8;
    float v[8];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const uint32_t word = n ? w.y : w.x;
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
        v[4 * n] = lo[0] * s; v[4 * n + 1] = lo[1] * s; v[4 * n + 2] = hi[0] * s; v[4 * n + 3] = hi[1] * s;
    }
    E e[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) e[n] = (E)v[n];
#pragma unroll
    for (int n = 0; n < (int)sizeof(E) / 2; ++n) ((u32x4 *)to)[n] = ((const u32x4 *)e)[n];
}

template <class E> hipError_t quantize(const Fp8QuantArgs &a, int block_rows, hipStream_t st)
{
    const int across = up(a.cols, kFp8Block);
    if (block_rows == 1) {
        const int64_t groups = (int64_t)a.rows * across * 16;
        fp8_quantize_rows_kernel<E><<<(groups + 255) / 256, 256, 0, st>>>(a, across * 16, groups);
    } else {
        fp8_quantize_blocks_kernel<E><<<(int64_t)up(a.rows, 128) * across, 256, 0, st>>>(a, across);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_quantize(const Fp8QuantArgs &a, int block_rows, int dtype, hipStream_t st)
{
    return dtype == TAPOUT_F32 ? quantize<float>(a, block_rows, st) : quantize<__bf16>(a, block_rows, st);
}

hipError_t launch_fp8_dequantize(const Fp8DequantArgs &a, int dtype, hipStream_t st)
{
    const int per = up(a.cols, kFp8Block) * 16;
    const int64_t grid = ((int64_t)a.rows * per + 255) / 256;
    if (dtype == TAPOUT_F32) fp8_dequantize_kernel<float><<<grid, 256, 0, st>>>(a, per);
    else fp8_dequantize_kernel<__bf16><<<grid, 256, 0, st>>>(a, per);
    return hipGetLastError();
}

}  // namespace tapout
