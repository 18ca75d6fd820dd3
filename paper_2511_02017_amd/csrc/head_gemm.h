// The matrix-core tile that the draft head's operators share:  acc[i][j] = sum_k I[i][k] * J[j][k], both operands with k
// contiguous.  I is always the long side that is streamed (vocabulary rows, or columns of a gradient), J the tokens.
//
// A stage is a piece of k that both operands bring into LDS by the asynchronous global-to-LDS loads (16 bytes a lane, no
// registers in between); two stages alternate, the next one is under way while the matrix instructions work on this one.
// Rows of a stage lie behind each other without padding (the loads write 64 x 16 bytes in a row), so the 16-byte chunks of a
// row are exchanged by an XOR with bits of the row number: the 16 lanes that read one chunk column of 16 rows then meet every
// bank once.  The exchange is made on the source address, which stays within the row.
#pragma once

#include "common.h"

namespace tapout {

using f32x4 = float __attribute__((ext_vector_type(4)));
using i32x8 = int __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));

// What the two operands of a product are.
enum TileKind {
    kTileF32,    // both binary32
    kTileBf16,   // both bfloat16
    kTileMx4,    // both 4-bit codes with a scale byte for 32 of them
    kTileMx4W    // I: 4-bit codes with scales; J: bfloat16
};

// Bytes of an operand's row in a stage, elements of k in a stage, and matrix steps: a step takes 64 bytes of each of 16 I rows
// (16 a lane).
template <int KIND> struct Kind {
    static constexpr int elems = KIND == kTileF32 ? 32 : KIND == kTileBf16 ? 64 : KIND == kTileMx4 ? 256 : 128;
    static constexpr int row_i = KIND == kTileMx4W ? 64 : 128;
    static constexpr int row_j = KIND == kTileMx4W ? 256 : 128;
    static constexpr int steps = row_i / 64;
    static constexpr int step_elems = elems / steps;
    static constexpr int scale_i = KIND == kTileMx4 || KIND == kTileMx4W ? elems / 32 : 0;     // scale bytes of a row in a stage
    static constexpr int scale_j = KIND == kTileMx4 ? elems / 32 : 0;
};

struct Operand {
    const void *p;          // row 0, 16-byte aligned
    int64_t stride;         // bytes from row to row, a multiple of 16; 256 of them within 2^31 (checked on the host)
    int32_t rows;
    int32_t row_bytes;      // bytes of a row that may be read
    const uint8_t *scales;  // kTileMx4, and I of kTileMx4W
    int32_t scale_stride;   // bytes, a multiple of 4
};

// Exchange of a row's 16-byte chunks.  A 16-byte LDS read serves its 64 lanes sixteen at a time, lanes 0-3, 12-15 and 20-27, then
// 4-11, 16-19 and 28-31, then the same of the upper half; with lane l at row l % 16 and chunk l / 16 of its row these sixteen meet
// 64 different banks.  (With chunk ^ (row & 7), which suits sixteen lanes in a row, half of the LDS cycles were conflicts.)
template <int R> __device__ __forceinline__ int chunk_swap(int row)
{
    if constexpr (R == 64) return -(row >> 2) & 3;                            // four rows to 64 banks, lane's chunk l / 16
    else if constexpr (R == 128) return (row >> 1) & 7;                       // two rows
    else return (row & 3) | (row & 8) | (row & 8) >> 1;                       // one row; lane's chunk 4 (l / 16) + t
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, int64_t bytes)
{
    const uint32_t n = bytes <= 0 ? 0u : bytes > 0xfffffff0ll ? 0xfffffff0u : (uint32_t)bytes;
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)n, 0x00020000);
}

// T rows of R bytes of a stage, in pieces of 1 KB (a wavefront's load), dealt out to NW wavefronts.  Every wavefront makes the same
// number of loads, since it waits for them by their number: where the pieces do not come out even, some are loaded twice.
template <int T, int R, int NW> struct Stager {
    static constexpr int pieces = T * R / 1024, per = (pieces + NW - 1) / NW;
    uint32_t off[per];
    __device__ void init(int rows_left, int64_t stride, int wave, int lane)
    {
#pragma unroll
        for (int n = 0; n < per; ++n) {
            const int row = (wave + n * NW) % pieces * (1024 / R) + lane / (R / 16);
            const int chunk = (lane % (R / 16)) ^ chunk_swap<R>(row);
            off[n] = (uint32_t)(min(row, rows_left - 1) * stride) + chunk * 16;      // rows behind the last one: the last one again
        }
    }
    __device__ __forceinline__ void issue_one(int n, __amdgpu_buffer_rsrc_t rsrc, char *lds, uint32_t k_byte, int wave) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave + n * NW) % pieces * 1024), 16, off[n], k_byte, 0, 0);
    }
};

// The scale bytes of a stage: S (4 or 8) a row, four a lane, 256 bytes a piece.
template <int T, int S, int NW> struct ScaleStager {
    static constexpr int pieces = (T * S + 255) / 256, per = (pieces + NW - 1) / NW;
    uint32_t off[per];
    __device__ void init(int rows_left, int stride, int wave, int lane)
    {
#pragma unroll
        for (int n = 0; n < per; ++n) {
            const int word = (wave + n * NW) % pieces * 64 + lane, row = word / (S / 4);
            off[n] = (uint32_t)min(row, rows_left - 1) * (uint32_t)stride + (word % (S / 4)) * 4;
        }
    }
    __device__ __forceinline__ void issue_one(int n, __amdgpu_buffer_rsrc_t rsrc, char *lds, uint32_t k_byte, int wave) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave + n * NW) % pieces * 256), 4, off[n], k_byte, 0, 0);
    }
};
template <int T, int NW> struct ScaleStager<T, 0, NW> {
    static constexpr int per = 0;
    __device__ void init(int, int, int, int) {}
    __device__ void issue_one(int, __amdgpu_buffer_rsrc_t, char *, uint32_t, int) const {}
};

__device__ __forceinline__ f32x4 mma_f32(u32x4 a, u32x4 b, f32x4 c)
{
    // four k a lane, one matrix instruction each; the order of k is the same on both sides
#pragma unroll
    for (int n = 0; n < 4; ++n) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, a)[n], __builtin_bit_cast(f32x4, b)[n], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4 mma_bf16(u32x4 a, u32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma_mx4(u32x4 a, uint32_t sa, u32x4 b, uint32_t sb, f32x4 c)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)sa, 0, (int)sb);
}

// A scale byte as the conversions take it: they read the exponent field alone, 0 as 2^-127 and 255 as NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes as bfloat16.  E2M1 times a power of two is exact in bfloat16 (whose exponents are binary32's).
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t w, float scale)
{
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    return r;
}

template <int N> __device__ __forceinline__ void wait_loads_and_barrier()
{
    // the LDS reads of this wavefront are done, all of its loads but the last N have landed, and those of the others
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// TI x TJ results by WI x WJ wavefronts; a wavefront holds MI x NJ blocks of 16 x 16.  acc[mi][nj][r] of lane l is
//   i = (wave's i) + 16 mi + 4 (l / 16) + r,   j = (wave's j) + 16 nj + l % 16.
// I's part of a stage has three places in LDS, J's two: that is what 160 KB hold of 256 x 256 (128 x 128: twice a compute unit).
template <int KIND, int TI_, int TJ_, int WI_, int WJ_> struct Tile {
    using K = Kind<KIND>;
    static constexpr int kind = KIND, TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, NW = WI * WJ, threads = NW * 64;
    static constexpr int MI = TI / WI / 16, NJ = TJ / WJ / 16;
    static constexpr int up256(int n) { return (n + 255) & ~255; }
    static constexpr int oSI = TI * K::row_i, bytes_i = oSI + up256(TI * K::scale_i);
    static constexpr int oSJ = TJ * K::row_j, bytes_j = oSJ + up256(TJ * K::scale_j);
    static constexpr int ring_i = KIND == kTileMx4 ? 2 : 3, ring_j = 2, lds_bytes = ring_i * bytes_i + ring_j * bytes_j;
    using Acc = f32x4[MI][NJ];

    // What a wavefront multiplies in one step.
    struct Frags {
        u32x4 a[MI], b[NJ];
        uint32_t sa[K::scale_i ? MI : 1], sb[K::scale_j ? NJ : 1];
    };
    // Read n of the NJ + MI of a step, J's first: the next step begins with all of J and the first of I.
    static constexpr int reads = NJ + MI;
    static __device__ __forceinline__ void load_one(int n, const char *pi, const char *pj, int s, int wi, int wj, int lane, Frags &f)
    {
        const int r16 = lane & 15, g = lane >> 4;
        if (n < NJ) {
            const int row = wj * NJ * 16 + r16;
            f.b[n] = *(const u32x4 *)(pj + row * K::row_j + (((s * 4 + g) ^ chunk_swap<K::row_j>(r16)) * 16) + n * 16 * K::row_j);
            // four scales, of the four lanes that share a row; the matrix instruction takes the low byte
            if constexpr (K::scale_j > 0) f.sb[n] = *(const uint32_t *)(pj + oSJ + row * K::scale_j + s * 4 + n * 16 * K::scale_j);
        } else {
            const int m = n - NJ, row = wi * MI * 16 + r16;
            f.a[m] = *(const u32x4 *)(pi + row * K::row_i + (((s * 4 + g) ^ chunk_swap<K::row_i>(r16)) * 16) + m * 16 * K::row_i);
            if constexpr (K::scale_i > 0) f.sa[m] = *(const uint32_t *)(pi + oSI + row * K::scale_i + s * 4 + m * 16 * K::scale_i);
        }
    }
    static __device__ __forceinline__ void multiply_row(int mi, const Frags &f, int lane, Acc &acc)
    {
        const int g8 = (lane >> 4) * 8;
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj)
            acc[mi][nj] = KIND == kTileF32 ? mma_f32(f.a[mi], f.b[nj], acc[mi][nj])
                        : KIND == kTileBf16 ? mma_bf16(f.a[mi], f.b[nj], acc[mi][nj])
                                            : mma_mx4(f.a[mi], f.sa[K::scale_i ? mi : 0] >> g8, f.b[nj], f.sb[K::scale_j ? nj : 0] >> g8, acc[mi][nj]);
    }
    // kTileMx4W: a lane holds the 32 codes of block g of its row: four matrix instructions of 8 codes a lane, whose k are
    // 32 g + 8 t .. + 7 on both sides.
    static __device__ __forceinline__ void compute_w(const char *pi, const char *pj, int wi, int wj, int lane, Acc &acc)
    {
        const int r16 = lane & 15, g = lane >> 4;
        const char *si = pi + (wi * MI * 16 + r16) * K::row_i, *sj = pj + (wj * NJ * 16 + r16) * K::row_j;
        const int xi = chunk_swap<K::row_i>(r16), xj = chunk_swap<K::row_j>(r16);
        u32x4 a[MI];
        float sa[MI];
        const char *ssi = pi + oSI + (wi * MI * 16 + r16) * K::scale_i;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            a[mi] = *(const u32x4 *)(si + mi * 16 * K::row_i + ((g ^ xi) * 16));
            sa[mi] = scale_value((*(const uint32_t *)(ssi + mi * 16 * K::scale_i) >> (8 * g)) & 255u);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u32x4 b[NJ];
#pragma unroll
            for (int nj = 0; nj < NJ; ++nj) b[nj] = *(const u32x4 *)(sj + nj * 16 * K::row_j + (((g * 4 + t) ^ xj) * 16));
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) {
                const u32x4 w = codes_to_bf16(a[mi][t], sa[mi]);
#pragma unroll
                for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = mma_bf16(w, b[nj], acc[mi][nj]);
            }
        }
    }

    // acc = the sums over stages [first, first + n); the last stage of k (index n_all - 1) has last_steps steps.  All
    // wavefronts of the workgroup come here; LDS is free again when it returns.
    static __device__ __forceinline__ void run(const Operand &I, const Operand &J, int i0, int j0, int first, int n, int n_all, int last_steps,
                                               char *lds, Acc &acc)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wi = wave / WJ, wj = wave % WJ;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int64_t left_i = I.rows - i0, left_j = J.rows - j0;
        const __amdgpu_buffer_rsrc_t ri = buffer_of((const char *)I.p + i0 * I.stride, (left_i - 1) * I.stride + I.row_bytes);
        const __amdgpu_buffer_rsrc_t rj = buffer_of((const char *)J.p + j0 * J.stride, (left_j - 1) * J.stride + J.row_bytes);
        Stager<TI, K::row_i, NW> gi;
        Stager<TJ, K::row_j, NW> gj;
        gi.init((int)min(left_i, (int64_t)TI), I.stride, wave, lane);
        gj.init((int)min(left_j, (int64_t)TJ), J.stride, wave, lane);
        ScaleStager<TI, K::scale_i, NW> hi;
        ScaleStager<TJ, K::scale_j, NW> hj;
        __amdgpu_buffer_rsrc_t rsi = ri, rsj = rj;
        if constexpr (K::scale_i > 0) {
            rsi = buffer_of(I.scales + (int64_t)i0 * I.scale_stride, left_i * I.scale_stride);
            hi.init((int)min(left_i, (int64_t)TI), I.scale_stride, wave, lane);
        }
        if constexpr (K::scale_j > 0) {
            rsj = buffer_of(J.scales + (int64_t)j0 * J.scale_stride, left_j * J.scale_stride);
            hj.init((int)min(left_j, (int64_t)TJ), J.scale_stride, wave, lane);
        }
        // Load n of a stage's loads of either operand.  Behind the last stage: the last one again, into memory that nobody reads.
        constexpr int loads_i = gi.per + hi.per, loads_j = gj.per + hj.per;
        auto load_i = [&](int x, int s, char *to) {
            const uint32_t at = (uint32_t)(first + min(s, n - 1));
            if (x < gi.per) gi.issue_one(x, ri, to, at * K::row_i, wave);
            else hi.issue_one(x - gi.per, rsi, to + oSI, at * K::scale_i, wave);
        };
        auto load_j = [&](int x, int s, char *to) {
            const uint32_t at = (uint32_t)(first + min(s, n - 1));
            if (x < gj.per) gj.issue_one(x, rj, to, at * K::row_j, wave);
            else hj.issue_one(x - gj.per, rsj, to + oSJ, at * K::scale_j, wave);
        };
        char *const lj = lds + ring_i * bytes_i;
        if (n > 0) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int x = 0; x < loads_i; ++x) load_i(x, s, lds + s * bytes_i);
#pragma unroll
                for (int x = 0; x < loads_j; ++x) load_j(x, s, lj + s * bytes_j);
            }
            wait_loads_and_barrier<loads_i + loads_j>();
        }
        // places of I's stages s, s + 1, s + 2
        char *i0p = lds, *i1p = lds + bytes_i, *i2p = ring_i == 3 ? lds + 2 * bytes_i : i0p;
        if constexpr (K::steps == 1) {
            for (int s = 0; s < n; ++s) {
                char *now = lj + (s & 1) * bytes_j;
#pragma unroll
                for (int x = 0; x < loads_i; ++x) load_i(x, s + 2, i2p);
                compute_w(i0p, now, wi, wj, lane, acc);
                wait_loads_and_barrier<loads_i>();
#pragma unroll
                for (int x = 0; x < loads_j; ++x) load_j(x, s + 2, now);
                char *t = i0p; i0p = i1p; i1p = i2p; i2p = t;
            }
        } else if (n > 0) {
            // The operands of a step are read while the step before multiplies; the barrier that hands J's place on lies between the
            // last reads of the stage and its last products.  Reads and loads are dealt out between the products: a wavefront that
            // issues all its loads at once waits for the others' loads to be taken, with no product under way.
            Frags f0, f1;
#pragma unroll
            for (int x = 0; x < reads; ++x) load_one(x, i0p, lj, 0, wi, wj, lane, f0);
            for (int s = 0; s + 1 < n; ++s) {
                char *now = lj + (s & 1) * bytes_j, *next = lj + ((s + 1) & 1) * bytes_j;
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) {
                    constexpr int fast = MI > 1 ? (MI + 1) / 2 : 1;          // all reads in the first half: the barrier waits for them
#pragma unroll
                    for (int x = mi * loads_i / MI; x < (mi + 1) * loads_i / MI; ++x)
                        if (ring_i == 3) load_i(x, s + 2, i2p);
#pragma unroll
                    for (int x = mi * reads / fast; x < (mi + 1) * reads / fast && x < reads; ++x) load_one(x, i0p, now, 1, wi, wj, lane, f1);
                    multiply_row(mi, f0, lane, acc);
                    __builtin_amdgcn_sched_barrier(0);
                }
                wait_loads_and_barrier<ring_i == 3 ? loads_i : 0>();
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
                    for (int x = mi * loads_i / MI; x < (mi + 1) * loads_i / MI; ++x)
                        if (ring_i == 2) load_i(x, s + 2, i0p);
#pragma unroll
                    for (int x = mi * loads_j / MI; x < (mi + 1) * loads_j / MI; ++x) load_j(x, s + 2, now);
#pragma unroll
                    for (int x = mi * reads / MI; x < (mi + 1) * reads / MI; ++x) load_one(x, i1p, next, 0, wi, wj, lane, f0);
                    multiply_row(mi, f1, lane, acc);
                    __builtin_amdgcn_sched_barrier(0);
                }
                char *t = i0p; i0p = i1p; i1p = ring_i == 3 ? i2p : t; i2p = t;
            }
            const bool two = first + n < n_all || last_steps == 2;
            if (two) {
#pragma unroll
                for (int x = 0; x < reads; ++x) load_one(x, i0p, lj + ((n - 1) & 1) * bytes_j, 1, wi, wj, lane, f1);
            }
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) multiply_row(mi, f0, lane, acc);
            if (two) {
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) multiply_row(mi, f1, lane, acc);
            }
        }
        wait_loads_and_barrier<0>();
        __syncthreads();
    }
};

// Workgroup -> tile.  Consecutive workgroups go to the eight dies in turn, each with an L2 of its own: die x gets a run of
// tiles, and a run walks blocks of `band` I tiles by all J tiles, I fastest, so that the workgroups a die has at a time
// share both operands.
struct TileAt { int i, j; };
__device__ __forceinline__ TileAt tile_at(int bid, int ni, int nj, int band)
{
    const int n = ni * nj, x = bid & 7, q = n >> 3, r = n & 7;
    const int at = x * q + min(x, r) + (bid >> 3);
    const int per = band * nj, b = at / per, in = at - b * per, h = min(band, ni - b * band);
    return TileAt{b * band + in % h, in / h};
}

}  // namespace tapout
