// The matrix-core tile that the draft head's operators share:  acc[i][j] = sum_k I[i][k] * J[j][k], both operands with k
// contiguous.  I is always the long side that is streamed (vocabulary rows, or columns of a gradient), J the tokens.
//
// A stage is a piece of k that both operands bring into LDS by the asynchronous global-to-LDS loads (16 bytes a lane, no
// registers in between).  I has places for three stages and J for two (both two where three do not fit), so that up to two stages
// are under way while the matrix instructions work on a third, across the tiles of a workgroup too.
// Rows of a stage lie behind each other without padding (the loads write 64 x 16 bytes in a row), so the 16-byte chunks of a
// row are exchanged by an XOR with bits of the row number: the 16 lanes that read one chunk column of 16 rows then meet every
// bank once.  The exchange is made on the source address, which stays within the row.
#pragma once

#include <type_traits>

#include "common.h"

namespace tapout {

using f32x4 = float __attribute__((ext_vector_type(4)));
using i32x8 = int __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

// What the two operands of a product are.
enum TileKind {
    kTileF32,    // both binary32, multiplied as they are
    kTileF32x3,  // both binary32, multiplied as sums of three bfloat16 each (see split3)
    kTileBf16,   // both bfloat16
    kTileMx4,    // both 4-bit codes with a scale byte for 32 of them
    kTileMx4W    // I: 4-bit codes with scales; J: bfloat16
};

// Bytes of an operand's row in a stage, elements of k in a stage, and matrix steps: a step takes 64 bytes of each of 16 I rows
// (16 a lane).
template <int KIND> struct Kind {
    static constexpr int elems = KIND == kTileF32 || KIND == kTileF32x3 ? 32 : KIND == kTileBf16 ? 64 : KIND == kTileMx4 ? 256 : 128;
    static constexpr int row_i = KIND == kTileMx4W ? 64 : 128;
    static constexpr int row_j = KIND == kTileMx4W ? 256 : 128;
    static constexpr int steps = row_i / 64;
    static constexpr int scale_i = KIND == kTileMx4 || KIND == kTileMx4W ? elems / 32 : 0;     // scale bytes of a row in a stage
    static constexpr int scale_j = KIND == kTileMx4 ? elems / 32 : 0;
};

struct Operand {
    const void *p;          // row 0, 16-byte aligned (I turned: step 0 of k)
    int64_t stride;         // bytes from row to row, a multiple of 16; 256 of them within 2^31 (checked on the host)
    int32_t rows;
    int32_t row_bytes;      // bytes of a row, a multiple of 16: what lies behind counts as zeros
    const uint8_t *scales;  // kTileMx4, and I of kTileMx4W
    int32_t scale_stride;   // bytes of a row's scales, a multiple of 4
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

// The memory of `bytes` bytes from p on, at most 2^31 - 1 of them: loads of what lies behind bring zeros, into LDS too.  The compiler
// leaves the scalar offset of a buffer load out of what it says of the range check, so the whole address is a lane's offset.
constexpr uint32_t kNoMemory = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes <= 0 ? 0 : (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff), 0x00020000);
}

// Which row of the tile lies at row q of its part of LDS, that is, which row a matrix instruction takes as its q % 16th.  A lane's
// four results of one instruction are rows 4 (l / 16) .. + 3 of I and one row of J; with this order the results of two
// instructions that are neighbours in I are eight neighbouring rows of I, and those of NJ neighbours in J are NJ neighbouring
// rows of J, so that results leave the registers in 16-byte pieces, in either orientation, without passing through LDS.
__device__ __forceinline__ int row_of_i(int q) { return (q & ~31) | (q & 12) << 1 | (q & 16) >> 2 | (q & 3); }
template <int NJ> __device__ __forceinline__ int row_of_j(int q) { return q / (16 * NJ) * (16 * NJ) + (q & 15) * NJ + (q >> 4) % NJ; }
template <int NJ> __device__ __forceinline__ int tile_row(int q) { if constexpr (NJ == 0) return row_of_i(q); else return row_of_j<NJ>(q); }

// A wavefront's load of 64 x 16 bytes into LDS.  HIDDEN: not as the builtin, whose loads the compiler takes to be meant by every turning
// read that follows, and waits for (a product by 1503 hidden states in twice as many runs of k as now: 754 instead of 293 us).  There are no registers to be written
// but M0; this wavefront and the others wait by number, below.
template <bool HIDDEN> __device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rsrc, char *lds, uint32_t off)
{
    const auto to = (__attribute__((address_space(3))) void *)lds;
    if constexpr (HIDDEN) {
        const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)to);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(rsrc) : "memory", "m0");
    } else {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, to, 16, off, 0, 0, 0);
    }
}

// T rows of R bytes of a stage, in pieces of a wavefront's load, W bytes a lane.  Every wavefront makes the same number of loads,
// since it waits for them by their number: where there are fewer pieces than wavefronts, some are loaded twice.  Rows behind the
// operand's last one and bytes behind a row's last one come as zeros.
template <int T, int R, int W, int NW, int NJ, bool HIDDEN = false> struct Stager {           // NJ = 0: I's rows
    static constexpr int pieces = T * R / (64 * W) < 1 ? 1 : T * R / (64 * W), per = (pieces + NW - 1) / NW, rows = 64 * W / R, lanes = R / W;
    static_assert(pieces % NW == 0 || pieces < NW, "");
    uint32_t off, now, at;           // of this lane: from the tile's first row; the same of a stage, or nowhere; its first byte in a row's R
    __device__ __forceinline__ void init(int64_t stride, int wave, int lane)
    {
        const int q = wave % pieces * rows + lane / lanes;
        at = (uint32_t)((lane % lanes) ^ (W == 16 ? chunk_swap<R>(q) : 0)) * W;
        off = (uint32_t)(tile_row<NJ>(q) * stride) + at;
    }
    __device__ __forceinline__ void stage(int s, int row_bytes) { now = s * R + (int)at < row_bytes ? off + (uint32_t)(s * R) : kNoMemory; }
    // The row orders exchange bits of a row's number, and the wavefronts' pieces of one n differ in bits of their own.  All rows of a tile lie
    // within 2^31 bytes, so the sum does not wrap, of a lane that is nowhere either.
    __device__ __forceinline__ void issue(int n, __amdgpu_buffer_rsrc_t rsrc, char *lds, int64_t stride, int wave) const
    {
        char *to = lds + (wave % pieces + n * NW) * (64 * W);
        const uint32_t from = now + (uint32_t)(tile_row<NJ>(n * NW * rows) * stride);
        if constexpr (W == 16) load_to_lds<HIDDEN>(rsrc, to, from);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)to, 4, from, 0, 0, 0);
    }
};
// The same of an operand whose rows are steps of k (its columns the rows of I): KS of them, T columns of E bytes each, 16 bytes a lane.
// A lane of a matrix instruction wants neighbours in k of one column; the reads below turn them round.  They serve rows 8 g + 0..3 (bfloat16,
// sixteen columns in 32 bytes) or 4 g + j (binary32, 64 bytes) of neighbouring g at a time, which the exchange of slots of that size
// by bits of the row spreads over the banks.
template <int T, int KS, int E, int NW> struct TurnedStager {
    static constexpr int R = T * E, pieces = R * KS / 1024, per = pieces / NW, rows = 1024 / R, lanes = R / 16;
    static_assert(pieces % NW == 0 && NW * rows % 8 == 0, "");
    static __device__ __forceinline__ uint32_t swap(int row) { return E == 2 ? ((row & 3) | (row >> 1 & 4)) * 32u : (uint32_t)(row >> 2 & 3) * 64u; }
    uint32_t row_off, chunk[2];      // of this lane's first row; its bytes in a row, of even and odd n
    __device__ __forceinline__ void init(int64_t stride, int wave, int lane)
    {
        const int q = wave * rows + lane / lanes;
        row_off = (uint32_t)(q * stride);
#pragma unroll
        for (int n = 0; n < 2; ++n) chunk[n] = (uint32_t)(lane % lanes) * 16u ^ swap(q + n * NW * rows);
    }
    __device__ __forceinline__ void issue(int n, __amdgpu_buffer_rsrc_t rsrc, char *lds, int64_t stride, int wave) const
    {
        load_to_lds<E == 2>(rsrc, lds + (wave + n * NW) * 1024, row_off + chunk[NW * rows % 16 ? n & 1 : 0] + (uint32_t)(n * NW * rows * stride));
    }
};
struct NoStager {
    static constexpr int per = 0;
    __device__ __forceinline__ void init(int64_t, int, int) {}
    __device__ __forceinline__ void stage(int, int) {}
    __device__ __forceinline__ void issue(int, __amdgpu_buffer_rsrc_t, char *, int64_t, int) const {}
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
// Eight binary32 as three bfloat16 each, x = h + m + l: each part is the upper half of what is left, taken off exactly, and 24 bits are
// three times eight, so nothing is left behind l.  With |m| < 2^-7 |x| and |l| < 2^-15 |x|, the three smallest of the nine products of two
// such sums are below 2^-21 |x y| together, 2^-24 in the mean, and are left out.  Six bfloat16 products take 96 cycles of the matrix unit for
// 16 x 16 x 32, the binary32 ones 256.  Parts cut off are a third fewer vector instructions than parts rounded by conversions (cross
// entropy of 1000 / 3000 rows, V = 32000, dim = 1024: 375 / 1030 us instead of 425 / 1160, with no look for a NaN yet); the splitting between the products of the
// row of blocks before, two instructions each, gains nothing there (385 / 1026).  An infinity becomes a NaN (see Tile::multiply_as_they_are).
struct Split3 { u32x4 h, m, l; };
__device__ __forceinline__ Split3 split3(u32x4 a, u32x4 b)
{
    Split3 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float x = __uint_as_float(q < 2 ? a[2 * q] : b[2 * q - 4]), y = __uint_as_float(q < 2 ? a[2 * q + 1] : b[2 * q - 3]);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint32_t u = __float_as_uint(x), w = __float_as_uint(y);
            (p == 0 ? r.h : p == 1 ? r.m : r.l)[q] = __builtin_amdgcn_perm(w, u, 0x07060302u);
            x -= __uint_as_float(u & 0xffff0000u);
            y -= __uint_as_float(w & 0xffff0000u);
        }
    }
    return r;
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

// The same with one of two numbers.  The branch is inside, where the compiler does not see it: it would move the products behind it.
template <int N0, int N1> __device__ __forceinline__ void wait_loads_and_barrier(int which)
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_cmp_eq_u32 %0, 0\n\ts_cbranch_scc1 .Lfirst%=\n\ts_waitcnt vmcnt(%2) lgkmcnt(0)\n\ts_branch .Lboth%=\n.Lfirst%=:\n\t"
                 "s_waitcnt vmcnt(%1) lgkmcnt(0)\n.Lboth%=:\n\ts_barrier" ::"s"(which), "n"(N0), "n"(N1) : "memory", "scc");
    __builtin_amdgcn_sched_barrier(0);
}

// A workgroup's way through ni x nj tiles by `splits` runs of k.  Consecutive workgroups go to the eight dies in turn, each with an
// L2 of its own: die x gets a run of tiles, of which its workgroups take every S-th, and a run walks bands of eight rows of
// tiles (at the end four, two, one) by all J tiles, I fastest, so that the workgroups of a die share both operands at any
// time.  Each step is a few additions: divisions would take longer than a stage of a short product.
struct Walk {
    int ni, nj, left, step;          // left: tiles of this workgroup's run from here on
    int split, base, shift, in;      // band of 1 << shift rows of tiles from `base`, tile `in` of the band
    __device__ __forceinline__ void band(int b)
    {
        base = b;
        const int rest = ni - b;
        shift = rest >= 8 ? 3 : rest >= 4 ? 2 : rest >= 2 ? 1 : 0;
    }
    __device__ __forceinline__ void settle()
    {
        while (in >= nj << shift) {
            in -= nj << shift;
            int b = base + (1 << shift);
            if (b >= ni) { b = 0; ++split; }
            band(b);
        }
    }
    __device__ __forceinline__ Walk(int ni_, int nj_, int splits) : ni(ni_), nj(nj_)
    {
        const int n = ni * nj * splits, x = blockIdx.x & 7, q = n >> 3, r = n & 7, at = blockIdx.x >> 3;
        left = q + (x < r) - at;
        step = (gridDim.x + 7) >> 3;               // of a whole number of eights, or a tile for each workgroup
        const int from = x * q + min(x, r) + at, one = ni * nj, b = (from % one) / (nj * 8);
        split = from / one;
        in = from % one - b * nj * 8;
        band(b * 8);
        settle();
    }
    __device__ __forceinline__ bool more() const { return left > step; }
    __device__ __forceinline__ void next()
    {
        left -= step;
        in += step;
        settle();
    }
    __device__ __forceinline__ int i() const { return base + (in & ((1 << shift) - 1)); }
    __device__ __forceinline__ int j() const { return in >> shift; }
};

// A tile at (i0, j0) over stages [first, first + n) of k.
struct Work { int i0, j0, first, n; };

// TI x TJ results by WI x WJ wavefronts; a wavefront holds MI x NJ blocks of 16 x 16.  acc[mi][nj][r] of a lane is
//   i = i_of(mi) + r,   j = j_of(nj).
// I's part of a stage has ring_i places in LDS, J's two: three and two are what 160 KB hold of 256 x 256 (128 x 128: twice a
// compute unit).
// TURNED: I lies with its columns contiguous; results of one lane are then four neighbours in I only.
template <int KIND, int TI_, int TJ_, int WI_, int WJ_, bool TURNED = false> struct Tile {
    using K = Kind<KIND>;
    static_assert(!TURNED || KIND == kTileF32 || KIND == kTileF32x3 || KIND == kTileBf16, "");
    static constexpr int esz = KIND == kTileF32 || KIND == kTileF32x3 ? 4 : 2;
    static constexpr bool split = KIND == kTileF32x3;
    static constexpr bool turned = TURNED;
    static constexpr int kind = KIND, TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, NW = WI * WJ, threads = NW * 64;
    static constexpr int MI = TI / WI / 16, NJ = TJ / WJ / 16;
    static_assert(MI % 2 == 0, "rows of I are ordered by pairs of blocks");
    static constexpr int up256(int n) { return (n + 255) & ~255; }
    static constexpr int oSI = TI * K::row_i, bytes_i = oSI + up256(TI * K::scale_i);
    static constexpr int oSJ = TJ * K::row_j, bytes_j = oSJ + up256(TJ * K::scale_j);
    static constexpr int ring_i = KIND == kTileMx4 || KIND == kTileF32x3 ? 2 : 3, ring_j = 2, ring_bytes = ring_i * bytes_i + ring_j * bytes_j;
    static constexpr int per_cu = 163840 / ring_bytes < 1 ? 1 : 163840 / ring_bytes > 2048 / threads ? 2048 / threads : 163840 / ring_bytes;
    // wavefronts that have to fit a SIMD: where a tile is multiplied a second time (below) the compiler takes more registers than leave room
    // for a unit's second workgroup (gradient of 1000 x 32000 x 1024 by the logits: 556 us instead of 413)
    static constexpr int per_simd = split ? per_cu * NW / 4 : 1;
    using Acc = f32x4[MI][NJ];
    using StagerI = std::conditional_t<TURNED, TurnedStager<TI, K::elems, esz, NW>, Stager<TI, K::row_i, 16, NW, 0>>;
    using StagerJ = Stager<TJ, K::row_j, 16, NW, NJ, TURNED && KIND == kTileBf16>;
    using ScalesI = std::conditional_t<(K::scale_i > 0), Stager<TI, (K::scale_i > 0 ? K::scale_i : 4), 4, NW, 0>, NoStager>;
    using ScalesJ = std::conditional_t<(K::scale_j > 0), Stager<TJ, (K::scale_j > 0 ? K::scale_j : 4), 4, NW, NJ>, NoStager>;
    static constexpr int li = StagerI::per + ScalesI::per, lj = StagerJ::per + ScalesJ::per;       // loads of a wavefront and stage

    static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ int i_of(int mi)
    {
        const int g = lane() >> 4;
        return wave() / WJ * (MI * 16) + (TURNED ? mi * 16 + g * 4 : (mi >> 1) * 32 + g * 8 + (mi & 1) * 4);
    }
    static __device__ __forceinline__ int j_of(int nj) { return wave() % WJ * (NJ * 16) + (lane() & 15) * NJ + nj; }

    // What a wavefront multiplies: blocks of I (those of the next step replace them one by one), and of J for two steps.
    struct Frags {
        u32x4 a[KIND == kTileMx4W || split ? 2 : 1][MI], b[2][NJ];
        uint32_t sa[KIND == kTileMx4W ? 2 : 1][K::scale_i ? MI : 1], sb[2][K::scale_j ? NJ : 1];
    };
    // Where this lane reads: its row of the first block, and the chunk of step 0; steps exchange bits of the chunk.
    struct Places {
        uint32_t a, b, sa, sb, turn = 0;
        __device__ __forceinline__ Places()
        {
            const int r16 = lane() & 15, g = lane() >> 4, ra = wave() / WJ * MI * 16 + r16, rb = wave() % WJ * NJ * 16 + r16;
            a = ra * K::row_i + (g ^ chunk_swap<K::row_i>(r16)) * 16;
            if constexpr (TURNED) {
                // row of step 0 and its bytes there, without the exchange of slots: bfloat16 a row for every four lanes, 8 bytes each
                const int row = KIND == kTileBf16 ? g * 8 + r16 / 4 : g * 4;
                a = row * (TI * esz) + (KIND == kTileBf16 ? r16 % 4 * 8 : r16 * 4);
                turn = StagerI::swap(row);
            }
            b = rb * K::row_j + ((KIND == kTileMx4W ? g * 4 : g) ^ chunk_swap<K::row_j>(r16)) * 16;
            sa = oSI + ra * K::scale_i + g;
            sb = oSJ + rb * K::scale_j + g;
        }
    };
    static __device__ __forceinline__ void read_a(int set, int m, const char *pi, int s, const Places &at, Frags &f)
    {
        if constexpr (TURNED) {
            const char *p = pi + at.a + (((wave() / WJ * MI + m) * 16 * esz) ^ at.turn) + s * (K::elems / 2) * (TI * esz);
            if constexpr (KIND == kTileBf16) {
                using s16x4 = short __attribute__((ext_vector_type(4)));
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p + 4 * TI * esz));
                const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                f.a[set][m] = u32x4{l.x, l.y, h.x, h.y};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) f.a[set][m][j] = *(const uint32_t *)(p + j * TI * esz);
            }
        } else {
            f.a[set][m] = *(const u32x4 *)(pi + (at.a ^ (s * 64)) + m * 16 * K::row_i);
        }
        // a byte of its own for every lane: shifted out of a word that four lanes read, it would hold up the matrix instructions, which
        // wait for results of the vector ALU (6.6 and 4.1 PFLOP/s of 4-bit products with nothing else in the loop)
        if constexpr (K::scale_i > 0) f.sa[set][m] = *(const uint8_t *)(pi + at.sa + s * 4 + m * 16 * K::scale_i);
    }
    static __device__ __forceinline__ void read_b(int set, int n, const char *pj, int s, const Places &at, Frags &f)
    {
        f.b[set][n] = *(const u32x4 *)(pj + (at.b ^ (s * (KIND == kTileMx4W ? 16 : 64))) + n * 16 * K::row_j);
        if constexpr (K::scale_j > 0) f.sb[set][n] = *(const uint8_t *)(pj + at.sb + s * 4 + n * 16 * K::scale_j);
    }
    // Row mi of blocks times the J blocks of `set`.  kTileMx4W: a lane holds the 32 codes of block l / 16 of its row; matrix
    // instruction t of four takes codes 8 t .. + 7 of every lane, and the same k of J.
    static __device__ __forceinline__ void multiply_row(int mi, int set_a, int set_b, int t, const Frags &f, Acc &acc)
    {
        u32x4 a = f.a[set_a][mi];
        if constexpr (KIND == kTileMx4W) a = codes_to_bf16(a[t], scale_value(f.sa[set_a][mi]));
#pragma unroll
        for (int nj = 0; nj < NJ; ++nj) {
            if constexpr (KIND == kTileF32) acc[mi][nj] = mma_f32(a, f.b[set_b][nj], acc[mi][nj]);
            else if constexpr (KIND == kTileMx4) acc[mi][nj] = mma_mx4(a, f.sa[set_a][mi], f.b[set_b][nj], f.sb[set_b][nj], acc[mi][nj]);
            else acc[mi][nj] = mma_bf16(a, f.b[set_b][nj], acc[mi][nj]);
        }
        // here and not where the sums are next used, to which the compiler would move the scaled products, past the loads and the barrier
        if constexpr (KIND == kTileMx4) {
#pragma unroll
            for (int nj = 0; nj < NJ; ++nj) asm volatile("" : "+v"(acc[mi][nj]));
        }
    }

    // The tile of `w` once more, as binary32 products, each lane's operands straight from memory.  Parts of an infinity are no number, nor is
    // its product with a part that is zero, so a tile of split products has a NaN wherever one of its operands is infinite; where the
    // logits of a vocabulary row that is masked by infinite weights are infinite they have to come out so.  A wavefront whose results hold a
    // NaN makes them again; the others go on (cross entropy of 1000 x 32000 x 1024 with one masked vocabulary row 482 us, without 386).
    static __device__ __forceinline__ void multiply_as_they_are(const Operand &I, const Operand &J, const Work &w, Acc &acc)
    {
        const int r16 = lane() & 15, g = lane() >> 4, qi = wave() / WJ * MI * 16 + r16, qj = wave() % WJ * NJ * 16 + r16;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int k0 = w.first * K::elems; k0 < (w.first + w.n) * K::elems; k0 += 16) {
            const int k = k0 + g * 4;
            u32x4 b[NJ];
#pragma unroll
            for (int n = 0; n < NJ; ++n) {
                const int j = w.j0 + row_of_j<NJ>(qj + n * 16);
                b[n] = u32x4{0, 0, 0, 0};
                if (j < J.rows && k * 4 < J.row_bytes) b[n] = *(const u32x4 *)((const char *)J.p + j * J.stride + k * 4);
            }
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) {
                const int q = qi + mi * 16, i = w.i0 + (TURNED ? q : row_of_i(q));
                u32x4 a = {0, 0, 0, 0};
                if constexpr (TURNED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (k + e < I.rows && i * 4 < I.row_bytes) a[e] = *(const uint32_t *)((const char *)I.p + (k + e) * I.stride + i * 4);
                } else {
                    if (i < I.rows && k * 4 < I.row_bytes) a = *(const u32x4 *)((const char *)I.p + i * I.stride + k * 4);
                }
#pragma unroll
                for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = mma_f32(a, b[nj], acc[mi][nj]);
            }
        }
    }

    // Works through the tiles of `walk`.  where(walk): its Work, with n >= 1; before(w): fetches what its results need from memory; finish(w, acc): hands the results on, out of the registers, and says
    // whether it made STORES stores exactly.  LOST_J: results of a row of J that is not finite are lost either way (a token whose hidden state
    // holds an infinity has no finite lse: none of its logits is finite).
    //
    // Stages of all tiles form one stream, of which the loads are two stages ahead of the products: a tile is finished while the
    // first stages of the next one arrive.  Stores count like loads where a wavefront waits for its loads by number: behind a
    // tile whose stores are known in number, the next stage is not waited for longer on their account.
    template <int STORES, bool LOST_J, class Where, class Before, class Finish>
    static __device__ __forceinline__ void work(const Operand &I, const Operand &J, Walk walk, char *lds, Where where, Before before, Finish finish)
    {
        const int wave = Tile::wave(), lane = Tile::lane();
        if (walk.left <= 0) return;
        const Places places;
        __amdgpu_buffer_rsrc_t ri, rj, rsi, rsj;
        StagerI gi;
        StagerJ gj;
        ScalesI hi;
        ScalesJ hj;
        gi.init(I.stride, wave, lane);
        gj.init(J.stride, wave, lane);
        hi.init(I.scale_stride, wave, lane);
        hj.init(J.scale_stride, wave, lane);
        Work w = where(walk);                                    // the tile that is multiplied
        Walk ahead_walk = walk;                                  // the tile that is loaded
        int from_i = 0, ahead = 0, ahead_n = 0;                              // the next stage to be loaded, and where its tile's stages end
        auto stage = [&] {
            if constexpr (TURNED) {
                const int64_t k = (int64_t)ahead * K::elems;
                ri = buffer_of((const char *)I.p + k * I.stride + from_i * esz, (I.rows - 1 - k) * I.stride + I.row_bytes - from_i * esz);
            } else {
                gi.stage(ahead, I.row_bytes);
            }
            gj.stage(ahead, J.row_bytes);
            hi.stage(ahead, I.scale_stride);
            hj.stage(ahead, J.scale_stride);
        };
        auto load_from = [&](const Work &v) {
            const int64_t left_i = I.rows - v.i0, left_j = J.rows - v.j0;
            from_i = v.i0;
            if constexpr (!TURNED) ri = buffer_of((const char *)I.p + v.i0 * I.stride, (left_i - 1) * I.stride + I.row_bytes);
            rj = buffer_of((const char *)J.p + v.j0 * J.stride, (left_j - 1) * J.stride + J.row_bytes);
            if constexpr (K::scale_i > 0) rsi = buffer_of(I.scales + (int64_t)v.i0 * I.scale_stride, left_i * I.scale_stride);
            if constexpr (K::scale_j > 0) rsj = buffer_of(J.scales + (int64_t)v.j0 * J.scale_stride, left_j * J.scale_stride);
            ahead = v.first;
            ahead_n = v.first + v.n;
            stage();
        };
        // Load x of either operand's part of stage `ahead`.  Behind the last tile: its last stage again, into memory that nobody reads.
        auto load_i = [&](int x, char *to) {
            if constexpr (TURNED) gi.issue(x, ri, to, I.stride, wave);
            else if (x < gi.per) gi.issue(x, ri, to, I.stride, wave);
            else hi.issue(x - gi.per, rsi, to + oSI, I.scale_stride, wave);
        };
        auto load_j = [&](int x, char *to) {
            if (x < gj.per) gj.issue(x, rj, to, J.stride, wave);
            else hj.issue(x - gj.per, rsj, to + oSJ, J.scale_stride, wave);
        };
        auto advance = [&] {
            if (ahead + 1 < ahead_n) {
                ++ahead;
                stage();
            } else if (ahead_walk.more()) {
                ahead_walk.next();
                load_from(where(ahead_walk));
            }
        };
        load_from(w);
        // places of I's stages s, s + 1, s + 2, and of J's s, s + 1
        char *i0p = lds, *i1p = lds + bytes_i, *i2p = ring_i == 3 ? lds + 2 * bytes_i : i0p, *j0p = lds + ring_i * bytes_i, *j1p = j0p + bytes_j;
#pragma unroll
        for (int x = 0; x < li; ++x) load_i(x, i0p);
#pragma unroll
        for (int x = 0; x < lj; ++x) load_j(x, j0p);
        advance();
#pragma unroll
        for (int x = 0; x < li; ++x) load_i(x, i1p);
#pragma unroll
        for (int x = 0; x < lj; ++x) load_j(x, j1p);
        advance();
        wait_loads_and_barrier<li + lj>();
        Frags f;
#pragma unroll
        for (int x = 0; x < NJ; ++x) read_b(0, x, j0p, 0, places, f);
#pragma unroll
        for (int x = 0; x < MI; ++x) read_a(0, x, i0p, 0, places, f);
        if constexpr (split) {
#pragma unroll
            for (int x = 0; x < NJ; ++x) read_b(1, x, j0p, 1, places, f);
#pragma unroll
            for (int x = 0; x < MI; ++x) read_a(1, x, i0p, 1, places, f);
        }
        int stores = 0;                                          // 1: STORES stores are younger than the loads that are waited for next
        constexpr int steps = KIND == kTileMx4W ? 4 : K::steps, last = steps - 1;
        constexpr int hold = KIND == kTileMx4W || MI < 4 ? 0 : 1;          // the row of blocks behind which a stage is handed on
        static_assert(steps % 2 == 0, "a stage begins with J's first set of blocks");
        for (;;) {
            before(w);
            Acc acc;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int nj = 0; nj < NJ; ++nj) acc[mi][nj] = f32x4{0.f, 0.f, 0.f, 0.f};
            // The blocks of a step are read while the step before multiplies, each block of I into the place of one that is done
            // with.  Reads and loads are dealt out between the products: a wavefront that issues all its loads at once waits for the
            // others' loads to be taken, with no product under way.  The barrier that hands J's place on lies behind the last reads
            // of the stage, inside its last step.
            auto early_steps = [&] {
#pragma unroll
                for (int t = 0; t < last; ++t) {
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) {
                        constexpr int rows = last * MI, half = MI > 1 ? MI / 2 : 1;
#pragma unroll
                        for (int x = (t * MI + mi) * li / rows; x < (t * MI + mi + 1) * li / rows; ++x)
                            if (ring_i == 3) load_i(x, i2p);
                        // J's blocks within the first half: the next step begins with all of them
#pragma unroll
                        for (int x = mi * NJ / half; x < (mi + 1) * NJ / half && x < NJ; ++x) read_b((t + 1) & 1, x, j0p, t + 1, places, f);
                        multiply_row(mi, 0, t & 1, t, f, acc);
                        if constexpr (KIND != kTileMx4W) read_a(0, mi, i0p, t + 1, places, f);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            auto hand_on = [&] {
                constexpr int young = ring_i == 3 ? li : 0;
                if constexpr (STORES > 0) {
                    wait_loads_and_barrier<young, young + STORES>(__builtin_amdgcn_readfirstlane(stores));
                    stores = 0;
                } else {
                    wait_loads_and_barrier<young>();
                }
            };
            auto last_step = [&] {
                constexpr bool first = KIND == kTileMx4W;
                if (first) hand_on();
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) {
                    multiply_row(mi, 0, last & 1, last, f, acc);
                    if (!first && mi == hold) hand_on();
                    if (mi >= hold) {
                        constexpr int rest = MI - hold, half = rest > 1 ? rest / 2 : 1;
#pragma unroll
                        for (int x = (mi - hold) * lj / rest; x < (mi - hold + 1) * lj / rest; ++x) load_j(x, j0p);
#pragma unroll
                        for (int x = (mi - hold) * li / rest; x < (mi - hold + 1) * li / rest; ++x)
                            if (ring_i == 2) load_i(x, i0p);
#pragma unroll
                        for (int x = (mi - hold) * NJ / half; x < (mi - hold + 1) * NJ / half && x < NJ; ++x) read_b(0, x, j1p, 0, places, f);
#pragma unroll
                        for (int x = mi == hold ? 0 : mi; x <= mi; ++x) read_a(first ? 1 : 0, x, i1p, 0, places, f);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (first) {
#pragma unroll
                    for (int x = 0; x < MI; ++x) { f.a[0][x] = f.a[1][x]; f.sa[0][x] = f.sa[1][x]; }
                }
                advance();
                char *p = i0p; i0p = i1p; i1p = ring_i == 3 ? i2p : p; i2p = p;
                p = j0p; j0p = j1p; j1p = p;
            };
            // Split products: a stage's operands were read while the stage before multiplied, so the barrier that hands both places on comes
            // first; J's blocks are split once, I's as their rows come.
            auto split_stage = [&] {
                if constexpr (split) {
                    hand_on();
                    Split3 b[NJ];
#pragma unroll
                    for (int n = 0; n < NJ; ++n) b[n] = split3(f.b[0][n], f.b[1][n]);
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) {
                        const Split3 a = split3(f.a[0][mi], f.a[1][mi]);
#pragma unroll
                        for (int x = mi * lj / MI; x < (mi + 1) * lj / MI; ++x) load_j(x, j0p);
#pragma unroll
                        for (int x = mi * li / MI; x < (mi + 1) * li / MI; ++x) load_i(x, i0p);
#pragma unroll
                        for (int x = mi * NJ / MI; x < (mi + 1) * NJ / MI; ++x) {
                            read_b(0, x, j1p, 0, places, f);
                            read_b(1, x, j1p, 1, places, f);
                        }
                        read_a(0, mi, i1p, 0, places, f);
                        read_a(1, mi, i1p, 1, places, f);
#pragma unroll
                        for (int p = 0; p < 6; ++p)               // the smallest products first; neighbouring instructions have sums of their own
#pragma unroll
                            for (int n = 0; n < NJ; ++n)
                                acc[mi][n] = mma_bf16(p == 0 ? a.l : p == 2 || p == 3 ? a.m : a.h, p == 1 ? b[n].l : p == 2 || p == 4 ? b[n].m : b[n].h, acc[mi][n]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    advance();
                    char *p = i0p; i0p = i1p; i1p = p; i2p = p;
                    p = j0p; j0p = j1p; j1p = p;
                }
            };
            for (int s = 0; s < w.n; ++s) {
                if constexpr (split) split_stage();
                else {
                    early_steps();
                    last_step();
                }
            }
            if constexpr (split) {
                // an operand's row that is not finite has NaN results throughout, so one of J without any says that I's rows are finite; columns behind
                // those of a turned I hold anything (what lies behind its rows is zeros)
                bool again = LOST_J;
#pragma unroll
                for (int nj = 0; nj < NJ; ++nj) {
                    bool none = true;
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) {
                        const bool behind = TURNED && (w.i0 + i_of(mi)) * 4 >= I.row_bytes;
#pragma unroll
                        for (int r = 0; r < 4; ++r) none &= behind || acc[mi][nj][r] == acc[mi][nj][r];
                    }
                    uint64_t lanes = __ballot(none);
                    if constexpr (LOST_J) {
                        lanes &= lanes >> 32;                    // the four lanes of a row of J
                        lanes &= lanes >> 16;
                        again &= !(lanes & 0xffff);
                    } else {
                        again |= lanes != ~0ull;
                    }
                }
                if (again) multiply_as_they_are(I, J, w, acc);
            }
            stores = finish(w, acc);
            if (!walk.more()) break;
            walk.next();
            w = where(walk);
        }
        wait_loads_and_barrier<0>();                             // no load into LDS outlives the workgroup
    }
};

// Row and column of element base + off, base the same for the workgroup and off below 2^16, of rows of `per`: one long division for the
// workgroup, none for a lane (a division each was what quantising took longest for).
struct RowColumn {
    int r, c;
    __device__ __forceinline__ RowColumn(int64_t base, int off, int per)
    {
        const int64_t r0 = base / per;
        const int in = (int)(base - r0 * per) + off;
        int q = (int)((float)in * (1.f / (float)per));         // off by less than one: in < 2^17
        if (q * per > in) --q;
        if ((q + 1) * per <= in) ++q;
        r = (int)r0 + q;
        c = in - q * per;
    }
};

constexpr int kCUs = 256;
// Workgroups of a launch: as many as are resident at once.
template <class T> inline int grid_of(int64_t tiles) { return (int)(tiles < (int64_t)kCUs * T::per_cu ? tiles : (int64_t)kCUs * T::per_cu); }

}  // namespace tapout
