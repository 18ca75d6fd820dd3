// Internal declarations of the draft head's operators (head_loss.hip, head_mx4.hip, head_api.hip).
#pragma once

#include "head_gemm.h"

namespace tapout {

constexpr int kMx4Pad = 128;         // a row of codes is padded to whole matrix steps
inline int mx4_cols(int cols) { return (cols + kMx4Pad - 1) / kMx4Pad * kMx4Pad; }

// The target of row n if the row counts in the loss: a token of the vocabulary; -1: the row is left out, -2: no such token.
__host__ __device__ __forceinline__ int counted_target(int t, int V) { return t < 0 ? -1 : t < V ? t : -2; }

// A launch with `bytes` of LDS, which has to be asked for from 64 KB on.
template <class F> hipError_t with_lds(const void *kernel, int bytes, F launch)
{
    if (bytes > 65536) {
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    launch();
    return hipGetLastError();
}
inline int up(int a, int b) { return (a + b - 1) / b; }

// ---- cross entropy -----------------------------------------------------------------------------------
struct LossArgs {
    Operand weight, hidden;      // I: vocabulary rows, J: tokens
    int32_t N, V, D, rows_per_seq, B;
    const int32_t *target;       // [N]; NULL: the rows have lists
    float2 *part;                // [N, blocks]: maximum and sum of exp(z - maximum) over a wavefront's vocabulary rows
    int64_t part_cap;            // elements it has room for; a launch that needs more is refused
    float *target_logit;         // [N]
    float *loss, *lse;           // [N]
    uint32_t *flags;             // [B] or NULL
    // rows with lists of tokens in a target's place
    int32_t T;
    const int32_t *ids;          // [N, T] or NULL
    const float *logits, *teacher_lse;          // the teacher's: [N, T]; [N] or NULL
    float *top;                  // [N, T]
};
hipError_t launch_listed_join(const LossArgs &a, int blocks, int dtype, hipStream_t st);       // top, and from it and `part` the rest
hipError_t launch_head_loss(const LossArgs &a, int dtype, hipStream_t st);

// One piece of the vocabulary, rows [v0, v0 + n): its gradient by the logits, both ways round.
struct GradArgs {
    Operand weight, hidden;      // weight: the piece's rows
    int32_t N, V, D, v0, n;
    const int32_t *target;
    const float *lse, *row_weight;
    int32_t listed;              // 1: no target's term, which launch_listed_grad puts in its place
    void *g;                     // [N, n_pad]   n_pad = n rounded up to 64, zeros behind n
    int64_t g_stride;            // elements
    void *gt;                    // [n, N_pad]   N_pad = N rounded up to 32, zeros behind N
    int64_t gt_stride;
};
hipError_t launch_head_grad(const GradArgs &a, int dtype, hipStream_t st);

// Gradients by the listed tokens' logits.  Rows first: which count (state 0, else -1) and what their softmax is multiplied by; then, a piece at a
// time, the elements that lie in it, over what launch_head_grad wrote there.
struct ListedArgs {
    int32_t N, V, T;
    const int32_t *ids;
    const float *logits, *teacher_lse, *lse, *top, *row_weight;
    int32_t *state; float *factor;
};
hipError_t launch_listed_rows(const ListedArgs &a, hipStream_t st);
hipError_t launch_listed_grad(const ListedArgs &a, const GradArgs &piece, int dtype, hipStream_t st);

// dst [cols, rows_pad] = src [rows, cols]^T, zeros behind `rows`; with `target` given, rows that do not count are zeros.
struct TransposeArgs {
    const void *src; int64_t src_stride;       // elements
    void *dst; int64_t dst_stride;
    int32_t rows, cols, rows_pad, V;
    const int32_t *target; const float *lse, *row_weight;
};
hipError_t launch_head_transpose(const TransposeArgs &a, int dtype, hipStream_t st);

// out[j][i] = scale * sum over k of I[i][k] J[j][k], rounded; or, with part given, binary32 partial sums over `splits` runs of k, added to
// what is there unless `first`.  Then I is given turned: I.p[k][i], I.rows steps of k.
struct ProductArgs {
    Operand I, J;
    int32_t ni, nj, k;           // results and length of k in elements (not 0)
    int32_t splits, first;
    float *part;                 // [splits, nj, ni]
    void *out; int64_t out_stride;             // elements
    const float *scale;          // device, or NULL (1); the sums are zeros whatever it is where none of the rows counts
    int32_t rows, V;
    const int32_t *target; const float *lse, *row_weight;
};
hipError_t launch_head_product(const ProductArgs &a, int dtype, hipStream_t st);
int head_product_tiles(int ni, int nj, int dtype);       // tiles of one run of the turned product
int head_product_slots(int nj, int dtype);               // its workgroups resident at a time

// grad_hidden = scale * (sum of the partial sums), rows that do not count: zeros.
struct GradHiddenArgs {
    const float *part; int32_t splits, N, D, K, V;
    void *out; int64_t stride_b, stride_k;     // elements
    const float *scale;
    const int32_t *target; const float *lse, *row_weight;
};
hipError_t launch_head_grad_hidden(const GradHiddenArgs &a, int dtype, hipStream_t st);

// dst [B * K, cols] = src [B, K, cols].
struct PackArgs {
    const void *src; int64_t stride_b, stride_k;
    void *dst;
    int32_t N, K, cols;
};
hipError_t launch_head_pack(const PackArgs &a, int dtype, hipStream_t st);

// ---- 4-bit blocks -------------------------------------------------------------------------------------
struct QuantArgs {
    const void *src; int64_t stride_b, stride_k;    // elements; row r lies at (r / K) * stride_b + (r % K) * stride_k
    int32_t rows, K, cols;
    uint8_t *codes, *scales;                         // [rows, pad / 2], [rows, pad / 32]
};
hipError_t launch_mx4_quantize(const QuantArgs &a, int dtype, hipStream_t st);
struct DequantArgs {
    const uint8_t *codes, *scales;
    int32_t rows, cols;
    void *out; int64_t stride;                       // elements
};
hipError_t launch_mx4_dequantize(const DequantArgs &a, int dtype, hipStream_t st);

// ---- 8-bit blocks -------------------------------------------------------------------------------------
constexpr int kFp8Block = 128;       // elements of a row that share a scale; rows of codes are padded to whole blocks
struct Fp8QuantArgs {
    const void *src; int64_t stride_b, stride_k;     // elements; row r lies at (r / K) * stride_b + (r % K) * stride_k
    int32_t rows, K, cols;
    uint8_t *codes; float *scales;                   // [rows, pad], [rows / block_rows, pad / 128]
};
hipError_t launch_fp8_quantize(const Fp8QuantArgs &a, int block_rows, int dtype, hipStream_t st);
struct Fp8DequantArgs {
    const uint8_t *codes; const float *scales;
    int32_t rows, cols, block_rows;
    void *out; int64_t stride;                       // elements
};
hipError_t launch_fp8_dequantize(const Fp8DequantArgs &a, int dtype, hipStream_t st);

// ---- norm ---------------------------------------------------------------------------------------------
struct Rows { const void *p; int64_t stride_b, stride_k; };       // row r at (r / K) * stride_b + (r % K) * stride_k, elements; p NULL: none
struct NormArgs {
    Rows x, residual, sum, out;
    const void *weight;              // [D]
    float eps;
    int32_t N, K, D;
    uint8_t *codes; float *scales;   // [N, pad], [N, pad / 128], or both NULL
    float *rstd;                     // [N] or NULL
};
hipError_t launch_head_norm(const NormArgs &a, int dtype, hipStream_t st);
struct NormGradArgs {
    Rows grad_out, sum, grad_sum, grad_x;
    const void *weight;
    const float *rstd;
    int32_t N, K, D;
    float *part; int64_t part_cap;   // partial sums of grad_weight: room in floats
    void *grad_weight;               // [D]
};
hipError_t launch_head_norm_grad(const NormGradArgs &a, int dtype, hipStream_t st);

struct LogitsArgs {
    Operand weight, hidden;
    int32_t N, K, V, D;
    const int32_t *k_len;
    void *out; int64_t stride_b, stride_k;
};
hipError_t launch_head_logits(const LogitsArgs &a, int kind, int dtype_out, hipStream_t st);

}  // namespace tapout
