// C ABI of the draft head: argument validation, scratch ownership, launch sequencing.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "head.h"

using namespace tapout;

struct tapout_head {
    tapout_head_config cfg;
    float2 *part = nullptr;  size_t part_cap = 0;             // [N, blocks of a wavefront's vocabulary rows]: at least 64 of them, 32 up to N = 64
    float *target_logit = nullptr;       // [max_rows]
    void *packed = nullptr;              // [max_rows, dim]: hidden states whose rows lie unevenly
    uint8_t *act_codes = nullptr, *act_scales = nullptr;      // quantised hidden states (bfloat16 heads)
    uint8_t *act8_codes = nullptr; float *act8_scales = nullptr;         // the same in 8 bits
    // training only
    char *piece = nullptr;  size_t piece_cap = 0;             // a piece's gradient in both orientations
    void *hidden_t = nullptr;                                 // [dim, max_rows padded to 32]
    float *grad_part = nullptr;  size_t grad_cap = 0;         // partial sums of grad_hidden, or of the norm's grad_weight (floats)
    int32_t *row_state = nullptr; float *row_factor = nullptr;           // [max_rows]: rows with lists, see ListedArgs
    char err[256] = {0};
};

namespace {

constexpr int kMaxRows = 1 << 20, kMaxDim = 65536, kMaxVocab = 1 << 24;
constexpr int64_t kMaxHidden = 1ll << 33, kMaxWeights = 1ll << 35, kMaxBlocks = 1ll << 34, kMaxLists = 1ll << 30;      // elements: a grid has fewer than 2^32 lanes
constexpr int64_t kMaxRowBytes = 8 << 20;            // 255 rows of a tile lie within 2^31 bytes
constexpr size_t kPieceBytes = (size_t)1 << 30;
thread_local char g_err[256] = {0};

tapout_status fail(tapout_head *h, tapout_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(h ? h->err : g_err, 256, fmt, ap);
    va_end(ap);
    return st;
}

tapout_status hip_fail(tapout_head *h, hipError_t e, const char *what) { return fail(h, TAPOUT_EHIP, "%s: %s", what, hipGetErrorString(e)); }

struct DeviceGuard {
    int prev = -1; bool changed = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) changed = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() { if (changed) (void)hipSetDevice(prev); }
};

int size_of(int dtype) { return dtype == TAPOUT_F32 ? 4 : 2; }
int up_to(int a, int b) { return (a + b - 1) / b * b; }

tapout_status check_matrix(tapout_head *h, const tapout_matrix *m, const char *name)
{
    if (!m || !m->ptr) return fail(h, TAPOUT_EINVAL, "%s pointer is NULL", name);
    if (m->dtype != TAPOUT_F32 && m->dtype != TAPOUT_BF16) return fail(h, TAPOUT_EINVAL, "%s: unknown dtype %d", name, m->dtype);
    if (m->stride < 0) return fail(h, TAPOUT_EINVAL, "%s: negative stride", name);
    if ((uintptr_t)m->ptr % 16 || m->stride * size_of(m->dtype) % 16) return fail(h, TAPOUT_EINVAL, "%s: rows must be 16-byte aligned", name);
    return TAPOUT_OK;
}

tapout_status check_hidden(tapout_head *h, const tapout_logits *x, const char *name)
{
    if (!x || !x->ptr) return fail(h, TAPOUT_EINVAL, "%s pointer is NULL", name);
    if (x->dtype != h->cfg.dtype) return fail(h, TAPOUT_EINVAL, "%s: dtype %d, the head's is %d", name, x->dtype, h->cfg.dtype);
    if (x->stride_b < 0 || x->stride_k < 0) return fail(h, TAPOUT_EINVAL, "%s: negative stride", name);
    const int esz = size_of(x->dtype);
    if ((uintptr_t)x->ptr % 16 || x->stride_b * esz % 16 || x->stride_k * esz % 16) return fail(h, TAPOUT_EINVAL, "%s: rows must be 16-byte aligned", name);
    return TAPOUT_OK;
}

tapout_status check_weight(tapout_head *h, const tapout_matrix *m, const char *name, bool written)
{
    if (tapout_status st = check_matrix(h, m, name)) return st;
    if (m->dtype != h->cfg.dtype) return fail(h, TAPOUT_EINVAL, "%s: dtype %d, the head's is %d", name, m->dtype, h->cfg.dtype);
    if (m->stride * size_of(m->dtype) > kMaxRowBytes) return fail(h, TAPOUT_EUNSUPPORTED, "%s: row stride beyond 8 MiB", name);
    if (written && m->stride < h->cfg.dim) return fail(h, TAPOUT_EINVAL, "%s: rows overlap", name);
    return TAPOUT_OK;
}

tapout_status check_shape(tapout_head *h, int B, int K, int V)
{
    if (K < 1) return fail(h, TAPOUT_EINVAL, "K = %d is not positive", K);
    if (B < 0 || (int64_t)B * K > h->cfg.max_rows) return fail(h, TAPOUT_EINVAL, "B * K = %lld outside [0, max_rows = %d]", (long long)B * K, h->cfg.max_rows);
    if (V < 1 || V > h->cfg.vocab) return fail(h, TAPOUT_EINVAL, "V = %d outside [1, vocab = %d]", V, h->cfg.vocab);
    return TAPOUT_OK;
}

// Whether two of the B x K rows of `len` elements share memory.
bool rows_overlap(const tapout_logits *x, int B, int K, int len)
{
    const int64_t b = x->stride_b, k = x->stride_k;
    if (B == 1 || K == 1) return (K > 1 && k < len) || (B > 1 && b < len);
    return !(k >= len && b >= (K - 1) * k + len) && !(b >= len && k >= (B - 1) * b + len);
}

tapout_status check_out(tapout_head *h, const tapout_logits *out, int B, int K, int V)
{
    if (!out || !out->ptr) return fail(h, TAPOUT_EINVAL, "out pointer is NULL");
    if (out->dtype != TAPOUT_F32 && out->dtype != TAPOUT_BF16) return fail(h, TAPOUT_EINVAL, "out: unknown dtype %d", out->dtype);
    if ((uintptr_t)out->ptr % size_of(out->dtype)) return fail(h, TAPOUT_EINVAL, "out pointer is not element-aligned");
    if (out->stride_b < 0 || out->stride_k < 0) return fail(h, TAPOUT_EINVAL, "out: negative stride");
    if (rows_overlap(out, B, K, V)) return fail(h, TAPOUT_EINVAL, "out: rows overlap");
    return TAPOUT_OK;
}

// The hidden states as an operand of N rows: as they lie where their rows are evenly spaced, else packed.
hipError_t hidden_operand(tapout_head *h, const tapout_logits *x, int B, int K, hipStream_t st, Operand *op)
{
    const int N = B * K, D = h->cfg.dim, esz = size_of(x->dtype);
    const int64_t stride = K == 1 ? x->stride_b : x->stride_k;
    const bool even = B == 1 || K == 1 || x->stride_b == (int64_t)K * x->stride_k;
    if (even && stride * esz <= kMaxRowBytes) {
        *op = Operand{x->ptr, stride * esz, N, D * esz, nullptr, 0};
        return hipSuccess;
    }
    const PackArgs a{x->ptr, x->stride_b, x->stride_k, h->packed, N, K, D};
    *op = Operand{h->packed, (int64_t)D * esz, N, D * esz, nullptr, 0};
    return launch_head_pack(a, x->dtype, st);
}

size_t piece_bytes(int n_pad, int N, int esz) { return (size_t)n_pad * ((size_t)N + up_to(N, 32)) * esz; }

// `a`: what the rows are held against, and where the results go.
tapout_status run_loss(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int B, int K, int V, LossArgs a, hipStream_t st, const char *what)
{
    DeviceGuard guard(h->cfg.device);
    hipError_t e = hidden_operand(h, hidden, B, K, st, &a.hidden);
    if (e != hipSuccess) return hip_fail(h, e, "hidden states");
    const int esz = size_of(h->cfg.dtype);
    a.weight = Operand{weight->ptr, weight->stride * esz, V, h->cfg.dim * esz, nullptr, 0};
    a.N = B * K; a.V = V; a.D = h->cfg.dim; a.rows_per_seq = K; a.B = B;
    a.part = h->part; a.part_cap = (int64_t)h->part_cap; a.target_logit = h->target_logit;
    e = launch_head_loss(a, h->cfg.dtype, st);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, what);
}

tapout_status check_lists(tapout_head *h, int B, int K, int T)
{
    if (T < 1 || T > TAPOUT_MAX_TOP) return fail(h, TAPOUT_EINVAL, "T = %d outside [1, %d]", T, TAPOUT_MAX_TOP);
    if ((int64_t)B * K * T > kMaxLists) return fail(h, TAPOUT_EUNSUPPORTED, "B * K * T beyond 2^30");
    return TAPOUT_OK;
}

tapout_status check_grad(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int B, int K, int V,
                         const tapout_logits *grad_hidden, const tapout_matrix *grad_weight)
{
    if (!h->cfg.training) return fail(h, TAPOUT_EINVAL, "the head was created without training = 1");
    if (tapout_status st = check_shape(h, B, K, V)) return st;
    if (tapout_status st = check_weight(h, weight, "weight", false)) return st;
    if (tapout_status st = check_weight(h, grad_weight, "grad_weight", true)) return st;
    if (B * K == 0) return TAPOUT_OK;
    if (tapout_status st = check_hidden(h, hidden, "hidden")) return st;
    if (tapout_status st = check_hidden(h, grad_hidden, "grad_hidden")) return st;
    if (rows_overlap(grad_hidden, B, K, h->cfg.dim)) return fail(h, TAPOUT_EINVAL, "grad_hidden: rows overlap");
    return TAPOUT_OK;
}

// target: the rows' targets, or, with lists, their states (written here).
tapout_status run_grad(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int B, int K, int V,
                       const int32_t *target, const float *lse, const float *row_weight, const ListedArgs *lists, const float *scale,
                       const tapout_logits *grad_hidden, const tapout_matrix *grad_weight, hipStream_t st)
{
    const int N = B * K, D = h->cfg.dim, dt = h->cfg.dtype, esz = size_of(dt);
    DeviceGuard guard(h->cfg.device);
    if (N == 0) {                                              // a transposition of nothing, padded: zeros
        const TransposeArgs t{nullptr, 0, (void *)grad_weight->ptr, grad_weight->stride, 0, V, D, V, nullptr, nullptr, nullptr};
        const hipError_t e = launch_head_transpose(t, dt, st);
        return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "grad_weight");
    }
    const int N_pad = up_to(N, 32);
    Operand x{};
    hipError_t e = hidden_operand(h, hidden, B, K, st, &x);
    if (e != hipSuccess) return hip_fail(h, e, "hidden states");
    if (lists) {
        e = launch_listed_rows(*lists, st);
        if (e != hipSuccess) return hip_fail(h, e, "lists");
    }
    const TransposeArgs t{x.p, x.stride / esz, h->hidden_t, N_pad, N, D, N_pad, V, target, lse, row_weight};
    e = launch_head_transpose(t, dt, st);
    if (e != hipSuccess) return hip_fail(h, e, "hidden states transposed");
    // pieces of the vocabulary of equal length, as long as the scratch allows
    const size_t per = piece_bytes(1, N, esz);
    const int most = (int)std::min<size_t>(up_to(V, 256), h->piece_cap / per / 256 * 256);
    const int pieces = (V + most - 1) / most, len = up_to((V + pieces - 1) / pieces, 256);
    // runs of k of the product by the hidden states: as many as there are workgroups for at a time (twice as many: 293 us instead of 192 at
    // 1503 rows, dim = 1120, V = 50257, bfloat16), each long enough to be worth its partial sums
    const int tiles = head_product_tiles(D, N, dt), stages = up_to(std::min(len, V), 64) / (dt == TAPOUT_F32 ? 32 : 64);
    int splits = std::max(1, std::min({head_product_slots(N, dt) / tiles, stages / 4, (int)(h->grad_cap / ((size_t)N * D))}));
    splits = (stages + (stages + splits - 1) / splits - 1) / ((stages + splits - 1) / splits);        // runs of equal length, none of them empty
    for (int v0 = 0; v0 < V; v0 += len) {
        const int n = std::min(len, V - v0), n_pad = up_to(n, 64);
        const char *rows = (const char *)weight->ptr + v0 * weight->stride * esz;
        char *g = h->piece, *gt = g + (size_t)N * n_pad * esz;
        GradArgs a{};
        a.weight = Operand{rows, weight->stride * esz, n, D * esz, nullptr, 0};
        a.hidden = x;
        a.N = N; a.V = V; a.D = D; a.v0 = v0; a.n = n;
        a.target = target; a.lse = lse; a.row_weight = lists ? lists->factor : row_weight; a.listed = lists != nullptr;
        a.g = g; a.g_stride = n_pad; a.gt = gt; a.gt_stride = N_pad;
        e = launch_head_grad(a, dt, st);
        if (e != hipSuccess) return hip_fail(h, e, "head_grad");
        if (lists) {
            e = launch_listed_grad(*lists, a, dt, st);
            if (e != hipSuccess) return hip_fail(h, e, "lists");
        }
        ProductArgs p{};
        p.I = a.weight;
        p.J = Operand{g, (int64_t)n_pad * esz, N, n_pad * esz, nullptr, 0};
        p.ni = D; p.nj = N; p.k = n_pad; p.splits = splits; p.first = v0 == 0; p.part = h->grad_part;
        e = launch_head_product(p, dt, st);
        if (e != hipSuccess) return hip_fail(h, e, "grad_hidden");
        p = ProductArgs{};
        p.I = Operand{h->hidden_t, (int64_t)N_pad * esz, D, N_pad * esz, nullptr, 0};
        p.J = Operand{gt, (int64_t)N_pad * esz, n, N_pad * esz, nullptr, 0};
        p.ni = D; p.nj = n; p.k = N_pad; p.splits = 1;
        p.out = (char *)grad_weight->ptr + v0 * grad_weight->stride * esz; p.out_stride = grad_weight->stride; p.scale = scale;
        p.rows = N; p.V = V; p.target = target; p.lse = lse; p.row_weight = row_weight;
        e = launch_head_product(p, dt, st);
        if (e != hipSuccess) return hip_fail(h, e, "grad_weight");
    }
    const GradHiddenArgs a{h->grad_part, splits, N, D, K, V, (void *)grad_hidden->ptr, grad_hidden->stride_b, grad_hidden->stride_k,
                           scale, target, lse, row_weight};
    e = launch_head_grad_hidden(a, dt, st);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "grad_hidden");
}

// A row operand of the norm: NULL where it is optional and not wanted.
tapout_status norm_rows(tapout_head *h, const tapout_logits *x, const char *name, bool required, bool written, int B, int K, Rows *out)
{
    *out = Rows{nullptr, 0, 0};
    if (!x && !required) return TAPOUT_OK;
    if (tapout_status st = check_hidden(h, x, name)) return st;
    if (written && rows_overlap(x, B, K, h->cfg.dim)) return fail(h, TAPOUT_EINVAL, "%s: rows overlap", name);
    *out = Rows{x->ptr, x->stride_b, x->stride_k};
    return TAPOUT_OK;
}

tapout_status check_fp8(tapout_head *h, const uint8_t *codes, const float *scales, const char *what)
{
    if (!codes || !scales) return fail(h, TAPOUT_EINVAL, "%s: codes or scales is NULL", what);
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4) return fail(h, TAPOUT_EINVAL, "%s: codes must be 16-byte aligned, scales 4-byte aligned", what);
    return TAPOUT_OK;
}

tapout_status check_fp8_matrix(const tapout_matrix *m, const char *name, int rows, int cols, int block_rows)
{
    if (rows < 0) return fail(nullptr, TAPOUT_EINVAL, "rows = %d is negative", rows);
    if (cols < 32 || cols % 32 || cols > kMaxDim) return fail(nullptr, TAPOUT_EINVAL, "cols = %d is not a multiple of 32 in [32, %d]", cols, kMaxDim);
    if (block_rows != 1 && block_rows != kFp8Block) return fail(nullptr, TAPOUT_EUNSUPPORTED, "block_rows = %d: 1 or %d", block_rows, kFp8Block);
    if ((int64_t)rows * mx4_cols(cols) > kMaxBlocks) return fail(nullptr, TAPOUT_EUNSUPPORTED, "rows * cols beyond 2^34");
    return rows ? check_matrix(nullptr, m, name) : TAPOUT_OK;
}

}  // namespace

extern "C" {

tapout_status tapout_head_create(tapout_head **out, const tapout_head_config *cfg)
{
    if (!out) return fail(nullptr, TAPOUT_EINVAL, "out is NULL");
    *out = nullptr;
    if (!cfg) return fail(nullptr, TAPOUT_EINVAL, "cfg is NULL");
    if (cfg->max_rows < 1 || cfg->max_rows > kMaxRows) return fail(nullptr, TAPOUT_EINVAL, "max_rows = %d outside [1, %d]", cfg->max_rows, kMaxRows);
    if (cfg->dim < 32 || cfg->dim > kMaxDim || cfg->dim % 32) return fail(nullptr, TAPOUT_EINVAL, "dim = %d is not a multiple of 32 in [32, %d]", cfg->dim, kMaxDim);
    if (cfg->vocab < 1 || cfg->vocab > kMaxVocab) return fail(nullptr, TAPOUT_EINVAL, "vocab = %d outside [1, %d]", cfg->vocab, kMaxVocab);
    if (cfg->dtype != TAPOUT_F32 && cfg->dtype != TAPOUT_BF16) return fail(nullptr, TAPOUT_EINVAL, "unknown dtype %d", cfg->dtype);
    if (cfg->training != 0 && cfg->training != 1) return fail(nullptr, TAPOUT_EINVAL, "training must be 0 or 1");
    if ((int64_t)cfg->max_rows * cfg->dim > kMaxHidden) return fail(nullptr, TAPOUT_EUNSUPPORTED, "max_rows * dim beyond 2^33");
    if ((int64_t)cfg->vocab * cfg->dim > kMaxWeights) return fail(nullptr, TAPOUT_EUNSUPPORTED, "vocab * dim beyond 2^35");
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || cfg->device < 0 || cfg->device >= ndev)
        return fail(nullptr, TAPOUT_EHIP, "device %d not available (%d HIP devices)", cfg->device, ndev);
    tapout_head *h = new (std::nothrow) tapout_head;
    if (!h) return fail(nullptr, TAPOUT_ENOMEM, "host allocation failed");
    h->cfg = *cfg;
    DeviceGuard guard(cfg->device);
    const size_t N = cfg->max_rows, D = cfg->dim, esz = size_of(cfg->dtype), P = mx4_cols(cfg->dim);
    const size_t blocks = (cfg->vocab + 127) / 128;
    h->part_cap = (N + std::min<size_t>(N, 64)) * 2 * blocks;
    bool ok = hipMalloc(&h->part, h->part_cap * sizeof(float2)) == hipSuccess
           && hipMalloc(&h->target_logit, N * sizeof(float)) == hipSuccess
           && hipMalloc(&h->packed, N * D * esz) == hipSuccess
           && hipMalloc(&h->act8_codes, N * P) == hipSuccess && hipMalloc(&h->act8_scales, N * (P / kFp8Block) * sizeof(float)) == hipSuccess;
    if (ok && cfg->dtype == TAPOUT_BF16)
        ok = hipMalloc(&h->act_codes, N * P / 2) == hipSuccess && hipMalloc(&h->act_scales, N * P / 32) == hipSuccess;
    if (ok && cfg->training) {
        h->piece_cap = std::min(piece_bytes(up_to(cfg->vocab, 256), (int)N, (int)esz), std::max(kPieceBytes, piece_bytes(256, (int)N, (int)esz)));
        h->grad_cap = std::max(N * D, (size_t)16 << 20);
        ok = hipMalloc(&h->piece, h->piece_cap) == hipSuccess
          && hipMalloc(&h->hidden_t, D * up_to((int)N, 32) * esz) == hipSuccess
          && hipMalloc(&h->grad_part, h->grad_cap * sizeof(float)) == hipSuccess
          && hipMalloc(&h->row_state, N * sizeof(int32_t)) == hipSuccess && hipMalloc(&h->row_factor, N * sizeof(float)) == hipSuccess;
    }
    if (!ok) {
        (void)hipGetLastError();
        tapout_head_destroy(h);
        return fail(nullptr, TAPOUT_ENOMEM, "device allocation failed");
    }
    *out = h;
    return TAPOUT_OK;
}

tapout_status tapout_head_destroy(tapout_head *h)
{
    if (!h) return TAPOUT_OK;
    DeviceGuard guard(h->cfg.device);
    (void)hipFree(h->part); (void)hipFree(h->target_logit); (void)hipFree(h->packed); (void)hipFree(h->act_codes); (void)hipFree(h->act_scales);
    (void)hipFree(h->act8_codes); (void)hipFree(h->act8_scales);
    (void)hipFree(h->piece); (void)hipFree(h->hidden_t); (void)hipFree(h->grad_part); (void)hipFree(h->row_state); (void)hipFree(h->row_factor);
    delete h;
    return TAPOUT_OK;
}

const char *tapout_head_last_error(const tapout_head *h) { return h ? h->err : g_err; }

tapout_status tapout_mx4_quantize(const tapout_matrix *x, int32_t rows, int32_t cols, uint8_t *codes, uint8_t *scales, void *stream)
{
    if (rows < 0) return fail(nullptr, TAPOUT_EINVAL, "rows = %d is negative", rows);
    if (cols < 32 || cols % 32 || cols > kMaxDim) return fail(nullptr, TAPOUT_EINVAL, "cols = %d is not a multiple of 32 in [32, %d]", cols, kMaxDim);
    if ((int64_t)rows * mx4_cols(cols) > kMaxBlocks) return fail(nullptr, TAPOUT_EUNSUPPORTED, "rows * cols beyond 2^34");
    if (rows == 0) return TAPOUT_OK;
    if (tapout_status st = check_matrix(nullptr, x, "x")) return st;
    if (!codes || !scales) return fail(nullptr, TAPOUT_EINVAL, "codes or scales is NULL");
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4) return fail(nullptr, TAPOUT_EINVAL, "codes must be 16-byte aligned, scales 4-byte aligned");
    const QuantArgs a{x->ptr, x->stride, 0, rows, 1, cols, codes, scales};
    const hipError_t e = launch_mx4_quantize(a, x->dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(nullptr, e, "mx4_quantize");
}

tapout_status tapout_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int32_t rows, int32_t cols, const tapout_matrix *out, void *stream)
{
    if (rows < 0) return fail(nullptr, TAPOUT_EINVAL, "rows = %d is negative", rows);
    if (cols < 32 || cols % 32 || cols > kMaxDim) return fail(nullptr, TAPOUT_EINVAL, "cols = %d is not a multiple of 32 in [32, %d]", cols, kMaxDim);
    if ((int64_t)rows * mx4_cols(cols) > kMaxBlocks) return fail(nullptr, TAPOUT_EUNSUPPORTED, "rows * cols beyond 2^34");
    if (rows == 0) return TAPOUT_OK;
    if (tapout_status st = check_matrix(nullptr, out, "out")) return st;
    if (out->stride < cols && rows > 1) return fail(nullptr, TAPOUT_EINVAL, "out: rows overlap");
    if (!codes || !scales) return fail(nullptr, TAPOUT_EINVAL, "codes or scales is NULL");
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4) return fail(nullptr, TAPOUT_EINVAL, "codes must be 16-byte aligned, scales 4-byte aligned");
    const DequantArgs a{codes, scales, rows, cols, (void *)out->ptr, out->stride};
    const hipError_t e = launch_mx4_dequantize(a, out->dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(nullptr, e, "mx4_dequantize");
}

tapout_status tapout_head_logits_mx4(tapout_head *h, const tapout_logits *hidden, const uint8_t *codes, const uint8_t *scales,
                                     int32_t B, int32_t K, int32_t V, const int32_t *k_len, int32_t act_bits, const tapout_logits *out, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (h->cfg.dtype != TAPOUT_BF16) return fail(h, TAPOUT_EUNSUPPORTED, "4-bit heads multiply bfloat16 hidden states only");
    if (tapout_status st = check_shape(h, B, K, V)) return st;
    if (B * K == 0) return TAPOUT_OK;
    if (tapout_status st = check_hidden(h, hidden, "hidden")) return st;
    if (!codes || !scales) return fail(h, TAPOUT_EINVAL, "codes or scales is NULL");
    if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4) return fail(h, TAPOUT_EINVAL, "codes must be 16-byte aligned, scales 4-byte aligned");
    if (act_bits != 16 && act_bits != 4) return fail(h, TAPOUT_EUNSUPPORTED, "act_bits = %d: 16 or 4", act_bits);
    if (tapout_status st = check_out(h, out, B, K, V)) return st;
    const int N = B * K, D = h->cfg.dim, P = mx4_cols(D);
    DeviceGuard guard(h->cfg.device);
    hipStream_t st = (hipStream_t)stream;
    LogitsArgs a{};
    a.weight = Operand{codes, P / 2, V, P / 2, scales, P / 32};
    a.N = N; a.K = K; a.V = V; a.D = P;
    a.k_len = k_len; a.out = (void *)out->ptr; a.stride_b = out->stride_b; a.stride_k = out->stride_k;
    hipError_t e;
    if (act_bits == 4) {
        const QuantArgs q{hidden->ptr, hidden->stride_b, hidden->stride_k, N, K, D, h->act_codes, h->act_scales};
        e = launch_mx4_quantize(q, TAPOUT_BF16, st);
        a.hidden = Operand{h->act_codes, P / 2, N, P / 2, h->act_scales, P / 32};
    } else {
        e = hidden_operand(h, hidden, B, K, st, &a.hidden);
    }
    if (e != hipSuccess) return hip_fail(h, e, "hidden states");
    e = launch_head_logits(a, act_bits == 4 ? kTileMx4 : kTileMx4W, out->dtype, st);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "head_logits");
}

tapout_status tapout_fp8_quantize(const tapout_matrix *x, int32_t rows, int32_t cols, int32_t block_rows, uint8_t *codes, float *scales, void *stream)
{
    if (tapout_status st = check_fp8_matrix(x, "x", rows, cols, block_rows)) return st;
    if (rows == 0) return TAPOUT_OK;
    if (tapout_status st = check_fp8(nullptr, codes, scales, "x")) return st;
    const Fp8QuantArgs a{x->ptr, x->stride, 0, rows, 1, cols, codes, scales};
    const hipError_t e = launch_fp8_quantize(a, block_rows, x->dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(nullptr, e, "fp8_quantize");
}

tapout_status tapout_fp8_dequantize(const uint8_t *codes, const float *scales, int32_t rows, int32_t cols, int32_t block_rows, const tapout_matrix *out, void *stream)
{
    if (tapout_status st = check_fp8_matrix(out, "out", rows, cols, block_rows)) return st;
    if (rows == 0) return TAPOUT_OK;
    if (out->stride < cols && rows > 1) return fail(nullptr, TAPOUT_EINVAL, "out: rows overlap");
    if (tapout_status st = check_fp8(nullptr, codes, scales, "codes")) return st;
    const Fp8DequantArgs a{codes, scales, rows, cols, block_rows, (void *)out->ptr, out->stride};
    const hipError_t e = launch_fp8_dequantize(a, out->dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(nullptr, e, "fp8_dequantize");
}

tapout_status tapout_head_norm(tapout_head *h, const tapout_logits *x, const tapout_logits *residual, const void *weight, float eps, int32_t B, int32_t K,
                               const tapout_logits *sum, const tapout_logits *out, uint8_t *codes, float *scales, float *rstd, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_shape(h, B, K, 1)) return st;
    if (!(eps >= 0.f) || !(eps < INFINITY)) return fail(h, TAPOUT_EINVAL, "eps = %g is not a finite number from 0 on", (double)eps);
    if (B * K == 0) return TAPOUT_OK;
    NormArgs a{};
    if (tapout_status st = norm_rows(h, x, "x", true, false, B, K, &a.x)) return st;
    if (tapout_status st = norm_rows(h, residual, "residual", false, false, B, K, &a.residual)) return st;
    if (tapout_status st = norm_rows(h, sum, "sum", false, true, B, K, &a.sum)) return st;
    if (tapout_status st = norm_rows(h, out, "out", false, true, B, K, &a.out)) return st;
    if (!weight) return fail(h, TAPOUT_EINVAL, "weight is NULL");
    if ((uintptr_t)weight % 16) return fail(h, TAPOUT_EINVAL, "weight must be 16-byte aligned");
    if (codes || scales)
        if (tapout_status st = check_fp8(h, codes, scales, "norm")) return st;
    DeviceGuard guard(h->cfg.device);
    a.weight = weight; a.eps = eps; a.N = B * K; a.K = K; a.D = h->cfg.dim;
    a.codes = codes; a.scales = scales; a.rstd = rstd;
    const hipError_t e = launch_head_norm(a, h->cfg.dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "head_norm");
}

tapout_status tapout_head_norm_grad(tapout_head *h, const tapout_logits *grad_out, const tapout_logits *sum, const void *weight, const float *rstd,
                                    const tapout_logits *grad_sum, int32_t B, int32_t K, const tapout_logits *grad_x, void *grad_weight, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (!h->cfg.training) return fail(h, TAPOUT_EINVAL, "the head was created without training = 1");
    if (tapout_status st = check_shape(h, B, K, 1)) return st;
    if (!grad_weight) return fail(h, TAPOUT_EINVAL, "grad_weight is NULL");
    if ((uintptr_t)grad_weight % 16) return fail(h, TAPOUT_EINVAL, "grad_weight must be 16-byte aligned");
    DeviceGuard guard(h->cfg.device);
    const int D = h->cfg.dim;
    if (B * K == 0) {                                          // a transposition of nothing: zeros (one column)
        const TransposeArgs t{nullptr, 0, grad_weight, D, 0, 1, D, 0, nullptr, nullptr, nullptr};
        const hipError_t e = launch_head_transpose(t, h->cfg.dtype, (hipStream_t)stream);
        return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "grad_weight");
    }
    NormGradArgs a{};
    if (tapout_status st = norm_rows(h, grad_out, "grad_out", true, false, B, K, &a.grad_out)) return st;
    if (tapout_status st = norm_rows(h, sum, "sum", true, false, B, K, &a.sum)) return st;
    if (tapout_status st = norm_rows(h, grad_sum, "grad_sum", false, false, B, K, &a.grad_sum)) return st;
    if (tapout_status st = norm_rows(h, grad_x, "grad_x", true, true, B, K, &a.grad_x)) return st;
    if (!weight || !rstd) return fail(h, TAPOUT_EINVAL, "weight or rstd is NULL");
    if ((uintptr_t)weight % 16) return fail(h, TAPOUT_EINVAL, "weight must be 16-byte aligned");
    a.weight = weight; a.rstd = rstd; a.N = B * K; a.K = K; a.D = D;
    a.part = h->grad_part; a.part_cap = (int64_t)h->grad_cap; a.grad_weight = grad_weight;
    const hipError_t e = launch_head_norm_grad(a, h->cfg.dtype, (hipStream_t)stream);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "head_norm_grad");
}

tapout_status tapout_head_logits_fp8(tapout_head *h, const tapout_logits *hidden, const uint8_t *act_codes, const float *act_scales,
                                     const uint8_t *codes, const float *scales, int32_t B, int32_t K, int32_t V, const int32_t *k_len,
                                     const tapout_logits *out, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_shape(h, B, K, V)) return st;
    if (B * K == 0) return TAPOUT_OK;
    if (hidden && (act_codes || act_scales)) return fail(h, TAPOUT_EINVAL, "hidden states are given twice: as they are and in 8 bits");
    if (hidden || (!act_codes && !act_scales)) {
        if (tapout_status st = check_hidden(h, hidden, "hidden")) return st;
    } else if (tapout_status st = check_fp8(h, act_codes, act_scales, "hidden")) return st;
    if (tapout_status st = check_fp8(h, codes, scales, "weight")) return st;
    if (tapout_status st = check_out(h, out, B, K, V)) return st;
    const int N = B * K, D = h->cfg.dim, P = mx4_cols(D);
    DeviceGuard guard(h->cfg.device);
    hipStream_t st = (hipStream_t)stream;
    if (hidden) {
        const Fp8QuantArgs q{hidden->ptr, hidden->stride_b, hidden->stride_k, N, K, D, h->act8_codes, h->act8_scales};
        const hipError_t e = launch_fp8_quantize(q, 1, h->cfg.dtype, st);
        if (e != hipSuccess) return hip_fail(h, e, "hidden states");
        act_codes = h->act8_codes; act_scales = h->act8_scales;
    }
    const int scale_bytes = P / kFp8Block * (int)sizeof(float);
    LogitsArgs a{};
    a.weight = Operand{codes, P, V, P, (const uint8_t *)scales, scale_bytes};
    a.hidden = Operand{act_codes, P, N, P, (const uint8_t *)act_scales, scale_bytes};
    a.N = N; a.K = K; a.V = V; a.D = P;
    a.k_len = k_len; a.out = (void *)out->ptr; a.stride_b = out->stride_b; a.stride_k = out->stride_k;
    const hipError_t e = launch_head_logits(a, kTileF8, out->dtype, st);
    return e == hipSuccess ? TAPOUT_OK : hip_fail(h, e, "head_logits_fp8");
}

tapout_status tapout_head_loss(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int32_t B, int32_t K, int32_t V,
                               const int32_t *target, float *loss, float *lse, uint32_t *flags, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_shape(h, B, K, V)) return st;
    if (B * K == 0) return TAPOUT_OK;
    if (tapout_status st = check_hidden(h, hidden, "hidden")) return st;
    if (tapout_status st = check_weight(h, weight, "weight", false)) return st;
    if (!target || !loss || !lse) return fail(h, TAPOUT_EINVAL, "target, loss or lse is NULL");
    LossArgs a{};
    a.target = target; a.loss = loss; a.lse = lse; a.flags = flags;
    return run_loss(h, hidden, weight, B, K, V, a, (hipStream_t)stream, "head_loss");
}

tapout_status tapout_head_distill(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int32_t B, int32_t K, int32_t V,
                                  const int32_t *top_ids, const float *top_logits, int32_t T, const float *teacher_lse,
                                  float *loss, float *lse, float *top, uint32_t *flags, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_shape(h, B, K, V)) return st;
    if (tapout_status st = check_lists(h, B, K, T)) return st;
    if (B * K == 0) return TAPOUT_OK;
    if (tapout_status st = check_hidden(h, hidden, "hidden")) return st;
    if (tapout_status st = check_weight(h, weight, "weight", false)) return st;
    if (!top_ids || !top_logits || !loss || !lse || !top) return fail(h, TAPOUT_EINVAL, "top_ids, top_logits, loss, lse or top is NULL");
    LossArgs a{};
    a.T = T; a.ids = top_ids; a.logits = top_logits; a.teacher_lse = teacher_lse; a.top = top;
    a.loss = loss; a.lse = lse; a.flags = flags;
    return run_loss(h, hidden, weight, B, K, V, a, (hipStream_t)stream, "head_distill");
}

tapout_status tapout_head_loss_grad(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int32_t B, int32_t K, int32_t V,
                                    const int32_t *target, const float *lse, const float *row_weight, const float *scale,
                                    const tapout_logits *grad_hidden, const tapout_matrix *grad_weight, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_grad(h, hidden, weight, B, K, V, grad_hidden, grad_weight)) return st;
    if (B * K > 0 && (!target || !lse)) return fail(h, TAPOUT_EINVAL, "target or lse is NULL");
    return run_grad(h, hidden, weight, B, K, V, target, lse, row_weight, nullptr, scale, grad_hidden, grad_weight, (hipStream_t)stream);
}

tapout_status tapout_head_distill_grad(tapout_head *h, const tapout_logits *hidden, const tapout_matrix *weight, int32_t B, int32_t K, int32_t V,
                                       const int32_t *top_ids, const float *top_logits, int32_t T, const float *teacher_lse,
                                       const float *lse, const float *top, const float *row_weight, const float *scale,
                                       const tapout_logits *grad_hidden, const tapout_matrix *grad_weight, void *stream)
{
    if (!h) return fail(nullptr, TAPOUT_EINVAL, "head is NULL");
    if (tapout_status st = check_grad(h, hidden, weight, B, K, V, grad_hidden, grad_weight)) return st;
    if (tapout_status st = check_lists(h, B, K, T)) return st;
    const int N = B * K;
    if (N > 0 && (!top_ids || !top_logits || !lse || !top)) return fail(h, TAPOUT_EINVAL, "top_ids, top_logits, lse or top is NULL");
    const ListedArgs lists{N, V, T, top_ids, top_logits, teacher_lse, lse, top, row_weight, h->row_state, h->row_factor};
    return run_grad(h, hidden, weight, B, K, V, h->row_state, lse, nullptr, &lists, scale, grad_hidden, grad_weight, (hipStream_t)stream);
}

}  // extern "C"
