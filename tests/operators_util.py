"""Plain 64-bit forms of the norm, the 8-bit blocks, the filtered sampling and the distillation, and the error bounds that the tests
hold the kernels to (torch, on the CPU)."""
import math

import torch

from tests import head_util as hu

U32 = hu.U32                           # half a step of binary32
HALF = hu.HALF
TOP = 448.0
INV_TOP = torch.tensor(1.0, dtype=torch.float32) / torch.tensor(TOP, dtype=torch.float32)


# ---- 8-bit blocks --------------------------------------------------------------------------------------------
def fp8(x, block_rows=1):
    """x [rows, cols]: (codes as values of the 8-bit type [rows, P], float64, scales float32 [ceil(rows / block_rows), P / 128]); every step is
    defined in binary32 with one rounding."""
    rows, cols = x.shape
    R, P = -(-rows // block_rows), -(-cols // 128) * 128
    y = torch.zeros(R * block_rows, P, dtype=torch.float32)
    y[:rows, :cols] = x.float()
    y = y.view(R, block_rows, P // 128, 128)
    bad = ~torch.isfinite(y).all(3, keepdim=True).all(1, keepdim=True)
    top = torch.where(bad, 1.0, y.abs().amax((1, 3), keepdim=True)).clamp(min=TOP * 2.0 ** -126)
    scale = torch.where(bad, math.nan, top * INV_TOP)
    q = (torch.where(bad, 0.0, y) / torch.where(bad, 1.0, scale)).to(torch.float8_e4m3fn).double()
    q = torch.where(bad, math.nan, q)
    return q.reshape(R * block_rows, P)[:rows], scale.view(R, P // 128)


def spread(scale, rows, block_rows=1):
    return scale.double().repeat_interleave(block_rows, 0).repeat_interleave(128, 1)[:rows]


def code_values(codes):
    return codes.cpu().view(torch.float8_e4m3fn).double()


def logits_fp8(qa, sa, qw, sw, dtype):
    """(z, bound) of codes' values qa [N, P], qw [V, P] with their scales.  Each block of 128 products leaves the matrix unit in binary32; of the 8-bit ones
    (results in bfloat16) each product may be off by 2^-16 of the block's largest, products of bfloat16 are summed in binary32.  The block's factor, the
    products with it and the sums: two roundings a block."""
    N, V, nb = qa.shape[0], qw.shape[0], qa.shape[1] // 128
    z = torch.zeros(N, V, dtype=torch.float64)
    off = torch.zeros_like(z)
    size = torch.zeros_like(z)
    for b in range(nb):
        s = sa[:, b].double()[:, None] * sw[torch.arange(V) // 128, b].double()[None]
        p = qa[:, None, b * 128:(b + 1) * 128] * qw[None, :, b * 128:(b + 1) * 128]
        z += s * p.sum(-1)
        size += s * p.abs().sum(-1)
        off += s * (2.0 ** -9 * p.abs().amax(-1) if dtype == torch.bfloat16 else 130 * 2 * U32 * p.abs().sum(-1))
    return z, off + 2 * (nb + 2) * U32 * size + HALF[dtype] * z.abs() * (dtype == torch.bfloat16)


# ---- norm ------------------------------------------------------------------------------------------------------
def norm(s, w, eps):
    """(y, rstd) of the rows s [N, D], float64."""
    r = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s * r * w, r


# rstd is rounded once; s r and that times w: once each
def norm_bound(y, dtype):
    return 4 * U32 * y.abs() + (HALF[dtype] * y.abs() * (1 + 4 * U32) if dtype == torch.bfloat16 else 0) + 1e-44


def norm_grad(g, s, w, eps, more, dtype):
    """(dx, dw, bounds) in float64."""
    _, r = norm(s, w, eps)
    h, u = s * r, g * w
    D, N = s.shape[1], s.shape[0]
    mean = (u * h).mean(-1, keepdim=True)
    dx = r * (u - h * mean)
    # u and h are off by a rounding and by two, their products' sums (in binary64) by that; the difference, r and the sum with the other gradient: one each
    off = 4 * U32 * r * (u.abs() + 2 * h.abs() * mean.abs() + 2 * h.abs() * (u * h).abs().mean(-1, keepdim=True))
    if more is not None:
        dx = dx + more
        off = off + 2 * U32 * dx.abs()
    dw = (g * h).sum(0)
    dw_off = (N + 64) * 2 * U32 * (g * h).abs().sum(0)
    return dx, dw, off + (HALF[dtype] + U32) * dx.abs() + 1e-44, dw_off + (HALF[dtype] + U32) * (dw.abs() + dw_off) + 1e-44


# ---- sampling --------------------------------------------------------------------------------------------------
def filtered(x, T, k, p, least, u):
    """One row: dict(bad), or dict(keep mask, d, n, token, logq)."""
    x = x.double()
    V = len(x)
    if math.isnan(T) or torch.isnan(x).any() or not math.isfinite(x.max()):
        return dict(bad=True)
    if T < 2.0 ** -126:
        best = int((x == x.max()).nonzero()[0])
        keep = torch.zeros(V, dtype=torch.bool)
        keep[best] = True
        return dict(bad=False, keep=keep, d=torch.zeros(V, dtype=torch.float64), n=1, token=best, logq=0.0)
    d = torch.where(x == -math.inf, -math.inf, (x - x.max()) / T)
    w = torch.exp(d)
    order = torch.argsort(-x, stable=True)
    order = order[x[order] > -math.inf]
    if 0 < k < V:
        order = order[:k]
    if p < 1:
        before = torch.cat((torch.zeros(1, dtype=torch.float64), w[order].cumsum(0)[:-1]))
        keep = before < p * w[order].sum()
        keep[0] = True
        order = order[keep]
    if least > 0:
        order = order[d[order] >= math.log(min(least, 1.0))]             # w >= least, where w of a d next to 0 would be rounded to 1
    keep = torch.zeros(V, dtype=torch.bool)
    keep[order] = True
    out = dict(bad=False, keep=keep, d=d, n=len(order))
    if u is not None:
        cum = torch.where(keep, w, 0.0).cumsum(0)
        above = (cum > u * cum[-1]).nonzero()
        out["token"] = int(above[0]) if len(above) else int((torch.where(keep, w, 0.0) > 0).nonzero()[-1])
        out["logq"] = float(d[out["token"]] - torch.log(cum[-1]))
    return out


# ---- distillation ------------------------------------------------------------------------------------------------
def distillation(h, w, ids, logits, given, row_weight, scale, dtype):
    """(loss, lse, counts, dh, dw, bounds of loss, lse, dh, dw) for rows h [N, D] with lists ids, logits [N, T] and given lse [N] or None."""
    z, dz = hu.logits(h, w)
    V = w.shape[0]
    lse = torch.logsumexp(z, -1)
    real = ids >= 0
    at = ids.clamp(0, V - 1).long()
    tl = torch.where(real, logits.double(), -math.inf)
    ref = torch.logsumexp(tl, -1) if given is None else given.double()
    log_t = torch.where(real & (tl > -math.inf), tl - ref[:, None], 0.0)
    t = torch.where(real & (tl > -math.inf), torch.exp(log_t), 0.0)
    mass = t.sum(-1)
    zt, dzt = z.gather(1, at), dz.gather(1, at)
    loss = torch.where(t > 0, t * (log_t - zt + lse[:, None]), 0.0).sum(-1)
    counts = real.any(-1) & torch.isfinite(lse) & torch.isfinite(mass) & ~(real & (ids >= V)).any(-1) & (row_weight != 0)
    dlse = hu.lse_bound(z, dz, lse)
    dloss = (t * (dzt + dlse[:, None] + 2 * U32 * (log_t.abs() + zt.abs() + lse.abs()[:, None]))).sum(-1) + 2 * U32 * loss.abs()
    rw = torch.where(counts, row_weight.double(), 0.0)[:, None]
    p = torch.exp(z - lse[:, None]) * mass[:, None]
    g = p.clone().scatter_add_(1, at, -t)
    g = torch.where(counts[:, None], g, 0.0) * rw
    h = torch.where(counts[:, None], h.double(), 0.0)
    w = w.double()
    dp = p * (dz + dlse[:, None] + 2.0 ** -19)
    T = ids.shape[1]
    dt = torch.zeros_like(p).scatter_add_(1, at, t * (T + 2) * U32)
    dg = torch.where(counts[:, None], (dp + dt + 4 * U32 * p) * rw.abs() + (HALF[dtype] + U32) * g.abs(), 0.0)
    N = len(h)
    dh, dw = scale * (g @ w), scale * (g.T @ h)
    bh = abs(scale) * (dg @ w.abs() + (V + 64) * 2 * U32 * (g.abs() @ w.abs()))
    bw = abs(scale) * (dg.T @ h.abs() + (N + 64) * 2 * U32 * (g.abs().T @ h.abs()))
    return (loss, lse, counts, dh, dw, dloss, dlse, bh + (HALF[dtype] + U32) * (dh.abs() + bh) + 1e-37, bw + (HALF[dtype] + U32) * (dw.abs() + bw) + 1e-37)
