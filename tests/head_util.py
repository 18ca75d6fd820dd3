"""Plain 64-bit forms of the draft head's operators and the error bounds that the tests hold them to (torch, on the CPU)."""
import torch

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
U32 = 2.0 ** -24                       # half a step of binary32
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def mx4(x):
    """x [rows, cols] float64: (codes 0..15 [rows, P], scale bytes [rows, P / 32], values [rows, cols])."""
    rows, cols = x.shape
    P = -(-cols // 128) * 128
    y = torch.zeros(rows, P, dtype=torch.float64)
    y[:, :cols] = x.double()
    y = y.view(rows, P // 32, 32)
    bad = ~torch.isfinite(y).all(-1)
    top = torch.where(bad, 1.0, y.abs().amax(-1))
    _, e = torch.frexp(top)                                     # top = m 2^e, m in [1/2, 1)
    e = torch.where(top > 0, e - 3, -127).clamp(min=-127)
    unit = torch.ldexp(torch.ones_like(top), e)
    a = torch.where(bad[..., None], 0.0, y.abs() / unit[..., None])
    # nearest, ties to the even code, by distance
    grid = torch.tensor(GRID, dtype=torch.float64)
    d = (a[..., None] - grid).abs()
    best = d.amin(-1, keepdim=True)
    tied = d == best
    even = torch.arange(8) % 2 == 0
    code = torch.where((tied & even).any(-1), (tied & even).to(torch.int8).argmax(-1), tied.to(torch.int8).argmax(-1))
    neg = torch.signbit(y)
    val = torch.where(neg, -1.0, 1.0) * grid[code] * unit[..., None]
    val = torch.where(bad[..., None], float("nan"), val)
    byte = torch.where(bad, 255, e + 127)
    return (code + 8 * neg).view(rows, P), byte, val.view(rows, P)[:, :cols]


def unpack(codes):
    c = codes.cpu().to(torch.int64)
    return torch.stack((c & 15, c >> 4), -1).flatten(1)


def logits(h, w):
    """(z, bound) of h [N, D], w [V, D]: the product and what a binary32 sum of its terms can be off by (two roundings a term, any order,
    truncated or rounded: 2 u a step)."""
    h, w = h.double(), w.double()
    z = h @ w.T
    return z, (h.shape[1] + 2) * 2 * U32 * (h.abs() @ w.abs().T)


def cross_entropy(h, w, t):
    """(loss, lse, z, dz) for targets t (any outside [0, V) gives loss 0)."""
    z, dz = logits(h, w)
    lse = torch.logsumexp(z, -1)
    V = w.shape[0]
    live = (t >= 0) & (t < V)
    loss = torch.where(live, lse - z.gather(1, t.clamp(0, V - 1).long()[:, None])[:, 0], 0.0)
    return loss, lse, z, dz


def lse_bound(z, dz, lse):
    """Off by the logits' own error, by sums of V positive terms (each with an exponential good to 2^-21 of itself for |z - max| up to 64: its
    argument is rounded twice) in runs of 256, and by the result's rounding."""
    return dz.amax(-1) + 2.0 ** -19 + 512 * U32 + 2 * U32 * lse.abs()


def gradients(h, w, t, lse, row_weight, scale, dtype):
    """(dh, dw, bound of dh, bound of dw)."""
    h, w = h.double(), w.double()
    z, dz = logits(h, w)
    V = w.shape[0]
    live = (t >= 0) & (t < V) & (row_weight != 0) & torch.isfinite(lse)
    p = torch.exp(z - torch.logsumexp(z, -1, keepdim=True))
    hot = torch.zeros_like(p)
    hot[torch.arange(len(t), device=t.device)[live], t[live].long()] = 1.0
    rw = torch.where(live, row_weight.double(), 0.0)[:, None]
    g = torch.where(live[:, None], p - hot, 0.0) * rw
    h = torch.where(live[:, None], h, 0.0)
    # g: p's relative error (the logits', lse's, the exponential's), the difference's and the product's rounding, then the operands' type
    dp = p * (dz + lse_bound(z, dz, torch.logsumexp(z, -1))[:, None] + 2.0 ** -19)
    dg = torch.where(live[:, None], (dp + 2 * U32) * rw.abs() + HALF[dtype] * g.abs(), 0.0)
    N, V = g.shape
    dh, dw = scale * (g @ w), scale * (g.T @ h)
    bh = abs(scale) * (dg @ w.abs() + (V + 64) * 2 * U32 * (g.abs() @ w.abs()))
    bw = abs(scale) * (dg.T @ h.abs() + (N + 64) * 2 * U32 * (g.abs().T @ h.abs()))
    return dh, dw, bh + HALF[dtype] * (dh.abs() + bh) + 1e-37, bw + HALF[dtype] * (dw.abs() + bw) + 1e-37
