"""Operators around the draft head that are timed and compared: the norm in front of it, its logits under 8-bit weights, the token
that is drawn from them, and its distillation from the target model's largest logits.

A case is a dict of plain values.  `op` names one pass:
  norm     root-mean-square norm of x + residual over the last axis.  pass_ "fp8": the sum and the normalised states in 8-bit floating
           point with a scale for 128 of them (returned as the values these stand for); "train": the sum, the normalised states, and
           the gradients by x (the residual's is the same) and by the norm's weight
  logits   the draft logits [B, K, V] of hidden states [B, K, D] under a head held in 8-bit floating point with a scale for each
           block of 128 x 128 weights; the hidden states are brought to 8 bits too, with a scale for 128 elements of a row
  sample   temperature, top-k, top-p and min-p: the filtered logits, and (draw) a token for each row at a given uniform number
  distill  divergence of the head's softmax from a teacher's, of which each row has the largest logits, and the mean's gradient by
           the hidden states and by the head's weights

Plain forms are written out here in elementary operations of 32 bits (64 where a token hangs on a sum's last bits); with `own` the
library's calls are made.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}
EPS = 1e-5
BLOCK = 128
TOP = 448.0                              # the largest finite value of the 8-bit type


def listed():
    return [
        # the last hidden states of a serving batch's next step, on their way to an 8-bit head: the smallest call
        dict(name="norm_step_fp8", op="norm", pass_="fp8", B=64, K=1, D=2048, dtype="bf16"),
        # a training step's texts
        dict(name="norm_train", op="norm", pass_="train", B=4, K=2048, D=2048, dtype="bf16"),
        # one user, one token, a small vocabulary
        dict(name="logits_one", op="logits", B=1, K=1, V=32000, D=1024, out="f32"),
        # one step of the draft loop for a serving batch
        dict(name="logits_step", op="logits", B=64, K=1, V=128256, D=2048, out="bf16"),
        # a large batch with long drafts
        dict(name="logits_large", op="logits", B=256, K=16, V=151936, D=2048, out="bf16"),
        # one user, one token: latency is all there is
        dict(name="sample_one", op="sample", B=1, K=1, V=32000, dtype="f32", filters="k", draw=True),
        # one step of the draft loop for a serving batch whose users ask for different filters
        dict(name="sample_step", op="sample", B=64, K=1, V=128256, dtype="bf16", filters="mixed", draw=True),
        # odd sizes: rows start at every alignment of their type
        dict(name="sample_odd_f32", op="sample", B=24, K=5, V=50257, dtype="f32", filters="mixed", draw=True),
        # the target's rows of a round, filtered before verification (which draws by itself)
        dict(name="sample_target_rows", op="sample", B=64, K=9, V=128256, dtype="bf16", filters="p", draw=False),
        # a step on one round's rows of a few users, binary32
        dict(name="distill_round_f32", op="distill", B=8, K=5, V=32000, D=1024, T=16, tail=False, dtype="f32"),
        # odd sizes everywhere: three texts of 501 tokens
        dict(name="distill_odd", op="distill", B=3, K=501, V=50257, D=1120, T=37, tail=True, dtype="bf16"),
        # the largest: a training step's tokens under a 128k-vocabulary head
        dict(name="distill_128k", op="distill", B=4, K=2048, V=128256, D=2048, T=64, tail=True, dtype="bf16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("norm", "logits", "sample", "sample", "distill"))
        V = _spread(rng, 8000, 256000)
        V += rng.choice((0, 1, -V % 8, -V % 128))
        D = 32 * _spread(rng, 8, 128)
        B, K = _spread(rng, 1, 512), rng.randint(1, 16)
        if op == "norm":
            c = dict(op=op, pass_=rng.choice(("fp8", "train")), B=B, K=K, D=D, dtype=rng.choice(("bf16", "bf16", "f32")))
            if c["pass_"] == "train":
                c["B"], c["K"] = rng.randint(1, 8), _spread(rng, 16, 2048)
            return c
        if op == "logits":
            c = dict(op=op, B=B, K=K, V=V, D=D, out=rng.choice(("bf16", "bf16", "f32")))
            if B * K * V * ESZ[c["out"]] <= 2e9 and B * K * V * D <= 1.3e12:
                return c
            continue
        if op == "sample":
            c = dict(op=op, B=B, K=K, V=V, dtype=rng.choice(("bf16", "bf16", "f32")), filters=rng.choice(("mixed", "mixed", "k", "p", "min")),
                     draw=rng.random() < 0.7)
            if B * K * V <= 7.5e7:
                return c
            continue
        if rng.random() < 0.5:
            B, K = rng.randint(1, 8), _spread(rng, 16, 2048)
        c = dict(op=op, B=B, K=K, V=V, D=D, T=_spread(rng, 1, 128), tail=rng.random() < 0.5, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
        # binary32 products run at a sixteenth of the bfloat16 rate: shorter texts
        if B * K * V * D <= (2.1e12 if c["dtype"] == "bf16" else 1.2e11):
            return c


# ---- 8-bit blocks, plainly -------------------------------------------------------------------------------
def _fp8(x, block_rows):
    """x [rows, cols], binary32, to (values of the 8-bit type, in binary32, [rows padded, cols padded], scales of its blocks)."""
    rows, cols = x.shape
    y = torch.zeros(-(-rows // block_rows) * block_rows, -(-cols // BLOCK) * BLOCK, dtype=torch.float32, device=x.device)
    y[:rows, :cols] = x
    y = y.view(-1, block_rows, y.shape[1] // BLOCK, BLOCK)
    scale = y.abs().amax((1, 3), keepdim=True).clamp(min=TOP * 2.0 ** -126) / TOP
    q = (y / scale).to(torch.float8_e4m3fn).float()
    return q.view(-1, q.shape[2] * BLOCK), scale.view(q.shape[0], q.shape[2])


def _spread_scales(scale, block_rows):
    return scale.repeat_interleave(block_rows, 0).repeat_interleave(BLOCK, 1)


# ---- inputs ----------------------------------------------------------------------------------------------
def _head(c, g, dtype):
    """A head whose logits of normalised hidden states spread by about 2, as those of the decode workloads do."""
    w = torch.randn(c["V"], c["D"], generator=g, device=DEV, dtype=torch.float32).mul_(2.0 / math.sqrt(c["D"]))
    return w.to(dtype)


def _filters(c, g, s):
    """What each sequence asks for: a temperature, and no more, or few, or several of the three filters; some want the best token."""
    B, kind = c["B"], c["filters"]
    u = torch.rand(7, B, generator=g, device=DEV)
    s["temperature"] = torch.where(u[0] < 0.1 if kind == "mixed" else u[0] < 0.0, 0.0, 0.5 + 0.8 * u[1])
    s["top_k"] = torch.where(u[2] < (0.5 if kind == "mixed" else 1.0), (20 + 180 * u[3]).int(), 0) if kind in ("mixed", "k") else None
    s["top_p"] = torch.where(u[4] < (0.6 if kind == "mixed" else 1.0), 0.8 + 0.18 * u[5], 1.0) if kind in ("mixed", "p") else None
    s["min_p"] = torch.where(u[6] < (0.3 if kind == "mixed" else 1.0), 0.02 + 0.1 * u[1], 0.0) if kind in ("mixed", "min") else None


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(7919 * seed + 13)
    s = dict(case=c)
    B, K = c["B"], c["K"]
    if c["op"] == "norm":
        dt = DTYPES[c["dtype"]]
        # a residual stream with a few large channels, and what the last layer adds to it
        big = 1.0 + 8.0 * (torch.rand(c["D"], generator=g, device=DEV) < 0.01)
        s["residual"] = (3.0 * torch.randn(B, K, c["D"], generator=g, device=DEV) * big).to(dt)
        s["x"] = torch.randn(B, K, c["D"], generator=g, device=DEV).to(dt)
        s["weight"] = (1.0 + 0.2 * torch.randn(c["D"], generator=g, device=DEV)).to(dt)
        if c["pass_"] == "train":
            s["grad_out"] = (0.1 * torch.randn(B, K, c["D"], generator=g, device=DEV)).to(dt)
    elif c["op"] == "logits":
        w = _head(c, g, torch.float32)
        q, s["scales"] = _fp8(w, BLOCK)
        s["codes"] = q[:c["V"]].to(torch.float8_e4m3fn).view(torch.uint8)
        s["hidden"] = torch.randn(B, K, c["D"], generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)
    elif c["op"] == "sample":
        # rows between peaked and flat; a few tokens of the vocabulary are masked in all of them
        base = 3.0 * torch.randn(B, K, c["V"], generator=g, device=DEV)
        base *= 0.6 + 1.4 * torch.rand(B, K, 1, generator=g, device=DEV)
        base.masked_fill_(torch.rand(c["V"], generator=g, device=DEV) < 0.002, -math.inf)
        s["logits"] = base.to(DTYPES[c["dtype"]])
        _filters(c, g, s)
        s["u"] = torch.rand(B, K, generator=g, device=DEV) if c["draw"] else None
    else:
        dt = DTYPES[c["dtype"]]
        V, D, T = c["V"], c["D"], c["T"]
        s["weight"] = w = _head(c, g, dt)
        # ids of a Zipf-like law at the top, spread over the vocabulary behind; logits that fall off like a target model's; lists of
        # uneven length, and rows without any (the prompts' tokens)
        top = torch.exp(torch.rand(B, K, 1, generator=g, device=DEV) * math.log(V)).long().clamp_(1, V) - 1
        step = 1 + (torch.rand(B, K, 1, generator=g, device=DEV) * (V // max(T, 1) - 1)).long()
        ids = (top * 7907 + step * torch.arange(T, device=DEV)) % V
        fall = 0.5 + 1.5 * torch.rand(B, K, 1, generator=g, device=DEV)
        z = 14.0 - fall * torch.log1p(torch.arange(T, device=DEV, dtype=torch.float32)) - torch.rand(B, K, T, generator=g, device=DEV) * 0.2
        n = torch.where(torch.rand(B, K, 1, generator=g, device=DEV) < 0.3, (1 + T * torch.rand(B, K, 1, generator=g, device=DEV)).long(), T)
        n = torch.where(torch.rand(B, K, 1, generator=g, device=DEV) < 0.06, 0, n)
        n[0, 0] = T
        s["top_ids"] = torch.where(torch.arange(T, device=DEV) < n, ids, -1).int()
        s["top_logits"] = z
        s["teacher_lse"] = None
        if c["tail"]:                    # what lies behind the list holds up to a third of the teacher's mass
            listed_mass = torch.exp(torch.where(s["top_ids"] >= 0, z, -math.inf)).sum(-1).clamp(min=1e-3)
            s["teacher_lse"] = torch.log(listed_mass * (1.0 + 0.5 * torch.rand(B, K, generator=g, device=DEV)))
        rows = w[ids[..., 0].view(-1)].float().view(B, K, D)
        lean = 7.0 * torch.rand(B, K, 1, generator=g, device=DEV)
        s["hidden"] = (torch.randn(B, K, D, generator=g, device=DEV) + lean * rows / rows.norm(dim=-1, keepdim=True)).to(dt)
        s["scale"] = 1.0 / (s["top_ids"][..., 0] >= 0).sum().float().view(1)     # the mean over the rows that count
    if own:
        from paper_2511_02017_amd import binding
        if c["op"] == "sample":
            s["ctx"] = binding.Tapout(B, K, c["V"])
        else:
            s["head"] = binding.DraftHead(B * K, c["D"], c.get("V", 1), dtype=DTYPES[c.get("dtype", "bf16")],
                                          training=c["op"] == "distill" or c.get("pass_") == "train")
    return s


def _run_own(s):
    from paper_2511_02017_amd import binding
    c = s["case"]
    if c["op"] == "norm":
        if c["pass_"] == "fp8":
            f = s["head"].norm(s["x"], s["weight"], residual=s["residual"], eps=EPS, fp8=True)
            return dict(sum=f["sum"], out=binding.fp8_dequantize(f["codes"], f["scales"], c["D"], dtype=torch.bfloat16))
        f = s["head"].norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        b = s["head"].norm_grad(s["grad_out"], f["sum"], s["weight"], f["rstd"])
        return dict(sum=f["sum"], out=f["out"], grad_x=b["grad_x"], grad_weight=b["grad_weight"])
    if c["op"] == "logits":
        return s["head"].logits_fp8(s["hidden"], s["codes"], s["scales"], dtype=DTYPES[c["out"]])
    if c["op"] == "sample":
        r = s["ctx"].sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                            kept=s["logits"].dtype)
        return {k: r[k] for k in (("token", "logq") if c["draw"] else ()) + ("n_kept", "kept")}
    f = s["head"].distill(s["hidden"], s["weight"], s["top_ids"], s["top_logits"], teacher_lse=s["teacher_lse"])
    b = s["head"].distill_grad(s["hidden"], s["weight"], s["top_ids"], s["top_logits"], f["lse"], f["top"], teacher_lse=s["teacher_lse"],
                               scale=s["scale"])
    return dict(loss=f["loss"], lse=f["lse"], grad_hidden=b["grad_hidden"], grad_weight=b["grad_weight"])


def _run_norm(s):
    c, dt = s["case"], s["x"].dtype
    total = (s["x"].float() + s["residual"].float()).to(dt)          # the residual stream, which is kept in its type
    v, w = total.float(), s["weight"].float()
    rstd = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    hat = v * rstd
    y = hat * w
    if c["pass_"] == "fp8":
        q, scale = _fp8(y.view(-1, c["D"]), 1)
        return dict(sum=total, out=(q * _spread_scales(scale, 1))[:, :c["D"]].to(torch.bfloat16).view(y.shape))
    g = s["grad_out"].float()
    gw = g * w
    gx = rstd * (gw - hat * (gw * hat).mean(-1, keepdim=True))
    return dict(sum=total, out=y.to(dt), grad_x=gx.to(dt), grad_weight=(g * hat).sum((0, 1)).to(dt))


def _run_logits(s):
    c = s["case"]
    w = s["codes"].view(torch.float8_e4m3fn).float()
    w *= _spread_scales(s["scales"], BLOCK)[:c["V"]]
    q, scale = _fp8(s["hidden"].float().view(-1, c["D"]), 1)
    return ((q * _spread_scales(scale, 1)) @ w.T).to(DTYPES[c["out"]]).view(c["B"], c["K"], c["V"])


def _run_sample(s):
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    per_row = lambda t, off: (torch.full((B,), off, device=DEV) if t is None else t).repeat_interleave(K)[:, None]      # noqa: E731
    temperature, k = per_row(s["temperature"], 1.0).double(), per_row(s["top_k"], 0)
    p, least = per_row(s["top_p"], 1.0).double(), per_row(s["min_p"], 0.0).double()
    x = s["logits"].view(B * K, V).double()
    greedy = temperature <= 0
    d = (x - x.amax(-1, keepdim=True)) / torch.where(greedy, 1.0, temperature)
    best_first, at = torch.sort(d, dim=-1, descending=True, stable=True)     # equal ones by index
    w = torch.exp(best_first)
    rank = torch.arange(V, device=DEV)
    in_k = (rank < k) | (k <= 0)
    total = torch.cumsum(torch.where(in_k, w, 0.0), -1)
    before = torch.zeros_like(total)
    before[:, 1:] = total[:, :-1]
    keep = in_k & ((before < p * total[:, -1:]) | (p >= 1)) & (w >= least) & torch.isfinite(best_first)
    keep = torch.where(greedy, False, keep)
    keep[:, 0] = True
    mask = torch.zeros_like(keep).scatter_(1, at, keep)
    d = torch.where(greedy, 0.0, d)
    out = dict(n_kept=mask.sum(-1).int().view(B, K), kept=torch.where(mask, d, -math.inf).to(s["logits"].dtype).view(B, K, V))
    if not c["draw"]:
        return out
    cum = torch.cumsum(torch.where(mask, torch.exp(d), 0.0), -1)
    token = (cum <= s["u"].view(-1, 1).double() * cum[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
    logq = d.gather(1, token) - torch.log(cum[:, -1:])
    return dict(token=token.int().view(B, K), logq=logq.float().view(B, K), **out)


def _run_distill(s):
    c = s["case"]
    B, K, V, D, T = c["B"], c["K"], c["V"], c["D"], c["T"]
    h, w = s["hidden"].float().view(B * K, D), s["weight"].float()
    ids = s["top_ids"].view(B * K, T).long()
    real, at = ids >= 0, ids.clamp(min=0)
    t = torch.where(real, s["top_logits"].view(B * K, T), -math.inf)
    counts = real.any(-1)
    lse_t = torch.logsumexp(torch.where(counts[:, None], t, 0.0), -1) if s["teacher_lse"] is None else s["teacher_lse"].view(-1)
    log_t = torch.where(real, t - lse_t[:, None], 0.0)
    t = torch.where(real, torch.exp(log_t), 0.0)
    mass = t.sum(-1)
    z = h @ w.T
    zt = z.gather(1, at)
    m = z.amax(-1)
    e = z.sub_(m[:, None]).exp_()
    sums = e.sum(-1)
    lse = m + sums.log()
    loss = (t * (log_t - zt + lse[:, None])).sum(-1)
    e *= (mass / sums)[:, None]
    e.scatter_add_(1, at, -t)
    e *= torch.where(counts, s["scale"], 0.0)[:, None]
    return dict(loss=loss.view(B, K), lse=lse.view(B, K), grad_hidden=(e @ w).to(s["hidden"].dtype).view(B, K, D), grad_weight=(e.T @ h).to(s["weight"].dtype))


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "logits": _run_logits, "sample": _run_sample, "distill": _run_distill}[state["case"]["op"]](state)


def work(case):
    c = case
    N = c["B"] * c["K"]
    if c["op"] == "norm":
        n = N * c["D"]
        if c["pass_"] == "fp8":          # x, residual, sum; a byte and its share of a scale
            return {"bytes": 3 * n * ESZ[c["dtype"]] + n + n // 32, "flops": 6 * n}
        return {"bytes": 7 * n * ESZ[c["dtype"]], "flops": 16 * n}
    if c["op"] == "logits":
        V, D = c["V"], c["D"]
        return {"bytes": V * D + 2 * N * D + N * V * ESZ[c["out"]], "flops": 2 * N * V * D}
    if c["op"] == "sample":
        return {"bytes": 2 * N * c["V"] * ESZ[c["dtype"]] + 12 * N, "flops": 4 * N * c["V"]}
    V, D, T = c["V"], c["D"], c["T"]
    return {"bytes": 2 * ((N + V) * D * ESZ[c["dtype"]] + 8 * N * T + 8 * N), "flops": 6 * N * V * D + 6 * N * T * D}


# ---- the definitions in 64 bits --------------------------------------------------------------------------
def _exact_fp8(x):
    """Values that x [rows, cols] (64 bits) has with a scale for 128 elements of a row.  By the definition the scale is a binary32 quotient, and
    so is what is rounded."""
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], BLOCK):
        b = x[:, k:k + BLOCK].float().double()
        scale = (torch.clamp(b.abs().max(-1, keepdim=True).values, min=TOP * 2.0 ** -126) / TOP).float().double()
        y = (b / scale).float().double()
        _, e = torch.frexp(y)
        unit = torch.ldexp(torch.ones_like(y), (e - 4).clamp(min=-9))           # four bits, down to 2^-9
        out[:, k:k + BLOCK] = torch.round(y / unit) * unit * scale
    return out


def _exact_sample(s):
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    at = lambda t, b, off: off if t is None else float(t[b])                        # noqa: E731
    kept = torch.full((B, K, V), -math.inf, dtype=torch.float64, device=DEV)
    n_kept = torch.zeros(B, K, dtype=torch.int32, device=DEV)
    token, logq = n_kept.clone(), torch.zeros(B, K, dtype=torch.float64, device=DEV)
    for b in range(B):
        tau, k = at(s["temperature"], b, 1.0), int(at(s["top_k"], b, 0))
        p, least = at(s["top_p"], b, 1.0), at(s["min_p"], b, 0.0)
        for i in range(K):
            x = s["logits"][b, i].double()
            if tau <= 0:
                best = int((x == x.max()).nonzero()[0])
                kept[b, i, best], n_kept[b, i], token[b, i] = 0.0, 1, best
                continue
            y = (x - x.max()) / tau
            w = torch.exp(y)
            order = torch.argsort(x.neg(), stable=True)
            order = order[:int((x > -math.inf).sum())]
            if k > 0:
                order = order[:k]
            if p < 1:
                mass = torch.cumsum(w[order], 0)
                order = order[:1 + int(torch.searchsorted(mass[:-1].contiguous(), p * mass[-1]))]      # masses below p of it: the next one stays too
            order = order[:max(1, int((w[order] >= least).sum()))]
            index = torch.sort(order).values
            kept[b, i, index] = y[index]
            n_kept[b, i] = len(index)
            if c["draw"]:
                mass = torch.cumsum(w[index], 0)
                j = min(int(torch.searchsorted(mass, float(s["u"][b, i]) * mass[-1], right=True)), len(index) - 1)
                token[b, i] = index[j]
                logq[b, i] = y[index[j]] - torch.log(mass[-1])
    return dict(token=token, logq=logq, n_kept=n_kept, kept=kept) if c["draw"] else dict(n_kept=n_kept, kept=kept)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, K = c["B"], c["K"]
    if c["op"] == "sample":
        return _exact_sample(s)
    if c["op"] == "norm":
        D = c["D"]
        total = (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
        v, w = total.double().view(-1, D), s["weight"].double()
        rms = torch.sqrt(torch.sum(v ** 2, 1) / D + EPS)[:, None]
        if c["pass_"] == "fp8":
            return dict(sum=total.double(), out=_exact_fp8(w * v / rms).view(B, K, D))
        g = s["grad_out"].double().view(-1, D)
        inner = torch.sum(g * w * v, 1, keepdim=True)
        return dict(sum=total.double(), out=(w * v / rms).view(B, K, D), grad_x=(g * w / rms - v * inner / (D * rms ** 3)).view(B, K, D),
                    grad_weight=torch.sum(g * v / rms, 0))
    D, V = c["D"], c["V"]
    h = s["hidden"].double().reshape(-1, D)
    if c["op"] == "logits":
        h = _exact_fp8(h)
        out = torch.empty(B * K, V, dtype=torch.float64, device=DEV)
        for v in range(0, V, BLOCK):
            byte = s["codes"][v:v + BLOCK].int()
            e, m = byte // 8 % 16, (byte % 8).double()
            w = torch.where(e == 0, m * 2.0 ** -9, torch.ldexp(1 + m / 8, e - 7)) * torch.where(byte >= 128, -1.0, 1.0)
            w = w * s["scales"][v // BLOCK].double().repeat_interleave(BLOCK)
            out[:, v:v + BLOCK] = h @ w[:, :D].T
        return out.view(B, K, V)
    w, T = s["weight"].double(), c["T"]
    ids, tl = s["top_ids"].reshape(-1, T).long(), s["top_logits"].double().reshape(-1, T)
    n = (ids[:, 0] >= 0).sum()
    loss, lse, gh = [], [], []
    gw = torch.zeros_like(w)
    for i in range(0, B * K, 1024):
        hi, ii = h[i:i + 1024], ids[i:i + 1024]
        weight = torch.where(ii >= 0, torch.exp(tl[i:i + 1024]), 0.0)
        norm = weight.sum(1) if s["teacher_lse"] is None else torch.exp(s["teacher_lse"].double().reshape(-1)[i:i + 1024])
        t = weight / torch.where(norm > 0, norm, 1.0)[:, None]
        z = torch.mm(hi, w.T)
        ls = torch.logsumexp(z, -1)
        lse.append(ls)
        logp = (z - ls[:, None]).gather(1, ii.clamp(min=0))
        loss.append(torch.sum(torch.special.xlogy(t, t) - t * logp, 1))
        g = torch.exp(z - ls[:, None]) * t.sum(1, keepdim=True)
        g.scatter_add_(1, ii.clamp(min=0), -t)
        g /= n
        gh.append(torch.mm(g, w))
        gw.addmm_(g.T, hi)
    return dict(loss=torch.cat(loss).view(B, K), lse=torch.cat(lse).view(B, K), grad_hidden=torch.cat(gh).view(B, K, D), grad_weight=gw)
