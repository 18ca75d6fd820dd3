"""The draft head's operators at the borders of their inputs: what lies behind the last rows, and what earlier calls left in the head's scratch."""
import pytest
import torch

from paper_2511_02017_amd import binding
from tests import head_util as hu
from tests.test_gpu_head import DEV, bf16, f32, loss_inputs, rand, same, within

pytestmark = pytest.mark.gpu
BEHIND = 300                             # rows: more than the largest tile has


def leading(x, junk):
    """x as the leading rows (axis 0) of a longer allocation whose other rows hold `junk`."""
    room = torch.full((x.shape[0] + BEHIND, *x.shape[1:]), junk, dtype=x.dtype, device=DEV)
    room[:x.shape[0]] = x
    return room[:x.shape[0]]


# tokens on every tile; vocabulary rows, tokens and dim that fill none of them
@pytest.mark.parametrize("dtype,N", [(bf16, 1), (bf16, 21), (bf16, 101), (bf16, 299), (f32, 1), (f32, 45), (f32, 101), (f32, 299)])
@pytest.mark.parametrize("V,D", [(1, 32), (333, 96), (777, 160)])
def test_what_lies_behind_the_rows_of_loss_and_gradient_is_not_read(dtype, N, V, D):
    h, w, t = (x.to(DEV) for x in loss_inputs(N, 1, V, D, dtype, seed=N + V))
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    got = []
    for x, y in ((h, w), (leading(h, float("nan")), leading(w, float("nan")))):
        f = head.loss(x, y, t)
        got.append(dict(f, **head.loss_grad(x, y, t, f["lse"])))
    torch.cuda.synchronize()
    assert all(torch.isfinite(v).all() for v in got[0].values())
    same(*got)


@pytest.mark.parametrize("dtype,N", [(bf16, 21), (bf16, 101), (bf16, 299), (f32, 45), (f32, 101), (f32, 299)])
@pytest.mark.parametrize("V,D", [(333, 96), (777, 160)])
def test_what_lies_beside_the_columns_of_loss_and_gradient_is_not_read(dtype, N, V, D):
    h, w, t = (x.to(DEV) for x in loss_inputs(N, 1, V, D, dtype, seed=N + V))
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    got = []
    for junk in (0.0, float("nan"), float("inf")):
        x, y = torch.full((N, 1, D + 64), junk, dtype=dtype, device=DEV)[..., :D], torch.full((V, D + 64), junk, dtype=dtype, device=DEV)[:, :D]
        x.copy_(h), y.copy_(w)
        f = head.loss(x, y, t)
        got.append(dict(f, **head.loss_grad(x, y, t, f["lse"])))
    torch.cuda.synchronize()
    assert all(torch.isfinite(v).all() for v in got[0].values())
    same(got[1], got[0])
    same(got[2], got[0])


@pytest.mark.parametrize("act", [16, 4])
@pytest.mark.parametrize("N", [1, 21, 50, 101, 299])
@pytest.mark.parametrize("V,D", [(1, 32), (333, 96), (777, 160)])
def test_what_lies_behind_the_rows_of_logits_is_not_read(act, N, V, D):
    h = rand(N, 1, D, seed=N, dtype=bf16).to(DEV)
    c, s = binding.mx4_quantize(rand(V, D, seed=V).to(DEV))
    head = binding.DraftHead(N, D, V)
    want = head.logits(h, c, s, act_bits=act)
    got = head.logits(leading(h, float("nan")), leading(c, 255), leading(s, 255), act_bits=act)
    torch.cuda.synchronize()
    assert torch.isfinite(want).all() and torch.equal(got, want)


@pytest.mark.parametrize("dtype,N", [(bf16, 21), (bf16, 101), (bf16, 299), (f32, 45), (f32, 101)])
def test_what_earlier_calls_left_in_the_scratch_is_not_read(dtype, N):
    """A larger call whose gradients are NaN throughout, hidden states that lie unevenly and are NaN, then a smaller call."""
    V, D, more = 333, 96, 400
    h, w, t = (x.to(DEV) for x in loss_inputs(1, N, V, D, dtype, seed=N))
    heads = [binding.DraftHead(more, D, 900, dtype=dtype, training=True) for _ in range(2)]
    H, W, T = (x.to(DEV) for x in loss_inputs(2, more // 2, 900, D, dtype, seed=2))
    lse = heads[0].loss(H, W, T)["lse"]
    heads[0].loss_grad(H, W, T, lse, row_weight=torch.full_like(lse, float("nan")))
    uneven = torch.full((2, more // 2 + 1, D), float("nan"), dtype=dtype, device=DEV)[:, 1:]
    heads[0].loss(uneven, W, T)
    c, s = binding.mx4_quantize(w)
    got = []
    for head in heads:
        f = head.loss(h, w, t)
        r = dict(f, **head.loss_grad(h, w, t, f["lse"]))
        if dtype == bf16:
            if head is heads[0]:
                head.logits(uneven, *binding.mx4_quantize(W), act_bits=4)
            r["z"] = head.logits(h, c, s, act_bits=4)
        got.append(r)
    torch.cuda.synchronize()
    assert all(torch.isfinite(v).all() for v in got[1].values())
    same(*got)


# vocabularies on every tile of the weights' gradient
@pytest.mark.parametrize("dtype,N,V", [(bf16, 5, 20), (bf16, 96, 100), (bf16, 300, 333), (f32, 5, 40), (f32, 96, 333), (f32, 300, 64)])
@pytest.mark.parametrize("factor", [float("inf"), -float("inf"), float("nan")])
def test_gradients_are_zeros_where_no_row_counts_whatever_the_factor(dtype, N, V, factor):
    """The mean over no rows has an infinite factor: a batch of prompts only leaves the weights as they are."""
    D = 96
    h, w, t = (x.to(DEV) for x in loss_inputs(1, N, V, D, dtype, seed=N + V))
    t[t < 0] = 0
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    lse = head.loss(h, w, t)["lse"]
    scale = torch.tensor([factor], device=DEV)
    none = torch.full_like(lse, float("nan"))
    for left_out in (dict(target=torch.full_like(t, -1), lse=lse), dict(target=t, lse=lse, row_weight=torch.zeros_like(lse)), dict(target=t, lse=none)):
        out = dict(grad_hidden=torch.ones_like(h), grad_weight=torch.ones_like(w))
        head.loss_grad(h, w, scale=scale, out=out, **left_out)
        torch.cuda.synchronize()
        assert (out["grad_hidden"] == 0).all() and (out["grad_weight"] == 0).all()
    # the last row alone counts: its gradient meets the factor
    last = torch.full_like(t, -1)
    last[0, -1] = t[0, -1]
    b = head.loss_grad(h, w, last, lse, scale=scale)
    torch.cuda.synchronize()
    assert not torch.isfinite(b["grad_hidden"][0, -1]).any() and (b["grad_hidden"][0, :-1] == 0).all()
    assert not torch.isfinite(b["grad_weight"][t[0, -1].long()]).any()


# binary32: the same products as they are up to 64 tokens, as sums of three bfloat16 from 65 on
@pytest.mark.parametrize("dtype,N", [(bf16, 20), (bf16, 100), (bf16, 299), (f32, 64), (f32, 65), (f32, 299)])
def test_vocabulary_rows_masked_by_infinite_weights(dtype, N):
    """A constant hidden element and a weight of -inf there: the token's logit is -inf, whatever the number of rows."""
    V, D = 700, 96
    h, w, t = loss_inputs(1, N, V, D, dtype, seed=N)
    masked = torch.zeros(V, dtype=torch.bool)
    masked[3], masked[256:400], masked[V - 1] = True, True, True
    h[..., 0] = 1.0
    t[0][(t[0] >= 0) & masked[t[0].clamp(min=0).long()]] = 5
    wm = w.clone()
    wm[masked, 0] = -float("inf")
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    hd, wd, td = h.to(DEV), wm.to(DEV), t.to(DEV)
    f = head.loss(hd, wd, td)
    b = head.loss_grad(hd, wd, td, f["lse"])
    torch.cuda.synchronize()
    assert (f["flags"] == 0).all()
    kept = torch.where(t[0] < 0, t[0], (torch.cumsum(~masked, 0) - 1).to(torch.int32)[t[0].clamp(min=0).long()])      # targets among the other rows
    loss, lse, z, dz = hu.cross_entropy(h[0], w[~masked], kept)
    bound = hu.lse_bound(z, dz, lse)
    within(f["lse"][0], lse, bound)
    within(f["loss"][0], loss, bound + dz.amax(-1) + 2 * hu.U32 * (loss.abs() + 1))
    dh, dw, bh, bw = hu.gradients(h[0], w[~masked], kept, lse, torch.ones(N), 1.0, dtype)
    live = t[0] >= 0
    within(b["grad_hidden"][0][:, 1:], dh[:, 1:], bh[:, 1:])
    assert b["grad_hidden"][0][live.to(DEV), 0].isnan().all() and (b["grad_hidden"][0][~live.to(DEV)] == 0).all()       # 0 times -inf
    within(b["grad_weight"][~masked.to(DEV)], dw, bw)
    assert (b["grad_weight"][masked.to(DEV)] == 0).all()
    # the target itself is masked: an infinite loss of a good row, whose gradient takes its hidden state off the masked row
    t[0, 2] = 3
    f = head.loss(hd, wd, t.to(DEV))
    b = head.loss_grad(hd, wd, t.to(DEV), f["lse"])
    torch.cuda.synchronize()
    assert (f["flags"] == 0).all() and f["loss"][0, 2] == float("inf") and torch.isfinite(f["lse"]).all()
    assert torch.equal(b["grad_weight"][3], -hd[0, 2])
    # logits of +inf: no finite lse
    h[0, 1, 0] = -1.0
    f = head.loss(h.to(DEV), wd, t.clamp(min=0).to(DEV))
    torch.cuda.synchronize()
    assert int(f["flags"][0]) == binding.FLAG_BAD_ROW and f["loss"][0, 1].isnan() and torch.isfinite(f["lse"][0, torch.arange(N) != 1]).all()


@pytest.mark.parametrize("N", [64, 65, 299])
def test_hidden_states_that_are_not_finite_beside_masked_vocabulary_rows(N):
    """Rows that are left out hold NaN and infinities, in every tile of tokens or in all of one but a few: the others as without them."""
    V, D = 700, 96
    h, w, t = loss_inputs(1, N, V, D, f32, seed=N)
    t[t < 0] = 1
    h[..., 0] = 1.0
    w[300, 0] = w[V - 1, 0] = -float("inf")
    t[0][(t[0] == 300) | (t[0] == V - 1)] = 5
    out = torch.zeros(N, dtype=torch.bool)
    out[::3], out[8:60] = True, True
    t[0, out] = -1
    dirty = h.clone()
    dirty[0, out] = torch.where(torch.arange(int(out.sum()))[:, None] % 2 == 0, float("nan"), float("inf"))
    head = binding.DraftHead(N, D, V, dtype=f32, training=True)
    hd, wd, td = dirty.to(DEV), w.to(DEV), t.to(DEV)
    f = head.loss(hd, wd, td)
    b = head.loss_grad(hd, wd, td, f["lse"])
    torch.cuda.synchronize()
    assert (f["flags"] == 0).all() and f["lse"][0, out.to(DEV)].isnan().all()
    rows = [v for v in range(V) if v not in (300, V - 1)]
    kept = t[0, ~out] - (t[0, ~out] > 300).to(torch.int32)
    loss, lse, z, dz = hu.cross_entropy(h[0, ~out], w[rows], kept)
    bound = hu.lse_bound(z, dz, lse)
    within(f["lse"][0, (~out).to(DEV)], lse, bound)
    within(f["loss"][0, (~out).to(DEV)], loss, bound + dz.amax(-1) + 2 * hu.U32 * (loss.abs() + 1))
    dh, dw, bh, bw = hu.gradients(h[0, ~out], w[rows], kept, lse, torch.ones(len(kept)), 1.0, f32)
    within(b["grad_hidden"][0, (~out).to(DEV)][:, 1:], dh[:, 1:], bh[:, 1:])
    within(b["grad_weight"][rows], dw, bw)
    assert (b["grad_hidden"][0, out.to(DEV)] == 0).all() and (b["grad_weight"][[300, V - 1]] == 0).all()


@pytest.mark.parametrize("N", [64, 65])
def test_binary32_results_by_infinite_operands_are_those_of_the_formula(N):
    """One vocabulary row against a row of zeros, hidden states with one element: each logit is one product."""
    inf, nan, D = float("inf"), float("nan"), 32
    pairs = [(1.0, -inf), (-1.0, inf), (2.0 ** -100, -inf), (1.0 + 2.0 ** -23, -inf), (0.0, 1.0), (3.0e38, -2.0), (1.0, nan), (0.0, -inf), (1.0, inf), (inf, 1.0), (-inf, 0.0)]
    head = binding.DraftHead(N, D, 2, dtype=f32)
    for x, y in pairs:
        h, w = torch.zeros(1, N, D), torch.zeros(2, D)
        h[..., 7], w[1, 7] = x, y
        f = head.loss(h.to(DEV), w.to(DEV), torch.zeros(1, N, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        z = torch.tensor(x) * torch.tensor(y) + (0.0 if abs(x) < inf else nan)               # inf times the row of zeros
        if z <= 0:
            assert (f["loss"] == (0.0 if z < 0 else torch.tensor(2.0).log())).all() and f["flags"][0] == 0, (x, y)
        else:
            assert f["loss"].isnan().all() and int(f["flags"][0]) == binding.FLAG_BAD_ROW, (x, y)


def test_binary32_split_products_are_as_precise_as_documented():
    """Off by 2^-21 of a product at most and 2^-24 in the mean where it is a sum of three bfloat16 by three: single products, so that nothing
    hides them.  Beside that a matrix instruction's sums: the last one a step of 2^-23 of the result, in the mean half of it, those before
    that add to less than 2^-6 of it a 64th each.  (Without the products by third parts: 2^-14 and 2^-16.)"""
    most, mean = 2.0 ** -21 + 2.0 ** -23 + 5 * 2.0 ** -29, 2.0 ** -24 + 2.0 ** -24 + 5 * 2.0 ** -30
    g = torch.Generator().manual_seed(1)

    def mantissas(*shape):
        return torch.exp2(torch.rand(*shape, generator=g)).float()

    def check(got, x, y):
        off = (got.double().cpu() / (x.double().cpu() * y.double().cpu()) - 1).abs()
        assert float(off.max()) <= most and float(off.mean()) <= mean, (float(off.max()), float(off.mean()))
    # logits: -z of a row with one element against 0 of a row of zeros; ln(1 + e^z) of z < -32 is below 2^-46
    N, D = 1024, 1024
    x, y = 8 * mantissas(N), -4 * mantissas(D)
    w = torch.zeros(2, D)
    w[1] = y
    h = torch.diag(x)[None]
    f = binding.DraftHead(N, D, 2, dtype=f32).loss(h.to(DEV), w.to(DEV), torch.ones(1, N, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    check(-f["loss"][0], x, y)
    # gradients: one row counts, so each element by the weights is g of its token times a hidden element, and with one vocabulary row that is not
    # zeros each by the hidden state is g times a weight; an element of 1 says what g is
    N, V = 70, 70
    h, w = torch.zeros(1, N, D), torch.zeros(V, D)
    h[0, 5], w[9] = mantissas(D) / 64, -mantissas(D) / 8
    h[0, 5, 0], w[9, 0] = 1.0, 1.0
    t = torch.full((1, N), -1, dtype=torch.int32)
    t[0, 5] = 3
    head = binding.DraftHead(N, D, V, dtype=f32, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    b = head.loss_grad(hd, wd, td, head.loss(hd, wd, td)["lse"])
    torch.cuda.synchronize()
    dh, dw = b["grad_hidden"][0, 5].cpu(), b["grad_weight"].cpu()
    check(dw, dw[:, :1], h[0, 5][None])
    check(dh, dh[:1], w[9])


# ---- the largest sizes -------------------------------------------------------------------------------------
def test_matrices_whose_offsets_pass_32_bits():
    """More than 2^32 bytes of weights, codes and logits: the far end as in a call that has it alone."""
    V, D, far = 1_100_033, 2048, 769
    w = torch.randn(V, D, dtype=bf16, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)) * 0.05
    c, s = binding.mx4_quantize(w)
    c1, s1 = binding.mx4_quantize(w[-far:])
    assert torch.equal(c[-far:], c1) and torch.equal(s[-far:], s1)
    assert torch.equal(binding.mx4_dequantize(c, s, D)[-far:], binding.mx4_dequantize(c1, s1, D))
    h = rand(1, 2100, D, seed=2, dtype=bf16).to(DEV)
    head = binding.DraftHead(2100, D, V)
    for act in (16, 4):
        z = head.logits(h, c, s, act_bits=act)
        assert z.numel() > 2 ** 31 and torch.equal(z[..., -far:], head.logits(h, c1, s1, act_bits=act))
        del z
    del head, c, s
    N = 40
    head = binding.DraftHead(N, D, V, training=True)
    h, t = h[:, :N], torch.arange(V - N, V, dtype=torch.int32, device=DEV)[None]
    f = head.loss(h, w, t)
    b = head.loss_grad(h, w, t, f["lse"])
    torch.cuda.synchronize()
    z = torch.cat([h[0].float() @ p.float().T for p in w.split(65536)], 1).double()
    lse = torch.logsumexp(z, -1)
    # binary32 products of the reference too: both are within (D + 2) / 2^23 of sum |h w|, at most |h| |w| a row
    dz = 2 * (D + 2) * 2.0 ** -23 * h[0].float().norm(dim=-1).double() * float(w.float().norm(dim=-1).max())
    within(f["lse"][0], lse.cpu(), (dz + 2.0 ** -18 + 1024 * hu.U32 + 2 * hu.U32 * lse.abs()).cpu())
    p = torch.exp(z[:, -far:] - lse[:, None])
    p[torch.arange(N), torch.arange(far - N, far)] -= 1.0
    dw = p.T @ h[0].double()
    bw = ((2 * dz[:, None] + 2.0 ** -8 + 2.0 ** -16) * p.abs()).T @ h[0].double().abs()
    within(b["grad_weight"][-far:], dw.cpu(), (bw + 2.0 ** -8 * (dw.abs() + bw) + 1e-9).cpu())


@pytest.mark.parametrize("dtype,N", [(bf16, 20), (bf16, 101), (bf16, 299), (f32, 45), (f32, 101)])
def test_rows_as_far_apart_as_they_may_lie(dtype, N):
    """Weights and their gradient at 8 MiB a row, hidden states beyond that (which are copied first): as close together."""
    V, D = 300, 96
    stride = (8 << 20) // torch.tensor([], dtype=dtype).element_size()
    h, w, t = (x.to(DEV) for x in loss_inputs(1, N, V, D, dtype, seed=N))
    room = torch.full((V * stride,), float("nan"), dtype=dtype, device=DEV)
    far_w = room.as_strided((V, D), (stride, 1))
    far_w.copy_(w)
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    f = head.loss(h, w, t)
    want = dict(f, **head.loss_grad(h, w, t, f["lse"]))
    f = head.loss(h, far_w, t)
    got = head.loss_grad(h, far_w, t, f["lse"], out=dict(grad_hidden=torch.empty_like(h), grad_weight=room.as_strided((V, D), (stride, 1), 2 * D)))
    torch.cuda.synchronize()
    same({k: v.contiguous() for k, v in dict(f, **got).items()}, want)
    del room, far_w, got
    room = torch.full((N * (stride + 64),), float("nan"), dtype=dtype, device=DEV)
    far_h = room.as_strided((1, N, D), (0, stride + 64, 1))
    far_h.copy_(h)
    f = head.loss(far_h, w, t)
    got = head.loss_grad(far_h, w, t, f["lse"], out=dict(grad_hidden=room.as_strided((1, N, D), (0, stride + 64, 1), 2 * D), grad_weight=torch.empty_like(w)))
    torch.cuda.synchronize()
    same({k: v.contiguous() for k, v in dict(f, **got).items()}, want)
    with pytest.raises(binding.TapoutError, match="8 MiB"):
        head.loss(h, torch.empty(stride + 64 + D, device=DEV, dtype=dtype).as_strided((2, D), (stride + 64, 1)), t.clamp(max=1))


@pytest.mark.parametrize("dtype,N", [(bf16, 3), (bf16, 101), (bf16, 140), (f32, 3), (f32, 70)])
def test_the_longest_hidden_states(dtype, N):
    V, D = 130, 65536
    h, w, t = loss_inputs(1, N, V, D, dtype, seed=N)
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    f = head.loss(hd, wd, td)
    b = head.loss_grad(hd, wd, td, f["lse"])
    torch.cuda.synchronize()
    loss, lse, z, dz = hu.cross_entropy(hd[0], wd, td[0])
    within(f["lse"][0], lse.cpu(), hu.lse_bound(z, dz, lse).cpu())
    dh, dw, bh, bw = hu.gradients(hd[0], wd, td[0], f["lse"][0].double(), torch.ones(N, device=DEV), 1.0, dtype)
    within(b["grad_hidden"][0], dh.cpu(), bh.cpu())
    within(b["grad_weight"], dw.cpu(), bw.cpu())
    if dtype == bf16:
        c, s = binding.mx4_quantize(wd)
        values = binding.mx4_dequantize(c, s, D, dtype=f32)
        ch, sh = binding.mx4_quantize(hd[0])
        for act, x in ((16, hd[0]), (4, binding.mx4_dequantize(ch, sh, D, dtype=f32))):
            z, bound = hu.logits(x, values)
            within(head.logits(hd, c, s, act_bits=act, dtype=f32)[0], z.cpu(), (bound + 1e-37).cpu())


def test_a_closed_head_refuses_its_calls():
    h, w, t = (x.to(DEV) for x in loss_inputs(1, 3, 50, 64, bf16, seed=1))
    head = binding.DraftHead(3, 64, 50, training=True)
    c, s = binding.mx4_quantize(w)
    f = head.loss(h, w, t)
    head.close()
    head.close()
    for call in (lambda: head.loss(h, w, t), lambda: head.loss_grad(h, w, t, f["lse"]), lambda: head.logits(h, c, s)):
        with pytest.raises(binding.TapoutError, match="NULL"):
            call()
