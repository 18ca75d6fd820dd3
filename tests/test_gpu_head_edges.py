"""The draft head's operators at the borders of their inputs: what lies behind the last rows, and what earlier calls left in the head's scratch."""
import pytest
import torch

from paper_2511_02017_amd import binding
from tests.test_gpu_head import DEV, bf16, f32, loss_inputs, rand, same

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
