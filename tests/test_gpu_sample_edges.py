"""Sampling where runs end beside or among the smallest values, against the plain 64-bit form."""
import math

import pytest
import torch

from paper_2511_02017_amd import binding
from tests.test_gpu_sample import INF, bf16, check, columns, f32, run

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -16                                 # magnitudes below it are counted in one place


def place_beside_zeros(n, dtype, seed, below=0.0):
    """A row of n zeros and small values of both signs, n of the largest negative values beyond these, and light ones."""
    g = torch.Generator().manual_seed(seed)
    small = (torch.rand(n - n // 2, generator=g) * 2 - 1) * TINY * 0.99
    edge = -TINY * (1 + below * torch.rand(n, generator=g))
    x = torch.cat((torch.zeros(n // 2), small, edge, torch.full((n // 3 + 5,), -200.0)))
    return x[torch.randperm(len(x), generator=g)].to(dtype)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("n", [10, 300, 511, 513, 700, 3000, 9000])
@pytest.mark.parametrize("below", [0.0, 2.0 ** -8])
def test_top_p_ends_at_the_values_beside_the_smallest(dtype, n, below):
    """Of 2 n elements of weights next to 1 the run keeps the n larger ones and some of the others; masses that lie half a weight beside
    each border (all the weights together are off from 1 by 0.3 at most)."""
    x = place_beside_zeros(n, dtype, seed=n, below=below if dtype == f32 else 0.0)
    V = len(x)
    ends = [n + 1, n + n // 4, n + n // 2, 2 * n - 1]
    T, k, p, m = columns([(1.0, kk, (e - 0.5) / (2 * n), 0.0) for e in ends for kk in (0, max(2 * n, 1025))])
    B = len(T)
    many = x.expand(B, 2, V).contiguous()
    u = torch.rand(B, 2, generator=torch.Generator().manual_seed(1))
    check(many, run(binding.Tapout(B, 2, V), many, T, k, p, m, u, dtype), dtype, T, k, p, m, u)


def test_ten_zeros_and_ten_values_beside_the_smallest():
    x = torch.tensor([0.0] * 10 + [-1.53e-5] * 10).view(1, 1, 20)
    T, k, p, m = columns([(1.0, 0, 0.75, 0.0)])
    r = run(binding.Tapout(1, 1, 20), x, T, k, p, m, None, f32)
    assert int(r["n_kept"]) == 15 and (r["kept"].cpu().view(-1)[:15] > -INF).all() and (r["kept"].cpu().view(-1)[15:] == -INF).all()


@pytest.mark.parametrize("V", [60, 5003, 20011, 140009])
@pytest.mark.parametrize("zeros", [False, True])
def test_top_k_ends_among_small_values_and_top_p_before(V, zeros):
    """bfloat16 rows with up to 64 small values that top-k divides: top-p's share is that of those it leaves, at temperatures at which their weights differ."""
    g = torch.Generator().manual_seed(V)
    n = 10
    for seed in range(4):
        small = torch.full((20,), 1.4e-5) if seed == 0 else (torch.rand(20, generator=g) * 2 - 1) * 1.5e-5
        x = torch.full((V,), -3.0)
        at = torch.randperm(V, generator=g)
        x[at[:n]] = TINY
        x[at[n:n + 20]] = small
        if zeros:
            x[at[n + 20:n + 26]] = torch.tensor([0.0, -0.0] * 3)
        x = x.to(bf16)
        T, k, p, m = columns([(T, k, p, m) for T in (1e-6, 1e-5, 3e-6) for k in (14, 20, 25, 30) for p, m in ((0.9, 0.0), (0.35, 0.0), (0.97, 0.2))])
        B = len(T)
        many = x.expand(B, 1, V).contiguous()
        u = torch.rand(B, 1, generator=g)
        check(many, run(binding.Tapout(B, 1, V), many, T, k, p, m, u, bf16), bf16, T, k, p, m, u)


@pytest.mark.parametrize("V", [40, 30011])
def test_ten_largest_small_values_and_twenty_behind(V):
    x = torch.full((1, 1, V), -1.0)
    x[..., 3:13] = TINY
    x[..., 14:34] = 1.4e-5
    T, k, p, m = columns([(1e-6, 20, 0.9, 0.0)])
    r = run(binding.Tapout(1, 1, V), x.to(bf16), T, k, p, m, None, bf16)
    assert int(r["n_kept"]) == 16 and (r["kept"].cpu()[0, 0, 14:20] > -INF).all() and (r["kept"].cpu()[0, 0, 20:] == -INF).all()


def test_kept_rows_that_reach_into_the_logits_are_refused():
    V = 96
    flat = torch.randn(8 * V, device="cuda:0")
    x = flat[:4 * V].view(2, 2, V)
    tp = binding.Tapout(2, 1, V)
    rows = lambda at, b, k, dtype=f32: flat.view(dtype).as_strided((2, 2, V), (b, k, 1), at)          # noqa: E731
    for y in (x, rows(V, 2 * V, V), rows(4 * V - 1, 2 * V, V), rows(3 * V - 1, 3 * V, V), rows(8 * V - 2, 2 * V, V, bf16), rows(0, V, 3 * V)):
        with pytest.raises(binding.TapoutError, match="memory of logits"):
            tp.sample(x, out=dict(kept=y))
    want = tp.sample(x, kept=f32)
    for y in (rows(4 * V, 2 * V, V), rows(8 * V, 2 * V, V, bf16)):                                    # behind them
        got = tp.sample(x, out=dict(kept=y, n_kept=torch.empty(2, 2, dtype=torch.int32, device="cuda:0")))
        torch.cuda.synchronize()
        assert torch.equal(got["kept"], want["kept"].to(y.dtype)) and torch.equal(got["n_kept"], want["n_kept"])


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("kept", [f32, bf16])
@pytest.mark.parametrize("V", [7, 1003, 9001])
def test_kept_logits_are_rounded_once(V, dtype, kept):
    """(x - max) / T in binary64, where the difference, the inverse and their product are off by 2^-53 each, to binary32 and, of bfloat16, from
    there: half a step of each type, and of binary32's smallest numbers."""
    g = torch.Generator().manual_seed(V)
    x = torch.stack([torch.randn(V, generator=g) * s for s in (1.0, 3.0, 30.0, 1e-3, 1e6)]
                    + [30 - 40 * torch.rand(V, generator=g), 1e-30 * torch.randn(V, generator=g), 1e30 * torch.randn(V, generator=g)]).to(dtype)
    temperatures = (0.7, 1.3, 0.3333, 1.0, 7e-6, 3e38, 2e-38, INF)          # from 2^-126 on, about 1.2e-38, no greedy ones
    B, K = len(x), len(temperatures)
    T = torch.tensor(temperatures)
    many = x.expand(K, B, V).transpose(0, 1).reshape(B * K, 1, V).contiguous()
    r = run(binding.Tapout(B * K, 1, V), many, T.repeat(B), None, None, None, None, kept)
    d = (many.double() - many.double().amax(-1, keepdim=True)) / T.repeat(B).double()[:, None, None]
    inside = d.abs() < 3.3e38
    got = r["kept"].cpu().double()
    assert not torch.isnan(got).any() and (r["n_kept"].cpu() == V).all()
    half = 2.0 ** -24 + 2.0 ** -50
    bound = (half if kept == f32 else 2.0 ** -8 * (1 + half) + half) * d.abs() + (2.0 ** -150 if kept == f32 else 2.0 ** -133)
    assert ((got - d).abs()[inside] <= bound[inside]).all()
    assert (got[~inside] <= -3.3e38 * (1 - 2.0 ** -8)).all()


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_the_whole_range_under_an_infinite_temperature(dtype):
    """All weights are 1 and all kept logits 0, also of values whose difference is beyond binary32."""
    x = torch.tensor([3e38, -3e38, 0.0, -1.0, -INF, 3e38, -2e38, 1e30]).to(dtype).view(1, 1, 8)
    T = torch.tensor([INF])
    for u, token in ((0.0, 0), (0.2, 1), (0.5, 3), (0.6, 5), (0.99, 7)):
        r = run(binding.Tapout(1, 1, 8), x, T, None, None, None, torch.tensor([[u]]), dtype)
        kept = r["kept"].cpu().view(-1).tolist()
        assert [v == 0 for v in kept] == [True] * 4 + [False] + [True] * 3 and kept[4] == -INF
        assert int(r["token"]) == token and int(r["n_kept"]) == 7 and abs(float(r["logq"]) + math.log(7)) < 1e-6


def test_a_context_has_room_for_the_calls_it_takes():
    """Rows of more than 2^24 elements are not sampled: a context for them has no room for their slices (1.1 GB here), nor has it for more rows or slices
    than a call may have."""
    held = []
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    held.append(binding.Tapout(8, 16, 2 ** 30))
    assert free - torch.cuda.mem_get_info()[0] < 400e6
    with pytest.raises(binding.TapoutError, match="2\\^24"):
        held[0].sample(torch.zeros(1, device="cuda:0").expand(1, 1, 2 ** 24 + 1).contiguous(), kept=bf16)


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_as_many_rows_as_a_call_may_have(dtype):
    B, K, V = 65535, 64, 6
    row = torch.tensor([0.5, -1.0, 2.0, -INF, 1.0, 2.0]).to(dtype).to("cuda:0")
    tp = binding.Tapout(B, K, V)
    u = torch.full((B, K), 0.6, device="cuda:0")
    u[B // 2:] = 0.3
    r = tp.sample(row.expand(B, K, V), u, top_k=torch.full((B,), 2, dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    assert bool((r["n_kept"] == 2).all()) and bool((r["flags"] == 0).all())
    assert bool((r["token"][:B // 2] == 5).all()) and bool((r["token"][B // 2:] == 2).all())
    with pytest.raises(binding.TapoutError, match="rows beyond"):
        tp.sample(row.expand(B, K + 1, V), kept=dtype)


def test_as_many_slices_as_a_call_may_have():
    B, K, V = 23, 89, 2 ** 24                      # 2047 rows of 8193 slices
    row = torch.full((V,), -3.0, device="cuda:0")
    row[V - 1], row[5] = 4.0, 3.0
    tp = binding.Tapout(B, K, V)
    u = torch.rand(B, K, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1))
    u[0, 0], u[0, 1], u[B - 1, K - 1], u[B - 1, K - 2] = 0.0, 0.999, 0.999, 0.0
    r = tp.sample(row.expand(B, K, V), u, min_p=torch.full((B,), 0.1, device="cuda:0"))
    torch.cuda.synchronize()
    first = math.exp(-1) / (1 + math.exp(-1))
    assert bool((r["n_kept"] == 2).all()) and torch.equal(r["token"], torch.where(u.double() < first, 5, V - 1).int())
