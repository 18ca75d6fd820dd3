"""Sampling under a temperature, top-k, top-p and min-p against a plain 64-bit form: tokens, counts and what is kept have to be equal."""
import math

import pytest
import torch

from paper_2511_02017_amd import binding
from tests import operators_util as ou

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
f32, bf16, i32 = torch.float32, torch.bfloat16, torch.int32
NAN, INF = math.nan, math.inf


def check(x, r, kept_dtype, T=None, k=None, p=None, least=None, u=None, k_len=None):
    """x [B, K, V] on the CPU; r: what the call returned."""
    B, K, V = x.shape
    r = {n: v.cpu() for n, v in r.items()}
    val = lambda t, b, off: off if t is None else float(t[b])                         # noqa: E731
    for b in range(B):
        bad = False
        for i in range(K if k_len is None else int(k_len[b])):
            want = ou.filtered(x[b, i], val(T, b, 1.0), int(val(k, b, 0)), val(p, b, 1.0), val(least, b, 0.0), None if u is None else float(u[b, i]))
            what = (b, i, val(T, b, 1.0), val(k, b, 0), val(p, b, 1.0), val(least, b, 0.0), None if u is None else float(u[b, i]))
            bad |= want["bad"]
            if want["bad"]:
                assert (r["n_kept"][b, i] == 0) and ("kept" not in r or (r["kept"][b, i] == -INF).all()), what
                if u is not None:
                    assert r["token"][b, i] == -1 and math.isnan(r["logq"][b, i]), what
                continue
            assert int(r["n_kept"][b, i]) == want["n"], (what, int(r["n_kept"][b, i]), want["n"])
            if u is not None:
                assert int(r["token"][b, i]) == want["token"], (what, int(r["token"][b, i]), want["token"])
                # the sums' units, then one rounding
                assert abs(float(r["logq"][b, i]) - want["logq"]) <= 2 * ou.U32 * abs(want["logq"]) + 1e-10, what
            if "kept" in r:
                got, d = r["kept"][b, i].double(), torch.where(want["keep"], want["d"], -INF)
                assert not torch.isnan(got).any()
                out = d.abs() > 3.3e38                               # beyond the type: minus infinity
                assert torch.equal((got == -INF) | out, ~want["keep"] | out), what
                fine = want["keep"] & ~out
                # x - max, 1 / T and their product in binary32; then the type
                bound = 4 * ou.U32 * d.abs() + (ou.HALF[bf16] * d.abs() if kept_dtype == bf16 else 0) + 1.5e-38
                assert ((got - d).abs()[fine] <= bound[fine]).all(), what
        if k_len is None or int(k_len[b]) > 0:
            assert int(r["flags"][b]) == (binding.FLAG_BAD_ROW if bad else 0)


def rows(B, K, V, dtype, seed, sigma=3.0, masked=0.01):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, K, V, generator=g) * sigma * (0.4 + 1.2 * torch.rand(B, K, 1, generator=g))
    x[torch.rand(B, K, V, generator=g) < masked] = -INF
    x[..., 0] = torch.where(torch.isfinite(x).any(-1), x[..., 0], 0.0)
    return x.to(dtype)


FILTERS = [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (0.9, 0, 1.0, 0.05), (0.8, 40, 0.95, 0.02), (0.0, 0, 1.0, 0.0), (1.0, 1, 1.0, 0.0),
           (1.0, 0, 0.0, 0.0), (1.0, 0, 0.5, 0.0), (2.0, 300, 0.99, 0.0), (0.05, 0, 0.9, 0.0), (1.0, 0, 1.0, 1.0), (-1.0, 7, 0.5, 0.5), (1.0, -3, 2.0, -1.0),
           (INF, 0, 0.5, 0.0), (INF, 9, 0.3, 0.1), (1e-30, 4, 0.9, 0.0), (1e30, 0, 0.25, 0.0), (1e-42, 0, 1.0, 0.0), (1.0, 10 ** 9, 0.999999, 2.0),
           (1.0, 0, NAN, NAN), (NAN, 0, 1.0, 0.0), (0.6, 2, 0.1, 0.9), (1.0, 0, -0.5, 0.0)]


def columns(which):
    T, k, p, m = zip(*which)
    return torch.tensor(T), torch.tensor(k, dtype=i32), torch.tensor(p), torch.tensor(m)


def run(tp, x, T, k, p, m, u, kept, **kw):
    d = lambda t: None if t is None else t.to(DEV)                                    # noqa: E731
    r = tp.sample(x if x.is_cuda else x.to(DEV), d(u), temperature=d(T), top_k=d(k), top_p=d(p), min_p=d(m), kept=kept, **kw)
    torch.cuda.synchronize()
    return r


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 515, 4099, 8192, 16385, 32000, 70001])
def test_filters_and_tokens(V, dtype):
    B, K = len(FILTERS), 2
    x = rows(B, K, V, dtype, seed=V)
    T, k, p, m = columns(FILTERS)
    g = torch.Generator().manual_seed(V + 1)
    u = torch.rand(B, K, generator=g)
    u[::5, 0], u[1::5, 0] = 0.0, 1 - 2.0 ** -24
    tp = binding.Tapout(B, K, V)
    other = bf16 if dtype == f32 else f32
    check(x, run(tp, x, T, k, p, m, u, dtype), dtype, T, k, p, m, u)
    check(x, run(tp, x, T, k, p, m, None, other), other, T, k, p, m)
    check(x, run(tp, x, None, None, None, None, u, None), None, u=u)


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_every_alignment_stride_and_length(dtype):
    B, K, V = 3, 3, 1003
    wide = torch.full((B, K, 2 * V + 77), 50.0, dtype=dtype)
    lengths = torch.tensor([3, 0, 2], dtype=i32)
    T, k, p, m = columns([(0.9, 30, 0.9, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.02)])
    u = torch.rand(B, K, generator=torch.Generator().manual_seed(4))
    tp = binding.Tapout(B, K - 1, V)                                                  # K: target rows
    for off in range(9):
        x = rows(B, K, V, dtype, seed=off)
        wide[..., off:off + V] = x
        on = wide.to(DEV)
        # sequences inside positions, what lies around the rows is left as it is
        room = torch.full((K, B, V + 23), 7.0, dtype=f32 if off % 2 else bf16, device=DEV)
        out = dict(kept=room.transpose(0, 1)[..., off:off + V], token=torch.full((B, K), -7, dtype=i32, device=DEV),
                   logq=torch.full((B, K), 3.0, device=DEV), n_kept=torch.full((B, K), -9, dtype=i32, device=DEV), flags=torch.full((B,), 99, dtype=i32, device=DEV))
        run(tp, on[..., off:off + V], T, k, p, m, u, None, k_len=lengths.to(DEV), out=out)
        check(x, out, room.dtype, T, k, p, m, u, lengths)
        assert (out["flags"] == 0).all()
        for b in range(B):
            for i in range(int(lengths[b]), K):
                assert out["token"][b, i] == -7 and out["logq"][b, i] == 3 and out["n_kept"][b, i] == -9 and (room[i, b] == 7).all()
        assert (room[..., :off] == 7).all() and (room[..., off + V:] == 7).all()


def special(V, dtype):
    """Rows whose elements crowd: equal ones, few values, one place of the counting, small ones, large ones."""
    g = torch.Generator().manual_seed(5)
    r = torch.randn(V, generator=g)
    x = [torch.zeros(V), torch.where(r > 0, 0.0, -0.0), torch.full((V,), -3.5), (r * 2).round(), 1 + torch.rand(V, generator=g) * 2.0 ** -9,
         -1 - torch.rand(V, generator=g) * 2.0 ** -9, r * 1e-6, r * 1e-38, torch.where(r > 1, r, r * 1e-7), r * 1e-7 - 1e-5, r * 100, r * 3e37, 200 + r, -500 + r * 30,
         torch.where(r > 1.5, r, -INF), torch.where(torch.arange(V) == V // 2, 1.0, -INF), torch.where(r.abs() < 0.5, r * 1e-6, r.abs() * -5),
         r.clamp(max=0.5), torch.full((V,), 127.5), torch.where(r > 0, 128.0, -128.0), torch.where(r > 1, 1e-5, -2e-5), r * 2.0 ** -14]
    return torch.stack(x).to(dtype)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("V", [40, 5003, 33001])
@pytest.mark.parametrize("which", range(0, len(FILTERS), 4))
def test_crowded_rows(V, dtype, which):
    x = special(V, dtype)
    B = len(x)
    tp = binding.Tapout(B, 4, V)
    u = torch.rand(B, 4, generator=torch.Generator().manual_seed(which))
    u[0, 0], u[3, 1] = 0.0, 0.0
    for f in FILTERS[which:which + 4]:
        T, k, p, m = columns([f] * B)
        many = x[:, None].expand(B, 4, V)
        check(many, run(tp, many.to(DEV), T, k, p, m, u, dtype), dtype, T, k, p, m, u)


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_runs_that_end_among_equal_elements(dtype):
    """Thousands of equal ones of which k, then p of their mass, are kept: those with the smallest indices."""
    V = 40003
    x = torch.full((6, 1, V), -1.0)
    x[:, :, 7::3] = 2.0
    x[2:4, :, 100:140] = 5.0
    T, k, p, m = columns([(1.0, 5000, 1.0, 0.0), (1.0, 0, 0.3, 0.0), (0.5, 9000, 0.25, 0.0), (3.0, 0, 0.5, 0.1), (1.0, 20000, 0.9, 0.0), (1.0, 13333, 0.5, 0.0)])
    u = torch.rand(6, 1, generator=torch.Generator().manual_seed(1))
    x = x.to(dtype)
    check(x, run(binding.Tapout(6, 1, V), x, T, k, p, m, u, f32), f32, T, k, p, m, u)


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_bad_rows(dtype):
    V = 1500
    x = rows(7, 3, V, dtype, seed=1)
    x[0, 1, 700], x[1, 0, 0], x[2, 2, V - 1] = NAN, INF, NAN
    x[3, 1] = -INF
    x[4, 0, 3] = -NAN
    u = torch.rand(7, 3, generator=torch.Generator().manual_seed(1))
    T = torch.tensor([1.0, 0.0, 0.5, 1.0, 0.0, NAN, 1.0])
    p = torch.full((7,), 0.9)
    for K in (3, 1):
        y = x[:, :K]
        check(y, run(binding.Tapout(7, K, V), y.to(DEV), T, None, p, None, u[:, :K].contiguous(), dtype), dtype, T, None, p, None, u[:, :K])


def test_uniforms_outside_the_interval_and_no_sequences():
    V = 300
    x = rows(4, 1, V, f32, seed=2, masked=0)
    u = torch.tensor([[1.0], [1.5], [-0.25], [NAN]])
    r = run(binding.Tapout(4, 1, V), x, None, None, None, None, u, f32)
    w = torch.exp(x.double())
    assert int(r["token"][0, 0]) == V - 1 and int(r["token"][1, 0]) == V - 1 and int(r["token"][2, 0]) == 0 and 0 <= int(r["token"][3, 0]) < V
    assert w.min() > 0
    tp = binding.Tapout(4, 1, V)
    e = tp.sample(x[:0].to(DEV), u[:0].to(DEV), kept=f32)
    assert e["kept"].shape == (0, 1, V)


def test_a_vocabulary_of_many_slices():
    V = 2_500_007
    x = rows(1, 1, V, bf16, seed=3, masked=0)
    T, k, p, m = columns([(1.0, 0, 0.9, 0.0)])
    u = torch.tensor([[0.77]])
    check(x, run(binding.Tapout(1, 1, V), x, T, k, p, m, u, bf16), bf16, T, k, p, m, u)
    y = rows(1, 1, V, f32, seed=3, masked=0)
    check(y, run(binding.Tapout(1, 1, V), y, T, k, p, m, u, f32), f32, T, k, p, m, u)


def test_same_bits_on_another_stream_in_a_replayed_graph_and_beside_another_context():
    B, K, V = 20, 2, 9001
    T, k, p, m = (t.to(DEV) for t in columns(FILTERS[:20]))
    tps = [binding.Tapout(B, K, V) for _ in range(2)]
    sets = [(rows(B, K, V, bf16, seed=s).to(DEV), torch.rand(B, K, generator=torch.Generator().manual_seed(s)).to(DEV)) for s in range(3)]
    call = lambda tp, x, u, **kw: tp.sample(x, u, temperature=T, top_k=k, top_p=p, min_p=m, kept=bf16, **kw)         # noqa: E731

    def same(a, b):
        assert all(torch.equal(a[n].contiguous().view(torch.uint8), b[n].contiguous().view(torch.uint8)) for n in a)
    want = [call(tps[0], *s) for s in sets]
    streams = [torch.cuda.Stream() for _ in tps]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for i, st in enumerate(streams):
            got.append((i, call(tps[i], *sets[i], stream=st)))
    torch.cuda.synchronize()
    for i, g in got:
        same(g, want[i])
    held = [t.clone() for t in sets[0]]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = call(tps[0], *held)
    for s in (1, 0, 2, 1):
        for a, b in zip(held, sets[s]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        same(out, want[s])
        same(call(tps[0], *sets[2]), want[2])                          # eager work of the same context between the replays
        torch.cuda.synchronize()


def test_filtered_rows_make_a_round_of_speculative_sampling():
    """Draft tokens drawn from filtered rows, statistics and verification on the filtered rows: every emitted token is one that the target keeps."""
    B, K, V = 16, 4, 5000
    g = torch.Generator().manual_seed(8)
    base = torch.randn(B, K + 1, V, generator=g) * 3
    target = base.to(bf16).to(DEV)
    draft = (base[:, :K] + torch.randn(B, K, V, generator=g)).to(bf16).to(DEV)
    tp = binding.Tapout(B, K, V)
    T, k, p = torch.full((B,), 0.8, device=DEV), torch.full((B,), 50, dtype=i32, device=DEV), torch.full((B,), 0.9, device=DEV)
    u = torch.rand(B, K, generator=g).to(DEV)
    q = tp.sample(draft, u, temperature=T, top_k=k, top_p=p, kept=f32)
    t = tp.sample(target, temperature=T, top_k=k, top_p=p, kept=f32)
    ds = tp.draft_stats(q["kept"], draft_tok=q["token"])
    assert (ds["logq_tok"] - q["logq"]).abs().max() < 1e-5 and (ds["flags"] == 0).all()
    n = torch.full((B,), K, dtype=i32, device=DEV)
    v = tp.verify(t["kept"], q["kept"], ds["lse"], ds["logq_tok"], q["token"], n, torch.rand(B, K, generator=g).to(DEV), torch.rand(B, generator=g).to(DEV))
    assert (v["flags"] == 0).all() and 0 < int(v["accept_len"].sum()) < B * K
    for b in range(B):
        for i in range(int(v["n_out"][b])):
            assert torch.isfinite(t["kept"][b, i, v["out_tok"][b, i]]), (b, i)


def test_refusals():
    V = 100
    tp = binding.Tapout(2, 3, V)
    x = torch.zeros(2, 3, V, device=DEV)
    u = torch.rand(2, 3, device=DEV)
    with pytest.raises(binding.TapoutError, match="max_batch"):
        tp.sample(torch.zeros(3, 3, V, device=DEV), kept=f32)
    with pytest.raises(binding.TapoutError, match="max_k"):
        tp.sample(torch.zeros(2, 5, V, device=DEV), kept=f32)
    with pytest.raises(binding.TapoutError, match="vocab"):
        tp.sample(torch.zeros(2, 3, V + 1, device=DEV), kept=f32)
    with pytest.raises(binding.TapoutError, match="overlap"):
        tp.sample(x, out=dict(kept=torch.zeros(2, 1, V, device=DEV).expand(2, 3, V)))
    with pytest.raises(binding.TapoutError, match="token"):
        tp.sample(x, u, out=dict(n_kept=torch.zeros(2, 3, dtype=i32, device=DEV)))
    with pytest.raises(binding.TapoutError, match="need u"):
        tp.sample(x, out=dict(token=torch.zeros(2, 3, dtype=i32, device=DEV)))
    with pytest.raises(binding.TapoutError, match="nothing"):
        tp.sample(x, out=dict())
    with pytest.raises(ValueError, match="shape"):
        tp.sample(x, u[:, :2].contiguous())
    with pytest.raises(ValueError, match="shape"):
        tp.sample(x, u, top_k=torch.zeros(3, dtype=i32, device=DEV))
    with pytest.raises(ValueError):
        tp.sample(x, u, top_k=torch.zeros(2, device=DEV))
    with pytest.raises(ValueError, match="cpu"):
        tp.sample(x, u, temperature=torch.zeros(2))
    with pytest.raises(ValueError):
        tp.sample(x.half(), u)
    with pytest.raises(ValueError, match="shape"):
        tp.sample(x, u, out=dict(kept=torch.zeros(2, 3, V - 1, device=DEV), token=torch.zeros(2, 3, dtype=i32, device=DEV)))
    tp.close()
    with pytest.raises(binding.TapoutError, match="NULL"):
        tp.sample(x, u)


@pytest.mark.parametrize("V", [16391, 70001, 131075, 262153, 540009])
@pytest.mark.parametrize("before", [0, 3])
def test_few_rows_with_what_matters_far_apart(V, before):
    """Equal elements at which the run ends, and small values among zeros, from a row's start to its end; one bad value in its last part."""
    wide = torch.full((8, 1, V + 16), 9.0, dtype=bf16)
    x = wide[:, :, before:before + V]
    x.fill_(-2.0)
    x[:, :, 5::11] = 1.5
    x[1, :, -9:] = 3.0
    x[2] = 0.0
    x[2, :, 3::V // 40] = 2.0 ** -20
    x[3] = -INF
    x[3, :, 1::V // 70] = 2.0 ** -30                               # too many of them, in all parts together
    x[4, 0, -1] = 7.0
    x[5, 0, -2] = NAN
    x[6, 0, -1] = 300.0                                            # beyond what is counted
    x[7] = -INF
    n = V // 11
    T, k, p, m = columns([(1.0, n - 7, 1.0, 0.0), (1.0, 0, 0.6, 0.0), (0.3, n, 0.7, 0.0), (1.0, 33, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 5, 1.0, 0.0),
                          (200.0, n // 2, 1.0, 0.0), (1.0, 0, 1.0, 0.0)])
    u = torch.rand(8, 1, generator=torch.Generator().manual_seed(V))
    tp = binding.Tapout(8, 1, V)
    got = run(tp, wide.to(DEV)[:, :, before:before + V], T, k, p, m, u, bf16)
    check(x, got, bf16, T, k, p, m, u)


def test_kept_logits_are_not_written_over_the_logits():
    x = torch.zeros(2, 1, 64, device=DEV)
    with pytest.raises(binding.TapoutError, match="memory of logits"):
        binding.Tapout(2, 1, 64).sample(x, out=dict(kept=x))
    both = torch.randn(2, 1, 2, 64, device=DEV)                       # side by side they may lie
    r = binding.Tapout(2, 1, 64).sample(both[:, :, 0], out=dict(kept=both[:, :, 1], n_kept=torch.empty(2, 1, dtype=i32, device=DEV)))
    torch.cuda.synchronize()
    z = both[:, :, 0] - both[:, :, 0].amax(-1, keepdim=True)
    assert torch.equal(r["kept"], z) and bool((r["n_kept"] == 64).all())


@pytest.mark.parametrize("dtype", [f32, bf16])
def test_rows_beyond_32_bits_of_offsets(dtype):
    """300 rows of which the last begin more than 2^32 elements behind the first."""
    B, V, apart = 300, 9001, 2 ** 24
    flat = torch.empty((B - 1) * apart + V, dtype=dtype, device=DEV)
    x = flat.as_strided((B, 1, V), (apart, V, 1))
    data = rows(B, 1, V, dtype, seed=2)
    for b in range(B):
        x[b].copy_(data[b])
    kept = torch.empty((B - 1) * apart + V, dtype=bf16, device=DEV).as_strided((B, 1, V), (apart, V, 1))
    T, k, p, m = (t.repeat(B // len(FILTERS) + 1)[:B] for t in columns(FILTERS))
    u = torch.rand(B, 1, generator=torch.Generator().manual_seed(3))
    tp = binding.Tapout(B, 1, V)
    out = dict(token=torch.empty(B, 1, dtype=i32, device=DEV), logq=torch.empty(B, 1, device=DEV), n_kept=torch.empty(B, 1, dtype=i32, device=DEV),
               flags=torch.empty(B, dtype=i32, device=DEV), kept=kept)
    d = lambda t: t.to(DEV)                                                               # noqa: E731
    tp.sample(x, d(u), temperature=d(T), top_k=d(k), top_p=d(p), min_p=d(m), out=out)
    torch.cuda.synchronize()
    got = {n: t.cpu() for n, t in out.items() if n != "kept"}
    got["kept"] = torch.stack([kept[b].cpu() for b in range(B)])
    check(data, got, bf16, T, k, p, m, u)
