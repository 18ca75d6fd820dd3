"""The draft head's operators against plain 64-bit forms, at the sizes where a rule turns and the inputs where they can go wrong."""
import pytest
import torch

from paper_2511_02017_amd import binding
from tests import head_util as hu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
f32, bf16 = torch.float32, torch.bfloat16


def rand(*shape, seed, scale=1.0, dtype=f32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def within(got, want, bound):
    got, want, bound = got.cpu().double(), want.double(), bound.double()
    ok = (got - want).abs() <= bound
    assert ok.all(), (f"{int((~ok).sum())} of {ok.numel()} off, worst {float(((got - want).abs() / bound).nan_to_num(nan=float('inf')).max()):.3g} bounds; "
                      f"first at {ok.logical_not().nonzero()[0].tolist()}")


# ---- 4-bit blocks -------------------------------------------------------------------------------------
def special_rows(cols, dtype):
    x = rand(12, cols, seed=cols, dtype=dtype)
    x[0] = 0
    x[1] *= 2.0 ** -130                                  # below the smallest normal number
    x[2] *= 2.0 ** 120
    x[3, 0], x[4, cols // 2], x[5, cols - 1] = float("nan"), float("inf"), -float("inf")
    x[6] = torch.arange(cols).remainder(97).sub(48).div(8).to(dtype)      # every tie
    x[7] = -0.0
    x[8, 1:] = 0
    x[9] *= torch.exp2(torch.arange(cols).remainder(40).float() - 20).to(dtype)
    return x


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("cols", [32, 96, 128, 160, 1120])
def test_mx4_codes_scales_and_values(cols, dtype):
    x = special_rows(cols, dtype)
    code, byte, val = hu.mx4(x)
    c, s = binding.mx4_quantize(x.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(s.cpu().long(), byte)
    fine = (byte != 255).repeat_interleave(32, 1)
    assert torch.equal(hu.unpack(c)[fine], code[fine])
    for out in (bf16, f32):
        v = binding.mx4_dequantize(c, s, cols, dtype=out).cpu().double()
        assert torch.equal(v.nan_to_num(nan=1e300), val.nan_to_num(nan=1e300))


@pytest.mark.parametrize("rows", [0, 1, 2, 67, 1025])
def test_mx4_rows_strides_and_given_outputs(rows):
    wide = rand(rows, 3, 64, seed=rows, dtype=bf16).to(DEV)
    x = wide[:, 1]                                       # rows 192 elements apart
    c = torch.full((rows + 1, 64), 0xAB, dtype=torch.uint8, device=DEV)
    s = torch.full((rows + 1, 4), 0xCD, dtype=torch.uint8, device=DEV)
    binding.mx4_quantize(x, out=(c[:rows], s[:rows]))
    out = torch.full((rows + 1, 96), 7.0, dtype=bf16, device=DEV)
    binding.mx4_dequantize(c[:rows], s[:rows], 64, out=out[:rows, :64])
    torch.cuda.synchronize()
    _, byte, val = hu.mx4(x.cpu())
    assert torch.equal(out[:rows, :64].cpu().double(), val)
    assert (out[:, 64:] == 7).all() and (out[rows] == 7).all() and (c[rows] == 0xAB).all() and (s[rows] == 0xCD).all()
    assert (c[:rows, 32:] == 0).all() and (s[:rows, 2:] == 0).all()


@pytest.mark.parametrize("rows,cols,dtype", [(65539, 2048, bf16), (58301, 1120, f32), (524297, 32, f32)])
def test_mx4_of_more_values_than_the_caches_hold(rows, cols, dtype):
    """In one call as in calls of a few thousand rows; the first and last rows as the plain form."""
    x = (torch.randn(rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV) * 0.02).to(dtype)
    c, s = binding.mx4_quantize(x)
    for r in range(0, rows, 8000):
        c1, s1 = binding.mx4_quantize(x[r:r + 8000])
        assert torch.equal(c[r:r + 8000], c1) and torch.equal(s[r:r + 8000], s1)
    v = binding.mx4_dequantize(c, s, cols, dtype=dtype)
    for part in (slice(0, 40), slice(rows - 40, rows)):
        code, byte, val = hu.mx4(x[part].cpu())
        assert torch.equal(hu.unpack(c[part])[:, :code.shape[1]], code) and torch.equal(s[part].cpu().long(), byte.long())
        assert torch.equal(v[part].cpu().double(), val)


# ---- logits under a 4-bit head -----------------------------------------------------------------------------
def check_logits(B, K, V, D, act, out, seed=0, hidden=None, k_len=None, target=None):
    w = rand(V, D, seed=seed + 1, scale=2.0 / D ** 0.5)
    h = rand(B, K, D, seed=seed + 2, dtype=bf16).to(DEV) if hidden is None else hidden
    codes, scales = binding.mx4_quantize(w.to(DEV))
    head = binding.DraftHead(max(1, B * K), D, V)
    z = head.logits(h, codes, scales, k_len=k_len, act_bits=act, dtype=out, out=target)
    torch.cuda.synchronize()
    x = h.cpu().reshape(B * K, D)
    want, bound = hu.logits(hu.mx4(x)[2] if act == 4 else x, hu.mx4(w)[2])
    live = torch.ones(B, K, dtype=torch.bool) if k_len is None else torch.arange(K)[None] < k_len.cpu()[:, None]
    rows = live.view(-1)
    bound = bound + hu.HALF[out] * (want.abs() + bound) + 1e-37
    within(z.reshape(B * K, V)[rows.to(DEV)], want[rows], bound[rows])
    return z


@pytest.mark.parametrize("act", [16, 4])
@pytest.mark.parametrize("B,K,V,D", [
    (1, 1, 1, 32), (1, 1, 127, 128), (1, 5, 128, 96), (2, 1, 129, 160), (3, 5, 1000, 256),
    (16, 1, 257, 384), (17, 1, 500, 64), (1, 31, 640, 288), (4, 8, 333, 2048), (3, 11, 300, 512), (64, 1, 515, 1120), (5, 13, 700, 320),
    (16, 8, 385, 256), (43, 3, 511, 224), (64, 4, 513, 640), (37, 7, 777, 416), (2, 300, 259, 128),
])
def test_logits_sizes(B, K, V, D, act):
    check_logits(B, K, V, D, act, bf16, seed=V)
    check_logits(B, K, V, D, act, f32, seed=V + 1)


# so many tiles that a workgroup multiplies several, of a stage or two each
@pytest.mark.parametrize("act,out", [(16, bf16), (16, f32), (4, bf16), (4, f32)])
@pytest.mark.parametrize("B,K,V,D,lengths", [
    (5, 1, 300001, 32, False), (2, 8, 300000, 160, True), (31, 1, 150001, 64, False), (8, 4, 150016, 288, False), (5, 10, 150001, 96, False),
    (64, 1, 100224, 256, True), (13, 9, 70001, 64, False), (64, 2, 70144, 288, False), (300, 1, 70001, 32, False), (64, 4, 70144, 544, False),
    (30, 10, 70144, 96, True),
])
def test_logits_of_many_tiles(B, K, V, D, lengths, act, out):
    k_len = (torch.arange(B, dtype=torch.int32) % (K + 2)).clamp(max=K).to(DEV) if lengths else None
    check_logits(B, K, V, D, act, out, seed=V, k_len=k_len)


@pytest.mark.parametrize("act", [16, 4])
@pytest.mark.parametrize("out", [bf16, f32])
@pytest.mark.parametrize("B,K", [(3, 2), (9, 9), (40, 8)])
def test_logits_strides_lengths_and_neighbours(B, K, act, out):
    V, D = 391, 192
    # hidden states that are the last K of longer sequences; those behind a sequence's length hold anything
    full = rand(B, K + 3, D, seed=B, dtype=bf16).to(DEV)
    h = full[:, 3:]
    k_len = (torch.arange(B, dtype=torch.int32) % (K + 1)).to(DEV)
    dead = torch.arange(K, device=DEV)[None] >= k_len[:, None]
    h[dead] = float("nan")
    room = torch.full((B, K + 2, V + 9), -3.0, dtype=out, device=DEV)
    view = room[:, 1:K + 1, 5:5 + V]                      # rows at every alignment
    check_logits(B, K, V, D, act, out, hidden=h, k_len=k_len, target=view)
    assert (view[dead] == -3).all()
    for part in (room[:, 0], room[:, K + 1], room[..., :5], room[..., 5 + V:]):
        assert (part == -3).all()


@pytest.mark.parametrize("act", [16, 4])
@pytest.mark.parametrize("N", [3, 40, 300])
def test_logits_of_extreme_blocks(N, act):
    """Scale bytes 0 and 255, infinite products, NaN hidden states: each stays in its row or column."""
    V, D = 200, 128
    w = rand(V, D, seed=5, scale=0.1)
    codes, scales = binding.mx4_quantize(w.to(DEV))
    scales[7, 2] = 255
    codes[9] = 0
    scales[11] = 0
    h = rand(1, N, D, seed=6, dtype=bf16).to(DEV)
    h[0, 1, 5] = float("nan")
    z = binding.DraftHead(N, D, V).logits(h, codes, scales, act_bits=act, dtype=f32)[0].cpu()
    torch.cuda.synchronize()
    ok = torch.ones(N, dtype=torch.bool)
    ok[1] = False
    assert z[1].isnan().all() and z[:, 7].isnan().all()
    assert (z[ok][:, 9] == 0).all() and (z[ok][:, 11].abs() < 1e-33).all()
    rest = [v for v in range(V) if v != 7]
    assert torch.isfinite(z[ok][:, rest]).all()


# ---- cross entropy --------------------------------------------------------------------------------------------
def loss_inputs(B, K, V, D, dtype, seed, scale=2.0):
    w = rand(V, D, seed=seed, scale=scale / D ** 0.5, dtype=dtype)
    g = torch.Generator().manual_seed(seed + 9)
    t = torch.randint(0, V, (B, K), generator=g, dtype=torch.int32)
    lean = 5 * torch.rand(B, K, 1, generator=g)
    rows = w.float()[t.long()]
    h = (torch.randn(B, K, D, generator=g) + lean * rows / (rows.norm(dim=-1, keepdim=True) + 1e-6)).to(dtype)
    t[torch.rand(B, K, generator=g) < 0.1] = -1
    return h, w, t


SIZES = [(1, 1, 1, 32), (1, 1, 2, 32), (1, 5, 127, 64), (2, 2, 300, 96), (8, 4, 513, 160), (3, 11, 640, 128), (16, 2, 129, 2048),
         (5, 13, 1000, 96), (64, 2, 257, 224), (43, 3, 515, 256), (1, 256, 385, 64), (1, 257, 511, 160), (3, 211, 770, 96)]


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("B,K,V,D", SIZES)
def test_loss_and_gradients(B, K, V, D, dtype):
    h, w, t = loss_inputs(B, K, V, D, dtype, seed=V + D)
    head = binding.DraftHead(B * K + 3, D, V + 5, dtype=dtype, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    got = head.loss(hd, wd, td)
    rw = (torch.rand(B, K, generator=torch.Generator().manual_seed(1)) + 0.25)
    scale = torch.tensor([0.37])
    plain = head.loss_grad(hd, wd, td, got["lse"])
    weighted = head.loss_grad(hd, wd, td, got["lse"], row_weight=rw.to(DEV), scale=scale.to(DEV))
    torch.cuda.synchronize()
    flat, tf = h.reshape(-1, D), t.view(-1)
    loss, lse, z, dz = hu.cross_entropy(flat, w, tf)
    bound = hu.lse_bound(z, dz, lse)
    within(got["lse"].view(-1), lse, bound)
    within(got["loss"].view(-1), loss, bound + dz.amax(-1) + 2 * hu.U32 * (loss.abs() + 1))
    assert (got["loss"].cpu()[t < 0] == 0).all() and (got["flags"] == 0).all()
    for b, r, s in ((plain, torch.ones(B * K), 1.0), (weighted, rw.view(-1), float(scale))):
        dh, dw, bh, bw = hu.gradients(flat, w, tf, lse, r, s, dtype)
        within(b["grad_hidden"].reshape(-1, D), dh, bh)
        within(b["grad_weight"], dw, bw)
        assert (b["grad_hidden"].cpu()[t < 0] == 0).all()


# one more and one fewer token than a tile is chosen for, over vocabularies of more tiles than run at a time
@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("B,K,V,D", [(4, 8, 70001, 64), (33, 1, 40000, 96), (8, 8, 40001, 32), (13, 5, 40001, 96), (16, 8, 35000, 64), (3, 43, 70001, 32),
                                     (1, 40, 1300, 1120), (5, 17, 1280, 2080), (140, 1, 1111, 1120)])
def test_loss_and_gradients_over_long_axes(B, K, V, D, dtype):
    test_loss_and_gradients(B, K, V, D, dtype)


@pytest.mark.parametrize("dtype,N,V", [(bf16, 8192, 40000), (f32, 4096, 36000)])
def test_gradients_in_several_pieces_of_the_vocabulary(dtype, N, V):
    """So many rows that the scratch holds the gradient of a part of the vocabulary only; held to 64 bits on the GPU."""
    D = 64
    h, w, t = loss_inputs(4, N // 4, V, D, dtype, seed=3)
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    lse = head.loss(hd, wd, td)["lse"]
    got = head.loss_grad(hd, wd, td, lse)
    dh, dw, bh, bw = hu.gradients(hd.view(N, D), wd, td.view(-1), lse.view(-1).double(), torch.ones(N, device=DEV), 1.0, dtype)
    # the bounds hold for every term in the worst direction: the errors of sums this long stay far inside, which the norms say
    for got, want, bound in ((got["grad_hidden"].double().view(N, D), dh, bh), (got["grad_weight"].double(), dw, bw)):
        assert ((got - want).abs() <= bound).all()
        assert float((got - want).norm() / want.norm()) < (2.0 ** -8 if dtype == bf16 else 2.0 ** -17)


def test_gradient_is_the_slope_of_the_loss():
    """Central differences of the library's own loss along random directions."""
    B, K, V, D = 2, 9, 211, 64
    h, w, t = loss_inputs(B, K, V, D, f32, seed=21)
    head = binding.DraftHead(B * K, D, V, dtype=f32, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    scale = torch.tensor([1 / 16.0], device=DEV)
    grad = head.loss_grad(hd, wd, td, head.loss(hd, wd, td)["lse"], scale=scale)

    def mean(a, b):
        return head.loss(a, b, td)["loss"].double().sum().item() / 16
    eps = 2.0 ** -6
    for seed in range(4):
        for which in (0, 1):
            d = rand(*(h.shape if which == 0 else w.shape), seed=50 + seed).to(DEV)
            d /= d.norm()
            a, b = (mean(hd + s * eps * d, wd) if which == 0 else mean(hd, wd + s * eps * d) for s in (1, -1))
            slope = float(((grad["grad_hidden"] if which == 0 else grad["grad_weight"]).double() * d).sum())
            # 18 losses of up to 16 with an error of 2^-20 of that and weights 1/16, over 2 eps; the cubic term: |d| = 1 along rows of norm below 16 bounds
            # the third derivative of lse along d by 16^3 / 16 a row, times eps^2 / 6, for the weights, whose direction is spread over V rows: a 200th of it
            assert abs((a - b) / (2 * eps) - slope) < 18 * 16 * 2.0 ** -20 / 16 / (2 * eps) + 16 ** 3 / 16 * eps ** 2 / 6 / 100


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("N", [7, 96, 300])
def test_rows_that_do_not_count_and_bad_rows(N, dtype):
    V, D = 333, 96
    h, w, t = loss_inputs(1, N, V, D, dtype, seed=N)
    t[t < 0] = 1
    rw = torch.ones(1, N)
    for k, what in enumerate((float("nan"), float("inf"), 1e30)):         # left out: whatever their hidden states hold
        h[0, k] = what
    t[0, 0], t[0, 1], rw[0, 2] = -1, -100, 0.0
    t[0, 3] = V                                                            # no such token
    h[0, 4, 3] = float("nan")                                              # counts, and is bad
    head = binding.DraftHead(N, D, V, dtype=dtype, training=True)
    hd, wd, td = h.to(DEV), w.to(DEV), t.to(DEV)
    f = head.loss(hd, wd, td)
    b = head.loss_grad(hd, wd, td, f["lse"], row_weight=rw.to(DEV))
    torch.cuda.synchronize()
    loss = f["loss"].cpu()[0]
    assert (loss[:2] == 0).all() and loss[3:5].isnan().all() and torch.isfinite(loss[5:]).all()
    assert int(f["flags"][0]) & (binding.FLAG_BAD_ROW | binding.FLAG_BAD_TOKEN) == binding.FLAG_BAD_ROW | binding.FLAG_BAD_TOKEN
    keep = torch.ones(N, dtype=torch.bool)
    keep[:5] = False
    dh, dw, bh, bw = hu.gradients(h[0, keep], w, t[0, keep], f["lse"].cpu()[0, keep].double(), torch.ones(N - 5), 1.0, dtype)
    assert (b["grad_hidden"][0, :5] == 0).all()
    within(b["grad_hidden"][0, 5:], dh, bh)
    within(b["grad_weight"], dw, bw)
    # no row counts
    b = head.loss_grad(hd, wd, torch.full_like(td, -1), f["lse"])
    assert (b["grad_hidden"] == 0).all() and (b["grad_weight"] == 0).all()


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_large_logits_and_a_sure_row(dtype):
    V, D = 1000, 64
    h, w, t = loss_inputs(2, 4, V, D, dtype, seed=8, scale=200.0)         # logits spread by 200: single tokens hold everything
    head = binding.DraftHead(8, D, V, dtype=dtype)
    f = head.loss(h.to(DEV), w.to(DEV), t.to(DEV))
    loss, lse, z, dz = hu.cross_entropy(h.reshape(8, D), w, t.view(-1))
    bound = hu.lse_bound(z, dz, lse)
    within(f["lse"].view(-1), lse, bound)
    within(f["loss"].view(-1), loss, bound + dz.amax(-1) + 2 * hu.U32 * (loss.abs() + 1))


def test_no_rows():
    head = binding.DraftHead(4, 64, 300, training=True)
    h, t = torch.empty(0, 3, 64, dtype=bf16, device=DEV), torch.empty(0, 3, dtype=torch.int32, device=DEV)
    w = rand(300, 64, seed=1, dtype=bf16).to(DEV)
    f = head.loss(h, w, t)
    b = head.loss_grad(h, w, t, f["lse"], out=dict(grad_hidden=torch.empty_like(h), grad_weight=torch.ones_like(w)))
    torch.cuda.synchronize()
    assert (b["grad_weight"] == 0).all()
    c, s = binding.mx4_quantize(w)
    assert head.logits(h, c, s).shape == (0, 3, 300)


def test_no_rows_and_a_vocabulary_beyond_a_grid_axis():
    V = 4_200_001
    head = binding.DraftHead(1, 32, V, training=True)
    h, t = torch.empty(0, 1, 32, dtype=bf16, device=DEV), torch.empty(0, 1, dtype=torch.int32, device=DEV)
    w, lse = torch.zeros(V, 32, dtype=bf16, device=DEV), torch.empty(0, 1, device=DEV)
    gw = torch.ones_like(w)
    head.loss_grad(h, w, t, lse, out=dict(grad_hidden=torch.empty_like(h), grad_weight=gw))
    assert not gw.any()


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_one_hidden_state_for_all_rows(dtype):
    """Strides of zero, of the hidden states and of the weights: as copies of them."""
    B, K, V, D = 11, 7, 300, 96
    _, w, t = loss_inputs(B, K, V, D, dtype, seed=12)
    one = rand(1, 1, D, seed=13, dtype=dtype).to(DEV).expand(B, K, D)
    head = binding.DraftHead(B * K, D, V, dtype=dtype, training=True)
    wd, td = w.to(DEV), t.to(DEV)
    same = wd[:1].expand(V, D)
    for x, y in ((one, wd), (one, same)):
        a, b = head.loss(x, y, td), head.loss(x.contiguous(), y.contiguous(), td)
        assert torch.equal(a["loss"], b["loss"]) and torch.equal(a["lse"], b["lse"])
        a, b = head.loss_grad(x, y, td, a["lse"]), head.loss_grad(x.contiguous(), y.contiguous(), td, a["lse"])
        assert torch.equal(a["grad_hidden"], b["grad_hidden"]) and torch.equal(a["grad_weight"], b["grad_weight"])


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_loss_strides_and_neighbours(dtype):
    B, K, V, D = 5, 7, 130, 64
    h, w, t = loss_inputs(B, K, V, D, dtype, seed=4)
    wide = torch.full((B, K + 2, D), float("nan"), dtype=dtype, device=DEV)
    wide[:, 2:] = h.to(DEV)
    wr = torch.full((V, 2 * D), float("nan"), dtype=dtype, device=DEV)
    wr[:, :D] = w.to(DEV)
    head = binding.DraftHead(B * K, D, V, dtype=dtype, training=True)
    td = t.to(DEV)
    gh, gw = torch.full_like(wide, 5.0), torch.full_like(wr, 5.0)
    a = head.loss(h.to(DEV), w.to(DEV), td)
    b = head.loss(wide[:, 2:], wr[:, :D], td)
    assert torch.equal(a["loss"], b["loss"]) and torch.equal(a["lse"], b["lse"])
    x = head.loss_grad(h.to(DEV), w.to(DEV), td, a["lse"])
    head.loss_grad(wide[:, 2:], wr[:, :D], td, b["lse"], out=dict(grad_hidden=gh[:, 2:], grad_weight=gw[:, :D]))
    assert torch.equal(x["grad_hidden"], gh[:, 2:]) and torch.equal(x["grad_weight"], gw[:, :D])
    assert (gh[:, :2] == 5).all() and (gw[:, D:] == 5).all()


# ---- together, streams, graphs ------------------------------------------------------------------------------------
def test_a_training_step_then_a_round_under_the_quantised_head():
    """Loss, gradient, an update, 4-bit weights, logits, signals, drawn tokens, verification: as they are used together."""
    B, K, V, D = 6, 4, 1000, 128
    h, w, t = loss_inputs(B, K, V, D, bf16, seed=31)
    t[:, 0] = 3
    head = binding.DraftHead(B * K, D, V, training=True)
    tp = binding.Tapout(B, K, V, draft_sampling=True)
    hd, td = h.to(DEV), t.to(DEV)
    master = w.float().to(DEV)
    wd = master.to(bf16)
    f = head.loss(hd, wd, td)
    n = float((t >= 0).sum())
    g = head.loss_grad(hd, wd, td, f["lse"], scale=torch.tensor([1 / n], device=DEV))
    dh, dw, bh, bw = hu.gradients(h.reshape(-1, D), w, t.view(-1), f["lse"].cpu().view(-1).double(), torch.ones(B * K), 1 / n, bf16)
    within(g["grad_weight"], dw, bw)
    master -= 0.5 * g["grad_weight"].float()
    codes, scales = binding.mx4_quantize(master)
    z = head.logits(hd, codes, scales)
    arm = torch.zeros(B, dtype=torch.int32, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    u = torch.rand(B, K, generator=gen, device=DEV)
    ds = tp.draft_stats(z, arm=arm, u_draft=u)
    target = rand(B, K + 1, V, seed=77, scale=2.0).to(DEV)
    vf = tp.verify(target, z, ds["lse"], ds["logq_tok"], ds["sampled_tok"], ds["n_stop"], torch.rand(B, K, generator=gen, device=DEV),
                   torch.rand(B, generator=gen, device=DEV))
    torch.cuda.synchronize()
    zc = z.cpu().double()
    lse = torch.logsumexp(zc, -1)
    within(ds["lse"], lse, 1e-5 * (1 + lse.abs()))
    tok = ds["sampled_tok"].cpu().long()
    assert (tok >= 0).all() and (tok < V).all() and (ds["flags"] == 0).all() and (vf["flags"] == 0).all()
    within(ds["logq_tok"], zc.gather(2, tok[..., None])[..., 0] - lse, 1e-4 * torch.ones(B, K))
    # the drawn token is where the cumulative probability passes the uniform
    cum = torch.softmax(zc, -1).cumsum(-1)
    uc = u.cpu().double()[..., None]
    assert (cum.gather(2, tok[..., None]) > uc - 1e-5).all()
    assert ((cum.gather(2, (tok[..., None] - 1).clamp(min=0)) <= uc + 1e-5) | (tok[..., None] == 0)).all()
    n_out = vf["n_out"].cpu()
    assert (n_out == vf["accept_len"].cpu() + 1).all() and (n_out <= ds["n_stop"].cpu() + 1).all()


def all_calls(head, h, w, t, scale):
    f = head.loss(h, w, t)
    g = head.loss_grad(h, w, t, f["lse"], scale=scale)
    c, s = binding.mx4_quantize(w)
    return dict(f, **g, z16=head.logits(h, c, s), z4=head.logits(h, c, s, act_bits=4, dtype=f32), v=binding.mx4_dequantize(c, s, w.shape[1]))


def same(a, b):
    for k in a:
        assert torch.equal(a[k].view(torch.uint8) if a[k].is_contiguous() else a[k], b[k].view(torch.uint8) if b[k].is_contiguous() else b[k]), k


@pytest.mark.parametrize("B,K,V,D", [(1, 3, 500, 96), (9, 8, 1111, 256), (3, 150, 900, 128)])
def test_same_bits_on_another_stream_and_in_a_replayed_graph(B, K, V, D):
    head = binding.DraftHead(B * K, D, V, training=True)
    sets = [[x.to(DEV) for x in loss_inputs(B, K, V, D, bf16, seed=s)] for s in (1, 2, 3)]
    scale = torch.tensor([0.125], device=DEV)
    want = [all_calls(head, *x, scale) for x in sets]
    torch.cuda.synchronize()
    same(all_calls(head, *sets[0], scale), want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_calls(head, *sets[1], scale)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    same(got, want[1])
    # a stream given by argument, with outputs of the call's own
    f = head.loss(*sets[2], stream=side)
    g = head.loss_grad(*sets[2], f["lse"], scale=scale, stream=side)
    side.synchronize()
    assert torch.equal(g["grad_weight"], want[2]["grad_weight"])
    held = [x.clone() for x in sets[0]]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = all_calls(head, *held, scale)
    for k in (1, 0, 2, 1):
        for a, b in zip(held, sets[k]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        same(out, want[k])
        same(all_calls(head, *sets[0], scale), want[0])            # eager work of the same head between the replays
        torch.cuda.synchronize()


def test_two_heads_on_two_streams():
    """Calls of two heads under way at once: each as alone."""
    B, K, V, D = 8, 16, 3001, 160
    sets = [[x.to(DEV) for x in loss_inputs(B, K, V, D, bf16, seed=s)] for s in (5, 6)]
    heads = [binding.DraftHead(B * K, D, V, training=True) for _ in sets]
    scale = torch.tensor([0.5], device=DEV)
    want = [all_calls(heads[0], *x, scale) for x in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(all_calls(heads[i], *sets[i], scale))
    torch.cuda.synchronize()
    for i in (0, 1):
        for g in got[i]:
            same(g, want[i])


# ---- refusals -------------------------------------------------------------------------------------------------------
def test_refusals():
    head = binding.DraftHead(8, 64, 100)
    h, w, t = (x.to(DEV) for x in loss_inputs(2, 4, 100, 64, bf16, seed=1))
    c, s = binding.mx4_quantize(w)
    f = head.loss(h, w, t)
    with pytest.raises(binding.TapoutError, match="training"):
        head.loss_grad(h, w, t, f["lse"])
    with pytest.raises(binding.TapoutError, match="max_rows"):
        head.loss(torch.cat([h, h]), w, torch.cat([t, t]))
    with pytest.raises(binding.TapoutError, match="vocab"):
        head.loss(h, torch.cat([w, w]), t)
    with pytest.raises(binding.TapoutError, match="act_bits"):
        head.logits(h, c, s, act_bits=8)
    with pytest.raises(binding.TapoutError, match="overlap"):
        head.logits(h, c, s, out=torch.empty(2, 1, 100, dtype=bf16, device=DEV).expand(2, 4, 100))
    room = torch.empty(2 * 4 * 100, dtype=bf16, device=DEV)
    with pytest.raises(binding.TapoutError, match="overlap"):
        head.logits(h, c, s, out=room.as_strided((2, 4, 100), (100, 100, 1)))
    head.logits(h, c, s, out=room.as_strided((2, 4, 100), (100, 200, 1)))           # sequences inside positions: fine
    with pytest.raises(binding.TapoutError, match="aligned"):
        head.loss(torch.empty(2 * 4 * 64 + 1, dtype=bf16, device=DEV)[1:].view(2, 4, 64), w, t)
    with pytest.raises(ValueError, match="dim|must be"):
        head.loss(h[..., :32], w, t)
    with pytest.raises(ValueError):
        head.loss(h.float(), w, t)
    with pytest.raises(ValueError):
        head.loss(h, w, t.long())
    with pytest.raises(ValueError):
        head.logits(h, c[:50], s)
    with pytest.raises(ValueError, match="cpu"):
        head.loss(h, w, t.cpu())
    with pytest.raises(binding.TapoutError, match="bfloat16"):
        binding.DraftHead(8, 64, 100, dtype=f32).logits(h.float(), c, s)
    with pytest.raises(binding.TapoutError, match="cols"):
        binding.mx4_quantize(torch.zeros(4, 40, device=DEV))
