"""Host-side checks of the norm's, the 8-bit blocks', the sampling's and the distillation's calls, and of their plain forms: nothing
here touches a device."""
import ctypes as C
import math

import pytest
import torch

from paper_2511_02017_amd import binding
from tests import operators_util as ou


def test_null_handles():
    lib = binding.load_library()
    assert lib.tapout_sample(None, None, 1, 1, 1, *([None] * 12)) == 1
    assert "NULL" in lib.tapout_last_error(None).decode()
    assert lib.tapout_head_norm(None, None, None, None, 1e-5, 1, 1, *([None] * 6)) == 1
    assert lib.tapout_head_norm_grad(None, None, None, None, None, None, 1, 1, None, None, None) == 1
    assert lib.tapout_head_logits_fp8(None, None, None, None, None, None, 1, 1, 1, None, None, None) == 1
    assert lib.tapout_head_distill(None, None, None, 1, 1, 1, None, None, 1, *([None] * 6)) == 1
    assert lib.tapout_head_distill_grad(None, None, None, 1, 1, 1, None, None, 1, *([None] * 8)) == 1
    assert "NULL" in lib.tapout_head_last_error(None).decode()


@pytest.mark.parametrize("rows,cols,block,ptr,dtype,stride,codes,scales,status,word", [
    (-1, 64, 1, 4096, 1, 64, 4096, 4096, 1, "rows"), (2, 0, 1, 4096, 1, 64, 4096, 4096, 1, "cols"), (2, 40, 1, 4096, 1, 64, 4096, 4096, 1, "cols"),
    (2, 65568, 1, 4096, 1, 65568, 4096, 4096, 1, "cols"), (2, 64, 0, 4096, 1, 64, 4096, 4096, 2, "block_rows"), (2, 64, 64, 4096, 1, 64, 4096, 4096, 2, "block_rows"),
    (2, 64, 1, 0, 1, 64, 4096, 4096, 1, "NULL"), (2, 64, 128, 4098, 1, 64, 4096, 4096, 1, "aligned"), (2, 64, 1, 4096, 1, 65, 4096, 4096, 1, "aligned"),
    (2, 64, 1, 4096, 7, 64, 4096, 4096, 1, "dtype"), (2, 64, 1, 4096, 1, -64, 4096, 4096, 1, "stride"), (2, 64, 1, 4096, 1, 64, 0, 4096, 1, "NULL"),
    (2, 64, 1, 4096, 1, 64, 4096, 0, 1, "NULL"), (2, 64, 1, 4096, 1, 64, 4104, 4096, 1, "aligned"), (2, 64, 1, 4096, 1, 64, 4096, 4098, 1, "aligned"),
    ((1 << 18) + 1, 65536, 128, 4096, 1, 65536, 4096, 4096, 2, "2^34"),
])
def test_fp8_calls_refuse(rows, cols, block, ptr, dtype, stride, codes, scales, status, word):
    lib = binding.load_library()
    m = binding.TapoutMatrix(ptr, dtype, stride)
    assert lib.tapout_fp8_quantize(C.byref(m), rows, cols, block, codes, scales, None) == status
    assert word in lib.tapout_head_last_error(None).decode()
    assert lib.tapout_fp8_dequantize(codes, scales, rows, cols, block, C.byref(m), None) == status
    assert word in lib.tapout_head_last_error(None).decode()


def test_binding_refuses_cpu_tensors():
    with pytest.raises(ValueError, match="GPU"):
        binding.fp8_quantize(torch.zeros(4, 64))
    with pytest.raises(ValueError, match="GPU"):
        binding.fp8_dequantize(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1), 64, out=torch.zeros(4, 64))


def test_plain_form_of_the_8_bit_blocks():
    x = torch.zeros(3, 130)
    x[0, :4] = torch.tensor([448.0, 1.0, -17.0, 2.0 ** -10])
    x[1, 128] = 4.48
    x[2, 5] = math.inf
    q, s = ou.fp8(x)
    assert s[0].tolist()[0] == pytest.approx(1.0, rel=1e-7) and s[1, 1] == pytest.approx(0.01, rel=1e-6) and math.isnan(s[2, 0])
    assert q[0, :4].tolist() == [448.0, 1.0, -16.0, 0.0] and q[1, 128] == 448.0 and q[2, :128].isnan().all() and (q[2, 128:] == 0).all()
    assert (s[0, 1], s[1, 0]) == (s[1, 0], s[0, 1]) and float(s[1, 0]) > 0
    q, s = ou.fp8(torch.cat((x, torch.ones(130, 130))), 128)
    assert s.shape == (2, 2) and math.isnan(s[0, 0]) and q[:128, :128].isnan().all() and (q[128:, 128:130] == 448).all()


def test_plain_form_of_the_filters():
    x = torch.tensor([1.0, 3.0, -math.inf, 3.0, 2.0, 0.0])
    keep = lambda *a: ou.filtered(x, *a, None)["keep"].nonzero()[:, 0].tolist()          # noqa: E731
    assert keep(1.0, 0, 1.0, 0.0) == [0, 1, 3, 4, 5] and keep(1.0, 1, 1.0, 0.0) == [1] and keep(1.0, 3, 1.0, 0.0) == [1, 3, 4] and keep(0.0, 3, 1.0, 0.0) == [1]
    assert keep(1.0, 0, 0.5, 0.0) == [1, 3] and keep(1.0, 2, 0.5, 0.0) == [1] and keep(1.0, 0, 1.0, 0.3) == [1, 3, 4] and keep(1.0, 0, 1.0, 1.0) == [1, 3]
    a = ou.filtered(x, 1.0, 2, 1.0, 0.0, 0.5)
    assert a["token"] == 3 and a["logq"] == pytest.approx(math.log(0.5)) and ou.filtered(x, 1.0, 2, 1.0, 0.0, 0.49)["token"] == 1
    assert ou.filtered(x, math.nan, 0, 1.0, 0.0, 0.5)["bad"] and ou.filtered(torch.tensor([1.0, math.inf]), 1.0, 0, 1.0, 0.0, 0.5)["bad"]


def test_plain_form_of_the_distillation():
    """Against automatic differentiation of the formula."""
    g = torch.Generator().manual_seed(1)
    N, V, D, T = 5, 17, 8, 4
    h, w = torch.randn(N, D, generator=g, dtype=torch.float64).requires_grad_(), torch.randn(V, D, generator=g, dtype=torch.float64).requires_grad_()
    ids = torch.tensor([[1, 2, 3, 4], [5, -1, 6, -1], [-1, -1, -1, -1], [7, 7, 8, 7], [16, 0, 1, 2]], dtype=torch.int32)
    logits = torch.randn(N, T, generator=g)
    for given in (None, torch.logsumexp(logits, -1) + 0.3):
        real = ids >= 0
        tl = torch.where(real, logits.double(), -math.inf)
        ref = torch.logsumexp(torch.where(real.any(-1, keepdim=True), tl, 0.0), -1) if given is None else given.double()
        t = torch.exp(tl - ref[:, None])
        z = h @ w.T
        logp = torch.log_softmax(z, -1)
        loss = torch.where(real, t * (torch.where(real, tl - ref[:, None], 0.0) - logp.gather(1, ids.clamp(min=0).long())), 0.0).sum(-1)
        dh, dw = torch.autograd.grad(loss.sum(), (h, w))
        got = ou.distillation(h.detach(), w.detach(), ids, logits, given, torch.ones(N), 1.0, torch.float32)
        assert torch.allclose(got[0], loss) and torch.allclose(got[3], dh) and torch.allclose(got[4], dw)
        assert got[2].tolist() == [True, True, False, True, True]


def test_8_bit_codes_that_are_not_contiguous_are_refused_not_copied():
    """A copy would be made on the current stream, which nothing orders before the stream of the call."""
    codes, scales, out = torch.zeros(2, 4, 128, dtype=torch.uint8), torch.ones(2, 4, 1), torch.zeros(2, 2, 96)
    for c, s, word in ((codes[:, :2], scales[:, :2].contiguous(), "codes"), (codes[:, :2].contiguous(), scales[:, :2], "scales"),
                       (codes.transpose(0, 1)[:2], scales[:, :2].contiguous(), "codes")):
        with pytest.raises(ValueError, match=f"{word} must be contiguous"):
            binding.fp8_dequantize(c, s, 96, out=out)
