"""Host-side checks of the draft head's calls: every refusal comes before anything touches a device."""
import ctypes as C

import pytest
import torch

from paper_2511_02017_amd import binding
from tests import head_util as hu


def head_config(**kw):
    c = binding.TapoutHeadConfig(0, 64, 256, 1000, binding.BF16, 1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("change,word", [
    (dict(max_rows=0), "max_rows"), (dict(max_rows=(1 << 20) + 1), "max_rows"), (dict(dim=0), "dim"), (dict(dim=48), "dim"), (dict(dim=65568), "dim"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(dtype=2), "dtype"), (dict(training=2), "training"), (dict(device=-1), "device"),
])
def test_create_rejects_bad_configurations(change, word):
    lib = binding.load_library()
    h = C.c_void_p()
    assert lib.tapout_head_create(C.byref(h), C.byref(head_config(**change))) in (1, 4) and h.value is None
    assert word in lib.tapout_head_last_error(None).decode()


@pytest.mark.parametrize("change,word", [(dict(max_rows=1 << 20, dim=8224), "max_rows"), (dict(vocab=1 << 24, dim=2080), "vocab")])
def test_create_refuses_more_elements_than_a_grid_has_lanes(change, word):
    lib = binding.load_library()
    h = C.c_void_p()
    assert lib.tapout_head_create(C.byref(h), C.byref(head_config(**change))) == 2 and h.value is None
    assert word in lib.tapout_head_last_error(None).decode()


def test_mx4_calls_refuse_more_elements_than_a_grid_has_lanes():
    lib = binding.load_library()
    m = binding.TapoutMatrix(4096, binding.BF16, 65536)
    rows = (1 << 18) + 1
    assert lib.tapout_mx4_quantize(C.byref(m), rows, 65536, 4096, 4096, None) == 2
    assert "2^34" in lib.tapout_head_last_error(None).decode()
    assert lib.tapout_mx4_dequantize(4096, 4096, rows, 65536, C.byref(m), None) == 2
    assert "2^34" in lib.tapout_head_last_error(None).decode()


def test_null_handles():
    lib = binding.load_library()
    h = C.c_void_p()
    assert lib.tapout_head_create(None, C.byref(head_config())) == 1
    assert lib.tapout_head_create(C.byref(h), None) == 1
    assert lib.tapout_head_destroy(None) == 0
    assert lib.tapout_head_logits_mx4(None, None, None, None, 1, 1, 1, None, 16, None, None) == 1
    assert lib.tapout_head_loss(None, None, None, 1, 1, 1, None, None, None, None, None) == 1
    assert lib.tapout_head_loss_grad(None, None, None, 1, 1, 1, None, None, None, None, None, None, None) == 1
    assert "NULL" in lib.tapout_head_last_error(None).decode()


@pytest.mark.parametrize("rows,cols,ptr,dtype,stride,codes,scales,word", [
    (-1, 64, 4096, 1, 64, 4096, 4096, "rows"), (2, 0, 4096, 1, 64, 4096, 4096, "cols"), (2, 40, 4096, 1, 64, 4096, 4096, "cols"),
    (2, 64, 0, 1, 64, 4096, 4096, "NULL"), (2, 64, 4098, 1, 64, 4096, 4096, "aligned"), (2, 64, 4096, 1, 65, 4096, 4096, "aligned"),
    (2, 64, 4096, 7, 64, 4096, 4096, "dtype"), (2, 64, 4096, 1, -64, 4096, 4096, "stride"), (2, 64, 4096, 1, 64, 0, 4096, "NULL"),
    (2, 64, 4096, 1, 64, 4104, 4096, "aligned"), (2, 64, 4096, 1, 64, 4096, 4098, "aligned"),
])
def test_mx4_calls_refuse(rows, cols, ptr, dtype, stride, codes, scales, word):
    lib = binding.load_library()
    m = binding.TapoutMatrix(ptr, dtype, stride)
    assert lib.tapout_mx4_quantize(C.byref(m), rows, cols, codes, scales, None) == 1
    assert word in lib.tapout_head_last_error(None).decode()
    assert lib.tapout_mx4_dequantize(codes, scales, rows, cols, C.byref(m), None) == 1
    assert word in lib.tapout_head_last_error(None).decode()


def test_binding_refuses_cpu_tensors():
    with pytest.raises(ValueError, match="GPU"):
        binding.mx4_quantize(torch.zeros(4, 64))


def test_plain_form_of_the_4_bit_blocks():
    x = torch.tensor([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.1, 7.9, 4.0, 0.26, -0.2] + [0.0] * 20])
    c, s, v = hu.mx4(x)
    assert s[0, 0] == 127 and c[0, :12].tolist() == [0, 2, 2, 4, 4, 6, 6, 15, 7, 6, 1, 8]
    assert v[0, :12].tolist() == [0, 1, 1, 2, 2, 4, 4, -6, 6, 4, 0.5, 0]
    c, s, v = hu.mx4(torch.tensor([[3.0e-39] + [0.0] * 31, [float("inf")] + [1.0] * 31, [0.0] * 32, [2.0 ** 127] + [0.0] * 31], dtype=torch.float64))
    assert s[:, 0].tolist() == [0, 255, 0, 252] and v[1].isnan().all() and v[3, 0] == 2.0 ** 127
