"""The host's check that filtered logits are not written over the logits, against every byte of both."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

from paper_2511_02017_amd import binding

CSRC = os.path.join(os.path.dirname(os.path.abspath(binding.__file__)), "csrc")
INCLUDE = os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include")
SOURCE = """#include "%s/rows_meet.h"
extern "C" int meet(const tapout_logits *x, const tapout_logits *y, int B, int K, int V) { return tapout::rows_meet(*x, *y, B, K, V); }
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("rows_meet")
    (d / "m.cpp").write_text(SOURCE % CSRC)
    subprocess.run([cc, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", INCLUDE, "-o", str(d / "m.so"), str(d / "m.cpp")], check=True)
    f = C.CDLL(str(d / "m.so")).meet
    f.argtypes = [C.POINTER(binding.TapoutLogits)] * 2 + [C.c_int] * 3
    return lambda x, y, B, K, V: bool(f(C.byref(x), C.byref(y), B, K, V))


def bytes_of(t, B, K, V):
    e = 4 if t.dtype == binding.F32 else 2
    rows = [t.ptr + (b * t.stride_b + k * t.stride_k) * e for b in range(B) for k in range(K)]
    return [set(range(r, r + V * e)) for r in rows]


def test_against_every_byte(meet):
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    while min(seen.values()) < 1500:
        B, K, V = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 6)
        dt = [rng.choice((binding.F32, binding.BF16)) for _ in range(2)]
        strides = [rng.choice((0, V, V + 1, 2 * V, 2 * V + 3, K * V, 2 * K * V, 2 * K * V + 2, B * V, 3 * B * V)) for _ in range(4)]
        x = binding.TapoutLogits(4096 + 4 * rng.randint(-60, 60), dt[0], strides[0], strides[1])
        y = binding.TapoutLogits(4096, dt[1], strides[2], strides[3])
        rows = bytes_of(y, B, K, V)
        sb, sk = strides[2:]
        apart = (K == 1 or sk >= V) and (B == 1 or sb >= V) if 1 in (B, K) else (sk >= V and sb >= (K - 1) * sk + V) or (sb >= V and sk >= (B - 1) * sb + V)
        if not apart:                                          # refused before
            continue
        assert len(set().union(*rows)) == sum(map(len, rows))
        want = bool(set().union(*rows) & set().union(*bytes_of(x, B, K, V)))
        assert meet(x, y, B, K, V) == want, (x.ptr, dt, strides, B, K, V)
        seen[want] += 1


def test_what_a_program_does(meet):
    f32, bf16 = binding.F32, binding.BF16
    at = lambda p, dt, b, k: binding.TapoutLogits(p, dt, b, k)          # noqa: E731
    V, base = 128256, 1 << 40
    assert meet(at(base, bf16, 4 * V, V), at(base, bf16, 4 * V, V), 8, 4, V)                              # the logits themselves
    assert not meet(at(base, bf16, 4 * V, V), at(base + 8 * 4 * V * 2, bf16, 4 * V, V), 8, 4, V)          # behind them
    assert meet(at(base, bf16, 4 * V, V), at(base + (8 * 4 * V - 1) * 2, bf16, 4 * V, V), 8, 4, V)        # from their last element on
    assert not meet(at(base, f32, 8 * V, 2 * V), at(base + 4 * V, f32, 8 * V, 2 * V), 8, 4, V)            # side by side
    assert meet(at(base, f32, 8 * V, 2 * V), at(base + 4 * V - 4, f32, 8 * V, 2 * V), 8, 4, V)
    assert not meet(at(base, f32, 0, 0), at(base + 4 * V, f32, 4 * V, V), 8, 4, V)                        # one row for all
    assert meet(at(base, f32, 0, 0), at(base - 4, f32, 4 * V, V), 8, 4, V)
