"""Attention over pages within what its roundings allow (_attend_check.py), on each kernel: one lost key, tile or piece of a request is found."""
import random

import pytest
import torch

import _attend_check as A
from test_gpu_paged_attend import BF16, F32, make, run

pytestmark = pytest.mark.gpu


def case(monkeypatch, kernel, B, K, Hq, Hkv, d, page, lens, new=None, dtype=BF16, **kw):
    monkeypatch.delenv("ORTHRUS_TC_SMALL_ROWS", raising=False)
    if kernel in ("0", "1"):
        monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", kernel)
    new = [K] * B if new is None else new
    t = make(B, K, Hq, Hkv, d, page, dtype, lens, new, seed=B + K + d + page)
    A.plant(t, lens, new, True)
    v_top = float(t["v"].float().nan_to_num().abs().max())
    for causal in (True, False):
        want, spread = A.reference(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], lens, new, causal)
        got, status = run(t, Hq, causal, path="simt" if kernel == "simt" else None, **kw)
        assert status == 0
        assert A.faults(got, want, spread, new, v_top, dtype) == []
        for b, n in enumerate(new):
            assert bool((got[b, n:] == 7.0).all())


kernels = pytest.mark.parametrize("kernel", ["rule", "0", "1", "simt"])


@kernels
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 15, 63, 64, 65, 128, 1000])
def test_one_token(kernel, d, length, monkeypatch):
    case(monkeypatch, kernel, 2, 1, 8, 2, d, 16, [length, max(0, length - 7)])


@kernels
@pytest.mark.parametrize("B,Hkv,length", [(1, 1, 20000), (1, 2, 40001), (3, 1, 12345)])
def test_long_requests(kernel, B, Hkv, length, monkeypatch):
    case(monkeypatch, kernel, B, 1, 4 * Hkv, Hkv, 128, 64, [length - 1000 * b for b in range(B)])
    case(monkeypatch, kernel, B, 3, 3 * Hkv, Hkv, 64, 16, [length - 1000 * b for b in range(B)])


@kernels
@pytest.mark.parametrize("B,top", [(33, 300), (65, 90), (100, 40), (7, 3000), (2, 9000)])
def test_ragged_batches(kernel, B, top, monkeypatch):
    rng = random.Random(B)
    case(monkeypatch, kernel, B, 1, 4, 2, 128, 16, [rng.randint(0, top) for _ in range(B)])


@kernels
@pytest.mark.parametrize("K,Hq,Hkv,d", [(2, 8, 2, 128), (16, 8, 2, 128), (16, 6, 1, 64), (32, 8, 2, 128), (64, 4, 2, 64), (64, 14, 2, 128)])
def test_blocks(kernel, K, Hq, Hkv, d, monkeypatch):
    case(monkeypatch, kernel, 5, K, Hq, Hkv, d, 32, [0, 61, 130, 2000, 4097], [K, max(1, K - 1), K // 2, K, min(K, 3)])


@kernels
@pytest.mark.parametrize("hint", [1, 50, 700, 20000])
def test_bounds_below_and_above_the_lengths(kernel, hint, monkeypatch):
    case(monkeypatch, kernel, 3, 2, 8, 2, 128, 16, [5000, 20, 333], hint=hint)


@pytest.mark.parametrize("d,page,dtype", [(32, 16, BF16), (256, 16, BF16), (128, 1, BF16), (64, 4, F32), (128, 16, F32), (256, 32, F32)])
@pytest.mark.parametrize("lens,hint", [([5000, 0, 63], 0), ([64, 65, 127], 4000), ([1, 2047, 3000], 3000), ([9001], 9001), ([700, 20], 5)])
def test_shapes_of_the_plain_arithmetic(d, page, dtype, lens, hint, monkeypatch):
    B = len(lens)
    case(monkeypatch, "rule", B, 1, 6, 2, d, page, lens, dtype=dtype, hint=hint)
    case(monkeypatch, "rule", B, 3, 5, 1, d, page, lens, [3, 1, 2][:B], dtype=dtype, hint=hint)
