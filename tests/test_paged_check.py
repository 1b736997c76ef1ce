"""The check of paged attention results finds what it is there for: a lost key, a lost tile, a lost part, at every length that the tests on a GPU use."""
import math

import pytest
import torch

import _attend_check as A
from test_gpu_paged_attend import make

BF16, F64 = torch.bfloat16, torch.float64
SHAPES = [(1, 4, 1, 128, 64, 20000), (1, 8, 2, 128, 16, 40001), (3, 3, 1, 64, 16, 12345), (1, 8, 2, 64, 16, 1000), (2, 8, 2, 128, 64, 300), (1, 4, 1, 64, 16, 65),
          (2, 4, 2, 128, 32, 9000), (1, 8, 8, 128, 16, 129), (5, 8, 2, 64, 16, 2000)]


def honest(t, lens, new, causal):
    """What an exact evaluation with the roundings of the bf16 kernels gives."""
    B, K, Hq, d = t["q"].shape
    Hkv, page = t["k"].shape[1], t["k"].shape[2]
    out = torch.full(t["q"].shape, 7.0, dtype=BF16)
    for b in range(B):
        n = lens[b] + new[b]
        pos = torch.arange(n)
        at = t["table"][b][pos // page].long()
        k, v = (t[x][at, :, pos % page].to(F64).transpose(0, 1) for x in ("k", "v"))
        s = torch.einsum("ihgd,hnd->ihgn", t["q"][b, :new[b]].to(F64).view(new[b], Hkv, Hq // Hkv, d), k) / math.sqrt(d)
        if causal:
            s.masked_fill_((pos > lens[b] + torch.arange(new[b])[:, None])[:, None, None], -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.einsum("ihgn,hnd->ihgd", p.to(BF16).to(F64), v) / p.sum(-1, keepdim=True)
        out[b, :new[b]] = o.reshape(new[b], Hq, d).to(BF16)
    return out


@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_the_check_tells_right_from_wrong(shape, K):
    B, Hq, Hkv, d, page, length = shape
    lens, new = [max(length - 1000 * b, 50) for b in range(B)], [K] * B
    t = make(B, K, Hq, Hkv, d, page, BF16, lens, new, seed=length)
    A.plant(t, lens, new, True)
    t["k"], t["v"] = t["k"].nan_to_num(), t["v"].nan_to_num()
    v_top = float(t["v"].float().abs().max())
    want, spread = A.reference(t["q"], t["k"], t["v"], t["table"], lens, new, True)
    assert A.faults(honest(t, lens, new, True), want, spread, new, v_top, BF16) == []
    n = min(lens) + K
    tiles = -(-n // 64)
    for skip in [(0, 1), (n - K, n - K + 1), (n // 2, n // 2 + 1), (0, 64), (64 * (tiles // 2), 64 * (tiles // 2) + 64), (64 * (tiles - 1) - K, n - K), (n // 4, n // 2)]:
        if skip[1] - skip[0] >= n or skip[0] < 0:
            continue
        lost, _ = A.reference(t["q"], t["k"], t["v"], t["table"], lens, new, True, skip=[skip])
        where = [b for b in range(B) if lens[b] == min(lens)]
        found = A.faults(lost.to(BF16), want, spread, new, v_top, BF16)
        assert any(f.startswith(f"request {where[0]}:") for f in found), (skip, found)


def test_fp32_and_rows_that_do_not_exist():
    lens, new = [700, 5], [2, 0]
    t = make(2, 2, 4, 2, 64, 16, torch.float32, lens, new)
    t["k"], t["v"] = t["k"].nan_to_num(), t["v"].nan_to_num()
    want, spread = A.reference(t["q"], t["k"], t["v"], t["table"], lens, new, True)
    assert bool(torch.isnan(want[1]).all())
    assert A.faults(want.float(), want, spread, new, 4.0, torch.float32) == []
    lost, _ = A.reference(t["q"], t["k"], t["v"], t["table"], lens, new, True, skip=[(699, 700)])
    assert A.faults(lost.float(), want, spread, new, 4.0, torch.float32) != []
    nan = want.float()
    nan[0, 1, 2, 3] = math.nan
    assert A.faults(nan, want, spread, new, 4.0, torch.float32) != []
    bad = want.to(BF16)
    bad[0, 0, 0, 0] = math.nan
    assert len(A.faults(bad, want, spread, new, 4.0, BF16)) == 2
