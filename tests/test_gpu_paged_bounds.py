"""What attention over pages does with lengths and counts that a table cannot hold, on each of its kernels."""
import pytest
import torch

import _paged_ref as ref
from test_gpu_paged_attend import BF16, F32, check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", ["0", "1", "simt"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts", [None, [32, 20]])
@pytest.mark.parametrize("causal", [True, False])
def test_a_block_longer_than_the_table_is_cut_and_reported(kernel, dtype, counts, causal, monkeypatch):
    """A table of one page of 16 positions and a block of 32 rows: 16 of them are served, and the status word says so."""
    from paper_2605_12825_b200 import binding as B
    monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", kernel if kernel in "01" else "0")
    t = make(2, 16, 4, 2, 64, 16, dtype, [0, 0], [16, 16])
    want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], [0, 0], [16, 16], causal)
    t["q"] = torch.cat((t["q"], torch.full_like(t["q"], float("nan"))), 1)
    if counts:
        t["new"] = torch.tensor(counts, dtype=torch.int32)
    got, status = run(t, 4, causal, use_new=counts is not None, path="simt" if kernel == "simt" else None)
    assert status == B.DEV_BAD_CACHE_LEN
    check(got, torch.cat((want, want), 1), [16, 16], float(t["v"].float().nan_to_num().abs().max()), dtype)


@pytest.mark.parametrize("kernel", ["0", "1", "simt"])
def test_a_block_that_fills_the_table_is_in_order(kernel, monkeypatch):
    monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", kernel if kernel in "01" else "0")
    t = make(2, 32, 4, 2, 64, 16, BF16, [0, 0], [16, 16])            # (room for 16 rows, of 32 that the call brings)
    want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], [0, 0], [16, 16], True)
    got, status = run(t, 4, True, path="simt" if kernel == "simt" else None)
    assert status == 0
    check(got, want, [16, 16], float(t["v"].float().nan_to_num().abs().max()), BF16)
