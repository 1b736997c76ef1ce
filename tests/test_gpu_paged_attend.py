"""Attention over pages against the plain 64-bit implementation."""
import math
import random

import pytest
import torch

import _paged_ref as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(params=["by the rule", "0", "1"], autouse=True)
def kernel(request, monkeypatch):
    """Few rows run on either tensor-core kernel: as the rule has it, on the one that shares lengths out, on the keys kernel where it fits."""
    monkeypatch.delenv("ORTHRUS_TC_SMALL_ROWS", raising=False)
    if request.param in ("0", "1"):
        monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", request.param)


def make(B, K, Hq, Hkv, d, page, dtype, lens, new, seed=1, spare_width=0, q_scale=1.0):
    """Pages dealt at random; whatever no row of a request occupies is NaN, and table entries that no row needs are outside the pool."""
    g = torch.Generator().manual_seed(seed)
    width = max(1, max(-(-(n + a) // page) for n, a in zip(lens, new))) + spare_width
    n_pages = B * width + 2
    table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(torch.int32)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    k, v = rand(n_pages, Hkv, page, d).to(dtype), rand(n_pages, Hkv, page, d).to(dtype)
    live = torch.zeros(n_pages, page, dtype=torch.bool)
    for b in range(B):
        n = lens[b] + new[b] if new[b] else 0
        pos = torch.arange(n)
        live[table[b][pos // page].long(), pos % page] = True
        table[b, -(-n // page):] = 2 ** 30
    dead = ~live[:, None, :, None].expand_as(k)
    k[dead] = math.nan
    v[dead] = math.nan
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(q=(rand(B, K, Hq, d) * q_scale).to(dtype), k=k, v=v, table=table, len=i32(lens), new=i32(new))


def run(t, Hq, causal, hint=0, flags=0, use_new=True, scale=0.0, calls=1, path=None):
    from paper_2605_12825_b200 import binding as B
    d = {n: x.cuda() for n, x in t.items()}
    layer = B.make_paged_layer(d["k"], d["v"], d["table"], d["len"], Hq, t["q"].shape[1], d["new"] if use_new else None, hint, scale, flags)
    ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    n = d["q"].numel()
    buf = torch.full((n + 2048,), 7.0, dtype=t["q"].dtype, device="cuda")
    out = buf[1024:1024 + n].view(t["q"].shape)
    call = B.orthrus_paged_ar_attend if causal else B.orthrus_paged_diffusion_attend
    B.orthrus_set_path(path or "auto")
    try:
        for _ in range(calls):
            call(layer, d["q"], out, ws)
        status = B.orthrus_read_status(ws)
    finally:
        B.orthrus_set_path("auto")
    assert bool((buf[:1024] == 7.0).all()) and bool((buf[1024 + n:] == 7.0).all())
    return out.cpu(), status


def check(got, want, new, v_top, dtype):
    """Rows that exist within the tolerance, the others as they were.

    bf16: the output's rounding, half a step; probabilities rounded to bf16, half a step each of a sum whose terms are at most
    max |v| (2^-8 max|v|, reached only if all roundings agree in sign), and fp32 exponentials and sums.  fp32: sums of fp32 products over the keys."""
    for b, n in enumerate(new):
        assert bool((got[b, n:] == 7.0).all())
        g, w = got[b, :n].double(), want[b, :n]
        if dtype == BF16:
            assert bool(((g - w).abs() <= 2.0 ** -8 * w.abs() + 2.0 ** -8 * v_top).all())
            # roundings of thousands of terms do not all agree: the mean error is far below (a few 2^-9 / sqrt(keys that count))
            if w.numel() > 1000:
                assert float((g - w).norm() / w.norm()) < 2.0 ** -7
        else:
            assert bool(((g - w).abs() <= 2e-5 * v_top).all())


def case(B, K, Hq, Hkv, d, page, lens, new=None, dtype=BF16, **kw):
    new = [K] * B if new is None else new
    t = make(B, K, Hq, Hkv, d, page, dtype, lens, new, seed=B + K + d + page)
    v_top = float(t["v"].float().nan_to_num().abs().max())
    for causal in (True, False):
        want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], lens, new, causal)
        got, status = run(t, Hq, causal, **kw)
        assert status == 0
        check(got, want, new, v_top, dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 63, 64, 65, 127, 200, 1000])
def test_one_token(d, page, length):
    case(2, 1, 8, 2, d, page, [length, max(0, length - 7)])


@pytest.mark.parametrize("group,kv", [(1, 8), (2, 3), (4, 2), (5, 1), (7, 2), (8, 1), (16, 1), (17, 1), (32, 1), (48, 1), (71, 1), (130, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_one_token_groups(group, kv, d):
    case(3, 1, group * kv, kv, d, 16, [300, 0, 77])


@pytest.mark.parametrize("K", [1, 2, 5, 8, 16, 31, 64])
@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks(K, group, d):
    case(3, K, 2 * group, 2, d, 32, [0, 61, 130])


@pytest.mark.parametrize("K,group", [(1, 4), (4, 4), (6, 5), (16, 4), (33, 3)])
def test_some_rows_of_a_block_and_idle_requests(K, group):
    case(5, K, 2 * group, 2, 128, 16, [100, 90, 0, 500, 64], [K, 0, max(1, K - 1), K // 2, min(K, 3)])
    case(2, K, 2 * group, 2, 64, 16, [100, 90], [0, 0])


def test_ragged_batches():
    rng = random.Random(8)
    for B, top in ((33, 300), (65, 90), (100, 40), (7, 3000), (2, 9000)):
        case(B, 1, 4, 2, 128, 16, [rng.randint(0, top) for _ in range(B)])


@pytest.mark.parametrize("hint", [1, 50, 700, 2000])
def test_bound_below_the_lengths_is_served_too(hint):
    case(3, 2, 8, 2, 128, 16, [700, 20, 333], hint=hint)


@pytest.mark.parametrize("B,Hkv,length", [(1, 1, 20000), (1, 2, 40001), (3, 1, 12345)])
def test_long_requests_are_cut_and_joined(B, Hkv, length):
    case(B, 1, 4 * Hkv, Hkv, 128, 64, [length - 1000 * b for b in range(B)])
    case(B, 3, 3 * Hkv, Hkv, 64, 16, [length - 1000 * b for b in range(B)])


def test_flags_and_null_counts_give_the_same_bits():
    from paper_2605_12825_b200 import binding as B
    lens = [500, 17, 1200]
    t = make(3, 4, 8, 2, 128, 16, BF16, lens, [4] * 3)
    first, _ = run(t, 8, True)
    for kw in (dict(flags=B.LAYER_CACHE_QUIESCENT), dict(flags=B.LAYER_NO_EARLY_LAUNCH), dict(use_new=False), dict(calls=5),
               dict(flags=B.LAYER_CACHE_QUIESCENT, calls=20)):
        again, status = run(t, 8, True, **kw)
        assert status == 0 and torch.equal(first, again)


@pytest.mark.parametrize("d,page,dtype", [(32, 16, BF16), (256, 16, BF16), (64, 1, BF16), (128, 8, BF16), (32, 4, F32), (64, 16, F32),
                                          (128, 32, F32), (256, 1024, F32)])
def test_shapes_of_the_plain_arithmetic(d, page, dtype):
    case(3, 5, 6, 2, d, page, [100, 0, 33], [5, 2, 0], dtype=dtype)
    case(1, 1, 4, 1, d, page, [777], dtype=dtype)


def test_paths_agree():
    lens = [500, 17, 1200]
    t = make(3, 4, 8, 2, 128, 16, BF16, lens, [4] * 3)
    a, _ = run(t, 8, True)
    b, _ = run(t, 8, True, path="simt")
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -6


def test_softmax_scale():
    t = make(2, 2, 4, 2, 128, 16, BF16, [100, 5], [2, 2])
    want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], [100, 5], [2, 2], True, 0.3)
    got, _ = run(t, 4, True, scale=0.3)
    check(got, want, [2, 2], float(t["v"].float().nan_to_num().abs().max()), BF16)


@pytest.mark.parametrize("size", [30.0, -30.0, 300.0])
def test_large_scores(size):
    """Scores of hundreds of either sign: the running maximum moves, late keys win, exponentials vanish."""
    lens, new = [1000, 200], [2, 2]
    t = make(2, 2, 8, 2, 128, 16, BF16, lens, new, q_scale=abs(size))
    if size < 0:
        t["k"] = -t["k"].abs()
        t["q"] = t["q"].abs()
    want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], lens, new, True)
    got, _ = run(t, 8, True)
    v_top = float(t["v"].float().nan_to_num().abs().max())
    # a score of s is off by fp32 sums of 128 products, 2^-18 of it at most, and so is its exponential
    off = 2.0 ** -18 * float((t["q"].double().norm(dim=-1).max()) * t["k"].double().nan_to_num().norm(dim=-1).max()) / math.sqrt(128)
    for b in range(2):
        assert bool(((got[b].double() - want[b]).abs() <= 2.0 ** -8 * want[b].abs() + (2.0 ** -8 + 2 * off) * v_top).all())


def test_scores_of_minus_infinity_do_not_count():
    lens, new = [100], [1]
    t = make(1, 1, 2, 1, 128, 16, BF16, lens, new)
    t["q"][..., 0] = 1.0
    page = 16
    for pos in list(range(0, 64)) + [70, 99]:                # the whole first tile, and some later ones
        t["k"][t["table"][0, pos // page].long(), 0, pos % page, 0] = -math.inf
    want = ref.attend(t["q"], t["k"].nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf), t["v"].nan_to_num(), t["table"], lens, new, True)
    got, _ = run(t, 2, True)
    assert bool(torch.isfinite(want).all())
    check(got, want, new, float(t["v"].float().nan_to_num().abs().max()), BF16)


def test_bad_lengths_and_pages_are_reported():
    from paper_2605_12825_b200 import binding as B
    t = make(3, 2, 4, 2, 128, 16, BF16, [40, 40, 40], [2, 2, 2])
    want, _ = run(t, 4, True)
    t["len"][1] = 10 ** 6                    # clamped to what the table holds: 46 + 2 rows, the last ones NaN
    got, status = run(t, 4, True)
    assert status == B.DEV_BAD_CACHE_LEN
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    t["len"][1] = -5
    assert run(t, 4, True)[1] == B.DEV_BAD_CACHE_LEN
    t["len"][1] = 40
    t["new"][1] = 3
    assert run(t, 4, True)[1] == B.DEV_BAD_CACHE_LEN
    t["new"][1] = 2
    for bad in (-1, 2 ** 30):
        u = {n: x.clone() for n, x in t.items()}
        u["table"][1, 1] = bad
        for path in ("auto", "simt"):
            got, status = run(u, 4, True, path=path)
            assert status == B.DEV_BAD_PAGE
            if path == "auto":
                assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


def test_captured_with_lengths_that_change():
    """A captured graph serves whatever the lengths and tables hold when it is replayed; two graphs share a workspace in turn."""
    from paper_2605_12825_b200 import binding as B
    t = make(2, 1, 8, 2, 128, 16, BF16, [900, 900], [1, 1])
    t["k"], t["v"] = t["k"].nan_to_num(), t["v"].nan_to_num()
    d = {n: x.cuda() for n, x in t.items()}
    layer = B.make_paged_layer(d["k"], d["v"], d["table"], d["len"], 8, 1, d["new"])
    ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    out = [torch.zeros_like(d["q"]) for _ in range(2)]
    graphs = []
    for o, call in zip(out, (B.orthrus_paged_ar_attend, B.orthrus_paged_diffusion_attend)):
        call(layer, d["q"], o, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(layer, d["q"], o, ws)
        graphs.append(g)
    for lens, new in (([900, 900], [1, 1]), ([3, 700], [1, 1]), ([0, 0], [1, 0]), ([899, 1], [1, 1])):
        d["len"].copy_(torch.tensor(lens))
        d["new"].copy_(torch.tensor(new))
        for o in out:
            o.fill_(7.0)
        for g in graphs:
            g.replay()
        want = ref.attend(t["q"], t["k"], t["v"], t["table"], lens, new, True)
        assert B.orthrus_read_status(ws) == 0
        for o in out:
            check(o.cpu(), want, new, float(t["v"].float().abs().max()), BF16)


def test_another_stream():
    from paper_2605_12825_b200 import binding as B
    t = make(2, 1, 8, 2, 128, 16, BF16, [900, 100], [1, 1])
    want, _ = run(t, 8, True)
    d = {n: x.cuda() for n, x in t.items()}
    layer = B.make_paged_layer(d["k"], d["v"], d["table"], d["len"], 8, 1, d["new"])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    out = torch.zeros_like(d["q"])
    ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    torch.cuda.synchronize()
    B.orthrus_paged_ar_attend(layer, d["q"], out, ws, st)
    assert B.orthrus_read_status(ws, st) == 0
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("d,page,dtype", [(32, 16, BF16), (256, 16, BF16), (128, 1, BF16), (64, 4, F32), (128, 16, F32), (256, 32, F32)])
@pytest.mark.parametrize("lens,hint", [([5000, 0, 63], 0), ([64, 65, 127], 4000), ([1, 2047, 3000], 3000), ([9001], 9001), ([700, 20], 5)])
def test_plain_arithmetic_cut_over_the_keys(d, page, dtype, lens, hint):
    B = len(lens)
    case(B, 1, 6, 2, d, page, lens, dtype=dtype, hint=hint)
    case(B, 3, 5, 1, d, page, lens, [3, 1, 2][:B], dtype=dtype, hint=hint)


def test_plain_arithmetic_with_more_units_than_counts():
    case(40, 4, 12, 6, 32, 16, [(37 * b) % 300 for b in range(40)], dtype=F32)
    case(7, 64, 6, 2, 256, 16, [(97 * b) % 200 for b in range(7)])


def test_plain_arithmetic_leaves_values_alone_that_a_row_does_not_see():
    """Row 1 of the block is NaN and infinity throughout; row 0 does not see it."""
    t = make(1, 2, 4, 2, 256, 16, BF16, [300], [2])
    want = ref.attend(t["q"], t["k"].nan_to_num(), t["v"].nan_to_num(), t["table"], [300], [2], True)
    page, row = int(t["table"][0, 301 // 16]), 301 % 16
    t["k"][page, :, row], t["v"][page, :, row] = math.nan, math.inf
    got, status = run(t, 4, True)
    assert status == 0
    check(got[:, :1], want[:, :1], [1], float(t["v"].float().nan_to_num(posinf=0.0).abs().max()), BF16)


def test_calls_of_all_kinds_share_a_workspace():
    """What one call leaves in a workspace does not touch the next one, of whatever shape or kind."""
    from paper_2605_12825_b200 import binding as B
    torch.manual_seed(3)
    calls, size = [], 0
    for shape in ((1, 1, 8, 2, 128, 16, BF16, [9000], [1]), (2, 1, 8, 2, 256, 16, BF16, [3000, 500], [1, 1]),
                  (5, 4, 32, 8, 128, 64, BF16, [2000, 10, 777, 3500, 1], [4] * 5), (3, 1, 4, 2, 128, 16, F32, [2500, 1, 900], [1] * 3),
                  (2, 64, 4, 2, 64, 32, BF16, [3001, 50], [64, 7])):
        t = make(*shape)
        d = {n: x.cuda() for n, x in t.items()}
        layer = B.make_paged_layer(d["k"], d["v"], d["table"], d["len"], shape[2], shape[1], d["new"])
        out = torch.zeros_like(d["q"])
        size = max(size, B.orthrus_paged_attend_workspace_bytes(layer))
        calls.append((layer, d, out))
    kc, vc = (torch.randn(2, 2, 4096, 128, device="cuda").to(BF16) for _ in range(2))
    plain = B.make_layer(kc, vc, torch.tensor([4000, 300], dtype=torch.int32, device="cuda"), 8, 16, 4000)
    q, kb, vb = (torch.randn(2, 16, h, 128, device="cuda").to(BF16) for h in (8, 2, 2))
    out = torch.zeros_like(q)
    size = max(size, B.orthrus_attend_workspace_bytes(plain))
    logits, draft = torch.randn(8, 16, 5000, device="cuda"), torch.zeros(8, 16, dtype=torch.int32, device="cuda")
    counts = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in ((8,), (8, 16), (8, 16), (8,))]
    size = max(size, B.orthrus_consensus_workspace_bytes(8, 16, 5000))

    def everything(ws_of):
        results = []
        for layer, d, o in calls:
            o.zero_()
            B.orthrus_paged_ar_attend(layer, d["q"], o, ws_of())
            results.append(o.clone())
        B.orthrus_ar_verify_attend(plain, q, kb, vb, out, ws_of())
        B.orthrus_consensus_accept(logits, draft, *counts, ws_of())
        results += [out.clone()] + [c.clone() for c in counts]
        return results

    want = everything(lambda: B.new_workspace(size))
    ws = B.new_workspace(size)
    for _ in range(3):
        for a, b in zip(everything(lambda: ws), want):
            assert torch.equal(a, b)
    # what is in the workspace behind its header may be anything
    ws.view(torch.uint8)[256:].fill_(0x5a)
    for a, b in zip(everything(lambda: ws)[:5], want):
        assert torch.equal(a, b)
    assert B.orthrus_read_status(ws) == 0


def test_pool_past_32_bits():
    """A pool of 5 GB whose last pages are used: element offsets and byte offsets pass 2^31 and 2^32."""
    from paper_2605_12825_b200 import binding as B
    Hkv, page, d = 8, 64, 128
    n_pages = (5 << 30) // (Hkv * page * d * 2)
    k = torch.zeros(n_pages, Hkv, page, d, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator().manual_seed(4)
    length, ids = 500, [n_pages - 1 - 2 * j for j in range(8)]
    small_k, small_v = (torch.randn(8, Hkv, page, d, generator=g).to(BF16) for _ in range(2))
    k[ids], v[ids] = small_k.cuda(), small_v.cuda()
    q = torch.randn(1, 1, 32, d, generator=g).to(BF16)
    table, lens = torch.tensor([ids], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda")
    layer = B.make_paged_layer(k, v, table, lens, 32, 1)
    ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    # a row is written there and attended to
    slots = torch.tensor([[ids[length // page] * page + length % page]], device="cuda")
    new_k, new_v = (torch.randn(1, 1, Hkv, d, generator=g).to(BF16) for _ in range(2))
    B.orthrus_paged_kv_write(layer, slots, new_k.cuda(), new_v.cuda())
    small_k[length // page, :, length % page], small_v[length // page, :, length % page] = new_k[0, 0], new_v[0, 0]
    want = ref.attend(q, small_k, small_v, torch.arange(8).view(1, 8), [length], [1], True)
    for path in ("auto", "simt"):
        B.orthrus_set_path(path)
        out = torch.full_like(q, 7.0).cuda()
        B.orthrus_paged_ar_attend(layer, q.cuda(), out, ws)
        B.orthrus_set_path("auto")
        assert B.orthrus_read_status(ws) == 0
        check(out.cpu(), want, [1], float(small_v.float().abs().max()), BF16)
