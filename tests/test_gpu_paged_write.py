"""Writes into pages: copies bit for bit, rotations against 64 bits, nothing else touched."""
import pytest
import torch

import _paged_ref as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def make(B, K, Hq, Hkv, d, page, dtype, seed, lens, new, q_width=1.0):
    g = torch.Generator().manual_seed(seed)
    width = max(1, max(-(-(n + a) // page) for n, a in zip(lens, new)))
    n_pages = B * width + 3
    table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(torch.int32)
    slots = torch.full((B, K), -1, dtype=torch.int64)
    for b in range(B):
        for i in range(new[b]):
            pos = lens[b] + i
            slots[b, i] = int(table[b, pos // page]) * page + pos % page
    rand = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    return dict(k=rand(n_pages, Hkv, page, d), v=rand(n_pages, Hkv, page, d), table=table, slots=slots,
                lens=torch.tensor(lens, dtype=torch.int32), q=rand(B, K, Hq, d) * q_width, kb=rand(B, K, Hkv, d), vb=rand(B, K, Hkv, d))


def layer_of(t, Hq, K):
    from paper_2605_12825_b200 import binding as B
    d = {k: v.cuda() for k, v in t.items()}
    return B, d, B.make_paged_layer(d["k"], d["v"], d["table"], d["lens"], Hq, K)


SHAPES = [  # B, K, Hq, Hkv, d, page
    (1, 1, 1, 1, 32, 1), (3, 1, 4, 2, 64, 16), (2, 5, 6, 3, 128, 32), (4, 16, 32, 8, 128, 16), (1, 70, 10, 2, 64, 64),
    (2, 3, 7, 7, 256, 8), (1, 300, 5, 1, 128, 1024), (17, 2, 3, 3, 32, 4)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_copy_and_rotation(shape, dtype):
    B, K, Hq, Hkv, d, page = shape
    lens = [(37 * b * b + 5) % 900 for b in range(B)]
    new = [K if b % 3 != 2 else K // 2 for b in range(B)]
    t = make(B, K, Hq, Hkv, d, page, dtype, 5, lens, new)
    # the plain write
    b_, dv, layer = layer_of(t, Hq, K)
    ws = b_.new_workspace(256)
    b_.orthrus_paged_kv_write(layer, dv["slots"], dv["kb"], dv["vb"], ws)
    assert b_.orthrus_read_status(ws) == 0
    want_k, want_v = t["k"].clone(), t["v"].clone()
    for b in range(B):
        for i in range(new[b]):
            s = int(t["slots"][b, i])
            want_k[s // page, :, s % page] = t["kb"][b, i]
            want_v[s // page, :, s % page] = t["vb"][b, i]
    assert torch.equal(dv["k"].cpu(), want_k) and torch.equal(dv["v"].cpu(), want_v)
    # the rotary write
    b_, dv, layer = layer_of(t, Hq, K)
    q_out = torch.full_like(dv["q"], 7.0)
    b_.orthrus_rope_paged_kv_write(layer, dv["slots"], dv["q"], dv["kb"], dv["vb"], 10000.0, q_out)
    got_q, got_k, got_v = q_out.cpu(), dv["k"].cpu(), dv["v"].cpu()
    assert torch.equal(got_v, want_v)
    # A rounding of the result (half a step of the type), and what is lost before it, relative to the pair's size.  bf16 rows, fp32
    # arithmetic: the angle's fraction of a turn in float 2^-26 turns = 2^-23.3, sine and cosine two units 2^-23, two products and a
    # sum 3 * 2^-24, all times sqrt(2): below 2^-20.5.  fp32 rows, fp64: 1200 radians known to 4 * 2^-53 of themselves on both sides, 2^-39.
    half, inner = torch.finfo(dtype).eps / 2, 2.0 ** -20.5 if dtype == BF16 else 2.0 ** -39

    def check(got, want, src):
        size = torch.cat([torch.hypot(*src.double().chunk(2, -1))] * 2, -1)
        assert bool(((got.double() - want).abs() <= half * want.abs() * 1.0001 + inner * (1 + half) * size).all())

    rest = torch.ones(t["k"].shape[0], page, dtype=torch.bool)
    for b in range(B):
        for i in range(K):
            if i >= new[b]:
                assert bool((got_q[b, i] == 7.0).all())
                continue
            s = int(t["slots"][b, i])
            rest[s // page, s % page] = False
            check(got_q[b, i], ref.rotated(t["q"][b, i], lens[b] + i, 10000.0), t["q"][b, i])
            check(got_k[s // page, :, s % page], ref.rotated(t["kb"][b, i], lens[b] + i, 10000.0), t["kb"][b, i])
    keep = rest[:, None, :, None].expand_as(t["k"])
    assert torch.equal(got_k[keep], t["k"][keep])


@pytest.mark.parametrize("pos", [0, 1, 4095, 131071, 1_000_003])
def test_far_positions(pos):
    t = make(1, 1, 4, 2, 128, 1024, BF16, 9, [pos], [1])
    b_, dv, layer = layer_of(t, 4, 1)
    q_out = torch.empty_like(dv["q"])
    b_.orthrus_rope_paged_kv_write(layer, dv["slots"], dv["q"], dv["kb"], dv["vb"], 10000.0, q_out)
    want = ref.rotated(t["q"][0, 0], pos, 10000.0)
    size = torch.cat([torch.hypot(*t["q"][0, 0].double().chunk(2, -1))] * 2, -1)
    # the angle in turns: double, off by 2^-53 of itself; its fraction in float, off by 2^-25 turns; sine and cosine of that
    assert bool(((q_out[0, 0].cpu().double() - want).abs() <= 2.0 ** -9 * want.abs() * 1.0001 * 2 + 2.0 ** -20 * size).all())
    if pos == 0:
        assert torch.equal(q_out.cpu(), t["q"])


def test_in_place_queries_and_matching_the_contiguous_write():
    """The same rows through the contiguous cache's call: equal up to one rounding (its products are in 64 bits)."""
    from paper_2605_12825_b200 import binding as b_
    B, K, Hq, Hkv, d, page = 3, 4, 8, 2, 128, 16
    lens = [3, 40, 77]
    t = make(B, K, Hq, Hkv, d, page, BF16, 2, lens, [K] * B)
    _, dv, layer = layer_of(t, Hq, K)
    q = dv["q"].clone()
    b_.orthrus_rope_paged_kv_write(layer, dv["slots"], q, dv["kb"], dv["vb"], 10000.0, q)
    kc = torch.zeros(B, Hkv, 128, d, dtype=BF16, device="cuda")
    vc, q2 = torch.zeros_like(kc), torch.empty_like(q)
    flat = b_.make_layer(kc, vc, dv["lens"], Hq, K)
    b_.orthrus_rope_block_kv_write(flat, dv["q"], dv["kb"], dv["vb"], 10000.0, q2)
    step = torch.maximum(q.float().abs(), q2.float().abs()) * 2.0 ** -7 + 1e-6
    assert bool(((q.float() - q2.float()).abs() <= step).all())
    for b in range(B):
        for i in range(K):
            s = int(t["slots"][b, i])
            assert torch.equal(dv["v"][s // page, :, s % page], vc[b, :, lens[b] + i])


def test_slots_outside_the_pool_are_skipped_and_reported():
    B, K, Hq, Hkv, d, page = 2, 3, 4, 2, 64, 16
    t = make(B, K, Hq, Hkv, d, page, BF16, 4, [5, 9], [K] * B)
    total = t["k"].shape[0] * page
    t["slots"][0, 1] = total
    t["slots"][1, 2] = 2 ** 40
    b_, dv, layer = layer_of(t, Hq, K)
    ws = b_.new_workspace(256)
    b_.orthrus_paged_kv_write(layer, dv["slots"], dv["kb"], dv["vb"], ws)
    assert b_.orthrus_read_status(ws) == b_.DEV_BAD_PAGE
    want = t["v"].clone()
    for b in range(B):
        for i in range(K):
            s = int(t["slots"][b, i])
            if s < total:
                want[s // page, :, s % page] = t["vb"][b, i]
    assert torch.equal(dv["v"].cpu(), want)


def test_commit_len():
    t = make(4, 8, 2, 1, 64, 16, BF16, 4, [0, 10, 24, 30], [2] * 4)     # tables of two pages: 32 positions
    b_, dv, layer = layer_of(t, 2, 8)
    ws = b_.new_workspace(256)
    n = torch.tensor([8, 0, 8, 3], dtype=torch.int32, device="cuda")
    b_.orthrus_paged_commit_len(layer, n, ws)
    assert dv["lens"].tolist() == [8, 10, 32, 30] and b_.orthrus_read_status(ws) == b_.DEV_APPEND_OVERFLOW
