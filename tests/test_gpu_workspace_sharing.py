"""One workspace for calls of all kinds: what lies behind its header when a call starts does not matter to it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def contiguous(B, batch, hq, hkv, block, capacity, lens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    cache = rand(batch, hkv, capacity, 128), rand(batch, hkv, capacity, 128), torch.tensor(lens, dtype=torch.int32, device="cuda")
    layer = B.make_layer(*cache, hq, block, max(lens))
    layer.tensors = cache
    q, k, v = rand(batch, block, hq, 128), rand(batch, block, hkv, 128), rand(batch, block, hkv, 128)
    out = torch.empty_like(q)

    def call(ws):
        out.fill_(7.0)
        B.orthrus_ar_verify_attend(layer, q, k, v, out, ws)
        return out.clone()

    return call, B.orthrus_attend_workspace_bytes(layer)


def paged(B, batch, hq, hkv, block, length, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    width = -(-(length + block) // 64)
    table = torch.randperm(batch * width, generator=g, device="cuda").view(batch, width).to(torch.int32)
    layer = B.make_paged_layer(rand(batch * width, hkv, 64, 128), rand(batch * width, hkv, 64, 128), table,
                               torch.full((batch,), length, dtype=torch.int32, device="cuda"), hq, block)
    q = rand(batch, block, hq, 128)
    out = torch.empty_like(q)

    def call(ws):
        out.fill_(7.0)
        B.orthrus_paged_ar_attend(layer, q, out, ws)
        return out.clone()

    return call, B.orthrus_paged_attend_workspace_bytes(layer)


@pytest.mark.parametrize("schedule", ["stream", None])
def test_the_attention_calls_share_a_workspace(schedule, monkeypatch):
    """Both schedules of the contiguous attention, beside paged calls whose pieces reach far into the workspace."""
    from paper_2605_12825_b200 import binding as B
    monkeypatch.delenv("ORTHRUS_TC_SCHEDULE", raising=False)
    if schedule:
        monkeypatch.setenv("ORTHRUS_TC_SCHEDULE", schedule)
    monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", "0")
    made = [contiguous(B, 3, 32, 8, 16, 5000, [4500, 10, 2222], 1), paged(B, 32, 32, 8, 32, 1500, 2), contiguous(B, 40, 8, 2, 16, 700, [17 * b for b in range(40)], 3),
            paged(B, 2, 8, 2, 1, 9000, 4)]
    size = max(n for _, n in made)
    want = [call(B.new_workspace(size)) for call, _ in made]
    ws = B.new_workspace(size)
    for fill in (0x00, 0x5a, 0x01, 0xff):
        for call, first in zip((c for c, _ in made), want):
            ws[256:].fill_(fill)
            assert torch.equal(call(ws), first)
    for _ in range(3):
        for (call, _), first in zip(made, want):
            assert torch.equal(call(ws), first)
    assert B.orthrus_read_status(ws) == 0
