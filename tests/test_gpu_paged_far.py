"""Attention over pages at positions whose distance to the query, times the heads of a group, passes 31 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("rows", ["by the rule", "0", "1"])
@pytest.mark.parametrize("causal", [True, False])
def test_far_keys_count(causal, rows, monkeypatch):
    """20 million keys of one head, found through a table that names eight pages again and again, with a bound that asks for few CTAs.

    The keys of the first sixth are the likelier ones, and their values are around 1 where the others' are around -1.  Tolerance: a tile's product is added to an
    fp32 sum in four steps, each of which may cut it by 2^-23: keys / 16 * 2^-23 of the largest value where one CTA has all keys; probabilities and outputs
    in bf16, 2^-8 each, the sums of probabilities like the values."""
    from paper_2605_12825_b200 import binding as B
    monkeypatch.delenv("ORTHRUS_TC_SMALL_ROWS", raising=False)
    if rows != "by the rule":
        monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", rows)
    d, page, G, K, P = 64, 1024, 128, 1, 20 * 1000 * 1000 + 77
    n_table = -(-(P + K) // page)
    g = torch.Generator().manual_seed(G)
    k, v = (torch.randn(8, 1, page, d, generator=g) for _ in range(2))
    q = torch.randn(1, K, 1, d, generator=g) + 0.1 * torch.randn(1, K, G, d, generator=g)
    k[:4] += 2.5 * q[0, 0, 0] / q[0, 0, 0].norm()
    v = 0.2 * v + torch.tensor([1.0] * 4 + [-1.0] * 4).view(8, 1, 1, 1)
    q, k, v = q.to(BF16), k.to(BF16), v.to(BF16)
    far = n_table // 6
    table = torch.cat((torch.randint(0, 4, (far,), generator=g), torch.randint(4, 8, (n_table - far,), generator=g))).to(torch.int32)
    # every row of a page counts as often as the table names it; the last table entry ends with the block
    times = torch.bincount(table[:-1].long(), minlength=8).double().view(8, 1).repeat(1, page)
    times[int(table[-1]), :P + K - (n_table - 1) * page] += 1
    s = torch.einsum("hd,pjd->hpj", q[0, 0].double(), k[:, 0].double()) / d ** 0.5
    w = torch.exp(s - s.amax((1, 2), keepdim=True)) * times
    want = torch.einsum("hpj,pjd->hd", w, v[:, 0].double()) / w.sum((1, 2)).view(-1, 1)
    assert float(want.mean()) > 0.0                    # (without the first sixth it is around -1)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    layer = B.make_paged_layer(k.cuda(), v.cuda(), table.view(1, -1).cuda(), i32([P]), G, K, None, 1000)
    ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    out = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    (B.orthrus_paged_ar_attend if causal else B.orthrus_paged_diffusion_attend)(layer, q.cuda(), out, ws)
    assert B.orthrus_read_status(ws) == 0
    off = 2 * (P / 16) * 2.0 ** -23 + 2 * 2.0 ** -8
    assert float((out[0, 0].cpu().double() - want).abs().max()) <= off * float(v.float().abs().max())
