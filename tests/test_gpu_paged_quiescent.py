"""The promise of a quiescent cache with the write of the block's rows right ahead: the prefix may be read ahead of the wait, the block's rows and the queries
not."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("kernel", ["0", "1", "simt"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("K,Hq,Hkv,d,page,lens", [
    (1, 32, 8, 128, 16, [4095, 4096, 100, 0]), (1, 8, 2, 64, 16, [63, 64, 65, 1000] * 8), (16, 16, 4, 128, 32, [500, 2000, 48, 4000, 0, 64, 1, 3333]),
    (64, 8, 2, 128, 64, [1000, 10, 640, 127] * 6), (32, 12, 4, 64, 16, [77] * 40), (4, 32, 8, 128, 16, [8000])])
def test_rows_written_right_ahead_are_seen(kernel, causal, K, Hq, Hkv, d, page, lens, monkeypatch):
    """Many rounds of new rows to the same slots and attention to them, without a pause: each has to see its own round's rows.  The same rounds with plain
    stream order and without the promise say what it should be, bit for bit."""
    from paper_2605_12825_b200 import binding as B
    monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", kernel if kernel in "01" else "0")
    monkeypatch.delenv("ORTHRUS_NO_EARLY_LAUNCH", raising=False)
    g = torch.Generator(device="cuda").manual_seed(K + d)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    batch, rounds = len(lens), 12
    width = -(-(max(lens) + K) // page)
    n_pages = batch * width
    table = torch.randperm(n_pages, generator=g, device="cuda").view(batch, width).to(I32)
    ln = torch.tensor(lens, dtype=I32, device="cuda")
    pos = ln[:, None].long() + torch.arange(K, device="cuda")
    slots = table.gather(1, pos // page).long() * page + pos % page
    pages = rand(2, n_pages, Hkv, page, d)
    q, kb, vb = rand(rounds, batch, K, Hq, d), rand(rounds, batch, K, Hkv, d), rand(rounds, batch, K, Hkv, d) + torch.arange(rounds, device="cuda").view(-1, 1, 1, 1, 1).to(BF16)
    call = B.orthrus_paged_ar_attend if causal else B.orthrus_paged_diffusion_attend
    B.orthrus_set_path("simt" if kernel == "simt" else "auto")
    results = []
    try:
        for flags in (B.LAYER_NO_EARLY_LAUNCH, B.LAYER_CACHE_QUIESCENT, 0):
            k, v = pages[0].clone(), pages[1].clone()
            layer = B.make_paged_layer(k, v, table, ln, Hq, K, None, 0, 0.0, flags)
            ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
            q_rot, out = torch.zeros_like(q), torch.zeros_like(q)
            torch.cuda.synchronize()
            for _ in range(1 if flags == B.LAYER_NO_EARLY_LAUNCH else 4):
                for i in range(rounds):
                    B.orthrus_rope_paged_kv_write(layer, slots, q[i], kb[i], vb[i], 10000.0, q_rot[i])
                    call(layer, q_rot[i], out[i], ws)
            assert B.orthrus_read_status(ws) == 0
            results.append(out)
    finally:
        B.orthrus_set_path("auto")
    assert bool(torch.isfinite(results[0]).all()) and not torch.equal(results[0][0], results[0][1])
    for other in results[1:]:
        assert torch.equal(other, results[0])


@pytest.mark.parametrize("kernel", ["0", "1"])
def test_a_captured_step_with_the_promise(kernel, monkeypatch):
    """The promise in a graph of layers: each layer's write, then its attention, the lengths growing between replays."""
    from paper_2605_12825_b200 import binding as B
    monkeypatch.setenv("ORTHRUS_TC_SMALL_ROWS", kernel)
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    batch, K, Hq, Hkv, d, page, width, layers = 6, 1, 16, 4, 128, 16, 40, 3
    table = torch.randperm(batch * width, generator=g, device="cuda").view(batch, width).to(I32)
    q, kb, vb = rand(layers, batch, K, Hq, d), rand(layers, batch, K, Hkv, d), rand(layers, batch, K, Hkv, d)
    pool = rand(layers, 2, batch * width, Hkv, page, d)

    def loop(flags, steps=20):
        ln = torch.tensor([500, 63, 0, 64, 127, 300], dtype=I32, device="cuda")
        k = pool.clone()
        slots = torch.zeros(batch, K, dtype=torch.int64, device="cuda")
        descr = [B.make_paged_layer(k[n, 0], k[n, 1], table, ln, Hq, K, None, 0, 0.0, flags) for n in range(layers)]
        ws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(descr[0]))
        q_rot, out = torch.zeros_like(q), torch.zeros_like(q)

        def step():
            for n in range(layers):
                B.orthrus_rope_paged_kv_write(descr[n], slots, q[n], kb[n], vb[n], 10000.0, q_rot[n])
                B.orthrus_paged_ar_attend(descr[n], q_rot[n], out[n], ws)

        def prepare():
            slots.copy_(table.gather(1, (ln[:, None] // page).long()).long() * page + ln[:, None] % page)

        prepare()
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        seen = []
        for _ in range(steps):
            prepare()
            graph.replay()
            seen.append(out.clone())
            ln.add_(1)
            vb.mul_(-1)
        assert B.orthrus_read_status(ws) == 0
        return torch.stack(seen)

    want = loop(B.LAYER_NO_EARLY_LAUNCH)
    assert torch.equal(loop(B.LAYER_CACHE_QUIESCENT), want)
