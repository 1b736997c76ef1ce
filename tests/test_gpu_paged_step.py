"""The paged calls together, as a serving loop makes them: against the contiguous cache's calls, and captured into one graph."""
import pytest
import torch

import _paged_ref as ref

pytestmark = pytest.mark.gpu
BF16, I32, I64 = torch.bfloat16, torch.int32, torch.int64


class Pool:
    """Requests on a paged cache: tables, lengths, list of free pages."""

    def __init__(self, batch, hkv, d, page, n_pages, width, max_new):
        z = lambda *s, t=I32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.page = page
        self.k, self.v = (torch.full((n_pages, hkv, page, d), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
        self.len, self.new, self.held, self.granted = z(batch), z(batch), z(batch), z(batch)
        self.table = z(batch, width)
        self.free = torch.randperm(n_pages, device="cuda").to(I32)
        self.n_free = torch.full((1,), n_pages, dtype=I32, device="cuda")
        self.slots = z(batch, max_new, t=I64)

    def grow(self, B, ws):
        B.orthrus_page_tables(self.page, self.len, self.new, self.held, self.held, self.table, self.free, self.n_free, self.n_free, self.granted,
                              self.slots, ws)


@pytest.mark.parametrize("batch,hq,hkv,d,K,page", [(3, 8, 2, 128, 8, 16), (5, 16, 4, 128, 16, 32), (2, 4, 2, 64, 4, 16), (40, 8, 2, 128, 1, 16)])
def test_cycles_match_the_contiguous_cache(batch, hq, hkv, d, K, page):
    """Prompts, then generation cycles in place: both views, greedy consensus, the commit.  The contiguous calls get the same projections; their
    outputs agree as two roundings of one result do, and tokens, lengths and cache rows are equal."""
    from paper_2605_12825_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(batch)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    cap, vocab = 512, 200
    prompt = torch.randint(1, 150, (batch,), generator=g, device="cuda").to(I32)
    most = int(prompt.max())
    pool = Pool(batch, hkv, d, page, batch * (cap // page) + 3, cap // page, most)
    kc, vc = (torch.zeros(batch, hkv, cap, d, dtype=BF16, device="cuda") for _ in range(2))
    flat_len = torch.zeros(batch, dtype=I32, device="cuda")
    ws = B.new_workspace(256)
    # prompts: one write of ragged rows
    pool.new.copy_(prompt)
    pool.grow(B, ws)
    assert torch.equal(pool.granted, prompt)
    kb, vb = rand(batch, most, hkv, d), rand(batch, most, hkv, d)
    wide = B.make_paged_layer(pool.k, pool.v, pool.table, pool.len, hq, most, pool.granted)
    B.orthrus_paged_kv_write(wide, pool.slots, kb, vb, ws)
    for b in range(batch):
        n = int(prompt[b])
        kc[b, :, :n], vc[b, :, :n] = kb[b, :n].transpose(0, 1), vb[b, :n].transpose(0, 1)
    pool.len.copy_(prompt)
    flat_len.copy_(prompt)
    # cycles
    pool.slots = torch.zeros(batch, K, dtype=I64, device="cuda")
    layer = B.make_paged_layer(pool.k, pool.v, pool.table, pool.len, hq, K, pool.granted, cap - K)
    flat = B.make_layer(kc, vc, flat_len, hq, K, cap - K, 0.0, B.LAYER_BLOCK_IN_CACHE)
    aws = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))
    fws = B.new_workspace(B.orthrus_attend_workspace_bytes(flat))
    cws = B.new_workspace(B.orthrus_consensus_workspace_bytes(batch, K, vocab))
    i32 = lambda *s: torch.zeros(*s, dtype=I32, device="cuda")  # noqa: E731
    for cycle in range(6):
        pool.new.fill_(K)
        pool.grow(B, ws)
        assert bool((pool.granted == K).all())
        for paged_call, flat_call in ((B.orthrus_paged_diffusion_attend, B.orthrus_diffusion_block_attend),
                                      (B.orthrus_paged_ar_attend, B.orthrus_ar_verify_attend)):
            q, kb, vb = rand(batch, K, hq, d), rand(batch, K, hkv, d), rand(batch, K, hkv, d)
            q1, q2 = torch.empty_like(q), torch.empty_like(q)
            B.orthrus_rope_paged_kv_write(layer, pool.slots, q, kb, vb, 10000.0, q1, ws)
            B.orthrus_rope_block_kv_write(flat, q, kb, vb, 10000.0, q2, fws)
            o1, o2 = torch.empty_like(q), torch.empty_like(q)
            paged_call(layer, q1, o1, aws)
            flat_call(flat, q2, None, None, o2, fws)
            # each of queries and keys may be rounded another way in a few places, probabilities and outputs in all: 2^-8 each, of values up
            # to the largest of V
            assert float((o1.float() - o2.float()).abs().max()) <= 4 * 2.0 ** -8 * float(vb.float().abs().max())
            assert float((o1.float() - o2.float()).norm() / o2.float().norm()) < 2.0 ** -6
        logits, draft = rand(batch, K, vocab), torch.randint(0, vocab, (batch, K), generator=g, device="cuda").to(I32)
        n, com, arg, nxt = i32(batch), i32(batch, K), i32(batch, K), i32(batch)
        B.orthrus_consensus_accept(logits, draft, n, com, arg, nxt, cws)
        B.orthrus_paged_commit_len(layer, n, ws)
        B.orthrus_commit_len(flat, n, fws)
        assert torch.equal(pool.len, flat_len)
    assert B.orthrus_read_status(ws) == 0 and B.orthrus_read_status(aws) == 0 and B.orthrus_read_status(fws) == 0
    # the cache rows: values equal bit for bit, keys up to a rounding (the contiguous call rotates in 64 bits)
    for b in range(batch):
        m = int(pool.len[b])
        pos = torch.arange(m, device="cuda")
        at = pool.table[b][pos // page].long()
        assert torch.equal(pool.v[at, :, pos % page], vc[b, :, :m].transpose(0, 1))
        x, y = pool.k[at, :, pos % page].float(), kc[b, :, :m].transpose(0, 1).float()
        assert bool(((x - y).abs() <= 2.0 ** -7 * torch.maximum(x.abs(), y.abs()) + 1e-6).all())


def test_a_captured_decoding_step_serves_growing_requests():
    """One graph: pages, rotary write, attention, sampling, lengths.  Replayed as the requests grow, join and end, it leaves what the plain
    forms compute step by step."""
    from paper_2605_12825_b200 import binding as B
    batch, hq, hkv, d, page, width, vocab, n_pages = 4, 8, 2, 64, 16, 6, 300, 20
    g = torch.Generator(device="cuda").manual_seed(5)
    pool = Pool(batch, hkv, d, page, n_pages, width, 1)
    pool.k.zero_()
    pool.v.zero_()
    layer = B.make_paged_layer(pool.k, pool.v, pool.table, pool.len, hq, 1, pool.granted)
    q, kb, vb = (torch.zeros(batch, 1, h, d, dtype=BF16, device="cuda") for h in (hq, hkv, hkv))
    q_rot, out = torch.zeros_like(q), torch.zeros_like(q)
    head = torch.randn(hq * d, vocab, generator=g, device="cuda").to(BF16)
    logits = torch.zeros(batch, vocab, dtype=BF16, device="cuda")
    t, u = torch.full((batch,), 0.9, device="cuda"), torch.zeros(batch, device="cuda")
    k, p = torch.full((batch,), 40, dtype=I32, device="cuda"), torch.full((batch,), 0.9, device="cuda")
    token, logprob = torch.zeros(batch, dtype=I32, device="cuda"), torch.zeros(batch, device="cuda")
    ws, aws = B.new_workspace(256), B.new_workspace(B.orthrus_paged_attend_workspace_bytes(layer))

    def step():
        pool.grow(B, ws)
        B.orthrus_rope_paged_kv_write(layer, pool.slots, q, kb, vb, 10000.0, q_rot, ws)
        B.orthrus_paged_ar_attend(layer, q_rot, out, aws)
        torch.matmul(out.view(batch, -1), head, out=logits)
        B.orthrus_sample_tokens(logits, t, k, p, None, u, token, logprob)
        B.orthrus_paged_commit_len(layer, pool.granted, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                     # (new is 0: nothing grows)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rows = [([], []) for _ in range(batch)]        # what each request's cache should hold: rotated keys, values
    lens = [0] * batch
    for n in range(70):
        new = [1, int(n >= 10), int(n % 3 != 2), int(n < 60)]
        if n == 40:                                # request 2 ends, its pages go back
            pool.len[2] = 0
            lens[2], rows[2] = 0, ([], [])
            new[2] = 0
        pool.new.copy_(torch.tensor(new))
        for x in (q, kb, vb):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        u.copy_(torch.rand(batch, generator=g, device="cuda"))
        before = out.clone()
        graph.replay()
        torch.cuda.synchronize()
        granted = pool.granted.tolist()
        assert granted == new
        for b in range(batch):
            if not granted[b]:
                assert torch.equal(out[b], before[b])
                continue
            rows[b][0].append(ref.rotated(kb[b, 0].cpu(), lens[b], 10000.0).to(BF16))
            rows[b][1].append(vb[b, 0].cpu())
            lens[b] += 1
        assert pool.len.tolist() == lens
        if n % 10 == 9 or n in (40, 41):
            for b in range(batch):
                if not granted[b]:
                    continue
                ks, vs = torch.stack(rows[b][0]).double(), torch.stack(rows[b][1]).double()
                qr = ref.rotated(q[b, 0].cpu(), lens[b] - 1, 10000.0)
                want = torch.stack([torch.softmax(ks[:, h // (hq // hkv)] @ qr[h] / d ** 0.5, 0) @ vs[:, h // (hq // hkv)] for h in range(hq)])
                # queries and keys rounded (2^-8 of scores of a few units), probabilities, outputs
                assert float((out[b, 0].cpu().double() - want).abs().max()) <= 2.0 ** -4
                want_token, _, margin = ref.sample(logits[b].cpu(), float(t[b]), 40, float(p[b]), 0.0, float(u[b]))
                assert margin < 2.0 ** -26 or int(token[b]) == want_token
    held = pool.held.tolist()
    mine = [x for b in range(batch) for x in pool.table[b, :held[b]].tolist()]
    assert sorted(mine + pool.free[:int(pool.n_free)].tolist()) == list(range(n_pages))
    assert B.orthrus_read_status(ws) == 0 and B.orthrus_read_status(aws) == 0


def test_drafts_drawn_by_the_sampler_keep_the_verifiers_distribution():
    """Drafts sampled from the diffusion logits, tested by the sampled consensus: the first committed token is distributed as the AR view's,
    whatever the drafts' distribution is."""
    from paper_2605_12825_b200 import binding as B
    g = torch.Generator().manual_seed(3)
    vocab, n = 12, 40000
    ar, diff = torch.randn(vocab, generator=g) * 1.2, torch.randn(vocab, generator=g) * 1.2
    ar, diff = ar.to(BF16), diff.to(BF16)
    T = 0.8
    gpu = torch.Generator(device="cuda").manual_seed(4)
    lg_a, lg_d = ar.cuda().expand(n, 1, vocab).contiguous(), diff.cuda().expand(n, 1, vocab).contiguous()
    u = torch.rand(3, n, generator=gpu, device="cuda")
    draft = torch.zeros(n, dtype=I32, device="cuda")
    B.orthrus_sample_tokens(lg_d.view(n, vocab), torch.full((n,), T, device="cuda"), None, None, None, u[0].contiguous(), draft)
    count = torch.bincount(draft.long().cpu(), minlength=vocab).double() / n
    q = torch.softmax(diff.double() / T, 0)
    assert float(((count - q).abs() / (q * (1 - q) / n).sqrt()).max()) < 5.0        # five standard deviations
    i32 = lambda *s: torch.zeros(*s, dtype=I32, device="cuda")  # noqa: E731
    nc, com, nxt = i32(n), i32(n, 1), i32(n)
    ws = B.new_workspace(B.orthrus_consensus_sample_workspace_bytes(n, 1, vocab))
    B.orthrus_consensus_sample(lg_a, lg_d, draft.view(n, 1), u[1].view(n, 1).contiguous(), u[2].view(n, 1).contiguous(), T, nc, com, nxt, ws)
    count = torch.bincount(com.view(-1).long().cpu(), minlength=vocab).double() / n
    pa = torch.softmax(ar.double() / T, 0)
    assert float(((count - pa).abs() / (pa * (1 - pa) / n).sqrt()).max()) < 5.0
