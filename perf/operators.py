"""Performance cases of the operators of a serving step on a paged cache, with their plain forms.

Four kinds of work, each through the functions of the package's binding where `own` is true:

  tables   pages for the rows that the requests of a batch add, and the slot of every such row
  write    rotary embedding of a block's queries and keys, keys and values into their pages
  attend   attention of one new token, or of a block, over the pages of its request
  sample   a token per row of logits: temperature, top-k, top-p, min-p, from given uniforms

Lengths of a batch are spread evenly over their range and dealt to the requests by the seed, so that every
seed is the same amount of work.  A plain form is elementary torch operations in 32 bits, or in 64 where
angles of far positions, long sums or a comparison at a border need them.
"""
import math

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
I32, I64, F64 = torch.int32, torch.int64, torch.float64
THETA = 10000.0


# ------------------------------------------------------------------------------------------ cases

def _attend(name, batch, heads, kv_heads, head_dim, block, page, len_min, len_max, view, idle=0):
    return dict(name=name, kind="attend", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, block=block,
                page=page, len_min=len_min, len_max=len_max, view=view, idle=idle)


def _write(name, batch, heads, kv_heads, head_dim, page, len_min, len_max, new_min, new_max):
    return dict(name=name, kind="write", batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                len_min=len_min, len_max=len_max, new_min=new_min, new_max=new_max)


def _tables(name, batch, page, len_min, len_max, new_min, new_max, done):
    return dict(name=name, kind="tables", batch=batch, page=page, len_min=len_min, len_max=len_max, new_min=new_min,
                new_max=new_max, done=done)


def _sample(name, rows, vocab, dtype, std, temperature, top_k, top_p, min_p):
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, std=std, temperature=temperature,
                top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # one conversation: a step of plain decoding, where latency counts
        _attend("decode_one", 1, 32, 8, 128, 1, 16, 4096, 4096, "ar"),
        # a serving batch with conversations of all lengths, some places of the batch idle
        _attend("decode_ragged", 32, 32, 8, 128, 1, 16, 1024, 8192, "ar", 2),
        # long documents, large pages: the bandwidth of the memory
        _attend("decode_long", 4, 64, 8, 128, 1, 64, 32768, 32768, "ar"),
        # the verification of a drafted block
        _attend("verify_block", 8, 16, 4, 128, 16, 32, 512, 4096, "ar"),
        # a drafted block of a small model: narrow heads, an odd group, short and odd lengths
        _attend("draft_d64", 5, 10, 2, 64, 8, 16, 1, 1601, "diffusion"),
        # the rows of one cycle of a serving batch go to their pages
        _write("write_block", 32, 32, 8, 128, 16, 100, 2000, 16, 16),
        # prompts of unequal length go to their pages
        _write("write_prompts", 6, 16, 4, 128, 32, 0, 0, 301, 4097),
        # one cycle of a serving batch: most requests grow by a block, some have ended
        _tables("tables_cycle", 256, 16, 17, 8000, 16, 16, 9),
        # prompts are admitted
        _tables("tables_prompts", 64, 64, 0, 0, 1, 8191, 0),
        # a token for one conversation
        _sample("sample_one", 1, 151936, "bf16", 2.0, 0.8, 50, 0.95, 0.0),
        # a drafted block for every conversation of a serving batch, with settings of their own
        _sample("sample_ragged", 512, 128256, "bf16", 1.0, 0.0, -1, -1.0, -1.0),
        # logits in 32 bits, an odd vocabulary
        _sample("sample_fp32", 24, 32003, "fp32", 1.5, 1.3, 0, 0.9, 0.02),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "write", "tables", "sample", "sample"))
    if kind == "attend":
        kv, group, d = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8, 16)), rng.choice((64, 128, 128))
        block = rng.choice((1, 1, 1, 2, 5, 8, 16))
        batch, top = _log(rng, 1, 40), _log(rng, 1, 16000)
        top = min(top, max(1, 16000 * 32 // (batch * kv)))
        return _strip(_attend("", batch, kv * group, kv, d, block, rng.choice((16, 32, 64, 128)), rng.randint(0, top), top,
                              rng.choice(("ar", "diffusion")), rng.choice((0, 0, 1)) if batch > 1 else 0))
    if kind == "write":
        kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 4, 5, 8))
        batch, new = _log(rng, 1, 48), _log(rng, 1, 4000)
        new = min(new, max(1, 16000 // batch))
        return _strip(_write("", batch, kv * group, kv, rng.choice((64, 128)), rng.choice((16, 32, 64)), 0,
                             _log(rng, 1, 2000), rng.randint(1, new), new))
    if kind == "tables":
        batch, new = _log(rng, 1, 600), _log(rng, 1, 8000)
        new = min(new, max(1, 500000 // batch))
        return _strip(_tables("", batch, rng.choice((16, 32, 64, 128)), 0, _log(rng, 1, 8000), rng.randint(0, new), new,
                              rng.randint(0, batch // 4)))
    return _strip(_sample("", _log(rng, 1, 300), _log(rng, 1000, 152000), rng.choice(("bf16", "bf16", "fp32")),
                          rng.choice((0.5, 1.0, 2.0, 4.0)), round(rng.uniform(0.3, 2.0), 2), rng.choice((0, 1, 40, 1000)),
                          rng.choice((0.5, 0.9, 0.99, 1.0)), rng.choice((0.0, 0.0, 0.05))))


def _strip(case):
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------ inputs

def _spread(lo, hi, n):
    """n whole numbers from lo to hi at even distances, the same for every seed."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _dealt(values, g, dtype=I32):
    v = torch.tensor(values, dtype=dtype, device=DEV)
    return v[torch.randperm(len(values), generator=g, device=DEV)]


def _rows_of(case):
    """New rows of the requests, in the order of the spread (not yet dealt)."""
    if case["kind"] == "attend":
        return [case["block"]] * (case["batch"] - case["idle"]) + [0] * case["idle"]
    return _spread(case["new_min"], case["new_max"], case["batch"])


def _cdiv(a, b):
    return -(-a // b)


def _paged(case, lens, new_max, g):
    """A pool with pages for `new_max` more rows of each request, dealt at random, and some that nobody holds."""
    batch, page = case["batch"], case["page"]
    width = _cdiv(max(_spread(case["len_min"], case["len_max"], batch)) + new_max, page)
    n_pages = batch * width + max(4, batch * width // 16)
    pages = torch.randperm(n_pages, generator=g, device=DEV)[: batch * width].to(I32).view(batch, width)
    shape = (n_pages, case["kv_heads"], page, case["head_dim"])
    k = torch.randn(shape, generator=g, device=DEV, dtype=BF16)
    v = torch.randn(shape, generator=g, device=DEV, dtype=BF16)
    return k, v, pages.contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"attend": _prepare_attend, "write": _prepare_write, "tables": _prepare_tables,
            "sample": _prepare_sample}[case["kind"]](case, g)


def _prepare_attend(case, g):
    batch, block = case["batch"], case["block"]
    lens = _dealt(_spread(case["len_min"], case["len_max"], batch), g)
    k, v, table = _paged(case, lens, block, g)
    q = torch.randn(batch, block, case["heads"], case["head_dim"], generator=g, device=DEV, dtype=BF16)
    return dict(case=case, k=k, v=v, table=table, len=lens, new=_dealt(_rows_of(case), g), q=q, out=torch.zeros_like(q))


def _prepare_write(case, g):
    batch, block, page = case["batch"], case["new_max"], case["page"]
    lens = _dealt(_spread(case["len_min"], case["len_max"], batch), g)
    new = _dealt(_rows_of(case), g)
    k, v, table = _paged(case, lens, block, g)
    i = torch.arange(block, device=DEV)
    pos = lens.long()[:, None] + i
    slot = torch.where(i < new[:, None], table.long().gather(1, pos // page) * page + pos % page, -1)

    def rand(heads):
        return torch.randn(batch, block, heads, case["head_dim"], generator=g, device=DEV, dtype=BF16)

    q = rand(case["heads"])
    return dict(case=case, k=k, v=v, table=table, len=lens, new=new, slot=slot, q=q, k_blk=rand(case["kv_heads"]),
                v_blk=rand(case["kv_heads"]), q_out=torch.zeros_like(q))


def _prepare_tables(case, g):
    batch, page = case["batch"], case["page"]
    lens = _spread(case["len_min"], case["len_max"], batch)
    width = _cdiv(max(lens) + case["new_max"], page)
    new = _dealt(_rows_of(case), g)
    lens = _dealt(lens, g)
    held = (lens + page - 1) // page
    ended = torch.randperm(batch, generator=g, device=DEV)[: case["done"]]
    lens[ended] = 0
    new[ended] = 0
    n_pages = batch * width
    pages = torch.randperm(n_pages, generator=g, device=DEV).to(I32)
    j = torch.arange(width, device=DEV)
    mine = j < held[:, None]
    table = torch.zeros(batch, width, dtype=I32, device=DEV)
    table[mine] = pages[: int(mine.sum())]
    free = torch.zeros(n_pages, dtype=I32, device=DEV)
    rest = pages[int(mine.sum()):]
    free[: rest.numel()] = rest
    return dict(case=case, len=lens, new=new, held=held.to(I32), held_out=torch.zeros(batch, dtype=I32, device=DEV), table=table,
                free=free, n_free=torch.tensor([rest.numel()], dtype=I32, device=DEV),
                n_free_out=torch.zeros(1, dtype=I32, device=DEV), granted=torch.zeros(batch, dtype=I32, device=DEV),
                slot=torch.zeros(batch, case["new_max"], dtype=I64, device=DEV))


def _prepare_sample(case, g):
    rows, vocab = case["rows"], case["vocab"]
    logits = torch.randn(rows, vocab, generator=g, device=DEV) * case["std"]
    if case["dtype"] == "bf16":
        logits = logits.to(BF16)

    def setting(value, off, low, high, dtype=torch.float32):
        # a negative value: settings of their own for the rows, every third one `off`
        x = torch.rand(rows, generator=g, device=DEV) * (high - low) + low
        if value >= 0:
            return torch.full((rows,), value, dtype=dtype, device=DEV)
        x[::3] = off
        return x.to(dtype)

    own_settings = case["top_k"] < 0
    t = setting(-1.0 if own_settings else case["temperature"], 1.0, 0.3, 1.5)
    return dict(case=case, logits=logits, temperature=t, top_k=setting(case["top_k"], 0, 1, 2000, I32).roll(1),
                top_p=setting(case["top_p"], 1.0, 0.5, 1.0), min_p=setting(case["min_p"], 0.0, 0.0, 0.2).roll(2),
                u=torch.rand(rows, generator=g, device=DEV), token=torch.zeros(rows, dtype=I32, device=DEV),
                logprob=torch.zeros(rows, device=DEV))


# ------------------------------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(kind, state)
    return {"attend": _plain_attend, "write": _plain_write, "tables": _plain_tables, "sample": _plain_sample}[kind](state)


def _plan(kind, s):
    """Descriptor and workspace, which a program makes once for a batch and keeps."""
    from paper_2605_12825_b200 import binding as B
    case = s["case"]
    if kind in ("attend", "write"):
        s["layer"] = B.make_paged_layer(s["k"], s["v"], s["table"], s["len"], case["heads"], s["q"].shape[1], s["new"],
                                        case["len_max"])
    if kind == "attend":
        s["ws"] = B.new_workspace(B.orthrus_paged_attend_workspace_bytes(s["layer"]))
    s["B"] = B
    return B


def _own(kind, s):
    B = s.get("B") or _plan(kind, s)
    if kind == "attend":
        call = B.orthrus_paged_ar_attend if s["case"]["view"] == "ar" else B.orthrus_paged_diffusion_attend
        call(s["layer"], s["q"], s["out"], s["ws"])
        return s["out"]
    if kind == "write":
        B.orthrus_rope_paged_kv_write(s["layer"], s["slot"], s["q"], s["k_blk"], s["v_blk"], THETA, s["q_out"])
        return s["q_out"], s["k"], s["v"]
    if kind == "tables":
        B.orthrus_page_tables(s["case"]["page"], s["len"], s["new"], s["held"], s["held_out"], s["table"], s["free"], s["n_free"],
                              s["n_free_out"], s["granted"], s["slot"])
        return s["held_out"], s["table"], s["free"], s["n_free_out"], s["granted"], s["slot"]
    B.orthrus_sample_tokens(s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["token"], s["logprob"])
    return s["token"], s["logprob"]


def _plain_attend(s):
    case = s["case"]
    batch, block, heads, kv, d, page = (case[n] for n in ("batch", "block", "heads", "kv_heads", "head_dim", "page"))
    pos = torch.arange(case["len_max"] + block, device=DEV)
    at = s["table"].long()[:, pos // page]
    k = s["k"][at, :, pos % page].transpose(1, 2).float()                      # [B][Hkv][L][d]
    v = s["v"][at, :, pos % page].transpose(1, 2).float()
    q = s["q"].float().view(batch, block, kv, heads // kv, d).permute(0, 2, 1, 3, 4).reshape(batch, kv, -1, d)
    i = torch.arange(block, device=DEV)
    real = i < s["new"][:, None]                                               # [B][K]
    sees = s["len"][:, None] + (i + 1 if case["view"] == "ar" else s["new"][:, None])
    sees = torch.where(real, sees, 1).expand(batch, block)
    score = (q @ k.transpose(2, 3) / math.sqrt(d)).view(batch, kv, block, -1, pos.numel())
    score = score.masked_fill(pos >= sees[:, None, :, None, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True))
    o = (e.view(batch, kv, -1, pos.numel()) @ v).view(batch, kv, block, -1, d) / e.sum(-1, keepdim=True)
    o = o.permute(0, 2, 1, 3, 4).reshape(batch, block, heads, d)
    s["out"].copy_(torch.where(real[:, :, None, None], o, s["out"].float()))
    return s["out"]


def _rotated(x, angle):
    """Rotation of the halves of x [B][K][H][d] by angle [B][K][d/2], in 64 bits."""
    lo, hi = x.to(F64).chunk(2, -1)
    cos, sin = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1)


def _plain_write(s):
    case = s["case"]
    page, d = case["page"], case["head_dim"]
    block = s["q"].shape[1]
    freq = THETA ** (torch.arange(d // 2, device=DEV, dtype=F64) * (-2.0 / d))
    angle = (s["len"][:, None] + torch.arange(block, device=DEV)).to(F64)[:, :, None] * freq
    real = s["slot"] >= 0
    slot = s["slot"][real]
    s["q_out"][real] = _rotated(s["q"], angle)[real].to(BF16)
    s["k"][slot // page, :, slot % page] = _rotated(s["k_blk"], angle)[real].to(BF16)
    s["v"][slot // page, :, slot % page] = s["v_blk"][real]
    return s["q_out"], s["k"], s["v"]


def _plain_tables(s):
    page = s["case"]["page"]
    lens, new, held = s["len"].long(), s["new"].long(), s["held"].long()
    table, free = s["table"], s["free"]
    j = torch.arange(table.shape[1], device=DEV)
    need = (lens + new + page - 1) // page
    gives, takes = (held - need).clamp(min=0), (need - held).clamp(min=0)
    # pages that are given back, in the order of requests and pages, behind the free ones
    back = (j >= need[:, None]) & (j < held[:, None])
    place = s["n_free"].long() + (gives.cumsum(0) - gives)[:, None] + j - need[:, None]
    free[place[back]] = table[back]
    total = s["n_free"].long() + gives.sum()
    upto = takes.cumsum(0)
    granted = (upto <= total) | (takes == 0)
    # pages that are taken, from the end of the list
    gets = (j >= held[:, None]) & (j < need[:, None]) & granted[:, None]
    place = total - 1 - ((upto - takes)[:, None] + j - held[:, None])
    table[gets] = free[place[gets]]
    s["n_free_out"].copy_(total - torch.where(granted, upto, 0).amax().clamp(max=total))
    s["held_out"].copy_(torch.where(granted, need, held))
    s["granted"].copy_(torch.where(granted, new, 0))
    i = torch.arange(s["slot"].shape[1], device=DEV)
    pos = lens[:, None] + i
    slot = table.long().gather(1, (pos // page).clamp(max=table.shape[1] - 1)) * page + pos % page
    s["slot"].copy_(torch.where(i < s["granted"][:, None], slot, -1))
    return s["held_out"], table, free, s["n_free_out"], s["granted"], s["slot"]


def _plain_sample(s):
    # order: value falling, id rising; everything at a border in 64 bits
    x, order = torch.sort(s["logits"], dim=1, descending=True, stable=True)
    x = x.to(F64)
    greedy = ~(s["temperature"] > 0)
    t = torch.where(greedy, 1.0, s["temperature"]).to(F64)[:, None]
    vocab = x.shape[1]
    k = torch.where(s["top_k"] > 0, s["top_k"], vocab).long()
    k = torch.where(greedy, 1, k)[:, None]
    rank = torch.arange(vocab, device=DEV)
    w = torch.exp((x - x[:, :1]) / t)
    cum = w.cumsum(1)
    before = torch.cat((torch.zeros_like(cum[:, :1]), cum[:, :-1]), 1)
    mass_k = cum.gather(1, k.clamp(max=vocab) - 1)
    p = s["top_p"].to(F64)[:, None]
    keep = (rank < k) & ((before < p * mass_k) | (p >= 1)) & (w >= s["min_p"].to(F64)[:, None])
    n = keep.sum(1, keepdim=True).clamp(min=1)
    mass = cum.gather(1, n - 1)
    at = torch.minimum((cum <= s["u"].to(F64)[:, None] * mass).sum(1, keepdim=True), n - 1)
    s["token"].copy_(order.gather(1, at)[:, 0])
    s["logprob"].copy_(torch.log(w.gather(1, at) / mass)[:, 0])
    return s["token"], s["logprob"]


# ------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "write": _exact_write, "sample": _exact_sample}.get(case["kind"], lambda s: None)(s)


def _exact_attend(s):
    """Request by request: softmax(q k^T / sqrt(d)) v over the keys that a row sees."""
    case = s["case"]
    group, page, scale = case["heads"] // case["kv_heads"], case["page"], case["head_dim"] ** -0.5
    out = s["out"].to(F64)
    lens, news, table = s["len"].tolist(), s["new"].tolist(), s["table"].tolist()
    for b, (n, new) in enumerate(zip(lens, news)):
        if new == 0:
            continue
        pages = table[b][: _cdiv(n + new, page)]
        k = torch.cat([s["k"][p] for p in pages], 1)[:, : n + new].to(F64)      # [Hkv][L][d]
        v = torch.cat([s["v"][p] for p in pages], 1)[:, : n + new].to(F64)
        for i in range(new):
            m = n + i + 1 if case["view"] == "ar" else n + new
            q = s["q"][b, i].to(F64).view(case["kv_heads"], group, -1)
            w = torch.softmax(torch.einsum("hgd,hld->hgl", q, k[:, :m]) * scale, -1)
            out[b, i] = torch.einsum("hgl,hld->hgd", w, v[:, :m]).reshape(case["heads"], -1)
    return out


def _exact_write(s):
    """Pair by pair as a product of complex numbers, request by request."""
    case = s["case"]
    half, page = case["head_dim"] // 2, case["page"]
    k, v, q_out = s["k"].to(F64), s["v"].to(F64), s["q_out"].to(F64)
    table = s["table"].long()
    for b, (n, new) in enumerate(zip(s["len"].tolist(), s["new"].tolist())):
        pos = torch.arange(n, n + new, device=DEV)
        turn = torch.polar(torch.ones(new, half, dtype=F64, device=DEV),
                           pos.to(F64)[:, None] / torch.pow(torch.tensor(THETA, dtype=F64, device=DEV),
                                                            torch.arange(half, dtype=F64, device=DEV) / half))[:, None]
        at, off = table[b, pos // page], pos % page
        for src, put in ((s["q"], lambda y: q_out[b].__setitem__(slice(0, new), y)),
                         (s["k_blk"], lambda y: k.__setitem__((at, slice(None), off), y))):
            x = src[b, :new].to(F64)
            z = torch.complex(x[..., :half], x[..., half:]) * turn
            put(torch.cat((z.real, z.imag), -1))
        v[at, :, off] = s["v_blk"][b, :new].to(F64)
    return q_out, k, v


def _exact_sample(s):
    """Row by row with the set that each filter leaves.  The tokens are whole numbers; the log of the drawn one's share."""
    case = s["case"]
    out = []
    cols = [s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "u")]
    for r in range(case["rows"]):
        t, k, p, m, u = (c[r] for c in cols)
        x = s["logits"][r].to(F64)
        if t <= 0:
            out.append(0.0)
            continue
        prob = torch.softmax(x / t, 0)
        prob, ids = torch.sort(prob, descending=True, stable=True)
        top = prob[0].clone()
        if 0 < k < prob.numel():
            prob = prob[:k]
        share = prob / prob.sum()
        if p < 1:
            share = share[: max(1, int((share.cumsum(0) - share < p).sum()))]
            prob = prob[: share.numel()]
        prob = prob[: max(1, int((prob / top >= m).sum()))]
        share = prob / prob.sum()
        at = min(int(torch.searchsorted(share.cumsum(0), torch.tensor(u, dtype=F64, device=DEV), right=True)), share.numel() - 1)
        out.append(float(torch.log(share[at])))
    return None, torch.tensor(out, dtype=F64, device=DEV)


# ------------------------------------------------------------------------------------------ work

def work(case):
    if case["kind"] == "attend":
        batch, block, d = case["batch"], case["block"], case["head_dim"]
        lens = _spread(case["len_min"], case["len_max"], batch)
        # which requests are idle is the seed's; the mean length stands for each
        active = batch - case["idle"]
        mean = sum(lens) / batch
        keys = active * (mean + block)
        seen = active * (block * mean + (block * (block + 1) / 2 if case["view"] == "ar" else block * block))
        rows = active * block * case["heads"] * d * 2
        return {"bytes": keys * case["kv_heads"] * d * 4 + 2 * rows + 4 * keys / case["page"] + 8 * batch,
                "flops": 4 * d * case["heads"] * seen}
    if case["kind"] == "write":
        rows = sum(_rows_of(case))
        d = case["head_dim"]
        return {"bytes": rows * (2 * 2 * d * (case["heads"] + 2 * case["kv_heads"]) + 8) + 4 * case["batch"],
                "flops": 3 * rows * d * (case["heads"] + case["kv_heads"])}
    if case["kind"] == "tables":
        page = case["page"]
        rows = sum(_rows_of(case))
        pages = 0 if not rows else rows / page + case["batch"] / 2
        return {"bytes": 20 * case["batch"] + 8 * case["batch"] * case["new_max"] + 8 * pages + 12, "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": case["rows"] * case["vocab"] * 4}
