"""How far a paged attention result may be off, from the definition in 64 bits.

out = sum_j w_j v_j, w the softmax.  The bf16 kernels sum fp32 exponentials, but round each to bf16 ahead of the product with the values:
a term is off by at most 2^-8 w_j |v_j| (half a step), to either side, and the output by half a step of its own.  What fp32 scores, exponentials and sums
add is below 2^-14 of the largest value.
  Element by element: the roundings are independent and bounded, so that their sum passes t sqrt(sum_j (2^-8 w_j v_j)^2) with a probability below 2 exp(-t^2 / 2)
(Hoeffding): t = 7, 5e-11 an element.
  All elements of a request together: a rounding error that is bounded by c has a mean square of at most c^2 / 3 (it is uniform between its bounds where the
bound is met, smaller elsewhere).  The sum of squares may be three times its mean (which not even one rounding that is always at its bound passes); asked
for from 64 elements on, where it finds an error that is the same for all of them and small for each.
fp32: sums of fp32 products, 2e-5 of the largest value.
"""
import math

import torch

BF16 = torch.bfloat16
F64 = torch.float64


def reference(q, k_pages, v_pages, table, lens, new, causal, skip=(), scale=None):
    """out and sum_j (w_j v_j)^2, both [B][K][Hq][d]; rows that do not exist NaN.  skip: positions that are left out (of a result that is wrong on purpose)."""
    B, K, Hq, d = q.shape
    Hkv, page = k_pages.shape[1], k_pages.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    G = Hq // Hkv
    out, spread = (torch.full(q.shape, math.nan, dtype=F64) for _ in range(2))
    for b in range(B):
        n = lens[b] + new[b]
        if new[b] == 0:
            continue
        pos = torch.arange(n)
        at = table[b][pos // page].long()
        k, v = (x[at, :, pos % page].to(F64).transpose(0, 1) for x in (k_pages, v_pages))       # [Hkv][n][d]
        rows = q[b, :new[b]].to(F64).view(new[b], Hkv, G, d)
        s = torch.einsum("ihgd,hnd->ihgn", rows, k) * scale
        if causal:
            s.masked_fill_((pos > lens[b] + torch.arange(new[b])[:, None])[:, None, None], -math.inf)
        for lo, hi in skip:
            s[..., max(lo, 0):hi] = -math.inf
        w = torch.softmax(s, -1)
        out[b, :new[b]] = torch.einsum("ihgn,hnd->ihgd", w, v).reshape(new[b], Hq, d)
        spread[b, :new[b]] = torch.einsum("ihgn,hnd->ihgd", w * w, v * v).reshape(new[b], Hq, d)
    return out, spread


def faults(got, want, spread, new, v_top, dtype):
    """What is wrong with a result: a list of sentences, empty if nothing is."""
    bad = []
    for b, n in enumerate(new):
        if n == 0:
            continue
        g, w, s = got[b, :n].to(F64), want[b, :n], spread[b, :n]
        off = (g - w).abs()
        if dtype != BF16:
            if not bool((off <= 2e-5 * v_top).all()):
                bad.append(f"request {b}: off by {float(off.max())}")
            continue
        half = 2.0 ** -8
        if not bool((off <= half * w.abs() * (1 + half) + 7 * half * s.sqrt() + 2.0 ** -14 * v_top).all()):
            bad.append(f"request {b}: an element off by {float((off / (half * (w.abs() + s.sqrt()))).max())} half steps")
        if w.numel() >= 64:
            mean = float((half ** 2 * (w * w + s) / 3).sum())
            if not float((off * off).sum()) <= 3 * mean + w.numel() * (2.0 ** -16 * v_top) ** 2:
                bad.append(f"request {b}: squares {float((off * off).sum()) / mean} times their mean")
    return bad


def plant(t, lens, new, causal, bonus=2.0):
    """Keys at places where one is easily lost (the first and the last, at the edges of tiles and pages, in the middle) become likelier for all query rows of
    their head: exp(bonus) times the others, so that a result without one is far off however many there are."""
    page, (B, K, Hq, d) = t["k"].shape[2], t["q"].shape
    Hkv = t["k"].shape[1]
    for b in range(B):
        n = lens[b] + new[b]
        if new[b] == 0:
            continue
        q = t["q"][b, :new[b]].float().view(new[b], Hkv, Hq // Hkv, d)
        each = q / q.norm(dim=-1, keepdim=True) ** 2 * bonus * math.sqrt(d)
        # (a key that every row scores by `bonus`: the smallest such, where rows are few; else along their sum)
        along = each.sum((0, 2))
        for p in {0, n - 1, n // 2, min(63, n - 1), min(64, n - 1), min(page, n - 1), max(n - 65, 0), lens[b] if lens[b] < n else 0}:
            pg = int(t["table"][b, p // page])
            t["k"][pg, :, p % page] = (t["k"][pg, :, p % page].float() + along).to(t["k"].dtype)
