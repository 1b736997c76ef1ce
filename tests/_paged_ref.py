"""Plain 64-bit implementations of the paged-cache operators, on the CPU, request by request and row by row."""
import math

import torch

F64 = torch.float64


def page_tables(page, lens, new, held, table, free, n_free, n_pages, max_new):
    """Lists in, (held_out, table, free, n_free_out, granted, slots, trouble) out; `free` is the list's memory."""
    table, free = [r[:] for r in table], free[:]
    width = len(table[0])
    need = []
    trouble = set()
    for n, a, h in zip(lens, new, held):
        want = -(-(n + a) // page)
        ok = n >= 0 and 0 <= a <= max_new and 0 <= h <= width and want <= width
        if not ok:
            trouble.add("request")
        need.append(want if ok else None)
    for b, want in enumerate(need):
        for j in range(0 if want is None else want, held[b] if want is not None else 0):
            free[n_free] = table[b][j]
            n_free += 1
    held_out, granted, slots, asked, left = [], [], [], 0, n_free
    for b, want in enumerate(need):
        take = 0 if want is None else max(0, want - held[b])
        asked += take
        served = want is not None and (take == 0 or asked <= n_free)
        if want is not None and not served:
            trouble.add("pages")
        if served:
            for k in range(take):
                table[b][held[b] + k] = free[n_free - 1 - (asked - take) - k]
            left -= take
        held_out.append(want if served else held[b])
        granted.append(new[b] if served else 0)
        slots.append([table[b][(lens[b] + i) // page] * page + (lens[b] + i) % page if i < granted[b] else -1 for i in range(max_new)])
    return held_out, table, free, left, granted, slots, trouble


def rotated(x, pos, theta):
    """x [..., d] at position pos: pairs (c, c + d/2) as complex numbers."""
    half = x.shape[-1] // 2
    x = x.to(F64)
    angle = pos * theta ** (-torch.arange(half, dtype=F64) * 2 / (2 * half))
    z = torch.complex(x[..., :half], x[..., half:]) * torch.polar(torch.ones(half, dtype=F64), angle)
    return torch.cat((z.real, z.imag), -1)


def attend(q, k_pages, v_pages, table, lens, new, causal, scale=None):
    """[B][K][Hq][d] in 64 bits; rows that do not exist are NaN."""
    B, K, Hq, d = q.shape
    Hkv, page = k_pages.shape[1], k_pages.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    out = torch.full(q.shape, math.nan, dtype=F64)
    for b in range(B):
        n = lens[b] + new[b]
        if new[b] == 0:
            continue
        pos = torch.arange(n)
        at = table[b][pos // page].long()
        k = k_pages[at, :, pos % page].to(F64)               # [n][Hkv][d]
        v = v_pages[at, :, pos % page].to(F64)
        for i in range(new[b]):
            m = lens[b] + i + 1 if causal else n
            for h in range(Hq):
                g = h // (Hq // Hkv)
                w = torch.softmax(k[:m, g] @ q[b, i, h].to(F64) * scale, 0)
                out[b, i, h] = w @ v[:m, g]
    return out


def sample(x, t, top_k, top_p, min_p, u):
    """(token, log of its share, distance of the draw from the nearest border relative to the mass kept) for one row."""
    x = x.to(F64).clone()
    x[torch.isnan(x)] = -math.inf
    if bool((x == -math.inf).all()):
        return 0, math.nan, 1.0
    order = torch.sort(x, descending=True, stable=True).indices
    x = x[order]
    order = order[x > -math.inf]
    x = x[x > -math.inf]
    if not t > 0:
        return int(order[0]), 0.0, 1.0
    w = torch.where(x == x[0], torch.ones_like(x), torch.exp((x - x[0]) / t))
    margin = 1.0
    if 0 < top_k < len(w):
        w = w[:top_k]
    if top_p < 1:
        before = w.cumsum(0) - w
        want = max(top_p, 0.0) * float(w.sum())
        margin = min(margin, float((before[1:] - want).abs().min() / w.sum()) if len(w) > 1 else 1.0)
        w = w[:max(1, int((before < want).sum()))]
    if min_p > 0:
        keep = w >= min_p
        margin = min(margin, float((w / min_p - 1).abs().min()) if bool((w != 1).any()) else 1.0)
        w = w[:max(1, int(keep.sum()))]
    upto = w.cumsum(0)
    target = min(max(u, 0.0), 1 - 2.0 ** -24) * float(upto[-1])
    at = min(int((upto <= target).sum()), len(w) - 1)
    margin = min(margin, float((upto - target).abs().min() / upto[-1]))
    return int(order[at]), float(torch.log(w[at] / upto[-1])), margin
