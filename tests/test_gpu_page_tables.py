"""Block tables and slot maps against the plain implementation: whole numbers, equal everywhere."""
import random

import pytest
import torch

import _paged_ref as ref

pytestmark = pytest.mark.gpu
I32 = torch.int32


def run(page, lens, new, held, table, free, n_free, max_new, in_place=False, stream=None):
    from paper_2605_12825_b200 import binding as B
    dev = lambda v, t=I32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    n = len(lens)
    h, f = dev(held), dev([n_free])
    ho, fo = (h if in_place in (True, "held") else dev([-7] * n)), (f if in_place in (True, "free") else dev([-7]))
    tb, fl, gr = dev(table), dev(free), dev([-7] * n)
    slots = torch.full((n, max_new), -9, dtype=torch.int64, device="cuda")
    ws = B.new_workspace(256)
    B.orthrus_page_tables(page, dev(lens), dev(new), h, ho, tb, fl, f, fo, gr, slots, ws)
    status = B.orthrus_read_status(ws)
    return ho.tolist(), tb.tolist(), fl.tolist(), fo.tolist()[0], gr.tolist(), slots.tolist(), status


def state(rng, batch, page, len_max, new_max, spare, done=0, short=0):
    """Requests that hold what their lengths ask for, some with pages to spare, some that have ended."""
    lens = [rng.randint(0, len_max) for _ in range(batch)]
    new = [rng.randint(0, new_max) for _ in range(batch)]
    held = [-(-n // page) + rng.choice((0, 0, 1, 2)) for n in lens]
    for b in rng.sample(range(batch), done):
        lens[b] = new[b] = 0
    width = max(-(-(len_max + new_max) // page), max(held))
    n_pages = sum(held) + spare
    pages = list(range(n_pages))
    rng.shuffle(pages)
    table, at = [], 0
    for h in held:
        table.append(pages[at:at + h] + [-5] * (width - h))
        at += h
    free = pages[at:] + [-3] * at
    return lens, new, held, table, free, spare


def compare(page, s, max_new, **kw):
    lens, new, held, table, free, n_free = s
    want = ref.page_tables(page, lens, new, held, table, free, n_free, len(free), max_new)
    got = run(page, lens, new, held, table, free, n_free, max_new, **kw)
    from paper_2605_12825_b200 import binding as B
    assert got[:6] == tuple(want[:6])
    bits = (B.DEV_BAD_CACHE_LEN if "request" in want[6] else 0) | (B.DEV_NO_PAGES if "pages" in want[6] else 0)
    assert got[6] == bits
    return want


@pytest.mark.parametrize("batch,page,len_max,new_max,done", [
    (1, 16, 0, 1, 0), (1, 1, 3, 5, 0), (2, 1024, 5000, 2, 1), (7, 16, 100, 16, 2), (33, 32, 700, 33, 5), (256, 16, 300, 1, 9),
    (1023, 64, 90, 7, 40), (1025, 16, 40, 3, 100), (2500, 8, 20, 2, 300), (8192, 16, 20, 1, 1000), (12, 16, 10, 4099, 0),
    (64, 64, 0, 2500, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_against_the_plain_form(batch, page, len_max, new_max, done, in_place):
    rng = random.Random(batch * 7 + page)
    s = state(rng, batch, page, len_max, new_max, batch * (-(-new_max // page) + 1), done)
    compare(page, s, new_max, in_place=in_place)


@pytest.mark.parametrize("in_place", ["held", "free"])
@pytest.mark.parametrize("batch,page,len_max,new_max,done", [(40, 16, 3000, 700, 20), (600, 8, 300, 100, 300)])
def test_one_of_the_counts_in_place(batch, page, len_max, new_max, done, in_place):
    """Pages that one request gives back and another takes, with so many slots that several CTAs look them up."""
    rng = random.Random(batch)
    s = state(rng, batch, page, len_max, new_max, 3 + batch * (-(-new_max // page)) // 4, done)
    compare(page, s, new_max, in_place=in_place)
    compare(page, s, new_max)


@pytest.mark.parametrize("spare", [0, 1, 3, 10, 30])
def test_too_few_pages_serve_the_first_requests(spare):
    rng = random.Random(spare)
    s = state(rng, 40, 16, 50, 40, spare, 4)
    want = compare(16, s, 40)
    if spare < 10:
        assert "pages" in want[6]


def test_pages_given_back_in_the_same_call_are_handed_out():
    # no free page at all: request 0 ends, request 1 takes what it held, the last page first
    got = run(16, [0, 16], [0, 33], [3, 1], [[4, 2, 7, -5], [9, -5, -5, -5]], [-3] * 10, 0, 33)
    assert got[0] == [0, 4] and got[1][1] == [9, 7, 2, 4] and got[3] == 0 and got[4] == [0, 33]
    assert got[5][1][:17] == [7 * 16 + i for i in range(16)] + [2 * 16]


def test_requests_out_of_range_are_left_alone():
    page, width = 16, 4
    lens, new, held = [-1, 5, 5, 60, 64, 5, 5], [1, -1, 9, 8, 0, 8, 1], [1, 1, 1, 4, 4, 5, -1]
    table = [[10 * b + j for j in range(width)] for b in range(7)]
    free = list(range(100, 140))
    want = ref.page_tables(page, lens, new, held, table, free, 3, len(free), 8)
    got = run(page, lens, new, held, table, free, 3, 8)
    from paper_2605_12825_b200 import binding as B
    assert got[:6] == tuple(want[:6]) and got[6] == B.DEV_BAD_CACHE_LEN
    assert got[4] == [0, 0, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("n_free", [-1, 11, 9])
def test_a_list_of_free_pages_that_is_none_is_not_written_past_its_end(n_free):
    # 10 places; 9 free pages and two that are given back do not fit
    from paper_2605_12825_b200 import binding as B
    got = run(16, [0], [0], [2], [[50, 51]], list(range(10)), n_free, 1)
    assert got[6] & B.DEV_NO_PAGES and len(got[2]) == 10 and got[0] == [0]
    assert got[2][:9] == [50, 51, 2, 3, 4, 5, 6, 7, 8] if n_free == -1 else got[2][:9] == list(range(9))


def test_grow_shrink_and_grow_again_in_place_keeps_every_page_once():
    from paper_2605_12825_b200 import binding as B
    rng = random.Random(3)
    batch, page, width, n_pages = 20, 16, 12, 200
    dev = lambda v, t=I32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    held, n_free, granted = dev([0] * batch), dev([n_pages]), dev([0] * batch)
    table, free = torch.zeros(batch, width, dtype=I32, device="cuda"), torch.arange(n_pages, dtype=I32, device="cuda")
    slots = torch.zeros(batch, 64, dtype=torch.int64, device="cuda")
    lens = [0] * batch
    for step in range(30):
        new = [rng.randint(0, 30) for _ in range(batch)]
        for b in range(batch):
            if lens[b] + new[b] > width * page or rng.random() < 0.1:
                lens[b] = new[b] = 0
        B.orthrus_page_tables(page, dev(lens), dev(new), held, held, table, free, n_free, n_free, granted, slots)
        h, g, f = held.tolist(), granted.tolist(), int(n_free)
        mine = [p for b in range(batch) for p in table[b, :h[b]].tolist()]
        assert sorted(mine + free[:f].tolist()) == list(range(n_pages))
        used = [s for row in slots.tolist() for s in row if s >= 0]
        assert len(set(used)) == len(used) == sum(g)
        lens = [n + a for n, a in zip(lens, g)]


def test_captured_and_replayed():
    from paper_2605_12825_b200 import binding as B
    rng = random.Random(11)
    lens, new, held, table, free, n_free = state(rng, 50, 16, 200, 16, 200, 3)
    dev = lambda v, t=I32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    args = [dev(lens), dev(new), dev(held), dev(held), dev(table), dev(free), dev([n_free]), dev([0]), dev(held)]
    slots = torch.zeros(50, 16, dtype=torch.int64, device="cuda")
    B.orthrus_page_tables(16, *args, slots)
    torch.cuda.synchronize()
    first = [t.clone() for t in args[3:] + [slots]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.orthrus_page_tables(16, *args, slots)
    slots.fill_(-4)
    args[3].fill_(-4)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, args[3:] + [slots]))
