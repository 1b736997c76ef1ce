"""Token sampling against the plain 64-bit implementation: equal tokens wherever no border is within rounding of the draw."""
import math

import pytest
import torch

import _paged_ref as ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
# Weights are rounded to 2^-(62 - log2 V) of the largest: at most V * 2^-(63 - log2 V) of the mass for V tokens, below 2^-27 for
# the largest vocabulary here; both sides' exponentials and sums are doubles.
CLOSE = 2.0 ** -26


def run(x, t, k=None, p=None, m=None, u=None):
    from paper_2605_12825_b200 import binding as B
    f = lambda v, dt=F32: None if v is None else torch.tensor(v, dtype=dt, device="cuda")  # noqa: E731
    R = x.shape[0]
    token, logprob = torch.full((R,), -7, dtype=torch.int32, device="cuda"), torch.full((R,), 5.0, device="cuda")
    B.orthrus_sample_tokens(x, f(t), f(k, torch.int32), f(p), f(m), f(u), token, logprob)
    return token.tolist(), logprob.tolist()


def compare(x, t, k, p, m, u, most_close=0.02):
    token, logprob = run(x.cuda() if not x.is_cuda else x, t, k, p, m, u)
    f32 = lambda v: torch.tensor(v, dtype=F32).tolist()  # noqa: E731
    t, p, m, u = f32(t), None if p is None else f32(p), None if m is None else f32(m), f32(u)
    close = 0
    for r in range(x.shape[0]):
        want, lp, margin = ref.sample(x[r].cpu(), t[r], k[r] if k else 0, p[r] if p else 1.0, m[r] if m else 0.0, u[r])
        if margin < CLOSE:
            close += 1
            continue
        assert token[r] == want, (r, token[r], want, margin)
        # log in double, rounded to float; half a step of it, and what the borders of the mass are known to
        assert (math.isnan(lp) and math.isnan(logprob[r])) or abs(logprob[r] - lp) <= 2.0 ** -23 * abs(lp) + CLOSE, r
    assert close <= max(1, most_close * x.shape[0])
    return token


def settings(R, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda: torch.rand(R, generator=g)  # noqa: E731
    t = (r() * 1.7 + 0.2).tolist()
    k = torch.randint(0, 300, (R,), generator=g)
    k[::3] = 0
    p, m = r() * 0.6 + 0.4, r() * 0.2
    p[1::3] = 1.0
    m[2::3] = 0.0
    return t, k.tolist(), p.tolist(), m.tolist(), r().tolist()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (5, 31), (4, 257), (7, 1000), (2, 4099), (9, 8191), (3, 32003), (1, 151936), (40, 5001),
                                 (160, 2048), (330, 700)])
@pytest.mark.parametrize("std", [0.3, 2.0, 9.0])
def test_against_the_plain_form(dtype, R, V, std):
    g = torch.Generator().manual_seed(R * V)
    x = (torch.randn(R, V, generator=g) * std).to(dtype)
    t, k, p, m, u = settings(R, V)
    compare(x, t, k, p, m, u)
    compare(x, t, None, None, None, u)
    compare(x, t, k, None, None, u)
    compare(x, t, None, p, None, u)
    compare(x, t, None, None, m, u)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [1e-8, 1e-6, 1e-3, 60.0, 1000.0, 1e30])
def test_scales_outside_the_usual(dtype, scale):
    """Tiny and huge logits: the bins of many values, refined."""
    g = torch.Generator().manual_seed(5)
    x = (torch.randn(6, 3000, generator=g) * scale).to(dtype)
    t = [max(scale, 1e-30) * 0.7] * 3 + [1.0] * 3
    u = torch.rand(6, generator=g).tolist()
    compare(x, t, [0, 5, 100, 0, 7, 2000], [0.9, 1.0, 0.5, 0.8, 1.0, 1.0], [0.0, 0.0, 0.01, 0.1, 0.3, 0.0], u)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mixed_scales_in_a_row(dtype):
    g = torch.Generator().manual_seed(6)
    x = torch.randn(8, 20000, generator=g) * 10.0 ** (torch.rand(8, 20000, generator=g) * 14 - 12)
    x[:, ::7] = 0.0
    x[:, 3::11] = -0.0
    compare(x.to(dtype), [0.5, 1.0, 2.0, 9.0] * 2, [0, 3, 15000, 0, 9000, 12000, 0, 0], [1.0, 1.0, 1.0, 0.7, 0.99, 1.0, 0.3, 0.97], [0.0] * 8,
            torch.rand(8, generator=g).tolist())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mixed_scales_where_a_row_has_one_cta(dtype):
    """As many rows as leave no SMs for clusters: bins of one value and of many, long stretches of ties."""
    g = torch.Generator().manual_seed(16)
    R, V = 100, 40000
    x = torch.randn(R, V, generator=g) * 10.0 ** (torch.rand(R, V, generator=g) * 14 - 12)
    x[:, ::7] = 0.0
    x[::2, 5::3] = 0.25
    t, k, p, m, u = settings(R, 17)
    compare(x.to(dtype), t, [n * 100 for n in k], p, None, u)
    compare(x.to(dtype), t, None, None, None, u)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [300, 9000])
def test_min_p_and_temperature_at_their_ends(dtype, V):
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(24, V, generator=g) * 3).to(dtype)
    x[20:, 5] = math.inf
    m = [1.0, 0.9999999, 0.5, 1e-3, 1e-30, 1e-38] * 4
    t = [1.0, 1e-6, 1e6, 0.3, 7.0, 1e-20] * 2 + [1e-38, 1.0, 50.0, 1e30, 0.1, 2.0] * 2
    u = torch.rand(24, generator=g).tolist()
    compare(x, t, None, None, m, u, most_close=0.3)
    token, _ = run(x.cuda(), t, None, None, m, u)
    assert token[20:] == [5] * 4


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ties_go_to_the_lowest_id(dtype):
    V = 1000
    flat = torch.full((7, V), 1.5).to(dtype)
    u = [0.0, 0.25, 0.5, 0.999, 1 - 2.0 ** -24, 0.125, 0.0009765625]
    token, lp = run(flat.cuda(), [1.0] * 7, None, None, None, u)
    assert token == [int(math.floor(v * V)) for v in torch.tensor(u).tolist()]
    assert all(abs(x + math.log(V)) < 1e-5 for x in lp)
    token, _ = run(flat.cuda(), [1.0] * 7, [10] * 7, None, None, u)
    assert token == [int(math.floor(v * 10)) for v in torch.tensor(u).tolist()]
    token, _ = run(flat.cuda(), [1.0] * 7, None, [0.25] * 7, None, u)
    assert token == [int(math.floor(v * 250)) for v in torch.tensor(u).tolist()]
    assert run(flat.cuda(), [0.0] * 7, None, None, None, u)[0] == [0] * 7
    two = flat.clone()
    two[:, 500:] = 2.0
    assert run(two.cuda(), [0.0] * 7, None, None, None, u)[0] == [500] * 7
    # zeros of both signs are one value
    z = torch.zeros(1, V).to(dtype)
    z[:, ::2] = -0.0
    assert run(z.cuda(), [1.0], None, None, None, [0.5])[0] == [500]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_numbers(dtype):
    x = torch.randn(8, 515, generator=torch.Generator().manual_seed(3)).to(dtype)
    x[0] = -math.inf
    x[1] = math.nan
    x[2, ::2] = math.nan
    x[3, ::2] = -math.inf
    x[4, 100] = math.inf
    x[5, [7, 300, 400]] = math.inf
    x[6, 1:] = -math.inf
    x[7, :] = -3.3e38
    u = [0.5, 0.5, 0.7, 0.7, 0.9, 0.9, 0.9, 0.5]
    token, lp = run(x.cuda(), [1.0] * 8, None, None, None, u)
    assert token[0] == 0 and math.isnan(lp[0]) and token[1] == 0 and math.isnan(lp[1])
    assert token[4] == 100 and token[5] == 400 and token[6] == 0
    assert lp[4] == 0.0 and abs(lp[5] + math.log(3)) < 1e-6
    assert token[7] == 257
    compare(x[2:4], [1.0] * 2, [0, 9], [0.9, 1.0], [0.0, 0.01], u[2:4])
    assert run(x[5:6].cuda(), [math.inf], None, None, None, [0.4])[0] == [300]


def test_settings_at_their_ends():
    g = torch.Generator().manual_seed(12)
    x = torch.randn(1, 3001, generator=g).to(BF16)
    best = int(x[0].float().argmax())
    R = 14
    xs = x.expand(R, -1).contiguous()
    nan, inf = math.nan, math.inf
    t = [0.0, -1.0, nan, 1.0, 1.0, 1.0, 1.0, 1.0, 1e-30, inf, 1.0, 1.0, 1.0, 1.0]
    k = [0, 0, 0, 1, 0, 0, 0, 0, 0, 0, -3, 3001, 5000, 2 ** 31 - 1]
    p = [1.0, 1.0, 1.0, 1.0, 0.0, -1.0, 1.0, 1.0, 1.0, 1.0, nan, 2.0, 1.0, 1.0]
    m = [0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1.0, 7.0, 0.0, 0.0, nan, -1.0, 0.0, 0.0]
    u = [0.99] * 8 + [0.99, 0.5, 0.3, 0.3, 0.3, 0.3]
    token, lp = run(xs.cuda(), t, k, p, m, u)
    ties = [int(i) for i in (x[0] == x[0, best]).nonzero()]
    assert [token[r] for r in (0, 1, 2, 3, 4, 5, 7)] == [ties[0]] * 7 and token[6] in ties and token[8] in ties
    order = torch.sort(x[0].float(), descending=True, stable=True).indices
    assert token[9] == int(order[1500]) and abs(lp[9] + math.log(3001)) < 1e-6
    assert token[10] == token[11] == token[12] == token[13] == ref.sample(x[0], 1.0, 0, 1.0, 0.0, float(torch.tensor(0.3)))[0]
    # uniforms outside [0, 1) are clamped
    token, _ = run(xs[:4].cuda(), [1.0] * 4, None, None, None, [-1.0, nan, 1.0, 9.0])
    assert token[0] == token[1] == ties[0] and token[2] == token[3] == ref.sample(x[0], 1.0, 0, 1.0, 0.0, 1.0)[0]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [0, 1, 3, 7])
def test_strided_and_unaligned_rows(dtype, shift):
    g = torch.Generator().manual_seed(shift)
    R, V = 5, 4097
    wide = torch.randn(R, V + 22 + shift, generator=g).to(dtype).cuda()
    x = wide[:, shift:shift + V]
    t, k, p, m, u = settings(R, 3)
    token = compare(x, t, k, p, m, u)
    assert token == run(x.contiguous(), t, k, p, m, u)[0]
    wide[:, :shift] = 100.0                       # neighbours do not count
    wide[:, shift + V:] = 100.0
    assert token == run(x, t, k, p, m, u)[0]


def test_frequencies():
    """20000 draws with uniforms at even distances: every token as often as its share, to one draw at each end of its stretch."""
    g = torch.Generator().manual_seed(1)
    R, V = 20000, 50
    row = (torch.randn(V, generator=g) * 1.5).to(BF16)
    u = ((torch.arange(R, dtype=torch.float64) + 0.5) / R).tolist()
    token, _ = run(row.expand(R, V).contiguous().cuda(), [0.8] * R, None, None, None, u)
    share = torch.softmax(row.double() / float(torch.tensor(0.8)), 0)
    n = torch.bincount(torch.tensor(token), minlength=V).double()
    assert bool(((n - share * R).abs() <= 2).all())


def test_many_rows_and_a_large_vocabulary():
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(70000, 40, generator=g, device="cuda").to(BF16)
    u = torch.rand(70000, generator=g, device="cuda")
    from paper_2605_12825_b200 import binding as B
    t = torch.ones(70000, device="cuda")
    token = torch.full((70000,), -1, dtype=torch.int32, device="cuda")
    B.orthrus_sample_tokens(x, t, None, None, None, u, token)
    assert bool(((token >= 0) & (token < 40)).all())
    for r in (0, 65534, 65535, 69999):
        assert int(token[r]) == ref.sample(x[r].cpu(), 1.0, 0, 1.0, 0.0, float(u[r]))[0]
    big = torch.randn(2, 1 << 21, generator=g, device="cuda").to(BF16)
    compare(big, [1.0, 0.7], [0, 1000], [0.9, 1.0], None, [0.3, 0.8], 1.0)


def test_captured_and_replayed_with_other_settings():
    from paper_2605_12825_b200 import binding as B
    g = torch.Generator().manual_seed(9)
    x = torch.randn(4, 3001, generator=g).to(BF16).cuda()
    t, k, p, m, u = settings(4, 1)
    f = lambda v, dt=F32: torch.tensor(v, dtype=dt, device="cuda")  # noqa: E731
    args = [f(t), f(k, torch.int32), f(p), f(m), f(u)]
    token, lp = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    B.orthrus_sample_tokens(x, *args, token, lp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.orthrus_sample_tokens(x, *args, token, lp)
    t, k, p, m, u = settings(4, 2)
    for a, v in zip(args, (t, k, p, m, u)):
        a.copy_(torch.tensor(v))
    graph.replay()
    assert token.tolist() == run(x, t, k, p, m, u)[0]
