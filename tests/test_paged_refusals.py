"""What the paged calls and the sampler refuse before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2605_12825_b200 import build
    build.build()
    from paper_2605_12825_b200 import binding
    return binding


def layer(lib, **kw):
    d = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, block=1, dtype=0, page_size=16, max_pages=64, n_pages=200, k_pages=0x1000,
             v_pages=0x2000, block_table=0x3000, cache_len=0x4000, n_new=None, max_len_hint=512, softmax_scale=0.0, flags=0)
    d.update(kw)
    return lib.PagedLayer(*[d[f[0]] for f in lib.PagedLayer._fields_])


BAD = [(dict(batch=0), 1), (dict(n_q_heads=7), 1), (dict(block=0), 1), (dict(max_pages=0), 1), (dict(n_pages=0), 1), (dict(max_len_hint=-1), 1),
       (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1), (dict(flags=4), 1), (dict(dtype=2), 2), (dict(head_dim=96), 2),
       (dict(page_size=24), 2), (dict(page_size=2048), 2), (dict(page_size=0), 2), (dict(max_pages=1 << 28), 2), (dict(n_pages=1 << 31), 2),
       (dict(k_pages=None), 1), (dict(v_pages=0x2008), 1)]


@pytest.mark.parametrize("bad,code", BAD + [(dict(block=65), 2), (dict(batch=16385), 2), (dict(block_table=None), 1), (dict(block_table=0x3002), 1),
                                            (dict(cache_len=None), 1), (dict(n_new=0x5001), 1)])
def test_attention(lib, bad, code):
    n0 = lib.orthrus_launch_count()
    L = layer(lib, **bad)
    for f in (lib.lib().orthrus_paged_ar_attend, lib.lib().orthrus_paged_diffusion_attend):
        assert f(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 1 << 30, None) == code
    assert lib.orthrus_launch_count() == n0


def test_positions_fit_31_bits_with_room(lib):
    """max_pages * page_size up to 2^31 - 2^16: what a kernel adds to a position to look ahead does not overflow."""
    size = lib.orthrus_paged_attend_workspace_bytes
    assert size(layer(lib, page_size=1024, max_pages=(1 << 21) - 64)) >= 256
    for width in ((1 << 21) - 63, 1 << 21, (1 << 31) - 1):
        L = layer(lib, page_size=1024, max_pages=width)
        assert size(L) == 0
        assert lib.lib().orthrus_paged_ar_attend(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 1 << 30, None) == 2
    # a grid of the plain-arithmetic kernel that cannot be launched
    L = layer(lib, dtype=1, batch=16384, n_kv_heads=1, n_q_heads=65535, block=64, k_pages=0x1000, v_pages=0x2000)
    assert lib.lib().orthrus_paged_ar_attend(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 1 << 40, None) == 2


def test_attention_arguments(lib):
    f, L = lib.lib().orthrus_paged_ar_attend, layer(lib)
    assert f(None, 0x10000, 0x20000, 0x30000, 1 << 30, None) == 1
    assert f(ctypes.byref(L), None, 0x20000, 0x30000, 1 << 30, None) == 1
    assert f(ctypes.byref(L), 0x10000, 0x20008, 0x30000, 1 << 30, None) == 1
    assert f(ctypes.byref(L), 0x10000, 0x20000, None, 1 << 30, None) == 1
    assert f(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 255, None) == 4
    size = lib.orthrus_paged_attend_workspace_bytes
    assert size(L) >= 256 and size(layer(lib, page_size=24)) == 0 and size(layer(lib, block=65)) == 0


@pytest.mark.parametrize("bad,code", BAD + [(dict(block=(1 << 20) + 1), 2)])
def test_writes(lib, bad, code):
    n0 = lib.orthrus_launch_count()
    L = layer(lib, **bad)
    assert lib.lib().orthrus_paged_kv_write(ctypes.byref(L), 0x10000, 0x20000, 0x30000, None, 0, None) == code
    assert lib.lib().orthrus_rope_paged_kv_write(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 0x40000, 1e4, 0x50000, None, 0, None) == code
    assert lib.orthrus_launch_count() == n0


def test_write_arguments(lib):
    L = layer(lib)
    w, r, c = lib.lib().orthrus_paged_kv_write, lib.lib().orthrus_rope_paged_kv_write, lib.lib().orthrus_paged_commit_len
    assert w(ctypes.byref(L), None, 0x20000, 0x30000, None, 0, None) == 1
    assert w(ctypes.byref(L), 0x10004, 0x20000, 0x30000, None, 0, None) == 1
    assert w(ctypes.byref(L), 0x10000, 0x20004, 0x30000, None, 0, None) == 1
    assert w(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 0x40000, 16, None) == 4
    assert r(ctypes.byref(L), 0x10000, None, 0x30000, 0x40000, 1e4, 0x50000, None, 0, None) == 1
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        assert r(ctypes.byref(L), 0x10000, 0x20000, 0x30000, 0x40000, theta, 0x50000, None, 0, None) == 1
    assert r(ctypes.byref(layer(lib, cache_len=None)), 0x10000, 0x20000, 0x30000, 0x40000, 1e4, 0x50000, None, 0, None) == 1
    assert c(ctypes.byref(L), None, None, 0, None) == 1 and c(ctypes.byref(layer(lib, cache_len=None)), 0x10000, None, 0, None) == 1


def test_page_tables(lib):
    f = lib.lib().orthrus_page_tables
    ok = [4, 16, 100, 8, 16] + [0x1000 * (k + 1) for k in range(10)] + [None, 0, None]
    n0 = lib.orthrus_launch_count()

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return f(*a)

    assert [call(_0=0), call(_2=0), call(_3=0), call(_4=0)] == [1] * 4
    assert [call(_0=8193), call(_1=24), call(_1=2048), call(_4=(1 << 24) + 1), call(_3=1 << 28)] == [2] * 5
    assert all(call(**{f"_{k}": None}) == 1 for k in range(5, 15))
    assert call(_5=0x1001) == 1 and call(_14=0xa004) == 1 and call(_15=0x20000, _16=16) == 4
    assert lib.orthrus_launch_count() == n0


def test_sampler(lib):
    f = lib.lib().orthrus_sample_tokens
    ok = [0x1000, 0, 4, 100, 100, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000, 0x7000, 0x8000, None]
    n0 = lib.orthrus_launch_count()

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return f(*a)

    assert [call(_2=0), call(_3=0), call(_4=99), call(_0=None), call(_5=None), call(_9=None), call(_10=None)] == [1] * 7
    assert [call(_0=0x1001), call(_0=0x1002, _1=1), call(_6=0x3002), call(_11=0x8001)] == [1] * 4
    assert [call(_1=2), call(_2=(1 << 20) + 1), call(_3=(1 << 24) + 1, _4=1 << 30)] == [2] * 3
    assert lib.orthrus_launch_count() == n0


@pytest.mark.parametrize("way", ["native", "ctypes"])
def test_bindings_refuse_tensors(lib, way):
    """Types, shapes, strides and devices, in the native marshalling and in the one over ctypes."""
    if way == "native":
        m = lib._native
    else:
        from paper_2605_12825_b200 import _marshal as m
        if lib._native is not m:
            m.bind(lib.lib(), lib._raise)
    L = layer(lib)
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    q = torch.zeros(2, 1, 8, 128, dtype=bf)
    kv = torch.zeros(2, 1, 2, 128, dtype=bf)
    slots = torch.zeros(2, 1, dtype=torch.int64)
    ws = torch.zeros(1024, dtype=torch.uint8)

    def refuses(kind, f, *args):
        with pytest.raises(kind):
            f(*args)

    refuses(ValueError, m.paged_ar_attend, L, q, q, ws, None)                        # not on a GPU
    refuses(TypeError, m.paged_ar_attend, L, q.float(), q, ws, None)
    refuses(ValueError, m.paged_ar_attend, L, q[:1], q, ws, None)
    refuses(ValueError, m.paged_diffusion_attend, L, q.transpose(0, 1), q, ws, None)
    refuses(TypeError, m.paged_ar_attend, L, None, q, ws, None)
    refuses(TypeError, m.paged_kv_write, L, slots.int(), kv, kv, None, None)
    refuses(ValueError, m.paged_kv_write, L, slots[:1], kv, kv, None, None)
    refuses(ValueError, m.paged_kv_write, L, slots, kv, kv, None, None)
    refuses(ValueError, m.rope_paged_kv_write, L, slots, q, kv, kv, 1e4, q, None, None)
    refuses(TypeError, m.paged_commit_len, L, slots[:, 0], None, None)
    n = torch.zeros(2, dtype=i32)
    one = torch.zeros(1, dtype=i32)
    table = torch.zeros(2, 8, dtype=i32)
    refuses(ValueError, m.page_tables, 16, n, n, n, n, table, n, one, one, n, slots, None, None)
    refuses(TypeError, m.page_tables, 16, n, n, n, n, table.long(), n, one, one, n, slots, None, None)
    x, r = torch.zeros(2, 50, dtype=bf), torch.zeros(2, dtype=f32)
    refuses(ValueError, m.sample_tokens, x, r, None, None, None, r, n, None, None)
    refuses(ValueError, m.sample_tokens, x[0], r, None, None, None, r, n, None, None)
    refuses(TypeError, m.sample_tokens, x.to(torch.float16), r, None, None, None, r, n, None, None)
    refuses(ValueError, lib.make_paged_layer, torch.zeros(4, 2, 16, 128, dtype=bf), torch.zeros(4, 2, 16, 128, dtype=bf), table, n, 8, 1)
    refuses(TypeError, lib.make_paged_layer, torch.zeros(4, 2, 16, 128, dtype=torch.float16), None, table, n, 8, 1)
