"""The argument marshalling of csrc/native_binding.cpp through ctypes: the same functions with the same arguments,
for an interpreter or a torch that the native module was not compiled for.  A call costs the host about 8 us
here and a third of one there (plus the launch either way)."""
import ctypes

import torch

_lib = _raise = None


def bind(lib, raiser):
    """`lib`: liborthrus.so with its argument types declared; `raiser(code, name)` raises for an error code."""
    global _lib, _raise
    _lib, _raise = lib, raiser


def _ptr(t):
    return None if t is None else t.data_ptr()


def _count(t):
    return 0 if t is None else t.numel()


def _stream(stream):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _dims(t, n):
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch tensor")
    if t.dim() != n:
        raise ValueError(f"expected a tensor of {n} dimensions, got {t.dim()}")
    return t.shape


def _dtype(t):
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {t.dtype}")
    return 0 if t.dtype == torch.bfloat16 else 1


def _call(name, *args):
    code = getattr(_lib, name)(*args)
    if code != 0:
        _raise(code, name)


def _attend(name, layer, q, k, v, out, workspace, stream):
    _call(name, ctypes.byref(layer), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(workspace), _count(workspace), _stream(stream))


def diffusion_block_attend(*args):
    _attend("orthrus_diffusion_block_attend", *args)


def ar_verify_attend(*args):
    _attend("orthrus_ar_verify_attend", *args)


def multi_block_attend(layer, anchors, q, k, v, out, workspace, stream):
    n_blocks = _dims(anchors, 2)[1]
    _call("orthrus_multi_block_attend", ctypes.byref(layer), n_blocks, _ptr(anchors), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
          _ptr(workspace), _count(workspace), _stream(stream))


def consensus_accept(logits, draft, n_commit, committed, ar_argmax, next_anchor, workspace, stream):
    B, K, V = _dims(logits, 3)
    _call("orthrus_consensus_accept", _ptr(logits), _dtype(logits), _ptr(draft), B, K, V, _ptr(n_commit), _ptr(committed),
          _ptr(ar_argmax), _ptr(next_anchor), _ptr(workspace), _count(workspace), _stream(stream))


def consensus_accept_static(logits, draft, n_commit, committed, ar_argmax, next_anchor, stream):
    B, K, V = _dims(logits, 3)
    _call("orthrus_consensus_accept_static", _ptr(logits), _dtype(logits), _ptr(draft), B, K, V, _ptr(n_commit),
          _ptr(committed), _ptr(ar_argmax), _ptr(next_anchor), _stream(stream))


def consensus_sample(ar, diff, draft, u_accept, u_resample, temperature, n_commit, committed, next_anchor, workspace, stream):
    B, K, V = _dims(ar, 3)
    if _dims(diff, 3) != ar.shape or diff.dtype != ar.dtype:
        raise TypeError("the two logit tensors must agree in shape and dtype")
    if u_accept.dtype != torch.float32 or u_resample.dtype != torch.float32:
        raise TypeError("the uniforms must be float32")
    _call("orthrus_consensus_sample", _ptr(ar), _ptr(diff), _dtype(ar), _ptr(draft), _ptr(u_accept), _ptr(u_resample),
          float(temperature), B, K, V, _ptr(n_commit), _ptr(committed), _ptr(next_anchor), _ptr(workspace), _count(workspace),
          _stream(stream))


def lm_head_consensus(hidden, lm_head, draft, n_commit, committed, ar_argmax, next_anchor, workspace, stream):
    (B, K, H), V = _dims(hidden, 3), _dims(lm_head, 2)[0]
    _call("orthrus_lm_head_consensus", _ptr(hidden), _ptr(lm_head), _dtype(hidden), H, _ptr(draft), B, K, V, _ptr(n_commit),
          _ptr(committed), _ptr(ar_argmax), _ptr(next_anchor), _ptr(workspace), _count(workspace), _stream(stream))


def kv_append(layer, k, v, n_commit, update_len, workspace, stream):
    _call("orthrus_kv_append", ctypes.byref(layer), _ptr(k), _ptr(v), _ptr(n_commit), 1 if update_len else 0, _ptr(workspace),
          _count(workspace), _stream(stream))


def kv_append_layers(layers, ks, vs, n_commit, update_len, workspace, stream):
    layers, ks, vs = list(layers), list(ks), list(vs)
    n = len(layers)
    if len(ks) != n or len(vs) != n:
        raise ValueError("one layer, one K and one V tensor per layer")
    arr = (type(layers[0]) * n)(*layers) if n else None
    kp, vp = ((ctypes.c_void_p * n)(*[t.data_ptr() for t in x]) for x in (ks, vs))
    _call("orthrus_kv_append_layers", arr, n, kp, vp, _ptr(n_commit), 1 if update_len else 0, _ptr(workspace),
          _count(workspace), _stream(stream))


def block_kv_write(layer, k, v, workspace, stream):
    _call("orthrus_block_kv_write", ctypes.byref(layer), _ptr(k), _ptr(v), _ptr(workspace), _count(workspace), _stream(stream))


def commit_len(layer, n_commit, workspace, stream):
    _call("orthrus_commit_len", ctypes.byref(layer), _ptr(n_commit), _ptr(workspace), _count(workspace), _stream(stream))


def rope_block_kv_write(layer, q, k, v, rope_theta, q_out, workspace, stream):
    _call("orthrus_rope_block_kv_write", ctypes.byref(layer), _ptr(q), _ptr(k), _ptr(v), float(rope_theta), _ptr(q_out),
          _ptr(workspace), _count(workspace), _stream(stream))


def _paged(t, name, dtype, shape, optional=False):
    """A tensor of a paged call: type, shape (None: any size), contiguous, on the current device; its address."""
    if t is None:
        if optional:
            return None
        raise TypeError(f"{name}: expected a torch tensor")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: wrong dtype {t.dtype}")
    if t.dim() != len(shape) or any(w >= 0 and n != w for n, w in zip(t.shape, shape)):
        raise ValueError(f"{name}: wrong shape {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: not on the current device")
    return t.data_ptr()


def _space(t):
    if t is None:
        return None, 0
    return _paged(t, "workspace", torch.uint8, (-1,)), t.numel()


def _here(layer):
    """Of a layer made of tensors: they are on the current device."""
    if layer.device is not None and layer.device != torch.cuda.current_device():
        raise ValueError(f"layer: on cuda:{layer.device}, but the current device is cuda:{torch.cuda.current_device()}")


def _rows(layer):
    return torch.float32 if layer.dtype else torch.bfloat16


def page_tables(page_size, cache_len, n_new, held_in, held_out, block_table, free_list, n_free_in, n_free_out, granted, slot_map,
                workspace, stream):
    i32 = torch.int32
    table = _paged(block_table, "block_table", i32, (-1, -1))
    B, width = block_table.shape
    per = [_paged(t, n, i32, (B,)) for t, n in ((cache_len, "cache_len"), (n_new, "n_new"), (held_in, "held_in"),
                                                (held_out, "held_out"))]
    free = _paged(free_list, "free_list", i32, (-1,))
    ends = [_paged(n_free_in, "n_free_in", i32, (1,)), _paged(n_free_out, "n_free_out", i32, (1,))]
    got = _paged(granted, "granted", i32, (B,))
    slots = _paged(slot_map, "slot_map", torch.int64, (B, -1))
    _call("orthrus_page_tables", B, page_size, free_list.shape[0], width, slot_map.shape[1], *per, table, free, *ends, got, slots,
          *_space(workspace), _stream(stream))


def _blocks(layer, q, q_out, k, v, slot_map):
    _here(layer)
    L, dt = layer, _rows(layer)
    qs, ks = (L.batch, L.block, L.n_q_heads, L.head_dim), (L.batch, L.block, L.n_kv_heads, L.head_dim)
    _paged(slot_map, "slot_map", torch.int64, (L.batch, L.block))
    for t, n, s in ((q, "q", qs), (k, "k_blk", ks), (v, "v_blk", ks), (q_out, "q_out", qs)):
        if t is not False:
            _paged(t, n, dt, s)


def paged_kv_write(layer, slot_map, k, v, workspace, stream):
    _blocks(layer, False, False, k, v, slot_map)
    _call("orthrus_paged_kv_write", ctypes.byref(layer), _ptr(slot_map), _ptr(k), _ptr(v), *_space(workspace), _stream(stream))


def rope_paged_kv_write(layer, slot_map, q, k, v, rope_theta, q_out, workspace, stream):
    _blocks(layer, q, q_out, k, v, slot_map)
    _call("orthrus_rope_paged_kv_write", ctypes.byref(layer), _ptr(slot_map), _ptr(q), _ptr(k), _ptr(v), float(rope_theta),
          _ptr(q_out), *_space(workspace), _stream(stream))


def paged_commit_len(layer, n_commit, workspace, stream):
    _here(layer)
    _call("orthrus_paged_commit_len", ctypes.byref(layer), _paged(n_commit, "n_commit", torch.int32, (layer.batch,)),
          *_space(workspace), _stream(stream))


def _paged_attend(name, layer, q, out, workspace, stream):
    _here(layer)
    shape = (layer.batch, layer.block, layer.n_q_heads, layer.head_dim)
    qp, op = _paged(q, "q", _rows(layer), shape), _paged(out, "out", _rows(layer), shape)
    _call(name, ctypes.byref(layer), qp, op, *_space(workspace), _stream(stream))


def paged_ar_attend(*args):
    _paged_attend("orthrus_paged_ar_attend", *args)


def paged_diffusion_attend(*args):
    _paged_attend("orthrus_paged_diffusion_attend", *args)


def sample_tokens(logits, temperature, top_k, top_p, min_p, u, token, logprob, stream):
    R, V = _dims(logits, 2)
    dt = _dtype(logits)
    if not logits.is_cuda or logits.device.index != torch.cuda.current_device():
        raise ValueError("logits: expected a CUDA tensor on the current device")
    if (V > 1 and logits.stride(1) != 1) or (R > 1 and logits.stride(0) < V):
        raise ValueError("logits: expected rows of neighbouring elements that do not overlap")
    f32, i32 = torch.float32, torch.int32
    t, up = _paged(temperature, "temperature", f32, (R,)), _paged(u, "u", f32, (R,))
    k, p = _paged(top_k, "top_k", i32, (R,), True), _paged(top_p, "top_p", f32, (R,), True)
    m, tok, lp = (_paged(min_p, "min_p", f32, (R,), True), _paged(token, "token", i32, (R,)),
                  _paged(logprob, "logprob", f32, (R,), True))
    _call("orthrus_sample_tokens", logits.data_ptr(), dt, R, V, logits.stride(0) if R > 1 else V, t, k, p, m, up, tok, lp,
          _stream(stream))
