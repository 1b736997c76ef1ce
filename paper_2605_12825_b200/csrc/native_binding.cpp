// Argument marshalling of the hot calls in native code.  A decoding loop makes dozens of these calls
// per cycle, each a kernel of a few microseconds: through ctypes a call cost the host 8 us (3 us of
// them to ask torch for the current stream, the rest pointer conversions), more than most of the
// kernels take.  Here a call costs what its launch costs plus about a third of a microsecond.
//
// Every function takes the arguments of the Python function of the same name in binding.py (tensors
// or None, the layer descriptor, scalars, and last the stream or None for the current one), hands
// the pointers to the C entry point and calls the registered raiser when that reports an error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <vector>
#include "orthrus.h"

namespace {

PyObject *g_raise = nullptr;      // binding._raise(code, name)

struct Failed {};                 // a Python exception is set

const at::Tensor *as_tensor(PyObject *o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

void *ptr(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (const at::Tensor *t = as_tensor(o)) return t->data_ptr();
    PyObject *r = PyObject_CallMethod(o, "data_ptr", nullptr);
    if (!r) throw Failed();
    void *p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (!p && PyErr_Occurred()) throw Failed();
    return p;
}

size_t count(PyObject *o)         // elements; 0 for None
{
    if (o == Py_None) return 0;
    if (const at::Tensor *t = as_tensor(o)) return (size_t)t->numel();
    PyObject *r = PyObject_CallMethod(o, "numel", nullptr);
    if (!r) throw Failed();
    const size_t n = PyLong_AsSize_t(r);
    Py_DECREF(r);
    if (n == (size_t)-1 && PyErr_Occurred()) throw Failed();
    return n;
}

const at::Tensor &need_tensor(PyObject *o, int dims)
{
    const at::Tensor *t = as_tensor(o);
    if (!t) { PyErr_SetString(PyExc_TypeError, "expected a torch tensor"); throw Failed(); }
    if (t->dim() != dims) {
        PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions, got %d", dims, (int)t->dim());
        throw Failed();
    }
    return *t;
}

int32_t dtype_of(const at::Tensor &t)
{
    if (t.scalar_type() == at::kBFloat16) return ORTHRUS_BF16;
    if (t.scalar_type() == at::kFloat) return ORTHRUS_FP32;
    PyErr_Format(PyExc_TypeError, "unsupported dtype %s", c10::toString(t.scalar_type()));
    throw Failed();
}

void *stream_of(PyObject *o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject *r = PyObject_GetAttrString(o, "cuda_stream");
    if (!r) throw Failed();
    void *p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (!p && PyErr_Occurred()) throw Failed();
    return p;
}

// the orthrus_layer_t behind a ctypes structure (a copy: 88 bytes)
orthrus_layer_t layer_of(PyObject *o)
{
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
    if (view.len != (Py_ssize_t)sizeof(orthrus_layer_t)) {
        PyBuffer_Release(&view);
        PyErr_SetString(PyExc_TypeError, "expected a Layer");
        throw Failed();
    }
    const orthrus_layer_t L = *static_cast<const orthrus_layer_t *>(view.buf);
    PyBuffer_Release(&view);
    return L;
}

double real(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Failed();
    return x;
}

bool truth(PyObject *o)
{
    const int t = PyObject_IsTrue(o);
    if (t < 0) throw Failed();
    return t != 0;
}

// runs `call` without the interpreter lock; None, or the raiser's exception
template <class Call> PyObject *finish(const char *name, Call call)
{
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = (int)call();
    Py_END_ALLOW_THREADS
    if (code == ORTHRUS_OK) Py_RETURN_NONE;
    PyObject *r = PyObject_CallFunction(g_raise, "is", code, name);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
    return nullptr;
}

template <class Body> PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, const char *name, Body body)
{
    if (given != wanted) return PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, wanted, given);
    try {
        return body();
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

template <class Fn> PyObject *attend(PyObject *const *a, Py_ssize_t n, const char *name, Fn fn)
{   // layer, q, k_blk, v_blk, out, workspace, stream
    return guarded(n, 7, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        void *q = ptr(a[1]), *k = ptr(a[2]), *v = ptr(a[3]), *out = ptr(a[4]), *ws = ptr(a[5]), *st = stream_of(a[6]);
        const size_t wb = count(a[5]);
        return finish(name, [&] { return fn(&L, q, k, v, out, ws, wb, st); });
    });
}

PyObject *diffusion_block_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return attend(a, n, "orthrus_diffusion_block_attend", orthrus_diffusion_block_attend);
}
PyObject *ar_verify_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return attend(a, n, "orthrus_ar_verify_attend", orthrus_ar_verify_attend);
}

PyObject *multi_block_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, anchors, q, k_blk, v_blk, out, workspace, stream
    const char *name = "orthrus_multi_block_attend";
    return guarded(n, 8, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        const at::Tensor &an = need_tensor(a[1], 2);
        const int32_t nb = (int32_t)an.size(1);
        const int32_t *ap = static_cast<const int32_t *>(an.data_ptr());
        void *q = ptr(a[2]), *k = ptr(a[3]), *v = ptr(a[4]), *out = ptr(a[5]), *ws = ptr(a[6]), *st = stream_of(a[7]);
        const size_t wb = count(a[6]);
        return finish(name, [&] { return orthrus_multi_block_attend(&L, nb, ap, q, k, v, out, ws, wb, st); });
    });
}

int32_t *iptr(PyObject *o) { return static_cast<int32_t *>(ptr(o)); }

PyObject *consensus_accept(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // ar_logits, draft, n_commit, committed, ar_argmax, next_anchor, workspace, stream
    const char *name = "orthrus_consensus_accept";
    return guarded(n, 8, name, [&]() -> PyObject * {
        const at::Tensor &x = need_tensor(a[0], 3);
        const int32_t B = (int32_t)x.size(0), K = (int32_t)x.size(1), V = (int32_t)x.size(2), dt = dtype_of(x);
        void *lg = x.data_ptr(), *ws = ptr(a[6]), *st = stream_of(a[7]);
        int32_t *draft = iptr(a[1]), *nc = iptr(a[2]), *com = iptr(a[3]), *arg = iptr(a[4]), *nx = iptr(a[5]);
        const size_t wb = count(a[6]);
        return finish(name, [&] { return orthrus_consensus_accept(lg, dt, draft, B, K, V, nc, com, arg, nx, ws, wb, st); });
    });
}

PyObject *consensus_accept_static(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // ar_logits, draft, n_commit, committed, ar_argmax, next_anchor, stream
    const char *name = "orthrus_consensus_accept_static";
    return guarded(n, 7, name, [&]() -> PyObject * {
        const at::Tensor &x = need_tensor(a[0], 3);
        const int32_t B = (int32_t)x.size(0), K = (int32_t)x.size(1), V = (int32_t)x.size(2), dt = dtype_of(x);
        void *lg = x.data_ptr(), *st = stream_of(a[6]);
        int32_t *draft = iptr(a[1]), *nc = iptr(a[2]), *com = iptr(a[3]), *arg = iptr(a[4]), *nx = iptr(a[5]);
        return finish(name, [&] { return orthrus_consensus_accept_static(lg, dt, draft, B, K, V, nc, com, arg, nx, st); });
    });
}

PyObject *consensus_sample(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // ar_logits, diff_logits, draft, u_accept, u_resample, temperature, n_commit, committed, next_anchor, workspace, stream
    const char *name = "orthrus_consensus_sample";
    return guarded(n, 11, name, [&]() -> PyObject * {
        const at::Tensor &x = need_tensor(a[0], 3), &y = need_tensor(a[1], 3);
        if (x.sizes() != y.sizes() || x.scalar_type() != y.scalar_type()) {
            PyErr_SetString(PyExc_TypeError, "the two logit tensors must agree in shape and dtype");
            throw Failed();
        }
        const at::Tensor *u[2] = {as_tensor(a[3]), as_tensor(a[4])};
        if (!u[0] || !u[1] || u[0]->scalar_type() != at::kFloat || u[1]->scalar_type() != at::kFloat) {
            PyErr_SetString(PyExc_TypeError, "the uniforms must be float32");
            throw Failed();
        }
        const int32_t B = (int32_t)x.size(0), K = (int32_t)x.size(1), V = (int32_t)x.size(2), dt = dtype_of(x);
        void *la = x.data_ptr(), *ld = y.data_ptr(), *ws = ptr(a[9]), *st = stream_of(a[10]);
        const float *u1 = static_cast<const float *>(u[0]->data_ptr()), *u2 = static_cast<const float *>(u[1]->data_ptr());
        const float temp = (float)real(a[5]);
        int32_t *draft = iptr(a[2]), *nc = iptr(a[6]), *com = iptr(a[7]), *nx = iptr(a[8]);
        const size_t wb = count(a[9]);
        return finish(name, [&] {
            return orthrus_consensus_sample(la, ld, dt, draft, u1, u2, temp, B, K, V, nc, com, nx, ws, wb, st);
        });
    });
}

PyObject *lm_head_consensus(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // hidden, lm_head, draft, n_commit, committed, ar_argmax, next_anchor, workspace, stream
    const char *name = "orthrus_lm_head_consensus";
    return guarded(n, 9, name, [&]() -> PyObject * {
        const at::Tensor &x = need_tensor(a[0], 3), &w = need_tensor(a[1], 2);
        const int32_t B = (int32_t)x.size(0), K = (int32_t)x.size(1), H = (int32_t)x.size(2), V = (int32_t)w.size(0);
        const int32_t dt = dtype_of(x);
        void *hp = x.data_ptr(), *wp = w.data_ptr(), *ws = ptr(a[7]), *st = stream_of(a[8]);
        int32_t *draft = iptr(a[2]), *nc = iptr(a[3]), *com = iptr(a[4]), *arg = iptr(a[5]), *nx = iptr(a[6]);
        const size_t wb = count(a[7]);
        return finish(name, [&] {
            return orthrus_lm_head_consensus(hp, wp, dt, H, draft, B, K, V, nc, com, arg, nx, ws, wb, st);
        });
    });
}

PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, k_ar_blk, v_ar_blk, n_commit, update_len, workspace, stream
    const char *name = "orthrus_kv_append";
    return guarded(n, 7, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        void *k = ptr(a[1]), *v = ptr(a[2]), *ws = ptr(a[5]), *st = stream_of(a[6]);
        const int32_t *nc = iptr(a[3]);
        const int upd = truth(a[4]) ? 1 : 0;
        const size_t wb = count(a[5]);
        return finish(name, [&] { return orthrus_kv_append(&L, k, v, nc, upd, ws, wb, st); });
    });
}

PyObject *kv_append_layers(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layers, k_ar_blks, v_ar_blks, n_commit, update_len, workspace, stream
    const char *name = "orthrus_kv_append_layers";
    return guarded(n, 7, name, [&]() -> PyObject * {
        PyObject *seq[3] = {nullptr, nullptr, nullptr};
        struct Release { PyObject **s; ~Release() { for (int i = 0; i < 3; ++i) Py_XDECREF(s[i]); } } release{seq};
        for (int i = 0; i < 3; ++i) {
            seq[i] = PySequence_Fast(a[i], "expected a sequence");
            if (!seq[i]) throw Failed();
        }
        const Py_ssize_t m = PySequence_Fast_GET_SIZE(seq[0]);
        if (PySequence_Fast_GET_SIZE(seq[1]) != m || PySequence_Fast_GET_SIZE(seq[2]) != m) {
            PyErr_SetString(PyExc_ValueError, "one layer, one K and one V tensor per layer");
            throw Failed();
        }
        std::vector<orthrus_layer_t> L((size_t)m);
        std::vector<const void *> kp((size_t)m), vp((size_t)m);
        for (Py_ssize_t i = 0; i < m; ++i) {
            L[(size_t)i] = layer_of(PySequence_Fast_GET_ITEM(seq[0], i));
            kp[(size_t)i] = ptr(PySequence_Fast_GET_ITEM(seq[1], i));
            vp[(size_t)i] = ptr(PySequence_Fast_GET_ITEM(seq[2], i));
        }
        const int32_t *nc = iptr(a[3]);
        const int upd = truth(a[4]) ? 1 : 0;
        void *ws = ptr(a[5]), *st = stream_of(a[6]);
        const size_t wb = count(a[5]);
        return finish(name, [&] {
            return orthrus_kv_append_layers(L.data(), (int32_t)m, kp.data(), vp.data(), nc, upd, ws, wb, st);
        });
    });
}

PyObject *block_kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, k_blk, v_blk, workspace, stream
    const char *name = "orthrus_block_kv_write";
    return guarded(n, 5, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        void *k = ptr(a[1]), *v = ptr(a[2]), *ws = ptr(a[3]), *st = stream_of(a[4]);
        const size_t wb = count(a[3]);
        return finish(name, [&] { return orthrus_block_kv_write(&L, k, v, ws, wb, st); });
    });
}

PyObject *commit_len(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, n_commit, workspace, stream
    const char *name = "orthrus_commit_len";
    return guarded(n, 4, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        const int32_t *nc = iptr(a[1]);
        void *ws = ptr(a[2]), *st = stream_of(a[3]);
        const size_t wb = count(a[2]);
        return finish(name, [&] { return orthrus_commit_len(&L, nc, ws, wb, st); });
    });
}

PyObject *rope_block_kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, q, k_blk, v_blk, rope_theta, q_out, workspace, stream
    const char *name = "orthrus_rope_block_kv_write";
    return guarded(n, 8, name, [&]() -> PyObject * {
        const orthrus_layer_t L = layer_of(a[0]);
        void *q = ptr(a[1]), *k = ptr(a[2]), *v = ptr(a[3]), *qo = ptr(a[5]), *ws = ptr(a[6]), *st = stream_of(a[7]);
        const float theta = (float)real(a[4]);
        const size_t wb = count(a[6]);
        return finish(name, [&] { return orthrus_rope_block_kv_write(&L, q, k, v, theta, qo, ws, wb, st); });
    });
}

// ---- the paged calls check their tensors: type, shape (below 0: any size), contiguous, on the current device
void *paged(PyObject *o, const char *name, at::ScalarType type, std::initializer_list<int64_t> shape, bool optional = false)
{
    if (o == Py_None && optional) return nullptr;
    const at::Tensor *t = as_tensor(o);
    if (!t) { PyErr_Format(PyExc_TypeError, "%s: expected a torch tensor", name); throw Failed(); }
    if (t->scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s: wrong dtype %s", name, c10::toString(t->scalar_type()));
        throw Failed();
    }
    bool ok = t->dim() == (int64_t)shape.size();
    int64_t k = 0;
    for (int64_t w : shape) { ok = ok && (w < 0 || t->size(k) == w); ++k; }
    if (!ok) { PyErr_Format(PyExc_ValueError, "%s: wrong shape", name); throw Failed(); }
    if (!t->is_contiguous()) { PyErr_Format(PyExc_ValueError, "%s: expected a contiguous tensor", name); throw Failed(); }
    if (!t->is_cuda()) { PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor", name); throw Failed(); }
    if (t->get_device() != c10::cuda::current_device()) {
        PyErr_Format(PyExc_ValueError, "%s: not on the current device", name);
        throw Failed();
    }
    return t->data_ptr();
}
struct Space { void *p; size_t n; };
Space space_of(PyObject *o)
{
    return Space{paged(o, "workspace", at::kByte, {-1}, true), o == Py_None ? 0 : count(o)};
}
orthrus_paged_layer_t paged_layer_of(PyObject *o)
{
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
    if (view.len != (Py_ssize_t)sizeof(orthrus_paged_layer_t)) {
        PyBuffer_Release(&view);
        PyErr_SetString(PyExc_TypeError, "expected a PagedLayer");
        throw Failed();
    }
    const orthrus_paged_layer_t L = *static_cast<const orthrus_paged_layer_t *>(view.buf);
    PyBuffer_Release(&view);
    // where its tensors are; None if it was not made of tensors
    PyObject *device = PyObject_GetAttrString(o, "device");
    if (!device) throw Failed();
    const long at = device == Py_None ? -1 : PyLong_AsLong(device);
    const bool known = device != Py_None;
    Py_DECREF(device);
    if (at == -1 && PyErr_Occurred()) throw Failed();
    if (known && at != c10::cuda::current_device()) {
        PyErr_Format(PyExc_ValueError, "layer: on cuda:%ld, but the current device is cuda:%d", at, (int)c10::cuda::current_device());
        throw Failed();
    }
    return L;
}
at::ScalarType type_of(const orthrus_paged_layer_t &L) { return L.dtype == ORTHRUS_FP32 ? at::kFloat : at::kBFloat16; }
int32_t whole(PyObject *o)
{
    const long x = PyLong_AsLong(o);
    if (x == -1 && PyErr_Occurred()) throw Failed();
    if (x < INT32_MIN || x > INT32_MAX) { PyErr_SetString(PyExc_ValueError, "a number out of range"); throw Failed(); }
    return (int32_t)x;
}
int32_t extent(const at::Tensor &t, int64_t k)
{
    if (t.size(k) > INT32_MAX) { PyErr_SetString(PyExc_ValueError, "a tensor that is too large"); throw Failed(); }
    return (int32_t)t.size(k);
}

PyObject *page_tables(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // page_size, cache_len, n_new, held_in, held_out, block_table, free_list, n_free_in, n_free_out, granted, slot_map, workspace, stream
    const char *name = "orthrus_page_tables";
    return guarded(n, 13, name, [&]() -> PyObject * {
        const int32_t page = whole(a[0]);
        auto i32 = [&](int k, const char *what, std::initializer_list<int64_t> s) { return static_cast<int32_t *>(paged(a[k], what, at::kInt, s)); };
        int32_t *table = i32(5, "block_table", {-1, -1});
        const int32_t B = extent(*as_tensor(a[5]), 0), W = extent(*as_tensor(a[5]), 1);
        int32_t *len = i32(1, "cache_len", {B}), *add = i32(2, "n_new", {B}), *hi = i32(3, "held_in", {B}), *ho = i32(4, "held_out", {B});
        int32_t *fl = i32(6, "free_list", {-1}), *fi = i32(7, "n_free_in", {1}), *fo = i32(8, "n_free_out", {1}), *gr = i32(9, "granted", {B});
        int64_t *sm = static_cast<int64_t *>(paged(a[10], "slot_map", at::kLong, {B, -1}));
        const int32_t N = extent(*as_tensor(a[6]), 0), M = extent(*as_tensor(a[10]), 1);
        const Space ws = space_of(a[11]);
        void *st = stream_of(a[12]);
        return finish(name, [&] { return orthrus_page_tables(B, page, N, W, M, len, add, hi, ho, table, fl, fi, fo, gr, sm, ws.p, ws.n, st); });
    });
}

PyObject *paged_kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, slot_map, k_blk, v_blk, workspace, stream
    const char *name = "orthrus_paged_kv_write";
    return guarded(n, 6, name, [&]() -> PyObject * {
        const orthrus_paged_layer_t L = paged_layer_of(a[0]);
        const int64_t *sm = static_cast<int64_t *>(paged(a[1], "slot_map", at::kLong, {L.batch, L.block}));
        void *k = paged(a[2], "k_blk", type_of(L), {L.batch, L.block, L.n_kv_heads, L.head_dim});
        void *v = paged(a[3], "v_blk", type_of(L), {L.batch, L.block, L.n_kv_heads, L.head_dim});
        const Space ws = space_of(a[4]);
        void *st = stream_of(a[5]);
        return finish(name, [&] { return orthrus_paged_kv_write(&L, sm, k, v, ws.p, ws.n, st); });
    });
}

PyObject *rope_paged_kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, slot_map, q, k_blk, v_blk, rope_theta, q_out, workspace, stream
    const char *name = "orthrus_rope_paged_kv_write";
    return guarded(n, 9, name, [&]() -> PyObject * {
        const orthrus_paged_layer_t L = paged_layer_of(a[0]);
        const int64_t *sm = static_cast<int64_t *>(paged(a[1], "slot_map", at::kLong, {L.batch, L.block}));
        void *q = paged(a[2], "q", type_of(L), {L.batch, L.block, L.n_q_heads, L.head_dim});
        void *k = paged(a[3], "k_blk", type_of(L), {L.batch, L.block, L.n_kv_heads, L.head_dim});
        void *v = paged(a[4], "v_blk", type_of(L), {L.batch, L.block, L.n_kv_heads, L.head_dim});
        const float theta = (float)real(a[5]);
        void *qo = paged(a[6], "q_out", type_of(L), {L.batch, L.block, L.n_q_heads, L.head_dim});
        const Space ws = space_of(a[7]);
        void *st = stream_of(a[8]);
        return finish(name, [&] { return orthrus_rope_paged_kv_write(&L, sm, q, k, v, theta, qo, ws.p, ws.n, st); });
    });
}

PyObject *paged_commit_len(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // layer, n_commit, workspace, stream
    const char *name = "orthrus_paged_commit_len";
    return guarded(n, 4, name, [&]() -> PyObject * {
        const orthrus_paged_layer_t L = paged_layer_of(a[0]);
        const int32_t *nc = static_cast<int32_t *>(paged(a[1], "n_commit", at::kInt, {L.batch}));
        const Space ws = space_of(a[2]);
        void *st = stream_of(a[3]);
        return finish(name, [&] { return orthrus_paged_commit_len(&L, nc, ws.p, ws.n, st); });
    });
}

template <class Fn> PyObject *paged_attend(PyObject *const *a, Py_ssize_t n, const char *name, Fn fn)
{   // layer, q, out, workspace, stream
    return guarded(n, 5, name, [&]() -> PyObject * {
        const orthrus_paged_layer_t L = paged_layer_of(a[0]);
        void *q = paged(a[1], "q", type_of(L), {L.batch, L.block, L.n_q_heads, L.head_dim});
        void *out = paged(a[2], "out", type_of(L), {L.batch, L.block, L.n_q_heads, L.head_dim});
        const Space ws = space_of(a[3]);
        void *st = stream_of(a[4]);
        return finish(name, [&] { return fn(&L, q, out, ws.p, ws.n, st); });
    });
}
PyObject *paged_ar_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return paged_attend(a, n, "orthrus_paged_ar_attend", orthrus_paged_ar_attend);
}
PyObject *paged_diffusion_attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return paged_attend(a, n, "orthrus_paged_diffusion_attend", orthrus_paged_diffusion_attend);
}

PyObject *sample_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{   // logits, temperature, top_k, top_p, min_p, u, token, logprob, stream
    const char *name = "orthrus_sample_tokens";
    return guarded(n, 9, name, [&]() -> PyObject * {
        const at::Tensor &x = need_tensor(a[0], 2);
        const int32_t R = extent(x, 0), V = extent(x, 1), dt = dtype_of(x);
        if (!x.is_cuda() || x.get_device() != c10::cuda::current_device()) {
            PyErr_SetString(PyExc_ValueError, "logits: expected a CUDA tensor on the current device");
            throw Failed();
        }
        if ((V > 1 && x.stride(1) != 1) || (R > 1 && x.stride(0) < V)) {
            PyErr_SetString(PyExc_ValueError, "logits: expected rows of neighbouring elements that do not overlap");
            throw Failed();
        }
        auto f32 = [&](int k, const char *what, bool optional) { return static_cast<float *>(paged(a[k], what, at::kFloat, {R}, optional)); };
        const float *t = f32(1, "temperature", false), *p = f32(3, "top_p", true), *m = f32(4, "min_p", true), *u = f32(5, "u", false);
        const int32_t *k = static_cast<int32_t *>(paged(a[2], "top_k", at::kInt, {R}, true));
        int32_t *tok = static_cast<int32_t *>(paged(a[6], "token", at::kInt, {R}));
        float *lp = f32(7, "logprob", true);
        void *lg = x.data_ptr(), *st = stream_of(a[8]);
        const int64_t stride = R > 1 ? x.stride(0) : V;
        return finish(name, [&] { return orthrus_sample_tokens(lg, dt, R, V, stride, t, k, p, m, u, tok, lp, st); });
    });
}

PyObject *set_raiser(PyObject *, PyObject *f)
{
    Py_XINCREF(f);
    Py_XSETREF(g_raise, f);
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FAST(diffusion_block_attend), FAST(ar_verify_attend), FAST(multi_block_attend), FAST(consensus_accept),
    FAST(consensus_accept_static), FAST(consensus_sample), FAST(lm_head_consensus), FAST(kv_append),
    FAST(kv_append_layers), FAST(block_kv_write), FAST(commit_len), FAST(rope_block_kv_write),
    FAST(page_tables), FAST(paged_kv_write), FAST(rope_paged_kv_write), FAST(paged_commit_len), FAST(paged_ar_attend),
    FAST(paged_diffusion_attend), FAST(sample_tokens),
    {"set_raiser", set_raiser, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
