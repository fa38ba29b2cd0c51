// CPython extension of the binding: argument checks, output and workspace allocation, and the calls into
// libbra, natively.  A small layer on one image takes 12 us of GPU time; checked and marshalled in Python
// (ctypes), its call took 14 us of host time and set the pace.
//
// Functions here take every argument by position; the Python functions of the package give them their names and
// defaults.  No kernel lives here and nothing is computed.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include "../../include/bra.h"

namespace {

PyObject *g_bra_error = nullptr;      // class BraError(code, text), set by init()

struct Raised {};                     // a Python exception is set

[[noreturn]] void value_error(const char *text)
{
    PyErr_SetString(PyExc_ValueError, text);
    throw Raised{};
}

void check(int rc)
{
    if (rc == BRA_OK) return;
    PyObject *e = PyObject_CallFunction(g_bra_error, "is", rc, bra_strerror(rc));
    if (e) {
        PyErr_SetObject(g_bra_error, e);
        Py_DECREF(e);
    }
    throw Raised{};
}

const at::Tensor *tensor(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name);
        throw Raised{};
    }
    return &THPVariable_Unpack(o);
}

const at::Tensor &need(PyObject *o)
{
    const at::Tensor *t = tensor(o);
    if (!t) value_error("a required tensor is None");
    return *t;
}

// ints and what converts to one without loss (numpy integers, anything with __index__); no floats, no strings
long long_integer(PyObject *o)
{
    PyObject *i = PyNumber_Index(o);
    if (!i) throw Raised{};
    const long v = PyLong_AsLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

int integer(PyObject *o) { return (int)long_integer(o); }

// what float() takes
double real(PyObject *o)
{
    PyObject *f = PyNumber_Float(o);
    if (!f) throw Raised{};
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}

float scale_of(PyObject *o) { return o == Py_None ? 0.f : (float)real(o); }

int dtype_of(const at::Tensor &X)
{
    if (X.scalar_type() == at::kFloat) return BRA_F32;
    if (X.scalar_type() == at::kBFloat16) return BRA_BF16;
    PyErr_SetString(PyExc_TypeError, "tensors must be float32 or bfloat16");
    throw Raised{};
}

bool dims_are(const at::Tensor &t, std::initializer_list<int64_t> d) { return t.sizes().equals(at::IntArrayRef(d.begin(), d.size())); }

void same_kind(const at::Tensor &t, const at::Tensor &X)
{
    if (!(t.is_cuda() && t.is_contiguous() && t.scalar_type() == X.scalar_type() && t.device() == X.device()))
        value_error("tensors must be contiguous, on one GPU and of one dtype");
}

// The layer's inputs; fills the shape (scale and path apart).
bra_shape layer_shape(const at::Tensor &X, const at::Tensor &Wqkv, const at::Tensor *Wo, const at::Tensor *Wlce, int S,
                      int k, int heads, PyObject *scale, PyObject *path)
{
    const float scale_value = scale_of(scale);
    if (X.dim() != 4) value_error("X must be [B, H, W, C]");
    const int64_t C = X.size(3);
    same_kind(X, X);
    same_kind(Wqkv, X);
    if (Wo) same_kind(*Wo, X);
    if (Wlce) same_kind(*Wlce, X);
    if (!dims_are(Wqkv, {C, 3 * C})) value_error("Wqkv must be [C, 3C]");
    if (Wo && !dims_are(*Wo, {C, C})) value_error("Wo must be [C, C]");
    if (Wlce && !dims_are(*Wlce, {C, 5, 5})) value_error("Wlce must be [C, 5, 5]");
    for (int d = 0; d < 4; ++d)
        if (X.size(d) > INT32_MAX) value_error("X is too large");
    return bra_shape{(int32_t)X.size(0), (int32_t)X.size(1), (int32_t)X.size(2), (int32_t)C, heads, S, k, dtype_of(X),
                     scale_value, integer(path)};
}

void check_index(const at::Tensor *Ir, const bra_shape &s, const char *text)
{
    if (Ir && !(Ir->is_cuda() && Ir->is_contiguous() && Ir->scalar_type() == at::kInt &&
                dims_are(*Ir, {s.B, (int64_t)s.S * s.S, s.k})))
        value_error(text);
}

void *data(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
void *stream_of(const at::Tensor &X) { return (void *)c10::hip::getCurrentHIPStream(X.device().index()).stream(); }

at::Tensor scratch(size_t bytes, const at::Tensor &X)
{
    return at::empty({(int64_t)std::max(bytes, (size_t)256)}, X.options().dtype(at::kByte));
}

at::Tensor new_index(const bra_shape &s, const at::Tensor &X)
{
    return at::empty({s.B, (int64_t)s.S * s.S, s.k}, X.options().dtype(at::kInt));
}

PyObject *wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

PyObject *tuple(std::initializer_list<PyObject *> items)
{
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}

// Runs `call` without the interpreter lock and turns its code into an exception.
template <typename F>
void run(F call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = call();
    Py_END_ALLOW_THREADS;
    check(rc);
}

template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F body)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        return body();
    } catch (const Raised &) {
        return nullptr;
    } catch (const c10::OutOfMemoryError &e) {
        PyObject *m = PyImport_ImportModule("torch"), *cls = m ? PyObject_GetAttrString(m, "OutOfMemoryError") : nullptr;
        PyErr_SetString(cls ? cls : PyExc_RuntimeError, e.what_without_backtrace());
        Py_XDECREF(cls);
        Py_XDECREF(m);
        return nullptr;
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// init(BraError)
PyObject *py_init(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 1, [&]() -> PyObject * {
        Py_INCREF(a[0]);
        Py_XDECREF(g_bra_error);
        g_bra_error = a[0];
        Py_RETURN_NONE;
    });
}

// route(X, Wqkv, S, k, heads, want_Ar, path, ws)
PyObject *py_route(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &Wqkv = need(a[1]);
        const bra_shape s = layer_shape(X, Wqkv, nullptr, nullptr, integer(a[2]), integer(a[3]), integer(a[4]), Py_None, a[6]);
        at::Tensor own;
        const at::Tensor *ws = tensor(a[7]);
        if (!ws) {
            size_t bytes = 0;
            check(bra_workspace_bytes(&s, &bytes));
            own = scratch(bytes, X);
            ws = &own;
        }
        const bool want_ar = PyObject_IsTrue(a[5]);
        at::Tensor Ir = new_index(s, X), Ar;
        const int64_t R = (int64_t)s.S * s.S;
        if (want_ar) Ar = at::empty({s.B, R, R}, X.options().dtype(at::kFloat));
        void *st = stream_of(X);
        run([&] {
            return bra_route(&s, X.data_ptr(), Wqkv.data_ptr(), (int32_t *)Ir.data_ptr(),
                             want_ar ? (float *)Ar.data_ptr() : nullptr, ws->data_ptr(), (size_t)ws->numel(), st);
        });
        return want_ar ? tuple({wrap(Ir), wrap(Ar)}) : wrap(Ir);
    });
}

// forward(X, Wqkv, Wo, Wlce, S, k, heads, scale, Ir_in, want_Ir, path, ws, out)
PyObject *py_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &Wqkv = need(a[1]), &Wo = need(a[2]), &Wlce = need(a[3]);
        const bra_shape s = layer_shape(X, Wqkv, &Wo, &Wlce, integer(a[4]), integer(a[5]), integer(a[6]), a[7], a[10]);
        const at::Tensor *Ir_in = tensor(a[8]), *ws = tensor(a[11]), *out = tensor(a[12]);
        at::Tensor own, Y, Ir;
        if (!ws) {
            size_t bytes = 0;
            check(bra_workspace_bytes(&s, &bytes));
            own = scratch(bytes, X);
            ws = &own;
        }
        Y = out ? *out : at::empty_like(X);
        const bool want_ir = PyObject_IsTrue(a[9]);
        if (want_ir) Ir = new_index(s, X);
        check_index(Ir_in, s, "Ir_in must be a contiguous int32 [B, S*S, k] device tensor");
        void *st = stream_of(X);
        run([&] {
            return bra_forward(&s, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(), Wlce.data_ptr(), Y.data_ptr(),
                               want_ir ? (int32_t *)Ir.data_ptr() : nullptr, (const int32_t *)data(Ir_in), ws->data_ptr(),
                               (size_t)ws->numel(), st);
        });
        PyObject *y;
        if (out) Py_INCREF(y = a[12]);
        else y = wrap(Y);
        return want_ir ? tuple({y, wrap(Ir)}) : y;
    });
}

// forward_static(X, Wqkv, Wo, Wlce, S, k, heads, out, Ir_out, Ir_in, scale, path)
PyObject *py_forward_static(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &Wqkv = need(a[1]), &Wo = need(a[2]), &Wlce = need(a[3]), &out = need(a[7]);
        const bra_shape s = layer_shape(X, Wqkv, &Wo, &Wlce, integer(a[4]), integer(a[5]), integer(a[6]), a[10], a[11]);
        const at::Tensor *Ir_out = tensor(a[8]), *Ir_in = tensor(a[9]);
        if (!(out.is_cuda() && out.is_contiguous() && out.scalar_type() == X.scalar_type() && out.sizes().equals(X.sizes())))
            value_error("out must be a contiguous device tensor of X's shape and dtype");
        check_index(Ir_out, s, "Ir_out must be a contiguous int32 [B, S*S, k] device tensor");
        check_index(Ir_in, s, "Ir_in must be a contiguous int32 [B, S*S, k] device tensor");
        void *st = stream_of(X);
        run([&] {
            return bra_forward_static(&s, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(), Wlce.data_ptr(), out.data_ptr(),
                                      (int32_t *)data(Ir_out), (const int32_t *)data(Ir_in), st);
        });
        Py_INCREF(a[7]);
        return a[7];
    });
}

// forward_padded(X, Wqkv, Wo, Wlce, S, k, heads, scale, Ir_in, want_Ir, path)
PyObject *py_forward_padded(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &Wqkv = need(a[1]), &Wo = need(a[2]), &Wlce = need(a[3]);
        const bra_shape s = layer_shape(X, Wqkv, &Wo, &Wlce, integer(a[4]), integer(a[5]), integer(a[6]), a[7], a[10]);
        size_t bytes = 0;
        check(bra_padded_workspace_bytes(&s, &bytes));
        at::Tensor ws = scratch(bytes, X), Y = at::empty_like(X), Ir;
        const bool want_ir = PyObject_IsTrue(a[9]);
        if (want_ir) Ir = new_index(s, X);
        const at::Tensor *Ir_in = tensor(a[8]);
        check_index(Ir_in, s, "Ir_in must be a contiguous int32 [B, S*S, k] device tensor");
        void *st = stream_of(X);
        run([&] {
            return bra_forward_padded(&s, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(), Wlce.data_ptr(), Y.data_ptr(),
                                      want_ir ? (int32_t *)Ir.data_ptr() : nullptr, (const int32_t *)data(Ir_in),
                                      ws.data_ptr(), (size_t)ws.numel(), st);
        });
        return want_ir ? tuple({wrap(Y), wrap(Ir)}) : wrap(Y);
    });
}

// backward(X, Wqkv, Wo, Wlce, Ir, dY, S, heads, scale, path, ws)
PyObject *py_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &Wqkv = need(a[1]), &Wo = need(a[2]), &Wlce = need(a[3]), &Ir = need(a[4]),
                         &dY = need(a[5]);
        if (Ir.dim() < 1) value_error("Ir must be a contiguous int32 [B, S*S, k] device tensor");
        const bra_shape s = layer_shape(X, Wqkv, &Wo, &Wlce, integer(a[6]), (int)Ir.size(-1), integer(a[7]), a[8], a[9]);
        check_index(&Ir, s, "Ir must be a contiguous int32 [B, S*S, k] device tensor");
        if (!(dY.is_cuda() && dY.is_contiguous() && dY.scalar_type() == X.scalar_type() && dY.sizes().equals(X.sizes())))
            value_error("dY must match X");
        at::Tensor own;
        const at::Tensor *ws = tensor(a[10]);
        if (!ws) {
            size_t bytes = 0;
            check(bra_backward_workspace_bytes(&s, &bytes));
            own = scratch(bytes, X);
            ws = &own;
        }
        const auto f32 = X.options().dtype(at::kFloat);
        const int64_t C = s.C;
        at::Tensor dX = at::empty_like(X), dWqkv = at::empty({C, 3 * C}, f32), dWo = at::empty({C, C}, f32),
                   dWlce = at::empty({C, 5, 5}, f32);
        void *st = stream_of(X);
        run([&] {
            return bra_backward(&s, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(), Wlce.data_ptr(),
                                (const int32_t *)Ir.data_ptr(), dY.data_ptr(), dX.data_ptr(), (float *)dWqkv.data_ptr(),
                                (float *)dWo.data_ptr(), (float *)dWlce.data_ptr(), ws->data_ptr(), (size_t)ws->numel(), st);
        });
        return tuple({wrap(dX), wrap(dWqkv), wrap(dWo), wrap(dWlce)});
    });
}

// block_forward(X, parameters in the order of bra_block_params (a tuple of 13), S, k, heads, eps, scale, Ir_in, want_Ir,
//               path, ws, out)
PyObject *py_block_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]);
        if (X.dim() != 4) value_error("X must be [B, H, W, C]");
        if (!(X.is_cuda() && X.is_contiguous())) value_error("X must be a contiguous device tensor");
        if (!PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 13) value_error("expected 13 parameter tensors");
        const at::Tensor *p[13];
        for (int i = 0; i < 13; ++i) p[i] = &need(PyTuple_GET_ITEM(a[1], i));
        const int64_t C = X.size(3), hidden = p[9]->dim() == 2 ? p[9]->size(1) : 0;
        const struct { const char *name; bool matrix; int nd; int64_t dims[3]; } want[13] = {
            {"Wpos", true, 3, {C, 3, 3}}, {"bpos", false, 1, {C}}, {"ln1_g", false, 1, {C}}, {"ln1_b", false, 1, {C}},
            {"Wqkv", true, 2, {C, 3 * C}}, {"Wo", true, 2, {C, C}}, {"Wlce", true, 3, {C, 5, 5}}, {"ln2_g", false, 1, {C}},
            {"ln2_b", false, 1, {C}}, {"W1", true, 2, {C, hidden}}, {"b1", false, 1, {hidden}}, {"W2", true, 2, {hidden, C}},
            {"b2", false, 1, {C}}};
        for (int i = 0; i < 13; ++i) {
            const at::Tensor &t = *p[i];
            if (!(t.is_cuda() && t.is_contiguous() && t.device() == X.device() &&
                  t.scalar_type() == (want[i].matrix ? X.scalar_type() : at::kFloat) &&
                  t.sizes().equals(at::IntArrayRef(want[i].dims, (size_t)want[i].nd)))) {
                PyErr_Format(PyExc_ValueError, "%s must be a contiguous device tensor %s, of the shape that fits X and W1",
                             want[i].name, want[i].matrix ? "of X's dtype" : "of float32");
                throw Raised{};
            }
        }
        for (int d = 0; d < 4; ++d)
            if (X.size(d) > INT32_MAX) value_error("X is too large");
        const bra_shape s = {(int32_t)X.size(0), (int32_t)X.size(1), (int32_t)X.size(2), (int32_t)C, integer(a[4]), integer(a[2]),
                             integer(a[3]), dtype_of(X), scale_of(a[6]), integer(a[9])};
        const double eps = real(a[5]);
        at::Tensor own, Xout, Ir;
        const at::Tensor *Ir_in = tensor(a[7]), *ws = tensor(a[10]), *out = tensor(a[11]);
        if (!ws) {
            size_t bytes = 0;
            check(bra_block_workspace_bytes(&s, (int32_t)hidden, &bytes));
            own = scratch(bytes, X);
            ws = &own;
        }
        Xout = out ? *out : at::empty_like(X);
        const bool want_ir = PyObject_IsTrue(a[8]);
        if (want_ir) Ir = new_index(s, X);
        check_index(Ir_in, s, "Ir_in must be a contiguous int32 [B, S*S, k] device tensor");
        const bra_block_params bp = {p[0]->data_ptr(), (const float *)p[1]->data_ptr(), (const float *)p[2]->data_ptr(),
                                     (const float *)p[3]->data_ptr(), p[4]->data_ptr(), p[5]->data_ptr(), p[6]->data_ptr(),
                                     (const float *)p[7]->data_ptr(), (const float *)p[8]->data_ptr(), p[9]->data_ptr(),
                                     (const float *)p[10]->data_ptr(), p[11]->data_ptr(), (const float *)p[12]->data_ptr()};
        void *st = stream_of(X);
        run([&] {
            return bra_block_forward(&s, (int32_t)hidden, (float)eps, X.data_ptr(), &bp, Xout.data_ptr(),
                                     want_ir ? (int32_t *)Ir.data_ptr() : nullptr, (const int32_t *)data(Ir_in), ws->data_ptr(),
                                     (size_t)ws->numel(), st);
        });
        PyObject *y;
        if (out) Py_INCREF(y = a[11]);
        else y = wrap(Xout);
        return want_ir ? tuple({y, wrap(Ir)}) : y;
    });
}

// A matrix or vector of the operators below, if it is there: on X's GPU, dense, of the type and the shape.
void same_place(const at::Tensor *t, const at::Tensor &X, at::ScalarType type, std::initializer_list<int64_t> dims, const char *text)
{
    if (t && !(t->is_cuda() && t->is_contiguous() && t->device() == X.device() && t->scalar_type() == type && dims_are(*t, dims))) value_error(text);
}

bool like(const at::Tensor &t, const at::Tensor &X)
{
    return t.is_cuda() && t.is_contiguous() && t.device() == X.device() && t.scalar_type() == X.scalar_type() && t.sizes().equals(X.sizes());
}

// The caller's workspace, or one of `bytes` on X's GPU.
const at::Tensor *workspace(const at::Tensor *ws, size_t bytes, const at::Tensor &X, at::Tensor &own)
{
    if (!ws) {
        own = scratch(bytes, X);
        return &own;
    }
    if (!(ws->is_cuda() && ws->is_contiguous() && ws->device() == X.device() && ws->scalar_type() == at::kByte)) value_error("ws must be a contiguous uint8 tensor on X's GPU");
    return ws;
}

// The gated block's operands; X [.., C].
bra_ffn_shape ffn_shape(const at::Tensor &X, const at::Tensor &W1, const at::Tensor &W2, const at::Tensor *b1, const at::Tensor *b2, PyObject *act)
{
    if (X.dim() < 1) value_error("X must be [.., C]");
    same_kind(X, X);
    const int64_t C = X.size(-1), h = W2.dim() == 2 ? W2.size(0) : 0;
    same_kind(W1, X);
    same_kind(W2, X);
    if (!dims_are(W2, {h, C})) value_error("W2 must be [hidden, C]");
    if (!dims_are(W1, {C, 2 * h})) value_error("W1 must be [C, 2 hidden]");
    same_place(b1, X, at::kFloat, {2 * h}, "b1 must be a contiguous float32 [2 hidden] tensor on X's GPU");
    same_place(b2, X, at::kFloat, {C}, "b2 must be a contiguous float32 [C] tensor on X's GPU");
    if (C < 1 || h < 1 || C > INT32_MAX || h > INT32_MAX) check(BRA_ERR_SHAPE);
    return bra_ffn_shape{X.numel() / C, (int32_t)C, (int32_t)h, dtype_of(X), integer(act)};
}

// ffn_forward(X, W1, W2, b1, b2, act, want_pre, ws, out)
PyObject *py_ffn_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &W1 = need(a[1]), &W2 = need(a[2]);
        const at::Tensor *b1 = tensor(a[3]), *b2 = tensor(a[4]), *out = tensor(a[8]);
        const bra_ffn_shape s = ffn_shape(X, W1, W2, b1, b2, a[5]);
        if (out && !like(*out, X)) value_error("out must be a contiguous tensor of X's shape and dtype on X's GPU");
        const c10::DeviceGuard guard(X.device());
        size_t bytes = 0;
        check(bra_ffn_workspace_bytes(&s, &bytes));
        at::Tensor own, Y = out ? *out : at::empty_like(X), pre;
        const at::Tensor *ws = workspace(tensor(a[7]), bytes, X, own);
        const bool want_pre = PyObject_IsTrue(a[6]);
        if (want_pre) {
            auto sizes = X.sizes().vec();
            sizes.back() = 2 * (int64_t)s.hidden;
            pre = at::empty(sizes, X.options());
        }
        void *st = stream_of(X);
        run([&] {
            return bra_ffn_forward(&s, X.data_ptr(), W1.data_ptr(), (const float *)data(b1), W2.data_ptr(), (const float *)data(b2), Y.data_ptr(),
                                   want_pre ? pre.data_ptr() : nullptr, ws->data_ptr(), (size_t)ws->numel(), st);
        });
        PyObject *y;
        if (out) Py_INCREF(y = a[8]);
        else y = wrap(Y);
        return want_pre ? tuple({y, wrap(pre)}) : y;
    });
}

// ffn_backward(X, W1, W2, dY, b1, pre, act, bias_grads, grad_dtype or -1, ws)
PyObject *py_ffn_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]), &W1 = need(a[1]), &W2 = need(a[2]), &dY = need(a[3]);
        const at::Tensor *b1 = tensor(a[4]), *pre = tensor(a[5]);
        const bra_ffn_shape s = ffn_shape(X, W1, W2, b1, nullptr, a[6]);
        if (!like(dY, X)) value_error("dY must be a contiguous tensor of X's shape and dtype on X's GPU");
        if (pre && !(pre->is_cuda() && pre->is_contiguous() && pre->device() == X.device() && pre->scalar_type() == X.scalar_type() && pre->dim() >= 1 &&
                     pre->size(-1) == 2 * (int64_t)s.hidden && pre->numel() == 2 * s.hidden * s.M))
            value_error("pre must be what bra_ffn_forward returned: contiguous [.., 2 hidden] of X's dtype on X's GPU");
        const c10::DeviceGuard guard(X.device());
        size_t bytes = 0;
        check(bra_ffn_backward_workspace_bytes(&s, &bytes));
        const int asked = integer(a[8]), kind = asked < 0 ? s.dtype : asked;
        const auto options = X.options().dtype(kind == BRA_F32 ? at::kFloat : at::kBFloat16);
        const bool biases = PyObject_IsTrue(a[7]);
        at::Tensor own, dX = at::empty_like(X), dW1 = at::empty(W1.sizes(), options), dW2 = at::empty(W2.sizes(), options), db1, db2;
        if (biases) {
            db1 = at::empty({2 * (int64_t)s.hidden}, options);
            db2 = at::empty({(int64_t)s.C}, options);
        }
        const at::Tensor *ws = workspace(tensor(a[9]), bytes, X, own);
        void *st = stream_of(X);
        run([&] {
            return bra_ffn_backward(&s, X.data_ptr(), W1.data_ptr(), (const float *)data(b1), W2.data_ptr(), data(pre), dY.data_ptr(), dX.data_ptr(), dW1.data_ptr(),
                                    dW2.data_ptr(), biases ? db1.data_ptr() : nullptr, biases ? db2.data_ptr() : nullptr, kind, ws->data_ptr(), (size_t)ws->numel(), st);
        });
        if (biases) return tuple({wrap(dX), wrap(dW1), wrap(dW2), wrap(db1), wrap(db2)});
        return tuple({wrap(dX), wrap(dW1), wrap(dW2)});
    });
}

// The norms' inputs; X [.., C].
struct NormCall {
    bra_norm_shape s;
    bra_norm_params p;
};
NormCall norm_call(const at::Tensor &X, const at::Tensor *Y, const at::Tensor *gamma, const at::Tensor *beta, const at::Tensor *post_gamma, const at::Tensor *post_beta,
                   const at::Tensor *scale, const at::Tensor *gate, PyObject *kind, PyObject *eps)
{
    if (X.dim() < 1) value_error("the map must be [.., C]");
    same_kind(X, X);
    const int64_t C = X.size(-1);
    if (C < 1 || C > INT32_MAX) check(BRA_ERR_SHAPE);
    if (Y && !like(*Y, X)) value_error("Y must be a contiguous tensor of the map's shape and dtype on its GPU");
    for (const at::Tensor *t : {gamma, beta, post_gamma, post_beta, scale})
        same_place(t, X, at::kFloat, {C}, "gamma, beta, post_gamma, post_beta and scale must be contiguous float32 [C] tensors on the map's GPU");
    if (beta && !gamma) value_error("beta without gamma");
    if (post_beta && !post_gamma) value_error("post_beta without post_gamma");
    if (!Y && (post_gamma || scale || gate)) value_error("post_gamma, scale and gate go with Y");
    int64_t groups = 1;
    if (gate) {
        if (!(gate->is_cuda() && gate->is_contiguous() && gate->device() == X.device() && gate->scalar_type() == X.scalar_type() && gate->dim() >= 1 && gate->size(-1) == C))
            value_error("gate must be a contiguous [.., C] tensor of the map's dtype on its GPU");
        int64_t lead = gate->dim() - 1;
        while (lead > 0 && gate->size(lead - 1) == 1) --lead;       // (of the map's size or standing for it: the groups are the same)
        if (lead > X.dim() - 1) value_error("gate has more dimensions than the map");
        for (int64_t d = 0; d < lead; ++d) {
            if (gate->size(d) != X.size(d)) value_error("gate's leading dimensions must be the map's first ones");
            groups *= gate->size(d);
        }
    }
    const int64_t rows = X.numel() / C;
    if (groups < 1) groups = 1;                       // no rows
    if (groups > INT32_MAX) check(BRA_ERR_SHAPE);
    return NormCall{{rows, (int32_t)groups, (int32_t)C, dtype_of(X), integer(kind), (float)real(eps)},
                    {(const float *)data(gamma), (const float *)data(beta), (const float *)data(post_gamma), (const float *)data(post_beta), (const float *)data(scale), data(gate)}};
}

// norm_forward(X, Y, gamma, beta, post_gamma, post_beta, scale, gate, kind, eps, out)
PyObject *py_norm_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const at::Tensor &X = need(a[0]);
        const at::Tensor *Y = tensor(a[1]), *gamma = tensor(a[2]), *out = tensor(a[10]);
        const NormCall c = norm_call(X, Y, gamma, tensor(a[3]), tensor(a[4]), tensor(a[5]), tensor(a[6]), tensor(a[7]), a[8], a[9]);
        if (!Y && !gamma) value_error("nothing to do: neither Y nor gamma");
        if (out && !Y) value_error("out goes with Y");
        if (out && !like(*out, X)) value_error("out must be a contiguous tensor of the map's shape and dtype on its GPU");
        const c10::DeviceGuard guard(X.device());
        at::Tensor R, N;
        if (Y) R = out ? *out : at::empty_like(X);
        if (gamma) N = at::empty_like(X);
        void *st = stream_of(X);
        run([&] {
            return bra_norm_forward(&c.s, X.data_ptr(), data(Y), &c.p, Y ? R.data_ptr() : nullptr, gamma ? N.data_ptr() : nullptr, st);
        });
        if (!Y) return wrap(N);
        PyObject *r;
        if (out) Py_INCREF(r = a[10]);
        else r = wrap(R);
        return gamma ? tuple({r, wrap(N)}) : r;
    });
}

// norm_backward(R, Y, gamma, post_gamma, post_beta, scale, gate, dN, dX, kind, eps, ws)
PyObject *py_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&]() -> PyObject * {
        const at::Tensor &R = need(a[0]);
        const at::Tensor *Y = tensor(a[1]), *gamma = tensor(a[2]), *post_gamma = tensor(a[3]), *post_beta = tensor(a[4]), *scale = tensor(a[5]), *gate = tensor(a[6]),
                         *dN = tensor(a[7]), *dR = tensor(a[8]);
        const NormCall c = norm_call(R, Y, gamma, nullptr, post_gamma, post_beta, scale, gate, a[9], a[10]);
        if (!dN && !dR) value_error("neither dN nor dX");
        if (dN && !gamma) value_error("dN without gamma");
        if ((dN && !like(*dN, R)) || (dR && !like(*dR, R))) value_error("dN and dX must be contiguous tensors of the map's shape and dtype on its GPU");
        const c10::DeviceGuard guard(R.device());
        size_t bytes = 0;
        check(bra_norm_backward_workspace_bytes(&c.s, post_gamma != nullptr, &bytes));
        PyObject *d = PyDict_New();
        if (!d) throw Raised{};
        struct Drop { PyObject *&o; ~Drop() { Py_XDECREF(o); } } drop{d};
        auto keep = [&](const char *name, at::Tensor t) {
            PyObject *o = wrap(t);
            const int rc = o ? PyDict_SetItemString(d, name, o) : -1;
            Py_XDECREF(o);
            if (rc) throw Raised{};
            return t.data_ptr();
        };
        // each vector has memory and a version of its own
        const auto options = R.options().dtype(at::kFloat);
        auto vector = [&](const char *name) { return (float *)keep(name, at::empty({(int64_t)c.s.C}, options)); };
        bra_norm_grads g{};
        g.dX = keep("dX", at::empty_like(R));
        if (dN) { g.dgamma = vector("dgamma"); g.dbeta = vector("dbeta"); }
        if (Y) {
            g.dY = keep("dY", at::empty_like(R));
            if (scale) g.dscale = vector("dscale");
            if (gate) g.dgate = keep("dgate", at::empty_like(*gate));
            if (post_gamma) { g.dpost_gamma = vector("dpost_gamma"); g.dpost_beta = vector("dpost_beta"); }
        }
        at::Tensor own;
        const at::Tensor *ws = workspace(tensor(a[11]), bytes, R, own);
        void *st = stream_of(R);
        run([&] {
            return bra_norm_backward(&c.s, R.data_ptr(), data(Y), &c.p, data(dN), data(dR), &g, ws->data_ptr(), (size_t)ws->numel(), st);
        });
        PyObject *out = d;
        d = nullptr;
        return out;
    });
}

// A list or tuple's items, held for the call.
struct Items {
    PyObject *fast;
    Py_ssize_t n;
    Items(PyObject *o, const char *text) : fast(PySequence_Fast(o, text)), n(0)
    {
        if (!fast) throw Raised{};
        n = PySequence_Fast_GET_SIZE(fast);
    }
    ~Items() { Py_XDECREF(fast); }
    Items(const Items &) = delete;
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

const at::Tensor &entry(PyObject *state, const char *key)
{
    PyObject *o = PyDict_GetItemString(state, key);
    if (!o) {
        PyErr_Format(PyExc_ValueError, "the state has no %s", key);
        throw Raised{};
    }
    return need(o);
}

// adamw_step(params, grads, state, step, lr, beta1, beta2, eps, weight_decay, copies, grad_scale)
PyObject *py_adamw_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const Items params(a[0], "params must be a list of tensors"), grads(a[1], "grads must be a list of tensors");
        if (params.n != grads.n) value_error("params and grads must be of one length");
        if (!PyDict_Check(a[2])) value_error("state must be a dict as adamw_state returns it");
        if (!params.n) Py_RETURN_NONE;
        const at::Tensor &first = need(params[0]);
        if (!first.is_cuda()) value_error("params must be contiguous float32 or bfloat16 tensors on one GPU");
        std::vector<bra_adamw_tensor> list((size_t)params.n);
        PyObject *copies_of = a[9] == Py_None ? a[0] : a[9];
        const Items copies(copies_of, "copies must be a list of tensors");
        const bool with_copies = a[9] != Py_None;
        if (with_copies && copies.n != params.n) value_error("copies must have an entry for each parameter");
        double decay = 0;
        const bool one_decay = PyFloat_Check(a[8]) || PyIndex_Check(a[8]);
        if (one_decay) decay = real(a[8]);
        const Items decays(one_decay ? a[0] : a[8], "weight_decay must be a number or one for each parameter");
        if (decays.n != params.n) value_error("weight_decay must be a number or one for each parameter");
        int64_t blocks = 0;
        for (Py_ssize_t i = 0; i < params.n; ++i) {
            const at::Tensor &p = need(params[i]);
            const at::Tensor *g = tensor(grads[i]), *c = with_copies ? tensor(copies[i]) : nullptr;
            if (!(p.is_cuda() && p.is_contiguous() && p.device() == first.device() && (p.scalar_type() == at::kFloat || p.scalar_type() == at::kBFloat16)))
                value_error("params must be contiguous float32 or bfloat16 tensors on one GPU");
            if (g && !(g->is_cuda() && g->is_contiguous() && g->device() == first.device() && g->sizes().equals(p.sizes()) &&
                       (g->scalar_type() == at::kFloat || g->scalar_type() == at::kBFloat16)))
                value_error("grads must be contiguous float32 or bfloat16 tensors of the parameters' shapes on their GPU");
            if (c && !(p.scalar_type() == at::kFloat && c->is_cuda() && c->is_contiguous() && c->device() == first.device() && c->sizes().equals(p.sizes()) &&
                       c->scalar_type() == at::kBFloat16))
                value_error("copies must be contiguous bfloat16 tensors of float32 parameters' shapes on their GPU");
            list[(size_t)i] = bra_adamw_tensor{p.data_ptr(), g && p.numel() ? g->data_ptr() : nullptr, data(c), p.numel(), (float)(one_decay ? decay : real(decays[i])),
                                               p.scalar_type() == at::kFloat ? BRA_F32 : BRA_BF16, g && g->scalar_type() == at::kFloat ? BRA_F32 : BRA_BF16};
            blocks += (p.numel() + BRA_ADAMW_BLOCK - 1) / BRA_ADAMW_BLOCK;
        }
        bra_adamw_args args{};
        args.lr = real(a[4]); args.beta1 = real(a[5]); args.beta2 = real(a[6]); args.eps = real(a[7]);
        args.bits = PyDict_GetItemString(a[2], "exp_avg_sq") ? 32 : 8;
        auto state = [&](const char *key, at::ScalarType type, int64_t size) {
            const at::Tensor &t = entry(a[2], key);
            if (!(t.is_cuda() && t.is_contiguous() && t.device() == first.device() && t.scalar_type() == type && t.numel() == size))
                value_error("the state is not that of these parameters");
            return t.data_ptr();
        };
        const int64_t values = blocks * BRA_ADAMW_BLOCK;
        if (args.bits == 32) {
            args.exp_avg = state("exp_avg", at::kFloat, values);
            args.exp_avg_sq = state("exp_avg_sq", at::kFloat, values);
        } else {
            args.exp_avg = state("exp_avg", at::kFloat8_e4m3fn, values);
            args.exp_avg_sq = state("exp_avg_root", at::kFloat8_e4m3fn, values);
            args.exp_avg_scale = state("exp_avg_scale", at::kFloat8_e8m0fnu, blocks);
            args.exp_avg_sq_scale = state("exp_avg_root_scale", at::kFloat8_e8m0fnu, blocks);
        }
        const at::Tensor *scale = tensor(a[10]);
        if (scale && !(scale->is_cuda() && scale->device() == first.device() && scale->scalar_type() == at::kFloat && scale->numel() == 1))
            value_error("grad_scale must be a one-element float32 tensor on the parameters' GPU");
        args.grad_scale = (const float *)data(scale);
        const c10::DeviceGuard guard(first.device());
        at::Tensor scalars;
        if (THPVariable_Check(a[3])) {
            const at::Tensor &t = THPVariable_Unpack(a[3]);
            if (!(t.is_cuda() && t.device() == first.device() && t.scalar_type() == at::kInt && t.numel() == 1)) value_error("step must be a number or a one-element int32 tensor on the parameters' GPU");
            args.step_device = (const int32_t *)t.data_ptr();
            scalars = at::empty({2}, first.options().dtype(at::kFloat));
            args.scalars = (float *)scalars.data_ptr();
        } else args.step = long_integer(a[3]);
        void *st = stream_of(first);
        run([&] { return bra_adamw_step(list.data(), (int32_t)params.n, &args, st); });
        Py_RETURN_NONE;
    });
}

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void *)py_init, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void *)py_route, METH_FASTCALL, nullptr},
    {"forward", (PyCFunction)(void *)py_forward, METH_FASTCALL, nullptr},
    {"forward_static", (PyCFunction)(void *)py_forward_static, METH_FASTCALL, nullptr},
    {"forward_padded", (PyCFunction)(void *)py_forward_padded, METH_FASTCALL, nullptr},
    {"backward", (PyCFunction)(void *)py_backward, METH_FASTCALL, nullptr},
    {"block_forward", (PyCFunction)(void *)py_block_forward, METH_FASTCALL, nullptr},
    {"ffn_forward", (PyCFunction)(void *)py_ffn_forward, METH_FASTCALL, nullptr},
    {"ffn_backward", (PyCFunction)(void *)py_ffn_backward, METH_FASTCALL, nullptr},
    {"norm_forward", (PyCFunction)(void *)py_norm_forward, METH_FASTCALL, nullptr},
    {"norm_backward", (PyCFunction)(void *)py_norm_backward, METH_FASTCALL, nullptr},
    {"adamw_step", (PyCFunction)(void *)py_adamw_step, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
