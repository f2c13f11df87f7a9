// Calls of the layer norm, the gated products and the embedding on torch tensors, and of what reads
// their 8-bit rows back (host code only).
//
// whtmix.py checks its arguments and allocates in Python, which takes 3 to 4 us of a call of a
// few rows whose kernel and launch take 3.  These functions make the same call where all of it is
// ordinary (contiguous tensors with elements, of the types and shapes asked for, on the current
// device, no `out` and no stream named) and return None otherwise: then whtmix.py goes its own way, which
// takes rows of wider tensors too and raises what there is to raise.  They decide nothing else.
// A layer norm of one row takes 5.7 us a call, 8.6 by way of Python; 17 embedded rows 5.0 and 7.4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

using at::Tensor;
typedef void *P;
typedef int64_t I;

// The entry points, in the order of bind()'s addresses.
enum Entry { LAYER_NORM, LAYER_NORM_MX, LAYER_NORM_BACKWARD, GATED, GATED_BACKWARD, GATED_MX,
             EMBEDDING, EMBEDDING_BACKWARD, DEQUANTIZE_MX, kEntries };
void *g_entry[kEntries];
PyObject *g_parameter;      // torch.nn.Parameter

// bind(addresses, torch.nn.Parameter)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs != 2 || !PyTuple_Check(args[0]) || PyTuple_GET_SIZE(args[0]) != kEntries) {
        PyErr_SetString(PyExc_TypeError, "bind() takes the entry points' addresses and a type");
        return nullptr;
    }
    for (int i = 0; i < kEntries; ++i) {
        g_entry[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args[0], i));
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[1]);
    Py_XSETREF(g_parameter, args[1]);
    Py_RETURN_NONE;
}

// A call on its way: what it has found to be ordinary, and what it will pass.
struct Call {
    bool ok = true;
    int device = -1, code = 0;
    at::ScalarType type = at::kFloat;

    // The tensor behind an object that is torch.Tensor or a parameter (no other subclass).
    const Tensor *tensor(PyObject *o)
    {
        ok = ok && (THPVariable_CheckExact(o) || (PyObject *)Py_TYPE(o) == g_parameter);
        return ok ? &THPVariable_Unpack(o) : nullptr;
    }
    // The first operand: its type and device are the others' too.
    const Tensor *first(PyObject *o, at::ScalarType only = at::ScalarType::Undefined)
    {
        const Tensor *t = tensor(o);
        if (!t) return nullptr;
        type = t->scalar_type();
        code = type == at::kBFloat16 ? 1 : 0;
        ok = t->is_cuda() && t->layout() == at::kStrided && t->numel() > 0 && t->is_contiguous() && !t->is_conj() &&
             !t->is_neg() &&
             (only == at::ScalarType::Undefined ? type == at::kFloat || type == at::kBFloat16
                                                : type == only);
        if (!ok) return nullptr;
        device = t->get_device();
        ok = device == c10::hip::current_device();
        return ok ? t : nullptr;
    }
    // Another one of this type and shape: its address, or null for None.
    P other(PyObject *o, at::ScalarType as, at::IntArrayRef shape, bool optional = false)
    {
        if (optional && o == Py_None) return nullptr;
        const Tensor *t = tensor(o);
        if (!t) return nullptr;
        ok = t->is_cuda() && t->scalar_type() == as && t->get_device() == device &&
             t->sizes() == shape && t->is_contiguous();
        return ok ? t->data_ptr() : nullptr;
    }
    Tensor fresh(at::IntArrayRef shape, at::ScalarType as) const
    {
        return at::empty(shape, at::TensorOptions().dtype(as).device(at::kCUDA, device));
    }
    P stream() const { return c10::hip::getCurrentHIPStream(device).stream(); }
};

bool number(PyObject *o, double &v)
{
    v = PyFloat_AsDouble(o);
    return !(v == -1.0 && PyErr_Occurred());
}

// A status as an int (which the caller raises on), or the result for success.
PyObject *result(int status, std::initializer_list<PyObject *> values)
{
    if (status != 0) {
        for (PyObject *v : values) Py_XDECREF(v);
        return PyLong_FromLong(status);
    }
    PyObject *t = PyTuple_New((Py_ssize_t)values.size());
    Py_ssize_t i = 0;
    for (PyObject *v : values) {
        if (t) PyTuple_SET_ITEM(t, i++, v);
        else Py_XDECREF(v);
    }
    return t;
}

PyObject *wrap(Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}
P address(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
PyObject *or_none(const Tensor &t) { return t.defined() ? wrap(t) : none(); }

// C++ exceptions (an allocation that fails) leave as Python's RuntimeError.
template <typename F> PyObject *guarded(const char *name, Py_ssize_t nargs, Py_ssize_t want, F f)
{
    if (nargs != want) {
        PyErr_Format(PyExc_TypeError, "%s() takes %zd arguments", name, want);
        return nullptr;
    }
    try {
        return f();
    } catch (const c10::OutOfMemoryError &) {
        Py_RETURN_NONE;         // the Python way meets it again and raises torch's own error
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

template <typename F, typename... A> int call(Entry e, A... a)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = ((F)g_entry[e])(a...);
    Py_END_ALLOW_THREADS
    return status;
}

int64_t mx_width(int64_t C) { return (C + 31) / 32 * 32; }

// Rows and width of a tensor [..., C].
bool rows_of(const Tensor &t, int64_t &rows, int64_t &C)
{
    if (t.dim() < 2 || (C = t.size(-1)) < 1) return false;
    rows = t.numel() / C;
    return true;
}

at::DimVector with_last(at::IntArrayRef shape, int64_t last)
{
    at::DimVector s(shape.begin(), shape.end());
    s.back() = last;
    return s;
}

// layer_norm(x, weight, bias, residual, eps) -> (y, h)
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("layer_norm", nargs, 5, [&]() -> PyObject * {
        Call c;
        int64_t rows, C;
        double eps;
        if (!number(args[4], eps)) return nullptr;
        const Tensor *x = c.first(args[0]);
        if (!x || !rows_of(*x, rows, C)) return none();
        const P w = c.other(args[1], at::kFloat, {C}), b = c.other(args[2], at::kFloat, {C}, true),
                r = c.other(args[3], c.type, x->sizes(), true);
        if (!c.ok) return none();
        Tensor y = c.fresh(x->sizes(), c.type), h;
        if (r) h = c.fresh(x->sizes(), c.type);
        const int st = call<int (*)(P, P, P, P, P, P, I, I, I, double, int, P)>(
            LAYER_NORM, x->data_ptr(), r, w, b, y.data_ptr(), address(h), rows, C, C, eps, c.code,
            c.stream());
        if (!r) Py_INCREF(args[0]);         // the stream is x itself
        return result(st, {wrap(y), r ? wrap(h) : args[0]});
    });
}

// layer_norm_mx(x, weight, bias, residual, eps) -> (q, scales, h)
PyObject *layer_norm_mx(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("layer_norm_mx", nargs, 5, [&]() -> PyObject * {
        Call c;
        int64_t rows, C;
        double eps;
        if (!number(args[4], eps)) return nullptr;
        const Tensor *x = c.first(args[0]);
        if (!x || !rows_of(*x, rows, C)) return none();
        const P w = c.other(args[1], at::kFloat, {C}), b = c.other(args[2], at::kFloat, {C}, true),
                r = c.other(args[3], c.type, x->sizes(), true);
        if (!c.ok) return none();
        Tensor q = c.fresh(with_last(x->sizes(), mx_width(C)), at::kFloat8_e4m3fn),
               s = c.fresh(with_last(x->sizes(), mx_width(C) / 32), at::kByte), h;
        if (r) h = c.fresh(x->sizes(), c.type);
        const int st = call<int (*)(P, P, P, P, P, P, P, I, I, I, double, int, P)>(
            LAYER_NORM_MX, x->data_ptr(), r, w, b, q.data_ptr(), s.data_ptr(), address(h), rows, C,
            C, eps, c.code, c.stream());
        if (!r) Py_INCREF(args[0]);
        return result(st, {wrap(q), wrap(s), r ? wrap(h) : args[0]});
    });
}

// layer_norm_backward(h, weight, dy, dh, eps, want_dweight, want_dbias) -> (dx, dweight, dbias)
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("layer_norm_backward", nargs, 7, [&]() -> PyObject * {
        Call c;
        int64_t rows, C;
        double eps;
        if (!number(args[4], eps)) return nullptr;
        const int dweight = PyObject_IsTrue(args[5]), dbias = PyObject_IsTrue(args[6]);
        if (dweight < 0 || dbias < 0) return nullptr;
        const Tensor *h = c.first(args[0]);
        if (!h || !rows_of(*h, rows, C)) return none();
        const P w = c.other(args[1], at::kFloat, {C}), dy = c.other(args[2], c.type, h->sizes()),
                dh = c.other(args[3], c.type, h->sizes(), true);
        if (!c.ok) return none();
        Tensor dx = c.fresh(h->sizes(), c.type), dw, db;
        if (dweight) dw = c.fresh({C}, at::kFloat);
        if (dbias) db = c.fresh({C}, at::kFloat);
        const int st = call<int (*)(P, P, P, P, P, P, P, I, I, double, int, P)>(
            LAYER_NORM_BACKWARD, h->data_ptr(), w, dy, dh, dx.data_ptr(), address(dw), address(db),
            rows, C, eps, c.code, c.stream());
        return result(st, {wrap(dx), or_none(dw), or_none(db)});
    });
}

// gated(x, w_gate, w_up, b_gate, b_up, activation, want_z) -> (y,) or (y, z_gate, z_up)
PyObject *gated(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("gated", nargs, 7, [&]() -> PyObject * {
        Call c;
        int64_t M, K;
        const long act = PyLong_AsLong(args[5]);
        if (act == -1 && PyErr_Occurred()) return nullptr;
        const int want = PyObject_IsTrue(args[6]);
        if (want < 0) return nullptr;
        const Tensor *x = c.first(args[0]);
        if (!x || !rows_of(*x, M, K)) return none();
        const Tensor *w = c.tensor(args[1]);
        if (!w || w->dim() != 2 || w->size(0) != K || w->size(1) < 1) return none();
        const int64_t N = w->size(1);
        const P wg = c.other(args[1], c.type, {K, N}), wu = c.other(args[2], c.type, {K, N}),
                bg = c.other(args[3], at::kFloat, {N}, true),
                bu = c.other(args[4], at::kFloat, {N}, true);
        if (!c.ok) return none();
        const at::DimVector shape = with_last(x->sizes(), N);
        Tensor y = c.fresh(shape, c.type), zg, zu;
        if (want) zg = c.fresh(shape, c.type), zu = c.fresh(shape, c.type);
        const int st = call<int (*)(P, P, P, P, P, P, P, P, I, I, I, I, int, int, P)>(
            GATED, x->data_ptr(), wg, wu, bg, bu, y.data_ptr(), address(zg), address(zu), M, K, N,
            K, (int)act, c.code, c.stream());
        if (!want) return result(st, {wrap(y)});
        return result(st, {wrap(y), wrap(zg), wrap(zu)});
    });
}

// gated_backward(x, w_gate, w_up, dy, z_gate, z_up, activation, want_dx, want_dw, want_dbias) ->
// (dx, dw_gate, dw_up, db_gate, db_up)
PyObject *gated_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("gated_backward", nargs, 10, [&]() -> PyObject * {
        Call c;
        int64_t M, K;
        const long act = PyLong_AsLong(args[6]);
        if (act == -1 && PyErr_Occurred()) return nullptr;
        const int dx = PyObject_IsTrue(args[7]), dw = PyObject_IsTrue(args[8]),
                  db = PyObject_IsTrue(args[9]);
        if (dx < 0 || dw < 0 || db < 0) return nullptr;
        const Tensor *x = c.first(args[0]);
        if (!x || !rows_of(*x, M, K) || !(dx || dw || db)) return none();
        const Tensor *w = c.tensor(args[1]);
        if (!w || w->dim() != 2 || w->size(0) != K || w->size(1) < 1) return none();
        const int64_t N = w->size(1);
        const at::DimVector shape = with_last(x->sizes(), N);
        const P wg = c.other(args[1], c.type, {K, N}), wu = c.other(args[2], c.type, {K, N}),
                dy = c.other(args[3], c.type, shape), zg = c.other(args[4], c.type, shape),
                zu = c.other(args[5], c.type, shape);
        if (!c.ok) return none();
        Tensor ox, og, ou, obg, obu;
        if (dx) ox = c.fresh(x->sizes(), c.type);
        if (dw) og = c.fresh({K, N}, c.type), ou = c.fresh({K, N}, c.type);
        if (db) obg = c.fresh({N}, at::kFloat), obu = c.fresh({N}, at::kFloat);
        const int st = call<int (*)(P, P, P, P, P, P, P, P, P, P, P, I, I, I, I, int, int, P)>(
            GATED_BACKWARD, x->data_ptr(), wg, wu, dy, zg, zu, address(ox), address(og),
            address(ou), address(obg), address(obu), M, K, N, K, (int)act, c.code, c.stream());
        return result(st, {or_none(ox), or_none(og), or_none(ou), or_none(obg), or_none(obu)});
    });
}

// gated_mx(xq, xs, wgq, wgs, wuq, wus, b_gate, b_up, activation, out_mx) -> (y,) in bfloat16 or
// (q, scales)
PyObject *gated_mx(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("gated_mx", nargs, 10, [&]() -> PyObject * {
        Call c;
        int64_t M, K;
        const long act = PyLong_AsLong(args[8]);
        if (act == -1 && PyErr_Occurred()) return nullptr;
        const int mx = PyObject_IsTrue(args[9]);
        if (mx < 0) return nullptr;
        const Tensor *x = c.first(args[0], at::kFloat8_e4m3fn);
        if (!x || !rows_of(*x, M, K) || K % 32) return none();
        const Tensor *w = c.tensor(args[2]);
        if (!w || w->dim() != 2 || w->size(1) != K || w->size(0) < 1) return none();
        const int64_t N = w->size(0);
        const P xs = c.other(args[1], at::kByte, with_last(x->sizes(), K / 32)),
                wg = c.other(args[2], c.type, {N, K}), gs = c.other(args[3], at::kByte, {N, K / 32}),
                wu = c.other(args[4], c.type, {N, K}), us = c.other(args[5], at::kByte, {N, K / 32}),
                bg = c.other(args[6], at::kFloat, {N}, true),
                bu = c.other(args[7], at::kFloat, {N}, true);
        if (!c.ok) return none();
        Tensor y, q, s;
        if (mx) {
            q = c.fresh(with_last(x->sizes(), mx_width(N)), at::kFloat8_e4m3fn);
            s = c.fresh(with_last(x->sizes(), mx_width(N) / 32), at::kByte);
        } else {
            y = c.fresh(with_last(x->sizes(), N), at::kBFloat16);
        }
        const int st = call<int (*)(P, P, P, P, P, P, P, P, P, P, P, I, I, I, int, int, P)>(
            GATED_MX, x->data_ptr(), xs, wg, gs, wu, us, bg, bu, address(y), address(q),
            address(s), M, K, N, (int)act, 1, c.stream());
        if (!mx) return result(st, {wrap(y)});
        return result(st, {wrap(q), wrap(s)});
    });
}

// dequantize_mx(q, scales, C, dtype code) -> (y,): what layer_norm_mx and gated_mx give, read back
PyObject *dequantize_mx(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("dequantize_mx", nargs, 4, [&]() -> PyObject * {
        Call c;
        int64_t rows, width;
        const long long C = PyLong_AsLongLong(args[2]);
        const long code = C == -1 && PyErr_Occurred() ? -1 : PyLong_AsLong(args[3]);
        if (PyErr_Occurred()) return nullptr;
        const Tensor *q = c.first(args[0], at::kFloat8_e4m3fn);
        if (!q || !rows_of(*q, rows, width) || width % 32) return none();
        const P s = c.other(args[1], at::kByte, with_last(q->sizes(), width / 32));
        if (!c.ok || C < 1 || mx_width(C) != width || (code != 0 && code != 1)) return none();
        Tensor y = c.fresh(with_last(q->sizes(), C), code == 1 ? at::kBFloat16 : at::kFloat);
        const int st = call<int (*)(P, P, P, I, I, int, P)>(
            DEQUANTIZE_MX, q->data_ptr(), s, y.data_ptr(), rows, (int64_t)C, (int)code, c.stream());
        return result(st, {wrap(y)});
    });
}

// The index code of token ids, or -1.
int index_of(const Tensor &t)
{
    return t.scalar_type() == at::kInt ? 0 : t.scalar_type() == at::kLong ? 1 : -1;
}

// embedding(ids, table, scale) -> (y,)
PyObject *embedding(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("embedding", nargs, 3, [&]() -> PyObject * {
        Call c;
        int64_t V, C;
        double scale;
        if (!number(args[2], scale)) return nullptr;
        const Tensor *table = c.first(args[1]);
        if (!table || table->dim() != 2 || !rows_of(*table, V, C)) return none();
        const Tensor *ids = c.tensor(args[0]);
        const int index = ids ? index_of(*ids) : -1;
        if (index < 0 || !ids->is_contiguous() || !ids->is_cuda() || ids->numel() == 0 ||
            ids->get_device() != c.device)
            return none();
        at::DimVector shape(ids->sizes().begin(), ids->sizes().end());
        shape.push_back(C);
        Tensor y = c.fresh(shape, c.type);
        const int st = call<int (*)(P, P, P, I, I, I, double, int, int, P)>(
            EMBEDDING, ids->data_ptr(), table->data_ptr(), y.data_ptr(), ids->numel(), V, C, scale,
            index, c.code, c.stream());
        return result(st, {wrap(y)});
    });
}

// embedding_backward(ids, dy, vocab, scale) -> (dtable,)
PyObject *embedding_backward(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return guarded("embedding_backward", nargs, 4, [&]() -> PyObject * {
        Call c;
        double scale;
        const long long V = PyLong_AsLongLong(args[2]);
        if ((V == -1 && PyErr_Occurred()) || !number(args[3], scale)) return nullptr;
        const Tensor *dy = c.first(args[1]);
        const Tensor *ids = dy ? c.tensor(args[0]) : nullptr;
        const int index = ids ? index_of(*ids) : -1;
        if (index < 0 || !ids->is_contiguous() || !ids->is_cuda() ||
            ids->get_device() != c.device || V < 1 || dy->dim() != ids->dim() + 1 ||
            dy->sizes().slice(0, ids->dim()) != ids->sizes() || dy->size(-1) < 1)
            return none();
        const int64_t C = dy->size(-1);
        Tensor dtable = c.fresh({(int64_t)V, C}, c.type);
        const int st = call<int (*)(P, P, P, I, I, I, double, int, int, P)>(
            EMBEDDING_BACKWARD, ids->data_ptr(), dy->data_ptr(), dtable.data_ptr(), ids->numel(),
            (int64_t)V, C, scale, index, c.code, c.stream());
        return result(st, {wrap(dtable)});
    });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, #name "(): see the source"}
PyMethodDef methods[] = {METHOD(bind),  METHOD(layer_norm),     METHOD(layer_norm_mx),
                         METHOD(layer_norm_backward), METHOD(gated), METHOD(gated_backward),
                         METHOD(gated_mx), METHOD(embedding), METHOD(embedding_backward),
                         METHOD(dequantize_mx),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_whtmix_torch",
                      "Calls of whtmix entry points on torch tensors", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__whtmix_torch(void) { return PyModule_Create(&module); }
