// A learner's operators from Python tensors to the C ABI in one native call: the checks
// of the binding, the result's and the scratch memory's allocation on torch's current stream,
// and the calls, with the interpreter's lock released. Through ctypes and torch's
// Python methods a call takes 13 to 16 us, more than most small operators themselves; so 5.
//
// Each function returns its result, or the status of a call that was refused, or None,
// with nothing done, for arguments that it does not take (tensor subclasses, wrong
// sizes, types or devices): the Python binding then makes the calls itself and raises
// what is to be raised.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ps_learner.h"

namespace {

// A device matrix with unit column stride, on the current device.
struct Matrix {
    at::Tensor t;
    void *p = nullptr;
    int dtype = PS_F32;
    int64_t rows = 0, cols = 0, ld = 0;
};

bool code_of(at::ScalarType s, int *code) {
    if (s == at::kFloat) *code = PS_F32;
    else if (s == at::kBFloat16) *code = PS_BF16;
    else return false;
    return true;
}

bool device_tensor(PyObject *o, at::Tensor *out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.device().index() != c10::hip::current_device())
        return false;
    *out = t;
    return true;
}

bool as_matrix(const at::Tensor &t, Matrix *m) {
    if (t.dim() != 2 || !code_of(t.scalar_type(), &m->dtype)) return false;
    m->rows = t.size(0);
    m->cols = t.size(1);
    if (m->cols > 1 && t.stride(1) != 1) return false;
    m->ld = t.stride(0);   // 0, of rows that share their memory, is refused by the library
    m->p = t.data_ptr();
    m->t = t;
    return true;
}

bool matrix(PyObject *o, Matrix *m) {
    at::Tensor t;
    return device_tensor(o, &t) && as_matrix(t, m);
}

// As at::empty, past the dispatcher: the six tensors of norm_grad in 12.4 us of a call instead of 14.2.
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType dtype, const at::Tensor &like) {
    return at::Tensor(at::detail::empty_cuda(sizes, dtype, like.device(), std::nullopt));
}

// rows x cols of `dtype` (a torch.dtype), or `out` if it is not None.
bool result(PyObject *out, PyObject *dtype, int64_t rows, int64_t cols, const at::Tensor &like,
            Matrix *m) {
    if (out != Py_None) return matrix(out, m) && m->rows == rows && m->cols == cols;
    if (!THPDtype_Check(dtype)) return false;
    const at::ScalarType s = reinterpret_cast<THPDtype *>(dtype)->scalar_type;
    int code;
    return code_of(s, &code) && as_matrix(empty({rows, cols}, s, like), m);
}

at::Tensor bytes(size_t n, const at::Tensor &like) {
    return empty({static_cast<int64_t>(n)}, at::kByte, like);
}

bool ids(PyObject *o, at::Tensor *t, int *type) {
    if (!device_tensor(o, t) || !t->is_contiguous()) return false;
    if (t->scalar_type() == at::kLong) *type = PL_I64;
    else if (t->scalar_type() == at::kInt) *type = PL_I32;
    else return false;
    return true;
}

// A Dropout (p, seed, offset) or None.
struct MaybeDrop {
    pl_drop d;
    const pl_drop *p = nullptr;
};

bool dropping(PyObject *o, MaybeDrop *out) {
    if (o == Py_None) return true;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) return false;
    out->d.p = static_cast<float>(PyFloat_AsDouble(PyTuple_GET_ITEM(o, 0)));
    out->d.seed = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(o, 1));
    out->d.offset = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(o, 2));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    out->p = &out->d;
    return true;
}

bool integer(PyObject *o, int64_t *out) {
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsLongLong(o);
    if (*out == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

bool number(PyObject *o, float *out) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    *out = static_cast<float>(PyFloat_AsDouble(o));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// Any object's truth, as Python has it.
bool flag(PyObject *o, bool *out) {
    const int truth = PyObject_IsTrue(o);
    if (truth < 0) PyErr_Clear();
    *out = truth > 0;
    return truth >= 0;
}

bool shape(const at::Tensor &t, int64_t rows, int64_t cols) {
    return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.is_contiguous();
}

// A matrix in 8-bit form from its parts (values, scales, rows, cols).
struct Fp8 {
    at::Tensor values, scales;
    pl_fp8 q;
    int64_t rows = 0, cols = 0;
};

bool fp8(PyObject *o, Fp8 *f) {
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 4) return false;
    if (!device_tensor(PyTuple_GET_ITEM(o, 0), &f->values) ||
        !device_tensor(PyTuple_GET_ITEM(o, 1), &f->scales) ||
        !integer(PyTuple_GET_ITEM(o, 2), &f->rows) || !integer(PyTuple_GET_ITEM(o, 3), &f->cols))
        return false;
    // a caller may have exchanged the tensors for others
    const int64_t words = (pl_fp8_ld(f->cols) / 128 + 3) / 4;
    if (f->values.scalar_type() != at::kFloat8_e4m3fn || f->scales.scalar_type() != at::kInt ||
        !shape(f->values, f->rows, pl_fp8_ld(f->cols)) || !shape(f->scales, words, f->rows))
        return false;
    f->q = pl_fp8{f->values.data_ptr(), static_cast<uint32_t *>(f->scales.data_ptr())};
    return true;
}

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Runs `f` (which returns a status and may not touch Python) without the lock, which is taken back
// when `f` throws, too: asking for the stream may.
template <class F>
int unlocked(F f) {
    struct Released {
        PyThreadState *state = PyEval_SaveThread();
        ~Released() { PyEval_RestoreThread(state); }
    } released;
    return f();
}

PyObject *give(int rc, PyObject *out, const at::Tensor &t) {
    if (rc != PS_OK) return PyLong_FromLong(rc);
    if (out != Py_None) {
        Py_INCREF(out);
        return out;
    }
    return THPVariable_Wrap(t);
}

// Wraps an entry: an exception of torch's (out of memory) becomes Python's.
template <PyObject *(*F)(PyObject *const *), int COUNT>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t count) {
    if (count != COUNT) return PyErr_Format(PyExc_TypeError, "%d arguments expected", COUNT);
    try {
        return F(a);
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// embedding(ids, table, scale, drop, dtype, out)
PyObject *embedding(PyObject *const *a) {
    at::Tensor id;
    Matrix table, out;
    MaybeDrop drop;
    int type;
    float scale;
    if (!ids(a[0], &id, &type) || !matrix(a[1], &table) || !number(a[2], &scale) ||
        !dropping(a[3], &drop) || !result(a[5], a[4], id.numel(), table.cols, table.t, &out))
        Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return pl_embedding(id.data_ptr(), type, id.numel(), table.p, table.dtype, table.rows, table.cols,
                            table.ld, scale, drop.p, out.p, out.dtype, out.ld, stream());
    });
    if (rc == PS_OK && a[5] == Py_None && id.dim() != 1) {
        std::vector<int64_t> shape(id.sizes().begin(), id.sizes().end());
        shape.push_back(table.cols);
        return THPVariable_Wrap(out.t.view(shape));
    }
    return give(rc, a[5], out.t);
}

// embedding_grad(ids, grad, rows, scale, drop, dtype, out, accumulate)
PyObject *embedding_grad(PyObject *const *a) {
    at::Tensor id;
    Matrix grad, out;
    MaybeDrop drop;
    int type;
    int64_t rows;
    float scale;
    bool accumulate;
    if (!flag(a[7], &accumulate) || !ids(a[0], &id, &type) || !matrix(a[1], &grad) || grad.rows != id.numel() ||
        !integer(a[2], &rows) || rows < 0 || !number(a[3], &scale) || !dropping(a[4], &drop) ||
        (accumulate && a[6] == Py_None) || !result(a[6], a[5], rows, grad.cols, grad.t, &out))
        Py_RETURN_NONE;
    const size_t need = pl_embedding_grad_workspace(id.numel(), rows, grad.cols);
    const at::Tensor work = bytes(need, grad.t);
    const int rc = unlocked([&] {
        return pl_embedding_grad(id.data_ptr(), type, id.numel(), grad.p, grad.dtype, grad.ld, grad.cols,
                                 scale, drop.p, out.p, out.dtype, out.ld, rows, accumulate,
                                 work.data_ptr(), need, stream());
    });
    return give(rc, a[6], out.t);
}

// dropout(x, drop, out), x a matrix
PyObject *dropout(PyObject *const *a) {
    Matrix x, out;
    MaybeDrop drop;
    if (!matrix(a[0], &x) || a[1] == Py_None || !dropping(a[1], &drop)) Py_RETURN_NONE;
    if (a[2] == Py_None) as_matrix(empty({x.rows, x.cols}, x.t.scalar_type(), x.t), &out);
    else if (!matrix(a[2], &out) || out.rows != x.rows || out.cols != x.cols || out.dtype != x.dtype)
        Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return pl_dropout(x.p, x.dtype, x.rows, x.cols, x.ld, drop.p, out.p, out.ld, stream());
    });
    return give(rc, a[2], out.t);
}

// A bias of n values, or none.
bool bias(PyObject *o, int64_t n, at::Tensor *t, const void **p, int *code) {
    *p = nullptr;
    *code = PS_F32;
    if (o == Py_None) return true;
    if (!device_tensor(o, t) || t->dim() != 1 || t->size(0) != n || !t->is_contiguous() ||
        !code_of(t->scalar_type(), code))
        return false;
    *p = t->data_ptr();
    return true;
}

// product(a, b, bias, relu, dtype, out, accumulate), a and b parts of 8-bit matrices
PyObject *product(PyObject *const *a) {
    Fp8 x, w;
    Matrix out;
    at::Tensor b;
    const void *pb;
    int bias_code;
    bool relu, accumulate;
    if (!flag(a[3], &relu) || !flag(a[6], &accumulate) || !fp8(a[0], &x) || !fp8(a[1], &w) ||
        x.cols != w.cols || !bias(a[2], w.rows, &b, &pb, &bias_code) ||
        (accumulate && a[5] == Py_None) || !result(a[5], a[4], x.rows, w.rows, x.scales, &out))
        Py_RETURN_NONE;
    const size_t need = pl_matmul_fp8_workspace(x.rows, w.rows, x.cols, out.dtype);
    at::Tensor work;
    if (need) work = bytes(need, out.t);
    const int rc = unlocked([&] {
        return pl_matmul_fp8(x.rows, w.rows, x.cols, &x.q, &w.q, pb, bias_code, relu, out.p, out.dtype,
                             out.ld, accumulate, need ? work.data_ptr() : nullptr, need, stream());
    });
    return give(rc, a[5], out.t);
}

// linear(x, w, bias, relu, dtype, out), w the parts of an 8-bit matrix
PyObject *linear(PyObject *const *a) {
    Matrix x, out;
    Fp8 w;
    at::Tensor b;
    const void *pb;
    int bias_code;
    bool relu;
    if (!flag(a[3], &relu) || !matrix(a[0], &x) || !fp8(a[1], &w) || x.cols != w.cols ||
        !bias(a[2], w.rows, &b, &pb, &bias_code) ||
        !result(a[5], a[4], x.rows, w.rows, x.t, &out))
        Py_RETURN_NONE;
    const size_t need = pl_linear_fp8_workspace(x.rows, w.rows, x.cols, x.dtype, out.dtype);
    at::Tensor work;
    if (need) work = bytes(need, out.t);
    const int rc = unlocked([&] {
        return pl_linear_fp8(x.p, x.dtype, x.rows, x.cols, x.ld, w.rows, &w.q, pb, bias_code, relu, out.p,
                             out.dtype, out.ld, need ? work.data_ptr() : nullptr, need, stream());
    });
    return give(rc, a[5], out.t);
}

// linear_grad(x, grad, w_t, dtype, weight_dtype, x_out, weight_out, accumulate)
PyObject *linear_grad(PyObject *const *a) {
    Matrix x, g, dx, dw;
    Fp8 w;   // inputs x outputs
    bool accumulate;
    if (!flag(a[7], &accumulate) || !matrix(a[0], &x) || !matrix(a[1], &g) || !fp8(a[2], &w) ||
        x.rows != g.rows || w.rows != x.cols || w.cols != g.cols || (accumulate && a[6] == Py_None) ||
        !result(a[5], a[3], x.rows, x.cols, x.t, &dx) || !result(a[6], a[4], g.cols, x.cols, x.t, &dw))
        Py_RETURN_NONE;
    const int64_t m = x.rows, k = x.cols, n = g.cols;
    const size_t need = pl_linear_fp8_grad_workspace(m, n, k, dx.dtype, dw.dtype);
    const at::Tensor work = bytes(need, x.t);
    const int rc = unlocked([&] {
        return pl_linear_fp8_grad(x.p, x.dtype, x.ld, g.p, g.dtype, g.ld, m, n, k, &w.q, dx.p, dx.dtype, dx.ld,
                                  dw.p, dw.dtype, dw.ld, accumulate, work.data_ptr(), need, stream());
    });
    if (rc != PS_OK) return PyLong_FromLong(rc);
    PyObject *px = give(rc, a[5], dx.t), *pw = give(rc, a[6], dw.t);
    if (px == nullptr || pw == nullptr) {
        Py_XDECREF(px);
        Py_XDECREF(pw);
        return nullptr;
    }
    return Py_BuildValue("(NN)", px, pw);
}

// `cols` contiguous values of a type that `*code` may already name (>= 0), or none.
bool values(PyObject *o, int64_t cols, at::Tensor *t, void **p, int *code) {
    *p = nullptr;
    if (o == Py_None) return true;
    int own;
    if (!device_tensor(o, t) || t->dim() != 1 || t->size(0) != cols || !t->is_contiguous() ||
        !code_of(t->scalar_type(), &own) || (*code >= 0 && own != *code))
        return false;
    *code = own;
    *p = t->data_ptr();
    return true;
}

// A gate: `cols` values for all rows, or a matrix; or none.
struct Gate {
    at::Tensor t;
    void *p = nullptr;
    int dtype = PS_F32;
    int64_t rows = 0, ld = 0;
};

bool gate(PyObject *o, int64_t cols, Gate *g) {
    if (o == Py_None) return true;
    Matrix m;
    // without rows it has no address, which stands for no gate
    if (!device_tensor(o, &g->t) || !as_matrix(g->t.dim() == 1 ? g->t.unsqueeze(0) : g->t, &m) || m.cols != cols ||
        m.rows == 0)
        return false;
    g->p = m.p;
    g->dtype = m.dtype;
    g->rows = m.rows;
    g->ld = m.ld;
    return true;
}

// rows x cols of `code`: `out` if it is not None, else new.
bool like(PyObject *out, int64_t rows, int64_t cols, int code, const at::Tensor &on, Matrix *m) {
    if (out == Py_None)
        return as_matrix(empty({rows, cols}, code == PS_F32 ? at::kFloat : at::kBFloat16, on), m);
    return matrix(out, m) && m->rows == rows && m->cols == cols && m->dtype == code;
}

// A new reference to `out`, or to the tensor that was made instead.
PyObject *same(PyObject *out, const at::Tensor &t) {
    if (out == Py_None) return THPVariable_Wrap(t);
    Py_INCREF(out);
    return out;
}

// norm(x, y, gate, after, before, scale, eps, dtype, out, normed_out): h and z, or without a y z
PyObject *norm(PyObject *const *a) {
    Matrix x, y, out, normed;
    Gate g;
    at::Tensor ta, tb;
    void *after, *before;
    float scale, eps;
    int code = -1;
    const bool block = a[1] != Py_None, next = !block || a[4] != Py_None;
    // empty tensors have no address: the Python route
    if (!matrix(a[0], &x) || x.rows == 0 || x.cols == 0) Py_RETURN_NONE;
    if (block && (!matrix(a[1], &y) || y.rows != x.rows || y.cols != x.cols)) Py_RETURN_NONE;
    if (!gate(a[2], x.cols, &g) || !values(a[3], x.cols, &ta, &after, &code) ||
        !values(a[4], x.cols, &tb, &before, &code) || !number(a[5], &scale) || !number(a[6], &eps))
        Py_RETURN_NONE;
    int y_code = y.dtype;
    if (!block) {
        y_code = x.dtype;
        if (a[7] != Py_None && (!THPDtype_Check(a[7]) ||
                                !code_of(reinterpret_cast<THPDtype *>(a[7])->scalar_type, &y_code)))
            Py_RETURN_NONE;
        if (a[9] != Py_None && a[7] == Py_None) {
            Matrix m;
            if (!matrix(a[9], &m)) Py_RETURN_NONE;
            y_code = m.dtype;
        }
    }
    if ((block ? !like(a[8], x.rows, x.cols, x.dtype, x.t, &out) : a[8] != Py_None) ||
        (next ? !like(a[9], x.rows, x.cols, y_code, x.t, &normed) : a[9] != Py_None))
        Py_RETURN_NONE;
    const int rc = unlocked([&] {
        return pl_norm(x.p, x.dtype, x.ld, y.p, y_code, y.ld, x.rows, x.cols, g.p, g.dtype, g.rows, g.ld, after,
                       before, code < 0 ? PS_F32 : code, scale, eps, out.p, out.ld, normed.p, normed.ld, stream());
    });
    if (rc != PS_OK) return PyLong_FromLong(rc);
    PyObject *z = Py_None;
    if (next) z = same(a[9], normed.t);
    else Py_INCREF(z);
    if (!block || z == nullptr) return z;
    PyObject *h = same(a[8], out.t);
    if (h == nullptr) {
        Py_DECREF(z);
        return nullptr;
    }
    return Py_BuildValue("(NN)", h, z);
}

// Where the gradient of `of` (None: there is none) goes; *code: of all that are named.
bool weight_out(PyObject *out, PyObject *of, const at::Tensor &like, int *code, bool accumulate, at::ScalarType dtype,
                at::Tensor *t, Matrix *m) {
    if (of == Py_None) return out == Py_None;
    if (out == Py_None) {
        if (accumulate) return false;
        *t = empty(like.sizes(), dtype, like);
    } else if (!device_tensor(out, t) || t->sizes() != like.sizes() || (t->dim() == 1 && !t->is_contiguous())) {
        return false;
    }
    if (!as_matrix(t->dim() == 1 ? t->unsqueeze(0) : *t, m) || (*code >= 0 && m->dtype != *code)) return false;
    *code = m->dtype;
    return true;
}

// norm_grad(h, y, grad, normed_grad, gate, after, before, scale, eps, weight_dtype, x_out, y_out, gate_out,
// after_out, before_out, accumulate): gradients for x, y, gate, after, before
PyObject *norm_grad(PyObject *const *a) {
    Matrix h, y, dh, dz, dx, dy, out[3];
    Gate g;
    at::Tensor ta, tb, made[3];
    void *after, *before;
    float scale, eps;
    bool accumulate;
    int code = -1, out_code = -1;
    const bool block = a[1] != Py_None, next = a[3] != Py_None;
    if (!flag(a[15], &accumulate) || !matrix(a[0], &h) || h.rows == 0 || h.cols == 0) Py_RETURN_NONE;
    auto fits = [&](PyObject *o, Matrix *m) { return matrix(o, m) && m->rows == h.rows && m->cols == h.cols; };
    if ((block && !fits(a[1], &y)) || (a[2] != Py_None && (!fits(a[2], &dh) || dh.dtype != h.dtype)) ||
        (next && (!fits(a[3], &dz) || (block && dz.dtype != y.dtype))) || (!next && a[6] != Py_None))
        Py_RETURN_NONE;
    const int y_code = block ? y.dtype : next ? dz.dtype : h.dtype;
    if (!gate(a[4], h.cols, &g) || !values(a[5], h.cols, &ta, &after, &code) ||
        !values(a[6], h.cols, &tb, &before, &code) || !number(a[7], &scale) || !number(a[8], &eps) ||
        !THPDtype_Check(a[9]) || !like(a[10], h.rows, h.cols, h.dtype, h.t, &dx) ||
        (block ? !like(a[11], h.rows, h.cols, y.dtype, h.t, &dy) : a[11] != Py_None))
        Py_RETURN_NONE;
    const at::ScalarType dtype = reinterpret_cast<THPDtype *>(a[9])->scalar_type;
    const at::Tensor *of[3] = {&g.t, &ta, &tb};
    for (int i = 0; i < 3; ++i)
        if (!weight_out(a[12 + i], a[4 + i], *of[i], &out_code, accumulate, dtype, &made[i], &out[i])) Py_RETURN_NONE;
    const size_t need = pl_norm_grad_workspace(h.rows, h.cols);
    const at::Tensor work = bytes(need, h.t);
    const int rc = unlocked([&] {
        return pl_norm_grad(h.p, h.dtype, h.ld, y.p, y_code, y.ld, dh.p, dh.ld, dz.p, dz.ld, h.rows, h.cols, g.p,
                            g.dtype, g.rows, g.ld, after, before, code < 0 ? PS_F32 : code, scale, eps, dx.p, dx.ld,
                            dy.p, dy.ld, out[0].p, out[0].ld, out[1].p, out[2].p, out_code < 0 ? PS_F32 : out_code,
                            accumulate, work.data_ptr(), need, stream());
    });
    if (rc != PS_OK) return PyLong_FromLong(rc);
    PyObject *result = PyTuple_New(5);
    if (result == nullptr) return nullptr;
    const at::Tensor *given[5] = {&dx.t, block ? &dy.t : nullptr, g.p ? &made[0] : nullptr, after ? &made[1] : nullptr,
                                  before ? &made[2] : nullptr};
    for (int i = 0; i < 5; ++i) {
        PyObject *o = Py_None;
        if (given[i] != nullptr) o = same(a[10 + i], *given[i]);
        else Py_INCREF(o);
        if (o == nullptr) {
            Py_DECREF(result);
            return nullptr;
        }
        PyTuple_SET_ITEM(result, i, o);
    }
    return result;
}

// A matrix of 8-bit integers from its parts (values, scales, rows, cols).
struct Int8 {
    at::Tensor values, scales;
    pl_int8 q;
    int64_t rows = 0, cols = 0;
};

bool int8(PyObject *o, Int8 *f) {
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 4) return false;
    if (!device_tensor(PyTuple_GET_ITEM(o, 0), &f->values) || !device_tensor(PyTuple_GET_ITEM(o, 1), &f->scales) ||
        !integer(PyTuple_GET_ITEM(o, 2), &f->rows) || !integer(PyTuple_GET_ITEM(o, 3), &f->cols))
        return false;
    // a caller may have exchanged the tensors for others
    if (f->values.scalar_type() != at::kChar || f->scales.scalar_type() != at::kFloat ||
        !shape(f->values, f->rows, pl_int8_ld(f->cols)) || f->scales.dim() != 1 || f->scales.size(0) != f->rows ||
        !f->scales.is_contiguous())
        return false;
    f->q = pl_int8{static_cast<int8_t *>(f->values.data_ptr()), static_cast<float *>(f->scales.data_ptr())};
    return true;
}

// product_int8(a, b, bias, relu, dtype, out), a and b parts of matrices of integers
PyObject *product_int8(PyObject *const *a) {
    Int8 x, w;
    Matrix out;
    at::Tensor b;
    const void *pb;
    int bias_code;
    bool relu;
    if (!flag(a[3], &relu) || !int8(a[0], &x) || !int8(a[1], &w) || x.cols != w.cols ||
        !bias(a[2], w.rows, &b, &pb, &bias_code) || !result(a[5], a[4], x.rows, w.rows, x.scales, &out))
        Py_RETURN_NONE;
    const size_t need = pl_matmul_int8_workspace(x.rows, w.rows, x.cols);
    at::Tensor work;
    if (need) work = bytes(need, out.t);
    const int rc = unlocked([&] {
        return pl_matmul_int8(x.rows, w.rows, x.cols, &x.q, &w.q, pb, bias_code, relu, out.p, out.dtype, out.ld,
                              need ? work.data_ptr() : nullptr, need, stream());
    });
    return give(rc, a[5], out.t);
}

// linear_int8(x, w, bias, relu, dtype, out), w the parts of a matrix of integers
PyObject *linear_int8(PyObject *const *a) {
    Matrix x, out;
    Int8 w;
    at::Tensor b;
    const void *pb;
    int bias_code;
    bool relu;
    if (!flag(a[3], &relu) || !matrix(a[0], &x) || !int8(a[1], &w) || x.cols != w.cols ||
        !bias(a[2], w.rows, &b, &pb, &bias_code) || !result(a[5], a[4], x.rows, w.rows, x.t, &out))
        Py_RETURN_NONE;
    const size_t need = pl_linear_int8_workspace(x.rows, w.rows, x.cols);
    at::Tensor work;
    if (need) work = bytes(need, out.t);
    const int rc = unlocked([&] {
        return pl_linear_int8(x.p, x.dtype, x.rows, x.cols, x.ld, w.rows, &w.q, pb, bias_code, relu, out.p, out.dtype,
                              out.ld, need ? work.data_ptr() : nullptr, need, stream());
    });
    return give(rc, a[5], out.t);
}

// An optimizer's states: m, v and, of 8 bits, their scales (else None), which a caller may have exchanged.
struct States {
    void *p[4] = {};
    at::Tensor t[4];
};

bool states(PyObject *const *a, int64_t room, int64_t bits, States *s) {
    for (int i = 0; i < 4; ++i) {
        if (i >= 2 && bits == 32) break;
        if (!device_tensor(a[i], &s->t[i]) || !s->t[i].is_contiguous() ||
            s->t[i].scalar_type() != (bits == 32 ? at::kFloat : at::kByte) ||
            s->t[i].numel() != (i < 2 ? room : room / 128))
            return false;
        s->p[i] = s->t[i].data_ptr();
    }
    return true;
}

// A number, or one fp32 on the device.
bool number_or_tensor(PyObject *o, float *x, at::Tensor *t, const float **at) {
    *at = nullptr;
    *x = 0.0f;
    if (number(o, x)) return true;
    if (!device_tensor(o, t) || t->scalar_type() != at::kFloat || t->numel() != 1) return false;
    *at = static_cast<const float *>(t->data_ptr());
    return true;
}

// adamw_step(m, v, m_scales, v_scales, plan, (parts, room, weight code, grad code, push, bits, seed), beta1,
// beta2, eps, lr, factor): None if it is not made, else its status
PyObject *adamw_step(PyObject *const *a) {
    int64_t k[6];
    if (!PyTuple_CheckExact(a[5]) || PyTuple_GET_SIZE(a[5]) != 7) Py_RETURN_NONE;
    for (int i = 0; i < 6; ++i)
        if (!integer(PyTuple_GET_ITEM(a[5], i), &k[i])) Py_RETURN_NONE;
    const uint64_t seed = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(a[5], 6));
    const double beta1 = PyFloat_AsDouble(a[6]), beta2 = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    States s;
    at::Tensor plan, tl, tf;
    float eps, lr, factor;
    const float *lr_at, *factor_at;
    if (!states(a, k[1], k[5], &s) || !device_tensor(a[4], &plan) || !plan.is_contiguous() ||
        plan.scalar_type() != at::kByte || static_cast<size_t>(plan.numel()) != pl_adamw_plan_bytes(k[0]) ||
        !number(a[8], &eps) || !number_or_tensor(a[9], &lr, &tl, &lr_at) ||
        !number_or_tensor(a[10], &factor, &tf, &factor_at))
        Py_RETURN_NONE;
    return PyLong_FromLong(unlocked([&] {
        return pl_adamw_step(plan.data_ptr(), k[0], static_cast<int>(k[2]), static_cast<int>(k[3]),
                             static_cast<int>(k[4]), static_cast<int>(k[5]), k[1], s.p[0], s.p[1],
                             static_cast<uint8_t *>(s.p[2]), static_cast<uint8_t *>(s.p[3]), beta1, beta2, eps, lr,
                             lr_at, factor, factor_at, seed, stream());
    }));
}

// adamw_moments(m, v, m_scales, v_scales, room, dtype), of states in 8 bits: m and v of dtype
PyObject *adamw_moments(PyObject *const *a) {
    States s;
    int64_t room;
    int code;
    if (!integer(a[4], &room) || !states(a, room, 8, &s) || !THPDtype_Check(a[5]) ||
        !code_of(reinterpret_cast<THPDtype *>(a[5])->scalar_type, &code))
        Py_RETURN_NONE;
    const at::ScalarType dtype = code == PS_F32 ? at::kFloat : at::kBFloat16;
    const at::Tensor m = empty({room}, dtype, s.t[0]), v = empty({room}, dtype, s.t[0]);
    const int rc = unlocked([&] {
        return pl_adamw_moments(room, s.p[0], s.p[1], static_cast<uint8_t *>(s.p[2]), static_cast<uint8_t *>(s.p[3]),
                                m.data_ptr(), v.data_ptr(), code, stream());
    });
    if (rc != PS_OK) return PyLong_FromLong(rc);
    PyObject *pm = THPVariable_Wrap(m), *pv = THPVariable_Wrap(v);
    if (pm == nullptr || pv == nullptr) {
        Py_XDECREF(pm);
        Py_XDECREF(pv);
        return nullptr;
    }
    return Py_BuildValue("(NN)", pm, pv);
}

#define ENTRY(name, f, count, doc)                                                                  \
    {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<f, count>)), METH_FASTCALL, doc}

PyMethodDef methods[] = {
    ENTRY("embedding", embedding, 6, "embedding(ids, table, scale, drop, dtype, out)"),
    ENTRY("embedding_grad", embedding_grad, 8,
          "embedding_grad(ids, grad, rows, scale, drop, dtype, out, accumulate)"),
    ENTRY("dropout", dropout, 3, "dropout(x, drop, out)"),
    ENTRY("product", product, 7, "product(a, b, bias, relu, dtype, out, accumulate)"),
    ENTRY("linear", linear, 6, "linear(x, w, bias, relu, dtype, out)"),
    ENTRY("linear_grad", linear_grad, 8,
          "linear_grad(x, grad, w_t, dtype, weight_dtype, x_out, weight_out, accumulate)"),
    ENTRY("norm", norm, 10, "norm(x, y, gate, after, before, scale, eps, dtype, out, normed_out)"),
    ENTRY("norm_grad", norm_grad, 16,
          "norm_grad(h, y, grad, normed_grad, gate, after, before, scale, eps, weight_dtype, x_out, y_out, "
          "gate_out, after_out, before_out, accumulate)"),
    ENTRY("product_int8", product_int8, 6, "product_int8(a, b, bias, relu, dtype, out)"),
    ENTRY("linear_int8", linear_int8, 6, "linear_int8(x, w, bias, relu, dtype, out)"),
    ENTRY("adamw_step", adamw_step, 11,
          "adamw_step(m, v, m_scales, v_scales, plan, fixed, beta1, beta2, eps, lr, factor)"),
    ENTRY("adamw_moments", adamw_moments, 6, "adamw_moments(m, v, m_scales, v_scales, room, dtype)"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_learner", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__learner(void) { return PyModule_Create(&module); }
