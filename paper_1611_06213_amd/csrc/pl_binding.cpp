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

#include <ATen/ops/empty.h>
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

// rows x cols of `dtype` (a torch.dtype), or `out` if it is not None.
bool result(PyObject *out, PyObject *dtype, int64_t rows, int64_t cols, const at::Tensor &like,
            Matrix *m) {
    if (out != Py_None) return matrix(out, m) && m->rows == rows && m->cols == cols;
    if (!THPDtype_Check(dtype)) return false;
    const at::ScalarType s = reinterpret_cast<THPDtype *>(dtype)->scalar_type;
    int code;
    return code_of(s, &code) && as_matrix(at::empty({rows, cols}, like.options().dtype(s)), m);
}

at::Tensor bytes(size_t n, const at::Tensor &like) {
    return at::empty({static_cast<int64_t>(n)}, like.options().dtype(at::kByte));
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
    if (a[2] == Py_None) as_matrix(at::empty({x.rows, x.cols}, x.t.options()), &out);
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
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_learner", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__learner(void) { return PyModule_Create(&module); }
