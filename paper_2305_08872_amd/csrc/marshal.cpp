// Argument marshalling of the calls a program makes most often, for the Python binding: checks the tensors, reads
// pointers, sizes and pitches and calls libamulet.so, in place of some thirty attribute reads and calls from
// Python.  It takes ordinary arguments only and returns None for anything else, without calling the library: the
// binding then goes through its own checks, which word the errors.  Per call of 64^3, the launch (2.7)
// included, us on the host: 6.3 from Python, 3.3 from here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <initializer_list>
#include <vector>

#include "amulet.h"

namespace {

PyObject *g_get_device, *g_raw_stream;   // torch._C: the current device's index, the raw handle of its current stream

struct Mat {
    void *p;
    int64_t rows, cols, ld;
};

// a dense device tensor of this type
const at::Tensor *device_tensor(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != type) return nullptr;
    return &t;
}

// the leading dimension: a tensor of one row or no values may have any; one of no elements between rows (an expanded one) stays as it is, for
// the call to refuse
int64_t pitch(int64_t rows, int64_t cols, int64_t ld)
{
    if (rows <= 1) ld = cols;
    return ld > 0 || (rows > 1 && cols > 0) ? ld : 1;
}

// ... of two dimensions with unit column stride
bool matrix(PyObject *o, at::ScalarType type, Mat &m)
{
    const at::Tensor *t = device_tensor(o, type);
    if (!t || t->dim() != 2) return false;
    m.rows = t->size(0);
    m.cols = t->size(1);
    if (m.cols > 1 && t->stride(1) != 1) return false;
    m.ld = pitch(m.rows, m.cols, t->stride(0));
    m.p = t->data_ptr();
    return true;
}

// ... of n contiguous values
bool values(PyObject *o, at::ScalarType type, int64_t n, void *&p)
{
    const at::Tensor *t = device_tensor(o, type);
    if (!t || !t->is_contiguous() || t->numel() != n) return false;
    p = t->data_ptr();
    return true;
}

bool integer(PyObject *o, int &v)
{
    if (!PyLong_Check(o)) return false;
    const long n = PyLong_AsLong(o);
    if (n < -0x7fffffffL || n > 0x7fffffffL) {
        PyErr_Clear();
        return false;
    }
    v = (int)n;
    return true;
}

bool stream_handle(PyObject *o, void *&s)
{
    PyObject *handle;
    if (o == Py_None) {
        PyObject *dev = PyObject_CallNoArgs(g_get_device);
        if (!dev) {
            PyErr_Clear();
            return false;
        }
        handle = PyObject_CallOneArg(g_raw_stream, dev);
        Py_DECREF(dev);
    } else if (PyLong_Check(o)) {
        handle = o;
        Py_INCREF(o);
    } else {
        handle = PyObject_GetAttrString(o, "cuda_stream");
    }
    if (!handle || !PyLong_Check(handle)) {
        PyErr_Clear();
        Py_XDECREF(handle);
        return false;
    }
    s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

PyObject *not_here() { Py_RETURN_NONE; }

template <class F> PyObject *status(F call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (task, A, B, params, R, stream)
PyObject *mmlike_f32(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, B, R;
    int task;
    void *params = nullptr, *s;
    if (n != 6 || !integer(a[0], task) || !matrix(a[1], at::kFloat, A) || !matrix(a[2], at::kFloat, B) || !matrix(a[4], at::kFloat, R) ||
        A.cols != B.rows || A.rows != R.rows || B.cols != R.cols)
        return not_here();
    const int rows = task == AMULET_DISCOUNT ? 2 : task == AMULET_BOOST || task == AMULET_COUNT_GT ? 1 : 0;
    if (rows > 0 && a[3] != Py_None && !values(a[3], at::kFloat, rows * R.cols, params)) return not_here();
    if (!stream_handle(a[5], s)) return not_here();
    return status([&] {
        return amulet_mmlike_f32(task, R.rows, R.cols, A.cols, (const float *)A.p, A.ld, (const float *)B.p, B.ld, (const float *)params,
                                 (float *)R.p, R.ld, s);
    });
}

// operands, thresholds and discounts of a general-form call
struct General {
    Mat A, B, R;
    int task, form, ta, tb, shape;
    int64_t K, ldt;
    void *thres, *dis, *stream;
};

// (task, A, B, thres, dis, R, thres_form, trans_a, trans_b, shape, stream)
bool general(PyObject *const *a, Py_ssize_t n, at::ScalarType type, General &g)
{
    if (n != 11 || !integer(a[0], g.task) || !integer(a[6], g.form) || !integer(a[7], g.ta) || !integer(a[8], g.tb) || !integer(a[9], g.shape) ||
        !matrix(a[1], type, g.A) || !matrix(a[2], type, g.B) || !matrix(a[5], type, g.R))
        return false;
    g.K = g.ta ? g.A.rows : g.A.cols;
    if ((g.ta ? g.A.cols : g.A.rows) != g.R.rows || (g.tb ? g.B.cols : g.B.rows) != g.K || (g.tb ? g.B.rows : g.B.cols) != g.R.cols)
        return false;
    g.thres = g.dis = nullptr;
    g.ldt = 0;
    if (g.task != AMULET_IDENTITY) {
        if (g.form == AMULET_THRES_ELEM) {
            Mat t;
            if (!matrix(a[3], type, t) || t.rows != g.R.rows || t.cols != g.R.cols) return false;
            g.thres = t.p;
            g.ldt = t.ld;
        } else {
            const int64_t want = g.form == AMULET_THRES_COL ? g.R.cols : g.form == AMULET_THRES_ROW ? g.R.rows : g.form == AMULET_THRES_CONST ? 1 : -1;
            if (!values(a[3], type, want, g.thres)) return false;
        }
    }
    if (g.task == AMULET_DISCOUNT && !values(a[4], type, g.R.cols, g.dis)) return false;
    return stream_handle(a[10], g.stream);
}

PyObject *mmlike_f32_general(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    General g;
    if (!general(a, n, at::kFloat, g)) return not_here();
    return status([&] {
        return amulet_mmlike_f32_general(g.task, g.form, g.ta, g.tb, g.shape, g.R.rows, g.R.cols, g.K, (const float *)g.A.p, g.A.ld,
                                         (const float *)g.B.p, g.B.ld, (const float *)g.thres, g.ldt, (const float *)g.dis, (float *)g.R.p,
                                         g.R.ld, g.stream);
    });
}

PyObject *mmlike_f64(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    General g;
    if (!general(a, n, at::kDouble, g)) return not_here();
    return status([&] {
        return amulet_mmlike_f64_shape(g.task, g.shape, g.form, g.ta, g.tb, g.R.rows, g.R.cols, g.K, (const double *)g.A.p, g.A.ld,
                                       (const double *)g.B.p, g.B.ld, (const double *)g.thres, g.ldt, (const double *)g.dis, (double *)g.R.p,
                                       g.R.ld, g.stream);
    });
}

bool count_operands(PyObject *const *a, bool ta, bool tb, Mat &A, Mat &B, Mat &R)
{
    return matrix(a[0], at::kChar, A) && matrix(a[1], at::kChar, B) && matrix(a[2], at::kInt, R) && (ta ? A.cols : A.rows) == R.rows &&
           (tb ? B.rows : B.cols) == R.cols && (ta ? A.rows : A.cols) == (tb ? B.cols : B.rows);
}

// (A, B, R, stream)
PyObject *count_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, B, R;
    void *s;
    if (n != 4 || !count_operands(a, false, false, A, B, R) || !stream_handle(a[3], s)) return not_here();
    return status([&] {
        return amulet_count_i8(R.rows, R.cols, A.cols, (const int8_t *)A.p, A.ld, (const int8_t *)B.p, B.ld, (int32_t *)R.p, R.ld, s);
    });
}

// (A, B, R, shape, stream)
PyObject *count_i8_assign(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, B, R;
    int shape;
    void *s;
    if (n != 5 || !count_operands(a, false, false, A, B, R) || !integer(a[3], shape) || !stream_handle(a[4], s)) return not_here();
    return status([&] {
        return amulet_count_i8_assign(shape, R.rows, R.cols, A.cols, (const int8_t *)A.p, A.ld, (const int8_t *)B.p, B.ld, (int32_t *)R.p, R.ld, s);
    });
}

// (A, B, R, workspace, trans_a, trans_b, stream)
PyObject *count_i8_general(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, B, R;
    int ta, tb;
    void *s, *w = nullptr;
    size_t bytes = 0;
    if (n != 7 || !integer(a[4], ta) || !integer(a[5], tb) || !count_operands(a, ta, tb, A, B, R)) return not_here();
    if (a[3] != Py_None) {
        if (!THPVariable_CheckExact(a[3])) return not_here();
        const at::Tensor &t = THPVariable_Unpack(a[3]);
        if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || !t.is_contiguous()) return not_here();
        w = t.data_ptr();
        bytes = t.nbytes();
    }
    if (!stream_handle(a[6], s)) return not_here();
    return status([&] {
        return amulet_count_i8_general(ta, tb, R.rows, R.cols, ta ? A.rows : A.cols, (const int8_t *)A.p, A.ld, (const int8_t *)B.p, B.ld,
                                       (int32_t *)R.p, R.ld, w, bytes, s);
    });
}

// ---- operators of a mixture-of-experts layer

const at::Tensor *tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// the type's code and torch's type of an fp32, bf16 or fp16 tensor
bool known_type(PyObject *o, int &code, at::ScalarType &type)
{
    const at::Tensor *t = tensor(o);
    if (!t || !t->defined()) return false;
    type = t->scalar_type();
    code = type == at::kFloat ? AMULET_FP32 : type == at::kBFloat16 ? AMULET_BF16 : type == at::kHalf ? AMULET_FP16 : -1;
    return code >= 0;
}

struct Groups {
    void *p;
    int64_t n, rows, cols, ld, apart;
};
bool groups(PyObject *o, at::ScalarType type, Groups &g)
{
    const at::Tensor *t = device_tensor(o, type);
    if (!t || t->dim() != 3) return false;
    g.n = t->size(0);
    g.rows = t->size(1);
    g.cols = t->size(2);
    if (g.cols > 1 && t->stride(2) != 1) return false;
    g.ld = pitch(g.rows, g.cols, t->stride(1));
    g.apart = g.n > 1 ? t->stride(0) : g.rows * g.ld;
    g.p = t->data_ptr();
    return true;
}

// None, or n contiguous values
bool values_or_none(PyObject *o, at::ScalarType type, int64_t n, void *&p)
{
    p = nullptr;
    return o == Py_None || values(o, type, n, p);
}
bool bytes_or_none(PyObject *o, void *&p, size_t &n)
{
    p = nullptr;
    n = 0;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o);
    if (!t || !t->defined() || !t->is_cuda() || t->layout() != at::kStrided || !t->has_storage() || !t->is_contiguous()) return false;
    p = t->data_ptr();
    n = t->nbytes();
    return true;
}
// rows and columns of a 2-D tensor, whatever else it is
bool shape2(PyObject *o, int64_t &rows, int64_t &cols)
{
    const at::Tensor *t = tensor(o);
    if (!t || !t->defined() || t->dim() != 2) return false;
    rows = t->size(0);
    cols = t->size(1);
    return true;
}
int64_t blocks128(int64_t n) { return (n + 127) / 128; }

// (logits, experts, weights, place, tokens, offsets, workspace, norm, stream)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat X;
    int type, norm;
    at::ScalarType t;
    int64_t T, k;
    void *e, *w, *p, *tok, *off, *ws, *s;
    size_t bytes;
    if (n != 9 || !known_type(a[0], type, t) || !matrix(a[0], t, X) || !shape2(a[1], T, k) || T != X.rows || !values(a[1], at::kInt, T * k, e) ||
        !values(a[2], at::kFloat, T * k, w) || !values(a[3], at::kInt, T * k, p) || !values(a[4], at::kInt, T * k, tok) ||
        !values(a[5], at::kInt, X.cols + 1, off) || !bytes_or_none(a[6], ws, bytes) || !integer(a[7], norm) || !stream_handle(a[8], s))
        return not_here();
    return status([&] {
        return amulet_route(type, T, X.cols, k, X.p, X.ld, norm, (int32_t *)e, (float *)w, (int32_t *)p, (int32_t *)tok, (int32_t *)off, ws, bytes, s);
    });
}

// (logits, experts, weights, dweights, dlogits, norm, stream)
PyObject *route_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat X, D;
    int type, norm;
    at::ScalarType t;
    int64_t T, k;
    void *e, *w, *dw, *s;
    if (n != 7 || !known_type(a[4], type, t) || !matrix(a[4], t, D) || !integer(a[5], norm) || !shape2(a[1], T, k) || T != D.rows ||
        !values(a[1], at::kInt, T * k, e) || !values(a[2], at::kFloat, T * k, w) || !values(a[3], at::kFloat, T * k, dw))
        return not_here();
    X.p = nullptr;
    X.ld = D.cols;
    if (!norm && a[0] != Py_None && (!matrix(a[0], t, X) || X.rows != D.rows || X.cols != D.cols)) return not_here();
    if (!stream_handle(a[6], s)) return not_here();
    return status([&] {
        return amulet_route_grad(type, T, D.cols, k, X.p, X.ld, norm, (const int32_t *)e, (const float *)w, (const float *)dw, D.p, D.ld, s);
    });
}

// (Y, weights, place, R, stream)
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat Y, R;
    int type;
    at::ScalarType t;
    int64_t T, k;
    void *w, *p, *s;
    if (n != 5 || !known_type(a[3], type, t) || !matrix(a[3], t, R) || !matrix(a[0], t, Y) || Y.cols != R.cols || !shape2(a[2], T, k) || T != R.rows ||
        !values_or_none(a[1], at::kFloat, T * k, w) || !values(a[2], at::kInt, T * k, p) || !stream_handle(a[4], s))
        return not_here();
    return status([&] { return amulet_combine(type, T, k, R.cols, Y.rows, Y.p, Y.ld, (const float *)w, (const int32_t *)p, R.p, R.ld, s); });
}

// (Y, weights, place, dR, dY, dweights, stream)
PyObject *combine_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat Y, D, dY;
    int type;
    at::ScalarType t;
    int64_t T, k;
    void *w, *p, *dw, *s;
    if (n != 7 || !known_type(a[3], type, t) || !matrix(a[3], t, D) || !matrix(a[4], t, dY) || dY.cols != D.cols || !shape2(a[2], T, k) || T != D.rows ||
        !values_or_none(a[1], at::kFloat, T * k, w) || !values(a[2], at::kInt, T * k, p) || !values_or_none(a[5], at::kFloat, T * k, dw))
        return not_here();
    Y.p = nullptr;
    Y.ld = D.cols;
    if (dw && (!matrix(a[0], t, Y) || Y.rows != dY.rows || Y.cols != dY.cols)) return not_here();
    if (a[5] != Py_None && !dw) return not_here();
    if (!stream_handle(a[6], s)) return not_here();
    return status([&] {
        return amulet_combine_grad(type, T, k, D.cols, dY.rows, Y.p, Y.ld, (const float *)w, (const int32_t *)p, D.p, D.ld, dY.p, dY.ld, (float *)dw, s);
    });
}

// (A, B, offsets, R, rows, trans_b, stream)
PyObject *grouped_mm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, R;
    Groups B;
    int type, out, tb;
    at::ScalarType t, tr;
    void *off, *rows, *s;
    if (n != 7 || !known_type(a[0], type, t) || !matrix(a[0], t, A) || !groups(a[1], t, B) || !known_type(a[3], out, tr) || !matrix(a[3], tr, R) ||
        !integer(a[5], tb) || (tb ? B.cols : B.rows) != A.cols || (tb ? B.rows : B.cols) != R.cols || !values_or_none(a[4], at::kInt, R.rows, rows) ||
        (a[4] == Py_None && A.rows != R.rows) || (a[4] != Py_None && !rows) || !values(a[2], at::kInt, B.n + 1, off) || !stream_handle(a[6], s))
        return not_here();
    return status([&] {
        return amulet_grouped_mm(type, out, tb, R.rows, R.cols, A.cols, B.n, A.p, A.ld, (const int32_t *)rows, A.rows, B.p, B.ld, B.apart,
                                 (const int32_t *)off, R.p, R.ld, s);
    });
}

// (A, D, offsets, R, workspace, rows, trans_r, stream)
PyObject *grouped_mm_wgrad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, D;
    Groups R;
    int type, out, tr;
    at::ScalarType t, to;
    void *off, *rows, *ws, *s;
    size_t bytes;
    if (n != 8 || !known_type(a[0], type, t) || !matrix(a[0], t, A) || !matrix(a[1], t, D) || !known_type(a[3], out, to) || !groups(a[3], to, R) ||
        !bytes_or_none(a[4], ws, bytes) || !integer(a[6], tr) || (tr ? R.cols : R.rows) != A.cols || (tr ? R.rows : R.cols) != D.cols ||
        !values_or_none(a[5], at::kInt, D.rows, rows) || (a[5] == Py_None && A.rows != D.rows) || (a[5] != Py_None && !rows) ||
        !values(a[2], at::kInt, R.n + 1, off) || !stream_handle(a[7], s))
        return not_here();
    return status([&] {
        return amulet_grouped_mm_wgrad(type, out, tr, D.rows, D.cols, A.cols, R.n, A.p, A.ld, (const int32_t *)rows, A.rows, D.p, D.ld,
                                       (const int32_t *)off, R.p, R.ld, R.apart, ws, bytes, s);
    });
}

// (X, Q, scales, stream)
PyObject *quantize_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat X, Q, S;
    int type;
    at::ScalarType t;
    void *s;
    if (n != 4 || !known_type(a[0], type, t) || !matrix(a[0], t, X) || !matrix(a[1], at::kFloat8_e4m3fn, Q) || !matrix(a[2], at::kFloat, S) ||
        Q.rows != X.rows || Q.cols != X.cols || S.rows != blocks128(X.cols) || S.cols != X.rows || !stream_handle(a[3], s))
        return not_here();
    return status([&] { return amulet_quantize_fp8(type, X.rows, X.cols, X.p, X.ld, Q.p, Q.ld, (float *)S.p, S.ld, s); });
}

// (X, Q, scales, stream)
PyObject *quantize_fp8_blocks(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Groups X, Q, S;
    int type;
    at::ScalarType t;
    void *s;
    if (n != 4 || !known_type(a[0], type, t) || !groups(a[0], t, X) || !groups(a[1], at::kFloat8_e4m3fn, Q) || !groups(a[2], at::kFloat, S) ||
        Q.n != X.n || Q.rows != X.rows || Q.cols != X.cols || S.n != X.n || S.rows != blocks128(X.rows) || S.cols != blocks128(X.cols) || !stream_handle(a[3], s))
        return not_here();
    return status([&] {
        return amulet_quantize_fp8_blocks(type, X.n, X.rows, X.cols, X.p, X.ld, X.apart, Q.p, Q.ld, Q.apart, (float *)S.p, S.ld, S.apart, s);
    });
}

// (A, scales_a, B, scales_b, offsets, R, rows, trans_b, stream)
PyObject *grouped_mm_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, SA, R;
    Groups B, SB;
    int out, tb;
    at::ScalarType tr;
    void *off, *rows, *s;
    if (n != 9 || !matrix(a[0], at::kFloat8_e4m3fn, A) || !matrix(a[1], at::kFloat, SA) || !groups(a[2], at::kFloat8_e4m3fn, B) || !groups(a[3], at::kFloat, SB) ||
        !known_type(a[5], out, tr) || !matrix(a[5], tr, R) || !integer(a[7], tb) || (tb ? B.cols : B.rows) != A.cols || (tb ? B.rows : B.cols) != R.cols ||
        SA.rows != blocks128(A.cols) || SA.cols != A.rows || SB.n != B.n || SB.rows != blocks128(B.rows) || SB.cols != blocks128(B.cols) ||
        !values_or_none(a[6], at::kInt, R.rows, rows) || (a[6] == Py_None && A.rows != R.rows) || (a[6] != Py_None && !rows) ||
        !values(a[4], at::kInt, B.n + 1, off) || !stream_handle(a[8], s))
        return not_here();
    return status([&] {
        return amulet_grouped_mm_fp8(out, tb, R.rows, R.cols, A.cols, B.n, A.p, A.ld, (const float *)SA.p, SA.ld, (const int32_t *)rows, A.rows,
                                     B.p, B.ld, B.apart, (const float *)SB.p, SB.ld, SB.apart, (const int32_t *)off, R.p, R.ld, s);
    });
}

// (A, scales_a, B, scales_b, R, trans_b, stream)
PyObject *mm_fp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat A, SA, B, SB, R;
    int out, tb;
    at::ScalarType tr;
    void *s;
    if (n != 7 || !matrix(a[0], at::kFloat8_e4m3fn, A) || !matrix(a[1], at::kFloat, SA) || !matrix(a[2], at::kFloat8_e4m3fn, B) || !matrix(a[3], at::kFloat, SB) ||
        !known_type(a[4], out, tr) || !matrix(a[4], tr, R) || !integer(a[5], tb) || (tb ? B.cols : B.rows) != A.cols || (tb ? B.rows : B.cols) != R.cols ||
        R.rows != A.rows || SA.rows != blocks128(A.cols) || SA.cols != A.rows || SB.rows != blocks128(B.rows) || SB.cols != blocks128(B.cols) || !stream_handle(a[6], s))
        return not_here();
    return status([&] {
        return amulet_mm_fp8(out, tb, R.rows, R.cols, A.cols, A.p, A.ld, (const float *)SA.p, SA.ld, B.p, B.ld, (const float *)SB.p, SB.ld, R.p, R.ld, s);
    });
}

// ---- low-rank adapters, the gradients' norm: tensors of the current device only

bool current_device(int &d)
{
    PyObject *dev = PyObject_CallNoArgs(g_get_device);
    if (!dev) {
        PyErr_Clear();
        return false;
    }
    const bool ok = integer(dev, d);
    Py_DECREF(dev);
    return ok;
}
bool on_device(int d, PyObject *const *a, std::initializer_list<int> which)
{
    for (int i : which) {
        if (a[i] == Py_None) continue;
        const at::Tensor *t = tensor(a[i]);
        if (!t || t->get_device() != d) return false;
    }
    return true;
}

// (X, W, A, B, offsets, T, R, adapters, scales, trans_w, trans_a, trans_b, stream)
PyObject *adapters_mm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat X, W, T, R;
    Groups A, B;
    int type, out, tw, ta, tb, d;
    at::ScalarType t, to;
    void *off, *ad, *sc, *s;
    if (n != 13 || !known_type(a[0], type, t) || !matrix(a[0], t, X) || !groups(a[2], t, A) || !groups(a[3], t, B) || !matrix(a[5], at::kFloat, T) ||
        !known_type(a[6], out, to) || !matrix(a[6], to, R) || !integer(a[9], tw) || !integer(a[10], ta) || !integer(a[11], tb))
        return not_here();
    W.p = nullptr;
    W.ld = 1;
    if (a[1] != Py_None && (!matrix(a[1], t, W) || (tw ? W.cols : W.rows) != X.cols || (tw ? W.rows : W.cols) != R.cols || !W.p)) return not_here();
    const int64_t r = T.cols;
    if (A.n != B.n || T.rows != X.rows || R.rows != X.rows || (ta ? A.cols : A.rows) != X.cols || (ta ? A.rows : A.cols) != r ||
        (tb ? B.cols : B.rows) != r || (tb ? B.rows : B.cols) != R.cols)
        return not_here();
    int64_t S = A.n;
    if (a[7] != Py_None) {
        const at::Tensor *x = tensor(a[7]);
        if (!x || !x->defined()) return not_here();
        S = x->numel();
    }
    if (!values_or_none(a[7], at::kInt, S, ad) || (a[7] != Py_None && !ad) || !values_or_none(a[8], at::kFloat, A.n, sc) || !values(a[4], at::kInt, S + 1, off) ||
        !current_device(d) || !on_device(d, a, {0, 1, 2, 3, 4, 5, 6, 7, 8}) || !stream_handle(a[12], s))
        return not_here();
    return status([&] {
        return amulet_adapters_mm(type, out, tw, ta, tb, X.rows, R.cols, X.cols, r, S, A.n, X.p, X.ld, W.p, W.ld, A.p, A.ld, A.apart, B.p, B.ld, B.apart,
                                  (const int32_t *)off, (const int32_t *)ad, (const float *)sc, (float *)T.p, T.ld, R.p, R.ld, s);
    });
}

// (X, T, offsets, R, workspace, adapters, trans_r, stream)
PyObject *adapters_wgrad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Mat X, T;
    Groups R;
    int type, out, tr, d;
    at::ScalarType t, to;
    void *off, *ad, *ws, *s;
    size_t bytes;
    if (n != 8 || !known_type(a[0], type, t) || !matrix(a[0], t, X) || !matrix(a[1], at::kFloat, T) || !known_type(a[3], out, to) || !groups(a[3], to, R) ||
        !bytes_or_none(a[4], ws, bytes) || !integer(a[6], tr) || T.rows != X.rows || (tr ? R.cols : R.rows) != X.cols || (tr ? R.rows : R.cols) != T.cols)
        return not_here();
    int64_t S = R.n;
    if (a[5] != Py_None) {
        const at::Tensor *x = tensor(a[5]);
        if (!x || !x->defined()) return not_here();
        S = x->numel();
    }
    if (!values_or_none(a[5], at::kInt, S, ad) || (a[5] != Py_None && !ad) || !values(a[2], at::kInt, S + 1, off) || !current_device(d) ||
        !on_device(d, a, {0, 1, 2, 3, 4, 5}) || !stream_handle(a[7], s))
        return not_here();
    return status([&] {
        return amulet_adapters_wgrad(type, out, tr, X.rows, X.cols, T.cols, S, R.n, X.p, X.ld, (const float *)T.p, T.ld, (const int32_t *)off, (const int32_t *)ad,
                                     R.p, R.ld, R.apart, ws, bytes, s);
    });
}

// The arrays that the calls take of a list of tensors (and of those they are written to, Py_None: in place)
struct Tensors {
    std::vector<int32_t> types;
    std::vector<int64_t> counts;
    std::vector<void *> in, out;

    bool read(PyObject *grads, PyObject *outs, int device)
    {
        if (!PyList_CheckExact(grads) || (outs != Py_None && !PyList_CheckExact(outs))) return false;
        const Py_ssize_t n = PyList_GET_SIZE(grads);
        if (outs != Py_None && PyList_GET_SIZE(outs) != n) return false;
        // (one more: no null pointers for an empty list)
        types.resize(n + 1);
        counts.resize(n + 1);
        in.resize(n + 1);
        out.resize(n + 1);
        for (Py_ssize_t i = 0; i < n; ++i) {
            const at::Tensor *t = dense(PyList_GET_ITEM(grads, i), device);
            if (!t) return false;
            const at::ScalarType type = t->scalar_type();
            types[i] = type == at::kFloat ? AMULET_FP32 : type == at::kBFloat16 ? AMULET_BF16 : AMULET_FP16;
            counts[i] = t->numel();
            in[i] = t->data_ptr();
            if (outs == Py_None) continue;
            const at::Tensor *o = dense(PyList_GET_ITEM(outs, i), device);
            if (!o || o->scalar_type() != type || o->sizes() != t->sizes() || (counts[i] > 0 && o->strides() != t->strides())) return false;
            out[i] = o->data_ptr();
        }
        return true;
    }
    static const at::Tensor *dense(PyObject *o, int device)
    {
        const at::Tensor *t = tensor(o);
        if (!t && PyObject_TypeCheck(o, (PyTypeObject *)THPVariableClass)) t = &THPVariable_Unpack(o);   // (parameters)
        if (!t || !t->defined() || !t->is_cuda() || t->layout() != at::kStrided || !t->has_storage() || t->get_device() != device) return nullptr;
        const at::ScalarType type = t->scalar_type();
        if (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf) return nullptr;
        return t->numel() == 0 || t->is_non_overlapping_and_dense() ? t : nullptr;
    }
};
bool number(PyObject *o, float &x)
{
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    x = (float)v;
    return true;
}

// (grads, norm, workspace, stream)
PyObject *grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        Tensors t;
        int d;
        void *norm, *ws, *s;
        size_t bytes;
        if (n != 4 || !current_device(d) || !t.read(a[0], Py_None, d) || !values(a[1], at::kFloat, 1, norm) || !bytes_or_none(a[2], ws, bytes) ||
            !on_device(d, a, {1, 2}) || !stream_handle(a[3], s))
            return not_here();
        return status([&] { return amulet_grad_norm((int64_t)t.types.size() - 1, t.types.data(), t.counts.data(), t.in.data(), (float *)norm, ws, bytes, s); });
    } catch (const std::exception &) {
        return not_here();
    }
}

// (grads, max_norm, norm, outs, stream)
PyObject *grad_clip(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        Tensors t;
        int d;
        float most;
        void *norm, *s;
        if (n != 5 || !current_device(d) || !t.read(a[0], a[3], d) || !number(a[1], most) || !values(a[2], at::kFloat, 1, norm) || !on_device(d, a, {2}) ||
            !stream_handle(a[4], s))
            return not_here();
        void *const *const out = a[3] == Py_None ? nullptr : t.out.data();
        return status([&] { return amulet_grad_clip((int64_t)t.types.size() - 1, t.types.data(), t.counts.data(), t.in.data(), out, most, (const float *)norm, s); });
    } catch (const std::exception &) {
        return not_here();
    }
}

// (grads, max_norm, norm, workspace, outs, stream)
PyObject *grad_norm_clip(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        Tensors t;
        int d;
        float most;
        void *norm, *ws, *s;
        size_t bytes;
        if (n != 6 || !current_device(d) || !t.read(a[0], a[4], d) || !number(a[1], most) || !values(a[2], at::kFloat, 1, norm) || !bytes_or_none(a[3], ws, bytes) ||
            !on_device(d, a, {2, 3}) || !stream_handle(a[5], s))
            return not_here();
        void *const *const out = a[4] == Py_None ? nullptr : t.out.data();
        return status([&] {
            return amulet_grad_norm_clip((int64_t)t.types.size() - 1, t.types.data(), t.counts.data(), t.in.data(), out, most, (float *)norm, ws, bytes, s);
        });
    } catch (const std::exception &) {
        return not_here();
    }
}

#define MARSHAL(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MARSHAL(mmlike_f32),      MARSHAL(mmlike_f32_general), MARSHAL(mmlike_f64), MARSHAL(count_i8),
                         MARSHAL(count_i8_assign), MARSHAL(count_i8_general),   MARSHAL(route),      MARSHAL(route_grad),
                         MARSHAL(combine),         MARSHAL(combine_grad),       MARSHAL(grouped_mm), MARSHAL(grouped_mm_wgrad),
                         MARSHAL(quantize_fp8),    MARSHAL(quantize_fp8_blocks), MARSHAL(grouped_mm_fp8), MARSHAL(mm_fp8),
                         MARSHAL(adapters_mm),     MARSHAL(adapters_wgrad),     MARSHAL(grad_norm),  MARSHAL(grad_clip),
                         MARSHAL(grad_norm_clip),  {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject *c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_raw_stream = g_get_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(c);
    if (!g_raw_stream) {   // a torch without them: the binding does without this module
        PyErr_SetString(PyExc_ImportError, "torch has no raw stream handles");
        return nullptr;
    }
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for_torch", BUILT_FOR_TORCH) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
