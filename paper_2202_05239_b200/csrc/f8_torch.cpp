// The binding's calls on real-valued tensors: checks torch tensors against each other, fills the descriptor and calls the entry point of
// the same name.  Reading shapes, strides and pointers here instead of through Python attributes and ctypes takes 1 us of a
// call instead of 5 to 7, which is what bounds a call on one token.
#include <Python.h>

#include <stdio.h>
#include <string.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/f8net.h"

namespace {

struct Refused {};           // a Python error is set

[[noreturn]] void refuse(const char *what, const char *why) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
    throw Refused();
}

enum : unsigned { U8 = 1, S8 = 2, S32 = 4, REAL = 8, F32 = 16, I64 = 32 };

// The library's code of a tensor's type, if `types` has it; -1 for int64.
int dtype_of(const at::Tensor &t, unsigned types, const char *what) {
    switch (t.scalar_type()) {
        case at::kByte: if (types & U8) return F8_U8; break;
        case at::kChar: if (types & S8) return F8_S8; break;
        case at::kInt: if (types & S32) return F8_S32; break;
        case at::kLong: if (types & I64) return -1; break;
        case at::kFloat: if (types & (REAL | F32)) return F8_F32; break;
        case at::kHalf: if (types & REAL) return F8_F16; break;
        case at::kBFloat16: if (types & REAL) return F8_BF16; break;
        default: break;
    }
    refuse(what, "a tensor of another type is needed");
}

// What the tensors of one call have in common: the device, which has to be the current one.
struct Call {
    int device = -1;
    const at::Tensor *tensor(PyObject *o, const char *what, bool optional) {
        if (o == Py_None) {
            if (optional) return nullptr;
            refuse(what, "a tensor is needed");
        }
        if (!THPVariable_Check(o)) refuse(what, "a tensor is needed");
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) refuse(what, "a tensor on the current CUDA device is needed");
        if (device < 0) device = c10::cuda::current_device();
        if (t.get_device() != device) refuse(what, "a tensor on the current CUDA device is needed");
        return &t;
    }
    cudaStream_t stream(PyObject *o) {
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
        PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
        if (!h) throw Refused();
        void *s = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!s && PyErr_Occurred()) throw Refused();
        return (cudaStream_t)s;
    }
};

// A matrix with unit stride along its rows, which do not overlap.
struct Matrix {
    void *p = nullptr;
    long long rows = 0, cols = 0, ld = 0;
    int dtype = 0;
    bool given = false;         // (a tensor without elements may have no memory)
    Matrix() {}
    Matrix(Call &c, PyObject *o, const char *what, unsigned types, bool optional = false) {
        const at::Tensor *t = c.tensor(o, what, optional);
        if (!t) return;
        given = true;
        dtype = dtype_of(*t, types, what);
        if (t->dim() != 2) refuse(what, "a matrix is needed");
        rows = t->size(0);
        cols = t->size(1);
        if (rows > 0x7fffffffll || cols > 0x7fffffffll) refuse(what, "extents beyond 2^31 - 1");
        ld = t->stride(0);
        if ((t->stride(1) != 1 && cols > 1) || (ld < cols && rows > 1)) refuse(what, "rows with unit stride that do not overlap are needed");
        if (rows <= 1 && ld < cols) ld = cols;
        p = const_cast<void *>(t->const_data_ptr());
    }
    void shaped(long long r, long long c, const char *what) const {
        if (given && (rows != r || cols != c)) refuse(what, "its shape does not fit the other tensors'");
    }
    void typed(int d, const char *what) const {
        if (given && dtype != d) refuse(what, "its type is not the other tensors'");
    }
};

// A dense tensor of `n` elements (or, where `one`, of a single one).
struct Vector {
    void *p = nullptr;
    long long n = 0;
    int dtype = 0;
    Vector(Call &c, PyObject *o, const char *what, unsigned types, long long count, bool one = false, bool optional = true) {
        const at::Tensor *t = c.tensor(o, what, optional);
        if (!t) return;
        dtype = dtype_of(*t, types, what);
        n = t->numel();
        if (n != count && !(one && n == 1)) refuse(what, "its number of elements does not fit the other tensors'");
        if (!t->is_contiguous()) refuse(what, "a dense tensor is needed");
        p = const_cast<void *>(t->const_data_ptr());
    }
};

long long integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
int small(PyObject *o) {
    const long long v = integer(o);
    if (v < -0x7fffffffll || v > 0x7fffffffll) refuse("argument", "an integer is too large");
    return (int)v;
}
float real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return (float)v;
}

// Lets other Python threads run, as a call through ctypes does: a launch waits where the queue of launches is full.
struct OthersRun {
    PyThreadState *state = PyEval_SaveThread();
    ~OthersRun() { PyEval_RestoreThread(state); }
};

template <typename F>
PyObject *guarded(Py_ssize_t got, Py_ssize_t want, F f) {
    if (got != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)f());
    } catch (const Refused &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// x, x_scale, w, w_scale, y, bias, stream
PyObject *linear_scaled(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 7, [&] {
        Call c;
        const Matrix x(c, a[0], "x", U8 | S8), w(c, a[2], "w", S8), y(c, a[4], "y", REAL);
        if (w.cols != x.cols) refuse("w", "its rows are not as long as x's");
        y.shaped(x.rows, w.rows, "y");
        const Vector xs(c, a[1], "x_scale", F32, x.rows, true, false), ws(c, a[3], "w_scale", F32, w.rows, true, false), b(c, a[5], "bias", REAL, w.rows);
        f8_scaled_desc d = {(int)x.rows, (int)x.cols, (int)w.rows, x.dtype, y.dtype, b.p ? b.dtype : F8_F32, (int)xs.n, (int)ws.n, x.ld, w.ld, y.ld};
        const cudaStream_t stream = c.stream(a[6]);
        const OthersRun others;
        return f8_linear_scaled(&d, x.p, (const float *)xs.p, (const int8_t *)w.p, (const float *)ws.p, b.p, y.p, stream);
    });
}

// x, q, scale, y, u, act, stream
PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 7, [&] {
        Call c;
        const Matrix x(c, a[0], "x", REAL), q(c, a[1], "q", S8, true), y(c, a[3], "y", REAL, true), u(c, a[4], "u", REAL, true);
        q.shaped(x.rows, x.cols, "q");
        y.shaped(x.rows, x.cols, "y");
        u.shaped(x.rows, x.cols, "u");
        y.typed(x.dtype, "y");
        u.typed(x.dtype, "u");
        const Vector s(c, a[2], "scale", F32, x.rows);
        f8_rows_desc d = {x.rows, (int)x.cols, x.dtype, small(a[5]), x.ld, u.ld, y.ld, q.ld};
        const cudaStream_t stream = c.stream(a[6]);
        const OthersRun others;
        return f8_quantize_rows(&d, x.p, u.p, (int8_t *)q.p, (float *)s.p, y.p, stream);
    });
}

// x, q, scale, y, residual, residual_out, gate, gate_act, post_norm, post_w, post_b, pre_norm, pre_w, pre_b, eps, weight_offset, branch_scale, stream
PyObject *norm_quantize(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 18, [&] {
        Call c;
        const Matrix x(c, a[0], "x", REAL), q(c, a[1], "q", S8, true), y(c, a[3], "y", REAL, true), r(c, a[4], "residual", REAL, true);
        const Matrix sum(c, a[5], "residual_out", REAL, true), g(c, a[6], "gate", REAL, true);
        q.shaped(x.rows, x.cols, "q");
        y.shaped(x.rows, x.cols, "y");
        r.shaped(x.rows, x.cols, "residual");
        sum.shaped(x.rows, x.cols, "residual_out");
        g.shaped(g.rows == 1 ? 1 : x.rows, x.cols, "gate");
        y.typed(x.dtype, "y");
        r.typed(x.dtype, "residual");
        sum.typed(x.dtype, "residual_out");
        g.typed(x.dtype, "gate");
        const Vector s(c, a[2], "scale", F32, x.rows), post_w(c, a[9], "post_w", REAL, x.cols), post_b(c, a[10], "post_b", REAL, x.cols);
        const Vector pre_w(c, a[12], "pre_w", REAL, x.cols), pre_b(c, a[13], "pre_b", REAL, x.cols);
        int wt = -1;
        for (const Vector *v : {&post_w, &post_b, &pre_w, &pre_b}) {
            if (!v->p) continue;
            if (wt >= 0 && v->dtype != wt) refuse("norm weights", "they are of different types");
            wt = v->dtype;
        }
        f8_norm_desc d = {x.rows, (int)x.cols, x.dtype, wt >= 0 ? wt : F8_F32, small(a[8]), small(a[11]), small(a[7]), g.p ? g.rows : 1,
                          real(a[14]), real(a[15]), real(a[16]), x.ld, g.ld, r.ld, sum.ld, y.ld, q.ld};
        const cudaStream_t stream = c.stream(a[17]);
        const OthersRun others;
        return f8_norm_quantize(&d, x.p, g.p, r.p, post_w.p, post_b.p, pre_w.p, pre_b.p, sum.p, (int8_t *)q.p, (float *)s.p, y.p, stream);
    });
}

// logits, tokens, logprobs, entropy, top_logprobs, top_ids, fl, inv_temperature, stream
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 9, [&] {
        Call c;
        const Matrix l(c, a[0], "logits", S32 | REAL);
        auto per_row = [&](int i, const char *what) -> long long {       // elements of each row's part of a tensor
            const at::Tensor *t = c.tensor(a[i], what, true);
            if (!t) return 0;
            if (l.rows == 0) return t->dim() == 2 ? t->size(1) : 0;
            if (t->numel() % l.rows) refuse(what, "its number of elements does not fit the other tensors'");
            return t->numel() / l.rows;
        };
        const long long tokens = per_row(1, "tokens"), top = std::max(per_row(4, "top_logprobs"), per_row(5, "top_ids"));
        if (tokens > 0x7fffffffll || top > 0x7fffffffll) refuse("tokens", "extents beyond 2^31 - 1");
        const Vector ids(c, a[1], "tokens", I64, l.rows * tokens), lp(c, a[2], "logprobs", F32, l.rows * tokens), h(c, a[3], "entropy", F32, l.rows);
        const Vector tl(c, a[4], "top_logprobs", F32, l.rows * top), ti(c, a[5], "top_ids", I64, l.rows * top);
        f8_logprobs_desc d = {l.rows, (int)l.cols, l.dtype, small(a[6]), (int)tokens, (int)top, real(a[7]), l.ld};
        const cudaStream_t stream = c.stream(a[8]);
        const OthersRun others;
        return f8_token_logprobs(&d, l.p, (const int64_t *)ids.p, (float *)lp.p, (float *)h.p, (float *)tl.p, (int64_t *)ti.p, stream);
    });
}

PyMethodDef methods[] = {{"linear_scaled", (PyCFunction)(void (*)())linear_scaled, METH_FASTCALL, nullptr},
                         {"quantize_rows", (PyCFunction)(void (*)())quantize_rows, METH_FASTCALL, nullptr},
                         {"norm_quantize", (PyCFunction)(void (*)())norm_quantize, METH_FASTCALL, nullptr},
                         {"token_logprobs", (PyCFunction)(void (*)())token_logprobs, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
// (the text by which the build knows whether the module was made for the Python and the torch at hand)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_f8torch", "Calls on torch tensors, " F8_MADE_FOR, -1, methods, nullptr, nullptr, nullptr, nullptr};

}   // namespace

PyMODINIT_FUNC PyInit__f8torch(void) { return PyModule_Create(&module); }
