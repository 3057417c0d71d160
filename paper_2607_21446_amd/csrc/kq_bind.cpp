// Native argument marshalling of the Python binding for the calls a serving or
// calibration loop repeats.  Each function takes the Python call's arguments and
// either makes the library call and returns its result, or returns None when an
// argument is not of the plain form checked here (another type, device, layout,
// size or stream object, a tensor without storage) or the library refuses the call:
// binding.py then runs its own checks and raises what they say.  A call that fails
// after that (KQ_ERROR_HIP) may have been enqueued, so it is not made again: its
// error is raised here.  A small call's time is the host's: 9.5 us through Python
// checks and ctypes for a kernel of 2.8.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

#include <algorithm>
#include <cmath>

#include "kroquant.h"

namespace {

constexpr int64_t kPackBytes = KQ_PACK_BYTES_PER_FACTOR;

// A plain torch.Tensor (or Parameter), not a subclass; null otherwise.
const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool dense(const at::Tensor* t, at::ScalarType dtype) {
    return t && t->scalar_type() == dtype && t->is_cuda() && t->is_contiguous();
}
bool matrix(const at::Tensor* t, at::ScalarType dtype) { return dense(t, dtype) && t->dim() == 2; }
// A contiguous tensor of exactly n elements on dev.
bool buffer(const at::Tensor* t, at::ScalarType dtype, int64_t n, at::Device dev) {
    return dense(t, dtype) && t->numel() == n && t->device() == dev;
}

bool stream_of(PyObject* o, void** st) {
    if (o == Py_None) {
        *st = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    *st = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

bool flag(PyObject* o, bool* v) {
    if (!PyBool_Check(o)) return false;
    *v = o == Py_True;
    return true;
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dtype, at::Device dev) {
    return at::empty(shape, at::TensorOptions().dtype(dtype).device(dev));
}

// An output: the caller's buffer, a new one, or (optional and not wanted) none.
struct Out {
    PyObject* given = nullptr;  // borrowed
    at::Tensor made;
    void* ptr = nullptr;
    PyObject* take() {  // new reference
        if (given) {
            Py_INCREF(given);
            return given;
        }
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_RETURN_NONE;
    }
};

bool output(PyObject* o, bool want, at::IntArrayRef shape, at::ScalarType dtype, int64_t n, at::Device dev, Out& out) {
    if (o != Py_None) {
        const at::Tensor* t = tensor(o);
        if (!buffer(t, dtype, n, dev)) return false;
        out.given = o;
        out.ptr = t->data_ptr();
    } else if (want) {
        out.made = empty(shape, dtype, dev);
        out.ptr = out.made.data_ptr();
    }
    return true;
}

// A call that the HIP runtime reported an error of.
struct Failed {
    kq_status status;
    const char* name;
};

// True if the call was made, false if the library refused its arguments.
template <class F>
bool call(const char* name, F f) {
    kq_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f();
    Py_END_ALLOW_THREADS;
    if (st == KQ_ERROR_HIP) throw Failed{st, name};
    return st == KQ_SUCCESS;
}

// Sets the binding's KQError.
PyObject* raise(const Failed& e) {
    PyObject* const m = PyImport_ImportModule("paper_2607_21446_amd.binding");
    PyObject* const cls = m ? PyObject_GetAttrString(m, "KQError") : nullptr;
    PyObject* const err = cls ? PyObject_CallFunction(cls, "iss", (int)e.status, kq_last_error_detail(), e.name) : nullptr;
    if (err) PyErr_SetObject(cls, err);
    Py_XDECREF(err);
    Py_XDECREF(cls);
    Py_XDECREF(m);
    return nullptr;
}

// Everything a function does runs in here: an exception of a tensor call means an
// argument that Python shall deal with.
template <class F>
PyObject* guarded(F f) {
    try {
        PyObject* r = f();
        if (r) return r;
    } catch (const Failed& e) {
        return raise(e);
    } catch (...) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

struct Quant {
    const at::Tensor* X;
    int64_t M, d;
    Out codes, scales, y;
    void* stream;
    // X, and the outputs' and stream arguments
    bool parse(PyObject* x, PyObject* c, PyObject* s, PyObject* yo, PyObject* want_y, PyObject* st) {
        X = tensor(x);
        if (!matrix(X, at::kBFloat16)) return false;
        M = X->size(0);
        d = X->size(1);
        const at::Device dev = X->device();
        bool want = false;
        if (want_y && !flag(want_y, &want)) return false;
        return stream_of(st, &stream) && output(c, true, {M, d / 2}, at::kByte, M * (d / 2), dev, codes) &&
               output(s, true, {M, d / 32}, at::kByte, M * (d / 32), dev, scales) &&
               (!yo || output(yo, want, {M, d}, at::kFloat, M * d, dev, y));
    }
    const uint16_t* x() const { return static_cast<const uint16_t*>(X->data_ptr()); }
    uint8_t* c() const { return static_cast<uint8_t*>(codes.ptr); }
    uint8_t* s() const { return static_cast<uint8_t*>(scales.ptr); }
    float* yp() const { return static_cast<float*>(y.ptr); }
    PyObject* result(bool with_y, Out* more = nullptr) {
        const int n = 2 + (with_y ? 1 : 0) + (more ? 1 : 0);
        PyObject* t = PyTuple_New(n);
        if (!t) return nullptr;
        PyTuple_SET_ITEM(t, 0, codes.take());
        PyTuple_SET_ITEM(t, 1, scales.take());
        if (with_y) PyTuple_SET_ITEM(t, 2, y.take());
        if (more) PyTuple_SET_ITEM(t, n - 1, more->take());
        return t;
    }
};

struct Pairs {
    const float *A, *B;
    int64_t a, b, nfac;
    bool parse(PyObject* pa, PyObject* pb, at::Device dev) {
        const at::Tensor *ta = tensor(pa), *tb = tensor(pb);
        if (!dense(ta, at::kFloat) || !dense(tb, at::kFloat) || ta->device() != dev || tb->device() != dev) return false;
        if (ta->dim() < 2 || tb->dim() < 2) return false;
        a = ta->size(-1);
        b = tb->size(-1);
        if (ta->size(-2) != a || tb->size(-2) != b || a < 1 || a > 32 || b < 1 || b > 32) return false;
        nfac = ta->numel() / (a * a);
        A = static_cast<const float*>(ta->data_ptr());
        B = static_cast<const float*>(tb->data_ptr());
        return tb->numel() == nfac * b * b;
    }
};

// (X, A, B, codes, scales, y, want_y, stream)
template <class F>
PyObject* kron(const char* name, PyObject* const* v, Py_ssize_t n, F f) {
    if (n != 8) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        Pairs p;
        if (!q.parse(v[0], v[3], v[4], v[5], v[6], v[7]) || !p.parse(v[1], v[2], q.X->device())) return nullptr;
        if (!call(name, [&] {
                return f(q.x(), q.M, q.d, p.A, p.B, (int)p.a, (int)p.b, p.nfac, q.c(), q.s(), q.yp(), q.stream);
            }))
            return nullptr;
        return q.result(true);
    });
}

PyObject* quantize(PyObject*, PyObject* const* v, Py_ssize_t n) { return kron("kq_quantize", v, n, kq_quantize); }
PyObject* quantize_exact(PyObject*, PyObject* const* v, Py_ssize_t n) { return kron("kq_quantize_exact", v, n, kq_quantize_exact); }

// (X, A, B, kpack, codes, scales, y, want_y, stream)
PyObject* quantize_packed(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        Pairs p;
        if (!q.parse(v[0], v[4], v[5], v[6], v[7], v[8]) || !p.parse(v[1], v[2], q.X->device())) return nullptr;
        const at::Tensor* k = tensor(v[3]);
        if (!buffer(k, at::kByte, p.nfac * kPackBytes, q.X->device())) return nullptr;
        if (!call("kq_quantize_packed", [&] {
                return kq_quantize_packed(q.x(), q.M, q.d, p.A, p.B, (int)p.a, (int)p.b, p.nfac, k->data_ptr(), q.c(),
                                          q.s(), q.yp(), q.stream);
            }))
            return nullptr;
        return q.result(true);
    });
}

// (X, lu, a, codes, scales, y, y16, want_y, want_y16, stream)
PyObject* quantize_lu(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 10) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        Out y16;
        bool want16 = false;
        if (!q.parse(v[0], v[3], v[4], v[5], v[7], v[9]) || !flag(v[8], &want16) || !PyLong_CheckExact(v[2])) return nullptr;
        const long a = PyLong_AsLong(v[2]);
        const at::Tensor* lu = tensor(v[1]);
        if (a < 1 || a > 32 || !dense(lu, at::kFloat) || lu->device() != q.X->device()) return nullptr;
        if (lu->numel() == 0 || lu->numel() % 15) return nullptr;
        if (!output(v[6], want16, {q.M, q.d}, at::kBFloat16, q.M * q.d, q.X->device(), y16)) return nullptr;
        if (!call("kq_quantize_lu", [&] {
                return kq_quantize_lu(q.x(), q.M, q.d, static_cast<const float*>(lu->data_ptr()), (int)a,
                                      lu->numel() / 15, q.c(), q.s(), q.yp(), static_cast<uint16_t*>(y16.ptr), q.stream);
            }))
            return nullptr;
        return q.result(true, &y16);
    });
}

// (X, mult, codes, scales, y, want_y, stream)
PyObject* smoothquant(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 7) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        if (!q.parse(v[0], v[2], v[3], v[4], v[5], v[6])) return nullptr;
        const at::Tensor* m = tensor(v[1]);
        if (!buffer(m, at::kFloat, q.d, q.X->device())) return nullptr;
        if (!call("kq_smoothquant_quantize", [&] {
                return kq_smoothquant_quantize(q.x(), q.M, q.d, static_cast<const float*>(m->data_ptr()), q.c(), q.s(),
                                               q.yp(), q.stream);
            }))
            return nullptr;
        return q.result(true);
    });
}

// (X, codes, scales, y, want_y, stream)
template <class F>
PyObject* plain(const char* name, PyObject* const* v, Py_ssize_t n, F f) {
    if (n != 6) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        if (!q.parse(v[0], v[1], v[2], v[3], v[4], v[5])) return nullptr;
        if (!call(name, [&] { return f(q.x(), q.M, q.d, q.c(), q.s(), q.yp(), q.stream); })) return nullptr;
        return q.result(true);
    });
}

PyObject* hadamard32(PyObject*, PyObject* const* v, Py_ssize_t n) { return plain("kq_hadamard32_quantize", v, n, kq_hadamard32_quantize); }
PyObject* fwht(PyObject*, PyObject* const* v, Py_ssize_t n) { return plain("kq_fwht_quantize", v, n, kq_fwht_quantize); }

// (X, codes, scales, stream)
PyObject* mxfp4(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 4) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Quant q;
        if (!q.parse(v[0], v[1], v[2], nullptr, nullptr, v[3])) return nullptr;
        if (!call("kq_mxfp4_quantize", [&] { return kq_mxfp4_quantize(q.x(), q.M, q.d, q.c(), q.s(), q.stream); })) return nullptr;
        return q.result(false);
    });
}

// (a_codes, a_scales, b_codes, b_scales, C, accumulate, stream, out_dtype)
PyObject* mxfp4_gemm(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 8) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        const at::Tensor* t[4];
        for (int i = 0; i < 4; ++i) {
            t[i] = tensor(v[i]);
            if (!matrix(t[i], at::kByte) || t[i]->device() != t[0]->device()) return nullptr;
        }
        const int64_t M = t[0]->size(0), N = t[2]->size(0), K = 2 * t[0]->size(1);
        if (2 * t[2]->size(1) != K || t[1]->size(0) != M || t[1]->size(1) != K / 32 || t[3]->size(0) != N ||
            t[3]->size(1) != K / 32)
            return nullptr;
        bool accumulate = false;
        void* st = nullptr;
        if (!flag(v[5], &accumulate) || !stream_of(v[6], &st)) return nullptr;
        at::ScalarType dtype = at::kFloat;
        Out C;
        if (v[4] != Py_None) {
            const at::Tensor* c = tensor(v[4]);
            if (!c || c->dim() != 2 || c->size(0) != M || c->size(1) != N) return nullptr;
            dtype = c->scalar_type();
        } else if (v[7] != Py_None) {
            if (!THPDtype_Check(v[7])) return nullptr;
            dtype = reinterpret_cast<THPDtype*>(v[7])->scalar_type;
        }
        if ((dtype != at::kFloat && dtype != at::kBFloat16) || (dtype == at::kBFloat16 && accumulate)) return nullptr;
        if (!output(v[4], true, {M, N}, dtype, M * N, t[0]->device(), C)) return nullptr;
        const int64_t ldc = (C.given ? *tensor(v[4]) : C.made).stride(0);
        const uint8_t* p[4];
        for (int i = 0; i < 4; ++i) p[i] = static_cast<const uint8_t*>(t[i]->data_ptr());
        if (!call(dtype == at::kFloat ? "kq_mxfp4_gemm" : "kq_mxfp4_gemm_bf16", [&] {
                return dtype == at::kFloat
                           ? kq_mxfp4_gemm(p[0], p[1], M, p[2], p[3], N, K, static_cast<float*>(C.ptr), ldc, accumulate, st)
                           : kq_mxfp4_gemm_bf16(p[0], p[1], M, p[2], p[3], N, K, static_cast<uint16_t*>(C.ptr), ldc, st);
            }))
            return nullptr;
        return C.take();
    });
}

// (X, W, Yneg, lu, lambdas, a, workspace, adam, grad, losses, stream); adam None only
PyObject* calib_step(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        const at::Tensor *X = tensor(v[0]), *W = tensor(v[1]), *Y = tensor(v[2]), *lu = tensor(v[3]), *lam = tensor(v[4]),
                         *ws = tensor(v[6]);
        if (!matrix(X, at::kBFloat16) || !matrix(W, at::kBFloat16) || W->device() != X->device()) return nullptr;
        const int64_t R = X->size(0), d = X->size(1), o = W->size(0);
        const at::Device dev = X->device();
        if (W->size(1) != d || !buffer(Y, at::kFloat, R * o, dev) || !dense(lu, at::kFloat) || lu->device() != dev ||
            lu->numel() == 0 || lu->numel() % 15 || !buffer(lam, at::kFloat, 2, dev) || !dense(ws, at::kByte) ||
            v[7] != Py_None || !PyLong_CheckExact(v[5]))
            return nullptr;
        const long a = PyLong_AsLong(v[5]);
        const int64_t nfac = lu->numel() / 15;
        Out grad, losses;
        void* st = nullptr;
        if (a < 1 || a > 32 || !stream_of(v[10], &st) || !output(v[8], true, {nfac, 5, 3}, at::kFloat, nfac * 15, dev, grad) ||
            !output(v[9], true, {4}, at::kDouble, 4, dev, losses))
            return nullptr;
        if (!call("kq_calib_step", [&] {
                return kq_calib_step(static_cast<const uint16_t*>(X->data_ptr()), R, d,
                                     static_cast<const uint16_t*>(W->data_ptr()), o, static_cast<const float*>(Y->data_ptr()),
                                     static_cast<float*>(lu->data_ptr()), (int)a, nfac,
                                     static_cast<const float*>(lam->data_ptr()), static_cast<float*>(grad.ptr),
                                     static_cast<double*>(losses.ptr), nullptr, nullptr, 0, 0.0f, ws->data_ptr(),
                                     (size_t)ws->numel(), st);
            }))
            return nullptr;
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, losses.take());
        PyTuple_SET_ITEM(r, 1, grad.take());
        return r;
    });
}

// fp32 or bf16, as the library's type.
bool float_type(const at::Tensor* t, int* type) {
    if (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16) return false;
    *type = t->scalar_type() == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32;
    return true;
}

bool number(PyObject* o, float* v) {
    if (!PyFloat_CheckExact(o)) return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

bool small_int(PyObject* o, int* v) {
    if (!PyLong_CheckExact(o)) return false;
    const long n = PyLong_AsLong(o);
    *v = (int)n;
    return *v == n && !(n == -1 && PyErr_Occurred());
}

bool float_dtype(PyObject* o, at::ScalarType* t) {
    if (!THPDtype_Check(o)) return false;
    *t = reinterpret_cast<THPDtype*>(o)->scalar_type;
    return *t == at::kFloat || *t == at::kBFloat16;
}

// Vectors of one type, [d] or [B, d] with contiguous rows.
struct Vectors {
    int type = -1;
    int64_t batches = -1;
    at::Device dev;
    explicit Vectors(at::Device d) : dev(d) {}
    int dtype() const { return type < 0 ? KQ_DTYPE_FP32 : type; }
    int64_t count() const { return batches < 0 ? 1 : batches; }
    bool add(PyObject* o, int64_t d, bool per_batch, const void** p, int64_t* stride) {
        *p = nullptr;
        *stride = 0;
        if (o == Py_None) return true;
        const at::Tensor* t = tensor(o);
        int ty;
        if (!t || !t->is_cuda() || t->device() != dev || !float_type(t, &ty) || (type >= 0 && ty != type)) return false;
        type = ty;
        const int64_t dim = t->dim();
        if (dim < 1 || dim > (per_batch ? 2 : 1) || t->size(dim - 1) != d || (d > 1 && t->stride(dim - 1) != 1)) return false;
        if (per_batch) {
            const int64_t n = dim == 2 ? t->size(0) : 1;
            if (batches >= 0 && n != batches) return false;
            batches = n;
            if (dim == 2) *stride = t->stride(0);
            if (*stride < 0) return false;
        }
        *p = t->data_ptr();
        return true;
    }
};

// A [rows, cols] array of the type `dtype` whose rows are contiguous: its row stride, -1 if it is none.
int64_t row_stride(const at::Tensor* t, int64_t rows, int64_t cols, at::ScalarType dtype, at::Device dev) {
    if (!t || !t->is_cuda() || t->scalar_type() != dtype || t->device() != dev || t->dim() != 2 || t->size(0) != rows ||
        t->size(1) != cols || (cols > 1 && t->stride(1) != 1) || (rows > 1 && t->stride(0) < cols))
        return -1;
    return rows > 1 ? t->stride(0) : cols;
}

// The output of a linear layer: the caller's, or a new one of out_dtype (else `dtype`).
bool linear_out(PyObject* given, PyObject* out_dtype, at::ScalarType dtype, int64_t rows, int64_t cols, at::Device dev, Out& out,
                int64_t* ldo, at::ScalarType* type) {
    *type = dtype;
    if (given != Py_None) {
        const at::Tensor* t = tensor(given);
        if (!t || (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16)) return false;
        *type = t->scalar_type();
        *ldo = row_stride(t, rows, cols, *type, dev);
        if (*ldo < 0) return false;
        out.given = given;
        out.ptr = t->data_ptr();
        return true;
    }
    if (out_dtype != Py_None && !float_dtype(out_dtype, type)) return false;
    out.made = empty({rows, cols}, *type, dev);
    out.ptr = out.made.data_ptr();
    *ldo = cols;
    return true;
}

struct Operands {
    const at::Tensor* t[4];
    int64_t M, N, K, E = 1;
    at::Device dev = at::kCPU;
    bool parse(PyObject* const* v, bool experts) {
        for (int i = 0; i < 4; ++i) {
            t[i] = tensor(v[i]);
            if (!dense(t[i], at::kByte) || t[i]->dim() != (experts && i >= 2 ? 3 : 2) || t[i]->device() != t[0]->device()) return false;
        }
        const int64_t b = experts ? 1 : 0;
        M = t[0]->size(0);
        K = 2 * t[0]->size(1);
        N = t[2]->size(b);
        if (experts) E = t[2]->size(0);
        dev = t[0]->device();
        return 2 * t[2]->size(b + 1) == K && t[1]->size(0) == M && t[1]->size(1) == K / 32 && t[3]->size(b) == N &&
               t[3]->size(b + 1) == K / 32 && (!experts || t[3]->size(0) == E);
    }
    const uint8_t* p(int i) const { return static_cast<const uint8_t*>(t[i]->data_ptr()); }
};

// (a_codes, a_scales, b_codes, b_scales, bias, act, gate, residual, out, out_dtype, stream)
PyObject* mxfp4_linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Operands o;
        int act;
        void* st = nullptr;
        if (!o.parse(v, false) || !small_int(v[5], &act) || !stream_of(v[10], &st)) return nullptr;
        const int64_t cols = act == KQ_ACT_SWIGLU ? o.N / 2 : o.N;
        if (act == KQ_ACT_SWIGLU && o.N % 2) return nullptr;
        Vectors vec(o.dev);
        const void *bias, *gate;
        int64_t none, stride;
        if (!vec.add(v[4], o.N, false, &bias, &none) || !vec.add(v[6], cols, true, &gate, &stride)) return nullptr;
        if (vec.count() <= 0 || o.M % vec.count()) return nullptr;
        at::ScalarType type = at::kBFloat16;
        const at::Tensor* res = nullptr;
        if (v[7] != Py_None) {
            res = tensor(v[7]);
            if (!res) return nullptr;
            type = res->scalar_type();
            if (type != at::kFloat && type != at::kBFloat16) return nullptr;
        }
        Out out;
        int64_t ldo, ldr = 0;
        if (!linear_out(v[8], v[9], type, o.M, cols, o.dev, out, &ldo, &type)) return nullptr;
        if (res && (ldr = row_stride(res, o.M, cols, type, o.dev)) < 0) return nullptr;
        if (!call("kq_mxfp4_linear", [&] {
                return kq_mxfp4_linear(o.p(0), o.p(1), o.M, o.p(2), o.p(3), o.N, o.K, bias, gate, stride,
                                       std::max<int64_t>(1, o.M / vec.count()), (kq_dtype)vec.dtype(), (kq_act)act,
                                       res ? res->data_ptr() : nullptr, ldr, out.ptr, ldo,
                                       type == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32, st);
            }))
            return nullptr;
        return out.take();
    });
}

// (a_codes, a_scales, b_codes, b_scales, offsets, rows, bias, act, row_scale, out, out_dtype, stream)
PyObject* mxfp4_grouped_linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 12) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Operands o;
        int act;
        void* st = nullptr;
        if (!o.parse(v, true) || !small_int(v[7], &act) || !stream_of(v[11], &st)) return nullptr;
        if (act == KQ_ACT_SWIGLU && o.N % 2) return nullptr;
        const at::Tensor* off = tensor(v[4]);
        if (!buffer(off, at::kInt, o.E + 1, o.dev)) return nullptr;
        int64_t R = o.M;
        const at::Tensor *rows = nullptr, *bias = nullptr, *scale = nullptr;
        if (v[5] != Py_None) {
            rows = tensor(v[5]);
            if (!dense(rows, at::kInt) || rows->device() != o.dev) return nullptr;
            R = rows->numel();
        }
        int vec = KQ_DTYPE_FP32;
        if (v[6] != Py_None) {
            bias = tensor(v[6]);
            if (!bias || !float_type(bias, &vec) || !dense(bias, bias->scalar_type()) || bias->device() != o.dev ||
                bias->dim() != 2 || bias->size(0) != o.E || bias->size(1) != o.N)
                return nullptr;
        }
        if (v[8] != Py_None) {
            scale = tensor(v[8]);
            if (!buffer(scale, at::kFloat, R, o.dev)) return nullptr;
        }
        Out out;
        int64_t ldo;
        at::ScalarType type;
        if (!linear_out(v[9], v[10], at::kBFloat16, R, act == KQ_ACT_SWIGLU ? o.N / 2 : o.N, o.dev, out, &ldo, &type)) return nullptr;
        if (!call("kq_mxfp4_grouped_linear", [&] {
                return kq_mxfp4_grouped_linear(o.p(0), o.p(1), o.M, rows ? static_cast<const int32_t*>(rows->data_ptr()) : nullptr,
                                               R, o.p(2), o.p(3), o.E, o.N, o.K, static_cast<const int32_t*>(off->data_ptr()),
                                               bias ? bias->data_ptr() : nullptr, (kq_dtype)vec, (kq_act)act,
                                               scale ? static_cast<const float*>(scale->data_ptr()) : nullptr, out.ptr, ldo,
                                               type == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32, st);
            }))
            return nullptr;
        return out.take();
    });
}

// A contiguous matrix as `like`, of one of the two types.
const at::Tensor* as_matrix(PyObject* o, const at::Tensor* like, int* type) {
    const at::Tensor* t = tensor(o);
    if (!t || !t->is_cuda() || !t->is_contiguous() || t->dim() != 2 || !float_type(t, type)) return nullptr;
    if (like && (t->size(0) != like->size(0) || t->size(1) != like->size(1) || t->device() != like->device())) return nullptr;
    return t;
}

// The five vectors of a norm, from v[0]: gate, post_weight, weight, scale, shift.
struct NormVectors {
    const void *gate, *post_weight, *weight, *scale, *shift;
    int64_t gs, ss, hs, none;
    Vectors vec;
    explicit NormVectors(at::Device dev) : vec(dev) {}
    bool parse(PyObject* const* v, int64_t M, int64_t d) {
        return vec.add(v[0], d, true, &gate, &gs) && vec.add(v[1], d, false, &post_weight, &none) &&
               vec.add(v[2], d, false, &weight, &none) && vec.add(v[3], d, true, &scale, &ss) &&
               vec.add(v[4], d, true, &shift, &hs) && vec.count() > 0 && M % vec.count() == 0;
    }
};

// (x, residual, gate, post_weight, weight, scale, shift, norm, post_norm, alpha, eps, h, y, h_dtype, stream)
PyObject* block_norm(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 15) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        int xt, ht, norm, post;
        float alpha, eps;
        void* st = nullptr;
        const at::Tensor* x = as_matrix(v[0], nullptr, &xt);
        if (!x || !small_int(v[7], &norm) || !small_int(v[8], &post) || !number(v[9], &alpha) || !number(v[10], &eps) ||
            !stream_of(v[14], &st) || norm == KQ_NORM_NONE)
            return nullptr;
        const int64_t M = x->size(0), d = x->size(1);
        ht = xt;
        const at::Tensor* res = nullptr;
        if (v[1] != Py_None && !(res = as_matrix(v[1], x, &ht))) return nullptr;
        if (!res && v[13] != Py_None) {
            at::ScalarType t;
            if (!float_dtype(v[13], &t)) return nullptr;
            ht = t == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32;
        }
        NormVectors vs(x->device());
        if (!vs.parse(v + 2, M, d)) return nullptr;
        const at::Tensor* const over = tensor(v[12]);  // h is x itself, unless y goes over it
        const bool plain = !res && !vs.gate && !post && alpha == 1.0f && ht == xt && v[11] == Py_None &&
                           !(over && over->data_ptr() == x->data_ptr());
        Out h, y;
        const at::ScalarType hs = ht == KQ_DTYPE_BF16 ? at::kBFloat16 : at::kFloat;
        if (v[11] != Py_None) {
            int t;
            if (!as_matrix(v[11], x, &t) || (res && t != ht)) return nullptr;
            ht = t;
            h.given = v[11];
            h.ptr = tensor(v[11])->data_ptr();
        } else if (!output(v[11], !plain, {M, d}, hs, M * d, x->device(), h)) {
            return nullptr;
        }
        int yt = xt;
        if (v[12] != Py_None && (!as_matrix(v[12], x, &yt) || yt != xt)) return nullptr;
        if (!output(v[12], true, {M, d}, x->scalar_type(), M * d, x->device(), y)) return nullptr;
        if (!call("kq_block_norm", [&] {
                return kq_block_norm(x->data_ptr(), (kq_dtype)xt, res ? res->data_ptr() : nullptr, (kq_dtype)ht, M, d,
                                     vs.vec.count(), vs.gate, vs.gs, vs.scale, vs.ss, vs.shift, vs.hs, vs.weight,
                                     vs.post_weight, (kq_dtype)vs.vec.dtype(), (kq_norm)norm, (kq_norm)post, alpha, eps, h.ptr,
                                     y.ptr, st);
            }))
            return nullptr;
        if (plain) h.given = v[0];
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, h.take());
        PyTuple_SET_ITEM(r, 1, y.take());
        return r;
    });
}

// ------------------------------------------------------------ a generation step

// The device is current: a launch, and the current stream, are on it.
bool current(at::Device dev) { return dev.is_cuda() && dev.index() == c10::hip::current_device(); }

// A [rows, heads, columns] array of fp32 or bf16 whose columns are contiguous.
struct Heads {
    const at::Tensor* t = nullptr;
    int type = 0;
    int64_t T = 0, H = 0, D = 0, row = 0, head = 0;
    bool parse(const at::Tensor* x) {
        t = x;
        if (!t || !t->is_cuda() || t->dim() != 3 || !float_type(t, &type)) return false;
        T = t->size(0);
        H = t->size(1);
        D = t->size(2);
        if (D > 1 && t->stride(2) != 1) return false;
        row = T > 1 ? t->stride(0) : H * D;
        head = H > 1 ? t->stride(1) : D;
        return true;
    }
};

// A result of x's sizes and type: a new one, x itself, or a contiguous one that shares no memory with x (others are
// left to Python's checks).
struct HeadsOut {
    Out out;
    int64_t row, head;
    bool parse(PyObject* o, const Heads& x) {
        row = x.H * x.D;
        head = x.D;
        if (o == Py_None) {
            out.made = empty({x.T, x.H, x.D}, x.t->scalar_type(), x.t->device());
            out.ptr = out.made.data_ptr();
            return true;
        }
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != x.t->scalar_type() || t->device() != x.t->device() || !t->sizes().equals(x.t->sizes()) ||
            !t->is_contiguous())
            return false;
        const bool same = t->data_ptr() == x.t->data_ptr() && t->strides().equals(x.t->strides());
        if (!same && t->storage().data() == x.t->storage().data()) return false;
        out.given = o;
        out.ptr = t->data_ptr();
        return true;
    }
};

// (x, positions, axes, theta, pairing, freqs, backward, out, stream)
PyObject* rope(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        Heads x;
        HeadsOut y;
        int pairing;
        bool backward;
        void* st = nullptr;
        double theta;
        if (!x.parse(tensor(v[0])) || !current(x.t->device()) || !small_int(v[4], &pairing) || !flag(v[6], &backward) ||
            !stream_of(v[8], &st))
            return nullptr;
        if (PyFloat_CheckExact(v[3])) theta = PyFloat_AS_DOUBLE(v[3]);
        else return nullptr;
        const at::Tensor* pos = tensor(v[1]);
        if (!pos || pos->device() != x.t->device()) return nullptr;
        int type;
        if (pos->scalar_type() == at::kInt) type = KQ_POSITION_INT32;
        else if (pos->scalar_type() == at::kLong) type = KQ_POSITION_INT64;
        else if (pos->scalar_type() == at::kFloat) type = KQ_POSITION_FP32;
        else return nullptr;
        int axes[4], count = 0;
        int64_t pairs = 0;
        if (PyLong_CheckExact(v[2])) {
            if (!small_int(v[2], &axes[count++])) return nullptr;
        } else {
            const bool list = PyList_CheckExact(v[2]);
            if (!list && !PyTuple_CheckExact(v[2])) return nullptr;
            const Py_ssize_t m = list ? PyList_GET_SIZE(v[2]) : PyTuple_GET_SIZE(v[2]);
            if (m < 1 || m > 4) return nullptr;
            while (count < m) {
                PyObject* const o = list ? PyList_GET_ITEM(v[2], count) : PyTuple_GET_ITEM(v[2], count);
                if (!small_int(o, &axes[count])) return nullptr;
                ++count;
            }
        }
        for (int i = 0; i < count; ++i) pairs += axes[i] / 2;
        const bool flat = pos->dim() == 1 && count == 1;
        if (!flat && (pos->dim() != 2 || pos->size(1) != count || (count > 1 && pos->stride(1) != 1))) return nullptr;
        if (pos->size(0) != x.T) return nullptr;
        const at::Tensor* freqs = nullptr;
        if (v[5] != Py_None) {
            freqs = tensor(v[5]);
            if (!buffer(freqs, at::kDouble, pairs, x.t->device())) return nullptr;
        }
        if (!y.parse(v[7], x)) return nullptr;
        if (!call("kq_rope", [&] {
                return kq_rope(x.t->data_ptr(), (kq_dtype)x.type, x.T, x.H, x.D, x.row, x.head, pos->data_ptr(), (kq_position)type,
                               x.T > 1 ? pos->stride(0) : count, axes, count, theta,
                               freqs ? static_cast<const double*>(freqs->data_ptr()) : nullptr, (kq_pairing)pairing, backward,
                               y.out.ptr, y.row, y.head, st);
            }))
            return nullptr;
        return y.out.take();
    });
}

// A KVCache (a named tuple of four).
bool cache_of(PyObject* o, kq_kv_cache* c, at::Device* dev) {
    if (!PyTuple_Check(o) || PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 4) return false;
    static PyObject* type = nullptr;  // (the GIL is held)
    if (!type) {
        PyObject* const m = PyImport_ImportModule("paper_2607_21446_amd.binding");
        type = m ? PyObject_GetAttrString(m, "KVCache") : nullptr;
        Py_XDECREF(m);
        if (!type) return false;
    }
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != type) return false;
    const bool scaled = PyTuple_GET_ITEM(o, 2) != Py_None;
    if (scaled != (PyTuple_GET_ITEM(o, 3) != Py_None)) return false;
    const at::Tensor* t[4] = {nullptr, nullptr, nullptr, nullptr};
    for (int i = 0; i < (scaled ? 4 : 2); ++i) {
        t[i] = tensor(PyTuple_GET_ITEM(o, i));
        if (!dense(t[i], scaled ? at::kByte : at::kBFloat16) || t[i]->dim() != 4 || t[i]->device() != t[0]->device()) return false;
        if (i % 2 && !t[i]->sizes().equals(t[i - 1]->sizes())) return false;
    }
    const int64_t row = t[0]->size(3);
    c->d = row;
    c->format = KQ_CACHE_BF16;
    if (scaled) {
        for (int i = 0; i < 3; ++i)
            if (t[2]->size(i) != t[0]->size(i)) return false;
        c->d = 32 * t[2]->size(3);
        if (row != c->d && 2 * row != c->d) return false;
        c->format = row == c->d ? KQ_CACHE_MXFP8 : KQ_CACHE_MXFP4;
    }
    c->k = t[0]->data_ptr();
    c->v = t[1]->data_ptr();
    c->k_scales = scaled ? static_cast<uint8_t*>(t[2]->data_ptr()) : nullptr;
    c->v_scales = scaled ? static_cast<uint8_t*>(t[3]->data_ptr()) : nullptr;
    c->pages = t[0]->size(0);
    c->heads = t[0]->size(1);
    c->page_size = t[0]->size(2);
    *dev = t[0]->device();
    return current(*dev);
}

const at::Tensor* slots_of(PyObject* o, at::Device dev) {
    const at::Tensor* t = tensor(o);
    return dense(t, at::kLong) && t->dim() == 1 && t->device() == dev ? t : nullptr;
}

// (cache, k, v, slots, stream)
PyObject* kv_cache_write(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 5) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        kq_kv_cache c;
        at::Device dev = at::kCPU;
        Heads h[2];
        void* st = nullptr;
        if (!cache_of(v[0], &c, &dev) || !stream_of(v[4], &st)) return nullptr;
        const at::Tensor* slots = slots_of(v[3], dev);
        if (!slots) return nullptr;
        for (int i = 0; i < 2; ++i) {
            if (!h[i].parse(tensor(v[1 + i])) || h[i].t->device() != dev || h[i].type != h[0].type || h[i].T != slots->numel() ||
                h[i].H != c.heads || h[i].D != c.d)
                return nullptr;
        }
        if (!call("kq_kv_cache_write", [&] {
                return kq_kv_cache_write(&c, h[0].t->data_ptr(), h[1].t->data_ptr(), (kq_dtype)h[0].type, h[0].T, h[0].row, h[0].head,
                                         h[1].row, h[1].head, static_cast<const int64_t*>(slots->data_ptr()), st);
            }))
            return nullptr;
        Py_INCREF(v[0]);
        return v[0];
    });
}

// (cache, slots, k, v, out_dtype, stream)
PyObject* kv_cache_read(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 6) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        kq_kv_cache c;
        at::Device dev = at::kCPU;
        void* st = nullptr;
        if (!cache_of(v[0], &c, &dev) || !stream_of(v[5], &st)) return nullptr;
        const at::Tensor* slots = slots_of(v[1], dev);
        if (!slots) return nullptr;
        at::ScalarType type = at::kBFloat16;
        if (v[4] != Py_None) {
            if (!float_dtype(v[4], &type)) return nullptr;
        } else if (v[2] != Py_None || v[3] != Py_None) {
            const at::Tensor* t = tensor(v[2] != Py_None ? v[2] : v[3]);
            if (!t) return nullptr;
            type = t->scalar_type();
        }
        if (type != at::kFloat && type != at::kBFloat16) return nullptr;
        const int64_t T = slots->numel();
        if (v[2] != Py_None && v[3] != Py_None) {  // (they may overlap)
            const at::Tensor *k = tensor(v[2]), *w = tensor(v[3]);
            if (!k || !w || k->storage().data() == w->storage().data()) return nullptr;
        }
        Out out[2];
        for (int i = 0; i < 2; ++i) {
            if (v[2 + i] != Py_None) {
                const at::Tensor* t = tensor(v[2 + i]);
                if (!t || t->dim() != 3 || t->size(0) != T || t->size(1) != c.heads || t->size(2) != c.d) return nullptr;
            }
            if (!output(v[2 + i], true, {T, c.heads, c.d}, type, T * c.heads * c.d, dev, out[i])) return nullptr;
        }
        if (!call("kq_kv_cache_read", [&] {
                return kq_kv_cache_read(&c, static_cast<const int64_t*>(slots->data_ptr()), T, out[0].ptr, out[1].ptr,
                                        type == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32, st);
            }))
            return nullptr;
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, out[0].take());
        PyTuple_SET_ITEM(r, 1, out[1].take());
        return r;
    });
}

// (q, cache, page_table, lengths, scale, window, out, lse, want_lse, workspace, stream)
PyObject* paged_attention(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        kq_kv_cache c;
        at::Device dev = at::kCPU;
        Heads q;
        HeadsOut out;
        void* st = nullptr;
        bool want = false;
        if (!cache_of(v[1], &c, &dev) || !q.parse(tensor(v[0])) || q.t->device() != dev || q.D != c.d || q.H < 1 || c.heads < 1 ||
            q.H % c.heads || !flag(v[8], &want) || !stream_of(v[10], &st))
            return nullptr;
        const at::Tensor *table = tensor(v[2]), *lengths = tensor(v[3]);
        if (!table || !table->is_cuda() || table->scalar_type() != at::kInt || table->device() != dev || table->dim() != 2 ||
            table->size(0) != q.T || (table->size(1) > 1 && table->stride(1) != 1) || !buffer(lengths, at::kInt, q.T, dev) ||
            lengths->dim() != 1)
            return nullptr;
        float scale = (float)(1.0 / std::sqrt((double)c.d));
        if (v[4] != Py_None && !number(v[4], &scale)) return nullptr;
        int64_t window = 0;
        if (v[5] != Py_None) {
            if (!PyLong_CheckExact(v[5])) return nullptr;
            window = PyLong_AsLongLong(v[5]);
            if (window < 1) return nullptr;
        }
        if (!out.parse(v[6], q)) return nullptr;
        Out lse;
        if (v[7] != Py_None || want) {
            if (!output(v[7], true, {q.T, q.H}, at::kFloat, q.T * q.H, dev, lse)) return nullptr;
        }
        size_t bytes = 0;
        at::Tensor made;
        void* work;
        if (v[9] != Py_None) {
            const at::Tensor* w = tensor(v[9]);
            if (!dense(w, at::kByte) || w->device() != dev) return nullptr;
            work = w->data_ptr();
            bytes = w->numel();
        } else {  // (one of the current stream's; for another stream Python makes it)
            if (v[10] != Py_None || kq_paged_attention_workspace_size(q.T, q.H, c.heads, c.d, &bytes) != KQ_SUCCESS) return nullptr;
            made = empty({(int64_t)bytes}, at::kByte, dev);
            work = made.data_ptr();
        }
        if (!call("kq_paged_attention", [&] {
                return kq_paged_attention(q.t->data_ptr(), (kq_dtype)q.type, q.T, q.H, q.row, q.head, &c,
                                          static_cast<const int32_t*>(table->data_ptr()), q.T > 1 ? table->stride(0) : table->size(1),
                                          table->size(1), static_cast<const int32_t*>(lengths->data_ptr()), scale, window, out.out.ptr,
                                          out.row, out.head, static_cast<float*>(lse.ptr), work, bytes, st);
            }))
            return nullptr;
        if (!lse.ptr && !lse.given && !lse.made.defined()) return out.out.take();
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, out.out.take());
        PyTuple_SET_ITEM(r, 1, lse.take());
        return r;
    });
}

// (x, b_codes, b_scales, bias, act, gate, residual, out, out_dtype, workspace, stream)
PyObject* w4a16_linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != 11) Py_RETURN_NONE;
    return guarded([&]() -> PyObject* {
        const at::Tensor *x = tensor(v[0]), *b = tensor(v[1]), *s = tensor(v[2]);
        int act, xt;
        void* st = nullptr;
        if (!x || !x->is_cuda() || x->dim() != 2 || !float_type(x, &xt) || !matrix(b, at::kByte) || !matrix(s, at::kByte) ||
            !small_int(v[4], &act) || !stream_of(v[10], &st))
            return nullptr;
        const at::Device dev = x->device();
        const int64_t M = x->size(0), K = x->size(1), N = b->size(0);
        if (!current(dev) || b->device() != dev || s->device() != dev || 2 * b->size(1) != K || s->size(0) != N || s->size(1) != K / 32)
            return nullptr;
        const int64_t ldx = row_stride(x, M, K, x->scalar_type(), dev), cols = act == KQ_ACT_SWIGLU ? N / 2 : N;
        if (ldx < 0 || (act == KQ_ACT_SWIGLU && N % 2)) return nullptr;
        Vectors vec(dev);
        const void *bias, *gate;
        int64_t none, stride;
        if (!vec.add(v[3], N, false, &bias, &none) || !vec.add(v[5], cols, true, &gate, &stride)) return nullptr;
        if (vec.count() <= 0 || M % vec.count()) return nullptr;
        at::ScalarType type = at::kBFloat16;
        const at::Tensor* res = nullptr;
        if (v[6] != Py_None) {
            res = tensor(v[6]);
            if (!res) return nullptr;
            type = res->scalar_type();
            if (type != at::kFloat && type != at::kBFloat16) return nullptr;
        }
        Out out;
        int64_t ldo, ldr = 0;
        if (!linear_out(v[7], v[8], type, M, cols, dev, out, &ldo, &type)) return nullptr;
        if (res && (ldr = row_stride(res, M, cols, type, dev)) < 0) return nullptr;
        if (out.given && tensor(v[7])->storage().data() == x->storage().data()) return nullptr;  // (they may overlap)
        size_t bytes = 0;
        at::Tensor made;
        void* work = nullptr;
        if (v[9] != Py_None) {
            const at::Tensor* w = tensor(v[9]);
            if (!dense(w, at::kByte) || w->device() != dev) return nullptr;
            bytes = w->numel();
            work = bytes ? w->data_ptr() : nullptr;
        } else {  // (one of the current stream's; for another stream Python makes it)
            if (kq_w4a16_workspace_size(M, N, K, (kq_dtype)xt, &bytes) != KQ_SUCCESS || (bytes && v[10] != Py_None)) return nullptr;
            if (bytes) {
                made = empty({(int64_t)bytes}, at::kByte, dev);
                work = made.data_ptr();
            }
        }
        if (!call("kq_w4a16_linear", [&] {
                return kq_w4a16_linear(x->data_ptr(), (kq_dtype)xt, M, ldx, static_cast<const uint8_t*>(b->data_ptr()),
                                       static_cast<const uint8_t*>(s->data_ptr()), N, K, bias, gate, stride,
                                       std::max<int64_t>(1, M / vec.count()), (kq_dtype)vec.dtype(), (kq_act)act,
                                       res ? res->data_ptr() : nullptr, ldr, out.ptr, ldo,
                                       type == at::kBFloat16 ? KQ_DTYPE_BF16 : KQ_DTYPE_FP32, work, bytes, st);
            }))
            return nullptr;
        return out.take();
    });
}

#define KQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {KQ_METHOD(quantize),    KQ_METHOD(quantize_exact), KQ_METHOD(quantize_packed),
                          KQ_METHOD(quantize_lu), KQ_METHOD(smoothquant),    KQ_METHOD(hadamard32),
                          KQ_METHOD(fwht),        KQ_METHOD(mxfp4),          KQ_METHOD(mxfp4_gemm),
                          KQ_METHOD(calib_step),  KQ_METHOD(mxfp4_linear),   KQ_METHOD(mxfp4_grouped_linear),
                          KQ_METHOD(block_norm),  KQ_METHOD(rope),           KQ_METHOD(kv_cache_write),
                          KQ_METHOD(kv_cache_read), KQ_METHOD(paged_attention), KQ_METHOD(w4a16_linear),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_kqbind", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kqbind() { return PyModule_Create(&kModule); }
