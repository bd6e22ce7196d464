// The per-token calls of the Python package, marshalled in native code: the products, the
// encode and the conversions take 3 to 7 us on the GPU, and checking the tensors, fetching
// the current stream and the foreign-function call took 9.7 us of Python per call (4.2 us
// now, of which the launch is about 3).
//
// Each function does its method's own checks on plain tensors and makes the call.  For
// whatever it does not take as it is (a tensor subclass, a wrong type, shape or device, a
// missing buffer that is not simply allocated) it returns None and has done nothing; the
// method's Python code then takes the call, or raises the error that names what is wrong.
// A failing library call raises through the package's own check.  Nothing is kept between
// calls.
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <new>
#include <vector>

#include "darb.h"

namespace {

struct PlanRef {
    darb_plan *plan;
    int64_t M, N, nnz, words;
};

const char kPlanName[] = "darb_plan";
PyObject *g_check = nullptr;             // the package's _check(code, where)
PyObject *g_stream_attr = nullptr;       // "cuda_stream"

void free_ref(PyObject *cap) {
    delete static_cast<PlanRef *>(PyCapsule_GetPointer(cap, kPlanName));
}

const PlanRef *plan_of(PyObject *o) {
    return static_cast<const PlanRef *>(PyCapsule_GetPointer(o, kPlanName));
}

// A plain device tensor with memory of its own, or null.
const at::Tensor *tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) return nullptr;
    return &t;
}

// A flat buffer of at least n elements of the given type.
const at::Tensor *buffer(PyObject *o, int64_t n, at::ScalarType type) {
    const at::Tensor *t = tensor(o);
    return t && t->scalar_type() == type && t->is_contiguous() && t->numel() >= n ? t : nullptr;
}

bool float_code(const at::Tensor &t, int *code) {
    if (t.scalar_type() == at::kFloat) *code = DARB_F32;
    else if (t.scalar_type() == at::kHalf) *code = DARB_F16;
    else return false;
    return true;
}

const at::Tensor *values_of(PyObject *o, int64_t nnz, int *code) {
    const at::Tensor *t = tensor(o);
    return t && float_code(*t, code) && t->is_contiguous() && t->numel() >= nnz ? t : nullptr;
}

// A [rows, cols] matrix of unit column stride: its leading dimension, or -1.
int64_t leading(const at::Tensor &t, int64_t rows, int64_t cols) {
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.stride(1) != 1) return -1;
    return rows > 1 ? t.stride(0) : (cols > t.stride(0) ? cols : t.stride(0));
}

// The stream's handle: the current one of the current device for None.
bool stream_of(PyObject *o, void **s) {
    if (o == Py_None) {
        *s = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    PyObject *v = PyObject_GetAttr(o, g_stream_attr);
    if (v && PyLong_Check(v)) *s = PyLong_AsVoidPtr(v);
    const bool ok = v && PyLong_Check(v) && !PyErr_Occurred();
    Py_XDECREF(v);
    if (!ok) PyErr_Clear();
    return ok;
}

// What a call allocates, while this lives, for its stream.  On another stream than the current one
// that is the other's memory: blocks of the current stream may still be in use by work queued there.
// Results (new or given) are then held until both streams are done with them.
class Memory {
  public:
    Memory(PyObject *o, void *s) : here_(c10::hip::getCurrentHIPStream()), there_(here_) {
        if (o == Py_None || s == static_cast<void *>(here_.stream())) return;
        there_ = c10::hip::getStreamFromExternal(static_cast<hipStream_t>(s), here_.device_index());
        other_ = true;
        c10::hip::setCurrentHIPStream(there_);
    }
    ~Memory() {
        if (other_) c10::hip::setCurrentHIPStream(here_);
    }
    Memory(const Memory &) = delete;
    Memory &operator=(const Memory &) = delete;
    void result(const at::Tensor &t) const {
        if (!other_ || !t.defined()) return;
        for (const auto &s : {here_, there_}) c10::hip::HIPCachingAllocator::recordStream(t.storage().data_ptr(), s);
    }

  private:
    c10::hip::HIPStream here_, there_;
    bool other_ = false;
};

void *ptr(const at::Tensor &t) { return t.data_ptr(); }

PyObject *none() { Py_RETURN_NONE; }

// The call with the interpreter lock released (as a foreign-function call does), then the
// result, or the package's error.
template <typename F> PyObject *finish(PyObject *result, const char *where, F &&call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    if (rc == DARB_OK) return result;
    Py_DECREF(result);
    PyObject *r = PyObject_CallFunction(g_check, "is", rc, where);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, where);
    return nullptr;
}

// Any C++ exception (a tensor without memory, an allocation that fails): the Python code
// takes the call and reports it.
template <typename F> PyObject *guarded(F &&f) {
    try {
        return f();
    } catch (...) {
        if (PyErr_Occurred()) PyErr_Clear();
        return none();
    }
}

// y [M] as given, or a new one on x's device.
PyObject *vector_out(PyObject *o, const PlanRef &p, const at::Tensor &x, at::Tensor *out) {
    if (o == Py_None) {
        *out = at::empty({p.M}, x.options().dtype(at::kFloat));
        return THPVariable_Wrap(*out);
    }
    const at::Tensor *y = buffer(o, p.M, at::kFloat);
    if (!y) return nullptr;
    *out = *y;
    Py_INCREF(o);
    return o;
}

PyObject *matrix_out(PyObject *o, const PlanRef &p, const at::Tensor &X, at::Tensor *out,
                     int64_t *ldy) {
    const int64_t B = X.size(1);
    if (o == Py_None) {
        *out = at::empty({p.M, B}, X.options().dtype(at::kFloat));
        *ldy = leading(*out, p.M, B);
        return THPVariable_Wrap(*out);
    }
    const at::Tensor *Y = tensor(o);
    if (!Y || Y->scalar_type() != at::kFloat) return nullptr;
    *ldy = leading(*Y, p.M, B);
    if (*ldy < 0) return nullptr;
    *out = *Y;
    Py_INCREF(o);
    return o;
}

// What a product multiplies by: values, or codes and scales; byte offsets, or packed words.
struct Format {
    const at::Tensor *values = nullptr, *scales = nullptr;
    const uint8_t *offsets = nullptr;
    const uint32_t *packed = nullptr;
    int code = 0;
};

bool offsets_of(PyObject *o, const PlanRef &p, Format *f) {
    const at::Tensor *t = buffer(o, p.nnz, at::kByte);
    if (t) f->offsets = static_cast<const uint8_t *>(ptr(*t));
    return t != nullptr;
}

bool packed_of(PyObject *o, const PlanRef &p, Format *f) {
    const at::Tensor *t = buffer(o, p.words, at::kInt);
    if (t) f->packed = static_cast<const uint32_t *>(ptr(*t));
    return t != nullptr;
}

template <typename F>
PyObject *vector_product(const PlanRef &p, PyObject *xo, PyObject *yo, PyObject *so,
                         const char *where, F &&call) {
    const at::Tensor *x = tensor(xo);
    int xcode;
    void *s;
    if (!x || !float_code(*x, &xcode) || x->dim() != 1 || x->size(0) != p.N ||
        !x->is_contiguous() || !stream_of(so, &s))
        return none();
    const Memory memory(so, s);
    at::Tensor y;
    PyObject *res = vector_out(yo, p, *x, &y);
    if (!res) return none();
    memory.result(y);
    const void *xp = ptr(*x);
    float *yp = static_cast<float *>(ptr(y));
    return finish(res, where, [&] { return call(xcode, xp, yp, s); });
}

template <typename F>
PyObject *matrix_product(const PlanRef &p, PyObject *xo, PyObject *yo, PyObject *so,
                         const char *where, F &&call) {
    const at::Tensor *X = tensor(xo);
    int xcode;
    void *s;
    if (!X || !float_code(*X, &xcode) || X->dim() != 2 || !stream_of(so, &s)) return none();
    const int64_t B = X->size(1), ldx = leading(*X, p.N, B);
    if (ldx < 0) return none();
    const Memory memory(so, s);
    at::Tensor Y;
    int64_t ldy;
    PyObject *res = matrix_out(yo, p, *X, &Y, &ldy);
    if (!res) return none();
    memory.result(Y);
    const void *xp = ptr(*X);
    float *yp = static_cast<float *>(ptr(Y));
    return finish(res, where, [&] { return call(xcode, B, xp, ldx, yp, ldy, s); });
}

#define DARB_ARGS(N)                                                                        \
    if (n != (N)) return none();                                                            \
    const PlanRef *p = plan_of(a[0]);                                                       \
    if (!p) {                                                                               \
        PyErr_Clear();                                                                      \
        return none();                                                                      \
    }

// (plan, values, offsets, x, y, stream)
PyObject *spmv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(6)
        Format f;
        if (!(f.values = values_of(a[1], p->nnz, &f.code)) || !offsets_of(a[2], *p, &f)) return none();
        const void *v = ptr(*f.values);
        return vector_product(*p, a[3], a[4], a[5], "darb_spmv",
                              [&](int xc, const void *x, float *y, void *s) {
                                  return darb_spmv(p->plan, f.code, v, f.offsets, xc, x, y, s);
                              });
    });
}

PyObject *spmv_packed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(6)
        Format f;
        if (!(f.values = values_of(a[1], p->nnz, &f.code)) || !packed_of(a[2], *p, &f)) return none();
        const void *v = ptr(*f.values);
        return vector_product(*p, a[3], a[4], a[5], "darb_spmv_packed",
                              [&](int xc, const void *x, float *y, void *s) {
                                  return darb_spmv_packed(p->plan, f.code, v, f.packed, xc, x, y, s);
                              });
    });
}

// (plan, values, offsets, X, Y, stream)
PyObject *spmm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(6)
        Format f;
        if (!(f.values = values_of(a[1], p->nnz, &f.code)) || !offsets_of(a[2], *p, &f)) return none();
        const void *v = ptr(*f.values);
        return matrix_product(
            *p, a[3], a[4], a[5], "darb_spmm",
            [&](int xc, int64_t B, const void *X, int64_t ldx, float *Y, int64_t ldy, void *s) {
                return darb_spmm(p->plan, f.code, v, f.offsets, xc, B, X, ldx, Y, ldy, s);
            });
    });
}

PyObject *spmm_packed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(6)
        Format f;
        if (!(f.values = values_of(a[1], p->nnz, &f.code)) || !packed_of(a[2], *p, &f)) return none();
        const void *v = ptr(*f.values);
        return matrix_product(
            *p, a[3], a[4], a[5], "darb_spmm_packed",
            [&](int xc, int64_t B, const void *X, int64_t ldx, float *Y, int64_t ldy, void *s) {
                return darb_spmm_packed(p->plan, f.code, v, f.packed, xc, B, X, ldx, Y, ldy, s);
            });
    });
}

bool i8_format(PyObject *codes, PyObject *scales, PyObject *offsets, PyObject *packed,
               const PlanRef &p, Format *f) {
    f->values = buffer(codes, p.nnz, at::kChar);
    f->scales = buffer(scales, p.M, at::kFloat);
    if (!f->values || !f->scales || (offsets == Py_None) == (packed == Py_None)) return false;
    return offsets != Py_None ? offsets_of(offsets, p, f) : packed_of(packed, p, f);
}

// (plan, codes, scales, x, offsets, packed, y, stream)
PyObject *spmv_i8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(8)
        Format f;
        if (!i8_format(a[1], a[2], a[4], a[5], *p, &f)) return none();
        const int8_t *q = static_cast<const int8_t *>(ptr(*f.values));
        const float *sc = static_cast<const float *>(ptr(*f.scales));
        return vector_product(*p, a[3], a[6], a[7], "darb_spmv_i8",
                              [&](int xc, const void *x, float *y, void *s) {
                                  return darb_spmv_i8(p->plan, q, sc, f.offsets, f.packed, xc, x,
                                                      y, s);
                              });
    });
}

PyObject *spmm_i8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(8)
        Format f;
        if (!i8_format(a[1], a[2], a[4], a[5], *p, &f)) return none();
        const int8_t *q = static_cast<const int8_t *>(ptr(*f.values));
        const float *sc = static_cast<const float *>(ptr(*f.scales));
        return matrix_product(
            *p, a[3], a[6], a[7], "darb_spmm_i8",
            [&](int xc, int64_t B, const void *X, int64_t ldx, float *Y, int64_t ldy, void *s) {
                return darb_spmm_i8(p->plan, q, sc, f.offsets, f.packed, xc, B, X, ldx, Y, ldy, s);
            });
    });
}

// (plan, W, values, offsets, stream)
PyObject *encode(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(5)
        const at::Tensor *W = tensor(a[1]);
        int wcode, vcode;
        void *s;
        if (!W || !float_code(*W, &wcode) || !stream_of(a[4], &s)) return none();
        const int64_t ldw = leading(*W, p->M, p->N);
        const at::Tensor *v = values_of(a[2], p->nnz, &vcode);
        const at::Tensor *o = buffer(a[3], p->nnz, at::kByte);
        if (ldw < 0 || !v || !o || vcode != wcode) return none();
        const void *wp = ptr(*W);
        void *vp = ptr(*v);
        uint8_t *op = static_cast<uint8_t *>(ptr(*o));
        PyObject *res = PyTuple_Pack(2, a[2], a[3]);
        if (!res) return nullptr;
        return finish(res, "darb_encode",
                      [&] { return darb_encode(p->plan, wcode, wp, ldw, vp, op, s); });
    });
}

// ---- evaluating and retraining a layer -------------------------------------------------

bool any_float_code(const at::Tensor &t, int *code) {
    if (t.scalar_type() != at::kBFloat16) return float_code(t, code);
    *code = DARB_BF16;
    return true;
}

bool here(const at::Tensor &t) { return t.get_device() == c10::hip::current_device(); }

// A non-empty [F, B] operand of either order on the current device, or null.
const at::Tensor *matrix(PyObject *o) {
    const at::Tensor *t = tensor(o);
    if (!t || t->dim() != 2 || t->numel() == 0 || !here(*t)) return nullptr;
    const int64_t F = t->size(0), B = t->size(1), fs = t->stride(0), bs = t->stride(1);
    return F == 1 || B == 1 || (fs == 1 && bs >= F) || (bs == 1 && fs >= B) ? t : nullptr;
}

const at::Tensor *matrix_like(PyObject *o, const at::Tensor &x) {
    const at::Tensor *t = matrix(o);
    return t && t->sizes() == x.sizes() && t->scalar_type() == x.scalar_type() ? t : nullptr;
}

// A flat buffer on the current device; None is a null pointer.
template <typename T> bool optional(PyObject *o, int64_t n, at::ScalarType type, T **p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = buffer(o, n, type);
    if (!t || !here(*t)) return false;
    *p = static_cast<T *>(ptr(*t));
    return true;
}

// A new dense tensor in x's memory order (contiguous where one token or feature leaves it open).
at::Tensor dense_like(const at::Tensor &x) {
    if (x.stride(0) == 1 && x.size(0) > 1 && x.size(1) > 1)
        return at::empty_strided(x.sizes(), {1, x.size(0)}, x.options());
    return at::empty(x.sizes(), x.options());
}

// The tensor given, or a new one by `make` for None; the new reference is the caller's.
template <typename F, typename C> PyObject *given_or(PyObject *o, at::Tensor *out, C &&check, F &&make) {
    if (o == Py_None) {
        *out = make();
        return THPVariable_Wrap(*out);
    }
    const at::Tensor *t = check(o);
    if (!t) return nullptr;
    *out = *t;
    Py_INCREF(o);
    return o;
}

// References that go with a failed or abandoned call.
struct Held {
    PyObject *o[3] = {};
    ~Held() {
        for (PyObject *p : o) Py_XDECREF(p);
    }
    PyObject *tuple(int n) {
        PyObject *t = PyTuple_New(n);
        if (!t) return nullptr;
        for (int i = 0; i < n; ++i) {
            PyTuple_SET_ITEM(t, i, o[i] ? o[i] : (Py_INCREF(Py_None), Py_None));
            o[i] = nullptr;
        }
        return t;
    }
};

// (logits, targets, top, stream): (logprob, entropy, lse, top_logprob, top_index)
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        int code;
        void *s;
        int64_t *t;
        if (n != 4) return none();
        const at::Tensor *z = matrix(a[0]);
        if (!z || !any_float_code(*z, &code) || !optional(a[1], z->size(1), at::kLong, &t) ||
            !PyLong_CheckExact(a[2]) || !stream_of(a[3], &s))
            return none();
        const int64_t V = z->size(0), B = z->size(1), fs = z->stride(0), bs = z->stride(1);
        const long long top = PyLong_AsLongLong(a[2]);
        int64_t bytes;
        if (top < 0 || darb_token_logprobs_workspace(code, V, B, fs, bs, top, &bytes) != DARB_OK) {
            PyErr_Clear();
            return none();
        }
        const Memory memory(a[3], s);
        const auto f32 = z->options().dtype(at::kFloat);
        at::Tensor out[5], workspace;
        for (int i = 0; i < 3; ++i) out[i] = at::empty({B}, f32);
        if (top) {
            out[3] = at::empty({B, int64_t(top)}, f32);
            out[4] = at::empty({B, int64_t(top)}, z->options().dtype(at::kLong));
        }
        if (bytes) workspace = at::empty({bytes}, z->options().dtype(at::kByte));
        for (const at::Tensor &t : out) memory.result(t);
        const void *zp = ptr(*z);
        float *p[4];
        for (int i = 0; i < 4; ++i) p[i] = out[i].defined() ? static_cast<float *>(ptr(out[i])) : nullptr;
        int64_t *ti = top ? static_cast<int64_t *>(ptr(out[4])) : nullptr;
        void *w = bytes ? ptr(workspace) : nullptr;
        PyObject *res = PyTuple_New(5);
        if (!res) return nullptr;
        for (int i = 0; i < 5; ++i)
            PyTuple_SET_ITEM(res, i, out[i].defined() ? THPVariable_Wrap(out[i]) : (Py_INCREF(Py_None), Py_None));
        return finish(res, "darb_token_logprobs", [&] {
            return darb_token_logprobs(code, V, B, zp, fs, bs, t, top, p[0], p[1], p[2], p[3], ti, w, bytes, s);
        });
    });
}

// (logits, targets, lse, grad_logprob, entropy, grad_entropy, out, stream)
PyObject *token_logprobs_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        int code;
        void *s;
        int64_t *t;
        float *lse, *g, *h, *gh;
        if (n != 8) return none();
        const at::Tensor *z = matrix(a[0]);
        if (!z || !any_float_code(*z, &code)) return none();
        const int64_t V = z->size(0), B = z->size(1);
        if (!optional(a[1], B, at::kLong, &t) || !optional(a[2], B, at::kFloat, &lse) || !lse ||
            !optional(a[3], B, at::kFloat, &g) || !optional(a[4], B, at::kFloat, &h) ||
            !optional(a[5], B, at::kFloat, &gh) || !stream_of(a[7], &s))
            return none();
        const Memory memory(a[7], s);
        at::Tensor dz;
        PyObject *res = given_or(a[6], &dz, [&](PyObject *o) { return matrix_like(o, *z); },
                                 [&] { return dense_like(*z); });
        if (!res) return none();
        memory.result(dz);
        const void *zp = ptr(*z);
        void *dp = ptr(dz);
        return finish(res, "darb_token_logprobs_grad", [&] {
            return darb_token_logprobs_grad(code, V, B, zp, z->stride(0), z->stride(1), t, lse, g, h, gh, dp,
                                            dz.stride(0), dz.stride(1), s);
        });
    });
}

// A weight [H]: fp32 or x's type, one type for both.
bool norm_weight(PyObject *o, const at::Tensor &x, int64_t H, int code, int *wcode, void **p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o);
    int c;
    if (!t || !any_float_code(*t, &c) || (c != DARB_F32 && c != code) || (*wcode >= 0 && *wcode != c) ||
        !t->is_contiguous() || t->numel() < H || !here(*t))
        return false;
    *wcode = c;
    *p = ptr(*t);
    return true;
}

// (x, weight, bias, eps, y, mean, rstd, stream)
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        int code, wcode = -1;
        void *s, *w, *b;
        if (n != 8) return none();
        const at::Tensor *x = matrix(a[0]);
        if (!x || !any_float_code(*x, &code)) return none();
        const int64_t H = x->size(0), B = x->size(1);
        if (!norm_weight(a[1], *x, H, code, &wcode, &w) || !norm_weight(a[2], *x, H, code, &wcode, &b) ||
            !PyFloat_CheckExact(a[3]) || !stream_of(a[7], &s))
            return none();
        const double eps = PyFloat_AS_DOUBLE(a[3]);
        const auto f32 = x->options().dtype(at::kFloat);
        auto vector = [&](PyObject *o) {
            const at::Tensor *t = buffer(o, B, at::kFloat);
            return t && here(*t) ? t : nullptr;
        };
        const Memory memory(a[7], s);
        at::Tensor y, mean, rstd;
        Held held;
        if (!(held.o[0] = given_or(a[4], &y, [&](PyObject *o) { return matrix_like(o, *x); },
                                   [&] { return dense_like(*x); })) ||
            !(held.o[1] = given_or(a[5], &mean, vector, [&] { return at::empty({B}, f32); })) ||
            !(held.o[2] = given_or(a[6], &rstd, vector, [&] { return at::empty({B}, f32); })))
            return none();
        for (const at::Tensor &t : {y, mean, rstd}) memory.result(t);
        const void *xp = ptr(*x);
        void *yp = ptr(y);
        float *mp = static_cast<float *>(ptr(mean)), *rp = static_cast<float *>(ptr(rstd));
        PyObject *res = held.tuple(3);
        if (!res) return nullptr;
        return finish(res, "darb_layer_norm", [&] {
            return darb_layer_norm(code, wcode < 0 ? int(DARB_F32) : wcode, H, B, xp, x->stride(0), x->stride(1), w,
                                   b, eps, yp, y.stride(0), y.stride(1), mp, rp, s);
        });
    });
}

// (dy, x, mean, rstd, weight, stream): all three gradients, new
PyObject *layer_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        int code, wcode = -1;
        void *s, *w;
        float *mean, *rstd;
        if (n != 6) return none();
        const at::Tensor *x = matrix(a[1]);
        if (!x || !any_float_code(*x, &code)) return none();
        const at::Tensor *dy = matrix_like(a[0], *x);
        const int64_t H = x->size(0), B = x->size(1);
        int64_t bytes;
        if (!dy || !optional(a[2], B, at::kFloat, &mean) || !mean || !optional(a[3], B, at::kFloat, &rstd) ||
            !rstd || !norm_weight(a[4], *x, H, code, &wcode, &w) || !stream_of(a[5], &s) ||
            darb_layer_norm_workspace(H, B, &bytes) != DARB_OK)
            return none();
        const Memory memory(a[5], s);
        const auto f32 = x->options().dtype(at::kFloat);
        at::Tensor dx = dense_like(*x), dw = at::empty({H}, f32), db = at::empty({H}, f32);
        at::Tensor workspace = at::empty({bytes}, x->options().dtype(at::kByte));
        for (const at::Tensor &t : {dx, dw, db}) memory.result(t);
        Held held;
        held.o[0] = THPVariable_Wrap(dx);
        held.o[1] = THPVariable_Wrap(dw);
        held.o[2] = THPVariable_Wrap(db);
        const void *xp = ptr(*x), *gp = ptr(*dy);
        void *dp = ptr(dx), *ws = ptr(workspace);
        float *wp = static_cast<float *>(ptr(dw)), *bp = static_cast<float *>(ptr(db));
        PyObject *res = held.tuple(3);
        if (!res) return nullptr;
        return finish(res, "darb_layer_norm_grad", [&] {
            return darb_layer_norm_grad(code, wcode < 0 ? int(DARB_F32) : wcode, H, B, gp, dy->stride(0),
                                        dy->stride(1), xp, x->stride(0), x->stride(1), mean, rstd, w, dp,
                                        dx.stride(0), dx.stride(1), wp, bp, ws, bytes, s);
        });
    });
}

// (plan, index, values, X, dY, stream): both gradients, new
PyObject *spmm_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        DARB_ARGS(6)
        int wcode, xcode;
        void *s;
        int64_t need, bytes;
        if (darb_transpose_bytes(p->plan, &need) != DARB_OK) return none();
        const at::Tensor *index = buffer(a[1], need, at::kByte), *values = values_of(a[2], p->nnz, &wcode);
        const at::Tensor *X = tensor(a[3]), *dY = tensor(a[4]);
        if (!index || !values || !X || !dY || !float_code(*X, &xcode) || dY->scalar_type() != at::kFloat ||
            dY->dim() != 2 || !stream_of(a[5], &s))
            return none();
        const int64_t B = dY->size(1), ldy = leading(*dY, p->M, B), ldx = leading(*X, p->N, B);
        if (ldy < 0 || ldx < 0 || darb_spmm_grad_workspace(p->plan, B, &bytes) != DARB_OK) return none();
        const Memory memory(a[5], s);
        const auto f32 = dY->options();
        at::Tensor dv = at::empty({p->nnz}, f32), dX = at::empty({p->N, B}, f32), workspace;
        if (bytes) workspace = at::empty({bytes}, f32.dtype(at::kByte));
        memory.result(dv);
        memory.result(dX);
        Held held;
        held.o[0] = THPVariable_Wrap(dv);
        held.o[1] = THPVariable_Wrap(dX);
        const void *ip = ptr(*index), *vp = ptr(*values), *xp = ptr(*X);
        const float *gp = static_cast<const float *>(ptr(*dY));
        float *dvp = static_cast<float *>(ptr(dv)), *dXp = static_cast<float *>(ptr(dX));
        void *ws = bytes ? ptr(workspace) : nullptr;
        const int64_t lddx = leading(dX, p->N, B);
        PyObject *res = held.tuple(2);
        if (!res) return nullptr;
        return finish(res, "darb_spmm_grad", [&] {
            return darb_spmm_grad(p->plan, ip, wcode, vp, xcode, B, xp, ldx, gp, ldy, dvp, dXp, lddx, ws, bytes, s);
        });
    });
}

// A list of tensors as pointers, each with its parameter's element count; false if one is not a
// plain contiguous tensor of that size (None is allowed: a null pointer).
bool pointers(PyObject *list, PyObject *params, bool any_type, std::vector<void *> *p, std::vector<int> *types) {
    if (!PyList_CheckExact(list) || !PyList_CheckExact(params)) return false;
    const Py_ssize_t n = PyList_GET_SIZE(params);
    if (PyList_GET_SIZE(list) != n) return false;
    p->assign(n, nullptr);
    types->assign(n, DARB_F32);
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject *o = PyList_GET_ITEM(list, i), *q = PyList_GET_ITEM(params, i);
        if (o == Py_None && any_type) continue;
        const at::Tensor *t = tensor(o), *of = tensor(q);
        int code;
        if (!t || !of || !any_float_code(*t, &code) || (!any_type && code != DARB_F32) || !t->is_contiguous() ||
            t->numel() != of->numel() || !here(*t))
            return false;
        (*p)[i] = t->numel() ? ptr(*t) : nullptr;
        (*types)[i] = code;
    }
    return true;
}

// (handle, params, grads, lr, beta1, beta2, eps, step, grad_scale, seed, stream): True
PyObject *adamw_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 11 || !PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[7]) || !PyLong_CheckExact(a[9]))
            return none();
        double k[4];
        for (int i = 0; i < 4; ++i) {
            if (!PyFloat_CheckExact(a[3 + i])) return none();
            k[i] = PyFloat_AS_DOUBLE(a[3 + i]);
        }
        std::vector<void *> p;
        std::vector<int> types;
        float *scale;
        void *s;
        if (!pointers(a[2], a[1], true, &p, &types) || !optional(a[8], 1, at::kFloat, &scale) ||
            !stream_of(a[10], &s))
            return none();
        const darb_adamw *h = static_cast<const darb_adamw *>(PyLong_AsVoidPtr(a[0]));
        const long long step = PyLong_AsLongLong(a[7]);
        const uint32_t seed = uint32_t(PyLong_AsUnsignedLongMask(a[9]));
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        Py_INCREF(Py_True);
        return finish(Py_True, "darb_adamw_step", [&] {
            return darb_adamw_step(h, p.data(), types.data(), int64_t(p.size()), k[0], k[1], k[2], k[3], step, scale,
                                   seed, s);
        });
    });
}

// (handle, params, m, v, stream): True
PyObject *adamw_moments(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        std::vector<void *> m, v;
        std::vector<int> types;
        void *s;
        if (n != 5 || !PyLong_CheckExact(a[0]) || !pointers(a[2], a[1], false, &m, &types) ||
            !pointers(a[3], a[1], false, &v, &types) || !stream_of(a[4], &s))
            return none();
        const darb_adamw *h = static_cast<const darb_adamw *>(PyLong_AsVoidPtr(a[0]));
        Py_INCREF(Py_True);
        return finish(Py_True, "darb_adamw_moments", [&] {
            return darb_adamw_moments(h, reinterpret_cast<float *const *>(m.data()),
                                      reinterpret_cast<float *const *>(v.data()), int64_t(m.size()), s);
        });
    });
}

darb_matrix as_matrix(const at::Tensor &t) { return {ptr(t), t.stride(0), t.stride(1)}; }

// A state fp32 [H, batch] on the current device; None is none.
bool state(PyObject *o, int64_t H, int64_t batch, darb_matrix *m, const darb_matrix **p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = tensor(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != H || t->size(1) != batch || !here(*t))
        return false;
    *m = as_matrix(*t);
    *p = m;
    return true;
}

at::Tensor state_like(const at::Tensor &x, int64_t H, int64_t batch) {
    const auto f32 = x.options().dtype(at::kFloat);
    if (x.stride(0) == 1 && H > 1 && x.size(1) > 1) return at::empty_strided({H, batch}, {1, H}, f32);
    return at::empty({H, batch}, f32);
}

// What both directions of the recurrence share.
struct Sequences {
    int code = 0, form = 0;
    int64_t H = 0, T = 0, batch = 0;
    const uint8_t *resets = nullptr;
    bool take(const at::Tensor &x, PyObject *batch_, PyObject *resets_, PyObject *form_) {
        if (!any_float_code(x, &code) || !PyLong_CheckExact(batch_) || !PyLong_CheckExact(form_)) return false;
        batch = PyLong_AsLongLong(batch_);
        form = int(PyLong_AsLong(form_));
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return false;
        }
        if (batch < 1 || x.size(1) % batch != 0 || form < 0) return false;
        H = x.size(0);
        T = x.size(1) / batch;
        if (resets_ == Py_None) return true;
        const at::Tensor *r = tensor(resets_);
        if (!r || (r->scalar_type() != at::kBool && r->scalar_type() != at::kByte) || r->dim() != 1 ||
            r->size(0) != x.size(1) || !r->is_contiguous() || !here(*r))
            return false;
        resets = static_cast<const uint8_t *>(ptr(*r));
        return true;
    }
};

// A new state, or the one given.
PyObject *state_or(PyObject *o, const at::Tensor &x, const Sequences &q, at::Tensor *out) {
    return given_or(o, out,
                    [&](PyObject *g) -> const at::Tensor * {
                        darb_matrix m;
                        const darb_matrix *p;
                        return state(g, q.H, q.batch, &m, &p) && p ? tensor(g) : nullptr;
                    },
                    [&] { return state_like(x, q.H, q.batch); });
}

// (gate, x, batch, h0, resets, form, h, h_last, stream): (h, h_last)
PyObject *gated_recurrence(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Sequences q;
        void *s;
        darb_matrix m0;
        const darb_matrix *h0;
        int64_t bytes;
        if (n != 9) return none();
        const at::Tensor *x = matrix(a[1]);
        if (!x) return none();
        const at::Tensor *gate = matrix_like(a[0], *x);
        if (!gate || !q.take(*x, a[2], a[4], a[5]) || !state(a[3], q.H, q.batch, &m0, &h0) || !stream_of(a[8], &s) ||
            darb_gated_recurrence_workspace(q.code, 0, q.H, q.T, q.batch, &bytes) != DARB_OK)
            return none();
        const Memory memory(a[8], s);
        at::Tensor h, last, workspace;
        Held held;
        if (!(held.o[0] = given_or(a[6], &h, [&](PyObject *o) { return matrix_like(o, *x); },
                                   [&] { return dense_like(*x); })) ||
            !(held.o[1] = state_or(a[7], *x, q, &last)))
            return none();
        if (bytes) workspace = at::empty({bytes}, x->options().dtype(at::kByte));
        memory.result(h);
        memory.result(last);
        const darb_matrix gm = as_matrix(*gate), xm = as_matrix(*x), hm = as_matrix(h), lm = as_matrix(last);
        void *w = bytes ? ptr(workspace) : nullptr;
        PyObject *res = held.tuple(2);
        if (!res) return nullptr;
        return finish(res, "darb_gated_recurrence", [&] {
            return darb_gated_recurrence(q.code, q.form, q.H, q.T, q.batch, &gm, &xm, q.resets, h0, &hm, &lm, w, bytes,
                                         s);
        });
    });
}

// (dh, gate, x, h, batch, h0, resets, dh_last, form, dgate, dx, dh0, stream): (dgate, dx, dh0)
PyObject *gated_recurrence_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Sequences q;
        void *s;
        darb_matrix m0, ml, xm;
        const darb_matrix *h0, *dl;
        int64_t bytes;
        if (n != 13) return none();
        const at::Tensor *gate = matrix(a[1]);
        if (!gate) return none();
        const at::Tensor *dh = matrix_like(a[0], *gate), *h = matrix_like(a[3], *gate);
        const at::Tensor *x = a[2] == Py_None ? nullptr : matrix_like(a[2], *gate);
        if (!dh || !h || (!x && a[2] != Py_None) || !q.take(*gate, a[4], a[6], a[8]) ||
            (!x && q.form != DARB_RECURRENCE_LINEAR) || !state(a[5], q.H, q.batch, &m0, &h0) ||
            !state(a[7], q.H, q.batch, &ml, &dl) || !stream_of(a[12], &s) ||
            darb_gated_recurrence_workspace(q.code, 1, q.H, q.T, q.batch, &bytes) != DARB_OK)
            return none();
        const Memory memory(a[12], s);
        at::Tensor dgate, dx, dh0, workspace;
        Held held;
        auto like = [&](PyObject *o) { return matrix_like(o, *gate); };
        auto dense = [&] { return dense_like(*gate); };
        if (!(held.o[0] = given_or(a[9], &dgate, like, dense)) || !(held.o[1] = given_or(a[10], &dx, like, dense)) ||
            !(held.o[2] = state_or(a[11], *gate, q, &dh0)))
            return none();
        if (bytes) workspace = at::empty({bytes}, gate->options().dtype(at::kByte));
        for (const at::Tensor &t : {dgate, dx, dh0}) memory.result(t);
        const darb_matrix dm = as_matrix(*dh), gm = as_matrix(*gate), hm = as_matrix(*h), zm = as_matrix(dgate),
                          dxm = as_matrix(dx), d0m = as_matrix(dh0);
        if (x) xm = as_matrix(*x);
        void *w = bytes ? ptr(workspace) : nullptr;
        PyObject *res = held.tuple(3);
        if (!res) return nullptr;
        return finish(res, "darb_gated_recurrence_grad", [&] {
            return darb_gated_recurrence_grad(q.code, q.form, q.H, q.T, q.batch, &dm, &gm, x ? &xm : nullptr, &hm,
                                              q.resets, h0, dl, &zm, &dxm, &d0m, w, bytes, s);
        });
    });
}

// fp32 [n] on the current device; None is none.
bool tokens(PyObject *o, int64_t n, const float **p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = buffer(o, n, at::kFloat);
    if (!t || t->dim() != 1 || t->size(0) != n || !here(*t)) return false;
    *p = static_cast<const float *>(ptr(*t));
    return true;
}

PyObject *tokens_or(PyObject *o, int64_t n, const at::TensorOptions &f32, at::Tensor *out) {
    return given_or(o, out,
                    [&](PyObject *g) -> const at::Tensor * {
                        const float *p;
                        return tokens(g, n, &p) && p ? tensor(g) : nullptr;
                    },
                    [&] { return at::empty({n}, f32); });
}

// (logprob, old, advantage, weight, low, high, ref, kl_coef, entropy, entropy_coef, grad_logprob,
// grad_entropy, stream): (loss, kl, clipped, grad_logprob, grad_entropy)
PyObject *policy_loss(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        void *s;
        const float *lp, *old, *adv, *w, *ref, *ent;
        double k[4];
        int64_t bytes;
        if (n != 13) return none();
        const at::Tensor *t = tensor(a[0]);
        if (!t) return none();
        const int64_t B = t->numel();
        const int at_[4] = {4, 5, 7, 9};
        for (int i = 0; i < 4; ++i) {
            if (!PyFloat_CheckExact(a[at_[i]])) return none();
            k[i] = PyFloat_AS_DOUBLE(a[at_[i]]);
        }
        if (!tokens(a[0], B, &lp) || !tokens(a[1], B, &old) || !tokens(a[2], B, &adv) || !old || !adv ||
            !tokens(a[3], B, &w) || !tokens(a[6], B, &ref) || !tokens(a[8], B, &ent) || !stream_of(a[12], &s) ||
            darb_policy_loss_workspace(B, &bytes) != DARB_OK)
            return none();
        const Memory memory(a[12], s);
        const auto f32 = t->options();
        at::Tensor stats = at::empty({3}, f32), grad, gent, workspace;
        Held held;
        if (!(held.o[0] = tokens_or(a[10], B, f32, &grad))) return none();
        if (ent && !(held.o[1] = tokens_or(a[11], B, f32, &gent))) return none();
        if (bytes) workspace = at::empty({bytes}, f32.dtype(at::kByte));
        for (const at::Tensor &r : {stats, grad, gent}) memory.result(r);
        float *sp = static_cast<float *>(ptr(stats)), *gp = static_cast<float *>(ptr(grad));
        float *ep = ent ? static_cast<float *>(ptr(gent)) : nullptr;
        void *ws = bytes ? ptr(workspace) : nullptr;
        PyObject *res = PyTuple_New(5);
        if (!res) return nullptr;
        {
            // views of a result of no gradient: nothing for automatic differentiation to record
            const at::AutoDispatchBelowADInplaceOrView plain;
            for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(res, i, THPVariable_Wrap(stats.select(0, i)));
        }
        for (int i = 0; i < 2; ++i) {
            PyTuple_SET_ITEM(res, 3 + i, held.o[i] ? held.o[i] : (Py_INCREF(Py_None), Py_None));
            held.o[i] = nullptr;
        }
        return finish(res, "darb_policy_loss", [&] {
            return darb_policy_loss(B, lp, old, adv, w, ref, ent, k[0], k[1], k[2], k[3], sp, gp, ep, ws, bytes, s);
        });
    });
}

// (logprob, ref, batch, starts, beta, smoothing, weight, grad_logprob, stream): (loss, margin,
// grad_logprob)
PyObject *preference_loss(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        void *s;
        const float *lp, *ref, *w;
        if (n != 9) return none();
        const at::Tensor *t = tensor(a[0]);
        if (!t || !PyFloat_CheckExact(a[4]) || !PyFloat_CheckExact(a[5]) || (a[2] == Py_None) == (a[3] == Py_None))
            return none();
        const int64_t B = t->numel();
        const int64_t *starts = nullptr;
        int64_t sequences;
        if (a[3] != Py_None) {
            const at::Tensor *st = tensor(a[3]);
            if (!st || st->scalar_type() != at::kLong || st->dim() != 1 || !st->is_contiguous() || !here(*st))
                return none();
            sequences = st->size(0) - 1;
            starts = static_cast<const int64_t *>(ptr(*st));
        } else {
            if (!PyLong_CheckExact(a[2])) return none();
            sequences = PyLong_AsLongLong(a[2]);
            if (PyErr_Occurred()) {
                PyErr_Clear();
                return none();
            }
            if (sequences > 0 && B % sequences != 0) return none();
        }
        if (sequences < 2 || sequences % 2 != 0 || !tokens(a[0], B, &lp) || !tokens(a[1], B, &ref) ||
            !tokens(a[6], sequences / 2, &w) || !stream_of(a[8], &s))
            return none();
        const int64_t P = sequences / 2;
        const double beta = PyFloat_AS_DOUBLE(a[4]), smoothing = PyFloat_AS_DOUBLE(a[5]);
        const Memory memory(a[8], s);
        at::Tensor out = at::empty({1 + P}, t->options()), grad;
        Held held;
        if (!(held.o[2] = tokens_or(a[7], B, t->options(), &grad))) return none();
        memory.result(out);
        memory.result(grad);
        {
            const at::AutoDispatchBelowADInplaceOrView plain;
            held.o[0] = THPVariable_Wrap(out.select(0, 0));
            held.o[1] = THPVariable_Wrap(out.slice(0, 1, 1 + P));
        }
        float *op = static_cast<float *>(ptr(out)), *gp = static_cast<float *>(ptr(grad));
        PyObject *res = held.tuple(3);
        if (!res) return nullptr;
        return finish(res, "darb_preference_loss", [&] {
            return darb_preference_loss(P, B, lp, ref, starts, w, beta, smoothing, op, op + 1, gp, s);
        });
    });
}

// (handle, M, N, nnz, packed words): what the functions above take as the plan
PyObject *plan_ref(PyObject *, PyObject *args) {
    unsigned long long h;
    long long M, N, nnz, words;
    if (!PyArg_ParseTuple(args, "KLLLL", &h, &M, &N, &nnz, &words)) return nullptr;
    PlanRef *p = new (std::nothrow)
        PlanRef{reinterpret_cast<darb_plan *>(uintptr_t(h)), M, N, nnz, words};
    if (!p) return PyErr_NoMemory();
    PyObject *cap = PyCapsule_New(p, kPlanName, free_ref);
    if (!cap) delete p;
    return cap;
}

// The current stream of the current device.
PyObject *current_stream(PyObject *, PyObject *) {
    return guarded([]() -> PyObject * {
        return PyLong_FromVoidPtr(c10::hip::getCurrentHIPStream().stream());
    });
}

// The package's function that raises for an error code.
PyObject *set_check(PyObject *, PyObject *f) {
    Py_INCREF(f);
    Py_XSETREF(g_check, f);
    Py_RETURN_NONE;
}

#define DARB_FAST(F) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(F)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    DARB_FAST(spmv), DARB_FAST(spmv_packed), DARB_FAST(spmv_i8),
    DARB_FAST(spmm), DARB_FAST(spmm_packed), DARB_FAST(spmm_i8),
    DARB_FAST(encode), DARB_FAST(spmm_grad),
    DARB_FAST(token_logprobs), DARB_FAST(token_logprobs_grad),
    DARB_FAST(layer_norm), DARB_FAST(layer_norm_grad),
    DARB_FAST(adamw_step), DARB_FAST(adamw_moments),
    DARB_FAST(gated_recurrence), DARB_FAST(gated_recurrence_grad),
    DARB_FAST(policy_loss), DARB_FAST(preference_loss),
    {"plan_ref", plan_ref, METH_VARARGS, nullptr},
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    {"set_check", set_check, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_darbcall", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__darbcall() {
    g_stream_attr = PyUnicode_InternFromString("cuda_stream");
    return g_stream_attr ? PyModule_Create(&module) : nullptr;
}
