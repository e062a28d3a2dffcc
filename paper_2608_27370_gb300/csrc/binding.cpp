// binding.cpp -- the Python binding's argument marshalling in native code.
//
// A call through ctypes spends 8-10 us on checking tensors attribute by
// attribute, building structures and asking torch for the stream, against 2.6 us
// in the library (validation, tensor maps, launch); a linear layer on a few
// hundred tokens is bound by that.  Each function here takes the arguments of
// the Python function of the same name, all positional, checks the tensors as
// the Python code does and calls the library: 11.7 -> 3.5 us for
// puro_fp8_quantize, 13.6 -> 3.8 us for puro_fp8_linear_fprop.
//
// Only the ordinary case is handled: plain torch.Tensor objects with storage,
// on CUDA, contiguous, of the expected dtype and not empty, and plain integers
// and floats.  For anything else the function returns None and does nothing,
// and the caller takes its general path, which raises the error or handles the
// case.  Otherwise the result is the library's status code.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "puro_fp8.h"

namespace {

PyObject *operand_type = nullptr;  // the binding's FP8Operand class

// The library's entry points, handed over by the binding (set_library): the
// same library its ctypes calls go to, also where a process holds two copies of
// the package.  Linked by name, the second copy's module got the first one's.
#define PURO_ENTRIES(X)                \
    X(puro_fp8_amax)                   \
    X(puro_fp8_quantize)               \
    X(puro_fp8_quantize_rmsnorm)       \
    X(puro_fp8_quantize_swiglu)        \
    X(puro_fp8_quantize_weights)       \
    X(puro_fp8_linear_fprop)           \
    X(puro_fp8_linear_dgrad)           \
    X(puro_fp8_linear_wgrad)           \
    X(puro_fp8_linear_wgrad_main_grad) \
    X(puro_fp8_linear_backward)        \
    X(puro_fp8_linear_dgrad_quantize)  \
    X(puro_bf16_linear_fprop)          \
    X(puro_bf16_linear_dgrad)          \
    X(puro_bf16_linear_wgrad)          \
    X(puro_fp8_linear_fprop_epilogue)  \
    X(puro_bf16_linear_fprop_epilogue) \
    X(puro_fp8_gated_fprop)            \
    X(puro_bf16_gated_fprop)           \
    X(puro_fp8_quantize_act_backward)  \
    X(puro_act_backward_bf16)          \
    X(puro_fp8_quantize_gated_backward) \
    X(puro_gated_backward_bf16)        \
    X(puro_qk_norm_rope)               \
    X(puro_qk_norm_rope_backward)      \
    X(puro_rope)                       \
    X(puro_rope_backward)              \
    X(puro_rope_tables)
struct Library {
#define PURO_FIELD(name) decltype(&::name) name;
    PURO_ENTRIES(PURO_FIELD)
#undef PURO_FIELD
};
Library lib{};
bool have_library = false;

// `ok` is cleared when an argument is not of the ordinary kind: the call is left to Python.
struct Args {
    PyObject *const *v;
    bool ok = true;
    int device = -1;     // of the first tensor
    bool mixed = false;  // another one's differs

    const at::Tensor *plain(PyObject *o) {
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.numel() == 0) return nullptr;
        if (device < 0) device = t.get_device();
        if (t.get_device() != device) mixed = true;
        return &t;
    }
    // Every tensor so far has to be on one device (the caller has compared the first with the current one).
    void one_device() {
        if (mixed) ok = false;
    }
    // Device pointer of a contiguous tensor of dtype dt or dt2.
    void *ptr_of(PyObject *o, at::ScalarType dt, at::ScalarType dt2) {
        const at::Tensor *t = plain(o);
        if (!t || !t->is_contiguous() || (t->scalar_type() != dt && t->scalar_type() != dt2)) return fail();
        return t->data_ptr();
    }
    void *ptr(int i, at::ScalarType dt) { return ptr_of(v[i], dt, dt); }
    void *opt(int i, at::ScalarType dt) { return v[i] == Py_None ? nullptr : ptr_of(v[i], dt, dt); }
    void *bits(int i) { return ptr_of(v[i], at::kInt, at::kUInt32); }
    void *opt_bits(int i) { return v[i] == Py_None ? nullptr : bits(i); }
    int32_t *status(int i) { return static_cast<int32_t *>(opt(i, at::kInt)); }
    // Scratch of any dtype, and its bytes.
    void *scratch(int i, size_t *bytes) {
        *bytes = 0;
        if (v[i] == Py_None) return nullptr;
        const at::Tensor *t = plain(v[i]);
        if (!t || !t->is_contiguous()) return fail();
        *bytes = t->nbytes();
        return t->data_ptr();
    }
    // Rows and columns of a 2-D tensor.
    void shape(int i, int64_t *rows, int64_t *cols) {
        *rows = *cols = 0;
        if (!ok) return;
        const at::Tensor &t = THPVariable_Unpack(v[i]);
        if (t.dim() != 2) {
            ok = false;
            return;
        }
        *rows = t.size(0);
        *cols = t.size(1);
    }
    int64_t integer_of(PyObject *o) {
        if (!PyLong_CheckExact(o)) return fail(), 0;
        int over = 0;
        const long long x = PyLong_AsLongLongAndOverflow(o, &over);
        if (over) return fail(), 0;
        return x;
    }
    int64_t i64(int i) { return integer_of(v[i]); }
    int32_t i32(int i) {
        const int64_t x = integer_of(v[i]);
        if (x < INT32_MIN || x > INT32_MAX) return fail(), 0;
        return static_cast<int32_t>(x);
    }
    bool flag(int i) {
        if (v[i] != Py_True && v[i] != Py_False) return fail(), false;
        return v[i] == Py_True;
    }
    float f32(int i) {
        if (!PyFloat_CheckExact(v[i])) return fail(), 0.0f;
        return static_cast<float>(PyFloat_AS_DOUBLE(v[i]));
    }
    void *stream(int i) {
        if (!ok) return nullptr;
        if (v[i] == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
        return fail();  // a Stream object or a raw handle
    }
    // An FP8Operand: its codes, scales and enums.
    void operand(int i, puro_fp8_tensor_t *t) {
        *t = puro_fp8_tensor_t{};
        if (reinterpret_cast<PyObject *>(Py_TYPE(v[i])) != operand_type) ok = false;
        static PyObject *names[5] = {
            PyUnicode_InternFromString("data"), PyUnicode_InternFromString("scale"), PyUnicode_InternFromString("fmt"),
            PyUnicode_InternFromString("scaling"), PyUnicode_InternFromString("role")};
        PyObject *f[5] = {};
        for (int k = 0; k < 5 && ok; ++k) {
            f[k] = PyObject_GetAttr(v[i], names[k]);
            if (!f[k]) {
                PyErr_Clear();
                ok = false;
            }
        }
        if (ok) {
            t->data = static_cast<const uint8_t *>(ptr_of(f[0], at::kByte, at::kByte));
            const at::Tensor *s = plain(f[1]);
            if (!s || !s->is_contiguous()) fail();
            if (ok) {
                const at::Tensor &d = THPVariable_Unpack(f[0]);
                if (d.dim() == 2) {
                    t->rows = d.size(0);
                    t->red = d.size(1);
                } else {
                    ok = false;
                }
                t->scale = s->data_ptr();
            }
            const int64_t e[3] = {integer_of(f[2]), integer_of(f[3]), integer_of(f[4])};
            for (int64_t x : e)
                if (x < INT32_MIN || x > INT32_MAX) ok = false;
            t->fmt = static_cast<int32_t>(e[0]);
            t->scaling = static_cast<int32_t>(e[1]);
            t->role = static_cast<int32_t>(e[2]);
        }
        for (PyObject *o : f) Py_XDECREF(o);  // the operand keeps its tensors
    }
    // Heads of tokens: a bf16 view [tokens, heads, channels] with unit channel stride.
    void heads(int i, puro_heads_t *h, int64_t *tokens, int64_t *channels) {
        *h = puro_heads_t{};
        *tokens = *channels = 0;
        const at::Tensor *t = plain(v[i]);
        if (!t || t->scalar_type() != at::kBFloat16 || t->dim() != 3 || t->stride(2) != 1 || t->size(1) > INT32_MAX) {
            ok = false;
            return;
        }
        h->data = t->data_ptr();
        h->token_stride = t->size(0) > 1 ? t->stride(0) : 0;
        h->head_stride = t->size(1) > 1 ? t->stride(1) : 0;
        h->heads = static_cast<int32_t>(t->size(1));
        *tokens = t->size(0);
        *channels = t->size(2);
    }
    // Two tables [positions, pairs] of one shape.
    void tables(int i, const float **co, const float **si, int64_t *positions, int32_t *rot) {
        *co = static_cast<const float *>(ptr_of(v[i], at::kFloat, at::kFloat));
        *si = static_cast<const float *>(ptr_of(v[i + 1], at::kFloat, at::kFloat));
        int64_t r[2] = {}, c[2] = {};
        shape(i, &r[0], &c[0]);
        shape(i + 1, &r[1], &c[1]);
        if (r[0] != r[1] || c[0] != c[1] || c[0] > 1024) ok = false;
        *positions = r[0];
        *rot = static_cast<int32_t>(2 * c[0]);
    }
    // Two bf16 views of one shape and row stride, with unit column stride.
    void gate_up(int i, const void **gate, const void **up, int64_t *rows, int64_t *cols, int64_t *ld) {
        *gate = *up = nullptr;
        *rows = *cols = *ld = 0;
        const at::Tensor *g = plain(v[i]), *u = plain(v[i + 1]);
        if (!g || !u || g->scalar_type() != at::kBFloat16 || u->scalar_type() != at::kBFloat16 || g->dim() != 2 ||
            u->dim() != 2 || g->sizes() != u->sizes() || g->size(0) < 2 || g->stride(1) != 1 || u->stride(1) != 1 ||
            g->stride(0) != u->stride(0)) {
            ok = false;
            return;
        }
        *gate = g->data_ptr();
        *up = u->data_ptr();
        *rows = g->size(0);
        *cols = g->size(1);
        *ld = g->stride(0);
    }
    // An optional bf16 [rows, cols] view with unit column stride, and its row stride.
    const void *rows_of(int i, int64_t rows, int64_t cols, int64_t *ld) {
        *ld = cols;
        if (v[i] == Py_None) return nullptr;
        const at::Tensor *t = plain(v[i]);
        if (!t || t->scalar_type() != at::kBFloat16 || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols ||
            t->stride(1) != 1)
            return fail();
        if (rows > 1) *ld = t->stride(0);
        return t->data_ptr();
    }
    // The scale vectors of an FP8 copy [rows, red] and (optional) of its transpose.
    void scales(int i, int it, int64_t rows, int64_t red) {
        numel(i, rows * ((red / 128 + 3) / 4) * 4);
        numel(it, red * ((rows / 128 + 3) / 4) * 4);
    }
    // A tensor's number of values has to be n.
    void numel(int i, int64_t n) {
        if (ok && v[i] != Py_None && THPVariable_Unpack(v[i]).numel() != n) ok = false;
    }
    std::nullptr_t fail() {
        ok = false;
        return nullptr;
    }
};

// Runs `call` without the GIL when every argument was ordinary.  It touches no
// tensor and must not throw: every pointer and size is taken before.
template <class F>
PyObject *finish(const Args &a, F call) {
    if (!a.ok) Py_RETURN_NONE;
    puro_status_t st;
    Py_BEGIN_ALLOW_THREADS;
    st = call();
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

#define PURO_NATIVE(name, nargs)                                                               \
    PyObject *name(PyObject *, PyObject *const *argv, Py_ssize_t n) {                          \
        if (n != (nargs) || !have_library) Py_RETURN_NONE;                                     \
        Args a{argv};                                                                          \
        try {                                                                                  \
            return name##_call(a);                                                             \
        } catch (const std::exception &) { /* e.g. a tensor whose memory cannot be accessed */ \
            Py_RETURN_NONE;                                                                    \
        }                                                                                      \
    }

constexpr at::ScalarType kBF16 = at::kBFloat16, kU8 = at::kByte, kF32 = at::kFloat;

uint8_t *u8(void *p) { return static_cast<uint8_t *>(p); }

// (x, amax_bits, stream)
PyObject *amax_call(Args &a) {
    const void *x = a.ptr(0, kBF16);
    uint32_t *bits = static_cast<uint32_t *>(a.bits(1));
    int64_t r, c;
    a.shape(0, &r, &c);
    void *s = a.stream(2);
    return finish(a, [&] { return lib.puro_fp8_amax(x, r, c, bits, s); });
}
PURO_NATIVE(amax, 3)

// (x, fmt, scaling, role, amax_bits, q, scale, q_t, scale_t, dev_status, stream)
PyObject *quantize_call(Args &a) {
    const void *x = a.ptr(0, kBF16);
    int64_t r, c;
    a.shape(0, &r, &c);
    const int32_t fmt = a.i32(1), scaling = a.i32(2), role = a.i32(3);
    const at::ScalarType sdt = scaling == PURO_SCALE_BLOCK ? kU8 : kF32;
    const uint32_t *bits = static_cast<const uint32_t *>(a.opt_bits(4));
    uint8_t *q = u8(a.opt(5, kU8)), *qt = u8(a.opt(7, kU8));
    void *sc = a.opt(6, sdt), *sct = a.opt(8, sdt);
    int32_t *st = a.status(9);
    void *s = a.stream(10);
    return finish(a, [&] { return lib.puro_fp8_quantize(x, r, c, fmt, scaling, role, bits, q, sc, qt, sct, st, s); });
}
PURO_NATIVE(quantize, 11)

// (h, gamma, eps, fmt, rstd, y, q, scale, q_t, scale_t, dev_status, stream)
PyObject *quantize_rmsnorm_call(Args &a) {
    const void *h = a.ptr(0, kBF16), *gamma = a.opt(1, kBF16);
    int64_t r, c;
    a.shape(0, &r, &c);
    const float eps = a.f32(2);
    const int32_t fmt = a.i32(3);
    float *rstd = static_cast<float *>(a.opt(4, kF32));
    void *y = a.opt(5, kBF16), *sc = a.opt(7, kU8), *sct = a.opt(9, kU8);
    uint8_t *q = u8(a.opt(6, kU8)), *qt = u8(a.opt(8, kU8));
    int32_t *st = a.status(10);
    void *s = a.stream(11);
    return finish(a, [&] { return lib.puro_fp8_quantize_rmsnorm(h, r, c, gamma, eps, fmt, rstd, y, q, sc, qt, sct, st, s); });
}
PURO_NATIVE(quantize_rmsnorm, 12)

// (gate, up, fmt, y, q, scale, q_t, scale_t, dev_status, stream): gate and up
// share their shape and row stride, with unit column stride
PyObject *quantize_swiglu_call(Args &a) {
    const at::Tensor *g = a.plain(a.v[0]), *u = a.plain(a.v[1]);
    if (!g || !u || g->scalar_type() != kBF16 || u->scalar_type() != kBF16 || g->dim() != 2 || u->dim() != 2 ||
        g->sizes() != u->sizes() || g->size(0) < 2 || g->stride(1) != 1 || u->stride(1) != 1 ||
        g->stride(0) != u->stride(0))
        Py_RETURN_NONE;
    const void *gp = g->data_ptr(), *up = u->data_ptr();
    const int64_t r = g->size(0), c = g->size(1), ld = g->stride(0);
    const int32_t fmt = a.i32(2);
    void *y = a.opt(3, kBF16), *sc = a.opt(5, kU8), *sct = a.opt(7, kU8);
    uint8_t *q = u8(a.opt(4, kU8)), *qt = u8(a.opt(6, kU8));
    int32_t *st = a.status(8);
    void *s = a.stream(9);
    return finish(a, [&] { return lib.puro_fp8_quantize_swiglu(gp, up, r, c, ld, fmt, y, q, sc, qt, sct, st, s); });
}
PURO_NATIVE(quantize_swiglu, 10)

// (address of the table, count, fmt, dev_status, stream)
PyObject *quantize_weights_call(Args &a) {
    const int64_t table = a.i64(0);
    const int32_t count = a.i32(1), fmt = a.i32(2);
    int32_t *st = a.status(3);
    void *s = a.stream(4);
    return finish(a, [&] {
        return lib.puro_fp8_quantize_weights(reinterpret_cast<const puro_fp8_weight_t *>(table), count, fmt, st, s);
    });
}
PURO_NATIVE(quantize_weights, 5)

// (a, b, out, workspace, dev_status, stream)
template <class Fn>
PyObject *gemm(Args &a, Fn fn, at::ScalarType out_dtype) {
    puro_fp8_tensor_t x, w;
    a.operand(0, &x);
    a.operand(1, &w);
    void *out = a.opt(2, out_dtype);
    size_t bytes;
    void *ws = a.scratch(3, &bytes);
    int32_t *st = a.status(4);
    void *s = a.stream(5);
    return finish(a, [&] { return fn(&x, &w, out, ws, bytes, st, s); });
}
PyObject *linear_fprop_call(Args &a) { return gemm(a, lib.puro_fp8_linear_fprop, kBF16); }
PyObject *linear_dgrad_call(Args &a) { return gemm(a, lib.puro_fp8_linear_dgrad, kBF16); }
PyObject *linear_wgrad_call(Args &a) { return gemm(a, lib.puro_fp8_linear_wgrad, kBF16); }
PyObject *linear_wgrad_main_grad_call(Args &a) {
    return gemm(a,
                [](const puro_fp8_tensor_t *x, const puro_fp8_tensor_t *w, void *out, void *ws, size_t bytes, int32_t *st,
                   void *s) {
                    return lib.puro_fp8_linear_wgrad_main_grad(x, w, static_cast<float *>(out), ws, bytes, st, s);
                },
                kF32);
}
PURO_NATIVE(linear_fprop, 6)
PURO_NATIVE(linear_dgrad, 6)
PURO_NATIVE(linear_wgrad, 6)
PURO_NATIVE(linear_wgrad_main_grad, 6)

// (dy, w_t, dx, dy_t, x_t, dw, workspace, dev_status, stream)
PyObject *linear_backward_call(Args &a) {
    puro_fp8_tensor_t dy, wt, dyt, xt;
    a.operand(0, &dy);
    a.operand(1, &wt);
    void *dx = a.opt(2, kBF16);
    a.operand(3, &dyt);
    a.operand(4, &xt);
    void *dw = a.opt(5, kBF16);
    size_t bytes;
    void *ws = a.scratch(6, &bytes);
    int32_t *st = a.status(7);
    void *s = a.stream(8);
    return finish(a, [&] { return lib.puro_fp8_linear_backward(&dy, &wt, dx, &dyt, &xt, dw, ws, bytes, st, s); });
}
PURO_NATIVE(linear_backward, 9)

// (dy, w_t, fmt, dx, dxq, dxq_scale, dxq_t, dxq_t_scale, dev_status, stream)
PyObject *linear_dgrad_quantize_call(Args &a) {
    puro_fp8_tensor_t dy, wt;
    a.operand(0, &dy);
    a.operand(1, &wt);
    const int32_t fmt = a.i32(2);
    void *dx = a.opt(3, kBF16), *sc = a.opt(5, kU8), *sct = a.opt(7, kU8);
    uint8_t *q = u8(a.opt(4, kU8)), *qt = u8(a.opt(6, kU8));
    int32_t *st = a.status(8);
    void *s = a.stream(9);
    return finish(a, [&] { return lib.puro_fp8_linear_dgrad_quantize(&dy, &wt, fmt, dx, q, sc, qt, sct, st, s); });
}
PURO_NATIVE(linear_dgrad_quantize, 10)

// (a, b, out, M, N, K, dev_status, stream)
template <class Fn>
PyObject *bf16(Args &a, Fn fn) {
    const void *x = a.opt(0, kBF16), *w = a.opt(1, kBF16);
    void *out = a.opt(2, kBF16);
    const int64_t M = a.i64(3), N = a.i64(4), K = a.i64(5);
    int32_t *st = a.status(6);
    void *s = a.stream(7);
    return finish(a, [&] { return fn(x, w, out, M, N, K, st, s); });
}
PyObject *bf16_fprop_call(Args &a) { return bf16(a, lib.puro_bf16_linear_fprop); }
PyObject *bf16_dgrad_call(Args &a) { return bf16(a, lib.puro_bf16_linear_dgrad); }
PyObject *bf16_wgrad_call(Args &a) { return bf16(a, lib.puro_bf16_linear_wgrad); }
PURO_NATIVE(bf16_fprop, 8)
PURO_NATIVE(bf16_dgrad, 8)
PURO_NATIVE(bf16_wgrad, 8)

// (x, w, y, bias, act, residual, z, workspace, dev_status, stream)
PyObject *linear_fprop_epilogue_call(Args &a) {
    puro_fp8_tensor_t x, w;
    a.operand(0, &x);
    a.operand(1, &w);
    void *y = a.ptr(2, kBF16), *z = a.opt(6, kBF16);
    const void *bias = a.opt(3, kBF16);
    const int32_t act = a.i32(4);
    int64_t ld;
    const void *res = a.rows_of(5, x.rows, w.rows, &ld);
    size_t bytes;
    void *ws = a.scratch(7, &bytes);
    int32_t *st = a.status(8);
    void *s = a.stream(9);
    for (int i : {2, 6}) a.numel(i, x.rows * w.rows);
    a.numel(3, w.rows);
    a.one_device();
    return finish(a, [&] { return lib.puro_fp8_linear_fprop_epilogue(&x, &w, bias, act, res, ld, z, y, ws, bytes, st, s); });
}
PURO_NATIVE(linear_fprop_epilogue, 10)

// (x, w, y, bias, act, residual, z, dev_status, stream)
PyObject *bf16_fprop_epilogue_call(Args &a) {
    const void *x = a.ptr(0, kBF16), *w = a.ptr(1, kBF16), *bias = a.opt(3, kBF16);
    void *y = a.ptr(2, kBF16), *z = a.opt(6, kBF16);
    int64_t M, K, N, K2, ld;
    a.shape(0, &M, &K);
    a.shape(1, &N, &K2);
    if (K != K2) a.ok = false;
    const int32_t act = a.i32(4);
    const void *res = a.rows_of(5, M, N, &ld);
    int32_t *st = a.status(7);
    void *s = a.stream(8);
    for (int i : {2, 6}) a.numel(i, M * N);
    a.numel(3, N);
    a.one_device();
    return finish(a, [&] { return lib.puro_bf16_linear_fprop_epilogue(x, w, M, N, K, bias, act, res, ld, z, y, st, s); });
}
PURO_NATIVE(bf16_fprop_epilogue, 9)

// (x, w, act, fmt, gate_up, h, hq, hq_scale, hq_t, hq_t_scale, dev_status, stream)
PyObject *gated_fprop_call(Args &a) {
    puro_fp8_tensor_t x, w;
    a.operand(0, &x);
    a.operand(1, &w);
    const int32_t act = a.i32(2), fmt = a.i32(3);
    void *gu = a.opt(4, kBF16), *h = a.opt(5, kBF16), *sc = a.opt(7, kU8), *sct = a.opt(9, kU8);
    uint8_t *q = u8(a.opt(6, kU8)), *qt = u8(a.opt(8, kU8));
    int32_t *st = a.status(10);
    void *s = a.stream(11);
    a.numel(4, x.rows * w.rows);
    for (int i : {5, 6, 8}) a.numel(i, x.rows * (w.rows / 2));
    a.scales(7, 9, x.rows, w.rows / 2);
    a.one_device();
    return finish(a, [&] { return lib.puro_fp8_gated_fprop(&x, &w, act, fmt, gu, h, q, sc, qt, sct, st, s); });
}
PURO_NATIVE(gated_fprop, 12)

// (x, w, act, gate_up, h, dev_status, stream)
PyObject *bf16_gated_fprop_call(Args &a) {
    const void *x = a.ptr(0, kBF16), *w = a.ptr(1, kBF16);
    int64_t M, K, N, K2;
    a.shape(0, &M, &K);
    a.shape(1, &N, &K2);
    if (K != K2 || N % 2) a.ok = false;
    const int32_t act = a.i32(2);
    void *gu = a.opt(3, kBF16), *h = a.ptr(4, kBF16);
    int32_t *st = a.status(5);
    void *s = a.stream(6);
    a.numel(3, M * N);
    a.numel(4, M * (N / 2));
    a.one_device();
    return finish(a, [&] { return lib.puro_bf16_gated_fprop(x, w, M, N / 2, K, act, gu, h, st, s); });
}
PURO_NATIVE(bf16_gated_fprop, 7)

// (dy, z, act, fmt, dz, dbias, workspace, q, scale, q_t, scale_t, dev_status, stream)
PyObject *quantize_act_backward_call(Args &a) {
    const void *dy = a.ptr(0, kBF16), *z = a.opt(1, kBF16);
    int64_t r, c;
    a.shape(0, &r, &c);
    const int32_t act = a.i32(2), fmt = a.i32(3);
    void *dz = a.opt(4, kBF16);
    float *db = static_cast<float *>(a.opt(5, kF32));
    size_t bytes;
    void *ws = a.scratch(6, &bytes);
    uint8_t *q = u8(a.opt(7, kU8)), *qt = u8(a.opt(9, kU8));
    void *sc = a.opt(8, kU8), *sct = a.opt(10, kU8);
    int32_t *st = a.status(11);
    void *s = a.stream(12);
    for (int i : {1, 4, 7, 9}) a.numel(i, r * c);
    a.numel(5, c);
    a.scales(8, 10, r, c);
    a.one_device();
    return finish(a, [&] {
        return lib.puro_fp8_quantize_act_backward(dy, z, r, c, act, fmt, dz, db, ws, bytes, q, sc, qt, sct, st, s);
    });
}
PURO_NATIVE(quantize_act_backward, 13)

// (dy, z, act, dz, dbias, workspace, stream)
PyObject *act_backward_bf16_call(Args &a) {
    const void *dy = a.ptr(0, kBF16), *z = a.opt(1, kBF16);
    int64_t r, c;
    a.shape(0, &r, &c);
    const int32_t act = a.i32(2);
    void *dz = a.opt(3, kBF16);
    float *db = static_cast<float *>(a.opt(4, kF32));
    size_t bytes;
    void *ws = a.scratch(5, &bytes);
    void *s = a.stream(6);
    for (int i : {1, 3}) a.numel(i, r * c);
    a.numel(4, c);
    a.one_device();
    return finish(a, [&] { return lib.puro_act_backward_bf16(dy, z, r, c, act, dz, db, ws, bytes, s); });
}
PURO_NATIVE(act_backward_bf16, 7)

// (dh, gate, up, act, fmt, dgate_up, q, scale, q_t, scale_t, dev_status, stream)
PyObject *quantize_gated_backward_call(Args &a) {
    const void *dh = a.ptr(0, kBF16), *g, *u;
    int64_t r, c, ld, dr, dc;
    a.gate_up(1, &g, &u, &r, &c, &ld);
    a.shape(0, &dr, &dc);
    if (dr != r || dc != c) a.ok = false;
    const int32_t act = a.i32(3), fmt = a.i32(4);
    void *dgu = a.opt(5, kBF16), *sc = a.opt(7, kU8), *sct = a.opt(9, kU8);
    uint8_t *q = u8(a.opt(6, kU8)), *qt = u8(a.opt(8, kU8));
    int32_t *st = a.status(10);
    void *s = a.stream(11);
    for (int i : {5, 6, 8}) a.numel(i, 2 * r * c);
    a.scales(7, 9, r, 2 * c);
    a.one_device();
    return finish(a, [&] {
        return lib.puro_fp8_quantize_gated_backward(dh, g, u, r, c, ld, act, fmt, dgu, q, sc, qt, sct, st, s);
    });
}
PURO_NATIVE(quantize_gated_backward, 12)

// (dh, gate, up, act, dgate_up, stream)
PyObject *gated_backward_bf16_call(Args &a) {
    const void *dh = a.ptr(0, kBF16), *g, *u;
    int64_t r, c, ld, dr, dc;
    a.gate_up(1, &g, &u, &r, &c, &ld);
    a.shape(0, &dr, &dc);
    if (dr != r || dc != c) a.ok = false;
    const int32_t act = a.i32(3);
    void *dgu = a.ptr(4, kBF16);
    void *s = a.stream(5);
    a.numel(4, 2 * r * c);
    a.one_device();
    return finish(a, [&] { return lib.puro_gated_backward_bf16(dh, g, u, r, c, ld, act, dgu, s); });
}
PURO_NATIVE(gated_backward_bf16, 6)

// (q, k, q_gain, k_gain, eps, cos, sin, positions, interleaved, q_out, k_out,
// rstd, dev_status, stream)
PyObject *qk_norm_rope_call(Args &a) {
    puro_heads_t q, k, qo, ko;
    int64_t t[4], d[4], positions;
    a.heads(0, &q, &t[0], &d[0]);
    a.heads(1, &k, &t[1], &d[1]);
    const void *gq = a.opt(2, kBF16), *gk = a.opt(3, kBF16);
    const float eps = a.f32(4);
    const float *co, *si;
    int32_t rot;
    a.tables(5, &co, &si, &positions, &rot);
    const int32_t *pos = static_cast<const int32_t *>(a.opt(7, at::kInt));
    const bool inter = a.flag(8);
    a.heads(9, &qo, &t[2], &d[2]);
    a.heads(10, &ko, &t[3], &d[3]);
    float *rstd = static_cast<float *>(a.opt(11, kF32));
    int32_t *st = a.status(12);
    void *s = a.stream(13);
    for (int i = 1; i < 4; ++i)
        if (t[i] != t[0] || d[i] != d[0]) a.ok = false;
    a.numel(2, d[0]);
    a.numel(3, d[0]);
    a.numel(7, t[0]);
    a.numel(11, t[0] * (q.heads + k.heads));
    if (d[0] > 1024) a.ok = false;
    a.one_device();
    return finish(a, [&] {
        return lib.puro_qk_norm_rope(&q, &k, t[0], static_cast<int32_t>(d[0]), gq, gk, eps, co, si, positions, rot, inter, pos,
                                     &qo, &ko, rstd, st, s);
    });
}
PURO_NATIVE(qk_norm_rope, 14)

// (dq_out, dk_out, q, k, rstd, q_gain, k_gain, cos, sin, positions, interleaved,
// dq, dk, dq_gain, dk_gain, workspace, dev_status, stream)
PyObject *qk_norm_rope_backward_call(Args &a) {
    puro_heads_t h[6];
    int64_t t[6], d[6], positions;
    const int at_arg[6] = {0, 1, 2, 3, 11, 12};
    for (int i = 0; i < 6; ++i) a.heads(at_arg[i], &h[i], &t[i], &d[i]);
    const float *rstd = static_cast<const float *>(a.ptr(4, kF32));
    const void *gq = a.opt(5, kBF16), *gk = a.opt(6, kBF16);
    const float *co, *si;
    int32_t rot;
    a.tables(7, &co, &si, &positions, &rot);
    const int32_t *pos = static_cast<const int32_t *>(a.opt(9, at::kInt));
    const bool inter = a.flag(10);
    float *dgq = static_cast<float *>(a.opt(13, kF32)), *dgk = static_cast<float *>(a.opt(14, kF32));
    size_t bytes;
    void *ws = a.scratch(15, &bytes);
    int32_t *st = a.status(16);
    void *s = a.stream(17);
    for (int i = 1; i < 6; ++i)
        if (t[i] != t[0] || d[i] != d[0]) a.ok = false;
    a.numel(4, t[0] * (h[2].heads + h[3].heads));
    for (int i : {5, 6, 13, 14}) a.numel(i, d[0]);
    a.numel(9, t[0]);
    if (d[0] > 1024) a.ok = false;
    a.one_device();
    return finish(a, [&] {
        return lib.puro_qk_norm_rope_backward(&h[0], &h[1], &h[2], &h[3], rstd, t[0], static_cast<int32_t>(d[0]), gq, gk, co,
                                              si, positions, rot, inter, pos, &h[4], &h[5], dgq, dgk, ws, bytes, st, s);
    });
}
PURO_NATIVE(qk_norm_rope_backward, 18)

// (q, k, frequencies, positions, interleaved, q_out, k_out, scale, stream)
template <class Entry>
PyObject *rope_of(Args &a, Entry Library::*entry) {
    puro_heads_t q, k, qo, ko;
    int64_t t[4], d[4];
    a.heads(0, &q, &t[0], &d[0]);
    a.heads(1, &k, &t[1], &d[1]);
    const uint64_t *freq = static_cast<const uint64_t *>(a.ptr(2, at::kLong));
    const int64_t pairs = a.ok ? THPVariable_Unpack(a.v[2]).numel() : 0;
    const int32_t *pos = static_cast<const int32_t *>(a.opt(3, at::kInt));
    const bool inter = a.flag(4);
    a.heads(5, &qo, &t[2], &d[2]);
    a.heads(6, &ko, &t[3], &d[3]);
    const float scale = a.f32(7);
    void *s = a.stream(8);
    for (int i = 1; i < 4; ++i)
        if (t[i] != t[0] || d[i] != d[0]) a.ok = false;
    a.numel(3, t[0]);
    if (d[0] > 1024 || pairs > 1024) a.ok = false;
    a.one_device();
    return finish(a, [&] {
        return (lib.*entry)(&q, &k, t[0], static_cast<int32_t>(d[0]), freq, static_cast<int32_t>(2 * pairs), scale, inter, pos, &qo,
                            &ko, s);
    });
}
PyObject *rope_call(Args &a) { return rope_of(a, &Library::puro_rope); }
PURO_NATIVE(rope, 9)
PyObject *rope_backward_call(Args &a) { return rope_of(a, &Library::puro_rope_backward); }
PURO_NATIVE(rope_backward, 9)

// (frequencies, first, cos, sin, scale, stream)
PyObject *rope_tables_call(Args &a) {
    const uint64_t *freq = static_cast<const uint64_t *>(a.ptr(0, at::kLong));
    const int64_t pairs = a.ok ? THPVariable_Unpack(a.v[0]).numel() : 0, first = a.i64(1);
    float *co = static_cast<float *>(a.ptr(2, kF32)), *si = static_cast<float *>(a.ptr(3, kF32));
    int64_t rows[2], cols[2];
    a.shape(2, &rows[0], &cols[0]);
    a.shape(3, &rows[1], &cols[1]);
    const float scale = a.f32(4);
    void *s = a.stream(5);
    if (cols[0] != pairs || cols[1] != pairs || rows[0] != rows[1] || pairs > 1024) a.ok = false;
    a.one_device();
    return finish(a, [&] { return lib.puro_rope_tables(freq, static_cast<int32_t>(2 * pairs), scale, first, rows[0], co, si, s); });
}
PURO_NATIVE(rope_tables, 6)

// (the FP8Operand class)
PyObject *set_operand_type(PyObject *, PyObject *const *argv, Py_ssize_t n) {
    if (n != 1) {
        PyErr_SetString(PyExc_TypeError, "set_operand_type takes one class");
        return nullptr;
    }
    Py_INCREF(argv[0]);
    Py_XDECREF(operand_type);
    operand_type = argv[0];
    Py_RETURN_NONE;
}

// (name -> address of each entry point)
PyObject *set_library(PyObject *, PyObject *const *argv, Py_ssize_t n) {
    if (n != 1 || !PyDict_Check(argv[0])) {
        PyErr_SetString(PyExc_TypeError, "set_library takes one dict");
        return nullptr;
    }
    Library l{};
#define PURO_TAKE(name)                                                                    \
    {                                                                                      \
        PyObject *o = PyDict_GetItemString(argv[0], #name);                                \
        void *p = o ? PyLong_AsVoidPtr(o) : nullptr;                                       \
        if (!p) {                                                                          \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address of " #name); \
            return nullptr;                                                                \
        }                                                                                  \
        l.name = reinterpret_cast<decltype(l.name)>(p);                                    \
    }
    PURO_ENTRIES(PURO_TAKE)
#undef PURO_TAKE
    lib = l;
    have_library = true;
    Py_RETURN_NONE;
}

#define PURO_METHOD(py, fn) {py, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PURO_METHOD("set_operand_type", set_operand_type),
                         PURO_METHOD("set_library", set_library),
                         PURO_METHOD("puro_fp8_amax", amax),
                         PURO_METHOD("puro_fp8_quantize", quantize),
                         PURO_METHOD("puro_fp8_quantize_rmsnorm", quantize_rmsnorm),
                         PURO_METHOD("puro_fp8_quantize_swiglu", quantize_swiglu),
                         PURO_METHOD("puro_fp8_quantize_weights", quantize_weights),
                         PURO_METHOD("puro_fp8_linear_fprop", linear_fprop),
                         PURO_METHOD("puro_fp8_linear_dgrad", linear_dgrad),
                         PURO_METHOD("puro_fp8_linear_wgrad", linear_wgrad),
                         PURO_METHOD("puro_fp8_linear_wgrad_main_grad", linear_wgrad_main_grad),
                         PURO_METHOD("puro_fp8_linear_backward", linear_backward),
                         PURO_METHOD("puro_fp8_linear_dgrad_quantize", linear_dgrad_quantize),
                         PURO_METHOD("puro_bf16_linear_fprop", bf16_fprop),
                         PURO_METHOD("puro_bf16_linear_dgrad", bf16_dgrad),
                         PURO_METHOD("puro_bf16_linear_wgrad", bf16_wgrad),
                         PURO_METHOD("puro_fp8_linear_fprop_epilogue", linear_fprop_epilogue),
                         PURO_METHOD("puro_bf16_linear_fprop_epilogue", bf16_fprop_epilogue),
                         PURO_METHOD("puro_fp8_gated_fprop", gated_fprop),
                         PURO_METHOD("puro_bf16_gated_fprop", bf16_gated_fprop),
                         PURO_METHOD("puro_fp8_quantize_act_backward", quantize_act_backward),
                         PURO_METHOD("puro_act_backward_bf16", act_backward_bf16),
                         PURO_METHOD("puro_fp8_quantize_gated_backward", quantize_gated_backward),
                         PURO_METHOD("puro_gated_backward_bf16", gated_backward_bf16),
                         PURO_METHOD("puro_qk_norm_rope", qk_norm_rope),
                         PURO_METHOD("puro_qk_norm_rope_backward", qk_norm_rope_backward),
                         PURO_METHOD("puro_rope", rope),
                         PURO_METHOD("puro_rope_backward", rope_backward),
                         PURO_METHOD("puro_rope_tables", rope_tables),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Native argument marshalling of the Python binding.", -1, methods};

}  // namespace

// (native_for: the torch and the interpreter it was compiled for)
PyMODINIT_FUNC PyInit__native() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "native_for", PURO_NATIVE_FOR) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
