// The binding's test of one tensor argument, for lynx.py: a call makes up to 21
// of them, and a short kernel waits for the host.  In Python a test is five
// attribute reads, 0.6 us; here it is one call, 0.1.
//
//   typed(fn, what, t, nbytes, dtype, device) -> the pointer of tensor t
//
// None and ints pass through.  Anything that is not a contiguous tensor of that
// dtype on that device with nbytes bytes at least goes to the Python form of the
// test (set by `otherwise`), which says what is wrong.
//
// Whole calls, tests and C entry point, of the operators whose kernels are shorter
// than that (norms and rotation of one token: 8.6 us a call by typed() and ctypes, 4.6
// so; the launch is 3):
//
//   attn_hier, qk_norm_rope, blocks_extend, blocks_release
//       (address of the entry point, device, stream, the binding's arguments)
//       -> its status, or None where an argument does not pass: the binding's own
//       form then says what is wrong
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <algorithm>
#include <initializer_list>

namespace {

PyObject *g_otherwise = nullptr;

PyObject *typed(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "typed takes 6 arguments");
        return nullptr;
    }
    PyObject *t = args[2];
    if (t == Py_None || PyLong_CheckExact(t)) {
        Py_INCREF(t);
        return t;
    }
    if (THPVariable_Check(t) && THPDtype_Check(args[4]) && PyLong_Check(args[3]) && PyLong_Check(args[5])) {
        int over = 0, over_dev = 0;
        const long long nbytes = PyLong_AsLongLongAndOverflow(args[3], &over);
        const long dev = PyLong_AsLongAndOverflow(args[5], &over_dev);
        const at::Tensor &x = THPVariable_Unpack(t);
        try {
            if (!over && !over_dev && x.layout() == c10::kStrided && x.is_cuda() && x.get_device() == dev &&
                x.scalar_type() == reinterpret_cast<THPDtype *>(args[4])->scalar_type && x.is_contiguous() &&
                (long long)x.nbytes() >= nbytes)
                return PyLong_FromVoidPtr(x.data_ptr());
        } catch (const std::exception &) {  // (a tensor without storage: the Python form raises)
        }
    }
    if (!g_otherwise) {
        PyErr_SetString(PyExc_RuntimeError, "otherwise() has not been called");
        return nullptr;
    }
    return PyObject_Vectorcall(g_otherwise, args, n, nullptr);
}

// ---- whole calls ----
constexpr long long kHeadDim = 128;

// Arguments of one call.  `ok` falls where one is not what the call takes.
struct Call {
    PyObject *const *args;
    Py_ssize_t n;
    long dev = 0;
    bool ok = true;

    // An integer of 64 bits, or of 32.
    long long i64(PyObject *x) {
        if (!x || !(PyLong_Check(x) || PyIndex_Check(x))) {
            ok = false;
            return 0;
        }
        int over = 0;
        const long long v = PyLong_AsLongLongAndOverflow(x, &over);
        if (over || (v == -1 && PyErr_Occurred())) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    int32_t i32(PyObject *x) {
        const long long v = i64(x);
        if (v < INT32_MIN || v > INT32_MAX) ok = false;
        return (int32_t)v;
    }
    float f32(PyObject *x) {
        const double v = PyFloat_AsDouble(x);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return (float)v;
    }
    int32_t truth(PyObject *x) {
        const int v = PyObject_IsTrue(x);
        if (v < 0) {
            PyErr_Clear();
            ok = false;
        }
        return v > 0;
    }
    void *pointer(PyObject *x) { return x == Py_None ? nullptr : reinterpret_cast<void *>((uintptr_t)i64(x)); }
    const at::Tensor *of_type(PyObject *x, c10::ScalarType type) {
        if (!THPVariable_Check(x)) {
            ok = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(x);
        if (t.layout() != c10::kStrided || !t.is_cuda() || t.get_device() != dev || t.scalar_type() != type) {
            ok = false;
            return nullptr;
        }
        return &t;
    }
    // A contiguous tensor of nbytes at least; None is NULL, an int a pointer.
    void *tensor(PyObject *x, long long nbytes, c10::ScalarType type) {
        if (x == Py_None || PyLong_CheckExact(x)) return pointer(x);
        const at::Tensor *t = of_type(x, type);
        if (!t) return nullptr;
        if (!t->is_contiguous() || (long long)t->nbytes() < nbytes) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    // BF16 heads [tokens][heads][128], which may be part of a wider row.
    void *heads(PyObject *x, long long tokens, long long &n_heads, int64_t &stride) {
        const at::Tensor *t = of_type(x, c10::kBFloat16);
        if (!t) return nullptr;
        if (t->dim() != 3 || t->size(0) != tokens || t->size(2) != kHeadDim || t->stride(2) != 1 ||
            (t->stride(1) != kHeadDim && t->size(1) > 1)) {
            ok = false;
            return nullptr;
        }
        n_heads = t->size(1);
        stride = t->stride(0);
        if (tokens == 1) stride = std::max<int64_t>(stride, n_heads * kHeadDim) / 8 * 8;
        return t->data_ptr();
    }
    PyObject *attribute(PyObject *x, PyObject *name) {
        PyObject *v = PyObject_GetAttr(x, name);
        if (!v) {
            PyErr_Clear();
            ok = false;
        }
        return v;  // a new reference
    }
};

// lynx_layout's seven fields, in its order, and their names.
constexpr int kLayoutFields = 7, kMetaFields = 8;
const char *const kLayoutNames[kLayoutFields] = {"num_kv_heads", "head_dim", "k_group_tokens", "block_tokens",
                                                 "max_blocks_per_seq", "num_blocks", "max_tokens"};
const char *const kMetaNames[kMetaFields] = {"k_gmin", "k_gscale", "k_mu", "k_sigma", "v_gmin", "v_gscale", "v_mu", "v_sigma"};
PyObject *g_layout[kLayoutFields], *g_meta[kMetaFields];

struct Layout {
    int32_t kv_heads, head_dim, k_group, block_tokens, max_blocks, num_blocks, max_tokens;
};
Layout layout_of(Call &c, PyObject *x) {
    int32_t v[kLayoutFields] = {};
    for (int i = 0; i < kLayoutFields && c.ok; ++i) {
        PyObject *f = c.attribute(x, g_layout[i]);
        if (f) v[i] = c.i32(f);
        Py_XDECREF(f);
    }
    return {v[0], v[1], v[2], v[3], v[4], v[5], v[6]};
}

// Runs f where every argument passed; tensors that cannot say where they are (no
// storage) throw, and go to the binding's own form too.
template <typename F>
PyObject *whole_call(PyObject *const *args, Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "a whole call has another number of arguments");
        return nullptr;
    }
    Call c{args, n};
    int status = 0;
    try {
        c.dev = (long)c.i64(args[1]);
        if (c.ok) status = f(c);
    } catch (const std::exception &) {
        c.ok = false;
    }
    if (!c.ok) Py_RETURN_NONE;
    return PyLong_FromLong(status);
}
// The entry point itself, other threads running meanwhile.
template <typename Fn, typename... A>
int enter(PyObject *address, Call &c, Fn *, A... a) {
    Fn *fn = reinterpret_cast<Fn *>((uintptr_t)c.i64(address));
    if (!c.ok) return 0;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = fn(a...);
    Py_END_ALLOW_THREADS;
    return status;
}
long long positive(long long x) { return std::max(x, 0ll); }
// A size in bytes that no tensor has where the product passes 64 bits.
long long product(std::initializer_list<long long> factors) {
    long long p = 1;
    for (const long long f : factors)
        if (__builtin_mul_overflow(p, f, &p)) return INT64_MAX;
    return p;
}

constexpr auto kI32 = c10::kInt;
constexpr auto kF32 = c10::kFloat;
constexpr auto kU8 = c10::kByte;
constexpr auto kBF16 = c10::kBFloat16;

PyObject *attn_hier(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return whole_call(a, n, 22, [&](Call &c) {
        void *stream = c.pointer(a[2]);
        const Layout L = layout_of(c, a[3]);
        const int32_t B = c.i32(a[4]), Hq = c.i32(a[5]), k = c.i32(a[6]), most = c.i32(a[7]);
        const long long nb = positive(B), heads = nb * L.kv_heads, io = product({nb, positive(k), Hq, kHeadDim * 2});
        const int32_t full = c.truth(a[10]);
        const long long plane = product({L.num_blocks, L.kv_heads, L.block_tokens, full ? 128 : 64});
        void *lens = c.tensor(a[8], nb * 4, kI32), *table = c.tensor(a[9], product({nb, L.max_blocks, 4}), kI32);
        void *kp = c.tensor(a[11], plane, kU8), *vp = c.tensor(a[12], plane, kU8);
        const float alpha = c.f32(a[13]);
        const int32_t variant = c.i32(a[14]);
        void *meta[kMetaFields];
        for (int i = 0; i < kMetaFields && c.ok; ++i) {
            PyObject *f = c.attribute(a[15], g_meta[i]);
            const int per = kMetaNames[i][2] == 'g' ? 256 : 32;
            if (f) meta[i] = c.tensor(f, product({heads, (L.max_tokens + (long long)per - 1) / per, kHeadDim * 4}), kF32);
            Py_XDECREF(f);
        }
        void *q = c.tensor(a[16], io, kBF16);
        int32_t n_tail = 0;
        void *tail[2] = {nullptr, nullptr};
        if (a[17] == Py_None || a[18] == Py_None) {
            if (a[17] != a[18]) c.ok = false;
        } else if (const at::Tensor *t = c.of_type(a[17], kBF16)) {
            if (t->dim() != 4 || t->size(1) > INT32_MAX) {
                c.ok = false;
            } else {
                n_tail = (int32_t)t->size(1);
                for (int i = 0; i < 2; ++i) tail[i] = c.tensor(a[17 + i], product({heads, n_tail, kHeadDim * 2}), kBF16);
            }
        }
        void *out = c.tensor(a[19], io, kBF16), *lse = c.tensor(a[20], product({nb, positive(k), Hq, 4}), kF32);
        if (PyLong_CheckExact(a[21])) c.ok = false;  // (its size is not known)
        void *ws = c.tensor(a[21], 0, kU8);
        if (!c.ok) return 0;
        const size_t nws = a[21] == Py_None ? 0 : THPVariable_Unpack(a[21]).nbytes();
        using Fn = int(const Layout *, int32_t, int32_t, int32_t, int32_t, void *, void *, int32_t, void *, void *, float,
                       int32_t, void *, void *, int32_t, void *, void *, void *, void *, void *, size_t, void *);
        return enter(a[0], c, (Fn *)nullptr, &L, B, Hq, k, most, lens, table, full, kp, vp, alpha, variant, (void *)meta, q,
                     n_tail, tail[0], tail[1], out, lse, ws, nws, stream);
    });
}

PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return whole_call(a, n, 17, [&](Call &c) {
        void *stream = c.pointer(a[2]);
        const at::Tensor *first = c.of_type(a[3], kBF16);
        if (!first || first->dim() != 3 || first->size(0) > INT32_MAX) {
            c.ok = false;
            return 0;
        }
        const long long tokens = first->size(0);
        long long H[3] = {0, 0, 0};
        int64_t stride[3] = {0, 0, 0};
        void *x[3] = {nullptr, nullptr, nullptr};
        for (int i = 0; i < 3; ++i)
            if (i < 2 || a[5] != Py_None) x[i] = c.heads(a[3 + i], tokens, H[i], stride[i]);
        if (!c.ok || (x[2] && H[2] != H[1]) || H[0] < 1 || H[0] > INT32_MAX || H[1] > INT32_MAX ||
            (a[5] == Py_None) != (a[16] == Py_None) || !THPVariable_Check(a[14])) {
            c.ok = false;
            return 0;
        }
        const long long n_rows = THPVariable_Unpack(a[14]).numel() / (H[0] * kHeadDim);
        if (n_rows > INT32_MAX) c.ok = false;
        void *positions = c.tensor(a[6], tokens * 4, kI32), *rows = c.tensor(a[7], tokens * 4, kI32);
        void *qw = c.tensor(a[8], kHeadDim * 2, kBF16), *kw = c.tensor(a[9], kHeadDim * 2, kBF16);
        const float eps = c.f32(a[10]);
        int64_t rotary = 0;
        void *freq = nullptr;
        if (a[11] != Py_None) {
            const at::Tensor *t = c.of_type(a[11], kF32);
            if (!t || !t->is_contiguous() || t->numel() > kHeadDim) {
                c.ok = false;
                return 0;
            }
            rotary = 2 * t->numel();
            freq = t->data_ptr();
        }
        const int32_t pairs = c.truth(a[12]);
        const float scale = c.f32(a[13]);
        void *out[3];
        for (int i = 0; i < 3; ++i) out[i] = c.tensor(a[14 + i], i == 0 ? 0 : product({n_rows, H[1], kHeadDim * 2}), kBF16);
        if (!c.ok) return 0;
        using Fn = int(int32_t, int32_t, int32_t, int32_t, void *, int64_t, void *, int64_t, void *, int64_t, void *, void *,
                       int32_t, void *, void *, float, void *, int32_t, int32_t, float, void *, void *, void *, void *);
        return enter(a[0], c, (Fn *)nullptr, (int32_t)tokens, (int32_t)H[0], (int32_t)H[1], (int32_t)kHeadDim, x[0], stride[0],
                     x[1], stride[1], x[2], stride[2], positions, rows, (int32_t)n_rows, qw, kw, eps, freq, (int32_t)rotary,
                     pairs, scale, out[0], out[1], out[2], stream);
    });
}

PyObject *blocks_extend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return whole_call(a, n, 17, [&](Call &c) {
        void *stream = c.pointer(a[2]);
        const Layout L = layout_of(c, a[3]);
        const int32_t B = c.i32(a[4]), n_src = c.i32(a[5]);
        const long long nb = positive(B);
        void *lens = c.tensor(a[6], nb * 4, kI32), *counts = c.tensor(a[7], nb * 4, kI32);
        void *table = c.tensor(a[8], product({nb, L.max_blocks, 4}), kI32);
        void *stack = c.tensor(a[9], (long long)L.num_blocks * 4, kI32), *state = c.tensor(a[10], 8, kI32);
        void *granted = c.tensor(a[11], nb * 4, kI32), *starts = c.tensor(a[12], (nb + 1) * 4, kI32);
        long long rows = -1;
        for (int i = 13; i < 17; ++i)
            if (a[i] != Py_None) {
                if (!THPVariable_Check(a[i])) {
                    c.ok = false;
                    return 0;
                }
                const long long have = THPVariable_Unpack(a[i]).numel();
                rows = rows < 0 ? have : std::min(rows, have);
            }
        if (rows < 0) rows = std::min(nb * positive(n_src), 1ll << 30);
        if (rows > INT32_MAX) c.ok = false;
        void *out[4];
        for (int i = 0; i < 4; ++i) out[i] = c.tensor(a[13 + i], rows * 4, kI32);
        if (!c.ok) return 0;
        using Fn = int(const Layout *, int32_t, int32_t, int32_t, void *, void *, void *, void *, void *, void *, void *,
                       void *, void *, void *, void *, void *);
        return enter(a[0], c, (Fn *)nullptr, &L, B, n_src, (int32_t)rows, lens, counts, table, stack, state, granted, starts,
                     out[0], out[1], out[2], out[3], stream);
    });
}

PyObject *blocks_release(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return whole_call(a, n, 10, [&](Call &c) {
        void *stream = c.pointer(a[2]);
        const Layout L = layout_of(c, a[3]);
        const int32_t B = c.i32(a[4]);
        const long long nb = positive(B);
        void *lens = c.tensor(a[5], nb * 4, kI32), *keep = c.tensor(a[6], nb * 4, kI32);
        void *table = c.tensor(a[7], product({nb, L.max_blocks, 4}), kI32);
        void *stack = c.tensor(a[8], (long long)L.num_blocks * 4, kI32), *state = c.tensor(a[9], 8, kI32);
        if (!c.ok) return 0;
        using Fn = int(const Layout *, int32_t, void *, void *, void *, void *, void *, void *);
        return enter(a[0], c, (Fn *)nullptr, &L, B, lens, keep, table, stack, state, stream);
    });
}

PyObject *otherwise(PyObject *, PyObject *f) {
    Py_INCREF(f);
    Py_XSETREF(g_otherwise, f);
    Py_RETURN_NONE;
}

#define LYNX_FASTCALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    LYNX_FASTCALL(typed), LYNX_FASTCALL(attn_hier), LYNX_FASTCALL(qk_norm_rope), LYNX_FASTCALL(blocks_extend),
    LYNX_FASTCALL(blocks_release),
    {"otherwise", otherwise, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__args() {
    for (int i = 0; i < kLayoutFields; ++i)
        if (!(g_layout[i] = PyUnicode_InternFromString(kLayoutNames[i]))) return nullptr;
    for (int i = 0; i < kMetaFields; ++i)
        if (!(g_meta[i] = PyUnicode_InternFromString(kMetaNames[i]))) return nullptr;
    return PyModule_Create(&module);
}
