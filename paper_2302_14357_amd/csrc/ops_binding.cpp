// Python's way to the operators of an autoregressive model: checks of tensors, outputs and workspaces, and the calls of include/tbs.h on
// the current stream.  Host code only.  It exists because of what a call costs: the same through ctypes took 8 (linear) to 26
// (beam_reorder) us, as long as the smaller kernels themselves.
#include <torch/extension.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPStream.h>
#include <c10/hip/HIPGuard.h>

#include <optional>
#include <sstream>
#include <stdexcept>

#include "tbs.h"

namespace {

using at::Tensor;

// raised as ValueError
struct Bad : std::invalid_argument {
    using std::invalid_argument::invalid_argument;
};
#define WANT(ok, ...)                   \
    do {                                \
        if (!(ok)) {                    \
            std::ostringstream text;    \
            text << __VA_ARGS__;        \
            throw Bad(text.str());      \
        }                               \
    } while (0)

// the library's error code; raised by what ops.py gave (TbsError)
struct Refused {
    int code;
};
PyObject *g_raise = nullptr;

// whether the caller records gradients (the calls themselves do not)
bool g_grad = false;

const Tensor *tensor(PyObject *o, const char *name, bool may_lack = false) {
    if (o == Py_None && may_lack) return nullptr;
    WANT(THPVariable_Check(o), name << " has to be a tensor");
    const Tensor &t = THPVariable_Unpack(o);
    WANT(!g_grad || !t.requires_grad(), name << " requires a gradient, and this operator has none: call it under torch.no_grad(), or on a detached tensor");
    return &t;
}

int32_t dtype_of(const Tensor &t, const char *name) {
    switch (t.scalar_type()) {
        case at::kFloat: return TBS_F32;
        case at::kBFloat16: return TBS_BF16;
        case at::kHalf: return TBS_F16;
        default: WANT(false, name << " is " << t.scalar_type() << ": float32, bfloat16 or float16 is wanted");
    }
    return -1;
}

void on(const Tensor &t, const char *name, const at::Device &d) { WANT(t.device() == d, name << " is on " << t.device() << ", not on " << d); }

at::Device gpu(const Tensor &t) {
    WANT(t.is_cuda(), "the tensors have to be on the GPU: this library has no CPU path");
    return t.device();
}

int32_t number(PyObject *o, const char *name) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        WANT(false, name << " has to be a whole number");
    }
    WANT(v >= INT32_MIN && v <= INT32_MAX, name << " = " << v << " is no 32-bit number");
    return (int32_t)v;
}

int32_t size32(int64_t v, const char *name) {
    WANT(v <= INT32_MAX, name << " = " << v << " is too large");
    return (int32_t)v;
}

Tensor made(at::IntArrayRef shape, at::ScalarType type, const at::Device &d) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(d));
}

// 2-D, a row's elements side by side: its row stride (of one row: any)
int64_t rows_of(const Tensor &t, const char *name, int64_t rows, int64_t cols) {
    WANT(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, name << " has shape " << t.sizes() << ": [" << rows << ", " << cols << "] is wanted");
    WANT(cols <= 1 || t.stride(1) == 1, name << ": elements of a row have to lie side by side");
    return rows > 1 ? t.stride(0) : cols;
}

void *vector_of(const Tensor &t, const char *name, int64_t rows, at::ScalarType type, const at::Device &d) {
    WANT(t.scalar_type() == type && t.dim() == 1 && t.size(0) == rows && (rows <= 1 || t.stride(0) == 1),
         name << " has shape " << t.sizes() << " and " << t.scalar_type() << ": [" << rows << "] in " << type << ", contiguous, is wanted");
    on(t, name, d);
    return t.data_ptr();
}

const uint8_t *flags_of(const Tensor *t, int64_t rows, const at::Device &d) {
    return t ? (const uint8_t *)vector_of(*t, "finished", rows, t->scalar_type() == at::kByte ? at::kByte : at::kBool, d) : nullptr;
}

// [rows, heads, dim], a head's elements side by side (strides of one row or one head: any)
void heads_of(const Tensor &t, const char *name, int64_t rows, int64_t heads, int64_t dim, at::ScalarType type, const at::Device &d, int64_t &row, int64_t &head) {
    WANT(t.dim() == 3 && t.size(0) == rows && t.size(1) == heads && t.size(2) == dim && t.scalar_type() == type,
         name << " has shape " << t.sizes() << " and " << t.scalar_type() << ": [" << rows << ", " << heads << ", " << dim << "] in " << type << " is wanted");
    WANT(t.stride(2) == 1 || dim <= 1, name << ": elements of a head have to lie side by side");
    on(t, name, d);
    row = rows > 1 ? t.stride(0) : heads * dim;
    head = heads > 1 ? t.stride(1) : dim;
}

// [pages, page, heads, dim] (a stride that nothing is reached by says nothing)
void cache_of(const Tensor &t, const char *name, at::ScalarType type, const at::Device &d, int64_t &page, int64_t &token, int64_t &head) {
    WANT(t.dim() == 4 && t.scalar_type() == type, name << " has shape " << t.sizes() << " and " << t.scalar_type() << ": [pages, page, heads, dim] in " << type << " is wanted");
    WANT(t.stride(3) == 1 || t.size(3) <= 1, name << ": elements of a head have to lie side by side");
    on(t, name, d);
    page = t.size(0) > 1 ? t.stride(0) : t.numel();
    token = t.size(1) > 1 ? t.stride(1) : t.size(2) * t.size(3);
    head = t.size(2) > 1 ? t.stride(2) : t.size(3);
}

template <class Args>
void call(int (*fn)(const Args *, void *), const Args &a, const at::Device &d) {
    const c10::hip::HIPGuard guard(d.index());
    const int rc = fn(&a, (void *)c10::hip::getCurrentHIPStream(d.index()).stream());
    if (rc) throw Refused{rc};
}

// A tensor of the caller's was written: autograd sees that what it had kept of it is gone (a tensor made in inference mode has no version)
void written(const Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A call's workspace, kept until it is enqueued (the allocator hands its memory on in the order of the stream).
template <class Args>
Tensor workspace(int64_t (*fn)(const Args *), Args &a, const at::Device &d) {
    const int64_t n = fn(&a);
    if (n < 0) throw Refused{(int)n};
    if (n == 0) return Tensor();
    Tensor t = made({n}, at::kByte, d);
    a.workspace = t.data_ptr();
    a.workspace_bytes = n;
    return t;
}

template <class F>
PyObject *guarded(F f) {
    try {
        g_grad = at::GradMode::is_enabled();
        const at::NoGradGuard no_grad;
        return f();
    } catch (const Refused &r) {
        PyObject *x = PyObject_CallFunction(g_raise, "i", r.code);
        Py_XDECREF(x);
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "the library refused the call");
    } catch (const Bad &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

#define ARGS(n) \
    WANT(nargs == (n), "wrong number of arguments")

// x, weight, bias, act, residual, out, float32 result (None: as out or x)
PyObject *py_linear(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject * {
        ARGS(7);
        const Tensor &x = *tensor(o[0], "x"), &w = *tensor(o[1], "weight");
        const Tensor *bias = tensor(o[2], "bias", true), *residual = tensor(o[4], "residual", true), *out = tensor(o[5], "out", true);
        WANT(w.dim() == 2 && x.dim() >= 1, "x [..., K] and weight [N, K] are wanted");
        tbs_linear_args a = {};
        a.dtype = dtype_of(x, "x");
        a.act = number(o[3], "act");
        const int64_t n = w.size(0), k = w.size(1);
        WANT(x.size(-1) == k && w.scalar_type() == x.scalar_type(),
             "x has " << x.size(-1) << " columns in " << x.scalar_type() << ", weight " << k << " in " << w.scalar_type());
        const at::Device d = gpu(x);
        on(w, "weight", d);
        const at::ScalarType kind = o[6] == Py_True ? at::kFloat : o[6] == Py_False ? x.scalar_type() : out ? out->scalar_type() : x.scalar_type();
        WANT(kind == x.scalar_type() || kind == at::kFloat, "the result in " << kind << ": x's type or float32 is wanted");
        a.out_dtype = kind == at::kFloat ? (int32_t)TBS_F32 : a.dtype;
        c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = n;
        const Tensor x2 = x.dim() == 2 ? x : x.reshape({-1, k});
        const int64_t m = x2.size(0);
        Tensor result, o2, r2;
        if (out) {
            WANT(out->scalar_type() == kind && out->sizes() == at::IntArrayRef(shape),
                 "out has shape " << out->sizes() << " and " << out->scalar_type() << ": " << at::IntArrayRef(shape) << " in " << kind << " is wanted");
            on(*out, "out", d);
            result = *out;
            o2 = out->dim() == 2 ? *out : out->view({-1, n});
        } else {
            result = made(shape, kind, d);
            o2 = result.dim() == 2 ? result : result.view({-1, n});
        }
        a.ld_out = rows_of(o2, "out", m, n);
        if (residual) {
            WANT(residual->scalar_type() == kind && residual->sizes() == at::IntArrayRef(shape),
                 "residual has shape " << residual->sizes() << " and " << residual->scalar_type() << ": " << at::IntArrayRef(shape) << " in " << kind << " is wanted");
            on(*residual, "residual", d);
            r2 = residual->dim() == 2 ? *residual : residual->reshape({-1, n});
            a.residual = r2.data_ptr();
            a.ld_residual = rows_of(r2, "residual", m, n);
        }
        if (bias) a.bias = (const float *)vector_of(*bias, "bias", n, at::kFloat, d);
        if (m > 0) {
            a.x = x2.data_ptr(), a.w = w.data_ptr(), a.out = o2.data_ptr();
            a.ld_x = rows_of(x2, "x", m, k), a.ld_w = rows_of(w, "weight", n, k);
            a.m = size32(m, "rows"), a.n = size32(n, "N"), a.k = size32(k, "K");
            call(tbs_linear, a, d);
        }
        if (out) {
            written(*out);
            Py_INCREF(o[5]);
            return o[5];
        }
        return THPVariable_Wrap(std::move(result));
    });
}

// q, k_cache, v_cache, tables, lens, k_new, v_new, scale, beams, max_len, out
PyObject *py_attend(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject * {
        ARGS(11);
        const Tensor &q = *tensor(o[0], "q"), &kc = *tensor(o[1], "k_cache"), &vc = *tensor(o[2], "v_cache"), &tables = *tensor(o[3], "tables"), &lens = *tensor(o[4], "lens");
        const Tensor *kn = tensor(o[5], "k_new", true), *vn = tensor(o[6], "v_new", true), *out = tensor(o[10], "out", true);
        tbs_attend_args a = {};
        a.dtype = dtype_of(q, "q");
        const at::ScalarType kind = q.scalar_type();
        WANT(q.dim() == 3 && kc.dim() == 4 && tables.dim() == 2, "q [rows, heads, dim], k_cache [pages, page, kv_heads, dim] and tables [rows, table width] are wanted");
        const int64_t rows = q.size(0), heads = q.size(1), dim = q.size(2), kv = kc.size(2);
        WANT(kc.size(3) == dim && vc.sizes() == kc.sizes(), "q has heads of " << dim << ", k_cache is " << kc.sizes() << ", v_cache " << vc.sizes());
        WANT(tables.scalar_type() == at::kInt, "tables is " << tables.scalar_type() << ": int32 is wanted");
        WANT(!kn == !vn, "k_new and v_new belong together");
        const at::Device d = gpu(q);
        on(tables, "tables", d);
        heads_of(q, "q", rows, heads, dim, kind, d, a.q_row, a.q_head);
        cache_of(kc, "k_cache", kind, d, a.k_page, a.k_token, a.k_head);
        cache_of(vc, "v_cache", kind, d, a.v_page, a.v_token, a.v_head);
        if (kn) {
            heads_of(*kn, "k_new", rows, kv, dim, kind, d, a.k_new_row, a.k_new_head);
            heads_of(*vn, "v_new", rows, kv, dim, kind, d, a.v_new_row, a.v_new_head);
            a.k_new = kn->data_ptr(), a.v_new = vn->data_ptr();
        }
        a.ld_tables = rows_of(tables, "tables", rows, tables.size(1));
        a.lens = (const int32_t *)vector_of(lens, "lens", rows, at::kInt, d);
        Tensor result = out ? *out : made({rows, heads, dim}, kind, d);
        heads_of(result, "out", rows, heads, dim, kind, d, a.out_row, a.out_head);
        a.q = q.data_ptr(), a.k_cache = kc.data_ptr(), a.v_cache = vc.data_ptr(), a.tables = (const int32_t *)tables.data_ptr(), a.out = result.data_ptr();
        a.rows = size32(rows, "rows"), a.heads = size32(heads, "heads"), a.kv_heads = size32(kv, "kv_heads"), a.dim = size32(dim, "dim");
        a.page = size32(kc.size(1), "page"), a.pages = size32(kc.size(0), "pages"), a.table_width = size32(tables.size(1), "table width");
        a.max_len = o[9] == Py_None ? 0 : number(o[9], "max_len");
        a.beams = number(o[8], "beams");
        if (o[7] != Py_None) {
            const double s = PyFloat_AsDouble(o[7]);
            if (s == -1.0 && PyErr_Occurred()) {
                PyErr_Clear();
                WANT(false, "scale has to be a number");
            }
            WANT((float)s != 0.f, "scale has to be other than 0");
            a.scale = (float)s;
        }
        if (rows > 0) {
            const Tensor work = workspace(tbs_attend_workspace, a, d);
            call(tbs_attend_paged, a, d);
            if (kn) written(kc), written(vc);
        }
        if (out) {
            written(*out);
            Py_INCREF(o[10]);
            return o[10];
        }
        return THPVariable_Wrap(std::move(result));
    });
}

PyObject *tuple_of(std::initializer_list<Tensor> list) {
    PyObject *t = PyTuple_New((Py_ssize_t)list.size());
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    for (const Tensor &x : list) {
        PyObject *p = THPVariable_Wrap(x);
        if (!p) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i++, p);
    }
    return t;
}

// logits, scores, beams, finished, eos
PyObject *py_select(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject * {
        ARGS(5);
        const Tensor &logits = *tensor(o[0], "logits"), &scores = *tensor(o[1], "scores");
        const Tensor *finished = tensor(o[3], "finished", true);
        tbs_beam_select_args a = {};
        a.dtype = dtype_of(logits, "logits");
        WANT(logits.dim() == 2, "logits [rows, vocabulary] is wanted");
        const int64_t rows = logits.size(0);
        const at::Device d = gpu(logits);
        a.scores = (const double *)vector_of(scores, "scores", rows, at::kDouble, d);
        a.finished = flags_of(finished, rows, d);
        a.ld_logits = rows_of(logits, "logits", rows, logits.size(1));
        a.rows = size32(rows, "rows"), a.beams = number(o[2], "beams"), a.vocab = size32(logits.size(1), "vocabulary"), a.eos = number(o[4], "eos");
        Tensor s = made({rows}, at::kDouble, d), t = made({rows}, at::kInt, d), p = made({rows}, at::kInt, d), f = made({rows}, at::kBool, d);
        if (rows > 0) {
            a.logits = logits.data_ptr();
            a.out_scores = (double *)s.data_ptr(), a.out_tokens = (int32_t *)t.data_ptr(), a.out_parents = (int32_t *)p.data_ptr(), a.out_finished = (uint8_t *)f.data_ptr();
            const Tensor work = workspace(tbs_beam_select_workspace, a, d);
            call(tbs_beam_select, a, d);
        }
        return tuple_of({s, t, p, f});
    });
}

// parents, tables, lens, caches, beams, finished, appended, status
PyObject *py_reorder(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
    return guarded([&]() -> PyObject * {
        ARGS(8);
        const Tensor &parents = *tensor(o[0], "parents"), &tables = *tensor(o[1], "tables"), &lens = *tensor(o[2], "lens");
        const Tensor *finished = tensor(o[5], "finished", true), *status = tensor(o[7], "status", true);
        const int appended = PyObject_IsTrue(o[6]);
        if (appended < 0) PyErr_Clear();
        WANT(appended >= 0, "appended has to be True or False");
        const at::Device d = parents.device();
        WANT(tables.dim() == 2 && tables.scalar_type() == at::kInt, "tables [rows, table width] in int32 is wanted");
        const int64_t rows = tables.size(0), width = tables.size(1);
        on(tables, "tables", d);
        // a list or tuple of tensors, or one tensor with their number in front
        c10::SmallVector<void *, 64> ptrs;
        Tensor first;
        auto caches = [&](auto f) {   // of a list or tuple, or the one
            if (THPVariable_Check(o[3])) f(THPVariable_Unpack(o[3]));
            else
                for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(o[3]); ++i) f(THPVariable_Unpack(PySequence_Fast_GET_ITEM(o[3], i)));
        };
        if (THPVariable_Check(o[3])) {
            const Tensor &all = *tensor(o[3], "caches");
            WANT(all.dim() == 5 && all.size(0) > 0, "caches has shape " << all.sizes() << ": [caches, pages, page, kv_heads, dim] is wanted");
            first = all.select(0, 0);
            for (int64_t i = 0; i < all.size(0); ++i) ptrs.push_back((char *)all.data_ptr() + i * all.stride(0) * all.element_size());
        } else {
            WANT(PyList_Check(o[3]) || PyTuple_Check(o[3]), "caches has to be a list of tensors or a tensor");
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(o[3]);
            WANT(n > 0, "caches: one at least is wanted");
            PyObject **items = PySequence_Fast_ITEMS(o[3]);
            first = *tensor(items[0], "caches[0]");
            for (Py_ssize_t i = 0; i < n; ++i) {
                const Tensor &c = *tensor(items[i], "a cache");
                WANT(c.sizes() == first.sizes() && c.strides() == first.strides() && c.scalar_type() == first.scalar_type() && c.device() == d,
                     "the caches have to be alike in shape, strides and type, on the device of the tables");
                ptrs.push_back(c.data_ptr());
            }
        }
        gpu(parents);
        tbs_beam_reorder_args a = {};
        a.dtype = dtype_of(first, "caches");
        cache_of(first, "caches", first.scalar_type(), d, a.cache_page, a.cache_token, a.cache_head);
        a.pages = size32(first.size(0), "pages"), a.page = size32(first.size(1), "page"), a.kv_heads = size32(first.size(2), "kv_heads"), a.dim = size32(first.size(3), "dim");
        a.parents = (const int32_t *)vector_of(parents, "parents", rows, at::kInt, d);
        a.lens = (const int32_t *)vector_of(lens, "lens", rows, at::kInt, d);
        a.finished = flags_of(finished, rows, d);
        a.ld_tables = rows_of(tables, "tables", rows, width);
        a.ld_out_tables = width;
        if (status) {
            WANT(status->scalar_type() == at::kInt && status->numel() == 1, "status: one number in int32 is wanted");
            on(*status, "status", d);
            a.status = (int32_t *)status->data_ptr();
        }
        a.rows = size32(rows, "rows"), a.beams = number(o[4], "beams"), a.table_width = size32(width, "table width");
        a.appended = appended;
        Tensor t = made({rows, width}, at::kInt, d), n = made({rows}, at::kInt, d);
        if (rows > 0) {
            a.tables = (const int32_t *)tables.data_ptr(), a.out_tables = (int32_t *)t.data_ptr(), a.out_lens = (int32_t *)n.data_ptr();
            for (size_t i = 0; i < ptrs.size(); i += TBS_MAX_CACHES) {   // (every launch writes the same tables)
                a.caches = ptrs.data() + i;
                a.n_caches = (int32_t)std::min<size_t>(ptrs.size() - i, TBS_MAX_CACHES);
                if (i) a.status = nullptr;
                call(tbs_beam_reorder, a, d);
            }
            caches(written);
            if (status) written(*status);
        }
        return tuple_of({t, n});
    });
}

PyObject *py_raise_by(PyObject *, PyObject *f) {
    Py_XDECREF(g_raise);
    Py_INCREF(f);
    g_raise = f;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"linear", (PyCFunction)(void *)py_linear, METH_FASTCALL, nullptr},
                         {"attend_paged", (PyCFunction)(void *)py_attend, METH_FASTCALL, nullptr},
                         {"beam_select", (PyCFunction)(void *)py_select, METH_FASTCALL, nullptr},
                         {"beam_reorder", (PyCFunction)(void *)py_reorder, METH_FASTCALL, nullptr},
                         {"raise_by", py_raise_by, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tbs_ops", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tbs_ops(void) { return PyModule_Create(&module); }
