// CPython extension of the binding: reads the tensors of a call and calls the C
// ABI of liblsgd.so. Every function returns the call's lsgd_status, or None
// where an argument is anything but what the call plainly takes (another type
// or dtype, another device, not contiguous, another size, a tensor subclass
// with its own dispatch, ...): the caller then takes the general Python path,
// which checks each argument and raises its error. Reading 130 tensors' dtype,
// device, size, layout and address from Python cost 80 to 90 us of a 95 us
// call; here it is 3 to 4.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "layers/lsgd_layers.h"
#include "lsgd.h"
#include "marshal_call.h"

namespace {

// A plain dense GPU tensor, or null: a torch.Tensor or Parameter itself, as a
// subclass may answer for its address, size or dtype with __torch_function__.
const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.unsafeGetTensorImpl()->is_python_dispatch() ||
        t.is_conj() || t.is_neg() || !t.is_contiguous())
        return nullptr;
    return &t;
}

// A plain tensor of `dtype` with n elements (n < 0: any) on device `dev`.
const at::Tensor* plain(PyObject* o, at::ScalarType dtype, int64_t n, int dev) {
    const at::Tensor* t = plain(o);
    return t && t->scalar_type() == dtype && (n < 0 || t->numel() == n) && t->get_device() == dev ? t : nullptr;
}

// Addresses of a list or tuple of n-element tensors of one dtype (float32 or
// bfloat16; 0 entries: float32). False where it is anything else.
bool addresses(PyObject* seq, int64_t n, int dev, void** out, int most, int* count, lsgd_dtype* dt) {
    if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(seq);
    if (k > most) return false;
    at::ScalarType type = at::kFloat;
    for (Py_ssize_t i = 0; i < k; ++i) {
        PyObject* o = PySequence_Fast_GET_ITEM(seq, i);
        if (i == 0) {
            const at::Tensor* t = plain(o);
            if (!t) return false;
            type = t->scalar_type();
            if (type != at::kFloat && type != at::kBFloat16) return false;
        }
        const at::Tensor* t = plain(o, type, n, dev);
        if (!t) return false;
        out[i] = t->data_ptr();
    }
    *count = static_cast<int>(k);
    *dt = type == at::kBFloat16 ? LSGD_BF16 : LSGD_F32;
    return true;
}

bool small_int(PyObject* o, int32_t* out) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v < INT32_MIN || v > INT32_MAX) return false;
    *out = static_cast<int32_t>(v);
    return true;
}

// group_of_worker of exactly `count` entries.
bool membership(PyObject* seq, int count, int32_t* out) {
    if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) return false;
    if (PySequence_Fast_GET_SIZE(seq) != count) return false;
    for (int i = 0; i < count; ++i)
        if (!small_int(PySequence_Fast_GET_ITEM(seq, i), &out[i])) return false;
    return true;
}

bool number(PyObject* o, float* out) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) {   // an int beyond the double range
        PyErr_Clear();
        return false;
    }
    *out = static_cast<float>(v);
    return true;
}

void* stream_of(PyObject* o) { return PyLong_AsVoidPtr(o); }

// A C++ exception of a tensor accessor (a tensor without storage): the general
// path meets the same tensor and reports it. (without_gil lets none of the
// library's through.)
template <typename Body>
PyObject* guarded(const Body& body) {
    try {
        return body();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// step(params, momentum, grads, gow, n_groups, lr, mu, wd, replicas, reduction,
//      broadcast, lr_device or None, device, stream)
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        if (na != 14) Py_RETURN_NONE;
        int32_t dev, groups, reduction, bcast;
        const at::Tensor* p = plain(a[0]);
        if (!p || !small_int(a[12], &dev) || !(p = plain(a[0], at::kFloat, -1, dev))) Py_RETURN_NONE;
        const int64_t n = p->numel();
        const at::Tensor* m = plain(a[1], at::kFloat, n, dev);
        void *grads[LSGD_MAX_WORKERS], *reps[LSGD_MAX_REPLICAS];
        int32_t gow[LSGD_MAX_WORKERS];
        int N, R;
        lsgd_dtype gdt, rdt;
        float lr, mu, wd;
        if (!m || !addresses(a[2], n, dev, grads, LSGD_MAX_WORKERS, &N, &gdt) || !membership(a[3], N, gow) ||
            !small_int(a[4], &groups) || !number(a[5], &lr) || !number(a[6], &mu) || !number(a[7], &wd) ||
            !addresses(a[8], n, dev, reps, LSGD_MAX_REPLICAS, &R, &rdt) || !small_int(a[9], &reduction) ||
            !small_int(a[10], &bcast))
            Py_RETURN_NONE;
        lsgd_step_options o = {reduction, bcast, nullptr};
        if (a[11] != Py_None) {
            const at::Tensor* l = plain(a[11], at::kFloat, -1, dev);
            if (!l || l->numel() < 1) Py_RETURN_NONE;
            o.lr_device = static_cast<const float*>(l->data_ptr());
        }
        float* pp = static_cast<float*>(p->data_ptr());
        float* mp = static_cast<float*>(m->data_ptr());
        void* stream = stream_of(a[13]);
        return without_gil([&] {
            return lsgd_step_ex(pp, mp, grads, gdt, N, gow, groups, n, lr, mu, wd, reps, R, rdt, &o, stream);
        });
    });
}

// group_mean(grads, gow, n_groups, out, device, stream)
PyObject* group_mean(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev, groups;
        if (na != 6 || !small_int(a[2], &groups) || !small_int(a[4], &dev)) Py_RETURN_NONE;
        if ((!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) || PySequence_Fast_GET_SIZE(a[0]) < 1) Py_RETURN_NONE;
        const at::Tensor* first = plain(PySequence_Fast_GET_ITEM(a[0], 0));
        if (!first) Py_RETURN_NONE;
        const int64_t n = first->numel();
        void *grads[LSGD_MAX_WORKERS], *out[LSGD_MAX_WORKERS];
        int32_t gow[LSGD_MAX_WORKERS];
        int N, G;
        lsgd_dtype gdt, odt;
        if (!addresses(a[0], n, dev, grads, LSGD_MAX_WORKERS, &N, &gdt) || !membership(a[1], N, gow) ||
            !addresses(a[3], n, dev, out, LSGD_MAX_WORKERS, &G, &odt) || G != groups || odt != LSGD_F32)
            Py_RETURN_NONE;
        void* stream = stream_of(a[5]);
        return without_gil([&] {
            return lsgd_group_mean(grads, gdt, N, gow, groups, n, reinterpret_cast<float* const*>(out), stream);
        });
    });
}

// global_mean(means, out, device, stream)
PyObject* global_mean(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        if (na != 4 || !small_int(a[2], &dev)) Py_RETURN_NONE;
        const at::Tensor* out = plain(a[1], at::kFloat, -1, dev);
        if (!out) Py_RETURN_NONE;
        const int64_t n = out->numel();
        void* in[LSGD_MAX_WORKERS];
        int G;
        lsgd_dtype dt;
        if (!addresses(a[0], n, dev, in, LSGD_MAX_WORKERS, &G, &dt) || dt != LSGD_F32) Py_RETURN_NONE;
        float* op = static_cast<float*>(out->data_ptr());
        void* stream = stream_of(a[3]);
        return without_gil([&] { return lsgd_global_mean(reinterpret_cast<const float* const*>(in), G, n, op, stream); });
    });
}

// sgd_step(params, momentum, grad_mean, lr, mu, wd, replicas, device, stream)
PyObject* sgd_step(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        if (na != 9 || !small_int(a[7], &dev)) Py_RETURN_NONE;
        const at::Tensor* p = plain(a[0], at::kFloat, -1, dev);
        if (!p) Py_RETURN_NONE;
        const int64_t n = p->numel();
        const at::Tensor *m = plain(a[1], at::kFloat, n, dev), *g = plain(a[2], at::kFloat, n, dev);
        void* reps[LSGD_MAX_REPLICAS];
        int R;
        lsgd_dtype rdt;
        float lr, mu, wd;
        if (!m || !g || !number(a[3], &lr) || !number(a[4], &mu) || !number(a[5], &wd) ||
            !addresses(a[6], n, dev, reps, LSGD_MAX_REPLICAS, &R, &rdt))
            Py_RETURN_NONE;
        float *pp = static_cast<float*>(p->data_ptr()), *mp = static_cast<float*>(m->data_ptr());
        const float* gp = static_cast<const float*>(g->data_ptr());
        void* stream = stream_of(a[8]);
        return without_gil([&] { return lsgd_sgd_step(pp, mp, gp, n, lr, mu, wd, reps, R, rdt, stream); });
    });
}

// copy_out(params, replicas, device, stream)
PyObject* copy_out(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        if (na != 4 || !small_int(a[2], &dev)) Py_RETURN_NONE;
        const at::Tensor* p = plain(a[0], at::kFloat, -1, dev);
        if (!p) Py_RETURN_NONE;
        const int64_t n = p->numel();
        void* reps[LSGD_MAX_REPLICAS];
        int R;
        lsgd_dtype rdt;
        if (!addresses(a[1], n, dev, reps, LSGD_MAX_REPLICAS, &R, &rdt)) Py_RETURN_NONE;
        const float* pp = static_cast<const float*>(p->data_ptr());
        void* stream = stream_of(a[3]);
        return without_gil([&] { return lsgd_copy_out(pp, n, reps, R, rdt, stream); });
    });
}

// ---- the layer operators ----

bool float_dtype(const at::Tensor& t, lsgd_dtype* dt) {
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) return false;
    *dt = t.scalar_type() == at::kBFloat16 ? LSGD_BF16 : LSGD_F32;
    return true;
}
bool index_type(const at::Tensor& t, lsgd_index_type* it) {
    if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) return false;
    *it = t.scalar_type() == at::kLong ? LSGD_I64 : LSGD_I32;
    return true;
}
// A plain tensor on device `dev` (of n elements, n < 0: any), float32 or bfloat16.
const at::Tensor* floats(PyObject* o, int64_t n, int dev, lsgd_dtype* dt) {
    const at::Tensor* t = plain(o);
    return t && t->get_device() == dev && (n < 0 || t->numel() == n) && float_dtype(*t, dt) ? t : nullptr;
}
// A tensor as a matrix of its last dimension.
bool matrix(const at::Tensor& t, int64_t* rows, int64_t* cols) {
    if (t.dim() < 1) return false;
    *cols = t.size(-1);
    *rows = 1;
    for (int64_t i = 0; i + 1 < t.dim(); ++i) *rows *= t.size(i);
    return true;
}
// Codes or scales: `type` or uint8, n bytes (n < 0: any).
const at::Tensor* bytes8(PyObject* o, at::ScalarType type, int64_t n, int dev) {
    const at::Tensor* t = plain(o);
    return t && t->get_device() == dev && (n < 0 || t->numel() == n) &&
                   (t->scalar_type() == type || t->scalar_type() == at::kByte)
               ? t
               : nullptr;
}
constexpr at::ScalarType kCodes = at::ScalarType::Float8_e4m3fn, kScales = at::ScalarType::Float8_e8m0fnu;
int64_t blocks(int64_t n, int64_t of) { return (n + of - 1) / of; }

// embed_lookup(table, tokens, out, scale, device, stream)
PyObject* embed_lookup(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        lsgd_dtype tdt, odt;
        lsgd_index_type it;
        float scale;
        int64_t rows, dim;
        if (na != 6 || !small_int(a[4], &dev) || !number(a[3], &scale)) Py_RETURN_NONE;
        const at::Tensor *table = floats(a[0], -1, dev, &tdt), *tokens = plain(a[1]);
        if (!table || !matrix(*table, &rows, &dim) || !tokens || tokens->get_device() != dev || !index_type(*tokens, &it))
            Py_RETURN_NONE;
        const int64_t n = tokens->numel();
        const at::Tensor* out = floats(a[2], n * dim, dev, &odt);
        if (!out) Py_RETURN_NONE;
        const void *tp = table->data_ptr(), *kp = tokens->data_ptr();
        void *op = out->data_ptr(), *stream = stream_of(a[5]);
        return without_gil(
            [&] { return lsgd_embed_lookup(tp, tdt, rows, dim, kp, it, n, scale, op, odt, stream); });
    });
}

// embed_grad(grads, tokens, out, scale, accumulate, device, stream): the
// workspace is torch's, on the current stream, which has to be `stream`
PyObject* embed_grad(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev, accumulate;
        lsgd_dtype gdt, odt;
        lsgd_index_type it = LSGD_I32;
        float scale;
        int64_t rows, dim;
        if (na != 7 || !small_int(a[5], &dev) || !number(a[3], &scale) || !small_int(a[4], &accumulate)) Py_RETURN_NONE;
        const at::Tensor* out = floats(a[2], -1, dev, &odt);
        if (!out || !matrix(*out, &rows, &dim) || (!PyList_CheckExact(a[1]) && !PyTuple_CheckExact(a[1]))) Py_RETURN_NONE;
        const Py_ssize_t k = PySequence_Fast_GET_SIZE(a[1]);
        if (k < 1 || k > LSGD_MAX_WORKERS) Py_RETURN_NONE;
        void *grads[LSGD_MAX_WORKERS], *tokens[LSGD_MAX_WORKERS];
        int64_t n = 0;
        at::ScalarType type = at::kInt;
        for (Py_ssize_t i = 0; i < k; ++i) {
            const at::Tensor* t = plain(PySequence_Fast_GET_ITEM(a[1], i));
            if (!t || t->get_device() != dev || (i ? t->numel() != n || t->scalar_type() != type : !index_type(*t, &it)))
                Py_RETURN_NONE;
            n = t->numel();
            type = t->scalar_type();
            tokens[i] = t->data_ptr();
        }
        int workers;
        if (!addresses(a[0], n * dim, dev, grads, LSGD_MAX_WORKERS, &workers, &gdt) || workers != k) Py_RETURN_NONE;
        size_t need = 0;
        if (lsgd_embed_grad_workspace_size(workers, n, rows, dim, &need) != LSGD_OK) Py_RETURN_NONE;
        at::Tensor ws;
        if (need) ws = at::empty({static_cast<int64_t>(need)}, out->options().dtype(at::kByte));
        void *op = out->data_ptr(), *wp = need ? ws.data_ptr() : nullptr, *stream = stream_of(a[6]);
        return without_gil([&] {
            return lsgd_embed_grad(grads, gdt, tokens, it, workers, n, rows, dim, scale, op, odt, accumulate, wp, need,
                                   stream);
        });
    });
}

// quant8(x, codes, scales, device, stream)
PyObject* quant8(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        lsgd_dtype xdt;
        int64_t rows, cols;
        if (na != 5 || !small_int(a[3], &dev)) Py_RETURN_NONE;
        const at::Tensor* x = floats(a[0], -1, dev, &xdt);
        if (!x || !matrix(*x, &rows, &cols)) Py_RETURN_NONE;
        const at::Tensor *q = bytes8(a[1], kCodes, rows * lsgd_pitch8(cols), dev),
                         *s = bytes8(a[2], kScales, rows * lsgd_scale_pitch8(cols), dev);
        if (!q || !s) Py_RETURN_NONE;
        const void* xp = x->data_ptr();
        void *qp = q->data_ptr(), *sp = s->data_ptr(), *stream = stream_of(a[4]);
        return without_gil([&] { return lsgd_quant8(xp, xdt, rows, cols, qp, sp, stream); });
    });
}

// A list or tuple of (codes, scales) tuples of a rows by cols matrix, block 128.
bool copies8(PyObject* seq, int64_t rows, int64_t cols, int dev, void** codes, void** scales, int* count) {
    if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(seq);
    if (k > LSGD_MAX_REPLICAS) return false;
    for (Py_ssize_t i = 0; i < k; ++i) {
        PyObject* pair = PySequence_Fast_GET_ITEM(seq, i);
        if (!PyTuple_CheckExact(pair) || PyTuple_GET_SIZE(pair) != 2) return false;
        const at::Tensor *q = bytes8(PyTuple_GET_ITEM(pair, 0), kCodes, rows * lsgd_pitch8(cols), dev),
                         *s = bytes8(PyTuple_GET_ITEM(pair, 1), kScales, blocks(rows, 128) * lsgd_scale_pitch8(cols), dev);
        if (!q || !s) return false;
        codes[i] = q->data_ptr();
        scales[i] = s->data_ptr();
    }
    *count = static_cast<int>(k);
    return true;
}

// copy_out8(params, replicas, transposed, device, stream)
PyObject* copy_out8(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        int64_t rows, cols;
        if (na != 5 || !small_int(a[3], &dev)) Py_RETURN_NONE;
        const at::Tensor* p = plain(a[0], at::kFloat, -1, dev);
        if (!p || !matrix(*p, &rows, &cols)) Py_RETURN_NONE;
        void *q[LSGD_MAX_REPLICAS], *s[LSGD_MAX_REPLICAS], *qt[LSGD_MAX_REPLICAS], *st[LSGD_MAX_REPLICAS];
        int n, nt;
        if (!copies8(a[1], rows, cols, dev, q, s, &n) || !copies8(a[2], cols, rows, dev, qt, st, &nt)) Py_RETURN_NONE;
        const float* pp = static_cast<const float*>(p->data_ptr());
        void* stream = stream_of(a[4]);
        return without_gil([&] { return lsgd_copy_out8(pp, rows, cols, q, s, n, qt, st, nt, stream); });
    });
}

// matmul8(a, a_scales, b, b_scales, out, device, stream)
PyObject* matmul8(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev;
        if (na != 7 || !small_int(a[5], &dev)) Py_RETURN_NONE;
        const at::Tensor *q[2], *s[2];
        int64_t rows[2], pitch[2];
        int32_t block[2];
        for (int i = 0; i < 2; ++i) {
            q[i] = bytes8(a[2 * i], kCodes, -1, dev);
            s[i] = bytes8(a[2 * i + 1], kScales, -1, dev);
            if (!q[i] || !s[i] || !matrix(*q[i], &rows[i], &pitch[i]) || pitch[i] % 128) Py_RETURN_NONE;
            const int64_t sp = lsgd_scale_pitch8(pitch[i]), n = s[i]->numel();
            block[i] = n == rows[i] * sp ? 1 : n == blocks(rows[i], 128) * sp ? 128 : 0;
            if (!block[i]) Py_RETURN_NONE;
        }
        lsgd_dtype odt;
        const at::Tensor* out = floats(a[4], rows[0] * rows[1], dev, &odt);
        if (!out || pitch[0] != pitch[1]) Py_RETURN_NONE;
        const void *qa = q[0]->data_ptr(), *sa = s[0]->data_ptr(), *qb = q[1]->data_ptr(), *sb = s[1]->data_ptr();
        void *op = out->data_ptr(), *stream = stream_of(a[6]);
        return without_gil([&] {
            return lsgd_matmul8(qa, sa, block[0], rows[0], qb, sb, block[1], rows[1], pitch[0], op, odt, stream);
        });
    });
}

// weight_grad8(grad, x, x_scales, out, accumulate, device, stream); workspace as embed_grad
PyObject* weight_grad8(PyObject*, PyObject* const* a, Py_ssize_t na) {
    return guarded([&]() -> PyObject* {
        int32_t dev, accumulate;
        lsgd_dtype odt;
        int64_t n, k, m, gn;
        if (na != 7 || !small_int(a[5], &dev) || !small_int(a[4], &accumulate)) Py_RETURN_NONE;
        const at::Tensor *out = floats(a[3], -1, dev, &odt), *g = plain(a[0], at::kBFloat16, -1, dev);
        if (!out || !g || !matrix(*out, &n, &k) || !matrix(*g, &m, &gn) || gn != n) Py_RETURN_NONE;
        const at::Tensor *q = bytes8(a[1], kCodes, m * lsgd_pitch8(k), dev),
                         *s = bytes8(a[2], kScales, m * lsgd_scale_pitch8(k), dev);
        size_t need = 0;
        if (!q || !s || lsgd_weight_grad8_workspace_size(m, n, k, &need) != LSGD_OK) Py_RETURN_NONE;
        at::Tensor ws;
        if (need) ws = at::empty({static_cast<int64_t>(need)}, out->options().dtype(at::kByte));
        const void *gp = g->data_ptr(), *qp = q->data_ptr(), *sp = s->data_ptr();
        void *op = out->data_ptr(), *wp = need ? ws.data_ptr() : nullptr, *stream = stream_of(a[6]);
        return without_gil([&] {
            return lsgd_weight_grad8(gp, qp, sp, m, n, k, op, odt, accumulate, wp, need, stream);
        });
    });
}

PyMethodDef methods[] = {
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(step)), METH_FASTCALL, nullptr},
    {"group_mean", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(group_mean)), METH_FASTCALL, nullptr},
    {"global_mean", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(global_mean)), METH_FASTCALL, nullptr},
    {"sgd_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(sgd_step)), METH_FASTCALL, nullptr},
    {"copy_out", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(copy_out)), METH_FASTCALL, nullptr},
    {"embed_lookup", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(embed_lookup)), METH_FASTCALL, nullptr},
    {"embed_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(embed_grad)), METH_FASTCALL, nullptr},
    {"quant8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quant8)), METH_FASTCALL, nullptr},
    {"copy_out8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(copy_out8)), METH_FASTCALL, nullptr},
    {"matmul8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(matmul8)), METH_FASTCALL, nullptr},
    {"weight_grad8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(weight_grad8)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "torch_build", LSGD_TORCH_BUILD) < 0) Py_CLEAR(m);
    return m;
}
