// The hot calls of binding.py in native code: tensors to pointers, torch's current stream, the call.  A decode step of one sequence
// takes 4 us on the GPU and took 5.4 on the host, 3 of them in looking at nine tensors through their Python attributes and in ctypes.
// Through these calls one after the other take 3.6 to 4.4 us (6.0), about the rate at which launches follow each other on the GPU; a
// call that is waited for gains the same 2 us of about 18.  16 heads of fp32 attention decode 6.4 -> 4.4.
// Every function returns the library's status, or None for arguments that are anything but contiguous GPU tensors and plain
// numbers: the caller then goes the general way, which says what is wrong with them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "dsla.h"

namespace {

// torch._C._cuda_getDevice, _cuda_getCurrentRawStream; torch.nn.Parameter, binding.DslaDesc, DslaCache, DslaBatch, DslaRope, DslaNorm, DslaHeads
PyObject *g_device, *g_raw_stream, *g_parameter, *g_desc, *g_cache, *g_batch, *g_rope, *g_norm, *g_heads;
struct Entries {
    decltype(&dsla_decode) decode;
    decltype(&dsla_decode_slots) decode_slots;
    decltype(&dsla_prefill) prefill;
    decltype(&dsla_prefill_varlen) prefill_varlen;
    decltype(&dsla_attention_decode) attention_decode;
    decltype(&dsla_attention_prefill) attention_prefill;
    decltype(&dsla_project) project;
    decltype(&dsla_cache_extend) cache_extend;
    decltype(&dsla_cache_fork) cache_fork;
    decltype(&dsla_cache_truncate) cache_truncate;
    decltype(&dsla_cache_accept) cache_accept;
    decltype(&dsla_cache_compact) cache_compact;
    decltype(&dsla_qk_rope) qk_rope;
    decltype(&dsla_attention_paged) attention_paged;
    decltype(&dsla_residual_norm) residual_norm;
    decltype(&dsla_head_norm) head_norm;
    decltype(&dsla_quantize) quantize;
    decltype(&dsla_project_fp8) project_fp8;
} g_entry;

// A tensor whose memory can be handed over; other subclasses answer for themselves in Python.
const at::Tensor *gpu_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o) && reinterpret_cast<PyObject *>(Py_TYPE(o)) != g_parameter) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

struct Args {
    PyObject *const *o;
    bool ok = true;
    explicit Args(PyObject *const *args) : o(args) {}
    void *pointer(int i, bool optional = false)
    {
        if (optional && o[i] == Py_None) return nullptr;
        const at::Tensor *t = gpu_tensor(o[i]);
        if (!t) ok = false;
        return t ? t->data_ptr() : nullptr;
    }
    void *buffer(int i, size_t *bytes)
    {
        *bytes = 0;
        if (o[i] == Py_None) return nullptr;
        const at::Tensor *t = gpu_tensor(o[i]);
        if (!t) {
            ok = false;
            return nullptr;
        }
        *bytes = static_cast<size_t>(t->numel()) * t->element_size();
        return t->data_ptr();
    }
    // a structure of binding.py  (a copy: the caller's may change while the call runs without the interpreter's lock)
    template <class S>
    S structure(int i, PyObject *type)
    {
        S d;
        std::memset(&d, 0, sizeof(d));
        Py_buffer view;
        if (reinterpret_cast<PyObject *>(Py_TYPE(o[i])) != type) {   // (bytes of that size have a buffer too)
            ok = false;
            return d;
        }
        if (PyObject_GetBuffer(o[i], &view, PyBUF_SIMPLE) != 0) {
            ok = false;
            return d;
        }
        if (view.len == static_cast<Py_ssize_t>(sizeof(d))) std::memcpy(&d, view.buf, sizeof(d));
        else ok = false;
        PyBuffer_Release(&view);
        return d;
    }
    dsla_desc desc(int i) { return structure<dsla_desc>(i, g_desc); }
    // a tensor on the current device, of that type and number of elements (n < 0: any)
    void *here(int i, at::ScalarType type, int64_t n, bool optional = false)
    {
        if (optional && o[i] == Py_None) return nullptr;
        const at::Tensor *t = gpu_tensor(o[i]);
        if (!t || t->scalar_type() != type || (n >= 0 && t->numel() != n) || t->get_device() != device()) {
            ok = false;
            return nullptr;
        }
        return t->data_ptr();
    }
    int32_t *ints(int i, int64_t n) { return static_cast<int32_t *>(here(i, at::kInt, n)); }
    void *scratch(int i, size_t *bytes)
    {
        void *p = buffer(i, bytes);
        if (p && gpu_tensor(o[i])->get_device() != device()) ok = false;
        return p;
    }
    int64_t integer(int i)
    {
        if (!PyLong_CheckExact(o[i])) {
            ok = false;
            return 0;
        }
        const int64_t x = PyLong_AsLongLong(o[i]);
        if (x == -1 && PyErr_Occurred()) ok = false;
        return x;
    }
    float real(int i)
    {
        if (!PyFloat_CheckExact(o[i])) ok = false;
        return ok ? static_cast<float>(PyFloat_AS_DOUBLE(o[i])) : 0.f;
    }
    int64_t current = -1;   // torch's current device, once asked for
    int64_t device()
    {
        if (current < 0) {
            PyObject *d = PyObject_CallNoArgs(g_device);
            current = d ? PyLong_AsLongLong(d) : -1;
            Py_XDECREF(d);
            if (PyErr_Occurred()) ok = false;
        }
        return current;
    }
    void *stream()
    {
        if (!ok) return nullptr;
        PyObject *device = current >= 0 ? PyLong_FromLongLong(current) : PyObject_CallNoArgs(g_device), *s = device ? PyObject_CallOneArg(g_raw_stream, device) : nullptr;
        Py_XDECREF(device);
        void *p = s ? PyLong_AsVoidPtr(s) : nullptr;
        Py_XDECREF(s);
        if (PyErr_Occurred()) ok = false;
        return p;
    }
};

// [B][T][H][d] of a bf16 or fp32 tensor
bool shape_of(PyObject *o, int32_t (&dims)[3], int64_t *T, int32_t *dtype)
{
    const at::Tensor *t = gpu_tensor(o);
    if (!t || t->dim() != 4) return false;
    const auto s = t->sizes();
    for (int i = 0; i < 4; ++i)
        if (s[i] > 0x7fffffff) return false;
    dims[0] = static_cast<int32_t>(s[0]);
    *T = s[1];
    dims[1] = static_cast<int32_t>(s[2]);
    dims[2] = static_cast<int32_t>(s[3]);
    if (t->scalar_type() == at::kBFloat16) *dtype = DSLA_BF16;
    else if (t->scalar_type() == at::kFloat) *dtype = DSLA_F32;
    else return false;
    return true;
}

// Runs f(args) -> status without the interpreter's lock; None where the arguments were not what it takes.
template <class F>
PyObject *guarded(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t want, F &&f)
{
    if (nargs == want) {
        try {
            Args a(args);
            const int status = f(a);
            if (a.ok) return PyLong_FromLong(status);
        } catch (const std::exception &) {
        }
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}
#define CALL(status, a, ...)                                                                                       \
    do {                                                                                                           \
        if (!(a).ok) return 0;                                                                                     \
        Py_BEGIN_ALLOW_THREADS                                                                                     \
        status = __VA_ARGS__;                                                                                      \
        Py_END_ALLOW_THREADS                                                                                       \
    } while (0)

PyObject *decode(PyObject *, PyObject *const *args, Py_ssize_t n)   // desc, q, k, v, g1, g2, S1, S2, o
{
    return guarded(args, n, 9, [](Args &a) -> int {
        const dsla_desc d = a.desc(0);
        void *p[9];
        for (int i = 1; i < 9; ++i) p[i] = a.pointer(i);
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.decode(&d, p[1], p[2], p[3], p[4], p[5], static_cast<float *>(p[6]), static_cast<float *>(p[7]), p[8], s));
        return status;
    });
}

PyObject *decode_slots(PyObject *, PyObject *const *args, Py_ssize_t n)   // desc, q, k, v, g1, g2, row_index, state_slot, S1, S2, o
{
    return guarded(args, n, 11, [](Args &a) -> int {
        const dsla_desc d = a.desc(0);
        void *p[11];
        for (int i = 1; i < 11; ++i) p[i] = a.pointer(i, i == 6 || i == 7);
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.decode_slots(&d, p[1], p[2], p[3], p[4], p[5], static_cast<int32_t *>(p[6]), static_cast<int32_t *>(p[7]),
                                             static_cast<float *>(p[8]), static_cast<float *>(p[9]), p[10], s));
        return status;
    });
}

PyObject *prefill(PyObject *, PyObject *const *args, Py_ssize_t n)   // desc, T, q, k, v, g1, g2, S1, S2, o, workspace
{
    return guarded(args, n, 11, [](Args &a) -> int {
        const dsla_desc d = a.desc(0);
        const int64_t T = a.integer(1);
        void *p[10];
        for (int i = 2; i < 10; ++i) p[i] = a.pointer(i);
        size_t bytes;
        void *ws = a.buffer(10, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.prefill(&d, T, p[2], p[3], p[4], p[5], p[6], static_cast<float *>(p[7]), static_cast<float *>(p[8]), p[9], ws, bytes, s));
        return status;
    });
}

// desc, total_T, max_T, cu_seqlens, seq_index, state_slot, q, k, v, g1, g2, S1, S2, o, workspace
PyObject *prefill_varlen(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 15, [](Args &a) -> int {
        const dsla_desc d = a.desc(0);
        const int64_t total = a.integer(1), longest = a.integer(2);
        void *p[14];
        for (int i = 3; i < 14; ++i) p[i] = a.pointer(i, i == 4 || i == 5);
        size_t bytes;
        void *ws = a.buffer(14, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.prefill_varlen(&d, total, longest, static_cast<int32_t *>(p[3]), static_cast<int32_t *>(p[4]), static_cast<int32_t *>(p[5]),
                                               p[6], p[7], p[8], p[9], p[10], static_cast<float *>(p[11]), static_cast<float *>(p[12]), p[13], ws, bytes, s));
        return status;
    });
}

PyObject *attention_decode(PyObject *, PyObject *const *args, Py_ssize_t n)   // q, k, v, o, scale, workspace, seq_lens
{
    return guarded(args, n, 7, [](Args &a) -> int {
        int32_t dims[3] = {}, dtype = 0;
        int64_t T = 0;
        if (!shape_of(a.o[1], dims, &T, &dtype)) a.ok = false;
        void *q = a.pointer(0), *k = a.pointer(1), *v = a.pointer(2), *o = a.pointer(3);
        const float scale = a.real(4);
        size_t bytes;
        void *ws = a.buffer(5, &bytes), *lens = a.pointer(6, true), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.attention_decode(dims[0], dims[1], dims[2], T, dtype, scale, q, k, v, static_cast<int32_t *>(lens), o, ws, bytes, s));
        return status;
    });
}

PyObject *attention_prefill(PyObject *, PyObject *const *args, Py_ssize_t n)   // q, k, v, o, scale
{
    return guarded(args, n, 5, [](Args &a) -> int {
        int32_t dims[3] = {}, dtype = 0;
        int64_t T = 0;
        if (!shape_of(a.o[0], dims, &T, &dtype)) a.ok = false;
        void *q = a.pointer(0), *k = a.pointer(1), *v = a.pointer(2), *o = a.pointer(3);
        const float scale = a.real(4);
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.attention_prefill(dims[0], dims[1], dims[2], T, dtype, scale, q, k, v, o, s));
        return status;
    });
}

PyObject *project(PyObject *, PyObject *const *args, Py_ssize_t n)   // x, W, outs, bias
{
    return guarded(args, n, 4, [](Args &a) -> int {
        constexpr int kMost = 16;
        void *po[kMost];
        const at::Tensor *x = gpu_tensor(a.o[0]), *w = gpu_tensor(a.o[1]);
        if (!x || !w || !PyList_CheckExact(a.o[2]) || x->dim() != 2 || w->dim() != 2) {
            a.ok = false;
            return 0;
        }
        const int64_t M = x->size(0), K = x->size(1), n_out = PyList_GET_SIZE(a.o[2]);
        if (n_out < 1 || n_out > kMost || w->size(0) > 0x7fffffff || K > 0x7fffffff || w->size(0) % n_out != 0 || w->size(1) != K) {
            a.ok = false;
            return 0;
        }
        const int64_t width = w->size(0) / n_out;
        for (int64_t i = 0; i < n_out; ++i) {
            const at::Tensor *t = gpu_tensor(PyList_GET_ITEM(a.o[2], i));
            if (!t || t->numel() != M * width) {
                a.ok = false;
                return 0;
            }
            po[i] = t->data_ptr();
        }
        void *px = a.pointer(0), *pw = a.pointer(1), *bias = a.pointer(3, true), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.project(M, static_cast<int32_t>(K), static_cast<int32_t>(n_out), static_cast<int32_t>(width), px, pw,
                                        static_cast<float *>(bias), po, s));
        return status;
    });
}

at::ScalarType type_of(int32_t dtype) { return dtype == DSLA_BF16 ? at::kBFloat16 : at::kFloat; }
int64_t pool_size(const dsla_cache &c) { return static_cast<int64_t>(c.n_pages) * c.H_kv * c.page * c.d; }
// the array of a binding.Pools: its length and address
void *const *pools(Args &a, int i, int32_t *n)
{
    *n = static_cast<int32_t>(a.integer(i));
    return reinterpret_cast<void *const *>(a.integer(i + 1));
}

PyObject *cache_extend(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, batch, n_pools, pools, workspace
{
    return guarded(args, n, 5, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        const dsla_batch x = a.structure<dsla_batch>(1, g_batch);
        int32_t np;
        void *const *p = pools(a, 2, &np);
        size_t bytes;
        void *ws = a.scratch(4, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.cache_extend(&c, &x, np, p, ws, bytes, s));
        return status;
    });
}

PyObject *cache_fork(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, parent
{
    return guarded(args, n, 2, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        const int32_t *parent = a.ints(1, c.n_seqs);
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.cache_fork(&c, parent, s));
        return status;
    });
}

PyObject *cache_truncate(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, new_lens
{
    return guarded(args, n, 2, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        const int32_t *lens = a.ints(1, c.n_seqs);
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.cache_truncate(&c, lens, s));
        return status;
    });
}

PyObject *cache_accept(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, batch, path, n_accepted, n_pools, pools, workspace
{
    return guarded(args, n, 7, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        const dsla_batch x = a.structure<dsla_batch>(1, g_batch);
        const int32_t *path = a.ints(2, x.total), *accepted = a.ints(3, x.B);
        int32_t np;
        void *const *p = pools(a, 4, &np);
        size_t bytes;
        void *ws = a.scratch(6, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.cache_accept(&c, &x, path, accepted, np, p, ws, bytes, s));
        return status;
    });
}

PyObject *cache_compact(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, n_live, n_pools, pools, workspace
{
    return guarded(args, n, 5, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        int32_t *live = a.ints(1, 1), np;
        void *const *p = pools(a, 2, &np);
        size_t bytes;
        void *ws = a.scratch(4, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.cache_compact(&c, live, np, p, ws, bytes, s));
        return status;
    });
}

PyObject *qk_rope(PyObject *, PyObject *const *args, Py_ssize_t n)   // rope, total, q, k, v, q_out, k_out, cache, batch, k_pages, v_pages
{
    return guarded(args, n, 11, [](Args &a) -> int {
        const dsla_rope r = a.structure<dsla_rope>(0, g_rope);
        const int64_t total = a.integer(1), nq = total * r.H * r.d, nk = total * r.H_kv * r.d;
        const at::ScalarType type = type_of(r.io_dtype);
        void *q = a.here(2, type, nq), *k = a.here(3, type, nk), *v = a.here(4, type, nk, true), *q_out = a.here(5, type, nq), *k_out = a.here(6, type, nk, true);
        const bool cached = a.o[7] != Py_None && a.o[8] != Py_None;
        if (!cached && (a.o[7] != Py_None || a.o[8] != Py_None || a.o[9] != Py_None || a.o[10] != Py_None)) a.ok = false;
        dsla_cache c;
        dsla_batch x;
        void *kp = nullptr, *vp = nullptr;
        if (cached) {
            c = a.structure<dsla_cache>(7, g_cache);
            x = a.structure<dsla_batch>(8, g_batch);
            kp = a.here(9, type, pool_size(c));
            vp = a.here(10, type, pool_size(c));
        }
        void *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.qk_rope(&r, total, q, k, v, q_out, k_out, cached ? &c : nullptr, cached ? &x : nullptr, kp, vp, s));
        return status;
    });
}

PyObject *attention_paged(PyObject *, PyObject *const *args, Py_ssize_t n)   // cache, batch, q, k_pages, v_pages, o, scale, max_len, tree, workspace
{
    return guarded(args, n, 10, [](Args &a) -> int {
        const dsla_cache c = a.structure<dsla_cache>(0, g_cache);
        const dsla_batch x = a.structure<dsla_batch>(1, g_batch);
        const at::Tensor *t = gpu_tensor(a.o[2]);
        if (!t || t->dim() != 3 || t->size(1) > 0x7fffffff) {
            a.ok = false;
            return 0;
        }
        const int32_t H = static_cast<int32_t>(t->size(1));
        const at::ScalarType type = type_of(c.dtype);
        const int64_t nq = x.total * H * c.d;
        void *q = a.here(2, type, nq), *kp = a.here(3, type, pool_size(c)), *vp = a.here(4, type, pool_size(c)), *o = a.here(5, type, nq);
        const float scale = a.real(6);
        const int64_t max_len = a.integer(7);
        const uint64_t *tree = static_cast<uint64_t *>(a.here(8, at::kLong, x.total, true));
        size_t bytes;
        void *ws = a.scratch(9, &bytes), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.attention_paged(&c, &x, H, max_len, scale, q, kp, vp, tree, o, ws, bytes, s));
        return status;
    });
}

at::ScalarType type_of_result(int32_t dtype) { return dtype == DSLA_E4M3 ? at::ScalarType::Float8_e4m3fn : type_of(dtype); }
at::ScalarType type_of_scale(int32_t scale_type) { return scale_type == DSLA_SCALE_E8M0 ? at::ScalarType::Float8_e8m0fnu : at::kFloat; }

PyObject *residual_norm(PyObject *, PyObject *const *args, Py_ssize_t n)   // norm, x, y, gate, x_out, h, h_scale
{
    return guarded(args, n, 7, [](Args &a) -> int {
        const dsla_norm d = a.structure<dsla_norm>(0, g_norm);
        const at::Tensor *t = gpu_tensor(a.o[1]);
        if (!a.ok || !t || d.D <= 0) {
            a.ok = false;
            return 0;
        }
        const int64_t size = t->numel(), rows = size / d.D;
        const at::ScalarType tx = type_of(d.x_dtype), ty = type_of(d.y_dtype);
        void *x = a.here(1, tx, rows * d.D), *y = a.here(2, ty, size, true), *gate = a.here(3, ty, size, true), *x_out = a.here(4, tx, size, true);
        void *h = a.here(5, type_of_result(d.h_dtype), size, true);
        void *scale = a.here(6, type_of_scale(d.scale_type), rows * DSLA_SCALE_PITCH(static_cast<int64_t>(d.D)), true), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.residual_norm(&d, rows, x, y, gate, x_out, h, scale, s));
        return status;
    });
}

PyObject *head_norm(PyObject *, PyObject *const *args, Py_ssize_t n)   // heads, o, gate, out, out_scale
{
    return guarded(args, n, 5, [](Args &a) -> int {
        const dsla_heads d = a.structure<dsla_heads>(0, g_heads);
        const at::Tensor *t = gpu_tensor(a.o[1]);
        const int64_t width = static_cast<int64_t>(d.H) * d.d;
        if (!a.ok || !t || width <= 0) {
            a.ok = false;
            return 0;
        }
        const int64_t size = t->numel(), rows = size / width;
        const at::ScalarType type = type_of(d.io_dtype);
        void *o = a.here(1, type, rows * width), *gate = a.here(2, type, size, true), *out = a.here(3, type_of_result(d.out_dtype), size);
        void *scale = a.here(4, type_of_scale(d.scale_type), rows * DSLA_SCALE_PITCH(width), true), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.head_norm(&d, rows, o, gate, out, scale, s));
        return status;
    });
}

PyObject *quantize(PyObject *, PyObject *const *args, Py_ssize_t n)   // x, q, scale, block_rows
{
    return guarded(args, n, 4, [](Args &a) -> int {
        const at::Tensor *t = gpu_tensor(a.o[0]), *sc = gpu_tensor(a.o[2]);
        const int64_t per = a.integer(3);
        if (!a.ok || !t || !sc || t->dim() != 2 || t->size(1) > 0x7fffffff || (per != 1 && per != 128) ||
            (t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kFloat)) {
            a.ok = false;
            return 0;
        }
        const int64_t rows = t->size(0), cols = t->size(1);
        const int32_t st = sc->scalar_type() == at::kFloat ? DSLA_SCALE_F32 : DSLA_SCALE_E8M0;
        void *x = a.here(0, t->scalar_type(), rows * cols), *q = a.here(1, at::ScalarType::Float8_e4m3fn, rows * cols);
        void *scale = a.here(2, type_of_scale(st), (rows + per - 1) / per * DSLA_SCALE_PITCH(cols)), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.quantize(rows, static_cast<int32_t>(cols), t->scalar_type() == at::kFloat ? DSLA_F32 : DSLA_BF16, static_cast<int32_t>(per), st,
                                         x, q, scale, s));
        return status;
    });
}

PyObject *project_fp8(PyObject *, PyObject *const *args, Py_ssize_t n)   // x, x_scale, W, W_scale, outs, bias
{
    return guarded(args, n, 6, [](Args &a) -> int {
        void *po[DSLA_MAX_PROJECTIONS];
        int32_t widths[DSLA_MAX_PROJECTIONS];
        const at::Tensor *x = gpu_tensor(a.o[0]), *w = gpu_tensor(a.o[2]), *sc = gpu_tensor(a.o[1]);
        if (!x || !w || !sc || !PyList_CheckExact(a.o[4]) || x->dim() != 2 || w->dim() != 2 || x->size(1) > 0x7fffffff || w->size(1) != x->size(1)) {
            a.ok = false;
            return 0;
        }
        const int64_t M = x->size(0), K = x->size(1), n_out = PyList_GET_SIZE(a.o[4]), P = DSLA_SCALE_PITCH(K);
        const int32_t st = sc->scalar_type() == at::kFloat ? DSLA_SCALE_F32 : DSLA_SCALE_E8M0;
        if (n_out < 1 || n_out > DSLA_MAX_PROJECTIONS) {
            a.ok = false;
            return 0;
        }
        int64_t N = 0, blocks = 0;
        at::ScalarType type = at::kFloat;
        for (int64_t i = 0; i < n_out; ++i) {
            const at::Tensor *t = gpu_tensor(PyList_GET_ITEM(a.o[4], i));
            if (i == 0 && t) type = t->scalar_type();
            if (!t || t->dim() != 2 || t->size(0) != M || t->size(1) > (1 << 24) || t->scalar_type() != type || t->get_device() != a.device() ||
                (type != at::kFloat && type != at::kBFloat16)) {
                a.ok = false;
                return 0;
            }
            po[i] = t->data_ptr();
            widths[i] = static_cast<int32_t>(t->size(1));
            N += widths[i];
            blocks += (widths[i] + 127) / 128;
        }
        void *px = a.here(0, at::ScalarType::Float8_e4m3fn, M * K), *xs = a.here(1, type_of_scale(st), M * P);
        void *pw = a.here(2, at::ScalarType::Float8_e4m3fn, N * K), *ws = a.here(3, type_of_scale(st), blocks * P);
        void *bias = a.here(5, at::kFloat, N, true), *s = a.stream();
        int status = 0;
        CALL(status, a, g_entry.project_fp8(M, static_cast<int32_t>(K), static_cast<int32_t>(n_out), widths, st, px, xs, pw, ws, static_cast<float *>(bias),
                                            type == at::kFloat ? DSLA_F32 : DSLA_BF16, po, s));
        return status;
    });
}

// device, raw_stream, parameter type, the structures' types, addresses of the entry points in the order of Entries
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    constexpr int kEntries = sizeof(Entries) / sizeof(void *);
    constexpr int kObjects = 9;
    if (n != kObjects + kEntries) {
        PyErr_SetString(PyExc_TypeError, "bind: number of arguments");
        return nullptr;
    }
    void *p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(args[kObjects + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    std::memcpy(&g_entry, p, sizeof(p));
    PyObject **to[kObjects] = {&g_device, &g_raw_stream, &g_parameter, &g_desc, &g_cache, &g_batch, &g_rope, &g_norm, &g_heads};
    for (int i = 0; i < kObjects; ++i) {
        Py_INCREF(args[i]);
        Py_XDECREF(*to[i]);
        *to[i] = args[i];
    }
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {METHOD(bind), METHOD(decode), METHOD(decode_slots), METHOD(prefill), METHOD(prefill_varlen), METHOD(attention_decode),
                           METHOD(attention_prefill), METHOD(project), METHOD(cache_extend), METHOD(cache_fork), METHOD(cache_truncate), METHOD(cache_accept),
                           METHOD(cache_compact), METHOD(qk_rope), METHOD(attention_paged), METHOD(residual_norm), METHOD(head_norm),
                           METHOD(quantize), METHOD(project_fp8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__marshal(void)
{
    PyObject *m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "built_for", DSLA_BUILT_FOR) != 0) Py_CLEAR(m);   // (build.py: marshal_stamp)
    return m;
}
