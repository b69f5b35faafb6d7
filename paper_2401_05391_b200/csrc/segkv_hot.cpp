// The calls of the decode loop without the interpreter in between: argument checks and the library call of
// segkv_decode_step, segkv_append, segkv_decode_sdpa, segkv_truncate_last and segkv_steps for one handle of the segment cache, and of
// segkv_pages_append, segkv_pages_sdpa and segkv_pages_read for one handle of the paged cache.
//
// Six tensors checked from Python cost about 3 us of a call and marshalling them through ctypes another one, which is
// as much as a small layer's step takes on the GPU.  Here each check reads the tensor object directly.  A call
// whose arguments are not plainly what the step expects (a tensor of another shape, type or place, a tensor subclass, a
// step that is no int) is not made: the method answers None, and the caller takes its general path, which
// raises what it has always raised.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

struct Fns {
    int (*decode_step)(void*, int, const int32_t*, const void*, const void*, const void*, void*, const float*, void*);
    int (*append)(void*, int, const int32_t*, const void*, const void*, void*);
    int (*decode_sdpa)(void*, const void*, void*, const float*, void*);
    int (*truncate_last)(void*);
    int (*steps)(void*);
};

struct Hot {
    PyObject_HEAD
    void* handle;
    Fns fn;
    long long rows, heads, kv_heads, head_dim;
    at::ScalarType dtype;
};

// Device address of a plain contiguous CUDA tensor of this type and shape; None stands for a null pointer.
bool tensor(PyObject* o, at::ScalarType type, const long long* shape, int dims, void** p) {
    *p = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || t.dim() != dims) return false;
    const auto sizes = t.sizes();
    for (int i = 0; i < dims; ++i)
        if (sizes[i] != shape[i]) return false;
    if (!t.is_contiguous()) return false;
    *p = t.data_ptr();
    return true;
}

bool step_of(PyObject* o, int* step) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v != (long)(int)v) return false;
    *step = (int)v;
    return true;
}

// The checks, then the call.  An exception of the tensor library (a tensor without storage, say) leaves the call to the
// general path.
template <typename Check, typename Run>
PyObject* checked(Check check, Run run) {
    void* st = nullptr;
    try {
        if (!check()) Py_RETURN_NONE;
        st = c10::cuda::getCurrentCUDAStream().stream();
    } catch (...) {
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = run(st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// decode_step(step, beam_parent, k_new, v_new, q, out, slopes)
PyObject* hot_decode_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Hot* h = reinterpret_cast<Hot*>(self);
    int step = 0;
    void *par, *k, *v, *q, *out, *sl;
    const long long kv[3] = {h->rows, h->kv_heads, h->head_dim}, qs[3] = {h->rows, h->heads, h->head_dim};
    return checked(
        [&] {
            return n == 7 && step_of(a[0], &step) && tensor(a[1], at::kInt, kv, 1, &par) && tensor(a[2], h->dtype, kv, 3, &k) &&
                   tensor(a[3], h->dtype, kv, 3, &v) && tensor(a[4], h->dtype, qs, 3, &q) && tensor(a[5], h->dtype, qs, 3, &out) &&
                   tensor(a[6], at::kFloat, &h->heads, 1, &sl);
        },
        [&](void* st) { return h->fn.decode_step(h->handle, step, (const int32_t*)par, k, v, q, out, (const float*)sl, st); });
}

// append(step, beam_parent, k_new, v_new)
PyObject* hot_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Hot* h = reinterpret_cast<Hot*>(self);
    int step = 0;
    void *par, *k, *v;
    const long long kv[3] = {h->rows, h->kv_heads, h->head_dim};
    return checked(
        [&] {
            return n == 4 && step_of(a[0], &step) && tensor(a[1], at::kInt, kv, 1, &par) && tensor(a[2], h->dtype, kv, 3, &k) &&
                   tensor(a[3], h->dtype, kv, 3, &v);
        },
        [&](void* st) { return h->fn.append(h->handle, step, (const int32_t*)par, k, v, st); });
}

// decode_sdpa(q, out, slopes)
PyObject* hot_decode_sdpa(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    const Hot* h = reinterpret_cast<Hot*>(self);
    void *q, *out, *sl;
    const long long qs[3] = {h->rows, h->heads, h->head_dim};
    return checked(
        [&] {
            return n == 3 && tensor(a[0], h->dtype, qs, 3, &q) && tensor(a[1], h->dtype, qs, 3, &out) &&
                   tensor(a[2], at::kFloat, &h->heads, 1, &sl);
        },
        [&](void* st) { return h->fn.decode_sdpa(h->handle, q, out, (const float*)sl, st); });
}

PyObject* hot_truncate_last(PyObject* self, PyObject*) {
    const Hot* h = reinterpret_cast<Hot*>(self);
    return PyLong_FromLong(h->fn.truncate_last(h->handle));
}

PyObject* hot_steps(PyObject* self, PyObject*) {
    const Hot* h = reinterpret_cast<Hot*>(self);
    return PyLong_FromLong(h->fn.steps(h->handle));
}

// Hot(handle, rows, heads, kv_heads, head_dim, bf16, (addresses of decode_step, append, decode_sdpa, truncate_last, steps))
PyObject* hot_new(PyTypeObject* type, PyObject* args, PyObject*) {
    unsigned long long handle, f[5];
    long long rows, heads, kv_heads, head_dim;
    int bf16;
    if (!PyArg_ParseTuple(args, "KLLLLp(KKKKK)", &handle, &rows, &heads, &kv_heads, &head_dim, &bf16, &f[0], &f[1], &f[2], &f[3], &f[4]))
        return nullptr;
    Hot* h = reinterpret_cast<Hot*>(type->tp_alloc(type, 0));
    if (!h) return nullptr;
    h->handle = reinterpret_cast<void*>(handle);
    h->rows = rows;
    h->heads = heads;
    h->kv_heads = kv_heads;
    h->head_dim = head_dim;
    h->dtype = bf16 ? at::kBFloat16 : at::kHalf;
    h->fn.decode_step = reinterpret_cast<decltype(Fns::decode_step)>(f[0]);
    h->fn.append = reinterpret_cast<decltype(Fns::append)>(f[1]);
    h->fn.decode_sdpa = reinterpret_cast<decltype(Fns::decode_sdpa)>(f[2]);
    h->fn.truncate_last = reinterpret_cast<decltype(Fns::truncate_last)>(f[3]);
    h->fn.steps = reinterpret_cast<decltype(Fns::steps)>(f[4]);
    return reinterpret_cast<PyObject*>(h);
}

PyMethodDef methods[] = {
    {"decode_step", (PyCFunction)(void (*)(void))hot_decode_step, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))hot_append, METH_FASTCALL, nullptr},
    {"decode_sdpa", (PyCFunction)(void (*)(void))hot_decode_sdpa, METH_FASTCALL, nullptr},
    {"truncate_last", hot_truncate_last, METH_NOARGS, nullptr},
    {"steps", hot_steps, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

// ------------------------------------------------------------------------------------------------------------- the paged cache
struct PagesFns {
    int (*append)(void*, int, int, const void*, long long, const void*, long long, const int32_t*, int, const int32_t*, const int32_t*,
                  const void*, long long, void*, const float*, const float*, int, int, void*);
    int (*sdpa)(void*, int, int, const void*, long long, void*, const int32_t*, int, const int32_t*, const float*, void*);
    int (*read)(void*, int, int, void*, void*, const int32_t*, int, const int32_t*, const int32_t*, void*);
};

struct Pages {
    PyObject_HEAD
    void* handle;
    PagesFns fn;
    long long heads, kv_heads, head_dim;
    int device;
    at::ScalarType dtype;
};

const at::Tensor* plain(const Pages* h, PyObject* o, at::ScalarType type, int dims) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.device().index() != h->device || t.scalar_type() != type || t.layout() != at::kStrided || t.dim() != dims) return nullptr;
    return &t;
}

// table [n, entries] and lens [n]
bool index_of(const Pages* h, PyObject* table, PyObject* lens, int* n, int* entries, void** tp, void** lp) {
    const at::Tensor *a = plain(h, table, at::kInt, 2), *b = plain(h, lens, at::kInt, 1);
    if (!a || !b || a->size(0) != b->size(0) || !a->is_contiguous() || !b->is_contiguous()) return false;
    if (b->size(0) > 0x7FFFFFFF || a->size(1) > 0x7FFFFFFF) return false;
    *n = (int)b->size(0);
    *entries = (int)a->size(1);
    *tp = a->data_ptr();
    *lp = b->data_ptr();
    return true;
}

bool optional_lens(const Pages* h, PyObject* o, int n, void** p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(h, o, at::kInt, 1);
    if (!t || t->size(0) != n || !t->is_contiguous()) return false;
    *p = t->data_ptr();
    return true;
}

// [n, tokens, heads, head_dim] with each token's heads contiguous and the tokens evenly spaced; *tokens is filled in, or compared where it is set
bool rows_of(const Pages* h, PyObject* o, int n, long long* tokens, long long heads, void** p, long long* stride) {
    const at::Tensor* t = plain(h, o, h->dtype, 4);
    if (!t || t->numel() == 0) return false;
    const auto z = t->sizes(), s = t->strides();
    if (z[0] != n || z[2] != heads || z[3] != h->head_dim || s[3] != 1 || (heads > 1 && s[2] != h->head_dim)) return false;
    if (*tokens >= 0 ? z[1] != *tokens : z[1] > 0x7FFFFFFF) return false;
    *tokens = z[1];
    const long long row = z[1] > 1 ? s[1] : n > 1 ? s[0] : heads * h->head_dim;
    if ((n > 1 && s[0] != row * z[1]) || row < heads * h->head_dim || row % 8) return false;
    *p = t->data_ptr();
    *stride = row;
    return true;
}

bool dense_of(const Pages* h, PyObject* o, int n, long long tokens, long long heads, void** p) {
    const at::Tensor* t = plain(h, o, h->dtype, 4);
    if (!t || !t->is_contiguous()) return false;
    const auto z = t->sizes();
    if (z[0] != n || z[1] != tokens || z[2] != heads || z[3] != h->head_dim) return false;
    *p = t->data_ptr();
    return true;
}

bool current(const Pages* h) { return c10::cuda::current_device() == h->device; }

// append(k, v, table, lens, new_lens, q, q_out, rope_cos, rope_sin, style)
PyObject* pages_append(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
    const Pages* h = reinterpret_cast<Pages*>(self);
    int n = 0, entries = 0, style = 0, positions = 0;
    long long tokens = -1, ks = 0, vs = 0, qs = 0;
    void *k, *v, *tab, *lens, *fresh, *q = nullptr, *q_out = nullptr, *cos = nullptr, *sin = nullptr;
    return checked(
        [&] {
            if (nargs != 10 || !current(h) || !index_of(h, a[2], a[3], &n, &entries, &tab, &lens) || !optional_lens(h, a[4], n, &fresh)) return false;
            if (!rows_of(h, a[0], n, &tokens, h->kv_heads, &k, &ks) || !rows_of(h, a[1], n, &tokens, h->kv_heads, &v, &vs)) return false;
            if ((a[5] == Py_None) != (a[6] == Py_None) || (a[7] == Py_None) != (a[8] == Py_None)) return false;
            if (a[5] != Py_None && (!rows_of(h, a[5], n, &tokens, h->heads, &q, &qs) || !dense_of(h, a[6], n, tokens, h->heads, &q_out))) return false;
            if (a[7] == Py_None) return true;
            const at::Tensor *c = plain(h, a[7], at::kFloat, 2), *s = plain(h, a[8], at::kFloat, 2);
            if (!c || !s || !c->is_contiguous() || !s->is_contiguous() || c->sizes() != s->sizes() || c->size(1) != h->head_dim / 2) return false;
            if (c->size(0) > 0x7FFFFFFF || !step_of(a[9], &style)) return false;
            cos = c->data_ptr();
            sin = s->data_ptr();
            positions = (int)c->size(0);
            return true;
        },
        [&](void* st) {
            return h->fn.append(h->handle, n, (int)tokens, k, ks, v, vs, (const int32_t*)tab, entries, (const int32_t*)lens, (const int32_t*)fresh, q, qs,
                                q_out, (const float*)cos, (const float*)sin, positions, style, st);
        });
}

// sdpa(q, table, lens, out, slopes)
PyObject* pages_sdpa(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
    const Pages* h = reinterpret_cast<Pages*>(self);
    int n = 0, entries = 0;
    long long tokens = -1, qs = 0;
    void *q, *tab, *lens, *out, *slopes = nullptr;
    return checked(
        [&] {
            if (nargs != 5 || !current(h) || !index_of(h, a[1], a[2], &n, &entries, &tab, &lens)) return false;
            if (!rows_of(h, a[0], n, &tokens, h->heads, &q, &qs) || !dense_of(h, a[3], n, tokens, h->heads, &out)) return false;
            if (a[4] == Py_None) return true;
            const at::Tensor* s = plain(h, a[4], at::kFloat, 1);
            if (!s || s->size(0) != h->heads || !s->is_contiguous()) return false;
            slopes = s->data_ptr();
            return true;
        },
        [&](void* st) {
            return h->fn.sdpa(h->handle, n, (int)tokens, q, qs, out, (const int32_t*)tab, entries, (const int32_t*)lens, (const float*)slopes, st);
        });
}

// read(table, lens, tokens, new_lens, k, v)
PyObject* pages_read(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
    const Pages* h = reinterpret_cast<Pages*>(self);
    int n = 0, entries = 0, tokens = 0;
    void *tab, *lens, *fresh, *k, *v;
    return checked(
        [&] {
            return nargs == 6 && current(h) && index_of(h, a[0], a[1], &n, &entries, &tab, &lens) && step_of(a[2], &tokens) && tokens >= 0 &&
                   optional_lens(h, a[3], n, &fresh) && dense_of(h, a[4], n, tokens, h->kv_heads, &k) && dense_of(h, a[5], n, tokens, h->kv_heads, &v);
        },
        [&](void* st) { return h->fn.read(h->handle, n, tokens, k, v, (const int32_t*)tab, entries, (const int32_t*)lens, (const int32_t*)fresh, st); });
}

// Pages(handle, heads, kv_heads, head_dim, device, bf16, (addresses of append, sdpa, read))
PyObject* pages_new(PyTypeObject* type, PyObject* args, PyObject*) {
    unsigned long long handle, f[3];
    long long heads, kv_heads, head_dim;
    int device, bf16;
    if (!PyArg_ParseTuple(args, "KLLLip(KKK)", &handle, &heads, &kv_heads, &head_dim, &device, &bf16, &f[0], &f[1], &f[2])) return nullptr;
    Pages* h = reinterpret_cast<Pages*>(type->tp_alloc(type, 0));
    if (!h) return nullptr;
    h->handle = reinterpret_cast<void*>(handle);
    h->heads = heads;
    h->kv_heads = kv_heads;
    h->head_dim = head_dim;
    h->device = device;
    h->dtype = bf16 ? at::kBFloat16 : at::kHalf;
    h->fn.append = reinterpret_cast<decltype(PagesFns::append)>(f[0]);
    h->fn.sdpa = reinterpret_cast<decltype(PagesFns::sdpa)>(f[1]);
    h->fn.read = reinterpret_cast<decltype(PagesFns::read)>(f[2]);
    return reinterpret_cast<PyObject*>(h);
}

PyMethodDef pages_methods[] = {
    {"append", (PyCFunction)(void (*)(void))pages_append, METH_FASTCALL, nullptr},
    {"sdpa", (PyCFunction)(void (*)(void))pages_sdpa, METH_FASTCALL, nullptr},
    {"read", (PyCFunction)(void (*)(void))pages_read, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject pages_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject hot_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "segkv_hot", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_segkv_hot(void) {
    hot_type.tp_name = "segkv_hot.Hot";
    hot_type.tp_basicsize = sizeof(Hot);
    hot_type.tp_flags = Py_TPFLAGS_DEFAULT;
    hot_type.tp_new = hot_new;
    hot_type.tp_methods = methods;
    if (PyType_Ready(&hot_type) < 0) return nullptr;
    PyObject* m = PyModule_Create(&module);
    if (!m) return nullptr;
    Py_INCREF(&hot_type);
    if (PyModule_AddObject(m, "Hot", reinterpret_cast<PyObject*>(&hot_type)) < 0) return nullptr;
    pages_type.tp_name = "segkv_hot.Pages";
    pages_type.tp_basicsize = sizeof(Pages);
    pages_type.tp_flags = Py_TPFLAGS_DEFAULT;
    pages_type.tp_new = pages_new;
    pages_type.tp_methods = pages_methods;
    if (PyType_Ready(&pages_type) < 0) return nullptr;
    Py_INCREF(&pages_type);
    if (PyModule_AddObject(m, "Pages", reinterpret_cast<PyObject*>(&pages_type)) < 0) return nullptr;
    return m;
}
