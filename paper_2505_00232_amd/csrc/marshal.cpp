// The calls of binding.py whose arguments are in order, without Python's attribute look-ups: a small layer takes the GPU 3 us, and the checks and the
// conversion of its arguments in Python took the host as long.  Whatever is not in order returns -1 and is looked at again there, for the message.
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qfc.h"

namespace {

decltype(&qfc_forward) g_forward = nullptr;
decltype(&qfc_forward_fused) g_forward_fused = nullptr;
PyObject *g_stream = nullptr;  // torch's current stream, asked for once the arguments are in order

// Pointer of a contiguous binary16 matrix on a GPU with `cols` columns and (if rows >= 0) that many rows, which are returned; null: something else.
// Plain tensors with memory of their own only: subclasses and wrappers (tracing, vmap) go the other way.
void *matrix(PyObject *o, int64_t &rows, int64_t cols) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.scalar_type() != at::kHalf || t.dim() != 2 || !t.is_contiguous()) return nullptr;
    const auto sizes = t.sizes();
    if (sizes[1] != cols || (rows >= 0 && sizes[0] != rows)) return nullptr;
    rows = sizes[0];
    return t.mutable_data_ptr();
}

void *vector(PyObject *o, int64_t size) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.scalar_type() != at::kHalf || t.dim() != 1 || t.sizes()[0] != size || !t.is_contiguous()) return nullptr;
    return t.mutable_data_ptr();
}

// False with Python's error set where there is none
bool current_stream(void *&stream) {
    PyObject *s = PyObject_CallNoArgs(g_stream);
    if (!s) return false;
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return !PyErr_Occurred();
}

// bind(address of qfc_forward, address of qfc_forward_fused, function that returns the current stream)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) return PyErr_Format(PyExc_TypeError, "two addresses and a function");
    void *f = PyLong_AsVoidPtr(a[0]), *g = PyLong_AsVoidPtr(a[1]);
    if (PyErr_Occurred()) return nullptr;
    g_forward = reinterpret_cast<decltype(g_forward)>(f);
    g_forward_fused = reinterpret_cast<decltype(g_forward_fused)>(g);
    Py_INCREF(a[2]);
    Py_XSETREF(g_stream, a[2]);
    Py_RETURN_NONE;
}

// forward(handle, x, y, N, K) -> status, or -1
PyObject *forward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 5 || !g_forward) return PyLong_FromLong(-1);
    void *h = PyLong_AsVoidPtr(a[0]);
    const long N = PyLong_AsLong(a[3]), K = PyLong_AsLong(a[4]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return PyLong_FromLong(-1);
    }
    int64_t M = -1;
    void *x = nullptr, *y = nullptr;
    try {
        x = matrix(a[1], M, K);
        if (x) y = matrix(a[2], M, N);
    } catch (...) {
        y = nullptr;
    }
    if (!x || !y || M < 1 || M > INT32_MAX) return PyLong_FromLong(-1);
    void *stream;
    if (!current_stream(stream)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_forward(static_cast<qfc_handle_t>(h), x, (int32_t)M, y, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// forward_fused(handle, x, y, N, K, gate, activation, residual, gated_output, norm_gamma, norm_eps, norm_offset) -> status, or -1
PyObject *forward_fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 12 || !g_forward_fused) return PyLong_FromLong(-1);
    void *h = PyLong_AsVoidPtr(a[0]);
    const long N = PyLong_AsLong(a[3]), K = PyLong_AsLong(a[4]), activation = PyLong_AsLong(a[6]);
    const int gated = PyObject_IsTrue(a[8]);
    qfc_fusion_t f = {};
    f.norm_eps = (float)PyFloat_AsDouble(a[10]);
    f.norm_offset = (float)PyFloat_AsDouble(a[11]);
    if (PyErr_Occurred()) {
        PyErr_Clear();  // (an argument of another type: as the other way takes it)
        return PyLong_FromLong(-1);
    }
    if (activation < INT32_MIN || activation > INT32_MAX || (gated && a[7] != Py_None)) return PyLong_FromLong(-1);
    f.activation = (int32_t)activation;
    f.gated_output = gated;
    int64_t M = -1;
    void *x = nullptr, *y = nullptr;
    bool ok = false;
    try {
        x = matrix(a[1], M, K);
        if (x) y = matrix(a[2], M, gated ? N / 2 : N);
        ok = x && y;
        if (ok && a[5] != Py_None) ok = (f.gate = matrix(a[5], M, K)) != nullptr;
        if (ok && a[7] != Py_None) ok = (f.residual = matrix(a[7], M, N)) != nullptr;
        if (ok && a[9] != Py_None) ok = (f.norm_gamma = vector(a[9], K)) != nullptr;
    } catch (...) {
        ok = false;
    }
    if (!ok || M < 1 || M > INT32_MAX) return PyLong_FromLong(-1);
    void *stream;
    if (!current_stream(stream)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = g_forward_fused(static_cast<qfc_handle_t>(h), x, (int32_t)M, y, &f, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// ---- pages: calls that a server makes once a step, a few microseconds of the GPU's each
decltype(&qfc_take_pages) g_take = nullptr;
decltype(&qfc_fork_pages) g_fork = nullptr;
decltype(&qfc_free_pages) g_free = nullptr;
decltype(&qfc_compact_pages) g_compact = nullptr;

// A contiguous plain tensor of a type on GPU `device`; null: something else
const at::Tensor *plain(PyObject *o, at::ScalarType type, int64_t dims, long device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != dims || !t.is_contiguous()) return nullptr;
    return &t;
}
int32_t *numbers(PyObject *o, int64_t count, long device) {
    const at::Tensor *t = plain(o, at::kInt, 1, device);
    return t && t->sizes()[0] == count ? static_cast<int32_t *>(t->mutable_data_ptr()) : nullptr;
}
struct Table {
    int32_t *at = nullptr;
    int32_t batch = 0, width = 0;
};
bool table(PyObject *o, long device, Table &out) {
    const at::Tensor *t = plain(o, at::kInt, 2, device);
    if (!t || t->sizes()[0] > INT32_MAX || t->sizes()[1] > INT32_MAX) return false;
    out.at = static_cast<int32_t *>(t->mutable_data_ptr()), out.batch = (int32_t)t->sizes()[0], out.width = (int32_t)t->sizes()[1];
    return true;
}
struct Space {
    void *at = nullptr;
    size_t bytes = 0;
};
bool space(PyObject *o, long device, Space &out) {
    const at::Tensor *t = THPVariable_CheckExact(o) ? plain(o, at::kByte, THPVariable_Unpack(o).dim(), device) : nullptr;
    if (!t) return false;
    out.at = t->mutable_data_ptr(), out.bytes = (size_t)t->numel();
    return true;
}
// null for None
bool maybe(PyObject *o, int64_t count, long device, int32_t *&out) {
    out = nullptr;
    return o == Py_None || (out = numbers(o, count, device)) != nullptr;
}

// What begins the arguments of all of them: address of the cache's description, its device, the current device, its pages
struct Pool {
    const qfc_q4_cache_t *cache;
    long device, pages;
    bool ok;
    explicit Pool(PyObject *const *a) {
        cache = static_cast<const qfc_q4_cache_t *>(PyLong_AsVoidPtr(a[0]));
        device = PyLong_AsLong(a[1]);
        const long now = PyLong_AsLong(a[2]);
        pages = PyLong_AsLong(a[3]);
        ok = !PyErr_Occurred() && cache && device == now;
        PyErr_Clear();
    }
};
// In order: `look` finds all arguments; call(stream): the library's status
template <class Look, class Call>
PyObject *page_call(bool ready, const Look &look, const Call &call) {
    bool ok = false;
    try {
        ok = ready && look();
    } catch (...) {
        ok = false;
    }
    if (!ok) return PyLong_FromLong(-1);
    void *stream;
    if (!current_stream(stream)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// bind_pages(addresses of qfc_take_pages, qfc_fork_pages, qfc_free_pages, qfc_compact_pages)
PyObject *bind_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "four addresses");
    void *f[4];
    for (int i = 0; i < 4; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    g_take = reinterpret_cast<decltype(g_take)>(f[0]), g_fork = reinterpret_cast<decltype(g_fork)>(f[1]);
    g_free = reinterpret_cast<decltype(g_free)>(f[2]), g_compact = reinterpret_cast<decltype(g_compact)>(f[3]);
    Py_RETURN_NONE;
}

// take_pages(cache, its device, current device, pages, references, table, positions, workspace, missing) -> status, or -1
PyObject *take_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return PyLong_FromLong(-1);
    const Pool p(a);
    int32_t *references, *positions, *missing;
    Table t;
    Space w;
    return page_call(
        p.ok && g_take,
        [&] {
            return (references = numbers(a[4], p.pages, p.device)) && table(a[5], p.device, t) && (positions = numbers(a[6], t.batch, p.device)) && space(a[7], p.device, w) &&
                   maybe(a[8], 1, p.device, missing);
        },
        [&](void *stream) { return g_take(p.cache, references, t.at, positions, t.batch, t.width, missing, w.at, w.bytes, stream); });
}

// fork_pages(cache, its device, current device, pages, references, source table, parents, positions, table, workspace, missing, address of bounds) -> status, or -1
PyObject *fork_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 12) return PyLong_FromLong(-1);
    const Pool p(a);
    const auto *bounds = static_cast<const qfc_page_bounds_t *>(PyLong_AsVoidPtr(a[11]));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return PyLong_FromLong(-1);
    }
    int32_t *references, *parents, *positions, *missing;
    Table from, t;
    Space w;
    return page_call(
        p.ok && g_fork,
        [&] {
            return (references = numbers(a[4], p.pages, p.device)) && table(a[5], p.device, from) && table(a[8], p.device, t) && (parents = numbers(a[6], t.batch, p.device)) &&
                   (positions = numbers(a[7], t.batch, p.device)) && space(a[9], p.device, w) && maybe(a[10], 1, p.device, missing);
        },
        [&](void *stream) {
            return g_fork(p.cache, references, from.at, from.batch, from.width, parents, positions, t.at, t.batch, t.width, missing, bounds, w.at, w.bytes, stream);
        });
}

// free_pages(cache, its device, current device, pages, references, table, keep) -> status, or -1
PyObject *free_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 7) return PyLong_FromLong(-1);
    const Pool p(a);
    int32_t *references, *keep;
    Table t;
    return page_call(
        p.ok && g_free, [&] { return (references = numbers(a[4], p.pages, p.device)) && table(a[5], p.device, t) && maybe(a[6], t.batch, p.device, keep); },
        [&](void *stream) { return g_free(p.cache, references, t.at, keep, t.batch, t.width, stream); });
}

// compact_pages(cache, its device, current device, pages, references, table, workspace, used, address of bounds) -> status, or -1
PyObject *compact_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return PyLong_FromLong(-1);
    const Pool p(a);
    const auto *bounds = static_cast<const qfc_page_bounds_t *>(PyLong_AsVoidPtr(a[8]));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return PyLong_FromLong(-1);
    }
    int32_t *references, *used;
    Table t;
    Space w;
    return page_call(
        p.ok && g_compact,
        [&] { return (references = numbers(a[4], p.pages, p.device)) && table(a[5], p.device, t) && space(a[6], p.device, w) && maybe(a[7], 1, p.device, used); },
        [&](void *stream) { return g_compact(p.cache, references, t.at, t.batch, t.width, used, bounds, w.at, w.bytes, stream); });
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(bind), METH_FASTCALL, nullptr},
    {"forward", reinterpret_cast<PyCFunction>(forward), METH_FASTCALL, nullptr},
    {"forward_fused", reinterpret_cast<PyCFunction>(forward_fused), METH_FASTCALL, nullptr},
    {"bind_pages", reinterpret_cast<PyCFunction>(bind_pages), METH_FASTCALL, nullptr},
    {"take_pages", reinterpret_cast<PyCFunction>(take_pages), METH_FASTCALL, nullptr},
    {"fork_pages", reinterpret_cast<PyCFunction>(fork_pages), METH_FASTCALL, nullptr},
    {"free_pages", reinterpret_cast<PyCFunction>(free_pages), METH_FASTCALL, nullptr},
    {"compact_pages", reinterpret_cast<PyCFunction>(compact_pages), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", QFC_BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
