// The binding's small calls in native code.  One token's projection takes 4.1 us on the GPU and took 5.3 on the host (4096 x 4096 int4), of
// which 3 went into reading the tensors' attributes one by one from Python and converting thirteen arguments; here they are read from the
// tensors themselves.  Only what needs no decision is done here: tensors of the plain types, all buffers given.  Anything else -- missing
// buffers, wrong types, subclasses, a tensor without storage -- returns None, and the Python code beside the call takes it from the start
// and raises what there is to raise.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <algorithm>
#include <cmath>

#include "../../include/rtn.h"

namespace {

decltype(&rtn_linear) linear_fn = nullptr;
decltype(&rtn_linear_asym) asym_fn = nullptr;
decltype(&rtn_cache_plan) plan_fn = nullptr;
decltype(&rtn_rope_cache) rope_fn = nullptr;
decltype(&rtn_paged_attention) attend_fn = nullptr;

bool plain(PyObject* o) {
    return Py_TYPE(o) == reinterpret_cast<PyTypeObject*>(THPVariableClass) || Py_TYPE(o) == reinterpret_cast<PyTypeObject*>(ParameterClass);
}

// (A, qweight, scales[, zeros], bits, group_size, out, workspace) -> status, or None
PyObject* call(PyObject* const* args, bool zp) {
    const int extra = zp ? 1 : 0;
    PyObject *const pa = args[0], *const pq = args[1], *const ps = args[2], *const pz = args[2 + extra], *const pbits = args[3 + extra],
             *const pg = args[4 + extra], *const pc = args[5 + extra], *const pw = args[6 + extra];
    for (PyObject* t : {pa, pq, ps, pz, pc, pw})
        if (!plain(t)) Py_RETURN_NONE;
    if (!PyLong_CheckExact(pbits) || !PyLong_CheckExact(pg)) Py_RETURN_NONE;
    const long bits = PyLong_AsLong(pbits), g = PyLong_AsLong(pg);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (bits != (int)bits || g != (int)g) Py_RETURN_NONE;
    const void *da, *dq, *ds, *dz = nullptr;
    void *dc, *dw, *stream;
    int64_t M, N, K;
    size_t bytes;
    try {
        const at::Tensor &a = THPVariable_Unpack(pa), &q = THPVariable_Unpack(pq), &s = THPVariable_Unpack(ps), &c = THPVariable_Unpack(pc),
                         &w = THPVariable_Unpack(pw);
        if (!a.is_cuda() || a.scalar_type() != at::kHalf || a.dim() != 2 || !a.is_contiguous() || s.dim() < 1) Py_RETURN_NONE;
        if (!w.is_cuda() || !w.is_contiguous() || w.device() != a.device()) Py_RETURN_NONE;
        da = a.data_ptr(); dq = q.data_ptr(); ds = s.data_ptr(); dc = c.data_ptr(); dw = w.data_ptr();
        if (zp) dz = THPVariable_Unpack(pz).data_ptr();
        M = a.size(0); K = a.size(1); N = s.size(0);
        bytes = zp ? (size_t)w.numel() : w.nbytes();
        stream = c10::hip::getCurrentHIPStream().stream();
    } catch (...) {                                       // no storage to point to
        Py_RETURN_NONE;
    }
    rtn_status st;
    Py_BEGIN_ALLOW_THREADS
    st = zp ? asym_fn(da, M, dq, ds, dz, N, K, (int)bits, (int)g, dc, dw, bytes, stream)
            : linear_fn(da, M, dq, ds, N, K, (int)bits, (int)g, dc, dw, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 7 || !linear_fn) Py_RETURN_NONE;
    return call(args, false);
}

PyObject* linear_asym(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 8 || !asym_fn) Py_RETURN_NONE;
    return call(args, true);
}

// ---- The paged cache's calls.  What they check is what the Python code checks; whatever fails goes there, to be refused.

bool ints(PyObject* o, int64_t n, int32_t** data, int64_t* have = nullptr) {      // a contiguous int32 vector of n (any, n < 0)
    if (!plain(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != 1 || !t.is_contiguous() || (n >= 0 && t.size(0) != n)) return false;
    *data = static_cast<int32_t*>(t.data_ptr());
    if (have) *have = t.size(0);
    return true;
}

int64_t row_stride(const at::Tensor& t) {                      // a single row may have any stride
    if (t.size(0) > 1) return t.stride(0);
    int64_t row = 0;
    if (t.size(0) == 1) {
        row = 1;
        for (int64_t d = 1; d < t.dim(); ++d) row *= t.size(d);
    }
    return std::max<int64_t>(t.stride(0), row);
}

bool table(PyObject* o, int64_t rows, int32_t** data, int64_t* stride, int64_t* width) {
    if (!plain(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != 2 || t.stride(1) != 1 || t.size(0) != rows || t.size(1) > INT32_MAX) return false;
    *data = static_cast<int32_t*>(t.data_ptr());
    *stride = row_stride(t);
    *width = t.size(1);
    return true;
}

bool whole(PyObject* o, long* v) {                             // an int of 32 bits
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsLong(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return *v == (int)*v;
}

at::ScalarType type_of(const rtn_kv_cache* c) { return c->dtype == RTN_TYPE_F16 ? at::kHalf : at::kBFloat16; }

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (step, cached_lens, block_table, free_pages, free_count, page_size, max_tokens, out) -> status, or None
PyObject* cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 8 || !plan_fn || !PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != 6) Py_RETURN_NONE;
    int32_t *step, *cached, *tab, *pages, *count, *o[6];
    int64_t B, stride, width, pool;
    long ps, tokens;
    void* stream;
    try {
        if (!whole(a[5], &ps) || !whole(a[6], &tokens) || tokens < 0 || !ints(a[0], -1, &step, &B) || B > INT32_MAX - 1 || !ints(a[1], B, &cached) ||
            !table(a[2], B, &tab, &stride, &width) || !ints(a[3], -1, &pages, &pool) || !ints(a[4], 1, &count))
            Py_RETURN_NONE;
        const int64_t sizes[6] = {B, B + 1, tokens, tokens, 1, 1};
        for (int i = 0; i < 6; ++i)
            if (!ints(PyTuple_GET_ITEM(a[7], i), sizes[i], &o[i])) Py_RETURN_NONE;
        stream = current_stream();
    } catch (...) {
        Py_RETURN_NONE;
    }
    rtn_status st;
    Py_BEGIN_ALLOW_THREADS
    st = plan_fn(step, cached, (int)B, (int)ps, tab, stride, (int)width, pages, pool, count, o[0], o[1], o[2], o[3], tokens, o[4], o[5], stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

// (qkv, q_heads, rope, positions, slots, cache's address, q_norm, k_norm, eps, interleaved, out) -> status, or None
PyObject* rope_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 11 || !rope_fn) Py_RETURN_NONE;
    const rtn_kv_cache* const c = static_cast<const rtn_kv_cache*>(PyLong_AsVoidPtr(a[5]));
    if (PyErr_Occurred() || !c) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    long heads;
    if (!whole(a[1], &heads) || heads < 1 || !plain(a[0]) || !plain(a[2]) || !plain(a[10]) || !PyFloat_CheckExact(a[8]) || !PyBool_Check(a[9])) Py_RETURN_NONE;
    const void* norm[2] = {nullptr, nullptr};
    int32_t *positions, *slots;
    const void *q, *rope;
    void *out, *stream;
    int64_t T, stride, rows, rotary;
    try {
        const at::ScalarType type = type_of(c);
        const at::Tensor &x = THPVariable_Unpack(a[0]), &r = THPVariable_Unpack(a[2]), &y = THPVariable_Unpack(a[10]);
        if (!x.is_cuda() || x.scalar_type() != type || x.dim() != 2 || x.size(1) != ((int64_t)heads + 2 * c->kv_heads) * c->head_dim || x.stride(1) != 1)
            Py_RETURN_NONE;
        if (!r.is_cuda() || r.scalar_type() != at::kFloat || r.dim() != 2 || !r.is_contiguous() || r.size(1) > INT32_MAX) Py_RETURN_NONE;
        T = x.size(0);
        if (!y.is_cuda() || y.scalar_type() != type || y.dim() != 3 || y.size(0) != T || y.size(1) != heads || y.size(2) != c->head_dim || !y.is_contiguous())
            Py_RETURN_NONE;
        if (!ints(a[3], T, &positions) || !ints(a[4], T, &slots)) Py_RETURN_NONE;
        for (int i = 0; i < 2; ++i) {
            if (a[6 + i] == Py_None) continue;
            if (!plain(a[6 + i])) Py_RETURN_NONE;
            const at::Tensor& w = THPVariable_Unpack(a[6 + i]);
            if (!w.is_cuda() || w.scalar_type() != type || w.dim() != 1 || w.size(0) != c->head_dim || !w.is_contiguous()) Py_RETURN_NONE;
            norm[i] = w.data_ptr();
        }
        q = x.data_ptr(); rope = r.data_ptr(); out = y.data_ptr();
        stride = row_stride(x); rows = r.size(0); rotary = r.size(1);
        stream = current_stream();
    } catch (...) {
        Py_RETURN_NONE;
    }
    const float eps = (float)PyFloat_AS_DOUBLE(a[8]);
    const int interleaved = a[9] == Py_True;
    rtn_status st;
    Py_BEGIN_ALLOW_THREADS
    st = rope_fn(q, T, stride, (int)heads, static_cast<const float*>(rope), (int)rotary, rows, interleaved, positions, slots, norm[0], norm[1], eps, c, out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

// (q, cache's address, block_table, seq_lens, query_start, max_new, scale, softcap, window, out, workspace) -> status, or None
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 11 || !attend_fn) Py_RETURN_NONE;
    const rtn_kv_cache* const c = static_cast<const rtn_kv_cache*>(PyLong_AsVoidPtr(a[1]));
    if (PyErr_Occurred() || !c) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    long most, window;
    if (!whole(a[5], &most) || !whole(a[8], &window) || !plain(a[0]) || !plain(a[9]) || !plain(a[10]) || !(a[6] == Py_None || PyFloat_CheckExact(a[6])) ||
        !PyFloat_CheckExact(a[7]))
        Py_RETURN_NONE;
    int32_t *tab, *seq, *start;
    const void* q;
    void *out, *ws, *stream;
    int64_t T, H, B, qs, stride, width;
    size_t bytes;
    try {
        const at::ScalarType type = type_of(c);
        const at::Tensor &x = THPVariable_Unpack(a[0]), &y = THPVariable_Unpack(a[9]), &w = THPVariable_Unpack(a[10]);
        if (!x.is_cuda() || x.scalar_type() != type || x.dim() != 3 || x.size(2) != c->head_dim || x.stride(2) != 1 || x.size(1) > INT32_MAX) Py_RETURN_NONE;
        T = x.size(0); H = x.size(1);
        if (H != 1 && x.stride(1) != x.size(2)) Py_RETURN_NONE;
        if (!y.is_cuda() || y.scalar_type() != type || y.sizes() != x.sizes() || !y.is_contiguous()) Py_RETURN_NONE;
        if (!w.is_cuda() || !w.is_contiguous() || w.device() != x.device()) Py_RETURN_NONE;
        if (!ints(a[3], -1, &seq, &B) || B > INT32_MAX - 1 || !ints(a[4], B + 1, &start) || !table(a[2], B, &tab, &stride, &width)) Py_RETURN_NONE;
        q = x.data_ptr(); out = y.data_ptr(); ws = w.data_ptr();
        qs = row_stride(x); bytes = w.nbytes();
        stream = current_stream();
    } catch (...) {
        Py_RETURN_NONE;
    }
    const float scale = (float)(a[6] == Py_None ? 1.0 / std::sqrt((double)c->head_dim) : PyFloat_AS_DOUBLE(a[6])), cap = (float)PyFloat_AS_DOUBLE(a[7]);
    rtn_status st;
    Py_BEGIN_ALLOW_THREADS
    st = attend_fn(q, T, qs, (int)H, c, tab, stride, (int)width, seq, start, (int)B, (int)most, scale, cap, (int)window, out, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

// bind(rtn_linear, rtn_linear_asym, rtn_cache_plan, rtn_rope_cache, rtn_paged_attention): their addresses in the loaded library
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind takes five addresses");
        return nullptr;
    }
    void* f[5];
    for (int i = 0; i < 5; ++i) {
        f[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    linear_fn = reinterpret_cast<decltype(linear_fn)>(f[0]);
    asym_fn = reinterpret_cast<decltype(asym_fn)>(f[1]);
    plan_fn = reinterpret_cast<decltype(plan_fn)>(f[2]);
    rope_fn = reinterpret_cast<decltype(rope_fn)>(f[3]);
    attend_fn = reinterpret_cast<decltype(attend_fn)>(f[4]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"linear_asym", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_asym)), METH_FASTCALL, nullptr},
    {"cache_plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_plan)), METH_FASTCALL, nullptr},
    {"rope_cache", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rope_cache)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attention)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the PyTorch and Python of this build
PyMODINIT_FUNC PyInit__native() {
    PyObject* const m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", RTN_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
