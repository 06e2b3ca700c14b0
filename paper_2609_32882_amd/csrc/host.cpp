// Argument marshalling of the helpers around the attention (norm and rotation,
// the 8-bit cache, attention over it): torch tensors in, checks, outputs and
// workspaces from torch's allocator, one call of the C-ABI.
//
// These are the calls a server makes once per token and layer, where the host's
// time is what a call costs: the same marshalling through Python and ctypes took
// 11 to 35 us of a call whose launch takes 4.  Everything computed is in
// libvsa2.so; this file holds no arithmetic.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "vsa2.h"

namespace {

PyObject* g_error = nullptr;      // raises the package's error for (function, status)
thread_local int t_device = -1;   // the current GPU, on whose stream the call will run

// A Python error is set; unwinds to the entry point.
struct python_error {};

[[noreturn]] void fail(const std::string& what) {
    PyErr_SetString(PyExc_ValueError, what.c_str());
    throw python_error{};
}

std::string shape_text(at::IntArrayRef s) {
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + ")";
}

[[noreturn]] void unexpected(const char* name, const at::Tensor& t, const char* kind, at::IntArrayRef shape,
                             at::ScalarType dtype) {
    std::string strides;
    for (int64_t s : t.strides()) strides += (strides.empty() ? "" : ", ") + std::to_string(s);
    fail(std::string(name) + ": expected " + kind + " " + at::toString(dtype) + " " + shape_text(shape) +
         " on the GPU, got " + at::toString(t.scalar_type()) + " " + shape_text(t.sizes()) + " strides (" + strides +
         ") on " + t.device().str());
}

// A kernel of this GPU must not be handed another GPU's memory.
void on_current_device(const at::Tensor& t, const char* name) {
    if (t.device().index() != t_device)
        fail(std::string(name) + ": on " + t.device().str() + ", but the current device is cuda:" + std::to_string(t_device));
}

// Nor the memory whose addresses a structure has kept: `device` is the one it was filled on (-1: none).
int32_t integer32(PyObject* o, const char* name);
void filled_here(PyObject* device, const char* name) {
    const int32_t d = integer32(device, name);
    if (d >= 0 && d != t_device)
        fail(std::string(name) + ": its tensors are on cuda:" + std::to_string(d) + ", but the current device is cuda:" +
             std::to_string(t_device));
}

// The tensor in a Python object; null for None.
const at::Tensor* tensor(PyObject* o, const char* name) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) fail(std::string(name) + ": expected a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor& required(PyObject* o, const char* name) {
    const at::Tensor* t = tensor(o, name);
    if (!t) fail(std::string(name) + ": expected a tensor, got None");
    return *t;
}

template <typename P>
P* contiguous(const at::Tensor* t, at::IntArrayRef shape, at::ScalarType dtype, const char* name) {
    if (!t) return nullptr;
    if (t->sizes() != shape || t->scalar_type() != dtype || !t->is_cuda() || !t->is_contiguous())
        unexpected(name, *t, "contiguous", shape, dtype);
    on_current_device(*t, name);
    return static_cast<P*>(t->data_ptr());
}

// Rows of D contiguous elements with any strides.
vsa2_rows rows(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType dtype, const char* name) {
    if (t.sizes() != shape || t.scalar_type() != dtype || !t.is_cuda() || t.stride(3) != 1)
        unexpected(name, t, "rows of contiguous elements", shape, dtype);
    on_current_device(t, name);
    return vsa2_rows{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

// A C structure behind a ctypes one.
template <typename S>
S* structure(PyObject* o, const char* name) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw python_error{};
    void* p = b.buf;
    const bool fits = b.len == static_cast<Py_ssize_t>(sizeof(S));
    PyBuffer_Release(&b);          // the caller's reference keeps it alive
    if (!fits) fail(std::string(name) + ": not the structure this call takes");
    return static_cast<S*>(p);
}

int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error{};
    return v;
}
int32_t integer32(PyObject* o, const char* name) {
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(std::string(name) + ": outside 32 bits");
    return static_cast<int32_t>(v);
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1. && PyErr_Occurred()) throw python_error{};
    return v;
}
// The stream: what the caller's function says, asked once the tensors are checked.
hipStream_t stream_of(PyObject* current) {
    PyObject* r = PyObject_CallNoArgs(current);
    if (!r) throw python_error{};
    const int64_t v = PyLong_AsLongLong(r);
    Py_DECREF(r);
    if (v == -1 && PyErr_Occurred()) throw python_error{};
    return reinterpret_cast<hipStream_t>(static_cast<intptr_t>(v));
}

void check(const char* fn, vsa2_status st) {
    if (st == VSA2_OK) return;
    if (g_error) {
        PyObject* r = PyObject_CallFunction(g_error, "si", fn, static_cast<int>(st));
        if (r) {
            PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(r)), r);
            Py_DECREF(r);
        }
    } else {
        PyErr_SetString(PyExc_RuntimeError, fn);
    }
    throw python_error{};
}

at::ScalarType dtype_of(const vsa2_problem& p) { return p.dtype == VSA2_BF16 ? at::kBFloat16 : at::kFloat; }
int32_t code_of(at::ScalarType t, const char* name) {
    if (t == at::kBFloat16) return VSA2_BF16;
    if (t == at::kFloat) return VSA2_F32;
    fail(std::string(name) + ": expected torch.bfloat16 or torch.float32, got " + at::toString(t));
}

// Tokens of a sequence: in raster order, and in cube-major order with padding.
int64_t raster_tokens(const vsa2_problem& p) { return static_cast<int64_t>(p.T) * p.H * p.W + p.text_len; }
int64_t cube_tokens(const vsa2_problem& p) {
    if (p.Bt < 1 || p.Bh < 1 || p.Bw < 1) return 0;       // refused by the library
    const auto up = [](int64_t n, int64_t m) { return (n + m - 1) / m; };
    const int64_t block = static_cast<int64_t>(p.Bt) * p.Bh * p.Bw;
    return (up(p.T, p.Bt) * up(p.H, p.Bh) * up(p.W, p.Bw) + up(p.text_len, block)) * block;
}

// Three given outputs, or null.
PyObject* const* three(PyObject* o, const char* name) {
    if (o == Py_None) return nullptr;
    if (PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3) return &PyTuple_GET_ITEM(o, 0);
    if (PyList_Check(o) && PyList_GET_SIZE(o) == 3) return &PyList_GET_ITEM(o, 0);
    fail(std::string(name) + ": expected three tensors");
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

void count_args(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        throw python_error{};
    }
}

// (structure, axes, tables, origin, pairing) -> the device of the tables and origin, -1 without any
PyObject* fill_rope(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 5);
    vsa2_rope* r = structure<vsa2_rope>(a[0], "rope");
    PyObject *const *axes = three(a[1], "axes"), *const *tables = three(a[2], "tables");
    if (!axes || !tables) fail("axes, tables: expected three each");
    for (int i = 0; i < 3; ++i) {
        r->axis[i] = integer32(axes[i], "axes");
        r->rows[i] = 0;
        r->table[i] = nullptr;
        if (r->axis[i] == 0) continue;
        const at::Tensor* t = tensor(tables[i], "tables");
        if (!t) fail("tables[" + std::to_string(i) + "]: an axis of " + std::to_string(r->axis[i]) + " elements needs one");
        const int64_t rows = t->dim() ? t->size(0) : 0;
        r->table[i] = contiguous<float>(t, {rows, r->axis[i] / 2, 2}, at::kFloat, "tables");
        if (rows > INT32_MAX) fail("tables: too many rows");
        r->rows[i] = static_cast<int32_t>(rows);
    }
    const at::Tensor* origin = tensor(a[3], "origin");
    r->origin = origin ? contiguous<int32_t>(origin, {origin->dim() ? origin->size(0) : 0, 3}, at::kInt, "origin") : nullptr;
    r->pairing = integer32(a[4], "pairing");
    return PyLong_FromLong(r->axis[0] || r->axis[1] || r->axis[2] || origin ? t_device : -1);
}

// (structure, pool, table) -> their device
PyObject* fill_cache(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 3);
    vsa2_cache* c = structure<vsa2_cache>(a[0], "cache");
    const at::Tensor &pool = required(a[1], "pool"), &table = required(a[2], "table");
    if (pool.dim() != 3 || pool.size(2) < 256 || (pool.size(2) - 128) % 128)
        fail("pool: expected [pages, heads_kv, 128*D + 128], got " + shape_text(pool.sizes()));
    const bool lists = table.dim() == 3 && table.size(1) == pool.size(1);
    if (table.dim() != 2 && !lists)
        fail("table: expected [batch, max_pages] or [batch, " + std::to_string(pool.size(1)) + ", max_pages], got " +
             shape_text(table.sizes()));
    for (int64_t s : {pool.size(0), pool.size(1), pool.size(2), table.size(0), table.size(-1)})
        if (s > INT32_MAX) fail("cache: a size outside 32 bits");
    c->pool = contiguous<void>(&pool, pool.sizes(), at::kByte, "pool");
    c->table = contiguous<int32_t>(&table, table.sizes(), at::kInt, "table");
    c->batch = static_cast<int32_t>(table.size(0));
    c->heads_kv = static_cast<int32_t>(pool.size(1));
    c->head_dim = static_cast<int32_t>((pool.size(2) - 128) / 128);
    c->pages = static_cast<int32_t>(pool.size(0));
    c->max_pages = static_cast<int32_t>(table.size(-1));
    c->table_heads = lists ? c->heads_kv : 1;
    return PyLong_FromLong(t_device);
}

const vsa2_rope* rope_or_null(PyObject* o) { return o == Py_None ? nullptr : structure<vsa2_rope>(o, "rope"); }

// (problem, rope, eps, q, k, v, q_gain, k_gain, out, stream, rope's device) -> (q, k, v)
PyObject* norm_rope(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 11);
    filled_here(a[10], "rope");
    const vsa2_problem& p = *structure<vsa2_problem>(a[0], "problem");
    const vsa2_rope* r = rope_or_null(a[1]);
    const at::ScalarType dt = dtype_of(p);
    const int64_t tokens = raster_tokens(p), L = cube_tokens(p), D = p.head_dim;
    static const char* const names[3] = {"q", "k", "v"};
    PyObject* const* out = three(a[8], "out");
    vsa2_rows in[3];
    const vsa2_rows* given[3] = {};
    at::Tensor y[3];
    void* yp[3] = {};
    for (int i = 0; i < 3; ++i) {
        const at::Tensor* x = tensor(a[3 + i], names[i]);
        if (!x) continue;
        const int64_t heads = i ? p.heads_kv : p.heads_q;
        in[i] = rows(*x, {p.batch, heads, tokens, D}, dt, names[i]);
        given[i] = &in[i];
        y[i] = out ? required(out[i], "out") : at::empty({p.batch, heads, L, D}, x->options());
        yp[i] = contiguous<void>(&y[i], {p.batch, heads, L, D}, dt, "out");
    }
    const float* gain[2];
    for (int i = 0; i < 2; ++i) gain[i] = contiguous<const float>(tensor(a[6 + i], "gain"), {D}, at::kFloat, "gain");
    const float eps = static_cast<float>(real(a[2]));
    const hipStream_t s = stream_of(a[9]);
    check("vsa2_qk_norm_rope", vsa2_qk_norm_rope(&p, r, eps, given[0], gain[0], yp[0], given[1], gain[1], yp[1], given[2],
                                                 yp[2], s));
    PyObject* t = PyTuple_New(3);
    for (int i = 0; i < 3; ++i) {
        PyObject* o = given[i] ? (out ? out[i] : wrap(y[i])) : Py_None;
        if (!given[i] || out) Py_INCREF(o);
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
}

// (problem, rope, eps, dq, dk, dv, q, k, q_gain, k_gain, out, stream, rope's device)
//   -> (dq_in, dk_in, dv_in, dq_gain, dk_gain)
PyObject* norm_rope_bwd(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 13);
    filled_here(a[12], "rope");
    const vsa2_problem& p = *structure<vsa2_problem>(a[0], "problem");
    const vsa2_rope* r = rope_or_null(a[1]);
    const float eps = static_cast<float>(real(a[2]));
    const at::ScalarType dt = dtype_of(p);
    const int64_t tokens = raster_tokens(p), L = cube_tokens(p), D = p.head_dim;
    static const char* const names[3] = {"dq", "dk", "dv"};
    static const char* const xnames[2] = {"q", "k"};
    PyObject* const* out = three(a[10], "out");
    vsa2_rows in[2], dx_rows[3];
    const vsa2_rows *x_given[2] = {}, *dx_given[3] = {};
    const void* dy[3] = {};
    at::Tensor dx[3], dgain[2], ws;
    float* dgain_p[2] = {};
    for (int i = 0; i < 3; ++i) {
        const at::Tensor* g = tensor(a[3 + i], names[i]);
        if (!g) continue;
        const int64_t heads = i ? p.heads_kv : p.heads_q;
        dy[i] = contiguous<void>(g, {p.batch, heads, L, D}, dt, names[i]);
        dx[i] = out ? required(out[i], "out") : at::empty({p.batch, tokens, heads, D}, g->options()).transpose(1, 2);
        dx_rows[i] = rows(dx[i], {p.batch, heads, tokens, D}, dt, "out");
        dx_given[i] = &dx_rows[i];
        if (i == 2) continue;
        if (const at::Tensor* x = tensor(a[6 + i], xnames[i])) {
            in[i] = rows(*x, {p.batch, heads, tokens, D}, dt, xnames[i]);
            x_given[i] = &in[i];
        }
        if (eps > 0) {
            dgain[i] = at::empty({D}, g->options().dtype(at::kFloat));
            dgain_p[i] = dgain[i].data_ptr<float>();
        }
    }
    const float* gain[2];
    for (int i = 0; i < 2; ++i) gain[i] = contiguous<const float>(tensor(a[8 + i], "gain"), {D}, at::kFloat, "gain");
    size_t bytes = 0;
    void* wp = nullptr;
    if (dgain_p[0] || dgain_p[1]) {
        check("vsa2_qk_norm_rope_workspace", vsa2_qk_norm_rope_workspace(&p, &bytes));
        ws = at::empty({static_cast<int64_t>(bytes)}, dgain[dgain_p[0] ? 0 : 1].options().dtype(at::kByte));
        wp = ws.data_ptr();
    }
    const hipStream_t s = stream_of(a[11]);
    check("vsa2_qk_norm_rope_bwd",
          vsa2_qk_norm_rope_bwd(&p, r, eps, x_given[0], gain[0], dy[0], dx_given[0], dgain_p[0], x_given[1], gain[1],
                                dy[1], dx_given[1], dgain_p[1], dy[2], dx_given[2], wp, bytes, s));
    PyObject* t = PyTuple_New(5);
    for (int i = 0; i < 3; ++i) {
        PyObject* o = dx_given[i] ? (out ? out[i] : wrap(dx[i])) : Py_None;
        if (!dx_given[i] || out) Py_INCREF(o);
        PyTuple_SET_ITEM(t, i, o);
    }
    for (int i = 0; i < 2; ++i) {
        PyObject* o = dgain_p[i] ? wrap(dgain[i]) : Py_None;
        if (!dgain_p[i]) Py_INCREF(o);
        PyTuple_SET_ITEM(t, 3 + i, o);
    }
    return t;
}

// (cache, k, v, start, count, stream, cache's device)
PyObject* cache_write(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 7);
    filled_here(a[6], "cache");
    const vsa2_cache& c = *structure<vsa2_cache>(a[0], "cache");
    const at::Tensor &k = required(a[1], "k"), &v = required(a[2], "v");
    const at::ScalarType dt = k.scalar_type();
    if (k.dim() != 4 || k.size(2) > INT32_MAX) fail("k: expected [batch, heads_kv, n, D], got " + shape_text(k.sizes()));
    const int64_t shape[4] = {c.batch, c.heads_kv, k.size(2), c.head_dim};
    const vsa2_rows kr = rows(k, shape, dt, "k"), vr = rows(v, shape, dt, "v");
    const int32_t code = code_of(dt, "k");
    const int32_t* start = contiguous<int32_t>(&required(a[3], "start"), {c.batch}, at::kInt, "start");
    const int32_t* count = contiguous<int32_t>(tensor(a[4], "count"), {c.batch}, at::kInt, "count");
    const hipStream_t s = stream_of(a[5]);
    check("vsa2_cache_write", vsa2_cache_write(&c, code, static_cast<int32_t>(shape[2]), &kr, &vr, start, count, s));
    Py_RETURN_NONE;
}

// (cache, pool, n, start, count, dtype, k, v, stream, cache's device) -> (k, v); dtype is the code of new outputs
PyObject* cache_read(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 10);
    filled_here(a[9], "cache");
    const vsa2_cache& c = *structure<vsa2_cache>(a[0], "cache");
    const int32_t tokens = integer32(a[2], "n");
    if (tokens < 0) fail("n: expected 0 or more");
    const int64_t shape[4] = {c.batch, c.heads_kv, tokens, c.head_dim};
    const bool given = a[6] != Py_None;
    at::Tensor k, v;
    if (given) {
        k = required(a[6], "out");
        v = required(a[7], "out");
    } else {
        const auto like = required(a[1], "pool").options().dtype(integer(a[5]) == VSA2_F32 ? at::kFloat : at::kBFloat16);
        k = at::empty(shape, like);
        v = at::empty(shape, like);
    }
    const at::ScalarType dt = k.scalar_type();
    const vsa2_rows kr = rows(k, shape, dt, "out"), vr = rows(v, shape, dt, "out");
    const int32_t code = code_of(dt, "out");
    const int32_t* start = contiguous<int32_t>(&required(a[3], "start"), {c.batch}, at::kInt, "start");
    const int32_t* count = contiguous<int32_t>(tensor(a[4], "count"), {c.batch}, at::kInt, "count");
    const hipStream_t s = stream_of(a[8]);
    check("vsa2_cache_read", vsa2_cache_read(&c, code, tokens, &kr, &vr, start, count, s));
    PyObject* t = PyTuple_New(2);
    for (int i = 0; i < 2; ++i) {
        PyObject* o = given ? a[6 + i] : wrap(i ? v : k);
        if (given) Py_INCREF(o);
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
}

// (cache, q, length, count, causal, o, stream, cache's device) -> (o, lse)
PyObject* attn_cache(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 8);
    filled_here(a[7], "cache");
    const vsa2_cache& c = *structure<vsa2_cache>(a[0], "cache");
    const at::Tensor& q = required(a[1], "q");
    if (q.dim() != 4 || q.size(1) > INT32_MAX || q.size(2) > INT32_MAX)
        fail("q: expected [batch, heads_q, n, D], got " + shape_text(q.sizes()));
    const int64_t shape[4] = {c.batch, q.size(1), q.size(2), c.head_dim};
    const at::ScalarType dt = q.scalar_type();
    const int32_t code = code_of(dt, "q"), heads = static_cast<int32_t>(shape[1]), tokens = static_cast<int32_t>(shape[2]);
    const vsa2_rows qr = rows(q, shape, dt, "q");
    const bool given = a[5] != Py_None;
    const at::Tensor o = given ? required(a[5], "o") : at::empty(shape, q.options());
    const vsa2_rows orow = rows(o, shape, dt, "o");
    const at::Tensor lse = at::empty({shape[0], shape[1], shape[2]}, q.options().dtype(at::kFloat));
    size_t bytes = 0;
    check("vsa2_attn_cache_workspace", vsa2_attn_cache_workspace(&c, heads, tokens, &bytes));
    at::Tensor ws;
    if (bytes) ws = at::empty({static_cast<int64_t>(bytes)}, q.options().dtype(at::kByte));
    const int32_t* length = contiguous<int32_t>(&required(a[2], "length"), {c.batch}, at::kInt, "length");
    const int32_t* count = contiguous<int32_t>(tensor(a[3], "count"), {c.batch}, at::kInt, "count");
    const hipStream_t s = stream_of(a[6]);
    check("vsa2_attn_cache",
          vsa2_attn_cache(&c, code, heads, tokens, &qr, length, count, a[4] == Py_True ? 1 : 0, &orow,
                          lse.data_ptr<float>(), bytes ? ws.data_ptr() : nullptr, bytes, s));
    PyObject* t = PyTuple_New(2);
    if (given) Py_INCREF(a[5]);
    PyTuple_SET_ITEM(t, 0, given ? a[5] : wrap(o));
    PyTuple_SET_ITEM(t, 1, wrap(lse));
    return t;
}

PyObject* set_error(PyObject* const* a, Py_ssize_t n) {
    count_args(n, 1);
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    Py_RETURN_NONE;
}

// No exception leaves an entry point.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (hipGetDevice(&t_device) != hipSuccess) t_device = -1;      // without a GPU no tensor is on one
    try {
        return F(args, n);
    } catch (const python_error&) {
    } catch (const c10::OutOfMemoryError& e) {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* kind = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (kind) PyErr_SetString(kind, e.what_without_backtrace());
        Py_XDECREF(kind);
        Py_XDECREF(torch);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

#define VSA2_ENTRY(F) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {VSA2_ENTRY(fill_rope),   VSA2_ENTRY(fill_cache), VSA2_ENTRY(norm_rope), VSA2_ENTRY(norm_rope_bwd),
                           VSA2_ENTRY(cache_write), VSA2_ENTRY(cache_read), VSA2_ENTRY(attn_cache), VSA2_ENTRY(set_error),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_host", "Argument marshalling of the helpers around the attention.", -1,
                        g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&g_module); }
