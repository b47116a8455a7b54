// Python's side of the calls in 4 bits (dg4_mx4.h): checks of the tensors and the C call, for calls so short that looking at
// tensors from Python takes as long as the launch (a level's write: 6.2 us through ctypes, 3.0 of them outside the C call). No
// arithmetic. Functions take what binding.py's functions of the same names take, in order; what does not fit raises DG4Error.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "dg4_mx4.h"

namespace {

// What bind() gave: the library's entry points, the class of errors, the current stream of a device, the current device
decltype(&dg4_kv4_write) kv4_write;
decltype(&dg4_kv4_read) kv4_read;
decltype(&dg4_sparse_attn_kv4_fwd) attn_kv4;
decltype(&dg4_qkv_proj_mx4) proj_mx4;
decltype(&dg4_qkv_proj_kv4) proj_kv4;
decltype(&dg4_ffn_mx4_fwd) ffn_mx4;
PyObject *error_class, *stream_of, *current_device;
// attribute names
PyObject *n_hidden, *n_heads, *n_hops, *n_dtype, *n_ln_eps, *n_packed, *n_k, *n_n;

struct Refused {};                                // an argument that does not fit (a Python error may be set already)

PyObject* raise(int status, const char* where)
{
    if (PyErr_Occurred()) return nullptr;
    if (PyObject* e = PyObject_CallFunction(error_class, "is", status, where)) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    return nullptr;
}

struct Ref {                                      // an owned reference
    PyObject* p;
    explicit Ref(PyObject* o) : p(o) { if (!o) throw Refused{}; }
    ~Ref() { Py_DECREF(p); }
    Ref(const Ref&) = delete;
};
int64_t integer(PyObject* o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}
int64_t integer_of(PyObject* o, PyObject* name) { return integer(Ref(PyObject_GetAttr(o, name)).p); }
int32_t small_of(PyObject* o, PyObject* name)
{
    const int64_t v = integer_of(o, name);
    if (v != (int32_t)v) throw Refused{};
    return (int32_t)v;
}

const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) throw Refused{};
    return THPVariable_Unpack(o);
}

// Configuration, element type, device and stream of a call whose tensors are where `first` is
struct Call {
    dg4_layer_cfg cfg{};
    at::ScalarType type;
    int64_t dev;
    void* stream;
    Call(PyObject* c, const at::Tensor& first)
    {
        cfg.hidden = small_of(c, n_hidden);
        cfg.heads = small_of(c, n_heads);
        cfg.hops = small_of(c, n_hops);
        cfg.n_layers = 1;
        const Ref eps(PyObject_GetAttr(c, n_ln_eps));
        cfg.ln_eps = (float)PyFloat_AsDouble(eps.p);
        if (PyErr_Occurred()) throw Refused{};
        const Ref dtype(PyObject_GetAttr(c, n_dtype));
        if (!PyUnicode_Check(dtype.p)) throw Refused{};
        if (PyUnicode_CompareWithASCIIString(dtype.p, "f32") == 0) { cfg.dtype = DG4_F32; type = at::kFloat; }
        else if (PyUnicode_CompareWithASCIIString(dtype.p, "bf16") == 0) { cfg.dtype = DG4_BF16; type = at::kBFloat16; }
        else throw Refused{};
        dev = first.get_device();
        if (dev < 0 || dev != integer(Ref(PyObject_CallNoArgs(current_device)).p)) throw Refused{};
        const Ref on(PyLong_FromLongLong(dev));
        const Ref s(PyObject_CallOneArg(stream_of, on.p));
        stream = PyLong_AsVoidPtr(s.p);
        if (PyErr_Occurred()) throw Refused{};
    }
    // The address of `count` contiguous elements of one type on the call's device
    void* at(const at::Tensor& t, at::ScalarType of, int64_t count) const
    {
        if (t.scalar_type() != of || t.get_device() != dev || !t.is_contiguous() || t.numel() != count) throw Refused{};
        return t.data_ptr();
    }
    void* rows(PyObject* o, int64_t n) const { return at(tensor(o), type, n * cfg.hidden); }
};

// Rows [begin, end) of n
struct Range {
    int64_t begin, end;
    Range(PyObject* b, PyObject* e, int64_t n) : begin(integer(b)), end(e == Py_None ? n : integer(e))
    {
        if (end > n) throw Refused{};
    }
    bool empty() const { return begin == end && end == 0; }    // (an empty tensor has no address)
};
int64_t first_size(const at::Tensor& t)
{
    if (t.dim() == 0) throw Refused{};
    return t.size(0);
}

// A store in 4 bits, and the store rows of a call's n rows
struct Store {
    int64_t n;
    uint8_t *codes, *scales;
    const int32_t* ids;
    Store(const Call& c, PyObject* codes_, PyObject* scales_, PyObject* ids_, int64_t rows)
    {
        const at::Tensor& k = tensor(codes_);
        n = first_size(k);
        codes = (uint8_t*)c.at(k, at::kByte, n * c.cfg.hidden);
        const at::Tensor& s = tensor(scales_);
        if (s.dim() != 3 || s.size(0) != n || s.size(1) != c.cfg.heads || s.size(2) != 2) throw Refused{};
        scales = (uint8_t*)c.at(s, at::kByte, n * c.cfg.heads * 2);
        ids = ids_ == Py_None ? nullptr : (const int32_t*)c.at(tensor(ids_), at::kInt, rows);
        listed = ids_ != Py_None;
    }
    bool listed;
};

// Weights [k, n] of dg4_mx4_pack
struct Packed {
    Ref packed;
    void* at;
    int64_t bytes;
    Packed(const Call& c, PyObject* w, int64_t k, int64_t n) : packed(PyObject_GetAttr(w, n_packed))
    {
        if (integer_of(w, n_hidden) != c.cfg.hidden || integer_of(w, n_k) != k || integer_of(w, n_n) != n) throw Refused{};
        const at::Tensor& t = tensor(packed.p);
        bytes = t.numel();
        at = c.at(t, at::kByte, bytes);
    }
};

// f(arguments): the C call's status, raised where it is an error
template <typename F> PyObject* call(const char* where, PyObject* const* a, Py_ssize_t given, Py_ssize_t wanted, F&& f)
{
    if (given != wanted) return PyErr_Format(PyExc_TypeError, "%s: %zd arguments, not %zd", where, given, wanted);
    int rc = DG4_EINVAL;
    try {
        rc = f(a);
    } catch (const Refused&) {
        return raise(DG4_EINVAL, where);
    } catch (const std::exception&) {
        return raise(DG4_EINVAL, where);
    }
    if (rc != DG4_OK) return raise(rc, where);
    Py_RETURN_NONE;
}
template <typename F> int launched(F&& f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// (cfg, K, V, codes, scales, ids, row_begin, row_end)
PyObject* py_write(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_kv4_write", args, n, 8, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[3]));
        const int64_t rows = first_size(tensor(a[1]));
        const Range r(a[6], a[7], rows);
        const Store s(c, a[3], a[4], a[5], rows);
        void *k = c.rows(a[1], rows), *v = c.rows(a[2], rows);
        if (r.empty() || (s.n == 0 && s.listed)) return (int)DG4_OK;
        return launched([&] { return kv4_write(&c.cfg, k, v, r.begin, r.end, s.ids, s.codes, s.scales, s.n, c.stream); });
    });
}

// (cfg, codes, scales, K, V, ids, row_begin, row_end)
PyObject* py_read(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_kv4_read", args, n, 8, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[1]));
        const int64_t rows = first_size(tensor(a[3]));
        const Range r(a[6], a[7], rows);
        const Store s(c, a[1], a[2], a[5], rows);
        void *k = c.rows(a[3], rows), *v = c.rows(a[4], rows);
        if (r.empty() || (s.n == 0 && s.listed)) return (int)DG4_OK;
        return launched([&] { return kv4_read(&c.cfg, s.codes, s.scales, s.n, s.ids, r.begin, r.end, k, v, c.stream); });
    });
}

// (cfg, address of the graph, its gates, Q, codes, scales, rel_bias, A, ids, row_begin, row_end)
PyObject* py_attn(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_sparse_attn_kv4_fwd", args, n, 11, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[4]));
        const int64_t rows = first_size(tensor(a[3]));
        const Range r(a[9], a[10], rows);
        const Store s(c, a[4], a[5], a[8], rows);
        void *q = c.rows(a[3], rows), *out = c.rows(a[7], rows);
        auto* bias = (const float*)c.at(tensor(a[6]), at::kFloat, 4 * c.cfg.heads);
        auto* g = (dg4_graph*)PyLong_AsVoidPtr(a[1]);
        if (PyErr_Occurred() || s.n < integer(a[2])) throw Refused{};
        if (r.empty() || (s.n == 0 && s.listed)) return (int)DG4_OK;
        return launched([&] { return attn_kv4(&c.cfg, g, r.begin, r.end, s.ids, q, s.codes, s.scales, bias, out, c.stream); });
    });
}

// (cfg, weights, S, Q, K, V, row_begin, row_end)
PyObject* py_proj(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_qkv_proj_mx4", args, n, 8, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[2]));
        const int64_t rows = first_size(tensor(a[2]));
        const Range r(a[6], a[7], rows);
        const Packed w(c, a[1], c.cfg.hidden, 3 * (int64_t)c.cfg.hidden);
        void *s = c.rows(a[2], rows), *q = c.rows(a[3], rows), *k = c.rows(a[4], rows), *v = c.rows(a[5], rows);
        if (r.empty()) return (int)DG4_OK;
        return launched([&] { return proj_mx4(&c.cfg, w.at, w.bytes, s, r.begin, r.end, q, k, v, c.stream); });
    });
}

// (cfg, weights, S, Q, codes, scales, ids, row_begin, row_end)
PyObject* py_proj_store(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_qkv_proj_kv4", args, n, 9, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[2]));
        const int64_t rows = first_size(tensor(a[2]));
        const Range r(a[7], a[8], rows);
        const Packed w(c, a[1], c.cfg.hidden, 3 * (int64_t)c.cfg.hidden);
        const Store store(c, a[4], a[5], a[6], rows);
        void *s = c.rows(a[2], rows), *q = c.rows(a[3], rows);
        if (r.empty()) return (int)DG4_OK;
        if (store.n == 0) throw Refused{};        // (it has no address, and rows of Q would have to be written all the same)
        return launched([&] { return proj_kv4(&c.cfg, w.at, w.bytes, s, r.begin, r.end, store.ids, q, store.codes, store.scales, store.n, c.stream); });
    });
}

// (cfg, W1, W2, S, Out, row_begin, row_end)
PyObject* py_ffn(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return call("dg4_ffn_mx4_fwd", args, n, 7, [](PyObject* const* a) {
        const Call c(a[0], tensor(a[3]));
        const int64_t rows = first_size(tensor(a[3])), d = c.cfg.hidden;
        const Range r(a[5], a[6], rows);
        const Packed w1(c, a[1], d, 4 * d), w2(c, a[2], 4 * d, d);
        void *s = c.rows(a[3], rows), *out = c.rows(a[4], rows);
        if (r.empty()) return (int)DG4_OK;
        return launched([&] { return ffn_mx4(&c.cfg, w1.at, w1.bytes, w2.at, w2.bytes, s, r.begin, r.end, out, c.stream); });
    });
}

// (addresses of the six entry points in the order above, class of errors, stream of a device, current device)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 9) return PyErr_Format(PyExc_TypeError, "bind: nine arguments");
    void* at[6];
    for (int i = 0; i < 6; ++i) at[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
    kv4_write = (decltype(kv4_write))at[0];
    kv4_read = (decltype(kv4_read))at[1];
    attn_kv4 = (decltype(attn_kv4))at[2];
    proj_mx4 = (decltype(proj_mx4))at[3];
    proj_kv4 = (decltype(proj_kv4))at[4];
    ffn_mx4 = (decltype(ffn_mx4))at[5];
    Py_INCREF(a[6]); Py_INCREF(a[7]); Py_INCREF(a[8]);
    error_class = a[6]; stream_of = a[7]; current_device = a[8];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    { "bind", (PyCFunction)(void (*)())py_bind, METH_FASTCALL, nullptr },
    { "kv4_write", (PyCFunction)(void (*)())py_write, METH_FASTCALL, nullptr },
    { "kv4_read", (PyCFunction)(void (*)())py_read, METH_FASTCALL, nullptr },
    { "sparse_attn_kv4_fwd", (PyCFunction)(void (*)())py_attn, METH_FASTCALL, nullptr },
    { "qkv_proj_mx4", (PyCFunction)(void (*)())py_proj, METH_FASTCALL, nullptr },
    { "qkv_proj_kv4", (PyCFunction)(void (*)())py_proj_store, METH_FASTCALL, nullptr },
    { "ffn_mx4_fwd", (PyCFunction)(void (*)())py_ffn, METH_FASTCALL, nullptr },
    { nullptr, nullptr, 0, nullptr },
};
PyModuleDef module = { PyModuleDef_HEAD_INIT, "_dg4_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr };

}  // namespace

PyMODINIT_FUNC PyInit__dg4_marshal()
{
    struct { PyObject** to; const char* name; } names[] = { { &n_hidden, "hidden" }, { &n_heads, "heads" }, { &n_hops, "hops" }, { &n_dtype, "dtype" },
                                                            { &n_ln_eps, "ln_eps" }, { &n_packed, "packed" }, { &n_k, "k" }, { &n_n, "n" } };
    for (auto& x : names)
        if (!(*x.to = PyUnicode_InternFromString(x.name))) return nullptr;
    return PyModule_Create(&module);
}
