// The calls around the mixers as Python functions of torch tensors: each tensor is checked against the call's descriptor (shape, type, unit
// stride along a row, on the GPU), then the C ABI is called.  Host code only.  The same checks written in Python around ctypes cost a small
// call more than its kernel takes (layer norm of 16 x 32 rows of 2048: 7.4 us a call, now 3.9).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <initializer_list>
#include <string>

#include "bimamba.h"

namespace {

at::ScalarType scalar_of(int dtype) { return dtype == BIMAMBA_BF16 ? at::kBFloat16 : at::kFloat; }

std::string shape_of(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); i++) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

// What a call's arguments are read with.  The first one that is not as it has to be leaves an AssertionError; everything after it is
// passed over.
class Reader {
public:
    bool good() const { return good_; }

    // A descriptor: the bytes of a ctypes structure.
    template <typename Desc>
    Desc desc(PyObject* o)
    {
        Desc d{};
        Py_buffer b;
        if (!good_) return d;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
            good_ = false;
            return d;
        }
        if (b.len == (Py_ssize_t)sizeof d) std::memcpy(&d, b.buf, sizeof d);
        else fail("a descriptor of another call");
        PyBuffer_Release(&b);
        return d;
    }

    // [batch, L, width] activations, the channels contiguous.
    bimamba_tensor rows(PyObject* o, const char* what, int dtype, int64_t batch, int64_t L, int64_t width)
    {
        const at::Tensor* const t = tensor(o, what, scalar_of(dtype), {batch, L, width});
        if (!t) return {};
        if (t->stride(2) != 1 && width != 1 && t->numel() != 0) wrong(*t, what, scalar_of(dtype), {batch, L, width}, ", the channels contiguous");
        return bimamba_tensor{t->data_ptr(), t->stride(0), t->stride(1)};
    }
    bimamba_tokens ids(PyObject* o, const char* what, int64_t batch, int64_t L)
    {
        const at::Tensor* const t = tensor(o, what, at::kLong, {batch, L});
        if (!t) return {};
        return bimamba_tokens{static_cast<const int64_t*>(t->data_ptr()), t->stride(0), t->stride(1)};
    }
    // A contiguous array, or None.
    template <typename T = float>
    T* flat(PyObject* o, const char* what, std::initializer_list<int64_t> shape, at::ScalarType type = at::kFloat)
    {
        if (o == Py_None) return nullptr;
        const at::Tensor* const t = tensor(o, what, type, shape);
        if (!t) return nullptr;
        if (!t->is_contiguous()) wrong(*t, what, type, shape, ", contiguous");
        return static_cast<T*>(t->data_ptr());
    }
    // A parameter vector [d], or one for each batch element [batch, d], each contiguous; stride -1: None.
    struct Vector {
        float* p;
        int64_t stride;
    };
    Vector vector(PyObject* o, const char* what, int64_t batch, int64_t d)
    {
        if (o == Py_None || !good_) return {nullptr, -1};
        if (!is_tensor(o, what)) return {nullptr, -1};
        const at::Tensor& t = THPVariable_Unpack(o);
        const bool one = t.dim() == 1 && t.size(0) == d, each = t.dim() == 2 && t.size(0) == batch && t.size(1) == d;
        if (t.scalar_type() != at::kFloat || !t.is_cuda() || (!one && !each)) wrong(t, what, at::kFloat, {batch, d}, ", or one vector");
        else if (t.stride(-1) != 1 && d != 1 && t.numel() != 0) wrong(t, what, at::kFloat, {batch, d}, ", each vector contiguous");
        else if (each && batch > 1 && t.stride(0) < d) wrong(t, what, at::kFloat, {batch, d}, ", the vectors apart");
        if (!good_) return {nullptr, -1};
        return {static_cast<float*>(t.data_ptr()), one ? 0 : batch > 1 ? t.stride(0) : d};
    }
    struct Bytes {
        void* p;
        size_t n;
    };
    Bytes workspace(PyObject* o)
    {
        if (o == Py_None || !good_ || !is_tensor(o, "workspace")) return {nullptr, 0};
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) fail("workspace: wanted contiguous, on the GPU");
        return {t.data_ptr(), t.nbytes()};
    }
    void* stream(PyObject* o)
    {
        void* const p = PyLong_AsVoidPtr(o);
        if (PyErr_Occurred()) good_ = false;
        return p;
    }
    void fail(const std::string& text)
    {
        if (good_) PyErr_SetString(PyExc_AssertionError, text.c_str());
        good_ = false;
    }

private:
    bool is_tensor(PyObject* o, const char* what)
    {
        if (!THPVariable_Check(o)) fail(std::string(what) + ": not a tensor");
        return good_;
    }
    const at::Tensor* tensor(PyObject* o, const char* what, at::ScalarType type, std::initializer_list<int64_t> shape)
    {
        if (!good_ || !is_tensor(o, what)) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.scalar_type() == type && t.is_cuda() && t.sizes() == at::IntArrayRef(shape)) return &t;
        wrong(t, what, type, shape, "");
        return nullptr;
    }
    void wrong(const at::Tensor& t, const char* what, at::ScalarType type, at::IntArrayRef shape, const char* more)
    {
        fail(std::string(what) + ": " + at::toString(t.scalar_type()) + " " + shape_of(t.sizes()) + " with strides " + shape_of(t.strides()) + " on " +
             t.device().str() + ", wanted " + at::toString(type) + " " + shape_of(shape) + " on the GPU" + more);
    }
    bool good_ = true;
};

// The call itself, without the interpreter's lock; its status.
template <typename Call>
PyObject* status_of(const Reader& r, Call call)
{
    if (!r.good()) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

bool takes(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, wanted %zd", n, want);
    return n == want;
}

// No C++ exception passes into the interpreter.
template <PyObject* (*kCall)(PyObject* const*)>
PyObject* guarded(PyObject* const* a)
{
    try {
        return kCall(a);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
template <PyObject* (*kCall)(PyObject* const*), int kArgs>
PyObject* method(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return takes(n, kArgs) ? guarded<kCall>(a) : nullptr;
}

PyObject* embed(PyObject* const* a)   // desc, tokens, table, out, stream
{
    Reader r;
    const auto d = r.desc<bimamba_embed_desc>(a[0]);
    const auto tokens = r.ids(a[1], "tokens", d.batch, d.seqlen);
    void* const table = r.flat<void>(a[2], "table", {d.vocab, d.d_model}, scalar_of(d.table_dtype));
    const auto out = r.rows(a[3], "out", d.io_dtype, d.batch, d.seqlen, d.d_model);
    void* const st = r.stream(a[4]);
    return status_of(r, [&] { return bimamba_embed(&d, &tokens, table, &out, st); });
}
PyObject* embed_bwd(PyObject* const* a)   // desc, tokens, dout, dtable, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_embed_desc>(a[0]);
    const auto tokens = r.ids(a[1], "tokens", d.batch, d.seqlen);
    const auto dout = r.rows(a[2], "dout", d.io_dtype, d.batch, d.seqlen, d.d_model);
    float* const dtable = r.flat(a[3], "dtable", {d.vocab, d.d_model});
    const auto ws = r.workspace(a[4]);
    void* const st = r.stream(a[5]);
    return status_of(r, [&] { return bimamba_embed_bwd(&d, &tokens, &dout, dtable, ws.p, ws.n, st); });
}
PyObject* layer_norm(PyObject* const* a)   // desc, x, weight, bias, y, mean, rstd, stream
{
    Reader r;
    const auto d = r.desc<bimamba_norm_desc>(a[0]);
    const auto x = r.rows(a[1], "x", d.io_dtype, d.batch, d.seqlen, d.d_model);
    const auto w = r.vector(a[2], "weight", d.batch, d.d_model), b = r.vector(a[3], "bias", d.batch, d.d_model);
    if (w.stride >= 0 && b.stride >= 0 && w.stride != b.stride) r.fail("weight and bias: not of the same kind and stride");
    const auto y = r.rows(a[4], "y", d.io_dtype, d.batch, d.seqlen, d.d_model);
    float* const mean = r.flat(a[5], "mean", {d.batch, d.seqlen});
    float* const rstd = r.flat(a[6], "rstd", {d.batch, d.seqlen});
    void* const st = r.stream(a[7]);
    const int64_t stride = w.stride >= 0 ? w.stride : b.stride >= 0 ? b.stride : 0;
    return status_of(r, [&] { return bimamba_layer_norm(&d, &x, w.p, b.p, stride, &y, mean, rstd, st); });
}
PyObject* layer_norm_bwd(PyObject* const* a)   // desc, x, weight, mean, rstd, dy, dx, dweight, dbias, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_norm_desc>(a[0]);
    const auto x = r.rows(a[1], "x", d.io_dtype, d.batch, d.seqlen, d.d_model);
    auto w = r.vector(a[2], "weight", d.batch, d.d_model);
    float* const mean = r.flat(a[3], "mean", {d.batch, d.seqlen});
    float* const rstd = r.flat(a[4], "rstd", {d.batch, d.seqlen});
    const auto dy = r.rows(a[5], "dy", d.io_dtype, d.batch, d.seqlen, d.d_model);
    const auto dx = r.rows(a[6], "dx", d.io_dtype, d.batch, d.seqlen, d.d_model);
    if (w.stride < 0) {   // (no weight: the gradients' shape says whether each batch element has vectors of its own)
        const auto each = [](PyObject* o) { return o != Py_None && THPVariable_Check(o) && THPVariable_Unpack(o).dim() == 2; };
        w.stride = each(a[7]) || each(a[8]) ? d.d_model : 0;
    }
    const auto grad = [&](PyObject* o, const char* what) {
        return w.stride ? r.flat(o, what, {d.batch, d.d_model}) : r.flat(o, what, {d.d_model});
    };
    float* const dweight = grad(a[7], "dweight");
    float* const dbias = grad(a[8], "dbias");
    const auto ws = r.workspace(a[9]);
    void* const st = r.stream(a[10]);
    return status_of(r, [&] { return bimamba_layer_norm_bwd(&d, &x, w.p, w.stride, mean, rstd, &dy, &dx, dweight, dbias, ws.p, ws.n, st); });
}
PyObject* log_probs(PyObject* const* a)   // desc, logits, targets, logp, lse, entropy, top_logp, top_token, lse_rest, workspace, stream
{
    Reader r;
    auto d = r.desc<bimamba_logits_desc>(a[0]);
    const auto logits = r.rows(a[1], "logits", d.io_dtype, d.batch, d.seqlen, d.vocab);
    const bool has = a[2] != Py_None;
    const auto targets = has ? r.ids(a[2], "targets", d.batch, d.seqlen) : bimamba_tokens{};
    bimamba_scores out{};
    out.logp = r.flat(a[3], "logp", {d.batch, d.seqlen});
    out.lse = r.flat(a[4], "lse", {d.batch, d.seqlen});
    out.entropy = r.flat(a[5], "entropy", {d.batch, d.seqlen});
    out.top_logp = r.flat(a[6], "top_logp", {d.batch, d.seqlen, d.top_k});
    out.top_token = r.flat<int64_t>(a[7], "top_token", {d.batch, d.seqlen, d.top_k}, at::kLong);
    if (a[8] != Py_None) d.lse_rest = r.flat(a[8], "lse_rest", {d.batch, d.seqlen});
    const auto ws = r.workspace(a[9]);
    void* const st = r.stream(a[10]);
    return status_of(r, [&] { return bimamba_log_probs(&d, &logits, has ? &targets : nullptr, &out, ws.p, ws.n, st); });
}
PyObject* log_probs_bwd(PyObject* const* a)   // desc, logits, targets, lse, lse_rest, entropy, dlogp, dentropy, dlogits, stream
{
    Reader r;
    auto d = r.desc<bimamba_logits_desc>(a[0]);
    const auto logits = r.rows(a[1], "logits", d.io_dtype, d.batch, d.seqlen, d.vocab);
    const bool has = a[2] != Py_None;
    const auto targets = has ? r.ids(a[2], "targets", d.batch, d.seqlen) : bimamba_tokens{};
    const float* const lse = r.flat(a[3], "lse", {d.batch, d.seqlen});
    if (a[4] != Py_None) d.lse_rest = r.flat(a[4], "lse_rest", {d.batch, d.seqlen});
    const float* const entropy = r.flat(a[5], "entropy", {d.batch, d.seqlen});
    const float* const dlogp = r.flat(a[6], "dlogp", {d.batch, d.seqlen});
    const float* const dentropy = r.flat(a[7], "dentropy", {d.batch, d.seqlen});
    const auto dlogits = r.rows(a[8], "dlogits", d.io_dtype, d.batch, d.seqlen, d.vocab);
    void* const st = r.stream(a[9]);
    return status_of(r, [&] { return bimamba_log_probs_bwd(&d, &logits, has ? &targets : nullptr, lse, entropy, dlogp, dentropy, &dlogits, st); });
}
PyObject* clip_grads(PyObject* const* a)   // the host table's bytes, its copy on the device or None, max_norm, norm, workspace, stream
{
    Reader r;
    Py_buffer table;
    if (PyObject_GetBuffer(a[0], &table, PyBUF_SIMPLE) != 0) return nullptr;
    const int n = (int)(table.len / (Py_ssize_t)sizeof(bimamba_grad));
    const auto dev = r.workspace(a[1]);
    const double max_norm = PyFloat_AsDouble(a[2]);
    if (PyErr_Occurred()) {
        PyBuffer_Release(&table);
        return nullptr;
    }
    if (dev.n != (size_t)table.len) r.fail("the table and its copy: not of one length");
    float* const norm = r.flat(a[3], "norm", {1});
    const auto ws = r.workspace(a[4]);
    void* const st = r.stream(a[5]);
    PyObject* const rc = status_of(r, [&] {
        return bimamba_clip_grads(static_cast<const bimamba_grad*>(table.buf), n, dev.p, (float)max_norm, norm, ws.p, ws.n, st);
    });
    PyBuffer_Release(&table);
    return rc;
}

// A view, or None: a null pointer then.
struct Maybe {
    bimamba_tensor t;
    bool has;
    const bimamba_tensor* operator()() const { return has ? &t : nullptr; }
};
template <typename Desc>
Maybe maybe_rows(Reader& r, PyObject* o, const char* what, const Desc& d, int64_t width)
{
    const bool has = o != Py_None;
    return {has ? r.rows(o, what, d.io_dtype, d.batch, d.seqlen, width) : bimamba_tensor{}, has};
}

PyObject* recurrence(PyObject* const* a)   // desc, x, g, bias, add, lengths, h_in, y, h_out, states, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_recurrence_desc>(a[0]);
    const int64_t D = d.d_inner, kept = (int64_t(d.seqlen) + BIMAMBA_RECURRENCE_KEEP - 1) / BIMAMBA_RECURRENCE_KEEP;
    const auto x = r.rows(a[1], "x", d.io_dtype, d.batch, d.seqlen, D), g = r.rows(a[2], "g", d.io_dtype, d.batch, d.seqlen, D);
    const float* const bias = r.flat(a[3], "bias", {D});
    const auto add = maybe_rows(r, a[4], "add", d, D);
    const int64_t* const lengths = r.flat<int64_t>(a[5], "lengths", {d.batch}, at::kLong);
    const float* const h_in = r.flat(a[6], "h_in", {d.batch, D});
    const auto y = r.rows(a[7], "y", d.io_dtype, d.batch, d.seqlen, D);
    float* const h_out = r.flat(a[8], "h_out", {d.batch, D});
    float* const states = r.flat(a[9], "states", {d.batch, kept, D});
    const auto ws = r.workspace(a[10]);
    void* const st = r.stream(a[11]);
    return status_of(r, [&] { return bimamba_recurrence(&d, &x, &g, bias, add(), lengths, h_in, &y, h_out, states, ws.p, ws.n, st); });
}
PyObject* recurrence_bwd(PyObject* const* a)   // desc, x, g, bias, lengths, states, dy, dh_out, dx, dg, dbias, dh_in, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_recurrence_desc>(a[0]);
    const int64_t D = d.d_inner, kept = (int64_t(d.seqlen) + BIMAMBA_RECURRENCE_KEEP - 1) / BIMAMBA_RECURRENCE_KEEP;
    const auto view = [&](PyObject* o, const char* what) { return r.rows(o, what, d.io_dtype, d.batch, d.seqlen, D); };
    const auto x = view(a[1], "x"), g = view(a[2], "g");
    const float* const bias = r.flat(a[3], "bias", {D});
    const int64_t* const lengths = r.flat<int64_t>(a[4], "lengths", {d.batch}, at::kLong);
    const float* const states = r.flat(a[5], "states", {d.batch, kept, D});
    const auto dy = view(a[6], "dy");
    const float* const dh_out = r.flat(a[7], "dh_out", {d.batch, D});
    const auto dx = view(a[8], "dx"), dg = view(a[9], "dg");
    float* const dbias = r.flat(a[10], "dbias", {D});
    float* const dh_in = r.flat(a[11], "dh_in", {d.batch, D});
    const auto ws = r.workspace(a[12]);
    void* const st = r.stream(a[13]);
    return status_of(r, [&] {
        return bimamba_recurrence_bwd(&d, &x, &g, bias, lengths, states, &dy, dh_out, &dx, &dg, dbias, dh_in, ws.p, ws.n, st);
    });
}
PyObject* group_norm(PyObject* const* a)   // desc, x, z, weight, bias, y, mean, rstd, stream
{
    Reader r;
    const auto d = r.desc<bimamba_group_norm_desc>(a[0]);
    const int64_t D = d.d_inner;
    const auto x = r.rows(a[1], "x", d.io_dtype, d.batch, d.seqlen, D);
    const auto z = maybe_rows(r, a[2], "z", d, D);
    const float *const weight = r.flat(a[3], "weight", {D}), *const bias = r.flat(a[4], "bias", {D});
    const auto y = r.rows(a[5], "y", d.io_dtype, d.batch, d.seqlen, D);
    float* const mean = r.flat(a[6], "mean", {d.batch, d.seqlen, d.groups});
    float* const rstd = r.flat(a[7], "rstd", {d.batch, d.seqlen, d.groups});
    void* const st = r.stream(a[8]);
    return status_of(r, [&] { return bimamba_group_norm(&d, &x, z(), weight, bias, &y, mean, rstd, st); });
}
PyObject* group_norm_bwd(PyObject* const* a)   // desc, x, z, weight, bias, mean, rstd, dy, dx, dz, dweight, dbias, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_group_norm_desc>(a[0]);
    const int64_t D = d.d_inner;
    const auto x = r.rows(a[1], "x", d.io_dtype, d.batch, d.seqlen, D);
    const auto z = maybe_rows(r, a[2], "z", d, D);
    const float *const weight = r.flat(a[3], "weight", {D}), *const bias = r.flat(a[4], "bias", {D});
    const float* const mean = r.flat(a[5], "mean", {d.batch, d.seqlen, d.groups});
    const float* const rstd = r.flat(a[6], "rstd", {d.batch, d.seqlen, d.groups});
    const auto dy = r.rows(a[7], "dy", d.io_dtype, d.batch, d.seqlen, D), dx = r.rows(a[8], "dx", d.io_dtype, d.batch, d.seqlen, D);
    const auto dz = maybe_rows(r, a[9], "dz", d, D);
    float *const dweight = r.flat(a[10], "dweight", {D}), *const dbias = r.flat(a[11], "dbias", {D});
    const auto ws = r.workspace(a[12]);
    void* const st = r.stream(a[13]);
    return status_of(r, [&] { return bimamba_group_norm_bwd(&d, &x, z(), weight, bias, mean, rstd, &dy, &dx, dz(), dweight, dbias, ws.p, ws.n, st); });
}
const int64_t* key_of(Reader& r, PyObject* o)
{
    if (o == Py_None) r.fail("key: not a tensor");
    return r.flat<int64_t>(o, "key", {2}, at::kLong);
}
PyObject* dropout_add(PyObject* const* a)   // desc, key, x, gate, residual, out, stream
{
    Reader r;
    const auto d = r.desc<bimamba_dropout_desc>(a[0]);
    const int64_t* const key = key_of(r, a[1]);
    const auto x = r.rows(a[2], "x", d.io_dtype, d.batch, d.seqlen, d.d_model);
    const auto gate = r.vector(a[3], "gate", d.batch, d.d_model);
    const auto residual = maybe_rows(r, a[4], "residual", d, d.d_model);
    const auto out = r.rows(a[5], "out", d.io_dtype, d.batch, d.seqlen, d.d_model);
    void* const st = r.stream(a[6]);
    return status_of(r, [&] { return bimamba_dropout_add(&d, key, &x, gate.p, gate.stride < 0 ? 0 : gate.stride, residual(), &out, st); });
}
PyObject* dropout_add_bwd(PyObject* const* a)   // desc, key, x, gate, dout, dx, dgate, workspace, stream
{
    Reader r;
    const auto d = r.desc<bimamba_dropout_desc>(a[0]);
    const int64_t* const key = key_of(r, a[1]);
    const auto x = maybe_rows(r, a[2], "x", d, d.d_model);
    auto gate = r.vector(a[3], "gate", d.batch, d.d_model);
    const auto dout = r.rows(a[4], "dout", d.io_dtype, d.batch, d.seqlen, d.d_model), dx = r.rows(a[5], "dx", d.io_dtype, d.batch, d.seqlen, d.d_model);
    if (gate.stride < 0) gate.stride = a[6] != Py_None && THPVariable_Check(a[6]) && THPVariable_Unpack(a[6]).dim() == 2 ? d.d_model : 0;
    float* const dgate = gate.stride ? r.flat(a[6], "dgate", {d.batch, d.d_model}) : r.flat(a[6], "dgate", {d.d_model});
    const auto ws = r.workspace(a[7]);
    void* const st = r.stream(a[8]);
    return status_of(r, [&] { return bimamba_dropout_add_bwd(&d, key, x(), gate.p, gate.stride, &dout, &dx, dgate, ws.p, ws.n, st); });
}

#define BM_METHOD(name, args) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&method<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BM_METHOD(embed, 5),      BM_METHOD(embed_bwd, 6),      BM_METHOD(layer_norm, 8),
                         BM_METHOD(layer_norm_bwd, 11), BM_METHOD(log_probs, 11), BM_METHOD(log_probs_bwd, 10),
                         BM_METHOD(clip_grads, 6), BM_METHOD(recurrence, 12), BM_METHOD(recurrence_bwd, 14),
                         BM_METHOD(group_norm, 9), BM_METHOD(group_norm_bwd, 14), BM_METHOD(dropout_add, 7),
                         BM_METHOD(dropout_add_bwd, 9), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "The library's calls as functions of torch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
