// The calls of text generation from torch tensors: looks at the tensors, fills the descriptor, calls the library.
//
// A step of a few sequences has kernels of 4 to 8 us; looking at seven tensors from Python takes as long (0.1 us for every size, stride or
// type that is asked for), from here less than one.  What a tensor shows and the C side cannot see is checked here: types, shapes,
// elements that lie side by side, and that it is on a GPU.  The rest is the library's.

#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstddef>
#include <vector>

#include "freeride.h"

namespace {

struct Refused {};                         // (the Python error is set)

template <typename... X> [[noreturn]] void refuse(PyObject* kind, const char* text, X... x)
{
    PyErr_Format(kind, text, x...);
    throw Refused{};
}

int (*append)(const fr_kv_append_desc*, void*);
int (*attend)(const fr_attend_desc*, void*);
int (*sample)(const fr_sample_desc*, void*);
PyObject* current_stream;                  // (of a device's index: torch's current stream there)

bool given(PyObject* x) { return x != Py_None; }

const at::Tensor& tensor(PyObject* x, const char* name)
{
    if (!THPVariable_Check(x)) refuse(PyExc_TypeError, "%s: a torch tensor is needed", name);
    return THPVariable_Unpack(x);
}

int64_t whole(PyObject* x, const char* name, int64_t most = INT32_MAX)
{
    const long long y = PyLong_AsLongLong(x);
    if (y == -1 && PyErr_Occurred()) throw Refused{};
    if (y > most || y < -most - 1) refuse(PyExc_ValueError, "%s: %lld is out of range", name, y);
    return y;
}

int32_t number(int64_t x, const char* name)
{
    if (x > INT32_MAX) refuse(PyExc_ValueError, "%s: %lld is out of range", name, (long long)x);
    return (int32_t)x;
}

void* address(PyObject* stream, c10::Device device)
{
    PyObject* made = given(stream) ? nullptr : PyObject_CallFunction(current_stream, "i", (int)device.index());
    PyObject* of = given(stream) ? stream : made;
    PyObject* y = !of ? nullptr : PyLong_Check(of) ? Py_NewRef(of) : PyObject_GetAttrString(of, "cuda_stream");
    Py_XDECREF(made);
    if (!y) throw Refused{};
    void* p = PyLong_AsVoidPtr(y);
    Py_DECREF(y);
    if (!p && PyErr_Occurred()) throw Refused{};
    return p;
}

at::ScalarType type_of(int32_t dtype) { return dtype == FR_DTYPE_BF16 ? at::kBFloat16 : dtype == FR_DTYPE_F16 ? at::kHalf : at::kFloat; }

// The tensors of a call, to be looked at once more when everything else is right.
struct Call {
    const at::Tensor* seen[16];
    const char* names[16];
    int n = 0;

    void* of(const at::Tensor& t, const char* name)
    {
        seen[n] = &t;
        names[n++] = name;
        return t.data_ptr();
    }
    // Elements of a type that the C side cannot see, side by side in the last dimension; shape: sizes that are needed.
    template <typename P = void> P* typed(PyObject* x, const char* name, at::ScalarType type, std::initializer_list<int64_t> shape = {})
    {
        if (!given(x)) return nullptr;
        const at::Tensor& t = tensor(x, name);
        if (t.scalar_type() != type || (t.dim() && t.stride(-1) != 1 && t.size(-1) > 1))
            refuse(PyExc_TypeError, "%s: %s elements side by side are needed", name, c10::toString(type));
        if (shape.size() && !t.sizes().equals(shape)) refuse(PyExc_ValueError, "%s: another shape is needed", name);
        return static_cast<P*>(of(t, name));
    }
    // [tokens, heads, dim], a token's heads side by side
    void* rows(PyObject* x, const char* name, int64_t tokens, int64_t heads, int64_t dim, at::ScalarType type, int64_t& stride)
    {
        const at::Tensor& t = tensor(x, name);
        if (!t.sizes().equals({tokens, heads, dim}))
            refuse(PyExc_ValueError, "%s: shape (%lld, %lld, %lld) is needed", name, (long long)tokens, (long long)heads, (long long)dim);
        if (t.scalar_type() != type) refuse(PyExc_TypeError, "%s: not of the cache's type", name);
        if (t.numel() && ((dim > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != dim)))
            refuse(PyExc_ValueError, "%s: heads of a token have to lie side by side", name);
        stride = tokens > 1 ? t.stride(0) : heads * dim;
        return of(t, name);
    }
    void workspace(PyObject* x, void*& p, uint64_t& bytes)
    {
        if (!given(x)) return;
        const at::Tensor& t = tensor(x, "workspace");
        p = of(t, "workspace");
        bytes = t.nbytes();
    }
    void on_gpu() const
    {
        for (int i = 0; i < n; ++i) {
            if (!seen[i]->is_cuda()) refuse(PyExc_ValueError, "%s: not on a GPU", names[i]);
            if (seen[i]->device() != seen[0]->device()) refuse(PyExc_ValueError, "%s: on another GPU than %s", names[i], names[0]);
        }
    }
};

template <typename D> PyObject* made(int (*entry)(const D*, void*), const D& d, const Call& call, PyObject* stream)
{
    call.on_gpu();
    const c10::DeviceGuard guard(call.seen[0]->device());      // (the null stream is the current device's)
    void* s = address(stream, call.seen[0]->device());
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = entry(&d, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(code);
}

// x: the pages' descriptor, as bytes, and the two tensors that it was made of, which the kernels read and write as well
fr_kv_pages cache_of(PyObject* const* x, Call& call)
{
    fr_kv_pages cache;
    if (!PyBytes_Check(x[0]) || PyBytes_GET_SIZE(x[0]) != sizeof(cache) || !PyTuple_Check(x[1]) || PyTuple_GET_SIZE(x[1]) != 2)
        refuse(PyExc_TypeError, "cache: a KvPages is needed");
    memcpy(&cache, PyBytes_AS_STRING(x[0]), sizeof(cache));
    call.of(tensor(PyTuple_GET_ITEM(x[1], 0), "cache"), "cache k");
    call.of(tensor(PyTuple_GET_ITEM(x[1], 1), "cache"), "cache v");
    return cache;
}

// cache (two), k, v, slot, q, q_out, position, rotary, style, stream
PyObject* of_append(PyObject* const* x)
{
    fr_kv_append_desc d = {};
    Call call;
    d.cache = cache_of(x, call);
    ++x;
    const int64_t dim = d.cache.head_dim, heads = d.cache.n_kv_heads;
    const at::ScalarType type = type_of(d.cache.dtype);
    const at::Tensor& k = tensor(x[1], "k");
    const int64_t tokens = k.dim() ? k.size(0) : 0;
    d.n_tokens = number(tokens, "k");
    d.k = call.rows(x[1], "k", tokens, heads, dim, type, d.k_stride);
    d.v = call.rows(x[2], "v", tokens, heads, dim, type, d.v_stride);
    d.slot = call.typed<int64_t>(x[3], "slot", at::kLong, {tokens});
    if (given(x[4])) {
        const at::Tensor& q = tensor(x[4], "q");
        const int64_t n = q.dim() > 1 ? q.size(1) : 0;
        d.n_q_heads = number(n, "q");
        if (n) {
            d.q = call.rows(x[4], "q", tokens, n, dim, type, d.q_stride);
            d.q_out = call.rows(x[5], "q_out", tokens, n, dim, type, d.q_out_stride);
        }
    }
    if (given(x[7])) {
        const at::Tensor& t = tensor(x[7], "rotary");
        if (t.dim() != 2 || !t.is_contiguous()) refuse(PyExc_ValueError, "rotary: [positions, rotary_dim], rows side by side, is needed");
        d.rotary = call.typed<float>(x[7], "rotary", at::kFloat);
        d.n_positions = number(t.size(0), "rotary");
        d.rotary_dim = number(t.size(1), "rotary");
        if (d.rotary_dim) d.position = call.typed<int32_t>(x[6], "position", at::kInt, {tokens});
    }
    d.style = (int32_t)whole(x[8], "style");
    return made(append, d, call, x[9]);
}

// cache (two), q, out, pages, own_len, scale, prefix_len, max_own_len, prefix_pages, q_begin, max_q, lse, workspace, stream
PyObject* of_attend(PyObject* const* x)
{
    fr_attend_desc d = {};
    Call call;
    d.cache = cache_of(x, call);
    ++x;
    const int64_t dim = d.cache.head_dim, page = d.cache.page_size;
    const at::ScalarType type = type_of(d.cache.dtype);
    const at::Tensor& q = tensor(x[1], "q");
    if (q.dim() != 3) refuse(PyExc_ValueError, "q: [tokens, heads, head_dim] is needed");
    const int64_t tokens = q.size(0), heads = q.size(1);
    d.n_tokens = number(tokens, "q");
    d.n_q_heads = number(heads, "q");
    d.q = call.rows(x[1], "q", tokens, heads, dim, type, d.q_stride);
    d.out = call.rows(x[2], "out", tokens, heads, dim, type, d.out_stride);
    d.prefix_len = (int32_t)whole(x[6], "prefix_len");
    d.max_own_len = (int32_t)whole(x[7], "max_own_len");
    d.max_q = (int32_t)whole(x[10], "max_q");
    d.scale = (float)PyFloat_AsDouble(x[5]);
    if (PyErr_Occurred()) throw Refused{};
    int64_t seqs = tokens;
    if (given(x[9])) {
        const at::Tensor& t = tensor(x[9], "q_begin");
        if (t.dim() != 1 || t.size(0) < 1) refuse(PyExc_ValueError, "q_begin: [sequences + 1] is needed");
        seqs = t.size(0) - 1;
        d.q_begin = call.typed<int32_t>(x[9], "q_begin", at::kInt);
    }
    d.n_seqs = number(seqs, "q_begin");
    if (given(x[11])) {
        if (!tensor(x[11], "lse").is_contiguous()) refuse(PyExc_ValueError, "lse: rows have to lie side by side");
        d.lse = call.typed<float>(x[11], "lse", at::kFloat, {tokens, heads});
    }
    if (given(x[8])) {
        const at::Tensor& t = tensor(x[8], "prefix_pages");
        if (t.dim() != 1 || t.numel() * page < d.prefix_len) refuse(PyExc_ValueError, "prefix_pages: too few for prefix_len");
        d.prefix_pages = call.typed<int32_t>(x[8], "prefix_pages", at::kInt);
    }
    if (given(x[3])) {
        const at::Tensor& t = tensor(x[3], "pages");
        if (t.dim() != 2 || t.size(0) != seqs || t.size(1) * page < d.max_own_len)
            refuse(PyExc_ValueError, "pages: [n_seqs, at least max_own_len / page_size] is needed");
        d.pages = call.typed<int32_t>(x[3], "pages", at::kInt);
        d.pages_stride = seqs > 1 ? t.stride(0) : t.size(1);
        d.own_len = call.typed<int32_t>(x[4], "own_len", at::kInt, {seqs});
    }
    call.workspace(x[12], d.workspace, d.workspace_bytes);
    return made(attend, d, call, x[13]);
}

// logits, uniform, token, temperature, top_k, top_p, min_p, workspace, stream
PyObject* of_sample(PyObject* const* x)
{
    fr_sample_desc d = {};
    Call call;
    const at::Tensor& t = tensor(x[0], "logits");
    if (t.dim() != 2) refuse(PyExc_ValueError, "logits: [rows, vocabulary] is needed");
    const int64_t n = t.size(0), vocab = t.size(1);
    if (vocab > 1 && t.stride(1) != 1) refuse(PyExc_ValueError, "logits: the entries of a row have to lie side by side");
    const at::ScalarType type = t.scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf && type != at::kFloat)
        refuse(PyExc_TypeError, "logits: the library takes bfloat16, float16 and float32");
    d.dtype = type == at::kBFloat16 ? FR_DTYPE_BF16 : type == at::kHalf ? FR_DTYPE_F16 : FR_DTYPE_F32;
    d.n_rows = number(n, "logits");
    d.n_vocab = number(vocab, "logits");
    d.row_stride = n > 1 ? t.stride(0) : vocab;
    d.logits = call.of(t, "logits");
    d.uniform = call.typed<float>(x[1], "uniform", at::kFloat, {n});
    d.token = call.typed<int32_t>(x[2], "token", at::kInt, {n});
    d.temperature = call.typed<float>(x[3], "temperature", at::kFloat, {n});
    d.top_k = call.typed<int32_t>(x[4], "top_k", at::kInt, {n});
    d.top_p = call.typed<float>(x[5], "top_p", at::kFloat, {n});
    d.min_p = call.typed<float>(x[6], "min_p", at::kFloat, {n});
    call.workspace(x[7], d.workspace, d.workspace_bytes);
    return made(sample, d, call, x[8]);
}

// No C++ exception leaves: what was refused has its Python error set, anything else becomes one.
template <PyObject* (*kCall)(PyObject* const*), int kArguments> PyObject* guarded(PyObject*, PyObject* const* x, Py_ssize_t n)
{
    if (n != kArguments) return PyErr_Format(PyExc_TypeError, "%d arguments are needed", kArguments);
    try {
        return kCall(x);
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// the library's entries, as addresses: fr_kv_append, fr_attend_shared, fr_sample; and what gives torch's current stream of a device
PyObject* entries(PyObject*, PyObject* const* x, Py_ssize_t n)
{
    void* p[3];
    if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments are needed");
    for (int i = 0; i < 3; ++i)
        if (!(p[i] = PyLong_AsVoidPtr(x[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "an address is needed");
    append = reinterpret_cast<decltype(append)>(p[0]);
    attend = reinterpret_cast<decltype(attend)>(p[1]);
    sample = reinterpret_cast<decltype(sample)>(p[2]);
    Py_XSETREF(current_stream, Py_NewRef(x[3]));
    Py_RETURN_NONE;
}

// Where the fields of the descriptors lie, and their sizes, as this file was compiled: to be compared with the binding's.
PyObject* layout(PyObject*, PyObject* const*, Py_ssize_t)
{
#define AT(S, f) (long)offsetof(S, f)
    static const std::vector<long> structs[] = {
#define F(f) AT(fr_kv_pages, f)
        {F(k), F(v), F(n_pages), F(page_stride), F(head_stride), F(slot_stride), F(n_kv_heads), F(head_dim), F(page_size), F(dtype), sizeof(fr_kv_pages)},
#undef F
#define F(f) AT(fr_kv_append_desc, f)
        {F(cache), F(k), F(v), F(q), F(q_out), F(k_stride), F(v_stride), F(q_stride), F(q_out_stride), F(slot), F(position), F(rotary), F(n_positions),
         F(rotary_dim), F(style), F(n_tokens), F(n_q_heads), F(reserved), sizeof(fr_kv_append_desc)},
#undef F
#define F(f) AT(fr_attend_desc, f)
        {F(cache), F(q), F(out), F(lse), F(q_stride), F(out_stride), F(q_begin), F(prefix_pages), F(pages), F(own_len), F(pages_stride), F(n_tokens),
         F(n_seqs), F(n_q_heads), F(max_q), F(prefix_len), F(max_own_len), F(scale), F(reserved), F(workspace), F(workspace_bytes), sizeof(fr_attend_desc)},
#undef F
#define F(f) AT(fr_sample_desc, f)
        {F(logits), F(row_stride), F(dtype), F(n_rows), F(n_vocab), F(reserved), F(temperature), F(top_k), F(top_p), F(min_p), F(uniform), F(token),
         F(workspace), F(workspace_bytes), sizeof(fr_sample_desc)},
#undef F
#undef AT
    };
    PyObject* all = PyList_New(0);
    for (const auto& s : structs)
        for (long x : s) {
            PyObject* y = all ? PyLong_FromLong(x) : nullptr;
            if (!y || PyList_Append(all, y)) Py_CLEAR(all);
            Py_XDECREF(y);
        }
    return all;
}

template <typename F> PyCFunction method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef methods[] = {
    {"layout", method(layout), METH_FASTCALL, nullptr},
    {"entries", method(entries), METH_FASTCALL, nullptr},
    {"kv_append", method(guarded<of_append, 11>), METH_FASTCALL, nullptr},
    {"attend_shared", method(guarded<of_attend, 15>), METH_FASTCALL, nullptr},
    {"sample", method(guarded<of_sample, 9>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module_def); }
