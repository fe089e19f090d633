// The plain forms of the smallest calls without the interpreter's part: rows in, new buffers out, on the current stream.  A call of a
// few microseconds on the GPU is bound by what happens before it; the checks, the allocations and the argument marshalling of
// binding.py take 6 us, here about one.  Whatever is not plain (given buffers, other types, shapes, strides or devices, anything
// that throws) is answered with None, and binding.py does the call or raises as it always did: there is no second set of rules.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/bfq.h"

namespace {

using ForwardQuant = int (*)(bfq_plan*, const void*, bfq_dtype, int64_t, int64_t, int, uint8_t*, uint16_t*, void*);
using Rows = int (*)(bfq_plan*, const void*, bfq_dtype, int64_t, int64_t, void*, bfq_dtype, int64_t, void*);
ForwardQuant forward_quant_fn = nullptr;
Rows forward_fn = nullptr, inverse_fn = nullptr;
decltype(&bfq_kv_append) append_fn = nullptr;
decltype(&bfq_kv_read) read_fn = nullptr;
decltype(&bfq_kv_attend_workspace) workspace_fn = nullptr;
decltype(&bfq_kv_attend) attend_fn = nullptr;

struct Call {
    bfq_plan* plan;
    int64_t n;
    int device;
    const at::Tensor* x;
    bfq_dtype type;
    int64_t rows, ld;
};

// arguments (plan handle, n, device index, x): false if x is not plain rows of n numbers on that device
bool plain_rows(PyObject* const* args, Call* call) {
    if (!THPVariable_CheckExact(args[3])) return false;
    call->plan = static_cast<bfq_plan*>(PyLong_AsVoidPtr(args[0]));
    call->n = PyLong_AsLongLong(args[1]);
    call->device = static_cast<int>(PyLong_AsLong(args[2]));
    if (PyErr_Occurred() || call->plan == nullptr) {
        PyErr_Clear();
        return false;
    }
    const at::Tensor& x = THPVariable_Unpack(args[3]);
    if (!x.is_cuda() || x.get_device() != call->device || x.dim() != 2) return false;
    const auto type = x.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) return false;
    call->x = &x, call->type = type == at::kFloat ? BFQ_F32 : BFQ_BF16;
    call->rows = x.size(0), call->ld = x.stride(0);
    return call->rows > 0 && x.size(1) == call->n && x.stride(1) == 1 && call->ld >= call->n;
}

// f(stream) without the interpreter's lock
template <class F>
int launch(int device, F&& f) {
    void* stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(stream);
    Py_END_ALLOW_THREADS
    return status;
}

// forward_quant(plan, n, device, x, bits) -> (codes, scales), or a status, or None
PyObject* forward_quant(PyObject*, PyObject* const* args, Py_ssize_t count) {
    try {
        Call call;
        if (count != 5 || forward_quant_fn == nullptr || !PyLong_CheckExact(args[4]) || !plain_rows(args, &call)) Py_RETURN_NONE;
        const long bits = PyLong_AsLong(args[4]);
        if (bits != 2 && bits != 4 && bits != 8) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const c10::Device device(c10::kCUDA, static_cast<c10::DeviceIndex>(call.device));
        at::Tensor codes = at::empty({call.rows, call.n * bits / 8}, at::TensorOptions().dtype(at::kByte).device(device));
        at::Tensor scales = at::empty({call.rows}, at::TensorOptions().dtype(at::kHalf).device(device));
        const void* x = call.x->data_ptr();
        uint8_t* to = static_cast<uint8_t*>(codes.data_ptr());
        uint16_t* scale = static_cast<uint16_t*>(scales.data_ptr());
        const int status = launch(call.device, [&](void* stream) {
            return forward_quant_fn(call.plan, x, call.type, call.rows, call.ld, static_cast<int>(bits), to, scale, stream);
        });
        if (status != BFQ_OK) return PyLong_FromLong(status);
        PyObject* first = THPVariable_Wrap(std::move(codes));
        PyObject* second = first != nullptr ? THPVariable_Wrap(std::move(scales)) : nullptr;
        PyObject* both = second != nullptr ? PyTuple_Pack(2, first, second) : nullptr;
        Py_XDECREF(first), Py_XDECREF(second);
        return both;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// forward / inverse(plan, n, device, x) -> rows in the type of x, or a status, or None
PyObject* rows_call(Rows fn, PyObject* const* args, Py_ssize_t count) {
    try {
        Call call;
        if (count != 4 || fn == nullptr || !plain_rows(args, &call)) Py_RETURN_NONE;
        at::Tensor y = at::empty({call.rows, call.n}, call.x->options());
        const void* x = call.x->data_ptr();
        void* to = y.data_ptr();
        const int status = launch(call.device, [&](void* stream) { return fn(call.plan, x, call.type, call.rows, call.ld, to, call.type, call.n, stream); });
        if (status != BFQ_OK) return PyLong_FromLong(status);
        return THPVariable_Wrap(std::move(y));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t count) { return rows_call(forward_fn, args, count); }
PyObject* inverse(PyObject*, PyObject* const* args, Py_ssize_t count) { return rows_call(inverse_fn, args, count); }

// ---- the paged cache of keys and values -------------------------------------------------------------------------------
// The plan's head dimension and device, and its cache; every check below is binding.py's and kv_cache.py's.
struct CacheCall {
    bfq_plan* plan;
    int64_t n;
    int device;
    bfq_kv_cache cache;
};
bool here(const CacheCall& call, const at::Tensor& t) { return t.is_cuda() && t.get_device() == call.device; }

// a tensor of this type and number of dimensions on the plan's device; null: anything else
const at::Tensor* tensor(const CacheCall& call, PyObject* o, at::ScalarType type, int64_t dims) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return here(call, t) && t.scalar_type() == type && t.dim() == dims ? &t : nullptr;
}
const at::Tensor* vector(const CacheCall& call, PyObject* o, at::ScalarType type, int64_t size) {
    const at::Tensor* t = tensor(call, o, type, 1);
    return t != nullptr && t->size(0) == size && t->is_contiguous() ? t : nullptr;
}

// arguments (plan handle, n, device index, k_codes, k_scales, v_codes, v_scales, bits)
constexpr int kCacheArgs = 8;
bool cache_call(PyObject* const* args, CacheCall* call) {
    call->plan = static_cast<bfq_plan*>(PyLong_AsVoidPtr(args[0]));
    call->n = PyLong_AsLongLong(args[1]);
    call->device = static_cast<int>(PyLong_AsLong(args[2]));
    const long bits = PyLong_AsLong(args[7]);
    if (PyErr_Occurred() || call->plan == nullptr || (bits != 4 && bits != 8)) {
        PyErr_Clear();
        return false;
    }
    const at::Tensor* t[4];
    for (int i = 0; i < 4; ++i)
        if ((t[i] = tensor(*call, args[3 + i], i % 2 == 0 ? at::kByte : at::kHalf, 4 - i % 2)) == nullptr) return false;
    const int64_t pages = t[0]->size(0), heads = t[0]->size(1), places = t[0]->size(2), width = t[0]->size(3);
    if (pages < 1 || heads < 1 || heads > 1024 || places < 1 || places > 256 || width * 8 != call->n * bits) return false;
    for (int i = 0; i < 4; ++i) {
        const at::Tensor& x = *t[i];
        const int64_t row = i % 2 == 0 ? width : 1;
        if (x.size(0) != pages || x.size(1) != heads || x.size(2) != places || (i % 2 == 0 && (x.size(3) != width || x.stride(3) != 1))) return false;
        if (x.stride(2) != row || (heads > 1 && x.stride(1) != places * row) || (pages > 1 && x.stride(0) < heads * places * row)) return false;
    }
    auto far = [&](const at::Tensor& x, int64_t row) { return pages > 1 ? x.stride(0) : heads * places * row; };
    bfq_kv_cache& c = call->cache;
    c.k_codes = static_cast<uint8_t*>(t[0]->data_ptr()), c.k_scales = static_cast<uint16_t*>(t[1]->data_ptr());
    c.v_codes = static_cast<uint8_t*>(t[2]->data_ptr()), c.v_scales = static_cast<uint16_t*>(t[3]->data_ptr());
    c.k_codes_page = far(*t[0], width), c.k_scales_page = far(*t[1], 1), c.v_codes_page = far(*t[2], width), c.v_scales_page = far(*t[3], 1);
    c.pages = pages, c.heads = static_cast<int>(heads), c.page_size = static_cast<int>(places), c.bits = static_cast<int>(bits);
    return true;
}
// rows [tokens][heads][n] of this type; -1: any number
bool head_rows(const CacheCall& call, PyObject* o, at::ScalarType type, int64_t tokens, int64_t heads, bfq_heads* out) {
    const at::Tensor* t = tensor(call, o, type, 3);
    if (t == nullptr || t->size(2) != call.n || t->stride(2) != 1 || t->size(0) < 1 || t->size(1) < 1 || t->size(1) > 1 << 20) return false;
    if ((tokens >= 0 && t->size(0) != tokens) || (heads >= 0 && t->size(1) != heads)) return false;
    out->data = t->data_ptr(), out->heads = static_cast<int>(t->size(1));
    out->token = t->size(0) > 1 ? t->stride(0) : t->size(1) * call.n, out->head = t->size(1) > 1 ? t->stride(1) : call.n;
    return true;
}
at::Tensor room(const CacheCall& call, at::IntArrayRef shape, at::ScalarType type) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, static_cast<c10::DeviceIndex>(call.device))));
}

// append_kv(cache arguments, k, v, slots, q, positions, rope, interleaved, q_norm, k_norm, eps) -> the queries or True, or a status, or None
PyObject* append_kv(PyObject*, PyObject* const* args, Py_ssize_t count) {
    try {
        CacheCall call;
        if (count != kCacheArgs + 10 || append_fn == nullptr || !cache_call(args, &call)) Py_RETURN_NONE;
        args += kCacheArgs;
        if (!THPVariable_CheckExact(args[0]) || !PyFloat_CheckExact(args[9])) Py_RETURN_NONE;
        const at::ScalarType type = THPVariable_Unpack(args[0]).scalar_type();
        if (type != at::kBFloat16 && type != at::kFloat) Py_RETURN_NONE;
        bfq_heads k, v, q{}, q_out{};
        if (!head_rows(call, args[0], type, -1, call.cache.heads, &k)) Py_RETURN_NONE;
        const int64_t tokens = THPVariable_Unpack(args[0]).size(0);
        const at::Tensor* slots = vector(call, args[2], at::kLong, tokens);
        if (slots == nullptr || !head_rows(call, args[1], type, tokens, call.cache.heads, &v)) Py_RETURN_NONE;
        const bool queries = args[3] != Py_None;
        if (queries && !head_rows(call, args[3], type, tokens, -1, &q)) Py_RETURN_NONE;
        bfq_kv_positions at{};
        if (args[4] != Py_None) {
            const at::Tensor *positions = vector(call, args[4], at::kInt, tokens), *table = tensor(call, args[5], at::kFloat, 2);
            if (positions == nullptr || table == nullptr || !table->is_contiguous() || table->size(0) < 1 || table->size(1) < 16 || table->size(1) > call.n ||
                table->size(1) % 16 != 0)
                Py_RETURN_NONE;
            at.positions = static_cast<const int32_t*>(positions->data_ptr()), at.table = static_cast<const float*>(table->data_ptr());
            at.rows = table->size(0), at.dims = static_cast<int>(table->size(1)), at.interleaved = args[6] == Py_True;
            if (args[6] != Py_True && args[6] != Py_False) Py_RETURN_NONE;
        } else if (args[5] != Py_None) {
            Py_RETURN_NONE;
        }
        for (int i = 0; i < 2; ++i) {
            if (args[7 + i] == Py_None) continue;
            const at::Tensor* w = vector(call, args[7 + i], at::kFloat, call.n);
            if (w == nullptr || (i == 0 && !queries)) Py_RETURN_NONE;
            (i == 0 ? at.q_norm : at.k_norm) = static_cast<const float*>(w->data_ptr());
        }
        at.eps = static_cast<float>(PyFloat_AS_DOUBLE(args[9]));
        at::Tensor out;
        if (queries) {
            out = room(call, {tokens, q.heads, call.n}, at::kBFloat16);
            q_out = bfq_heads{out.data_ptr(), q.heads * call.n, call.n, q.heads};
        }
        const int64_t* at_slots = static_cast<const int64_t*>(slots->data_ptr());
        const int status = launch(call.device, [&](void* stream) {
            return append_fn(call.plan, &call.cache, at_slots, tokens, type == at::kFloat ? BFQ_F32 : BFQ_BF16, &k, &v, queries ? &q : nullptr,
                             queries ? &q_out : nullptr, &at, stream);
        });
        if (status != BFQ_OK) return PyLong_FromLong(status);
        if (!queries) Py_RETURN_TRUE;
        return THPVariable_Wrap(std::move(out));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// read_kv(cache arguments, slots) -> (k, v) in bf16, or a status, or None
PyObject* read_kv(PyObject*, PyObject* const* args, Py_ssize_t count) {
    try {
        CacheCall call;
        if (count != kCacheArgs + 1 || read_fn == nullptr || !cache_call(args, &call)) Py_RETURN_NONE;
        const at::Tensor* slots = tensor(call, args[kCacheArgs], at::kLong, 1);
        if (slots == nullptr || !slots->is_contiguous() || slots->size(0) < 1) Py_RETURN_NONE;
        const int64_t tokens = slots->size(0);
        const at::Tensor both = room(call, {2, tokens, call.cache.heads, call.n}, at::kBFloat16);
        at::Tensor k = both.select(0, 0), v = both.select(0, 1);
        const int64_t* at_slots = static_cast<const int64_t*>(slots->data_ptr());
        void *to_k = k.data_ptr(), *to_v = v.data_ptr();
        const int status = launch(call.device, [&](void* stream) { return read_fn(call.plan, &call.cache, at_slots, tokens, BFQ_BF16, to_k, to_v, stream); });
        if (status != BFQ_OK) return PyLong_FromLong(status);
        PyObject* first = THPVariable_Wrap(std::move(k));
        PyObject* second = first != nullptr ? THPVariable_Wrap(std::move(v)) : nullptr;
        PyObject* pair = second != nullptr ? PyTuple_Pack(2, first, second) : nullptr;
        Py_XDECREF(first), Py_XDECREF(second);
        return pair;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// attend_kv(cache arguments, q, block_table, lengths, scale, q_starts, max_new, prefix, prefix_length) -> out, or a status, or None
PyObject* attend_kv(PyObject*, PyObject* const* args, Py_ssize_t count) {
    try {
        CacheCall call;
        if (count != kCacheArgs + 8 || attend_fn == nullptr || workspace_fn == nullptr || !cache_call(args, &call)) Py_RETURN_NONE;
        args += kCacheArgs;
        bfq_kv_queries a{};
        if (!head_rows(call, args[0], at::kBFloat16, -1, -1, &a.q)) Py_RETURN_NONE;
        a.tokens = THPVariable_Unpack(args[0]).size(0);
        if (a.q.heads % call.cache.heads != 0 || a.q.heads / call.cache.heads > 128) Py_RETURN_NONE;
        const at::Tensor *lengths = tensor(call, args[2], at::kInt, 1), *table = tensor(call, args[1], at::kInt, 2);
        if (lengths == nullptr || table == nullptr || !lengths->is_contiguous()) Py_RETURN_NONE;
        const int64_t batch = lengths->size(0), width = table->size(1);
        if (batch < 1 || batch > 1 << 20 || width > 1 << 30 || table->size(0) != batch || (width > 1 && table->stride(1) != 1) || (batch > 1 && table->stride(0) < width))
            Py_RETURN_NONE;
        a.batch = static_cast<int>(batch), a.lengths = static_cast<const int32_t*>(lengths->data_ptr());
        a.block_table = static_cast<const int32_t*>(table->data_ptr()), a.table_ld = batch > 1 ? table->stride(0) : width, a.table_width = static_cast<int>(width);
        a.max_new = 1;
        if (args[4] != Py_None) {
            const at::Tensor* starts = vector(call, args[4], at::kInt, batch + 1);
            const long most = PyLong_CheckExact(args[5]) ? PyLong_AsLong(args[5]) : -1;
            if (starts == nullptr || most < 1) {
                PyErr_Clear();
                Py_RETURN_NONE;
            }
            a.q_starts = static_cast<const int32_t*>(starts->data_ptr()), a.max_new = static_cast<int>(most < a.tokens ? most : a.tokens);
        } else if (a.tokens < batch) {
            Py_RETURN_NONE;
        }
        if (!PyLong_CheckExact(args[7])) Py_RETURN_NONE;
        a.prefix_length = PyLong_AsLongLong(args[7]);
        if (args[6] != Py_None) {
            const at::Tensor* prefix = tensor(call, args[6], at::kInt, 1);
            if (prefix == nullptr || !prefix->is_contiguous() || prefix->size(0) > 1 << 30 || a.prefix_length < 0 || a.prefix_length > prefix->size(0) * call.cache.page_size) {
                PyErr_Clear();
                Py_RETURN_NONE;
            }
            a.prefix = static_cast<const int32_t*>(prefix->data_ptr()), a.prefix_pages = static_cast<int>(prefix->size(0));
        } else if (a.prefix_length != 0) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        if (args[3] != Py_None && !PyFloat_CheckExact(args[3])) Py_RETURN_NONE;
        a.scale = static_cast<float>(args[3] != Py_None ? PyFloat_AS_DOUBLE(args[3]) : 1.0 / std::sqrt(static_cast<double>(call.n)));
        at::Tensor out = room(call, {a.tokens, a.q.heads, call.n}, at::kBFloat16);
        a.out = bfq_heads{out.data_ptr(), a.q.heads * call.n, call.n, a.q.heads};
        const size_t bytes = workspace_fn(call.plan, &call.cache, &a);
        const at::Tensor workspace = room(call, {static_cast<int64_t>(bytes)}, at::kByte);  // torch's blocks are 512 bytes apart
        void* at_workspace = workspace.data_ptr();
        const int status = launch(call.device, [&](void* stream) { return attend_fn(call.plan, &call.cache, &a, at_workspace, bytes, stream); });
        if (status == BFQ_ERR_ALIGN) Py_RETURN_NONE;  // or they are not: binding.py makes room for that
        if (status != BFQ_OK) return PyLong_FromLong(status);
        return THPVariable_Wrap(std::move(out));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// attach(path of libbfq.so): the library binding.py has loaded
PyObject* attach(PyObject*, PyObject* path) {
    const char* name = PyUnicode_AsUTF8(path);
    if (name == nullptr) return nullptr;
    void* lib = dlopen(name, RTLD_NOW | RTLD_LOCAL);
    constexpr int kNames = 7;
    void* found[kNames] = {};
    const char* names[kNames] = {"bfq_forward_quant", "bfq_forward", "bfq_inverse", "bfq_kv_append", "bfq_kv_read", "bfq_kv_attend_workspace", "bfq_kv_attend"};
    for (int i = 0; i < kNames; ++i)
        if (lib == nullptr || (found[i] = dlsym(lib, names[i])) == nullptr) {
            const char* why = dlerror();
            PyErr_SetString(PyExc_OSError, why != nullptr ? why : names[i]);
            return nullptr;
        }
    forward_quant_fn = reinterpret_cast<ForwardQuant>(found[0]);
    forward_fn = reinterpret_cast<Rows>(found[1]), inverse_fn = reinterpret_cast<Rows>(found[2]);
    append_fn = reinterpret_cast<decltype(append_fn)>(found[3]), read_fn = reinterpret_cast<decltype(read_fn)>(found[4]);
    workspace_fn = reinterpret_cast<decltype(workspace_fn)>(found[5]), attend_fn = reinterpret_cast<decltype(attend_fn)>(found[6]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"attach", attach, METH_O, nullptr},
    {"forward_quant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward_quant)), METH_FASTCALL, nullptr},
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL, nullptr},
    {"inverse", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(inverse)), METH_FASTCALL, nullptr},
    {"append_kv", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append_kv)), METH_FASTCALL, nullptr},
    {"read_kv", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(read_kv)), METH_FASTCALL, nullptr},
    {"attend_kv", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attend_kv)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_fast_calls() {
    PyObject* m = PyModule_Create(&module);
    // calls nothing of torch's: the binding asks for this before it uses the module with the torch that is there
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", BFQ_TORCH) < 0) Py_CLEAR(m);
    return m;
}
