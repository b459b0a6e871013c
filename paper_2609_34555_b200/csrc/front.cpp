// Checks of the tensors that the calls on the 4-bit path are given, and the calls themselves, for binding.py.
//
// The calls are small: a decode step's rotation or attention of one sequence keeps the GPU for a few microseconds, and the
// same checks written in Python took longer than the launch.  This module does what binding._dev and the methods beside
// it do for the other calls -- type, device, contiguity, shape -- and hands raw pointers to the C ABI; every computation
// stays behind include/pulseinfer.h.  It does not link the CUDA library: binding.py loads that and passes the addresses.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "pulseinfer.h"

namespace {

struct Calls {
    decltype(&pi_assign_pages) assign_pages;
    decltype(&pi_qk_norm_rope) qk_norm_rope;
    decltype(&pi_kv4_store) kv4_store;
    decltype(&pi_kv4_load) kv4_load;
    decltype(&pi_append_kv4) append_kv4;
    decltype(&pi_recall_kv4) recall_kv4;
    decltype(&pi_sparse_decode_attn_kv4) sparse_decode_attn_kv4;
} g_calls;

// What a context's calls look at: its address, device and shape.
struct Shape {
    pi_ctx* ctx;
    int64_t device, hq, hkv, d, b, slots, blocks, budget, block4;
};

struct Raised {};                                  // a Python error is set

[[noreturn]] void refuse(PyObject* kind, const std::string& text) {
    PyErr_SetString(kind, text.c_str());
    throw Raised();
}

std::string text_of(c10::IntArrayRef v) {
    std::string s = "(";
    for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + (v[i] < 0 ? std::string("...") : std::to_string(v[i]));
    return s + ")";
}

const char* name_of(at::ScalarType t) {
    switch (t) {
        case at::kInt: return "torch.int32";
        case at::kLong: return "torch.int64";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kFloat: return "torch.float32";
        default: return "torch.uint8";
    }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + ": expected a tensor");
    return THPVariable_Unpack(o);
}

void same_device(const Shape& s, const at::Tensor& t, const char* name) {
    if (t.get_device() != s.device)
        refuse(PyExc_ValueError, std::string(name) + ": on " + t.device().str() + ", the context is on cuda:" + std::to_string(s.device));
}

// A contiguous tensor of one type on the context's device; a negative size in `shape` stands for any.
const at::Tensor& on(const Shape& s, PyObject* o, at::ScalarType type, const char* name, std::initializer_list<int64_t> shape = {}) {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous())
        refuse(PyExc_TypeError, std::string(name) + ": expected a contiguous CUDA tensor of " + name_of(type));
    same_device(s, t, name);
    if (shape.size()) {
        const auto have = t.sizes();
        bool fits = have.size() == shape.size();
        size_t i = 0;
        for (int64_t want : shape) { fits = fits && (want < 0 || have[i] == want); ++i; }
        if (!fits) refuse(PyExc_ValueError, std::string(name) + ": expected shape " + text_of(c10::IntArrayRef(shape.begin(), shape.size())) + ", got " + text_of(have));
    }
    return t;
}

template <typename T>
T* ptr(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

template <typename T>
T* maybe(const Shape& s, PyObject* o, at::ScalarType type, const char* name, std::initializer_list<int64_t> shape) {
    return o == Py_None ? nullptr : ptr<T>(on(s, o, type, name, shape));
}

// At least so many values.
template <typename T>
T* table(const Shape& s, PyObject* o, at::ScalarType type, const char* name, int64_t values) {
    const at::Tensor& t = on(s, o, type, name);
    if (t.numel() < values) refuse(PyExc_ValueError, std::string(name) + ": expected at least " + std::to_string(values) + " values, got " + std::to_string(t.numel()));
    return ptr<T>(t);
}

struct NotPinned {};                               // PI_ERR_NOT_PINNED, as the C call would say

// A contiguous uint8 tensor [..., block4] of 4-bit blocks, on the device or (host) in pinned memory.
const at::Tensor& blocks4(const Shape& s, PyObject* o, const char* name, bool host, int64_t* blocks) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != at::kByte || !t.is_contiguous() || t.dim() < 2 || t.size(-1) != s.block4)
        refuse(PyExc_TypeError, std::string(name) + ": expected a contiguous uint8 tensor [..., " + std::to_string(s.block4) + "] of 4-bit blocks");
    if (t.is_cuda()) same_device(s, t, name);
    else if (!host) refuse(PyExc_TypeError, std::string(name) + ": expected a CUDA tensor");
    else if (!t.is_pinned()) throw NotPinned();
    *blocks = t.numel() / s.block4;
    return t;
}

void* pool4(const Shape& s, PyObject* o, int64_t batch) {
    int64_t n = 0;
    const at::Tensor& t = blocks4(s, o, "pool4", false, &n);
    if (n < batch * s.slots) refuse(PyExc_ValueError, "pool4: expected [batch][" + std::to_string(s.slots) + "] blocks");
    return t.data_ptr();
}

// A block-major or paged 4-bit store.
struct Store4 {
    void* base;
    int64_t stride, page_stride;
    const int32_t* pages;
    int32_t n_pages;
};
Store4 store4(const Shape& s, PyObject* store, PyObject* page_table, int64_t batch) {
    int64_t n = 0;
    Store4 r = {blocks4(s, store, "host_kv4", true, &n).data_ptr(), s.blocks * s.block4, 0, nullptr, 0};
    if (page_table != Py_None) {
        const at::Tensor& t = on(s, page_table, at::kInt, "page_table");
        if (t.dim() != 2 || t.size(0) < batch) refuse(PyExc_ValueError, "page_table: expected [batch][blocks]");
        r.stride = 0;
        r.page_stride = t.size(1);
        r.pages = ptr<int32_t>(t);
        r.n_pages = static_cast<int32_t>(n < INT32_MAX ? n : INT32_MAX);
    } else if (n < batch * s.blocks) {
        refuse(PyExc_ValueError, "host_kv4: expected [batch][" + std::to_string(s.blocks) + "] blocks");
    }
    return r;
}

int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}
int layer_of(PyObject* o) {
    const int64_t v = whole(o);
    return v < INT32_MIN || v > INT32_MAX ? -1 : static_cast<int>(v);       // (-1 is refused by the call)
}
int batch_of(const at::Tensor& t, const char* name) {
    if (t.dim() < 1) refuse(PyExc_ValueError, std::string(name) + ": expected at least one axis");
    return t.size(0) > INT32_MAX ? -1 : static_cast<int>(t.size(0));
}
void* stream_of(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}

using Args = PyObject* const*;

// The call itself, with the interpreter free for other threads (a launch may wait for room in the queue).  Arguments are
// values: nothing of Python is touched inside.
template <typename F, typename... A>
int call(F function, A... arguments) {
    PyThreadState* state = PyEval_SaveThread();
    const int rc = function(arguments...);
    PyEval_RestoreThread(state);
    return rc;
}

int assign_pages(const Shape& s, Args a) {
    const at::Tensor& old_len = on(s, a[0], at::kInt, "old_len", {-1});
    const int batch = batch_of(old_len, "old_len");
    const at::Tensor& new_len = on(s, a[1], at::kInt, "new_len", {batch});
    const at::Tensor& pages = on(s, a[2], at::kInt, "page_table", {-1, -1});
    if (pages.size(0) < batch) refuse(PyExc_ValueError, "page_table: expected [batch][blocks]");
    const at::Tensor& ring = on(s, a[3], at::kInt, "free_pages");
    const at::Tensor& state = on(s, a[4], at::kLong, "free_state", {4});
    int32_t* starts = maybe<int32_t>(s, a[5], at::kInt, "token_start", {batch + 1});
    const int64_t n = a[6] != Py_None ? on(s, a[6], at::kLong, "slot_map", {-1}).size(0) : a[7] != Py_None ? on(s, a[7], at::kInt, "positions", {-1}).size(0) : 0;
    int64_t* slots = maybe<int64_t>(s, a[6], at::kLong, "slot_map", {n});
    int32_t* positions = maybe<int32_t>(s, a[7], at::kInt, "positions", {n});
    // (a map of no entries has no address, which would say that none is wanted; with one, new tokens are refused for it)
    alignas(16) static int64_t none[2];
    if (a[6] != Py_None && n == 0) slots = none;
    if (a[7] != Py_None && n == 0) positions = reinterpret_cast<int32_t*>(none);
    return call(g_calls.assign_pages, s.ctx, batch, ptr<int32_t>(old_len), ptr<int32_t>(new_len), ptr<int32_t>(pages), pages.size(1), ptr<int32_t>(ring),
                                static_cast<int32_t>(ring.numel() < INT32_MAX ? ring.numel() : INT32_MAX), ptr<int64_t>(state), starts, n, slots, positions, stream_of(a[8]));
}

int qk_norm_rope(const Shape& s, Args a) {
    const float eps = static_cast<float>(number(a[8]));
    const int interleaved = truth(a[9]) ? 1 : 0;
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
    const int64_t T = q.dim() ? q.size(0) : 0;
    const auto type = q.scalar_type();
    const int dtype = type == at::kBFloat16 ? PI_DTYPE_BF16 : type == at::kHalf ? PI_DTYPE_FP16 : type == at::kFloat ? PI_DTYPE_FP32 : -1;
    auto rows = [&](const at::Tensor& t, int64_t heads, const char* name) {
        if (dtype < 0 || t.scalar_type() != type || !t.is_cuda()) refuse(PyExc_TypeError, std::string(name) + ": expected a CUDA tensor of bfloat16, float16 or float32, both of one type");
        same_device(s, t, name);
        if (t.dim() != 3 || t.size(0) != T || t.size(1) != heads || t.size(2) != s.d) {
            const int64_t want[3] = {T, heads, s.d};
            refuse(PyExc_ValueError, std::string(name) + ": expected shape " + text_of(want) + ", got " + text_of(t.sizes()));
        }
        if (T && (t.stride(2) != 1 || (heads > 1 && t.stride(1) != s.d))) refuse(PyExc_ValueError, std::string(name) + ": the rows of a token must be contiguous");
        return T > 1 ? t.stride(0) : heads * s.d;      // (of a single token the stride means nothing, and torch may report any)
    };
    const int64_t q_stride = rows(q, s.hq, "q"), k_stride = rows(k, s.hkv, "k");
    const at::Tensor& positions = on(s, a[2], at::kInt, "positions", {T});
    const at::Tensor* freq = a[3] == Py_None ? nullptr : &on(s, a[3], at::kFloat, "inv_freq");
    const int64_t rot = freq ? 2 * freq->numel() : 0;
    return call(g_calls.qk_norm_rope, s.ctx, T, dtype, q.data_ptr(), q_stride, k.data_ptr(), k_stride, ptr<int32_t>(positions),
                                maybe<float>(s, a[6], at::kFloat, "q_weight", {s.d}), maybe<float>(s, a[7], at::kFloat, "k_weight", {s.d}),
                                eps, freq ? ptr<float>(*freq) : nullptr, rot > 256 ? 256 : static_cast<int>(rot), interleaved,
                                on(s, a[4], at::kBFloat16, "q_out", {T, s.hq, s.d}).data_ptr(), on(s, a[5], at::kBFloat16, "k_out", {T, s.hkv, s.d}).data_ptr(), stream_of(a[10]));
}

int kv4_store(const Shape& s, Args a) {
    const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
    const int64_t dims = k.dim();
    if (dims != 3 && dims != 4) refuse(PyExc_ValueError, "k: expected [tokens][heads][channels] or [runs][tokens][heads][channels]");
    int64_t place[2][3];                           // strides of token, head and run
    int i = 0;
    for (const at::Tensor* t : {&k, &v}) {
        const char* name = i ? "v" : "k";
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16) refuse(PyExc_TypeError, std::string(name) + ": expected a CUDA tensor of torch.bfloat16");
        same_device(s, *t, name);
        if (t->sizes() != k.sizes() || t->size(-2) != s.hkv || t->size(-1) != s.d)
            refuse(PyExc_ValueError, std::string(name) + ": expected [..., " + std::to_string(s.hkv) + ", " + std::to_string(s.d) + "], k and v alike, got " + text_of(t->sizes()));
        if (t->numel() && t->stride(-1) != 1) refuse(PyExc_ValueError, std::string(name) + ": rows must be contiguous");
        // (of an axis of one entry the stride means nothing, and torch may report any)
        auto stride = [&](int64_t axis) { return t->size(axis) <= 1 ? int64_t(0) : t->stride(axis); };
        place[i][0] = stride(dims - 3); place[i][1] = stride(dims - 2); place[i][2] = dims == 4 ? stride(0) : 0;
        ++i;
    }
    const int64_t n = dims == 4 ? k.size(0) * k.size(1) : k.size(0);
    const int64_t* slots = maybe<int64_t>(s, a[3], at::kLong, "slot_map", {n});
    int64_t blocks = 0;
    void* store = blocks4(s, a[2], "store", true, &blocks).data_ptr();
    return call(g_calls.kv4_store, s.ctx, n, k.data_ptr(), place[0][0], place[0][1], place[0][2], v.data_ptr(), place[1][0], place[1][1], place[1][2],
                             dims == 4 ? k.size(1) : 0, slots, store, blocks, stream_of(a[4]));
}

int kv4_load(const Shape& s, Args a) {
    const at::Tensor* list = a[2] == Py_None ? nullptr : &on(s, a[2], at::kInt, "blocks");
    const at::Tensor& out = on(s, a[1], at::kBFloat16, "out", {list ? list->numel() : -1, s.hkv, 2, s.b, s.d});
    int64_t blocks = 0;
    void* store = blocks4(s, a[0], "store", true, &blocks).data_ptr();
    return call(g_calls.kv4_load, s.ctx, out.size(0), store, blocks, list ? ptr<int32_t>(*list) : nullptr, out.data_ptr(), stream_of(a[3]));
}

int append_kv4(const Shape& s, Args a) {
    const at::Tensor& ctx_len = on(s, a[4], at::kInt, "ctx_len", {-1});
    const int batch = batch_of(ctx_len, "ctx_len");
    uint32_t step = 0;
    const uint32_t* step_dev = nullptr;
    if (THPVariable_Check(a[1])) step_dev = table<uint32_t>(s, a[1], at::kInt, "step", 1);
    else {
        const int64_t v = whole(a[1]);
        step = v < 1 || v > UINT32_MAX ? 0u : static_cast<uint32_t>(v);     // (0 is refused by the call)
    }
    const at::Tensor &k = on(s, a[2], at::kBFloat16, "k_new", {batch, s.hkv, s.d}), &v = on(s, a[3], at::kBFloat16, "v_new", {batch, s.hkv, s.d});
    const Store4 st = store4(s, a[5], a[11], batch);
    return call(g_calls.append_kv4, s.ctx, layer_of(a[0]), batch, step, step_dev, k.data_ptr(), v.data_ptr(), ptr<int32_t>(ctx_len), st.base, st.stride, st.pages, st.page_stride,
                              st.n_pages, pool4(s, a[6], batch), table<int32_t>(s, a[7], at::kInt, "block_table", batch * s.blocks),
                              table<int32_t>(s, a[8], at::kInt, "slot_block", batch * s.slots), table<uint32_t>(s, a[9], at::kInt, "slot_stamp", batch * s.slots),
                              table<void>(s, a[10], at::kBFloat16, "digest", batch * s.blocks * 2 * s.d), stream_of(a[12]));
}

int recall_kv4(const Shape& s, Args a) {
    const at::Tensor& count = on(s, a[4], at::kInt, "recall_count", {-1});
    const int batch = batch_of(count, "recall_count");
    const at::Tensor& lists = on(s, a[3], at::kInt, "recall_list", {batch, -1, 4});
    const Store4 st = store4(s, a[1], a[5], batch);
    return call(g_calls.recall_kv4, s.ctx, layer_of(a[0]), batch, st.base, st.stride, st.pages, st.page_stride, st.n_pages, pool4(s, a[2], batch),
                              reinterpret_cast<const pi_extent*>(lists.data_ptr()), static_cast<int32_t>(lists.size(1) < INT32_MAX ? lists.size(1) : 0), ptr<int32_t>(count), stream_of(a[6]));
}

int sparse_decode_attn_kv4(const Shape& s, Args a) {
    const at::Tensor& q = on(s, a[1], at::kBFloat16, "q", {-1, s.hq, s.d});
    const int batch = batch_of(q, "q");
    void* pool = pool4(s, a[2], batch);
    return call(g_calls.sparse_decode_attn_kv4, s.ctx, layer_of(a[0]), batch, q.data_ptr(), pool, ptr<int32_t>(on(s, a[3], at::kInt, "sel_slots", {batch, s.budget})),
                                          ptr<int32_t>(on(s, a[4], at::kInt, "sel_blocks", {batch, s.budget})), ptr<int32_t>(on(s, a[5], at::kInt, "sel_count", {batch})),
                                          ptr<int32_t>(on(s, a[6], at::kInt, "ctx_len", {batch})), on(s, a[7], at::kBFloat16, "out", {batch, s.hq, s.d}).data_ptr(),
                                          maybe<float>(s, a[8], at::kFloat, "lse", {batch, s.hq}), stream_of(a[9]));
}

// module function: (shape, arguments...) -> the C call's return code
template <int (*CALL)(const Shape&, Args), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        if (n != N + 1) refuse(PyExc_TypeError, "wrong number of arguments");
        const Shape* s = static_cast<const Shape*>(PyCapsule_GetPointer(args[0], "pulseinfer.shape"));
        if (!s) throw Raised();
        return PyLong_FromLong(CALL(*s, args + 1));
    } catch (const Raised&) {
        return nullptr;
    } catch (const NotPinned&) {
        return PyLong_FromLong(PI_ERR_NOT_PINNED);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// shape(context address, device, Hq, Hkv, D, B, C, NB, K, bytes of a 4-bit block)
PyObject* make_shape(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        if (n != 10) refuse(PyExc_TypeError, "shape: wrong number of arguments");
        int64_t v[10];
        for (int i = 0; i < 10; ++i) v[i] = whole(args[i]);
        Shape* s = new Shape{reinterpret_cast<pi_ctx*>(v[0]), v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9]};
        return PyCapsule_New(s, "pulseinfer.shape", [](PyObject* c) { delete static_cast<Shape*>(PyCapsule_GetPointer(c, "pulseinfer.shape")); });
    } catch (const Raised&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// connect(addresses of the seven calls, in the order of Calls)
PyObject* connect(PyObject*, PyObject* const* args, Py_ssize_t n) {
    static_assert(sizeof(Calls) == 7 * sizeof(void*), "seven calls");
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "connect: expected seven addresses"); return nullptr; }
    void* p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "connect: a null address"); return nullptr; }
    }
    g_calls.assign_pages = reinterpret_cast<decltype(g_calls.assign_pages)>(p[0]);
    g_calls.qk_norm_rope = reinterpret_cast<decltype(g_calls.qk_norm_rope)>(p[1]);
    g_calls.kv4_store = reinterpret_cast<decltype(g_calls.kv4_store)>(p[2]);
    g_calls.kv4_load = reinterpret_cast<decltype(g_calls.kv4_load)>(p[3]);
    g_calls.append_kv4 = reinterpret_cast<decltype(g_calls.append_kv4)>(p[4]);
    g_calls.recall_kv4 = reinterpret_cast<decltype(g_calls.recall_kv4)>(p[5]);
    g_calls.sparse_decode_attn_kv4 = reinterpret_cast<decltype(g_calls.sparse_decode_attn_kv4)>(p[6]);
    Py_RETURN_NONE;
}

#define METHOD(name, function) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(function)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD("connect", connect),
    METHOD("shape", make_shape),
    METHOD("assign_pages", (&entry<assign_pages, 9>)),
    METHOD("qk_norm_rope", (&entry<qk_norm_rope, 11>)),
    METHOD("kv4_store", (&entry<kv4_store, 5>)),
    METHOD("kv4_load", (&entry<kv4_load, 4>)),
    METHOD("append_kv4", (&entry<append_kv4, 13>)),
    METHOD("recall_kv4", (&entry<recall_kv4, 7>)),
    METHOD("sparse_decode_attn_kv4", (&entry<sparse_decode_attn_kv4, 10>)),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_front", "Tensor checks and calls of the 4-bit path.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__front() { return PyModule_Create(&module); }
