// Argument marshalling of the serving calls (binding.py: baps_attention_window_fwd, baps_kv_*) against the interfaces of
// CPython and torch.
//
// What a call has to do on the host before its kernels start -- check the tensors' types, shapes, strides and device,
// allocate the outputs, pass pointers to the C ABI of include/baps.h, raise on a status -- and nothing else.  Kernels of the
// smallest calls take 3 to 10 us, so the host is what bounds them: one token appended took 12.7 us with these steps in Python,
// 8.8 with torch's Python methods called from C, 5.6 as here; a fork of beams 21.8, 18.1 and 11.5.  The library's functions
// come as addresses (bind), so that there is one loaded library, that of binding.load().
//
// The interpreter's lock is let go before anything is allocated or launched: torch's allocator may wait for other threads.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <limits>
#include <string>

#include "../../include/baps.h"

namespace {

PyObject* g_raise = nullptr;                       // binding._check(name, status)
PyObject* g_struct = nullptr;                      // "struct"
PyObject* g_members[4] = {};                       // "k", "v", "k_scale", "v_scale"
struct Library {
    decltype(&baps_attention_window_fwd) window;
    decltype(&baps_kv_append) append;
    decltype(&baps_kv_attention) attention;
    decltype(&baps_kv_attention_workspace) attention_workspace;
    decltype(&baps_kv_fork) fork;
    decltype(&baps_kv_compact) compact;
    decltype(&baps_kv_pages_workspace) pages_workspace;
};
Library lib;
constexpr int kFunctions = 7;
static_assert(sizeof(Library) == kFunctions * sizeof(void*), "one address each");

using at::Tensor;
using Sizes = at::IntArrayRef;
using at::kByte;
using at::kFloat;
using at::kInt;

struct Unlocked {                                  // the interpreter's lock let go for the life of this object
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// ---- checks -----------------------------------------------------------------------------------------------------------
struct Refused {                                   // becomes a Python error where the interpreter's lock is held
    PyObject* type;
    std::string text;
};
struct Raised {};                                  // a Python error is set already
[[noreturn]] void refuse(const char* name, const std::string& expected)
{
    throw Refused{PyExc_ValueError, std::string(name) + ": expected " + expected};
}
[[noreturn]] void out_of_range(const char* name) { throw Refused{PyExc_ValueError, std::string(name) + " is out of range"}; }

const Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(name) + ": expected a tensor"};
    return THPVariable_Unpack(o);
}
std::string text(Sizes s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}
// A contiguous tensor of this type, shape and device.
void* buffer(PyObject* o, const char* name, at::ScalarType type, Sizes shape, int device)
{
    const Tensor& t = tensor(o, name);
    if (t.scalar_type() != type || t.get_device() != device || t.sizes() != shape || !t.is_contiguous())
        refuse(name, std::string("a contiguous ") + c10::toString(type) + " tensor of shape " + text(shape) + " on cuda:" + std::to_string(device));
    return t.data_ptr();
}
int32_t* ints(PyObject* o, const char* name, Sizes shape, int device) { return static_cast<int32_t*>(buffer(o, name, kInt, shape, device)); }
void is_current(const char* name, int device)      // the library launches on the current device
{
    const int now = c10::cuda::current_device();
    if (device != now)
        throw Refused{PyExc_ValueError, std::string(name) + " is on cuda:" + std::to_string(device) + ", the current device is cuda:" + std::to_string(now)};
}
const Tensor& tensor16(PyObject* o, const char* name, int64_t dim, int& code)
{
    const Tensor& t = tensor(o, name);
    code = t.scalar_type() == at::kBFloat16 ? BAPS_DTYPE_BF16 : BAPS_DTYPE_F16;
    if ((t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kHalf) || !t.is_cuda()) refuse(name, "a bfloat16 or float16 CUDA tensor");
    if (t.dim() != dim) refuse(name, std::to_string(dim) + " dimensions");
    is_current(name, t.get_device());
    return t;
}
// A tensor of contiguous rows: its pointer, and the strides (elements) of the dimensions before the last; where a dimension
// has one element only, its stride does not matter and may be anything.
void* rows(const Tensor& t, const char* name, const Tensor& like, Sizes shape, int64_t* strides)
{
    if (t.scalar_type() != like.scalar_type() || t.get_device() != like.get_device() || t.sizes() != shape || t.strides().back() != 1)
        refuse(name, std::string("a ") + c10::toString(like.scalar_type()) + " tensor of shape " + text(shape) + " with contiguous rows on cuda:" +
                         std::to_string(like.get_device()));
    for (size_t i = 0; i + 1 < shape.size(); ++i) strides[i] = shape[i] > 1 ? t.strides()[i] : 8;
    return t.data_ptr();
}
int size_of(int64_t x)
{
    if (x > std::numeric_limits<int>::max()) out_of_range("a size");
    return static_cast<int>(x);
}
int whole(PyObject* o, const char* name, bool clamp = false)
{
    int over = 0;
    PyObject* n = PyNumber_Long(o);
    if (!n) throw Raised();
    const long long x = PyLong_AsLongLongAndOverflow(n, &over);
    Py_DECREF(n);
    if (over > 0 || x > std::numeric_limits<int>::max()) {
        if (!clamp) out_of_range(name);
        return std::numeric_limits<int>::max();
    }
    if (over < 0 || x < std::numeric_limits<int>::min()) out_of_range(name);
    return static_cast<int>(x);
}
int window_of(PyObject* o) { return whole(o, "window", true); }    // beyond an int it hides nothing
float real(PyObject* o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Raised();
    return static_cast<float>(x);
}
// The struct of a KvCache and its device, which has to be the current one.
struct Cache {
    baps_kv_cache c;
    int device, zero;                              // (no bytes that are nobody's: structs are compared as memory)
};
static_assert(sizeof(Cache) == sizeof(baps_kv_cache) + 2 * sizeof(int) && sizeof(baps_kv_cache) == 4 * sizeof(void*) + 4 * sizeof(int), "no padding");
// The struct of a KvCache's tensors.
Cache cache_of_tensors(PyObject* const* a)
{
    const Tensor& k = tensor(a[0], "k");
    const Sizes s = k.sizes();
    if (s.size() != 4 || !k.is_cuda()) refuse("k", "CUDA codes [n_pages,Hkv,page,D]");
    Cache cache;
    cache.device = k.get_device();
    cache.zero = 0;
    cache.c.k = static_cast<decltype(cache.c.k)>(buffer(a[0], "k", kByte, s, cache.device));
    cache.c.v = static_cast<decltype(cache.c.v)>(buffer(a[1], "v", kByte, s, cache.device));
    cache.c.k_scale = static_cast<float*>(buffer(a[2], "k_scale", kFloat, s.slice(0, 2), cache.device));
    cache.c.v_scale = static_cast<float*>(buffer(a[3], "v_scale", kFloat, s.slice(0, 2), cache.device));
    cache.c.n_pages = size_of(s[0]);
    cache.c.Hkv = size_of(s[1]);
    cache.c.page = size_of(s[2]);
    cache.c.D = size_of(s[3]);
    return cache;
}
Cache cache_of(PyObject* o)
{
    Cache cache;
    PyObject* bytes = PyObject_GetAttr(o, g_struct);
    if (!bytes) throw Raised();
    const bool ok = PyBytes_Check(bytes) && PyBytes_GET_SIZE(bytes) == static_cast<Py_ssize_t>(sizeof(Cache));
    if (ok) std::memcpy(&cache, PyBytes_AS_STRING(bytes), sizeof(Cache));
    Py_DECREF(bytes);
    if (!ok) refuse("cache", "a KvCache");
    // The struct's addresses are those of the tensors that the KvCache holds, or the memory may be another's by now.
    struct Held {
        PyObject* o[4] = {};
        ~Held() { for (PyObject* x : o) Py_XDECREF(x); }
    } held;
    for (int i = 0; i < 4; ++i)
        if (!(held.o[i] = PyObject_GetAttr(o, g_members[i]))) throw Raised();
    const Cache now = cache_of_tensors(held.o);
    if (std::memcmp(&now, &cache, sizeof(Cache)) != 0)
        throw Refused{PyExc_ValueError, "cache: its tensors were resized or given other storage since the KvCache was made; make a new one"};
    is_current("the cache", cache.device);
    return cache;
}
Sizes table_of(PyObject* o)
{
    const Sizes s = tensor(o, "table").sizes();
    if (s.size() != 2) refuse("table", "two dimensions");
    return s;
}

// ---- outputs ----------------------------------------------------------------------------------------------------------
Tensor empty(Sizes shape, at::ScalarType type, int device)
{
    return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, device), std::nullopt);
}
Tensor like(const Tensor& t) { return t.is_contiguous() ? empty(t.sizes(), t.scalar_type(), t.get_device()) : at::empty_like(t); }
int32_t* ints(const Tensor& t) { return static_cast<int32_t*>(t.data_ptr()); }
baps_stream stream_of(int device) { return c10::cuda::getCurrentCUDAStream(device).stream(); }

void check(const char* name, baps_status status)
{
    if (status == BAPS_OK) return;
    Py_XDECREF(PyObject_CallFunction(g_raise, "si", name, static_cast<int>(status)));
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
    throw Raised();
}
template <class... T>
PyObject* tuple(const T&... t)
{
    PyObject* o[] = {THPVariable_Wrap(t)...};
    PyObject* r = PyTuple_New(sizeof...(T));
    if (!r) throw Raised();
    for (size_t i = 0; i < sizeof...(T); ++i) PyTuple_SET_ITEM(r, i, o[i]);
    return r;
}

// ---- the calls --------------------------------------------------------------------------------------------------------
// (q, k, v, out | None, lse | None, lengths | None, window, sinks, scale) -> out
PyObject* call_window(PyObject* const* a)
{
    int code;
    int64_t st[12];
    const Tensor &q = tensor16(a[0], "q", 4, code), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const Sizes s = q.sizes(), ks = k.sizes();
    if (ks.size() != 4 || ks[0] != s[0] || ks[2] != s[2] || ks[3] != s[3]) refuse("k", "[B,Hkv,S,D] to match q [B,H,S,D]");
    const int device = q.get_device(), B = size_of(s[0]), H = size_of(s[1]), Hkv = size_of(ks[1]), S = size_of(s[2]), D = size_of(s[3]);
    const void *qp = rows(q, "q", q, s, st), *kp = rows(k, "k", q, ks, st + 3), *vp = rows(v, "v", q, ks, st + 6);
    void* op = a[3] == Py_None ? nullptr : rows(tensor(a[3], "out"), "out", q, s, st + 9);
    float* lse = a[4] == Py_None ? nullptr : static_cast<float*>(buffer(a[4], "lse", kFloat, s.slice(0, 3), device));
    const int32_t* lengths = a[5] == Py_None ? nullptr : ints(a[5], "lengths", s.slice(0, 1), device);
    const int win = window_of(a[6]), sinks = whole(a[7], "sinks");
    const float scale = real(a[8]);
    Tensor out;
    baps_status status;
    {
        Unlocked unlocked;
        if (a[3] == Py_None) op = rows(out = like(q), "out", q, s, st + 9);
        status = lib.window(qp, kp, vp, op, lse, lengths, st, B, H, Hkv, S, D, win, sinks, scale, code, stream_of(device));
    }
    check("baps_attention_window_fwd", status);
    return a[3] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[3]);
}

// (cache, k_new, v_new, table, lengths, starts, max_new | None)
PyObject* call_append(PyObject* const* a)
{
    int code;
    int64_t st[4];
    const Tensor &k = tensor16(a[1], "k_new", 3, code), &v = tensor(a[2], "v_new");
    const Cache cache = cache_of(a[0]);
    const Sizes ts = table_of(a[3]);
    const int64_t n = k.sizes()[0], shape[3] = {n, cache.c.Hkv, cache.c.D}, more[1] = {ts[0] + 1};
    const int B = size_of(ts[0]), width = size_of(ts[1]);
    const void *kp = rows(k, "k_new", k, shape, st), *vp = rows(v, "v_new", k, shape, st + 2);
    const int32_t *table = ints(a[3], "table", ts, cache.device), *lengths = ints(a[4], "lengths", ts.slice(0, 1), cache.device),
                  *starts = ints(a[5], "starts", more, cache.device);
    int64_t most = n;
    if (a[6] != Py_None) most = std::min<int64_t>(most, whole(a[6], "max_new", true));
    const int max_new = size_of(most);
    baps_status status;
    {
        Unlocked unlocked;
        status = lib.append(&cache.c, kp, vp, st, n, starts, lengths, table, width, B, max_new, code, stream_of(cache.device));
    }
    check("baps_kv_append", status);
    Py_RETURN_NONE;
}

// (q, cache, table, lengths, window, sinks, scale, out | None, want_lse, lse | None, workspace | None) -> out or (out, lse)
PyObject* call_attention(PyObject* const* a)
{
    int code;
    int64_t st[6];
    const Tensor& q = tensor16(a[0], "q", 4, code);
    const Cache cache = cache_of(a[1]);
    const Sizes s = q.sizes(), ts = table_of(a[2]);
    if (ts[0] != s[0] || s[3] != cache.c.D) throw Refused{PyExc_ValueError, "q does not match the cache, or table is not [B,width]"};
    const int device = cache.device, B = size_of(s[0]), H = size_of(s[1]), T = size_of(s[2]), width = size_of(ts[1]);
    const void* qp = rows(q, "q", q, s, st);
    const int32_t *table = ints(a[2], "table", ts, device), *lengths = ints(a[3], "lengths", ts.slice(0, 1), device);
    const int win = window_of(a[4]), sinks = whole(a[5], "sinks"), want_lse = PyObject_IsTrue(a[8]);
    const float scale = real(a[6]);
    if (want_lse < 0) throw Raised();
    void* op = a[7] == Py_None ? nullptr : rows(tensor(a[7], "out"), "out", q, s, st + 3);
    float* lp = a[9] == Py_None ? nullptr : static_cast<float*>(buffer(a[9], "lse", kFloat, s.slice(0, 3), device));
    void* wp = nullptr;
    size_t bytes = 0;
    if (a[10] != Py_None) {
        const Tensor& w = tensor(a[10], "workspace");
        if (w.scalar_type() != kByte || w.get_device() != device || !w.is_contiguous()) refuse("workspace", "a contiguous uint8 tensor on q's device");
        wp = w.data_ptr();
        bytes = w.numel();
    }
    Tensor out, lse, ws;
    baps_status status;
    {
        Unlocked unlocked;
        if (a[7] == Py_None) op = rows(out = like(q), "out", q, s, st + 3);
        if (want_lse && !lp) lp = static_cast<float*>((lse = empty(s.slice(0, 3), kFloat, device)).data_ptr());
        if (a[10] == Py_None && (bytes = lib.attention_workspace(B, H, cache.c.Hkv, T, cache.c.D, cache.c.page, width, win, sinks)) != 0)
            wp = (ws = empty({static_cast<int64_t>(bytes)}, kByte, device)).data_ptr();
        status = lib.attention(qp, op, lp, &cache.c, table, width, lengths, st, B, H, T, win, sinks, scale, code, wp, bytes, stream_of(device));
    }
    check("baps_kv_attention", status);
    PyObject* o = a[7] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[7]);
    if (!want_lse) return o;
    PyObject *l = a[9] == Py_None ? THPVariable_Wrap(lse) : Py_NewRef(a[9]), *pair = PyTuple_Pack(2, o, l);
    Py_DECREF(o);
    Py_DECREF(l);
    return pair;
}

// (cache, table, lengths, refs, parents, reserve, window, sinks) -> (new_table, new_lengths, new_refs)
PyObject* call_fork(PyObject* const* a)
{
    const Cache cache = cache_of(a[0]);
    const Sizes ts = table_of(a[1]), ps = tensor(a[4], "parents").sizes();
    if (ps.size() != 1) refuse("parents", "one dimension");
    const int device = cache.device, n_pages = cache.c.n_pages, n_rows = size_of(ts[0]), width = size_of(ts[1]), n_new = size_of(ps[0]);
    const int32_t *table = ints(a[1], "table", ts, device), *lengths = ints(a[2], "lengths", ts.slice(0, 1), device),
                  *refs = ints(a[3], "refs", {n_pages}, device), *parents = ints(a[4], "parents", ps, device);
    const int reserve = whole(a[5], "reserve"), win = window_of(a[6]), sinks = whole(a[7], "sinks");
    Tensor new_table, new_lengths, new_refs;
    baps_status status;
    {
        Unlocked unlocked;
        const size_t bytes = lib.pages_workspace(n_new, n_pages);
        new_table = empty({n_new, width}, kInt, device);
        new_lengths = empty({n_new}, kInt, device);
        new_refs = empty({n_pages}, kInt, device);
        const Tensor ws = empty({static_cast<int64_t>(bytes)}, kByte, device);
        status = lib.fork(&cache.c, table, lengths, n_rows, refs, parents, n_new, width, reserve, win, sinks, ints(new_table), ints(new_lengths),
                          ints(new_refs), ws.data_ptr(), bytes, stream_of(device));
    }
    check("baps_kv_fork", status);
    return tuple(new_table, new_lengths, new_refs);
}

// (cache, table, refs) -> (new_table, new_refs, page_map, n_live)
PyObject* call_compact(PyObject* const* a)
{
    const Cache cache = cache_of(a[0]);
    const Sizes ts = table_of(a[1]);
    const int device = cache.device, n_pages = cache.c.n_pages, n_rows = size_of(ts[0]), width = size_of(ts[1]);
    const int32_t *table = ints(a[1], "table", ts, device), *refs = ints(a[2], "refs", {n_pages}, device);
    Tensor new_table, new_refs, page_map, n_live;
    baps_status status;
    {
        Unlocked unlocked;
        const size_t bytes = lib.pages_workspace(0, n_pages);
        new_table = empty(ts, kInt, device);
        new_refs = empty({n_pages}, kInt, device);
        page_map = empty({n_pages}, kInt, device);
        n_live = empty({1}, kInt, device);
        const Tensor ws = empty({static_cast<int64_t>(bytes)}, kByte, device);
        status = lib.compact(&cache.c, table, n_rows, width, refs, ints(new_table), ints(new_refs), ints(page_map), ints(n_live), ws.data_ptr(),
                             bytes, stream_of(device));
    }
    check("baps_kv_compact", status);
    return tuple(new_table, new_refs, page_map, n_live);
}

// (KvCache, k, v, k_scale, v_scale): its members, past its own refusal of assignments
PyObject* fill_cache(PyObject* const* a)
{
    const Cache cache = cache_of_tensors(a + 1);
    PyObject* bytes = PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&cache), sizeof(cache));
    if (!bytes) throw Raised();
    int failed = PyObject_GenericSetAttr(a[0], g_struct, bytes);
    Py_DECREF(bytes);
    for (int i = 0; !failed && i < 4; ++i) failed = PyObject_GenericSetAttr(a[0], g_members[i], a[1 + i]);
    if (failed) throw Raised();
    Py_RETURN_NONE;
}

// (binding._check, addresses of the library's functions in Library's order)
PyObject* bind(PyObject* const* a)
{
    void* p[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        PyObject* x = PySequence_GetItem(a[1], i);
        if (!x) throw Raised();
        p[i] = PyLong_AsVoidPtr(x);
        Py_DECREF(x);
        if (PyErr_Occurred()) throw Raised();
        if (!p[i]) refuse("bind", "an address of each function");
    }
    std::memcpy(&lib, p, sizeof(lib));
    Py_XSETREF(g_raise, Py_NewRef(a[0]));
    Py_RETURN_NONE;
}

// No C++ exception passes the interpreter: they become Python's.
template <PyObject* (*kCall)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    try {
        if (n != kArgs) throw Refused{PyExc_TypeError, "expected " + std::to_string(kArgs) + " arguments, got " + std::to_string(n)};
        return kCall(a);
    } catch (const Refused& e) {
        PyErr_SetString(e.type, e.text.c_str());
        return nullptr;
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
template <PyObject* (*kCall)(PyObject* const*), int kArgs>
constexpr PyMethodDef method(const char* name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<kCall, kArgs>)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<bind, 2>("bind"),           method<fill_cache, 5>("fill_cache"), method<call_window, 9>("window"),
                           method<call_append, 7>("append"),       method<call_attention, 11>("attention"),      method<call_fork, 8>("fork"),
                           method<call_compact, 3>("compact"),     {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", "Argument marshalling of the serving calls.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving()
{
    const char* const members[] = {"k", "v", "k_scale", "v_scale"};
    for (int i = 0; i < 4; ++i)
        if (!(g_members[i] = PyUnicode_InternFromString(members[i]))) return nullptr;
    g_struct = PyUnicode_InternFromString("struct");
    return g_struct ? PyModule_Create(&g_module) : nullptr;
}
