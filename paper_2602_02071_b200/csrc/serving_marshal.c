/* Argument marshalling of the serving calls (binding.py: baps_attention_window_fwd, baps_kv_*), against the CPython API.
 *
 * What binding.py does for every call -- check the tensors' types, shapes, strides and device, allocate outputs through torch,
 * pass pointers to the C ABI of include/baps.h, raise on a status -- and nothing else.  In Python that took 8 to 15 us of calls
 * whose kernels take 3 to 10 (attribute by attribute 50 ns, but a hundred times that in interpreted checks).  No torch header is
 * used: tensors are asked through their Python methods.  The library's functions come as addresses (bind), so that
 * there is one loaded library, that of binding.load().
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>
#include "../../include/baps.h"

/* interned names, torch's objects, the library's functions; set once by bind() */
static PyObject *s_dtype, *s_shape, *s_stride, *s_get_device, *s_data_ptr, *s_new_empty, *s_struct, *s_k, *s_k_scale;
static PyObject *t_bf16, *t_f16, *t_f32, *t_i32, *t_u8, *t_empty_like, *t_device, *t_stream, *t_raise;
static struct {
    baps_status (*window)(const void *, const void *, const void *, void *, float *, const int32_t *, const int64_t *, int, int, int, int,
                          int, int, int, float, int, baps_stream);
    baps_status (*append)(const baps_kv_cache *, const void *, const void *, const int64_t *, int64_t, const int32_t *, const int32_t *,
                          const int32_t *, int, int, int, int, baps_stream);
    baps_status (*attention)(const void *, void *, float *, const baps_kv_cache *, const int32_t *, int, const int32_t *, const int64_t *,
                             int, int, int, int, int, float, int, void *, size_t, baps_stream);
    size_t (*attention_workspace)(int, int, int, int, int, int, int, int, int);
    baps_status (*fork)(const baps_kv_cache *, const int32_t *, const int32_t *, int, const int32_t *, const int32_t *, int, int, int, int,
                        int, int32_t *, int32_t *, int32_t *, void *, size_t, baps_stream);
    baps_status (*compact)(const baps_kv_cache *, const int32_t *, int, int, const int32_t *, int32_t *, int32_t *, int32_t *, int32_t *,
                           void *, size_t, baps_stream);
    size_t (*pages_workspace)(int, int);
} lib;

/* ---- tensors -------------------------------------------------------------------------------------- */
typedef struct {
    void *ptr;
    PyObject *dtype;                  /* a reference of torch's own, which outlives the call */
    int64_t dim, shape[4], stride[4], device;
} tensor;

static int long_of(PyObject *o, int64_t *x)      /* steals o */
{
    if (!o) return -1;
    *x = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return *x == -1 && PyErr_Occurred() ? -1 : 0;
}
static int tuple_of(PyObject *o, const char *name, int64_t *dim, int64_t *x)      /* steals o */
{
    if (!o) return -1;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) > 4) {
        Py_DECREF(o);
        PyErr_Format(PyExc_ValueError, "%s: expected a tensor of at most four dimensions", name);
        return -1;
    }
    *dim = PyTuple_GET_SIZE(o);
    for (Py_ssize_t i = 0; i < *dim; ++i) {
        x[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
        if (x[i] == -1 && PyErr_Occurred()) { Py_DECREF(o); return -1; }
    }
    Py_DECREF(o);
    return 0;
}
static int get_tensor(PyObject *o, const char *name, tensor *t)
{
    int64_t p, dim;
    t->dtype = PyObject_GetAttr(o, s_dtype);
    if (!t->dtype) return -1;
    Py_DECREF(t->dtype);
    if (long_of(PyObject_CallMethodNoArgs(o, s_get_device), &t->device) || tuple_of(PyObject_GetAttr(o, s_shape), name, &t->dim, t->shape) ||
        tuple_of(PyObject_CallMethodNoArgs(o, s_stride), name, &dim, t->stride) || long_of(PyObject_CallMethodNoArgs(o, s_data_ptr), &p))
        return -1;
    t->ptr = (void *)(intptr_t)p;
    return 0;
}
static int contiguous(const tensor *t)
{
    int64_t want = 1;
    for (int64_t i = t->dim - 1; i >= 0; --i) {
        if (t->shape[i] == 0) return 1;
        if (t->shape[i] != 1 && t->stride[i] != want) return 0;
        want *= t->shape[i];
    }
    return 1;
}
static int has_shape(const tensor *t, int64_t dim, const int64_t *shape)
{
    if (t->dim != dim) return 0;
    for (int64_t i = 0; i < dim; ++i)
        if (t->shape[i] != shape[i]) return 0;
    return 1;
}
static int refuse(const char *name, const char *why)
{
    PyErr_Format(PyExc_ValueError, "%s: expected %s", name, why);
    return -1;
}
/* A contiguous tensor of this type, device and shape. */
static int get_buffer(PyObject *o, const char *name, PyObject *dtype, const char *type, int64_t device, int64_t dim, const int64_t *shape,
                      tensor *t)
{
    if (get_tensor(o, name, t)) return -1;
    if (t->dtype != dtype || t->device != device || !has_shape(t, dim, shape) || !contiguous(t)) {
        PyErr_Format(PyExc_ValueError, "%s: expected a contiguous %s tensor on cuda:%lld that matches the other arguments", name, type,
                     (long long)device);
        return -1;
    }
    return 0;
}
/* A 16-bit tensor on the current device; its code in *code. */
static int get_16(PyObject *o, const char *name, int64_t dim, tensor *t, int *code)
{
    int64_t now;
    if (get_tensor(o, name, t)) return -1;
    *code = t->dtype == t_bf16 ? BAPS_DTYPE_BF16 : BAPS_DTYPE_F16;
    if ((t->dtype != t_bf16 && t->dtype != t_f16) || t->device < 0) return refuse(name, "a bfloat16 or float16 CUDA tensor");
    if (t->dim != dim) { PyErr_Format(PyExc_ValueError, "%s: expected %d dimensions", name, (int)dim); return -1; }
    if (long_of(PyObject_CallNoArgs(t_device), &now)) return -1;
    if (t->device != now) {
        PyErr_Format(PyExc_ValueError, "%s is on cuda:%lld, the current device is cuda:%lld", name, (long long)t->device, (long long)now);
        return -1;
    }
    return 0;
}
/* Strides (elements) of all dimensions but the last; where a dimension has one element, its stride does not matter. */
static int rows_of(const tensor *t, const char *name, const tensor *like, int64_t dim, const int64_t *shape, int64_t *out)
{
    if (t->dtype != like->dtype || t->device != like->device || !has_shape(t, dim, shape) || t->stride[dim - 1] != 1)
        return refuse(name, "a tensor of contiguous rows, of the type, device and shape that match the other arguments");
    for (int64_t i = 0; i + 1 < dim; ++i) out[i] = t->shape[i] > 1 ? t->stride[i] : 8;
    return 0;
}
static int fits_int(const char *name, int64_t x)
{
    if (x >= INT32_MIN && x <= INT32_MAX) return 0;
    PyErr_Format(PyExc_ValueError, "%s is out of range: %lld", name, (long long)x);
    return -1;
}
/* A whole number that fits an int; a window may be larger, and then hides nothing. */
static int int_arg(PyObject *o, const char *name, int is_window, int *out)
{
    int over;
    PyObject *n = PyNumber_Long(o);
    if (!n) return -1;
    const int64_t x = PyLong_AsLongLongAndOverflow(n, &over);
    Py_DECREF(n);
    if (is_window && (over > 0 || x > INT32_MAX)) { *out = INT32_MAX; return 0; }
    if (over) { PyErr_Format(PyExc_ValueError, "%s is out of range", name); return -1; }
    if (x == -1 && PyErr_Occurred()) return -1;
    if (fits_int(name, x)) return -1;
    *out = (int)x;
    return 0;
}
static int stream_of(int64_t device, baps_stream *s)
{
    int64_t x;
    PyObject *d = PyLong_FromLongLong(device);
    if (!d) return -1;
    PyObject *r = PyObject_CallOneArg(t_stream, d);
    Py_DECREF(d);
    if (long_of(r, &x)) return -1;
    *s = (baps_stream)(intptr_t)x;
    return 0;
}
/* like.new_empty(shape), or torch.empty_like(like) where dim < 0, and its pointer */
static PyObject *new_tensor(PyObject *like, int64_t dim, const int64_t *shape, void **ptr)
{
    int64_t p;
    PyObject *o;
    if (dim < 0) {
        o = PyObject_CallOneArg(t_empty_like, like);
    } else {
        PyObject *size = PyTuple_New(dim);
        if (!size) return NULL;
        for (int64_t i = 0; i < dim; ++i) {
            PyObject *n = PyLong_FromLongLong(shape[i]);
            if (!n) { Py_DECREF(size); return NULL; }
            PyTuple_SET_ITEM(size, i, n);
        }
        o = PyObject_CallMethodOneArg(like, s_new_empty, size);
        Py_DECREF(size);
    }
    if (!o) return NULL;
    if (long_of(PyObject_CallMethodNoArgs(o, s_data_ptr), &p)) { Py_DECREF(o); return NULL; }
    *ptr = (void *)(intptr_t)p;
    return o;
}
/* binding._check(name, status): raises */
static int check(const char *name, baps_status st)
{
    if (st == BAPS_OK) return 0;
    PyObject *r = PyObject_CallFunction(t_raise, "si", name, (int)st);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
    return -1;
}
/* The KvCache's struct and its device, which has to be the current one.  k, k_scale: its tensors (new references). */
static int get_cache(PyObject *o, baps_kv_cache *c, PyObject **k, PyObject **k_scale, int64_t *device)
{
    int64_t now;
    *k = *k_scale = NULL;
    PyObject *b = PyObject_GetAttr(o, s_struct);
    if (!b) return -1;
    if (!PyBytes_Check(b) || PyBytes_GET_SIZE(b) != (Py_ssize_t)sizeof(baps_kv_cache)) {
        Py_DECREF(b);
        return refuse("cache", "a KvCache");
    }
    memcpy(c, PyBytes_AS_STRING(b), sizeof(baps_kv_cache));
    Py_DECREF(b);
    if (!(*k = PyObject_GetAttr(o, s_k)) || !(*k_scale = PyObject_GetAttr(o, s_k_scale)) ||
        long_of(PyObject_CallMethodNoArgs(*k, s_get_device), device) || long_of(PyObject_CallNoArgs(t_device), &now))
        return -1;
    if (*device != now) {
        PyErr_Format(PyExc_ValueError, "the cache is on cuda:%lld, the current device is cuda:%lld", (long long)*device, (long long)now);
        return -1;
    }
    return 0;
}
static int arg_count(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return -1;
}

/* ---- window(q, k, v, out | None, lse | None, lengths | None, window, sinks, scale) -> out ----------------- */
static PyObject *call_window(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    tensor q, k, v, out, lse = {0}, len = {0};
    int64_t st[12];
    int code, window, sinks;
    baps_stream stream;
    if (arg_count(n, 9) || get_16(a[0], "q", 4, &q, &code) || get_tensor(a[1], "k", &k) || get_tensor(a[2], "v", &v)) return NULL;
    if (k.dim != 4 || k.shape[0] != q.shape[0] || k.shape[2] != q.shape[2] || k.shape[3] != q.shape[3]) {
        refuse("k", "[B,Hkv,S,D] to match q [B,H,S,D]");
        return NULL;
    }
    for (int i = 0; i < 4; ++i)
        if (fits_int("a size", q.shape[i]) || fits_int("a size", k.shape[i])) return NULL;
    const double scale = PyFloat_AsDouble(a[8]);
    if ((scale == -1.0 && PyErr_Occurred()) || int_arg(a[6], "window", 1, &window) || int_arg(a[7], "sinks", 0, &sinks)) return NULL;
    const int64_t rows[3] = {q.shape[0], q.shape[1], q.shape[2]};
    if (a[4] != Py_None && get_buffer(a[4], "lse", t_f32, "float32", q.device, 3, rows, &lse)) return NULL;
    if (a[5] != Py_None && get_buffer(a[5], "lengths", t_i32, "int32", q.device, 1, rows, &len)) return NULL;
    if (rows_of(&q, "q", &q, 4, q.shape, st) || rows_of(&k, "k", &q, 4, k.shape, st + 3) || rows_of(&v, "v", &q, 4, k.shape, st + 6)) return NULL;
    PyObject *o = a[3];
    if (o == Py_None) {
        void *p;
        if (!(o = new_tensor(a[0], -1, NULL, &p))) return NULL;
    } else {
        Py_INCREF(o);
    }
    if (get_tensor(o, "out", &out) || rows_of(&out, "out", &q, 4, q.shape, st + 9) || stream_of(q.device, &stream)) { Py_DECREF(o); return NULL; }
    baps_status status;
    Py_BEGIN_ALLOW_THREADS
    status = lib.window(q.ptr, k.ptr, v.ptr, out.ptr, lse.ptr, len.ptr, st, (int)q.shape[0], (int)q.shape[1], (int)k.shape[1],
                        (int)q.shape[2], (int)q.shape[3], window, sinks, (float)scale, code, stream);
    Py_END_ALLOW_THREADS
    if (check("baps_attention_window_fwd", status)) { Py_DECREF(o); return NULL; }
    return o;
}

/* ---- append(cache, k_new, v_new, table, lengths, starts, max_new | None) ------------------------------------ */
static PyObject *call_append(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    baps_kv_cache c;
    tensor k, v, table, len, starts;
    PyObject *ck = NULL, *cs = NULL, *result = NULL;
    int64_t device, st[4];
    int code;
    baps_stream stream;
    if (arg_count(n, 7) || get_cache(a[0], &c, &ck, &cs, &device) || get_16(a[1], "k_new", 3, &k, &code) || get_tensor(a[2], "v_new", &v) ||
        get_tensor(a[3], "table", &table))
        goto done;
    const int64_t shape[3] = {k.shape[0], c.Hkv, c.D}, more[1] = {table.shape[0] + 1};
    if (table.dim != 2) { refuse("table", "[B,width]"); goto done; }
    if (rows_of(&k, "k_new", &k, 3, shape, st) || rows_of(&v, "v_new", &k, 3, shape, st + 2) ||
        get_buffer(a[3], "table", t_i32, "int32", device, 2, table.shape, &table) ||
        get_buffer(a[4], "lengths", t_i32, "int32", device, 1, table.shape, &len) ||
        get_buffer(a[5], "starts", t_i32, "int32", device, 1, more, &starts) || fits_int("a size", table.shape[0]) ||
        fits_int("a size", table.shape[1]) || stream_of(device, &stream))
        goto done;
    int64_t most = k.shape[0];
    if (a[6] != Py_None) {
        int x;
        if (int_arg(a[6], "max_new", 0, &x)) goto done;
        if (x < most) most = x;
    }
    if (fits_int("max_new", most)) goto done;
    baps_status status;
    Py_BEGIN_ALLOW_THREADS
    status = lib.append(&c, k.ptr, v.ptr, st, k.shape[0], starts.ptr, len.ptr, table.ptr, (int)table.shape[1], (int)table.shape[0],
                        (int)most, code, stream);
    Py_END_ALLOW_THREADS
    if (!check("baps_kv_append", status)) result = Py_NewRef(Py_None);
done:
    Py_XDECREF(ck);
    Py_XDECREF(cs);
    return result;
}

/* ---- attention(q, cache, table, lengths, window, sinks, scale, out | None, want_lse, lse | None, workspace | None) ------ */
static PyObject *call_attention(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    baps_kv_cache c;
    tensor q, table, len, out, lse, ws;
    PyObject *ck = NULL, *cs = NULL, *o = NULL, *l = NULL, *w = NULL, *result = NULL;
    int64_t device, st[6];
    int code, window, sinks;
    baps_stream stream;
    if (arg_count(n, 11) || get_16(a[0], "q", 4, &q, &code) || get_cache(a[1], &c, &ck, &cs, &device) || get_tensor(a[2], "table", &table)) goto done;
    if (table.dim != 2 || table.shape[0] != q.shape[0] || q.shape[3] != c.D) { refuse("q and table", "[B,H,T,D] of the cache's D and [B,width]"); goto done; }
    const double scale = PyFloat_AsDouble(a[6]);
    if ((scale == -1.0 && PyErr_Occurred()) || int_arg(a[4], "window", 1, &window) || int_arg(a[5], "sinks", 0, &sinks)) goto done;
    if (get_buffer(a[2], "table", t_i32, "int32", device, 2, table.shape, &table) ||
        get_buffer(a[3], "lengths", t_i32, "int32", device, 1, table.shape, &len) || rows_of(&q, "q", &q, 4, q.shape, st) ||
        fits_int("a size", q.shape[0]) || fits_int("a size", q.shape[1]) || fits_int("a size", q.shape[2]) || fits_int("a size", table.shape[1]))
        goto done;
    const int want_lse = PyObject_IsTrue(a[8]);
    if (want_lse < 0) goto done;
    lse.ptr = NULL;
    if (a[9] != Py_None) {
        if (get_buffer(a[9], "lse", t_f32, "float32", device, 3, q.shape, &lse)) goto done;
        l = Py_NewRef(a[9]);
    } else if (want_lse && !(l = new_tensor(cs, 3, q.shape, &lse.ptr))) {
        goto done;
    }
    if (a[7] != Py_None) o = Py_NewRef(a[7]);
    else if (!(o = new_tensor(a[0], -1, NULL, &out.ptr))) goto done;
    if (get_tensor(o, "out", &out) || rows_of(&out, "out", &q, 4, q.shape, st + 3)) goto done;
    size_t bytes;
    ws.ptr = NULL;
    if (a[10] != Py_None) {
        if (get_tensor(a[10], "workspace", &ws)) goto done;
        if (ws.dtype != t_u8 || ws.device != device || !contiguous(&ws)) { refuse("workspace", "a contiguous uint8 tensor on q's device"); goto done; }
        bytes = 1;
        for (int64_t i = 0; i < ws.dim; ++i) bytes *= (size_t)ws.shape[i];
    } else {
        bytes = lib.attention_workspace((int)q.shape[0], (int)q.shape[1], c.Hkv, (int)q.shape[2], c.D, c.page, (int)table.shape[1], window, sinks);
        const int64_t size[1] = {(int64_t)bytes};
        if (bytes && !(w = new_tensor(ck, 1, size, &ws.ptr))) goto done;
    }
    if (stream_of(device, &stream)) goto done;
    baps_status status;
    Py_BEGIN_ALLOW_THREADS
    status = lib.attention(q.ptr, out.ptr, lse.ptr, &c, table.ptr, (int)table.shape[1], len.ptr, st, (int)q.shape[0], (int)q.shape[1],
                           (int)q.shape[2], window, sinks, (float)scale, code, ws.ptr, bytes, stream);
    Py_END_ALLOW_THREADS
    if (check("baps_kv_attention", status)) goto done;
    result = want_lse ? PyTuple_Pack(2, o, l) : Py_NewRef(o);
done:
    Py_XDECREF(ck);
    Py_XDECREF(cs);
    Py_XDECREF(o);
    Py_XDECREF(l);
    Py_XDECREF(w);
    return result;
}

/* ---- fork(cache, table, lengths, refs, parents, reserve, window, sinks) -> (new_table, new_lengths, new_refs) ------------- */
static PyObject *call_fork(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    baps_kv_cache c;
    tensor table, len, refs, parents;
    PyObject *ck = NULL, *cs = NULL, *nt = NULL, *nl = NULL, *nr = NULL, *w = NULL, *result = NULL;
    void *ntp, *nlp, *nrp, *wp;
    int64_t device;
    int reserve, window, sinks;
    baps_stream stream;
    if (arg_count(n, 8) || get_cache(a[0], &c, &ck, &cs, &device) || get_tensor(a[1], "table", &table) || get_tensor(a[4], "parents", &parents)) goto done;
    if (table.dim != 2 || parents.dim != 1) { refuse("table and parents", "[rows,width] and [new_rows]"); goto done; }
    const int64_t pages[1] = {c.n_pages}, shape[2] = {parents.shape[0], table.shape[1]};
    if (get_buffer(a[1], "table", t_i32, "int32", device, 2, table.shape, &table) ||
        get_buffer(a[2], "lengths", t_i32, "int32", device, 1, table.shape, &len) ||
        get_buffer(a[3], "refs", t_i32, "int32", device, 1, pages, &refs) ||
        get_buffer(a[4], "parents", t_i32, "int32", device, 1, parents.shape, &parents) || int_arg(a[5], "reserve", 0, &reserve) ||
        int_arg(a[6], "window", 1, &window) || int_arg(a[7], "sinks", 0, &sinks) || fits_int("a size", table.shape[0]) ||
        fits_int("a size", table.shape[1]) || fits_int("a size", parents.shape[0]))
        goto done;
    const size_t bytes = lib.pages_workspace((int)parents.shape[0], c.n_pages);
    const int64_t size[1] = {(int64_t)bytes};
    if (!(nt = new_tensor(a[1], shape[0] == table.shape[0] ? -1 : 2, shape, &ntp)) || !(nl = new_tensor(a[4], -1, NULL, &nlp)) ||
        !(nr = new_tensor(a[3], -1, NULL, &nrp)) || !(w = new_tensor(ck, 1, size, &wp)) || stream_of(device, &stream))
        goto done;
    baps_status status;
    Py_BEGIN_ALLOW_THREADS
    status = lib.fork(&c, table.ptr, len.ptr, (int)table.shape[0], refs.ptr, parents.ptr, (int)parents.shape[0], (int)table.shape[1], reserve,
                      window, sinks, ntp, nlp, nrp, wp, bytes, stream);
    Py_END_ALLOW_THREADS
    if (!check("baps_kv_fork", status)) result = PyTuple_Pack(3, nt, nl, nr);
done:
    Py_XDECREF(ck);
    Py_XDECREF(cs);
    Py_XDECREF(nt);
    Py_XDECREF(nl);
    Py_XDECREF(nr);
    Py_XDECREF(w);
    return result;
}

/* ---- compact(cache, table, refs) -> (new_table, new_refs, page_map, n_live) -------------------------------------------- */
static PyObject *call_compact(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    baps_kv_cache c;
    tensor table, refs;
    PyObject *ck = NULL, *cs = NULL, *nt = NULL, *nr = NULL, *pm = NULL, *live = NULL, *w = NULL, *result = NULL;
    void *ntp, *nrp, *pmp, *lp, *wp;
    int64_t device;
    baps_stream stream;
    if (arg_count(n, 3) || get_cache(a[0], &c, &ck, &cs, &device) || get_tensor(a[1], "table", &table)) goto done;
    if (table.dim != 2) { refuse("table", "[rows,width]"); goto done; }
    const int64_t pages[1] = {c.n_pages}, one[1] = {1};
    if (get_buffer(a[1], "table", t_i32, "int32", device, 2, table.shape, &table) ||
        get_buffer(a[2], "refs", t_i32, "int32", device, 1, pages, &refs) || fits_int("a size", table.shape[0]) || fits_int("a size", table.shape[1]))
        goto done;
    const size_t bytes = lib.pages_workspace(0, c.n_pages);
    const int64_t size[1] = {(int64_t)bytes};
    if (!(nt = new_tensor(a[1], -1, NULL, &ntp)) || !(nr = new_tensor(a[2], -1, NULL, &nrp)) || !(pm = new_tensor(a[2], -1, NULL, &pmp)) ||
        !(live = new_tensor(a[2], 1, one, &lp)) || !(w = new_tensor(ck, 1, size, &wp)) || stream_of(device, &stream))
        goto done;
    baps_status status;
    Py_BEGIN_ALLOW_THREADS
    status = lib.compact(&c, table.ptr, (int)table.shape[0], (int)table.shape[1], refs.ptr, ntp, nrp, pmp, lp, wp, bytes, stream);
    Py_END_ALLOW_THREADS
    if (!check("baps_kv_compact", status)) result = PyTuple_Pack(4, nt, nr, pm, live);
done:
    Py_XDECREF(ck);
    Py_XDECREF(cs);
    Py_XDECREF(nt);
    Py_XDECREF(nr);
    Py_XDECREF(pm);
    Py_XDECREF(live);
    Py_XDECREF(w);
    return result;
}

/* ---- cache_struct(k, v, k_scale, v_scale) -> bytes of baps_kv_cache ------------------------------------------------------ */
static PyObject *call_cache_struct(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    tensor k, v, ks, vs;
    if (arg_count(n, 4) || get_tensor(a[0], "k", &k)) return NULL;
    if (k.dtype != t_u8 || k.device < 0 || k.dim != 4 || !contiguous(&k)) { refuse("k", "contiguous uint8 CUDA codes [n_pages,Hkv,page,D]"); return NULL; }
    if (get_buffer(a[1], "v", t_u8, "uint8", k.device, 4, k.shape, &v) || get_buffer(a[2], "k_scale", t_f32, "float32", k.device, 2, k.shape, &ks) ||
        get_buffer(a[3], "v_scale", t_f32, "float32", k.device, 2, k.shape, &vs))
        return NULL;
    for (int i = 0; i < 4; ++i)
        if (fits_int("a size", k.shape[i])) return NULL;
    baps_kv_cache c;
    memset(&c, 0, sizeof(c));
    c.k = k.ptr; c.v = v.ptr; c.k_scale = ks.ptr; c.v_scale = vs.ptr;
    c.n_pages = (int)k.shape[0]; c.Hkv = (int)k.shape[1]; c.page = (int)k.shape[2]; c.D = (int)k.shape[3];
    return PyBytes_FromStringAndSize((const char *)&c, sizeof(c));
}

/* ---- bind(objects, addresses): torch's objects and the library's functions, in the order below ----------------------------- */
static PyObject *call_bind(PyObject *self, PyObject *args)
{
    (void)self;
    PyObject *o[9];
    unsigned long long f[7];
    if (!PyArg_ParseTuple(args, "(OOOOOOOOO)(KKKKKKK)", &o[0], &o[1], &o[2], &o[3], &o[4], &o[5], &o[6], &o[7], &o[8], &f[0], &f[1], &f[2],
                          &f[3], &f[4], &f[5], &f[6]))
        return NULL;
    PyObject **to[9] = {&t_bf16, &t_f16, &t_f32, &t_i32, &t_u8, &t_empty_like, &t_device, &t_stream, &t_raise};
    for (int i = 0; i < 9; ++i) Py_XSETREF(*to[i], Py_NewRef(o[i]));
    void *p[7];
    for (int i = 0; i < 7; ++i) p[i] = (void *)(uintptr_t)f[i];
    memcpy(&lib, p, sizeof(p));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", call_bind, METH_VARARGS, NULL},
    {"cache_struct", (PyCFunction)(void (*)(void))call_cache_struct, METH_FASTCALL, NULL},
    {"window", (PyCFunction)(void (*)(void))call_window, METH_FASTCALL, NULL},
    {"append", (PyCFunction)(void (*)(void))call_append, METH_FASTCALL, NULL},
    {"attention", (PyCFunction)(void (*)(void))call_attention, METH_FASTCALL, NULL},
    {"fork", (PyCFunction)(void (*)(void))call_fork, METH_FASTCALL, NULL},
    {"compact", (PyCFunction)(void (*)(void))call_compact, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", "Argument marshalling of the serving calls.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__serving(void)
{
    _Static_assert(sizeof(lib) == 7 * sizeof(void *), "seven addresses");
    PyObject **to[9] = {&s_dtype, &s_shape, &s_stride, &s_get_device, &s_data_ptr, &s_new_empty, &s_struct, &s_k, &s_k_scale};
    const char *names[9] = {"dtype", "shape", "stride", "get_device", "data_ptr", "new_empty", "struct", "k", "k_scale"};
    for (int i = 0; i < 9; ++i)
        if (!(*to[i] = PyUnicode_InternFromString(names[i]))) return NULL;
    return PyModule_Create(&module);
}
