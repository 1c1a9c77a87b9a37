/* Python entry points of the context-free operators (dt_rope, dt_add_rmsnorm, dt_cross_attn): argument marshalling only, in C
 * because on small tensors the marshalling is the call (through ctypes 8 to 11 us of host time a call, this way 5.7 to 6.1, against 3 to 5 us on the GPU).
 * Tensors are looked at through their Python attributes, so nothing here depends on torch's headers; the library's functions
 * are called through the addresses that binding.py hands to _bind. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/ditango.h"

enum { MAX_DIM = 8 };
enum { T_BF16 = DT_VALUE_BF16, T_FP16 = DT_VALUE_FP16, T_FP32 = DT_VALUE_FP32, T_FP64, T_I32, T_U8, T_BOOL, T_E4M3, T_COUNT, T_OTHER = -1 };

typedef struct {
    int64_t shape[MAX_DIM], stride[MAX_DIM];
    void *ptr;
    int nd, dtype;
    long device;
} Tensor;

static PyObject *dtypes[T_COUNT];
static PyObject *raw_stream, *get_device, *on_device, *raise_status;   /* callables of binding.py and torch */
static PyObject *s_shape, *s_stride, *s_data_ptr, *s_dtype, *s_get_device, *s_cuda_stream;
static dt_status (*f_rope)(const dt_rope_config *, const void *, const int64_t *, void *, const int64_t *, const void *, const int64_t *,
                           void *, const int64_t *, const double *, const int32_t *, const int64_t *, void *);
static dt_status (*f_norm)(const dt_norm_config *, const void *, const void *, const void *, void *, void *, float *, void *);
static dt_status (*f_cross)(const dt_cross_config *, const void *, const int64_t *, const void *, const int64_t *, const void *,
                            const int64_t *, const int32_t *, const uint8_t *, int64_t, void *, const int64_t *, float *, void *);

static int ints_of(PyObject *seq, int64_t *out) {   /* a tuple's integers; steals the reference; -1 with an error set */
    if (!seq) return -1;
    int n = -1;
    if (!PyTuple_Check(seq) || PyTuple_GET_SIZE(seq) > MAX_DIM) {
        PyErr_SetString(PyExc_AssertionError, "a tensor of at most 8 dimensions is wanted");
    } else {
        n = (int)PyTuple_GET_SIZE(seq);
        for (int i = 0; i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(seq, i));
        if (PyErr_Occurred()) n = -1;
    }
    Py_DECREF(seq);
    return n;
}

static int look(PyObject *t, Tensor *x) {   /* 0, or -1 with an error set */
    x->nd = ints_of(PyObject_GetAttr(t, s_shape), x->shape);
    if (x->nd < 0) return -1;
    const int n = ints_of(PyObject_CallMethodNoArgs(t, s_stride), x->stride);
    if (n < 0) return -1;
    if (n != x->nd) {
        PyErr_SetString(PyExc_AssertionError, "a strided tensor is wanted");
        return -1;
    }
    PyObject *o = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!o) return -1;
    x->ptr = PyLong_AsVoidPtr(o);
    Py_DECREF(o);
    o = PyObject_CallMethodNoArgs(t, s_get_device);
    if (!o) return -1;
    x->device = PyLong_AsLong(o);
    Py_DECREF(o);
    o = PyObject_GetAttr(t, s_dtype);
    if (!o) return -1;
    x->dtype = T_OTHER;
    for (int i = 0; i < T_COUNT; ++i)
        if (o == dtypes[i]) x->dtype = i;
    Py_DECREF(o);
    return PyErr_Occurred() ? -1 : 0;
}

static int same_shape(const Tensor *a, const Tensor *b) {
    if (a->nd != b->nd) return 0;
    for (int i = 0; i < a->nd; ++i)
        if (a->shape[i] != b->shape[i]) return 0;
    return 1;
}
static int is_shape(const Tensor *a, int nd, int64_t s0, int64_t s1, int64_t s2, int64_t s3) {
    const int64_t s[4] = {s0, s1, s2, s3};
    if (a->nd != nd) return 0;
    for (int i = 0; i < nd; ++i)
        if (a->shape[i] != s[i]) return 0;
    return 1;
}
static int contiguous(const Tensor *a) {
    int64_t want = 1;
    for (int i = a->nd - 1; i >= 0; --i) {
        if (a->shape[i] == 0) return 1;
        if (a->shape[i] != 1 && a->stride[i] != want) return 0;
        want *= a->shape[i];
    }
    return 1;
}

#define NEED(cond)                                                                        \
    do {                                                                                  \
        if (!(cond)) {                                                                    \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_AssertionError, #cond);          \
            return NULL;                                                                  \
        }                                                                                 \
    } while (0)

/* Positional and keyword arguments into `slot` (borrowed; NULL where not given). */
static int take(const char *name, const char *const *names, int count, int required, PyObject *const *args, Py_ssize_t nargs,
                PyObject *kwnames, PyObject **slot) {
    const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    if (nargs > count) {
        PyErr_Format(PyExc_TypeError, "%s() takes at most %d arguments", name, count);
        return -1;
    }
    for (int i = 0; i < count; ++i) slot[i] = i < nargs ? args[i] : NULL;
    for (Py_ssize_t k = 0; k < nkw; ++k) {
        PyObject *key = PyTuple_GET_ITEM(kwnames, k);
        int i = 0;
        while (i < count && PyUnicode_CompareWithASCIIString(key, names[i]) != 0) ++i;
        if (i == count || slot[i]) {
            PyErr_Format(PyExc_TypeError, i == count ? "%s() got an unexpected keyword argument '%U'" : "%s() got multiple values for argument '%U'", name, key);
            return -1;
        }
        slot[i] = args[nargs + k];
    }
    for (int i = 0; i < count; ++i) {
        if (slot[i] == Py_None && i >= required) slot[i] = NULL;   /* (an optional argument's None) */
        if (!slot[i] && i < required) {
            PyErr_Format(PyExc_TypeError, "%s() is missing argument '%s'", name, names[i]);
            return -1;
        }
    }
    return 0;
}

/* The stream's pointer, or the tensors' device is not current and `*again` is the call's result on it (NULL: error set). */
static int stream_of(PyObject *stream, long device, void **out) {
    PyObject *o;
    if (stream) {
        o = PyObject_GetAttr(stream, s_cuda_stream);
    } else {
        PyObject *i = PyLong_FromLong(device);
        if (!i) return -1;
        o = PyObject_CallOneArg(raw_stream, i);
        Py_DECREF(i);
    }
    if (!o) return -1;
    *out = PyLong_AsVoidPtr(o);
    Py_DECREF(o);
    return PyErr_Occurred() ? -1 : 0;
}
static int is_current(long device) {   /* 1, 0, or -1 with an error set */
    PyObject *o = PyObject_CallNoArgs(get_device);
    if (!o) return -1;
    const long d = PyLong_AsLong(o);
    Py_DECREF(o);
    return PyErr_Occurred() ? -1 : d == device;
}
/* binding.py makes `device` current and calls again with the same arguments */
static PyObject *call_on(long device, const char *name, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    PyObject *pos = PyTuple_New(nargs), *kw = PyDict_New(), *r = NULL;
    if (pos && kw) {
        for (Py_ssize_t i = 0; i < nargs; ++i) PyTuple_SET_ITEM(pos, i, Py_NewRef(args[i]));
        int ok = 1;
        for (Py_ssize_t k = 0; ok && kwnames && k < PyTuple_GET_SIZE(kwnames); ++k)
            ok = PyDict_SetItem(kw, PyTuple_GET_ITEM(kwnames, k), args[nargs + k]) == 0;
        if (ok) r = PyObject_CallFunction(on_device, "lsOO", device, name, pos, kw);
    }
    Py_XDECREF(pos);
    Py_XDECREF(kw);
    return r;
}
static PyObject *done(dt_status s) {
    if (s == DT_OK) Py_RETURN_NONE;
    return PyObject_CallFunction(raise_status, "i", (int)s);   /* raises */
}
#define ON_DEVICE(name, device)                                                  \
    do {                                                                         \
        const int cur_ = is_current(device);                                     \
        if (cur_ < 0) return NULL;                                               \
        if (!cur_) return call_on(device, name, args, nargs, kwnames);           \
    } while (0)

static PyObject *py_rope(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    static const char *const names[] = {"q", "k", "q_out", "k_out", "freqs", "positions", "layout", "attn_factor", "transpose", "stream"};
    PyObject *a[10];
    if (take("dt_rope", names, 10, 5, args, nargs, kwnames, a) < 0) return NULL;
    Tensor q, k, qo, ko, f, pos;
    if (look(a[0], &q) < 0 || look(a[2], &qo) < 0 || look(a[4], &f) < 0) return NULL;
    NEED(q.nd == 4 && q.device >= 0);
    NEED(same_shape(&q, &qo) && qo.dtype == q.dtype && qo.device == q.device);
    NEED(q.dtype == T_BF16 || q.dtype == T_FP16);
    NEED(f.dtype == T_FP64 && f.nd == 2 && contiguous(&f) && f.device == q.device);
    const int64_t B = q.shape[0], L = q.shape[1], axes = f.shape[0], pairs = f.shape[1];
    dt_rope_config c = {0};
    const int have_k = a[1] != Py_None;
    if (have_k) {
        if (look(a[1], &k) < 0 || look(a[3], &ko) < 0) return NULL;
        NEED(k.nd == 4 && is_shape(&k, 4, B, L, k.shape[2], q.shape[3]) && same_shape(&k, &ko));
        NEED(k.dtype == q.dtype && ko.dtype == q.dtype && k.device == q.device && ko.device == q.device);
    }
    int64_t ps[3] = {0, 0, 0};
    if (a[5]) {
        if (look(a[5], &pos) < 0) return NULL;
        NEED(pos.dtype == T_I32 && pos.device == q.device);
        NEED(is_shape(&pos, 3, B, L, axes, 0) || (axes == 1 && is_shape(&pos, 2, B, L, 0, 0)));
        for (int i = 0; i < pos.nd; ++i) ps[i] = pos.stride[i];
    }
    NEED(B <= INT32_MAX && L <= INT32_MAX && q.shape[2] <= INT32_MAX && q.shape[3] <= INT32_MAX && axes <= INT32_MAX && pairs <= INT32_MAX / 2);
    c.dtype = q.dtype;
    c.B = (int32_t)B; c.L = (int32_t)L; c.H = (int32_t)q.shape[2]; c.D = (int32_t)q.shape[3];
    if (have_k) {
        NEED(k.shape[2] <= INT32_MAX);
        c.H_k = (int32_t)k.shape[2];
    }
    c.rotary_dim = (int32_t)(2 * pairs);
    c.axes = (int32_t)axes;
    c.layout = a[6] ? (int32_t)PyLong_AsLong(a[6]) : DT_ROPE_INTERLEAVED;
    c.attn_factor = a[7] ? (float)PyFloat_AsDouble(a[7]) : 1.0f;
    c.transpose = a[8] ? PyObject_IsTrue(a[8]) : 0;
    if (PyErr_Occurred()) return NULL;
    ON_DEVICE("dt_rope", q.device);
    void *st;
    if (stream_of(a[9], q.device, &st) < 0) return NULL;
    return done(f_rope(&c, q.ptr, q.stride, qo.ptr, qo.stride, have_k ? k.ptr : NULL, have_k ? k.stride : NULL, have_k ? ko.ptr : NULL,
                       have_k ? ko.stride : NULL, f.ptr, a[5] ? pos.ptr : NULL, a[5] ? ps : NULL, st));
}

/* Leading dimensions of `t` collapsed into at most two (n, stride), outer first; 0 if they do not. */
static int rows_of(const Tensor *t, int64_t n[2], int64_t s[2]) {
    int64_t cn[MAX_DIM], cs[MAX_DIM];
    int m = 0;
    if (t->shape[t->nd - 1] != 1 && t->stride[t->nd - 1] != 1) return 0;
    for (int i = 0; i + 1 < t->nd; ++i) {
        if (t->shape[i] == 1) continue;
        if (m && cs[m - 1] == t->shape[i] * t->stride[i]) {
            cn[m - 1] *= t->shape[i];
            cs[m - 1] = t->stride[i];
        } else {
            cn[m] = t->shape[i];
            cs[m++] = t->stride[i];
        }
    }
    if (m > 2) return 0;
    n[0] = n[1] = 1;
    s[0] = s[1] = 0;
    for (int i = 0; i < m; ++i) {
        n[2 - m + i] = cn[i];
        s[2 - m + i] = cs[i];
    }
    return 1;
}
/* The rows of several tensors of one shape as one n0 x n1 with strides for each; 0 if there are no such. */
static int common_rows(const Tensor *const *t, int count, int64_t n[2], int64_t (*s)[2]) {
    int64_t each[4][2];
    int all = 1;
    for (int i = 0; i < count; ++i) all = all && contiguous(t[i]);
    if (all) {
        const int64_t w = t[0]->shape[t[0]->nd - 1];
        n[0] = n[1] = 1;
        for (int i = 0; i + 1 < t[0]->nd; ++i) n[1] *= t[0]->shape[i];
        for (int i = 0; i < count; ++i) {
            s[i][0] = 0;
            s[i][1] = w;
        }
        return 1;
    }
    for (int i = 0; i < count; ++i)
        if (!rows_of(t[i], each[i], s[i])) return 0;
    n[0] = each[0][0];
    n[1] = each[0][1];
    for (int i = 0; i < count; ++i)
        if (each[i][0] != 1) {
            n[0] = each[i][0];
            n[1] = each[i][1];
            break;
        }
    for (int i = 0; i < count; ++i) {
        if (each[i][0] == n[0] && each[i][1] == n[1]) continue;
        if (each[i][0] != 1 || each[i][1] != n[0] * n[1]) return 0;
        s[i][0] = n[1] * s[i][1];   /* its rows collapse further than another's: split the same way */
    }
    return 1;
}

static PyObject *py_norm(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    static const char *const names[] = {"x", "weight", "y", "eps", "residual", "residual_out", "scales", "stream"};
    PyObject *a[8];
    if (take("dt_add_rmsnorm", names, 8, 4, args, nargs, kwnames, a) < 0) return NULL;
    Tensor x, w, y, r, ro, sc;
    if (look(a[0], &x) < 0 || look(a[2], &y) < 0) return NULL;
    NEED(x.nd >= 1 && x.device >= 0 && (x.dtype == T_BF16 || x.dtype == T_FP16));
    const int q8 = y.dtype == T_E4M3;
    NEED(same_shape(&x, &y) && (q8 || y.dtype == x.dtype) && y.device == x.device);
    NEED((a[4] == NULL) == (a[5] == NULL));
    const Tensor *rows[4] = {&x, &y, &r, &ro};
    dt_norm_config c = {0};
    c.dtype = c.weight_dtype = c.residual_dtype = x.dtype;
    if (a[4]) {
        if (look(a[4], &r) < 0 || look(a[5], &ro) < 0) return NULL;
        NEED(same_shape(&x, &r) && same_shape(&x, &ro) && ro.dtype == r.dtype && r.device == x.device && ro.device == x.device);
        NEED(r.dtype == x.dtype || r.dtype == T_FP32);
        c.residual_dtype = r.dtype;
    }
    const int64_t width = x.shape[x.nd - 1];
    const int have_w = a[1] != Py_None;
    if (have_w) {
        if (look(a[1], &w) < 0) return NULL;
        NEED(is_shape(&w, 1, width, 0, 0, 0) && contiguous(&w) && w.device == x.device && (w.dtype == x.dtype || w.dtype == T_FP32));
        c.weight_dtype = w.dtype;
    }
    if (q8) {
        NEED(a[6] != NULL);
        if (look(a[6], &sc) < 0) return NULL;
        NEED(sc.dtype == T_FP32 && sc.nd == x.nd && contiguous(&sc) && sc.device == x.device);
        for (int i = 0; i + 1 < x.nd; ++i) NEED(sc.shape[i] == x.shape[i]);
        const int64_t per_row = sc.shape[sc.nd - 1];
        NEED(per_row > 0 && width % per_row == 0);
        NEED(width / per_row <= INT32_MAX);
        c.scale_group = per_row == 1 ? 0 : (int32_t)(width / per_row);
    }
    int64_t n[2], s[4][2] = {{0}};
    NEED(common_rows(rows, a[4] ? 4 : 2, n, s) && "rows of two strides at most, common to all, and values of stride 1");
    NEED(width <= INT32_MAX);
    c.out_kind = q8 ? DT_NORM_OUT_E4M3 : DT_NORM_OUT_SAME;
    c.n0 = n[0]; c.n1 = n[1];
    c.width = (int32_t)width;
    for (int d = 0; d < 2; ++d) {
        c.x_strides[d] = s[0][d]; c.y_strides[d] = s[1][d];
        c.residual_strides[d] = s[2][d]; c.residual_out_strides[d] = s[3][d];
    }
    c.eps = (float)PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return NULL;
    ON_DEVICE("dt_add_rmsnorm", x.device);
    void *st;
    if (stream_of(a[7], x.device, &st) < 0) return NULL;
    return done(f_norm(&c, x.ptr, have_w ? w.ptr : NULL, a[4] ? r.ptr : NULL, a[4] ? ro.ptr : NULL, y.ptr, q8 ? sc.ptr : NULL, st));
}

static PyObject *py_cross(PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames) {
    static const char *const names[] = {"q", "k", "v", "out", "softmax_scale", "key_lens", "key_mask", "lse_out", "stream"};
    PyObject *a[9];
    if (take("dt_cross_attn", names, 9, 5, args, nargs, kwnames, a) < 0) return NULL;
    Tensor q, k, v, o, lens, mask, lse;
    if (look(a[0], &q) < 0 || look(a[1], &k) < 0 || look(a[2], &v) < 0 || look(a[3], &o) < 0) return NULL;
    NEED(q.nd == 4 && q.device >= 0 && k.nd == 4);
    NEED(q.dtype == T_BF16 || q.dtype == T_FP16);
    NEED(k.shape[0] == q.shape[0] && k.shape[3] == q.shape[3] && same_shape(&k, &v) && same_shape(&q, &o));
    NEED(k.dtype == q.dtype && v.dtype == q.dtype && o.dtype == q.dtype);
    NEED(k.device == q.device && v.device == q.device && o.device == q.device);
    const int64_t B = q.shape[0], Lq = q.shape[1], H = q.shape[2], Lk = k.shape[1];
    NEED(B <= INT32_MAX && Lq <= INT32_MAX && H <= INT32_MAX && Lk <= INT32_MAX && k.shape[2] <= INT32_MAX && q.shape[3] <= INT32_MAX);
    if (a[5]) {
        if (look(a[5], &lens) < 0) return NULL;
        NEED(lens.dtype == T_I32 && is_shape(&lens, 1, B, 0, 0, 0) && contiguous(&lens) && lens.device == q.device);
    }
    if (a[6]) {
        if (look(a[6], &mask) < 0) return NULL;
        NEED((mask.dtype == T_U8 || mask.dtype == T_BOOL) && is_shape(&mask, 2, B, Lk, 0, 0) && mask.device == q.device);
        NEED(Lk <= 1 || mask.stride[1] == 1);
    }
    if (a[7]) {
        if (look(a[7], &lse) < 0) return NULL;
        NEED(lse.dtype == T_FP32 && is_shape(&lse, 3, B, H, Lq, 0) && contiguous(&lse) && lse.device == q.device);
    }
    dt_cross_config c = {0};
    c.dtype = q.dtype;
    c.B = (int32_t)B; c.Lq = (int32_t)Lq; c.Lk = (int32_t)Lk; c.H = (int32_t)H; c.H_kv = (int32_t)k.shape[2]; c.D = (int32_t)q.shape[3];
    c.softmax_scale = (float)PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) return NULL;
    ON_DEVICE("dt_cross_attn", q.device);
    void *st;
    if (stream_of(a[8], q.device, &st) < 0) return NULL;
    return done(f_cross(&c, q.ptr, q.stride, k.ptr, k.stride, v.ptr, v.stride, a[5] ? lens.ptr : NULL, a[6] ? mask.ptr : NULL,
                        a[6] ? mask.stride[0] : 0, o.ptr, o.stride, a[7] ? lse.ptr : NULL, st));
}

/* _norm_rows(tensors): (n0, n1, [(stride0, stride1), ...]) as dt_add_rmsnorm sees them (for tests) */
static PyObject *py_rows(PyObject *self, PyObject *list) {
    Tensor t[4];
    const Tensor *p[4] = {&t[0], &t[1], &t[2], &t[3]};
    if (!PyList_Check(list) || PyList_GET_SIZE(list) < 1 || PyList_GET_SIZE(list) > 4) {
        PyErr_SetString(PyExc_TypeError, "a list of one to four tensors");
        return NULL;
    }
    const int count = (int)PyList_GET_SIZE(list);
    for (int i = 0; i < count; ++i)
        if (look(PyList_GET_ITEM(list, i), &t[i]) < 0) return NULL;
    int64_t n[2], s[4][2];
    NEED(common_rows(p, count, n, s));
    PyObject *strides = PyList_New(count);
    if (!strides) return NULL;
    for (int i = 0; i < count; ++i) PyList_SET_ITEM(strides, i, Py_BuildValue("(LL)", (long long)s[i][0], (long long)s[i][1]));
    return Py_BuildValue("LLN", (long long)n[0], (long long)n[1], strides);
}

static PyObject *py_bind(PyObject *self, PyObject *args) {
    unsigned long long rope, norm, cross;
    PyObject *types, *calls[4];
    if (!PyArg_ParseTuple(args, "(KKK)O!(OOOO)", &rope, &norm, &cross, &PyTuple_Type, &types, &calls[0], &calls[1], &calls[2], &calls[3])) return NULL;
    NEED(PyTuple_GET_SIZE(types) == T_COUNT);
    f_rope = (void *)(uintptr_t)rope;
    f_norm = (void *)(uintptr_t)norm;
    f_cross = (void *)(uintptr_t)cross;
    for (int i = 0; i < T_COUNT; ++i) Py_XSETREF(dtypes[i], Py_NewRef(PyTuple_GET_ITEM(types, i)));
    Py_XSETREF(raw_stream, Py_NewRef(calls[0]));
    Py_XSETREF(get_device, Py_NewRef(calls[1]));
    Py_XSETREF(on_device, Py_NewRef(calls[2]));
    Py_XSETREF(raise_status, Py_NewRef(calls[3]));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"dt_rope", (PyCFunction)(void (*)(void))py_rope, METH_FASTCALL | METH_KEYWORDS,
     "dt_rope(q, k, q_out, k_out, freqs, positions=None, layout=DT_ROPE_INTERLEAVED, attn_factor=1.0, transpose=False, stream=None)\n\n"
     "Rotary positions on q [B, L, H, D] and k [B, L, H_k, D] (k and k_out may be None) into q_out, k_out (which may be q, k).\n"
     "freqs is float64 [axes, rotary_dim / 2] on the device, positions int32 [B, L, axes] ([B, L] for one axis; any strides,\n"
     "expanded batches too) or None for the token's index.  See ditango.h."},
    {"dt_add_rmsnorm", (PyCFunction)(void (*)(void))py_norm, METH_FASTCALL | METH_KEYWORDS,
     "dt_add_rmsnorm(x, weight, y, eps, residual=None, residual_out=None, scales=None, stream=None)\n\n"
     "Norm of x (+ residual) over the last dimension into y: x's type, or float8_e4m3fn with scales fp32 [..., width / group]\n"
     "(group: 32, 64, 128 or the whole row).  weight may be None; residual_out takes the sum and may be residual or x.\n"
     "See ditango.h."},
    {"dt_cross_attn", (PyCFunction)(void (*)(void))py_cross, METH_FASTCALL | METH_KEYWORDS,
     "dt_cross_attn(q, k, v, out, softmax_scale, key_lens=None, key_mask=None, lse_out=None, stream=None)\n\n"
     "Attention of q [B, Lq, H, D] to an encoder's k, v [B, Lk, H_kv, D]; key_lens int32 [B], key_mask uint8 or bool [B, Lk]\n"
     "(expanded batches too), lse_out fp32 [B, H, Lq].  See ditango.h."},
    {"_norm_rows", py_rows, METH_O, "rows of tensors as dt_add_rmsnorm sees them"},
    {"_bind", py_bind, METH_VARARGS, "addresses of the library's functions, torch's dtypes, callables"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ditango_ops", "Python entry points of libditango's context-free operators", -1, methods};

PyMODINIT_FUNC PyInit__ditango_ops(void) {
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!s_shape || !s_stride || !s_data_ptr || !s_dtype || !s_get_device || !s_cuda_stream) return NULL;
    return PyModule_Create(&module);
}
