/*
 * Argument marshalling of the Python binding's hot calls, as a CPython extension
 * (paper_2506_07416_gb300/_fastcall.so). Each function takes the arguments of the
 * C function of the same name (include/litevlm_select.h) as Python objects:
 * pointers as integers, numpy arrays or objects with data_ptr() (torch tensors),
 * host offset arrays as int32 numpy arrays (anything else goes through the binding's
 * own conversion), handles and numbers as ctypes takes them, and returns the status
 * code. No other object is a pointer, whatever memory it may show: the address of a
 * numpy scalar or of a bytes object is not the value it holds. The GIL is
 * released around the call. The C functions' addresses come from the library that
 * the binding loaded (bind).
 *
 * Why: with ctypes, a call's 12 to 18 argument conversions and numpy's ctypes
 * attribute took 15 to 20 us of a single-request step that needs 13 us of GPU time.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

enum { F_SCORE, F_FULL, F_SCORE_TOPK, F_TOPK, F_COMPACT, F_SPLICE, F_PROJECT, F_KEEP,
       F_APPEND, F_SPACE, F_ATTEND, F_EVICT, F_VERIFY, F_RESERVE, F_BOUNDS, F_PICK_SPACE, F_PICK, F_PICKED_SPACE,
       F_PICKED, F_APPEND_GRANTED, F_COUNT };
static const char *const kNames[F_COUNT] = {"score", "score_full_keys", "score_topk", "topk",
                                            "compact", "splice", "project", "keep_offsets",
                                            "cache_append", "cache_attend_workspace", "cache_attend", "cache_evict",
                                            "verify", "cache_reserve", "cache_bounds", "cache_pick_workspace",
                                            "cache_pick", "cache_attend_picked_workspace", "cache_attend_picked",
                                            "cache_append_granted"};
/* h handle / stream, i int32, l int64, f float, p pointer, n host int32 array */
static const char *const kSigs[F_COUNT] = {"hippnppnffph", "hippnppnppnpffph", "hippnppnffppnfppph", "hippnpnfppph",
                                           "", "hippnppnppnppnlpppph", "hliipppfippifph", "",
                                           "hippipplpllppnffpppph", "", "hippipplpnifpppplh", "hippipiiiipippph",
                                           "hiiippnpppppph", "hiipipppippnppph", "hipppippnh", "", "hippipplpniiiipplh", "",
                                           "hippipplpnpifpplh", "hippipplpllppnffppppph"};
static void *g_fn[F_COUNT];
static PyObject *g_host_i32;      /* the binding's conversion of a host offset array */
static PyObject *g_ndarray;       /* numpy.ndarray */
static PyObject *g_ctypes_value;  /* the value of a ctypes object of a signature's kind */
static PyObject *g_data_ptr;      /* "data_ptr" */

#define MAX_ARGS 24
typedef struct {
    Py_buffer buf[MAX_ARGS];
    PyObject *obj[MAX_ARGS];
    int nbuf, nobj;
} Held;

static void release(Held *h)
{
    while (h->nbuf > 0) PyBuffer_Release(&h->buf[--h->nbuf]);
    while (h->nobj > 0) Py_DECREF(h->obj[--h->nobj]);
}

static int as_ptr(PyObject *o, Held *h, void **out)
{
    if (o == Py_None) {
        *out = NULL;
        return 0;
    }
    if (PyLong_Check(o)) {
        *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
        return PyErr_Occurred() ? -1 : 0;
    }
    if (PyObject_TypeCheck(o, (PyTypeObject *)g_ndarray)) {
        Py_buffer *b = &h->buf[h->nbuf];
        if (PyObject_GetBuffer(o, b, PyBUF_STRIDED_RO) == 0) {
            ++h->nbuf;
            *out = b->buf;
            return 0;
        }
        PyErr_Clear(); /* a type without a buffer format */
        PyObject *c = PyObject_GetAttrString(o, "ctypes");
        PyObject *d = c ? PyObject_GetAttrString(c, "data") : NULL;
        Py_XDECREF(c);
        if (!d) return -1;
        *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(d);
        Py_DECREF(d);
        return PyErr_Occurred() ? -1 : 0;
    }
    PyObject *r = PyObject_CallMethodNoArgs(o, g_data_ptr);
    if (!r) return -1;
    *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(r);
    Py_DECREF(r);
    return PyErr_Occurred() ? -1 : 0;
}

/* a handle, a stream or a whole number: an int, an object with __index__ (not for
 * handles), or the ctypes object of its kind; longer ones are cut to 64 bits */
static int as_bits(PyObject *o, char kind, uint64_t *out)
{
    PyObject *v;
    if (kind == 'h' && o == Py_None) {
        *out = 0;
        return 0;
    }
    if (PyLong_Check(o)) v = Py_NewRef(o);
    else if (kind != 'h' && PyIndex_Check(o)) v = PyNumber_Index(o);
    else v = PyObject_CallFunction(g_ctypes_value, "OC", o, kind);
    if (!v) return -1;
    *out = (uint64_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int as_double(PyObject *o, double *out)
{
    *out = PyFloat_AsDouble(o);
    if (*out != -1.0 || !PyErr_Occurred()) return 0;
    PyErr_Clear();
    PyObject *v = PyObject_CallFunction(g_ctypes_value, "OC", o, 'f');
    if (!v) return -1;
    *out = PyFloat_AsDouble(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static int as_host_i32(PyObject *o, Held *h, const int32_t **out, Py_ssize_t *len)
{
    *out = NULL;
    if (len) *len = 0;
    if (o == Py_None) return 0;
    for (int tries = 0; tries < 2; ++tries) {
        if (PyObject_CheckBuffer(o)) {
            Py_buffer *b = &h->buf[h->nbuf];
            if (PyObject_GetBuffer(o, b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) == 0) {
                if (b->itemsize == 4 && b->format && b->format[0] == 'i' && !b->format[1]) {
                    ++h->nbuf;
                    *out = (const int32_t *)b->buf;
                    if (len) *len = b->len / 4;
                    return 0;
                }
                PyBuffer_Release(b);
            } else {
                PyErr_Clear();
            }
        }
        if (tries == 1) break;
        o = PyObject_CallOneArg(g_host_i32, o);
        if (!o) return -1;
        h->obj[h->nobj++] = o;
    }
    PyErr_SetString(PyExc_TypeError, "a host offset array is not an int32 array");
    return -1;
}

typedef union {
    void *p;
    int32_t i;
    int64_t l;
    float f;
} Arg;

static int convert(const char *sig, PyObject *const *args, Py_ssize_t n, Held *h, Arg *a)
{
    Py_ssize_t k = 0;
    for (; sig[k]; ++k) {
        if (k >= n) break;
        PyObject *o = args[k];
        switch (sig[k]) {
        case 'p':
            if (as_ptr(o, h, &a[k].p) != 0) return -1;
            break;
        case 'n': {
            const int32_t *q;
            if (as_host_i32(o, h, &q, NULL) != 0) return -1;
            a[k].p = (void *)q;
            break;
        }
        case 'h':
        case 'i':
        case 'l': {
            uint64_t v;
            if (as_bits(o, sig[k], &v) != 0) return -1;
            if (sig[k] == 'i') a[k].i = (int32_t)(uint32_t)v;
            else if (sig[k] == 'l') a[k].l = (int64_t)v;
            else a[k].p = (void *)(uintptr_t)v;
            break;
        }
        default: {
            double v;
            if (as_double(o, &v) != 0) return -1;
            a[k].f = (float)v;
        }
        }
    }
    if (sig[k] || k != n) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return -1;
    }
    return 0;
}

typedef void *P;
typedef int32_t I;

#define BEGIN(which)                                                                    \
    (void)self;                                                                         \
    Held h;                                                                             \
    h.nbuf = h.nobj = 0;                                                                \
    Arg a[MAX_ARGS];                                                                    \
    int rc = 0;                                                                         \
    if (convert(kSigs[which], args, n, &h, a) != 0) {                                   \
        release(&h);                                                                    \
        return NULL;                                                                    \
    }                                                                                   \
    Py_BEGIN_ALLOW_THREADS
#define END                                                                             \
    Py_END_ALLOW_THREADS                                                                \
    release(&h);                                                                        \
    return PyLong_FromLong(rc);

static PyObject *f_score(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_SCORE)
    rc = ((int (*)(P, I, P, P, P, P, P, P, float, float, P, P))g_fn[F_SCORE])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].f, a[9].f, a[10].p, a[11].p);
    END
}

static PyObject *f_full(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_FULL)
    rc = ((int (*)(P, I, P, P, P, P, P, P, P, P, P, P, float, float, P, P))g_fn[F_FULL])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].f,
        a[13].f, a[14].p, a[15].p);
    END
}

static PyObject *f_score_topk(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_SCORE_TOPK)
    rc = ((int (*)(P, I, P, P, P, P, P, P, float, float, P, P, P, float, P, P, P, P))g_fn[F_SCORE_TOPK])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].f, a[9].f, a[10].p, a[11].p, a[12].p,
        a[13].f, a[14].p, a[15].p, a[16].p, a[17].p);
    END
}

static PyObject *f_topk(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_TOPK)
    rc = ((int (*)(P, I, P, P, P, P, P, float, P, P, P, P))g_fn[F_TOPK])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].p, a[6].p, a[7].f, a[8].p, a[9].p, a[10].p, a[11].p);
    END
}

static PyObject *f_splice(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_SPLICE)
    rc = ((int (*)(P, I, P, P, P, P, P, P, P, P, P, P, P, P, int64_t, P, P, P, P, P))g_fn[F_SPLICE])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p, a[12].p,
        a[13].p, a[14].l, a[15].p, a[16].p, a[17].p, a[18].p, a[19].p);
    END
}

static PyObject *f_project(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_PROJECT)
    rc = ((int (*)(P, int64_t, I, I, P, P, P, float, I, P, P, I, float, P, P))g_fn[F_PROJECT])(
        a[0].p, a[1].l, a[2].i, a[3].i, a[4].p, a[5].p, a[6].p, a[7].f, a[8].i, a[9].p, a[10].p, a[11].i, a[12].f,
        a[13].p, a[14].p);
    END
}

static PyObject *f_append(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_APPEND)
    rc = ((int (*)(P, I, P, P, I, P, P, int64_t, P, int64_t, int64_t, P, P, P, float, float, P, P, P, P, P))
          g_fn[F_APPEND])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].p, a[7].l, a[8].p, a[9].l, a[10].l, a[11].p,
        a[12].p, a[13].p, a[14].f, a[15].f, a[16].p, a[17].p, a[18].p, a[19].p, a[20].p);
    END
}

static PyObject *f_append_granted(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_APPEND_GRANTED)
    rc = ((int (*)(P, I, P, P, I, P, P, int64_t, P, int64_t, int64_t, P, P, P, float, float, P, P, P, P, P, P))
          g_fn[F_APPEND_GRANTED])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].p, a[7].l, a[8].p, a[9].l, a[10].l, a[11].p,
        a[12].p, a[13].p, a[14].f, a[15].f, a[16].p, a[17].p, a[18].p, a[19].p, a[20].p, a[21].p);
    END
}

static PyObject *f_attend(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_ATTEND)
    rc = ((int (*)(P, I, P, P, I, P, P, int64_t, P, P, I, float, P, P, P, P, int64_t, P))
          g_fn[F_ATTEND])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].p, a[7].l, a[8].p, a[9].p, a[10].i, a[11].f,
        a[12].p, a[13].p, a[14].p, a[15].p, a[16].l, a[17].p);
    END
}

static PyObject *f_evict(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_EVICT)
    rc = ((int (*)(P, I, P, P, I, P, I, I, I, I, P, I, P, P, P, P))
          g_fn[F_EVICT])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].i, a[7].i, a[8].i, a[9].i, a[10].p, a[11].i,
        a[12].p, a[13].p, a[14].p, a[15].p);
    END
}

static PyObject *f_verify(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_VERIFY)
    rc = ((int (*)(P, I, I, I, P, P, P, P, P, P, P, P, P, P))
          g_fn[F_VERIFY])(
        a[0].p, a[1].i, a[2].i, a[3].i, a[4].p, a[5].p, a[6].p, a[7].p, a[8].p, a[9].p, a[10].p, a[11].p,
        a[12].p, a[13].p);
    END
}

static PyObject *f_reserve(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_RESERVE)
    rc = ((int (*)(P, I, I, P, I, P, P, P, I, P, P, P, P, P, P, P))g_fn[F_RESERVE])(
        a[0].p, a[1].i, a[2].i, a[3].p, a[4].i, a[5].p, a[6].p, a[7].p, a[8].i, a[9].p, a[10].p, a[11].p, a[12].p,
        a[13].p, a[14].p, a[15].p);
    END
}

static PyObject *f_bounds(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_BOUNDS)
    rc = ((int (*)(P, I, P, P, P, I, P, P, P, P))g_fn[F_BOUNDS])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].p, a[5].i, a[6].p, a[7].p, a[8].p, a[9].p);
    END
}

static PyObject *f_pick(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_PICK)
    rc = ((int (*)(P, I, P, P, I, P, P, int64_t, P, P, I, I, I, I, P, P, int64_t, P))g_fn[F_PICK])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].p, a[7].l, a[8].p, a[9].p, a[10].i, a[11].i, a[12].i,
        a[13].i, a[14].p, a[15].p, a[16].l, a[17].p);
    END
}

static PyObject *f_picked(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    BEGIN(F_PICKED)
    rc = ((int (*)(P, I, P, P, I, P, P, int64_t, P, P, P, I, float, P, P, int64_t, P))g_fn[F_PICKED])(
        a[0].p, a[1].i, a[2].p, a[3].p, a[4].i, a[5].p, a[6].p, a[7].l, a[8].p, a[9].p, a[10].p, a[11].i, a[12].f,
        a[13].p, a[14].p, a[15].l, a[16].p);
    END
}

/* bytes of a workspace from a handle, a batch, its offsets and three sizes, or -status */
static PyObject *bytes_of(int which, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return NULL;
    }
    Held h;
    h.nbuf = h.nobj = 0;
    const int32_t *off;
    uint64_t hd, batch, x[3] = {0, 0, 0};
    int bad = as_bits(args[0], 'h', &hd) || as_bits(args[1], 'i', &batch) || as_host_i32(args[2], &h, &off, NULL);
    for (int k = 0; k < 3 && !bad; ++k) bad = as_bits(args[3 + k], 'i', &x[k]);
    if (bad) {
        release(&h);
        return NULL;
    }
    int64_t bytes = 0;
    const I b = (I)(uint32_t)batch, x0 = (I)(uint32_t)x[0], x1 = (I)(uint32_t)x[1], x2 = (I)(uint32_t)x[2];
    const P handle = (P)(uintptr_t)hd;
    const int rc = ((int (*)(P, I, const int32_t *, I, I, I, int64_t *))g_fn[which])(handle, b, off, x0, x1, x2, &bytes);
    release(&h);
    return PyLong_FromLongLong(rc ? -(long long)rc : (long long)bytes);
}

/* pick_bytes(handle, batch, q_offsets_h, max_len, page_size, budget) */
static PyObject *f_pick_bytes(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    return bytes_of(F_PICK_SPACE, args, n);
}

/* picked_bytes(handle, batch, q_offsets_h, page_size, table_width, budget) */
static PyObject *f_picked_bytes(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    return bytes_of(F_PICKED_SPACE, args, n);
}

/* attend_bytes(handle, batch, q_offsets_h, max_len, weights): bytes of an attention call's workspace, or -status */
static PyObject *f_attend_bytes(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "attend_bytes takes five arguments");
        return NULL;
    }
    Held h;
    h.nbuf = h.nobj = 0;
    const int32_t *off;
    uint64_t hd, batch, len, weights;
    if (as_bits(args[0], 'h', &hd) || as_bits(args[1], 'i', &batch) || as_host_i32(args[2], &h, &off, NULL) ||
        as_bits(args[3], 'i', &len) || as_bits(args[4], 'i', &weights)) {
        release(&h);
        return NULL;
    }
    int64_t bytes = 0;
    const int rc = ((int (*)(P, I, const int32_t *, I, I, int64_t *))g_fn[F_SPACE])(
        (P)(uintptr_t)hd, (I)(uint32_t)batch, off, (I)(uint32_t)len, (I)(uint32_t)weights, &bytes);
    release(&h);
    return PyLong_FromLongLong(rc ? -(long long)rc : (long long)bytes);
}

/* fits(tensor, dtype, device index, sizes...): whether it is a contiguous tensor of this type on this CUDA device with
 * these sizes (-1: any). Written out in Python the checks of a call's tensors took half of its time. */
static PyObject *g_dtype, *g_get_device, *g_shape, *g_is_contiguous;
static int tensor_fits(PyObject *t, PyObject *dtype, PyObject *device, PyObject *const *sizes, Py_ssize_t n)
{
    int ok = 0;
    PyObject *r = PyObject_GetAttr(t, g_dtype);
    if (!r) goto other;
    ok = r == dtype;
    Py_DECREF(r);
    if (!ok) return 0;
    ok = 0;
    r = PyObject_CallMethodNoArgs(t, g_get_device);
    if (!r) goto other;
    ok = PyLong_Check(r) && PyLong_Check(device) && PyLong_AsLong(r) == PyLong_AsLong(device);
    Py_DECREF(r);
    if (!ok) return 0;
    ok = 0;
    r = PyObject_GetAttr(t, g_shape);
    if (!r) goto other;
    if (PyTuple_Check(r) && PyTuple_GET_SIZE(r) == n) {
        ok = 1;
        for (Py_ssize_t k = 0; k < n && ok; ++k) {
            const long long want = PyLong_AsLongLong(sizes[k]);
            ok = want < 0 || PyLong_AsLongLong(PyTuple_GET_ITEM(r, k)) == want;
        }
    }
    Py_DECREF(r);
    if (PyErr_Occurred()) goto other;
    if (!ok) return 0;
    r = PyObject_CallMethodNoArgs(t, g_is_contiguous);
    if (!r) goto other;
    ok = r == Py_True;
    Py_DECREF(r);
    return ok;
other: /* no tensor: the caller says what is wrong */
    PyErr_Clear();
    return 0;
}
static PyObject *f_fits(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n < 3) {
        PyErr_SetString(PyExc_TypeError, "fits takes a tensor, a type, a device and sizes");
        return NULL;
    }
    return PyBool_FromLong(tensor_fits(args[0], args[1], args[2], args + 3, n - 3));
}

/* all_fit(device index, dtype, (tensor, number of sizes, sizes...)...): whether every tensor fits; a decoding step's calls
 * check four to six */
static PyObject *f_all_fit(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    int ok = n >= 2;
    for (Py_ssize_t k = 2; k < n && ok;) {
        const Py_ssize_t sizes = k + 1 < n && PyLong_Check(args[k + 1]) ? PyLong_AsSsize_t(args[k + 1]) : -1;
        if (sizes < 0 || k + 2 + sizes > n) {
            PyErr_SetString(PyExc_TypeError, "all_fit takes a device, a type, and tensors with their numbers of sizes");
            return NULL;
        }
        ok = tensor_fits(args[k], args[1], args[0], args + k + 2, sizes);
        k += 2 + sizes;
    }
    return PyBool_FromLong(ok);
}

/* row_stride(tensor, dtype, device index, heads, d): elements from a row to the next of [rows, heads, d] rows whose heads
 * and channels lie side by side, on this CUDA device; -1 for anything else */
static PyObject *g_stride;
static PyObject *f_row_stride(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "row_stride takes five arguments");
        return NULL;
    }
    long long stride = -1;
    PyObject *t = args[0], *shape = NULL, *strides = NULL, *r = PyObject_GetAttr(t, g_dtype);
    if (!r) goto done;
    Py_DECREF(r);
    if (r != args[1]) goto done;
    r = PyObject_CallMethodNoArgs(t, g_get_device);
    if (!r) goto done;
    const int here = PyLong_Check(r) && PyLong_AsLong(r) == PyLong_AsLong(args[2]);
    Py_DECREF(r);
    if (!here) goto done;
    shape = PyObject_GetAttr(t, g_shape);
    strides = shape ? PyObject_CallMethodNoArgs(t, g_stride) : NULL;
    if (strides && PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 3 && PyTuple_Check(strides) &&
        PyTuple_GET_SIZE(strides) == 3) {
        long long v[6];
        for (int k = 0; k < 3; ++k) {
            v[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, k));
            v[3 + k] = PyLong_AsLongLong(PyTuple_GET_ITEM(strides, k));
        }
        const long long heads = PyLong_AsLongLong(args[3]), d = PyLong_AsLongLong(args[4]);
        if (v[1] == heads && v[2] == d && (v[0] == 0 || (v[5] == 1 && (heads == 1 || v[4] == d))))
            stride = v[0] > 1 ? v[3] : heads * d; /* (of no rows any stride will do) */
    }
done:
    Py_XDECREF(shape);
    Py_XDECREF(strides);
    if (PyErr_Occurred()) { /* no tensor: the caller says what is wrong */
        PyErr_Clear();
        stride = -1;
    }
    return PyLong_FromLongLong(stride);
}

/* compact(handle, total_kept, kept_idx, src_rows, srcs, dsts, row_bytes, stream): the three are lists */
static PyObject *f_compact(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 8 || !PyList_Check(args[4]) || !PyList_Check(args[5]) || !PyList_Check(args[6])) {
        PyErr_SetString(PyExc_TypeError, "compact takes eight arguments, three of them lists");
        return NULL;
    }
    const Py_ssize_t t = PyList_GET_SIZE(args[4]);
    if (t > 8 || PyList_GET_SIZE(args[5]) < t || PyList_GET_SIZE(args[6]) < t) {
        PyErr_SetString(PyExc_ValueError, "one destination and row size per source, at most 8");
        return NULL;
    }
    Held h;
    h.nbuf = h.nobj = 0;
    void *kept, *src[8], *dst[8];
    uint64_t hd, stream, total, rows, size;
    int64_t rb[8];
    int bad = as_bits(args[0], 'h', &hd) || as_bits(args[1], 'l', &total) || as_ptr(args[2], &h, &kept) ||
              as_bits(args[3], 'l', &rows) || as_bits(args[7], 'h', &stream);
    for (Py_ssize_t k = 0; k < t && !bad; ++k) {
        bad = as_ptr(PyList_GET_ITEM(args[4], k), &h, &src[k]) || as_ptr(PyList_GET_ITEM(args[5], k), &h, &dst[k]) ||
              as_bits(PyList_GET_ITEM(args[6], k), 'l', &size);
        if (!bad) rb[k] = (int64_t)size;
    }
    if (bad) {
        release(&h);
        return NULL;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(P, int64_t, P, int64_t, I, P, P, P, P))g_fn[F_COMPACT])(
        (P)(uintptr_t)hd, (int64_t)total, kept, (int64_t)rows, (I)t, src, dst, rb, (P)(uintptr_t)stream);
    Py_END_ALLOW_THREADS
    release(&h);
    return PyLong_FromLong(rc);
}

/* keep_total(seq_offsets_h, keep_k_h or None, keep_ratio): the batch's kept tokens, or -status */
static PyObject *f_keep_total(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "keep_total takes three arguments");
        return NULL;
    }
    Held h;
    h.nbuf = h.nobj = 0;
    const int32_t *so, *kk;
    Py_ssize_t len = 0;
    double ratio;
    if (as_double(args[2], &ratio) != 0 || as_host_i32(args[0], &h, &so, &len) != 0 ||
        as_host_i32(args[1], &h, &kk, NULL) != 0) {
        release(&h);
        return NULL;
    }
    int32_t small[65];
    int32_t *off = len <= 65 ? small : (int32_t *)PyMem_Malloc(sizeof(int32_t) * (size_t)len);
    if (!off) {
        release(&h);
        return PyErr_NoMemory();
    }
    const int rc = ((int (*)(I, const int32_t *, const int32_t *, float, int32_t *))g_fn[F_KEEP])((I)(len - 1), so, kk,
                                                                                             (float)ratio, off);
    const long total = rc ? -(long)rc : (long)off[len - 1];
    if (off != small) PyMem_Free(off);
    release(&h);
    return PyLong_FromLong(total);
}

/* bind({name: address}, host_i32, numpy.ndarray, ctypes_value) */
static PyObject *f_bind(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 4 || !PyDict_Check(args[0]) || !PyCallable_Check(args[1]) || !PyType_Check(args[2]) ||
        !PyCallable_Check(args[3])) {
        PyErr_SetString(PyExc_TypeError, "bind takes a dict of addresses, a callable, a type and a callable");
        return NULL;
    }
    for (int k = 0; k < F_COUNT; ++k) {
        PyObject *v = PyDict_GetItemString(args[0], kNames[k]);
        if (!v && k > F_KEEP && g_fn[k]) continue; /* these keep the address of an earlier bind */
        if (!v) {
            PyErr_Format(PyExc_KeyError, "%s", kNames[k]);
            return NULL;
        }
        g_fn[k] = PyLong_AsVoidPtr(v);
        if (PyErr_Occurred()) return NULL;
    }
    Py_INCREF(args[1]);
    Py_XSETREF(g_host_i32, args[1]);
    Py_INCREF(args[2]);
    Py_XSETREF(g_ndarray, args[2]);
    Py_INCREF(args[3]);
    Py_XSETREF(g_ctypes_value, args[3]);
    Py_RETURN_NONE;
}

#define DEF(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, NULL}
static PyMethodDef kMethods[] = {DEF("bind", f_bind), DEF("score", f_score), DEF("score_full_keys", f_full),
                                 DEF("score_topk", f_score_topk), DEF("topk", f_topk), DEF("compact", f_compact),
                                 DEF("splice", f_splice), DEF("project", f_project),
                                 DEF("keep_total", f_keep_total), DEF("cache_append", f_append),
                                 DEF("cache_append_granted", f_append_granted),
                                 DEF("cache_attend", f_attend), DEF("attend_bytes", f_attend_bytes),
                                 DEF("cache_evict", f_evict), DEF("verify", f_verify),
                                 DEF("cache_reserve", f_reserve), DEF("cache_bounds", f_bounds),
                                 DEF("pick_bytes", f_pick_bytes), DEF("cache_pick", f_pick),
                                 DEF("picked_bytes", f_picked_bytes), DEF("cache_attend_picked", f_picked),
                                 DEF("fits", f_fits), DEF("all_fit", f_all_fit), DEF("row_stride", f_row_stride), {NULL, NULL, 0, NULL}};
static struct PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, kMethods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void)
{
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_dtype = PyUnicode_InternFromString("dtype");
    g_get_device = PyUnicode_InternFromString("get_device");
    g_shape = PyUnicode_InternFromString("shape");
    g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    g_stride = PyUnicode_InternFromString("stride");
    return g_data_ptr && g_stride && g_dtype && g_get_device && g_shape && g_is_contiguous ? PyModule_Create(&kModule) : NULL;
}
