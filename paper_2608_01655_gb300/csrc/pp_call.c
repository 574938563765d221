/*
 * The calls of the paged cache for Python: argument conversion and tensor checks that a
 * serving step makes many times, at a fraction of what they cost through ctypes (2.0 to
 * 2.5 us a call with 20 to 30 arguments, 0.4 to 0.5 us a tensor, on the GPU's host).
 * The functions are libprefixplace's own, bound by address; the binding has the same
 * checks in Python and calls through ctypes where this module has not been built.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "prefixplace.h"

typedef union {
    int32_t i;
    int64_t l;
    size_t z;
    float f;
    void *p;
} slot_t;

#define MOST 32

static PyObject *s_value, *s_dtype, *s_shape, *s_get_device, *s_stride, *s_data_ptr, *s_is_contiguous;

/* i int32, l int64, z size_t, f float, p pointer: None, a number or a ctypes pointer */
static int convert(const char *types, PyObject *const *args, Py_ssize_t n, slot_t *v)
{
    Py_ssize_t k;
    for (k = 0; types[k]; ++k) {
        PyObject *x;
        if (k >= n) break;
        x = args[k];
        switch (types[k]) {
        case 'f':
            v[k].f = (float)PyFloat_AsDouble(x);
            break;
        case 'i': {
            const long y = PyLong_AsLong(x);
            if (y < INT32_MIN || y > INT32_MAX) {
                if (!PyErr_Occurred()) PyErr_Format(PyExc_OverflowError, "argument %zd does not fit in 32 bits", k);
                return -1;
            }
            v[k].i = (int32_t)y;
            break;
        }
        case 'l':
            v[k].l = PyLong_AsLongLong(x);
            break;
        case 'z':
            v[k].z = PyLong_AsSize_t(x);
            break;
        default:
            if (x == Py_None) {
                v[k].p = NULL;
            } else if (PyLong_Check(x)) {
                v[k].p = PyLong_AsVoidPtr(x);
            } else {
                PyObject *y = PyObject_GetAttr(x, s_value);
                if (!y) return -1;
                v[k].p = y == Py_None ? NULL : PyLong_AsVoidPtr(y);
                Py_DECREF(y);
            }
        }
        if (PyErr_Occurred()) return -1;
    }
    if (types[k] || k != n) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", (Py_ssize_t)strlen(types), n);
        return -1;
    }
    return 0;
}

#define ENTRY(NAME, TYPES, ...)                                                                   \
    static __typeof__(&NAME) f_##NAME;                                                            \
    static const char t_##NAME[] = TYPES;                                                         \
    static PyObject *c_##NAME(PyObject *self, PyObject *const *args, Py_ssize_t n)                \
    {                                                                                             \
        slot_t v[MOST];                                                                           \
        pp_status s;                                                                              \
        (void)self;                                                                               \
        if (!f_##NAME) {                                                                          \
            PyErr_SetString(PyExc_RuntimeError, #NAME " is not bound");                           \
            return NULL;                                                                          \
        }                                                                                         \
        if (convert(t_##NAME, args, n, v) < 0) return NULL;                                       \
        Py_BEGIN_ALLOW_THREADS                                                                    \
        s = f_##NAME(__VA_ARGS__);                                                                \
        Py_END_ALLOW_THREADS                                                                      \
        return PyLong_FromLong((long)s);                                                          \
    }

ENTRY(pp_block_tables, "pipppipipppipipppp", v[0].p, v[1].i, v[2].p, v[3].p, v[4].p, v[5].i, v[6].p, v[7].i, v[8].p, v[9].p,
      v[10].p, v[11].i, v[12].p, v[13].i, v[14].p, v[15].p, v[16].p, v[17].p)
ENTRY(pp_kv_write, "pipllpllpppp", v[0].p, v[1].i, v[2].p, v[3].l, v[4].l, v[5].p, v[6].l, v[7].l, v[8].p, v[9].p, v[10].p, v[11].p)
ENTRY(pp_paged_attention, "piiipllppipppiifpllpp", v[0].p, v[1].i, v[2].i, v[3].i, v[4].p, v[5].l, v[6].l, v[7].p, v[8].p, v[9].i,
      v[10].p, v[11].p, v[12].p, v[13].i, v[14].i, v[15].f, v[16].p, v[17].l, v[18].l, v[19].p, v[20].p)
ENTRY(pp_kv_rotate, "piipllpllppfpiipfpllpllpllpppp", v[0].p, v[1].i, v[2].i, v[3].p, v[4].l, v[5].l, v[6].p, v[7].l, v[8].l, v[9].p,
      v[10].p, v[11].f, v[12].p, v[13].i, v[14].i, v[15].p, v[16].f, v[17].p, v[18].l, v[19].l, v[20].p, v[21].l, v[22].l, v[23].p,
      v[24].l, v[25].l, v[26].p, v[27].p, v[28].p, v[29].p)
ENTRY(pp_kv_write8, "pipllpllpppppp", v[0].p, v[1].i, v[2].p, v[3].l, v[4].l, v[5].p, v[6].l, v[7].l, v[8].p, v[9].p, v[10].p, v[11].p,
      v[12].p, v[13].p)
ENTRY(pp_paged_attention8, "piiipllppppipppiifpllppzp", v[0].p, v[1].i, v[2].i, v[3].i, v[4].p, v[5].l, v[6].l, v[7].p, v[8].p, v[9].p,
      v[10].p, v[11].i, v[12].p, v[13].p, v[14].p, v[15].i, v[16].i, v[17].f, v[18].p, v[19].l, v[20].l, v[21].p, v[22].p, v[23].z,
      v[24].p)

/* bind(name, types, address): types have to be those that this file was written for */
static PyObject *bind(PyObject *self, PyObject *args)
{
    const char *name, *types;
    PyObject *address;
    void *p;
    (void)self;
    if (!PyArg_ParseTuple(args, "ssO", &name, &types, &address)) return NULL;
    p = PyLong_AsVoidPtr(address);
    if (PyErr_Occurred()) return NULL;
#define BIND(NAME)                                                                               \
    if (!strcmp(name, #NAME)) {                                                                   \
        if (strcmp(types, t_##NAME)) return PyErr_Format(PyExc_TypeError, "%s takes %s", name, t_##NAME); \
        f_##NAME = (__typeof__(&NAME))p;                                                          \
        Py_RETURN_NONE;                                                                           \
    }
    BIND(pp_block_tables)
    BIND(pp_kv_write)
    BIND(pp_paged_attention)
    BIND(pp_kv_rotate)
    BIND(pp_kv_write8)
    BIND(pp_paged_attention8)
    return PyErr_Format(PyExc_ValueError, "no call %s", name);
}

/* ---------------------------------------------------------------------------
 * Tensors.  Each check gives None where the tensor is another than asked for.
 * ------------------------------------------------------------------------- */
static int has_type(PyObject *t, PyObject *dtype)
{
    PyObject *x = PyObject_GetAttr(t, s_dtype);
    if (!x) return -1;
    Py_DECREF(x);
    return x == dtype;
}
static int on_device(PyObject *t, long device)
{
    PyObject *x = PyObject_CallMethodNoArgs(t, s_get_device);
    long d;
    if (!x) return -1;
    d = PyLong_AsLong(x);
    Py_DECREF(x);
    return PyErr_Occurred() ? -1 : d == device;
}
static int has_shape(PyObject *t, PyObject *shape)
{
    PyObject *x = PyObject_GetAttr(t, s_shape);
    int same;
    if (!x) return -1;
    same = PyObject_RichCompareBool(x, shape, Py_EQ);
    Py_DECREF(x);
    return same;
}
static PyObject *strides_of(PyObject *t, Py_ssize_t n)
{
    PyObject *x = PyObject_CallMethodNoArgs(t, s_stride);
    if (x && (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != n)) {
        Py_DECREF(x);
        PyErr_SetString(PyExc_TypeError, "stride() of a tensor is a tuple");
        return NULL;
    }
    return x;
}

/* contiguous(t, dtype, shape, device) -> pointer */
static PyObject *contiguous(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int ok;
    (void)self;
    if (n != 4) return PyErr_Format(PyExc_TypeError, "contiguous: 4 arguments");
    ok = has_type(a[0], a[1]);
    if (ok > 0) ok = has_shape(a[0], a[2]);
    if (ok > 0) ok = on_device(a[0], PyLong_AsLong(a[3]));
    if (ok > 0) {
        PyObject *x = PyObject_CallMethodNoArgs(a[0], s_is_contiguous);
        if (!x) return NULL;
        ok = PyObject_IsTrue(x);
        Py_DECREF(x);
    }
    if (ok < 0 || PyErr_Occurred()) return NULL;
    if (!ok) Py_RETURN_NONE;
    return PyObject_CallMethodNoArgs(a[0], s_data_ptr);
}

/* cache(t, dtype, shape, strides, device) -> pointer; an extent of 1 has no stride */
static PyObject *cache(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int ok, k;
    (void)self;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "cache: 5 arguments");
    ok = has_type(a[0], a[1]);
    if (ok > 0) ok = has_shape(a[0], a[2]);
    if (ok > 0) ok = on_device(a[0], PyLong_AsLong(a[4]));
    if (ok > 0) {
        PyObject *st = strides_of(a[0], 4);
        if (!st) return NULL;
        ok = PyLong_AsLong(PyTuple_GET_ITEM(st, 3)) == 1;
        for (k = 0; ok && k < 3; ++k)
            if (PyLong_AsLongLong(PyTuple_GET_ITEM(a[2], k)) != 1)
                ok = PyLong_AsLongLong(PyTuple_GET_ITEM(st, k)) == PyLong_AsLongLong(PyTuple_GET_ITEM(a[3], k));
        Py_DECREF(st);
    }
    if (ok < 0 || PyErr_Occurred()) return NULL;
    if (!ok) Py_RETURN_NONE;
    return PyObject_CallMethodNoArgs(a[0], s_data_ptr);
}

/* rows(t, dtype, tokens, heads, dim, device) -> pointer, token stride, head stride of [tokens][heads][dim] */
static PyObject *rows(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int ok;
    long long tokens, heads, dim, ht, tt;
    PyObject *shape, *st, *p;
    (void)self;
    if (n != 6) return PyErr_Format(PyExc_TypeError, "rows: 6 arguments");
    tokens = PyLong_AsLongLong(a[2]);
    heads = PyLong_AsLongLong(a[3]);
    dim = PyLong_AsLongLong(a[4]);
    ok = has_type(a[0], a[1]);
    if (ok > 0) {
        shape = PyObject_GetAttr(a[0], s_shape);
        if (!shape) return NULL;
        ok = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 3 && PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)) == tokens &&
             PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 1)) == heads && PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 2)) == dim;
        Py_DECREF(shape);
    }
    if (ok > 0) ok = on_device(a[0], PyLong_AsLong(a[5]));
    if (ok < 0 || PyErr_Occurred()) return NULL;
    if (!ok) Py_RETURN_NONE;
    st = strides_of(a[0], 3);
    if (!st) return NULL;
    /* an extent of 1 may carry any stride */
    ht = heads > 1 ? PyLong_AsLongLong(PyTuple_GET_ITEM(st, 1)) : dim;
    tt = tokens > 1 ? PyLong_AsLongLong(PyTuple_GET_ITEM(st, 0)) : heads * ht;
    ok = !tokens || PyLong_AsLongLong(PyTuple_GET_ITEM(st, 2)) == 1;
    Py_DECREF(st);
    if (PyErr_Occurred()) return NULL;
    if (!ok) Py_RETURN_NONE;
    p = PyObject_CallMethodNoArgs(a[0], s_data_ptr);
    return p ? Py_BuildValue("NLL", p, tt, ht) : NULL;
}

#define METHOD(NAME) {#NAME, (PyCFunction)(void (*)(void))c_##NAME, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    METHOD(pp_block_tables), METHOD(pp_kv_write),  METHOD(pp_paged_attention),
    METHOD(pp_kv_rotate),    METHOD(pp_kv_write8), METHOD(pp_paged_attention8),
    {"bind", bind, METH_VARARGS, NULL},
    {"contiguous", (PyCFunction)(void (*)(void))contiguous, METH_FASTCALL, NULL},
    {"cache", (PyCFunction)(void (*)(void))cache, METH_FASTCALL, NULL},
    {"rows", (PyCFunction)(void (*)(void))rows, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pp_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pp_call(void)
{
    s_value = PyUnicode_InternFromString("value");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_shape = PyUnicode_InternFromString("shape");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    if (!s_value || !s_dtype || !s_shape || !s_get_device || !s_stride || !s_data_ptr || !s_is_contiguous) return NULL;
    return PyModule_Create(&module);
}
