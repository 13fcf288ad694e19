/* The marshalling of the entry points that a decoder calls for every token (aircache_decode_attn and aircache_decode_step,
 * aircache_rotate, and aircache_append_quantized and aircache_decode_attn_quantized over the cache of 8 bits; with them
 * aircache_prompt_attn, for short prompts), natively: a kernel of theirs may take 2 to 5 us, and through ctypes the
 * arguments alone took 2.4 and 3.1 us of host time for the first two; here 0.6 and 0.8.  Same arguments, same function in
 * libaircache.so, same return code. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *s_shape, *s_ragged, *s_tokens, *s_rotary, *s_prompt, *s_quantized;   /* the binding's structure types */
static PyObject *s_get_device, *s_get_stream;    /* torch's current device and its current stream's raw handle */
static PyObject *s_int32, *s_int64, *s_float32, *s_bfloat16;   /* torch's types */
static PyObject *s_data_ptr, *s_numel, *s_element_size, *s_dtype, *s_is_contiguous;

static int struct_address(PyObject *o, PyObject *type, int64_t *w) {
    if (!PyObject_TypeCheck(o, (PyTypeObject *)type)) {
        PyErr_Format(PyExc_TypeError, "expected %s, got %s", ((PyTypeObject *)type)->tp_name, Py_TYPE(o)->tp_name);
        return -1;
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE)) return -1;
    *w = (int64_t)(intptr_t)view.buf;
    PyBuffer_Release(&view);   /* the caller's reference keeps the structure */
    return 0;
}

static int struct_or_null(PyObject *o, PyObject *type, int64_t *w) {
    if (o == Py_None) { *w = 0; return 0; }
    return struct_address(o, type, w);
}

static int as_int(PyObject *o, int64_t *w) {
    *w = (int64_t)PyLong_AsUnsignedLongLongMask(o);
    return *w == -1 && PyErr_Occurred() ? -1 : 0;
}

/* None, an address, or an object with data_ptr() */
static int address(PyObject *o, int64_t *w) {
    if (o == Py_None) { *w = 0; return 0; }
    if (PyLong_Check(o)) return as_int(o, w);
    PyObject *r = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!r) return -1;
    const int rc = as_int(r, w);
    Py_DECREF(r);
    return rc;
}

/* The same for a table of one type: a tensor of another one is a TypeError (torch makes 64-bit integers where it is not told
 * otherwise, and 32-bit positions read from them turn heads by wrong angles).  With `whole` also one with gaps, for tables that
 * programs cut out of larger ones.  (4 tokens of rotary positions, a call among others: 3.6 us without a look, 3.9 with these,
 * 4.1 with a look for gaps in all five tables.) */
static int table(PyObject *o, PyObject *dtype, int whole, int64_t *w) {
    if (o == Py_None || PyLong_Check(o)) return address(o, w);
    PyObject *r = PyObject_GetAttr(o, s_dtype);
    if (!r) {   /* no tensor */
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return -1;
        PyErr_Clear();
        return address(o, w);
    }
    Py_DECREF(r);   /* (torch keeps its types) */
    int fits = r == dtype;
    if (fits && whole) {
        if (!(r = PyObject_CallMethodNoArgs(o, s_is_contiguous))) return -1;
        Py_DECREF(r);
        fits = r == Py_True;
    }
    if (fits) return address(o, w);
    PyErr_SetString(PyExc_TypeError, "a table of another type, or with gaps");
    return -1;
}

/* numel() * element_size(); 0 for None and a raw address */
static int size_of(PyObject *o, int64_t *w) {
    *w = 0;
    if (o == Py_None || PyLong_Check(o)) return 0;
    int64_t n = 0, e = 0;
    PyObject *r = PyObject_CallMethodNoArgs(o, s_numel);
    if (!r || as_int(r, &n)) { Py_XDECREF(r); return -1; }
    Py_DECREF(r);
    r = PyObject_CallMethodNoArgs(o, s_element_size);
    if (!r || as_int(r, &e)) { Py_XDECREF(r); return -1; }
    Py_DECREF(r);
    *w = n * e;
    return 0;
}

/* None (torch's current stream), a raw handle, or an object with cuda_stream */
static int stream_handle(PyObject *o, int64_t *w) {
    PyObject *r;
    if (o == Py_None) {
        PyObject *d = PyObject_CallNoArgs(s_get_device);
        if (!d) return -1;
        r = PyObject_CallOneArg(s_get_stream, d);
        Py_DECREF(d);
    } else if (PyLong_Check(o)) {
        return as_int(o, w);
    } else {
        r = PyObject_GetAttrString(o, "cuda_stream");
    }
    if (!r) return -1;
    const int rc = as_int(r, w);
    Py_DECREF(r);
    return rc;
}

static int tail(PyObject *workspace, PyObject *stream, int64_t *w) {
    return address(workspace, w) || size_of(workspace, w + 1) || stream_handle(stream, w + 2) ? -1 : 0;
}

/* decode_attn(function address, shape, cache, q, out, workspace, stream) */
static PyObject *decode_attn(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[7];
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "decode_attn takes 7 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_shape, &w[0]) || struct_address(a[2], s_ragged, &w[1]) ||
        address(a[3], &w[2]) || address(a[4], &w[3]) || tail(a[5], a[6], &w[4]))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, const void *, const void *, float *, void *, int64_t, void *))(intptr_t)f)(
        (const void *)w[0], (const void *)w[1], (const void *)w[2], (float *)w[3], (void *)w[4], w[5], (void *)w[6]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* decode_step(function address, shape, cache, q, k_new, v_new, appended, out, workspace, stream) */
static PyObject *decode_step(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[10];
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "decode_step takes 10 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_shape, &w[0]) || struct_address(a[2], s_ragged, &w[1]) ||
        address(a[3], &w[2]) || address(a[4], &w[3]) || address(a[5], &w[4]) || as_int(a[6], &w[5]) ||
        address(a[7], &w[6]) || tail(a[8], a[9], &w[7]))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, void *, const void *, const void *, const void *, int32_t, float *, void *, int64_t,
                   void *))(intptr_t)f)((const void *)w[0], (void *)w[1], (const void *)w[2], (const void *)w[3],
                                        (const void *)w[4], (int32_t)w[5], (float *)w[6], (void *)w[7], w[8],
                                        (void *)w[9]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* decode_attn_quantized(function address, shape, cache, q, out, workspace, stream) */
static PyObject *decode_attn_quantized(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[7];
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "decode_attn_quantized takes 7 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_shape, &w[0]) || struct_address(a[2], s_quantized, &w[1]) ||
        address(a[3], &w[2]) || address(a[4], &w[3]) || tail(a[5], a[6], &w[4]))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, const void *, const void *, float *, void *, int64_t, void *))(intptr_t)f)(
        (const void *)w[0], (const void *)w[1], (const void *)w[2], (float *)w[3], (void *)w[4], w[5], (void *)w[6]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* append_quantized(function address, shape, cache, k_new, v_new, appended, stream) */
static PyObject *append_quantized(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[6];
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "append_quantized takes 7 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_shape, &w[0]) || struct_address(a[2], s_quantized, &w[1]) ||
        address(a[3], &w[2]) || address(a[4], &w[3]) || as_int(a[5], &w[4]) || stream_handle(a[6], &w[5]))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, void *, const void *, const void *, int32_t, void *))(intptr_t)f)(
        (const void *)w[0], (void *)w[1], (const void *)w[2], (const void *)w[3], (int32_t)w[4], (void *)w[5]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* rotate(function address, spec, q, k, v, positions, inv_freq, q_weight, k_weight, q_out, k_out, v_out, rows, n_rows, stream) */
static PyObject *rotate(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[14];
    if (n != 15) { PyErr_SetString(PyExc_TypeError, "rotate takes 15 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_rotary, &w[0])) return NULL;
    for (int i = 1; i < 4; ++i)
        if (struct_or_null(a[1 + i], s_tokens, &w[i]) || struct_or_null(a[8 + i], s_tokens, &w[7 + i])) return NULL;
    if (table(a[5], s_int32, 1, &w[4]) || table(a[6], s_float32, 0, &w[5]) || table(a[7], s_bfloat16, 0, &w[6]) ||
        table(a[8], s_bfloat16, 0, &w[7]))
        return NULL;
    if (table(a[12], s_int64, 1, &w[11]) || as_int(a[13], &w[12]) || stream_handle(a[14], &w[13])) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, const void *, const void *, const void *, const void *, const void *, const void *,
                   const void *, const void *, const void *, const void *, const void *, int64_t, void *))(intptr_t)f)(
        (const void *)w[0], (const void *)w[1], (const void *)w[2], (const void *)w[3], (const void *)w[4],
        (const void *)w[5], (const void *)w[6], (const void *)w[7], (const void *)w[8], (const void *)w[9],
        (const void *)w[10], (const void *)w[11], w[12], (void *)w[13]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* prompt_attn(function address, spec, q, k, v, q_offsets, k_offsets, out, stream) */
static PyObject *prompt_attn(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    int64_t f, w[8];
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "prompt_attn takes 9 arguments"); return NULL; }
    if (as_int(a[0], &f) || struct_address(a[1], s_prompt, &w[0]) || struct_or_null(a[2], s_tokens, &w[1]) ||
        struct_or_null(a[3], s_tokens, &w[2]) || struct_or_null(a[4], s_tokens, &w[3]) ||
        table(a[5], s_int32, 1, &w[4]) || table(a[6], s_int32, 1, &w[5]) || struct_or_null(a[7], s_tokens, &w[6]) || stream_handle(a[8], &w[7]))
        return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((int (*)(const void *, const void *, const void *, const void *, const void *, const void *, const void *,
                   void *))(intptr_t)f)((const void *)w[0], (const void *)w[1], (const void *)w[2], (const void *)w[3],
                                        (const void *)w[4], (const void *)w[5], (const void *)w[6], (void *)w[7]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* setup(Shape, Ragged, get_device, get_raw_stream[, Tokens, Rotary, Prompt, Quantized, int32, int64, float32, bfloat16]), once;
 * without the last eight, only decode_attn and decode_step may be called */
static PyObject *setup(PyObject *self, PyObject *args) {
    (void)self;
    PyObject *dev, *stream, *t[6] = {NULL, NULL, NULL, NULL, NULL, NULL}, *d[4] = {NULL, NULL, NULL, NULL};
    if (!PyArg_ParseTuple(args, "O!O!OO|O!O!O!O!OOOO", &PyType_Type, &t[0], &PyType_Type, &t[1], &dev, &stream, &PyType_Type,
                          &t[2], &PyType_Type, &t[3], &PyType_Type, &t[4], &PyType_Type, &t[5], &d[0], &d[1], &d[2], &d[3]))
        return NULL;
    Py_INCREF(dev); Py_INCREF(stream);
    for (int i = 0; i < 6; ++i) {
        if (!t[i]) t[i] = (PyObject *)&PyType_Type;   /* no structure is of this type: a TypeError */
        Py_INCREF(t[i]);
    }
    for (int i = 0; i < 4; ++i) Py_XINCREF(d[i]);
    s_get_device = dev; s_get_stream = stream;
    s_shape = t[0]; s_ragged = t[1]; s_tokens = t[2]; s_rotary = t[3]; s_prompt = t[4]; s_quantized = t[5];
    s_int32 = d[0]; s_int64 = d[1]; s_float32 = d[2]; s_bfloat16 = d[3];
    Py_RETURN_NONE;
}

static PyMethodDef s_methods[] = {
    {"setup", setup, METH_VARARGS, NULL},
    {"decode_attn", (PyCFunction)(void (*)(void))decode_attn, METH_FASTCALL, NULL},
    {"decode_step", (PyCFunction)(void (*)(void))decode_step, METH_FASTCALL, NULL},
    {"decode_attn_quantized", (PyCFunction)(void (*)(void))decode_attn_quantized, METH_FASTCALL, NULL},
    {"append_quantized", (PyCFunction)(void (*)(void))append_quantized, METH_FASTCALL, NULL},
    {"rotate", (PyCFunction)(void (*)(void))rotate, METH_FASTCALL, NULL},
    {"prompt_attn", (PyCFunction)(void (*)(void))prompt_attn, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef s_module = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, s_methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_element_size = PyUnicode_InternFromString("element_size");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    if (!s_data_ptr || !s_numel || !s_element_size || !s_dtype || !s_is_contiguous) return NULL;
    PyObject *const tables = PyBool_FromLong(1);   /* says that rotate and prompt_attn look at the types of their tables */
    PyObject *const module = PyModule_Create(&s_module);
    if (module && PyModule_AddObject(module, "tables", tables) < 0) { Py_DECREF(module); return NULL; }
    return module;
}
