/* The forward calls of dc.py, and those on 4-bit matrices, without ctypes: arguments are read from the Python objects here and the C entry point is
 * called through its address.  A small layer runs for 3-6 us, and marshalling its call through ctypes took 3.7 us of the host
 * (16 converted arguments, six pointers and the current stream fetched from Python); here about 1.
 *
 * Every function answers None for arguments that are not in the plain form it reads (a dtype it does not know, an act that
 * is no int, ...): dc.py then makes the call through ctypes, which reports what is wrong with them. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <float.h>

typedef int (*conv_fn)(const void *, int, int, int, const void *, const void *, const void *, int, const void *, void *, int,
                       void *, size_t, void *, int);
typedef int (*dw_fn)(const void *, int, int, int, int, int, int, int, const void *, const void *, int, void *, int, void *);
typedef int (*q4_quantize_fn)(const void *, long long, int, long long, int, int, float, void *, void *);
typedef int (*q4_dequantize_fn)(const void *, long long, int, int, float, void *, long long, int, void *);
typedef int (*q4_product_fn)(const void *, long long, int, const void *, int, int, float, const void *, int, const void *, void *, int, void *, size_t,
                             void *);
typedef int (*q4_forward_fn)(const void *, long long, int, const void *, int, int, float, float, const void *, int, const void *, void *, int, void *,
                             size_t, void *);
typedef int (*q4_query_fn)(long long, int, int, size_t *);
typedef int (*block_fn)(const void *, int, int, int, const void *, void *, int, void *, size_t, void *);

static conv_fn g_conv;
static dw_fn g_dw;
static block_fn g_block;
static q4_quantize_fn g_q4_quantize;
static q4_dequantize_fn g_q4_dequantize;
static q4_product_fn g_q4_product;
static q4_forward_fn g_q4_forward;
static q4_query_fn g_q4_query;
static PyObject *g_f32, *g_bf16, *g_geom, *g_block_type, *g_get_device, *g_get_stream;
static PyObject *s_data_ptr, *s_shape, *s_dtype, *s_numel, *s_element_size, *s_cuda_stream;
static PyObject *s_stride, *s_is_contiguous, *s_get_device, *s_rows, *s_cols, *s_fmt, *s_tensor_scale, *s_data, *s_nbytes;

/* each reader: 0 on success, -1 when the argument has another form (any Python error is cleared by the caller) */
static int read_size(PyObject *o, size_t *v) {
  if (!o) return -1;
  const size_t r = PyLong_Check(o) ? PyLong_AsSize_t(o) : (size_t)-1;
  Py_DECREF(o);
  if (r == (size_t)-1) return -1;
  *v = r;
  return 0;
}
static int read_ptr(PyObject *t, void **p) {
  size_t v = 0;
  *p = NULL;
  if (t == Py_None) return 0;
  if (read_size(PyObject_CallMethodNoArgs(t, s_data_ptr), &v)) return -1;
  *p = (void *)v;
  return 0;
}
static int read_int(PyObject *o, int *v) {
  int overflow = 0;
  if (!PyLong_Check(o)) return -1;
  const long r = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || r < -2147483647L - 1 || r > 2147483647L) return -1;
  *v = (int)r;
  return 0;
}
static int read_shape(PyObject *t, int *d) {
  PyObject *s = PyObject_GetAttr(t, s_shape);
  int bad = !s || !PyTuple_Check(s) || PyTuple_GET_SIZE(s) != 4;
  for (int i = 0; i < 4 && !bad; ++i) bad = read_int(PyTuple_GET_ITEM(s, i), &d[i]);
  Py_XDECREF(s);
  return bad ? -1 : 0;
}
static int read_dtype(PyObject *t, int *code) {
  PyObject *d = PyObject_GetAttr(t, s_dtype);
  Py_XDECREF(d);                                  /* dtypes are immortal singletons: compared, not used */
  if (d && d == g_f32) { *code = 0; return 0; }
  if (d && d == g_bf16) { *code = 1; return 0; }
  return -1;
}
static int read_bytes(PyObject *t, size_t *bytes) {
  size_t n = 0, e = 0;
  if (read_size(PyObject_CallMethodNoArgs(t, s_numel), &n) || read_size(PyObject_CallMethodNoArgs(t, s_element_size), &e)) return -1;
  *bytes = n * e;
  return 0;
}
static int read_stream(PyObject *stream, void **st) {
  size_t v = 0;
  if (stream == Py_None) {
    PyObject *dev = PyObject_CallNoArgs(g_get_device);
    if (!dev) return -1;
    PyObject *raw = PyObject_CallOneArg(g_get_stream, dev);
    Py_DECREF(dev);
    if (read_size(raw, &v)) return -1;
  } else if (read_size(PyObject_GetAttr(stream, s_cuda_stream), &v)) {
    return -1;
  }
  *st = (void *)v;
  return 0;
}
static PyObject *other_form(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

/* conv(x, geom, w_packed, bias, act, residual, y, workspace, stream, algo) */
static PyObject *conv(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int d[4], act, algo, code, st;
  void *x, *w, *b, *r, *y, *ws, *stream;
  size_t bytes;
  Py_buffer geom;
  if (n != 10 || !g_conv || (PyObject *)Py_TYPE(a[1]) != g_geom || read_shape(a[0], d) || read_dtype(a[0], &code) || read_ptr(a[0], &x) ||
      read_ptr(a[2], &w) || read_ptr(a[3], &b) || read_int(a[4], &act) || read_ptr(a[5], &r) || read_ptr(a[6], &y) ||
      read_ptr(a[7], &ws) || read_bytes(a[7], &bytes) || read_stream(a[8], &stream) || read_int(a[9], &algo) ||
      PyObject_GetBuffer(a[1], &geom, PyBUF_SIMPLE))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_conv(x, d[0], d[1], d[2], geom.buf, w, b, act, r, y, code, ws, bytes, stream, algo);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&geom);
  return PyLong_FromLong(st);
}

/* dwconv(x, k, stride, pad, w_packed, bias, act, y, stream) */
static PyObject *dwconv(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int d[4], k, s, p, act, code, st;
  void *x, *w, *b, *y, *stream;
  if (n != 9 || !g_dw || read_shape(a[0], d) || read_dtype(a[0], &code) || read_ptr(a[0], &x) || read_int(a[1], &k) || read_int(a[2], &s) ||
      read_int(a[3], &p) || read_ptr(a[4], &w) || read_ptr(a[5], &b) || read_int(a[6], &act) || read_ptr(a[7], &y) ||
      read_stream(a[8], &stream))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_dw(x, d[0], d[1], d[2], d[3], k, s, p, w, b, act, y, code, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* block(x, block, y, workspace, stream) */
static PyObject *block(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int d[4], code, st;
  void *x, *y, *ws, *stream;
  size_t bytes;
  Py_buffer blk;
  if (n != 5 || !g_block || (PyObject *)Py_TYPE(a[1]) != g_block_type || read_shape(a[0], d) || read_dtype(a[0], &code) ||
      read_ptr(a[0], &x) || read_ptr(a[2], &y) || read_ptr(a[3], &ws) || read_bytes(a[3], &bytes) || read_stream(a[4], &stream) ||
      PyObject_GetBuffer(a[1], &blk, PyBUF_SIMPLE))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_block(x, d[0], d[1], d[2], blk.buf, y, code, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&blk);
  return PyLong_FromLong(st);
}

/* ---- 4-bit matrices.  What dc.py checks of their tensors is checked here too; a tensor that fails goes back to dc.py, which says why. */
static int read_ll(PyObject *o, long long *v) {
  int overflow = 0;
  if (!o) return -1;
  const int is = PyLong_Check(o);
  const long long r = is ? PyLong_AsLongLongAndOverflow(o, &overflow) : 0;
  Py_DECREF(o);
  if (!is || overflow) return -1;
  *v = r;
  return 0;
}
static int read_float(PyObject *o, double *v) {
  if (!o) return -1;
  const int is = PyFloat_Check(o);
  if (is) *v = PyFloat_AS_DOUBLE(o);
  Py_DECREF(o);
  return is ? 0 : -1;
}
/* a tensor on the current device `dev`: its address; None: NULL */
static int read_here(PyObject *t, long long dev, void **p) {
  long long d;
  *p = NULL;
  if (t == Py_None) return 0;
  if (read_ll(PyObject_CallMethodNoArgs(t, s_get_device), &d) || d != dev) return -1;
  return read_ptr(t, p);
}
static int current_device(long long *dev) { return read_ll(PyObject_CallNoArgs(g_get_device), dev); }
typedef struct { long long rows, cols, fmt; double scale; void *data; } matrix;
static int read_matrix(PyObject *q, long long dev, matrix *m) {
  PyObject *d = NULL;
  if (read_ll(PyObject_GetAttr(q, s_rows), &m->rows) || read_ll(PyObject_GetAttr(q, s_cols), &m->cols) || read_ll(PyObject_GetAttr(q, s_fmt), &m->fmt) ||
      read_float(PyObject_GetAttr(q, s_tensor_scale), &m->scale) || !(d = PyObject_GetAttr(q, s_data)))
    return -1;
  long long have;
  size_t layout[4];                              /* dc_q4_layout; the last one its bytes */
  int bad = read_here(d, dev, &m->data) || !m->data || m->cols < 1 || m->cols > 2147483647LL || m->fmt < 0 || m->fmt > 1 ||
            read_ll(PyObject_GetAttr(d, s_nbytes), &have) || g_q4_query(m->rows, (int)m->cols, (int)m->fmt, layout) || have < 0 || (size_t)have < layout[3];
  if (!bad) {
    PyObject *dense = PyObject_CallMethodNoArgs(d, s_is_contiguous);
    bad = dense != Py_True;
    Py_XDECREF(dense);
  }
  Py_DECREF(d);
  return bad ? -1 : 0;
}
/* rows of `cols` neighbouring values at one distance: how many, and the distance */
static int read_rows(PyObject *t, long long cols, long long *rows, long long *step) {
  PyObject *sh = PyObject_GetAttr(t, s_shape), *st = PyObject_CallMethodNoArgs(t, s_stride);
  int bad = !sh || !st || !PyTuple_Check(sh) || !PyTuple_Check(st) || PyTuple_GET_SIZE(sh) < 2 || PyTuple_GET_SIZE(sh) != PyTuple_GET_SIZE(st);
  if (!bad) {
    const Py_ssize_t n = PyTuple_GET_SIZE(sh);
    long long have = 1, first = -1;
    bad = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, n - 1)) != cols || (cols > 1 && PyLong_AsLongLong(PyTuple_GET_ITEM(st, n - 1)) != 1);
    for (Py_ssize_t i = n - 2; i >= 0 && !bad; --i) {
      const long long size = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i)), stride = PyLong_AsLongLong(PyTuple_GET_ITEM(st, i));
      if (size == 1) continue;
      if (first < 0) first = stride;
      else bad = stride != first * have;
      have *= size;
    }
    *rows = have;
    *step = have > 1 ? first : cols;
  }
  Py_XDECREF(sh);
  Py_XDECREF(st);
  return bad || PyErr_Occurred() ? -1 : 0;
}
/* a dense tensor [..., cols] of `rows` rows (-1: any number) and this dtype code; None passes where `may_lack` */
static int read_dense(PyObject *t, long long dev, long long *rows, long long cols, int code, int may_lack, void **p) {
  int c;
  long long n;
  *p = NULL;
  if (t == Py_None) return may_lack ? 0 : -1;
  if (read_dtype(t, &c) || c != code) return -1;
  PyObject *sh = PyObject_GetAttr(t, s_shape);
  int bad = !sh || !PyTuple_Check(sh) || PyTuple_GET_SIZE(sh) < 1;
  if (!bad) {
    const Py_ssize_t d = PyTuple_GET_SIZE(sh);
    n = 1;
    for (Py_ssize_t i = 0; i < d - 1; ++i) n *= PyLong_AsLongLong(PyTuple_GET_ITEM(sh, i));
    bad = PyLong_AsLongLong(PyTuple_GET_ITEM(sh, d - 1)) != cols || (*rows >= 0 && n != *rows) || PyErr_Occurred();
    *rows = n;
  }
  Py_XDECREF(sh);
  if (bad) return -1;
  PyObject *dense = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  bad = dense != Py_True;
  Py_XDECREF(dense);
  return bad || read_here(t, dev, p) ? -1 : 0;
}
static int read_bias(PyObject *t, long long dev, long long n, void **p) {
  long long one = -1;
  if (t == Py_None) { *p = NULL; return 0; }
  return read_dense(t, dev, &one, n, 0, 0, p) || one != 1 ? -1 : 0;
}

/* q4_quantize(x, q, stream), q4_dequantize(q, y, stream) */
static PyObject *q4_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int code, st;
  long long dev, rows, step;
  matrix q;
  void *x, *stream;
  if (n != 3 || !g_q4_quantize || current_device(&dev) || read_matrix(a[1], dev, &q) || read_dtype(a[0], &code) || read_rows(a[0], q.cols, &rows, &step) ||
      rows != q.rows || read_here(a[0], dev, &x) || read_stream(a[2], &stream))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_q4_quantize(x, rows, (int)q.cols, step, code, (int)q.fmt, (float)q.scale, q.data, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
static PyObject *q4_dequantize(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int code, st;
  long long dev, rows, step;
  matrix q;
  void *y, *stream;
  if (n != 3 || !g_q4_dequantize || current_device(&dev) || read_matrix(a[0], dev, &q) || read_dtype(a[1], &code) || read_rows(a[1], q.cols, &rows, &step) ||
      rows != q.rows || read_here(a[1], dev, &y) || read_stream(a[2], &stream))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_q4_dequantize(q.data, rows, (int)q.cols, (int)q.fmt, (float)q.scale, y, step, code, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
/* a product of two tensor scales that fp32 rounds to 0, or to a subnormal number with fewer bits */
static int is_lost(double a, double b) {
  const double p = a * b;
  return (p == 0 && a != 0 && b != 0) || (p < FLT_MIN && p > -FLT_MIN && (double)(float)p != p);
}
/* q4_product(x, w, bias, act, residual, y, workspace, stream) */
static PyObject *q4_product(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int act, code, st;
  long long dev;
  matrix x, w;
  void *b, *r, *y, *ws, *stream;
  size_t bytes;
  if (n != 8 || !g_q4_product || current_device(&dev) || read_matrix(a[0], dev, &x) || read_matrix(a[1], dev, &w) || x.fmt != w.fmt || x.cols != w.cols ||
      is_lost(x.scale, w.scale) ||
      w.rows > 2147483647LL || read_dtype(a[5], &code) || read_bias(a[2], dev, w.rows, &b) || read_int(a[3], &act) ||
      read_dense(a[4], dev, &x.rows, w.rows, code, 1, &r) || read_dense(a[5], dev, &x.rows, w.rows, code, 0, &y) || read_here(a[6], dev, &ws) ||
      read_bytes(a[6], &bytes) || read_stream(a[7], &stream))
    return other_form();
  Py_BEGIN_ALLOW_THREADS
  st = g_q4_product(x.data, x.rows, (int)x.cols, w.data, (int)w.rows, (int)x.fmt, (float)(x.scale * w.scale), b, act, r, y, code, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
/* q4_forward(x, w, x_scale, bias, act, residual, y, workspace, stream) */
static PyObject *q4_forward(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  int act, code, st;
  long long dev, rows = -1;
  matrix w;
  double scale;
  void *x, *b, *r, *y, *ws, *stream;
  size_t bytes;
  if (n != 9 || !g_q4_forward || !PyFloat_Check(a[2]) || current_device(&dev) || read_matrix(a[1], dev, &w) || w.rows > 2147483647LL || read_dtype(a[0], &code) ||
      read_dense(a[0], dev, &rows, w.cols, code, 0, &x) || read_bias(a[3], dev, w.rows, &b) || read_int(a[4], &act) ||
      read_dense(a[5], dev, &rows, w.rows, code, 1, &r) || read_dense(a[6], dev, &rows, w.rows, code, 0, &y) || read_here(a[7], dev, &ws) ||
      read_bytes(a[7], &bytes) || read_stream(a[8], &stream))
    return other_form();
  scale = PyFloat_AS_DOUBLE(a[2]);
  Py_BEGIN_ALLOW_THREADS
  st = g_q4_forward(x, rows, (int)w.cols, w.data, (int)w.rows, (int)w.fmt, (float)scale, (float)w.scale, b, act, r, y, code, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
/* bind_q4(addresses of quantize, dequantize, product, forward, query) */
static PyObject *bind_q4(PyObject *self, PyObject *args) {
  unsigned long long q, d, p, f, l;
  (void)self;
  if (!PyArg_ParseTuple(args, "KKKKK", &q, &d, &p, &f, &l)) return NULL;
  g_q4_quantize = (q4_quantize_fn)(uintptr_t)q;
  g_q4_dequantize = (q4_dequantize_fn)(uintptr_t)d;
  g_q4_product = (q4_product_fn)(uintptr_t)p;
  g_q4_forward = (q4_forward_fn)(uintptr_t)f;
  g_q4_query = (q4_query_fn)(uintptr_t)l;
  Py_RETURN_NONE;
}

/* bind(conv address, dwconv address, block address, float32, bfloat16, Geom, Block, current device, current raw stream) */
static PyObject *bind(PyObject *self, PyObject *args) {
  unsigned long long c, w, b;
  PyObject *o[6];
  (void)self;
  if (!PyArg_ParseTuple(args, "KKKOOOOOO", &c, &w, &b, &o[0], &o[1], &o[2], &o[3], &o[4], &o[5])) return NULL;
  for (int i = 0; i < 6; ++i) Py_INCREF(o[i]);    /* kept for the life of the process */
  g_f32 = o[0]; g_bf16 = o[1]; g_geom = o[2]; g_block_type = o[3]; g_get_device = o[4]; g_get_stream = o[5];
  g_dw = (dw_fn)(uintptr_t)w;
  g_block = (block_fn)(uintptr_t)b;
  g_conv = (conv_fn)(uintptr_t)c;
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, NULL},
                                {"dwconv", (PyCFunction)(void (*)(void))dwconv, METH_FASTCALL, NULL},
                                {"block", (PyCFunction)(void (*)(void))block, METH_FASTCALL, NULL},
                                {"q4_quantize", (PyCFunction)(void (*)(void))q4_quantize, METH_FASTCALL, NULL},
                                {"q4_dequantize", (PyCFunction)(void (*)(void))q4_dequantize, METH_FASTCALL, NULL},
                                {"q4_product", (PyCFunction)(void (*)(void))q4_product, METH_FASTCALL, NULL},
                                {"q4_forward", (PyCFunction)(void (*)(void))q4_forward, METH_FASTCALL, NULL},
                                {"bind", bind, METH_VARARGS, NULL},
                                {"bind_q4", bind_q4, METH_VARARGS, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dccall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__dccall(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_shape = PyUnicode_InternFromString("shape");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_numel = PyUnicode_InternFromString("numel");
  s_element_size = PyUnicode_InternFromString("element_size");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_stride = PyUnicode_InternFromString("stride");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_rows = PyUnicode_InternFromString("rows");
  s_cols = PyUnicode_InternFromString("cols");
  s_fmt = PyUnicode_InternFromString("fmt");
  s_tensor_scale = PyUnicode_InternFromString("tensor_scale");
  s_data = PyUnicode_InternFromString("data");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  if (!s_stride || !s_is_contiguous || !s_get_device || !s_rows || !s_cols || !s_fmt || !s_tensor_scale || !s_data || !s_nbytes) return NULL;
  if (!s_data_ptr || !s_shape || !s_dtype || !s_numel || !s_element_size || !s_cuda_stream) return NULL;
  return PyModule_Create(&module);
}
