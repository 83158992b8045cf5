/* Calls of a decode step from Python with little host time: the tensors' addresses, shapes
 * and strides are read here, through the interpreter's C interface, and go straight to the
 * library. A call whose arguments are not as they should be is not made: the function
 * returns -1, and the binding's own checks (p4q.py) say what is wrong with it. (A step of
 * append and attention of a few sequences is bound by host time. Marshalled in Python with
 * ctypes an append took 14.8 us of it, 5.2 of these in the library and ctypes.) */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "p4q.h"

typedef p4q_status (*append_fn)(const uint16_t*, int, const uint16_t*, int, const uint16_t*, int, int, int, const float*,
                                const float*, int, int, int, const int32_t*, const int32_t*, const int32_t*,
                                const p4q_paged_kvq*, int, uint16_t*, int, uint16_t*, int, uint16_t*, int, p4q_stream_t);
typedef p4q_status (*attend_fn)(const uint16_t*, int, int, const p4q_paged_kvq*, int, const int32_t*, float, uint16_t*,
                                int, float*, void*, size_t, p4q_stream_t);
typedef p4q_status (*prefix_fn)(const uint16_t*, int, int, const p4q_paged_kv*, const int32_t*, const int32_t*,
                                const int32_t*, int, float, uint16_t*, int, float*, void*, size_t, p4q_stream_t);

static append_fn call_append;
static attend_fn call_attend;
static prefix_fn call_prefix;
static PyObject *get_stream, *get_device;                             /* torch's current stream and device */
static PyObject *t_f16, *t_bf16, *t_f32, *t_i32, *t_i8, *t_u8;         /* torch's types */
static PyObject *n_shape, *n_stride, *n_dtype, *n_is_cuda, *n_data_ptr, *n_cuda_stream;

typedef struct {
  void* p;
  PyObject* dtype; /* compared by identity only */
  int64_t shape[4], stride[4];
} tensor;

static int numbers(PyObject* t, int n, int64_t* out) {
  if (!t || !PyTuple_Check(t) || PyTuple_GET_SIZE(t) != n) return 0;
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (out[i] == -1 && PyErr_Occurred()) return 0;
  }
  return 1;
}

/* A CUDA tensor of nd dimensions; 0 if o is none. */
static int read_tensor(PyObject* o, int nd, tensor* t) {
  PyObject* v = PyObject_GetAttr(o, n_shape);
  int ok = numbers(v, nd, t->shape);
  Py_XDECREF(v);
  if (!ok) return 0;
  v = PyObject_CallMethodNoArgs(o, n_stride);
  ok = numbers(v, nd, t->stride);
  Py_XDECREF(v);
  if (!ok) return 0;
  v = PyObject_GetAttr(o, n_is_cuda);
  ok = v == Py_True;
  Py_XDECREF(v);
  if (!ok) return 0;
  t->dtype = PyObject_GetAttr(o, n_dtype);
  if (!t->dtype) return 0;
  Py_DECREF(t->dtype); /* (a type object of torch, which outlives this) */
  v = PyObject_CallMethodNoArgs(o, n_data_ptr);
  if (!v) return 0;
  t->p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

/* Rows of `cols` values of a type with unit column stride (cols, rows < 0: any), and their pitch. */
static int read_rows(PyObject* o, PyObject* dtype, int64_t rows, int64_t cols, tensor* t, int* pitch) {
  if (!read_tensor(o, 2, t) || t->dtype != dtype || (t->stride[1] != 1 && t->shape[1] > 1)) return 0;
  if ((rows >= 0 && t->shape[0] != rows) || (cols >= 0 && t->shape[1] != cols)) return 0;
  const int64_t ld = t->shape[0] > 1 ? t->stride[0] : (t->shape[1] + 7) / 8 * 8;
  if (ld < 0 || ld > INT32_MAX || t->shape[0] > INT32_MAX || t->shape[1] > INT32_MAX) return 0;
  *pitch = (int)ld;
  return 1;
}

static int read_vector(PyObject* o, PyObject* dtype, int64_t n, tensor* t) {
  return read_tensor(o, 1, t) && t->dtype == dtype && t->shape[0] == n && (n <= 1 || t->stride[0] == 1);
}

static int read_optional(PyObject* o, PyObject* dtype, int64_t n, tensor* t) {
  t->p = NULL;
  return o == Py_None || read_vector(o, dtype, n, t);
}

static int whole2(const tensor* t) { /* contiguous, 2-D */
  return (t->shape[1] <= 1 || t->stride[1] == 1) && (t->shape[0] <= 1 || t->stride[0] == t->shape[1]);
}

static int same4(const tensor* a, const tensor* b, int n) {
  if (a->dtype != b->dtype) return 0;
  for (int i = 0; i < n; ++i)
    if (a->shape[i] != b->shape[i] || a->stride[i] != b->stride[i]) return 0;
  return 1;
}

static int small(int64_t x) { return x >= 0 && x <= INT32_MAX; }

/* The page table and what the cache's first tensor says, as p4q.py packs them. */
static int read_table(PyObject* o, int32_t* seqs, int32_t* ld, int32_t* cols, const int32_t** p) {
  tensor t;
  if (!read_tensor(o, 2, &t) || t.dtype != t_i32 || (t.stride[1] != 1 && t.shape[1] > 1)) return 0;
  const int64_t pitch = t.shape[0] > 1 ? t.stride[0] : t.shape[1];
  if (!small(t.shape[0]) || !small(t.shape[1]) || !small(pitch)) return 0;
  *seqs = (int32_t)t.shape[0];
  *cols = (int32_t)t.shape[1];
  *ld = (int32_t)pitch;
  *p = (const int32_t*)t.p;
  return 1;
}

static int read_kvq(PyObject* const* a, p4q_paged_kvq* kv) { /* k, v, k_scale, v_scale, table */
  tensor k, v, ks, vs;
  if (!read_tensor(a[0], 4, &k) || !read_tensor(a[1], 4, &v) || !read_tensor(a[2], 3, &ks) || !read_tensor(a[3], 3, &vs))
    return 0;
  if ((k.dtype != t_i8 && k.dtype != t_u8) || k.stride[3] != 1 || !same4(&k, &v, 4)) return 0;
  if (ks.dtype != t_f32 || !same4(&ks, &vs, 3)) return 0;
  for (int i = 0; i < 4; ++i)
    if (!small(k.shape[i]) || (i < 3 && ks.shape[i] != k.shape[i])) return 0;
  kv->k = k.p;
  kv->v = v.p;
  kv->k_scale = (float*)ks.p;
  kv->v_scale = (float*)vs.p;
  const int64_t row = (k.shape[3] + 15) / 16 * 16; /* (the stride of a dimension of one says nothing) */
  kv->page_stride = k.shape[0] > 1 ? k.stride[0] : row;
  kv->token_stride = k.shape[1] > 1 ? k.stride[1] : row;
  kv->head_stride = k.shape[2] > 1 ? k.stride[2] : row;
  kv->scale_page_stride = k.shape[0] > 1 ? ks.stride[0] : 1;
  kv->scale_token_stride = k.shape[1] > 1 ? ks.stride[1] : 1;
  kv->scale_head_stride = k.shape[2] > 1 ? ks.stride[2] : 1;
  kv->bits = k.dtype == t_i8 ? 8 : 4;
  kv->pages = (int32_t)k.shape[0];
  kv->page_size = (int32_t)k.shape[1];
  kv->Hkv = (int32_t)k.shape[2];
  if (k.shape[3] > (1 << 20)) return 0;
  kv->dh = (int32_t)(k.dtype == t_i8 ? k.shape[3] : 2 * k.shape[3]);
  return kv->dh > 0 && read_table(a[4], &kv->seqs, &kv->table_ld, &kv->table_cols, &kv->table);
}

static int read_kv(PyObject* const* a, p4q_paged_kv* kv, PyObject** dtype) { /* k, v, table */
  tensor k, v;
  if (!read_tensor(a[0], 4, &k) || !read_tensor(a[1], 4, &v)) return 0;
  if ((k.dtype != t_f16 && k.dtype != t_bf16) || k.stride[3] != 1 || !same4(&k, &v, 4)) return 0;
  for (int i = 0; i < 4; ++i)
    if (!small(k.shape[i])) return 0;
  const int64_t dh = k.shape[3];
  kv->k = k.p;
  kv->v = v.p;
  kv->page_stride = k.shape[0] > 1 ? k.stride[0] : k.stride[0] > dh ? k.stride[0] : dh;
  kv->token_stride = k.shape[1] > 1 ? k.stride[1] : dh;
  kv->head_stride = k.shape[2] > 1 ? k.stride[2] : dh;
  kv->dtype = k.dtype == t_f16 ? P4Q_F16 : P4Q_BF16;
  kv->pages = (int32_t)k.shape[0];
  kv->page_size = (int32_t)k.shape[1];
  kv->Hkv = (int32_t)k.shape[2];
  kv->dh = (int32_t)dh;
  *dtype = k.dtype;
  return dh > 0 && read_table(a[2], &kv->seqs, &kv->table_ld, &kv->table_cols, &kv->table);
}

/* None: torch's current stream; else a torch.cuda.Stream. */
static int read_stream(PyObject* o, p4q_stream_t* s) {
  PyObject* v;
  if (o == Py_None) {
    PyObject* d = PyObject_CallNoArgs(get_device);
    if (!d) return 0;
    v = PyObject_CallOneArg(get_stream, d);
    Py_DECREF(d);
  } else {
    v = PyObject_GetAttr(o, n_cuda_stream);
  }
  if (!v) return 0;
  *s = (p4q_stream_t)PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

static int read_scale(PyObject* o, int dh, float* scale) {
  const double x = o == Py_None ? (dh == 64 ? 0.125 : dh == 128 ? 0.088388347648318447 : -1.0) : PyFloat_AsDouble(o);
  *scale = (float)x;
  return !(o == Py_None && x < 0) && !PyErr_Occurred();
}

static int row_type(PyObject* o, PyObject** dtype) { /* fp16 or bf16 */
  PyObject* v = PyObject_GetAttr(o, n_dtype);
  if (!v) return 0;
  Py_DECREF(v);
  *dtype = v;
  return v == t_f16 || v == t_bf16;
}

static PyObject* refused(void) {
  PyErr_Clear();
  return PyLong_FromLong(-1);
}

/* q, k, v, cos, sin, pos, k_cache, v_cache, k_scale, v_scale, table, q_out, k_out, v_out, seq, rot_pos, interleaved, stream */
static PyObject* rope_append_quant(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  p4q_paged_kvq kv;
  PyObject* dt;
  tensor q, k, v, c, s, pos, qo, ko, vo, seq, rot;
  int ldq, ldk, ldv, ldqo, ldko = 0, ldvo = 0;
  p4q_stream_t stream;
  if (n != 18 || !row_type(a[0], &dt) || !read_kvq(a + 6, &kv) || !read_rows(a[0], dt, -1, -1, &q, &ldq)) return refused();
  const int64_t T = q.shape[0], width = q.shape[1], nk = (int64_t)kv.Hkv * kv.dh;
  ko.p = vo.p = NULL;
  if (width % kv.dh || !read_rows(a[1], dt, T, nk, &k, &ldk) || !read_rows(a[2], dt, T, nk, &v, &ldv) ||
      !read_tensor(a[3], 2, &c) || !read_tensor(a[4], 2, &s) || c.dtype != t_f32 || s.dtype != t_f32 || !whole2(&c) ||
      !whole2(&s) || c.shape[0] != s.shape[0] || c.shape[1] != s.shape[1] || !small(c.shape[0]) || c.shape[1] > (1 << 20) ||
      !read_vector(a[5], t_i32, T, &pos) || !read_rows(a[11], dt, T, width, &qo, &ldqo) ||
      (a[12] != Py_None && !read_rows(a[12], dt, T, nk, &ko, &ldko)) ||
      (a[13] != Py_None && !read_rows(a[13], dt, T, nk, &vo, &ldvo)) || !read_optional(a[14], t_i32, T, &seq) ||
      !read_optional(a[15], t_i32, T, &rot) || !read_stream(a[17], &stream))
    return refused();
  const int inter = PyObject_IsTrue(a[16]);
  if (inter < 0) return refused();
  p4q_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = call_append(q.p, ldq, k.p, ldk, v.p, ldv, (int)T, (int)(width / kv.dh), c.p, s.p, (int)c.shape[0], (int)(2 * c.shape[1]),
                   inter, pos.p, rot.p, seq.p, &kv, dt == t_f16 ? P4Q_F16 : P4Q_BF16, qo.p, ldqo, ko.p, ldko, vo.p, ldvo, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

static int read_ws(PyObject* o, tensor* t) {
  return read_tensor(o, 1, t) && t->dtype == t_u8 && (t->shape[0] <= 1 || t->stride[0] == 1);
}

static int read_lse(PyObject* o, int64_t seqs, int64_t heads, tensor* t) {
  t->p = NULL;
  return o == Py_None || (read_tensor(o, 2, t) && t->dtype == t_f32 && whole2(t) && t->shape[0] == seqs && t->shape[1] == heads);
}

/* q, k_cache, v_cache, k_scale, v_scale, table, lens, o, ws, scale, lse, stream */
static PyObject* paged_attention_quant(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  p4q_paged_kvq kv;
  PyObject* dt;
  tensor q, lens, o, ws, lse;
  int ldq, ldo;
  float scale;
  p4q_stream_t stream;
  if (n != 12 || !row_type(a[0], &dt) || !read_kvq(a + 1, &kv) || !read_rows(a[0], dt, kv.seqs, -1, &q, &ldq)) return refused();
  const int64_t width = q.shape[1];
  if (width % kv.dh || !read_vector(a[6], t_i32, kv.seqs, &lens) || !read_rows(a[7], dt, kv.seqs, width, &o, &ldo) ||
      !read_ws(a[8], &ws) || !read_scale(a[9], kv.dh, &scale) || !read_lse(a[10], kv.seqs, width / kv.dh, &lse) ||
      !read_stream(a[11], &stream))
    return refused();
  p4q_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = call_attend(q.p, ldq, (int)(width / kv.dh), &kv, dt == t_f16 ? P4Q_F16 : P4Q_BF16, lens.p, scale, o.p, ldo, lse.p, ws.p,
                   (size_t)ws.shape[0], stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

/* q, k_cache, v_cache, table, lens, group_start, prefix_lens, o, ws, scale, lse, stream */
static PyObject* prefix_attention(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  p4q_paged_kv kv;
  PyObject* dt;
  tensor q, lens, start, prefix, o, ws, lse;
  int ldq, ldo;
  float scale;
  p4q_stream_t stream;
  if (n != 12 || !read_kv(a + 1, &kv, &dt) || !read_rows(a[0], dt, kv.seqs, -1, &q, &ldq)) return refused();
  const int64_t width = q.shape[1];
  if (width % kv.dh || !read_vector(a[4], t_i32, kv.seqs, &lens) || !read_tensor(a[6], 1, &prefix) ||
      !small(prefix.shape[0]) || prefix.dtype != t_i32 || (prefix.shape[0] > 1 && prefix.stride[0] != 1) ||
      !read_vector(a[5], t_i32, prefix.shape[0] + 1, &start) || !read_rows(a[7], dt, kv.seqs, width, &o, &ldo) ||
      !read_ws(a[8], &ws) || !read_scale(a[9], kv.dh, &scale) || !read_lse(a[10], kv.seqs, width / kv.dh, &lse) ||
      !read_stream(a[11], &stream))
    return refused();
  p4q_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = call_prefix(q.p, ldq, (int)(width / kv.dh), &kv, lens.p, start.p, prefix.p, (int)prefix.shape[0], scale, o.p, ldo, lse.p,
                   ws.p, (size_t)ws.shape[0], stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

/* bind((addresses of the three entry points), (fp16, bf16, fp32, int32, int8, uint8), current stream, current device) */
static PyObject* bind(PyObject* self, PyObject* args) {
  (void)self;
  unsigned long long f[3];
  PyObject *types[6], *stream, *device;
  if (!PyArg_ParseTuple(args, "(KKK)(OOOOOO)OO", &f[0], &f[1], &f[2], &types[0], &types[1], &types[2], &types[3], &types[4],
                        &types[5], &stream, &device))
    return NULL;
  call_append = (append_fn)(uintptr_t)f[0];
  call_attend = (attend_fn)(uintptr_t)f[1];
  call_prefix = (prefix_fn)(uintptr_t)f[2];
  PyObject** const kept[] = {&t_f16, &t_bf16, &t_f32, &t_i32, &t_i8, &t_u8};
  for (int i = 0; i < 6; ++i) *kept[i] = Py_NewRef(types[i]);
  get_stream = Py_NewRef(stream);
  get_device = Py_NewRef(device);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, NULL},
    {"rope_append_quant", (PyCFunction)(void (*)(void))rope_append_quant, METH_FASTCALL, NULL},
    {"paged_attention_quant", (PyCFunction)(void (*)(void))paged_attention_quant, METH_FASTCALL, NULL},
    {"prefix_attention", (PyCFunction)(void (*)(void))prefix_attention, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "p4q_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit_p4q_call(void) {
  n_shape = PyUnicode_InternFromString("shape");
  n_stride = PyUnicode_InternFromString("stride");
  n_dtype = PyUnicode_InternFromString("dtype");
  n_is_cuda = PyUnicode_InternFromString("is_cuda");
  n_data_ptr = PyUnicode_InternFromString("data_ptr");
  n_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!n_shape || !n_stride || !n_dtype || !n_is_cuda || !n_data_ptr || !n_cuda_stream) return NULL;
  return PyModule_Create(&module);
}
