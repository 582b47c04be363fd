/* CPython module behind heatkv.py: the checks and the call of the functions of the paged cache that a model's step repeats, in one go.  A small
 * call takes longer in Python than on the GPU (a table call 9.4 us from there through ctypes, 6.1 from here, its kernel 3 to 4).
 * Each gives the call's status, or None where an argument does not pass: heatkv.py then looks again and says which. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>

#include "heatkv.h"

static PyObject *s_data_ptr, *s_stride, *s_dtype, *s_shape, *s_numel, *s_nbytes, *s_is_contiguous, *s_get_device, *s_cuda_stream, *s_addr, *s_device,
    *s_torch_dtype;
static PyObject *type_int32, *type_float32;
static PyObject *hook_device, *hook_stream;      /* torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream */

/* whole number that a method (or, attribute != 0, an attribute) gives; INT64_MIN where there is none */
static int64_t number(PyObject* x, PyObject* name, int attribute) {
  PyObject* v = attribute ? PyObject_GetAttr(x, name) : PyObject_CallMethodNoArgs(x, name);
  const int64_t r = v ? PyLong_AsLongLong(v) : -1;
  Py_XDECREF(v);
  if (!PyErr_Occurred()) return r;
  PyErr_Clear();
  return INT64_MIN;
}
static int contiguous(PyObject* t) {
  PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  if (!v) PyErr_Clear();
  Py_XDECREF(v);
  return v == Py_True;
}
/* a tensor's address, if it has the type and lies on the device */
static int placed(PyObject* t, PyObject* type, int64_t device, void** out) {
  PyObject* v = PyObject_GetAttr(t, s_dtype);
  if (!v) PyErr_Clear();
  Py_XDECREF(v);
  if (v != type || number(t, s_get_device, 0) != device) return 0;
  v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  *out = v ? PyLong_AsVoidPtr(v) : NULL;
  Py_XDECREF(v);
  if (!PyErr_Occurred()) return 1;
  PyErr_Clear();
  return 0;
}
static int vector(PyObject* t, int64_t n, int64_t device, void** out) {
  return placed(t, type_int32, device, out) && number(t, s_numel, 0) == n && contiguous(t);
}
/* `dims` numbers of a tensor's shape, or (method != 0) of its strides */
static int extents(PyObject* t, PyObject* name, int method, int dims, int64_t* out) {
  PyObject* v = method ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
  const int ok = v && PyTuple_Check(v) && PyTuple_GET_SIZE(v) == dims;
  for (int i = 0; ok && i < dims; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
  Py_XDECREF(v);
  if (!PyErr_Occurred()) return ok;
  PyErr_Clear();
  return 0;
}
/* [tokens, heads (0: any number), d] activations, d contiguous */
typedef struct {
  void* p;
  int64_t heads, tok, head;
} Rows;
static int rows(PyObject* t, PyObject* type, int64_t device, int64_t tokens, int64_t heads, int64_t d, Rows* out) {
  int64_t x[3];
  if (!placed(t, type, device, &out->p) || !extents(t, s_shape, 0, 3, x) || x[0] != tokens || x[2] != d || (heads && x[1] != heads)) return 0;
  out->heads = x[1];
  out->tok = x[1] * d;
  out->head = d;
  if (contiguous(t)) return 1;
  if (!extents(t, s_stride, 1, 3, x) || x[2] != 1) return 0;
  out->tok = x[0];
  out->head = x[1];
  return 1;
}
/* the stream's handle, if `device` is the current one */
static int stream_of(PyObject* stream, int64_t device, void** out) {
  if (device < 0 || !hook_device) return 0;
  PyObject* here = PyObject_CallNoArgs(hook_device);
  PyObject* v = NULL;
  if (here && PyLong_AsLongLong(here) == device)
    v = stream == Py_None ? PyObject_CallOneArg(hook_stream, here) : PyLong_Check(stream) ? Py_NewRef(stream) : PyObject_GetAttr(stream, s_cuda_stream);
  *out = v ? PyLong_AsVoidPtr(v) : NULL;
  Py_XDECREF(here);
  Py_XDECREF(v);
  if (!PyErr_Occurred()) return v != NULL;
  PyErr_Clear();
  return 0;
}
/* a pool's or batch's structure, kept alive by the object that the caller holds */
static const void* structure(PyObject* x, int64_t* device) {
  const int64_t at = number(x, s_addr, 1);
  *device = number(x, s_device, 1);
  return at > 0 && *device >= 0 ? (const void*)(intptr_t)at : NULL;
}
static const heatkv_paged_pool* pool_of(PyObject* x, int64_t* device, PyObject** type) {
  const heatkv_paged_pool* pool = structure(x, device);
  *type = pool ? PyObject_GetAttr(x, s_torch_dtype) : NULL;       /* (held by torch, too) */
  if (!*type) PyErr_Clear();
  Py_XDECREF(*type);
  return *type ? pool : NULL;
}

static PyObject* py_paged_tables(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 11) Py_RETURN_NONE;
  const int64_t device = number(a[0], s_get_device, 0), n = number(a[0], s_numel, 0), n_pages = number(a[2], s_numel, 0),
                n_tokens = number(a[8], s_numel, 0);
  void *stream, *p[10];
  int64_t shape[2], strides[2];
  p[9] = NULL;
  if (!stream_of(a[10], device, &stream) || n < 0 || n > INT_MAX || n_pages < 0 || n_pages > INT_MAX || n_tokens < 0 || n_tokens > INT_MAX ||
      !vector(a[0], n, device, &p[0]) || !vector(a[1], n, device, &p[1]) || !vector(a[2], n_pages, device, &p[2]) ||
      !vector(a[3], 4, device, &p[3]) || !vector(a[4], 4, device, &p[4]) || !placed(a[5], type_int32, device, &p[5]) ||
      !extents(a[5], s_shape, 0, 2, shape) || !extents(a[5], s_stride, 1, 2, strides) || shape[0] != n || shape[1] > INT_MAX || strides[1] != 1 ||
      !vector(a[6], n + 1, device, &p[6]) || !vector(a[7], n, device, &p[7]) || !vector(a[8], n_tokens, device, &p[8]) ||
      (a[9] != Py_None && !vector(a[9], n_tokens, device, &p[9])))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_tables(p[0], p[1], (int)n, p[2], (int)n_pages, p[3], p[4], p[5], n > 1 ? strides[0] : shape[1], (int)shape[1], p[6], p[7], p[8],
                           p[9], (int)n_tokens, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_paged_store(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int64_t device, n;
  PyObject* type;
  const heatkv_paged_pool* pool;
  void *stream, *slots;
  Rows k, v;
  if (n_args != 5 || !(pool = pool_of(a[0], &device, &type)) || (n = number(a[3], s_numel, 0)) < 0 || n > INT_MAX ||
      !rows(a[1], type, device, n, pool->n_kv_heads, pool->d, &k) || !rows(a[2], type, device, n, pool->n_kv_heads, pool->d, &v) ||
      k.tok != v.tok || k.head != v.head || !vector(a[3], n, device, &slots) || !stream_of(a[4], device, &stream))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_store(pool, k.p, v.p, k.tok, k.head, slots, (int)n, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* what the calls over a batch have in common: (pool, batch, q, ..) and n_select lists of pages per token (sel None: none) */
typedef struct {
  const heatkv_paged_pool* pool;
  const heatkv_paged_batch* batch;
  int64_t device;
  PyObject* type;
  Rows q;
  void *lists, *stream;
  int64_t n_select;
} Call;
static int call_of(PyObject* pool, PyObject* batch, PyObject* q, PyObject* sel, PyObject* stream, Call* c) {
  int64_t other, x[3];
  if (!(c->pool = pool_of(pool, &c->device, &c->type)) || !(c->batch = structure(batch, &other)) || other != c->device ||
      !rows(q, c->type, c->device, c->batch->n_tokens, 0, c->pool->d, &c->q) || c->q.heads > INT_MAX || !stream_of(stream, c->device, &c->stream))
    return 0;
  if (!sel) return 1;
  if (!placed(sel, type_int32, c->device, &c->lists) || !extents(sel, s_shape, 0, 3, x) || x[0] != c->batch->n_tokens || x[1] != c->pool->n_kv_heads ||
      x[2] > INT_MAX || !contiguous(sel))
    return 0;
  c->n_select = x[2];
  return 1;
}
/* (.., out, lse | None, workspace): where results go */
typedef struct {
  Rows out;
  void *lse, *workspace;
  int64_t bytes;
} Results;
static int results_of(const Call* c, PyObject* out, PyObject* lse, PyObject* workspace, Results* r) {
  int64_t x[2];
  r->lse = NULL;
  if (!rows(out, c->type, c->device, c->batch->n_tokens, c->q.heads, c->pool->d, &r->out)) return 0;
  if (lse != Py_None && (!placed(lse, type_float32, c->device, &r->lse) || !extents(lse, s_shape, 0, 2, x) || x[0] != c->batch->n_tokens ||
                         x[1] != c->q.heads || !contiguous(lse)))
    return 0;
  PyObject* type = PyObject_GetAttr(workspace, s_dtype);
  if (!type) PyErr_Clear();
  Py_XDECREF(type);
  return type && placed(workspace, type, c->device, &r->workspace) && (r->bytes = number(workspace, s_nbytes, 1)) >= 0 && contiguous(workspace);
}

static PyObject* py_paged_attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {      /* pool, batch, q, out, lse, ws, causal, scale, stream */
  Call c;
  Results r;
  if (n_args != 9 || !call_of(a[0], a[1], a[2], NULL, a[8], &c) || !results_of(&c, a[3], a[4], a[5], &r)) Py_RETURN_NONE;
  const int causal = PyObject_IsTrue(a[6]);
  const double scale = PyFloat_AsDouble(a[7]);
  if (PyErr_Occurred()) return NULL;
  const heatkv_token_strides st = {c.q.tok, c.q.head, r.out.tok, r.out.head};
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_attention(c.pool, c.batch, (int)c.q.heads, c.q.p, &st, causal, (float)scale, r.out.p, r.lse, r.workspace, (uint64_t)r.bytes, c.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_paged_select(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {         /* pool, batch, q, sel, sink, local, stream */
  Call c;
  if (n_args != 7 || !call_of(a[0], a[1], a[2], a[3], a[6], &c)) Py_RETURN_NONE;
  const long sink = PyLong_AsLong(a[4]), local = PyLong_AsLong(a[5]);
  if (PyErr_Occurred()) return NULL;
  if (sink < INT_MIN || sink > INT_MAX || local < INT_MIN || local > INT_MAX) Py_RETURN_NONE;
  const heatkv_token_strides st = {c.q.tok, c.q.head, c.q.tok, c.q.head};
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_select(c.pool, c.batch, (int)c.q.heads, c.q.p, &st, (int)sink, (int)local, (int)c.n_select, c.lists, c.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_paged_sparse_attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {  /* pool, batch, q, sel, out, lse, ws, scale, stream */
  Call c;
  Results r;
  if (n_args != 9 || !call_of(a[0], a[1], a[2], a[3], a[8], &c) || !results_of(&c, a[4], a[5], a[6], &r)) Py_RETURN_NONE;
  const double scale = PyFloat_AsDouble(a[7]);
  if (PyErr_Occurred()) return NULL;
  const heatkv_token_strides st = {c.q.tok, c.q.head, r.out.tok, r.out.head};
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_sparse_attention(c.pool, c.batch, (int)c.q.heads, c.q.p, &st, c.lists, (int)c.n_select, (float)scale, r.out.p, r.lse, r.workspace,
                                     (uint64_t)r.bytes, c.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_set_hooks(PyObject* self, PyObject* args) {
  PyObject *device, *stream, *i, *f;
  if (!PyArg_ParseTuple(args, "OOOO", &device, &stream, &i, &f)) return NULL;
  hook_device = Py_NewRef(device);                              /* (once a process) */
  hook_stream = Py_NewRef(stream);
  type_int32 = Py_NewRef(i);
  type_float32 = Py_NewRef(f);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"tables", (PyCFunction)(void (*)(void))py_paged_tables, METH_FASTCALL,
     "(new_tokens, past_tokens, free_pages, state, state_out, block_table, q_begin, kv_len, slot_map, positions | None, stream | None)"},
    {"store", (PyCFunction)(void (*)(void))py_paged_store, METH_FASTCALL, "(pool, k_new, v_new, slot_map, stream | None)"},
    {"attention", (PyCFunction)(void (*)(void))py_paged_attention, METH_FASTCALL,
     "(pool, batch, q, out, lse | None, workspace, causal, sm_scale, stream | None)"},
    {"select", (PyCFunction)(void (*)(void))py_paged_select, METH_FASTCALL, "(pool, batch, q, sel, sink, local, stream | None)"},
    {"sparse_attention", (PyCFunction)(void (*)(void))py_paged_sparse_attention, METH_FASTCALL,
     "(pool, batch, q, sel, out, lse | None, workspace, sm_scale, stream | None)"},
    {"set_hooks", py_set_hooks, METH_VARARGS, "(current_device, raw_stream, torch.int32, torch.float32)"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__paged(void) {
  static const struct {
    PyObject** at;
    const char* name;
  } names[] = {{&s_data_ptr, "data_ptr"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_numel, "numel"}, {&s_nbytes, "nbytes"},
               {&s_is_contiguous, "is_contiguous"}, {&s_get_device, "get_device"}, {&s_cuda_stream, "cuda_stream"}, {&s_addr, "addr"},
               {&s_device, "device"}, {&s_torch_dtype, "torch_dtype"}};
  for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
    if (!(*names[i].at = PyUnicode_InternFromString(names[i].name))) return NULL;
  return PyModule_Create(&module);
}
