/* CPython module behind heatkv.py: the checks and the call of the functions of the paged cache that a model's step repeats, in one go.  A small
 * call takes longer in Python than on the GPU (a table call 9.4 us from there through ctypes, 6.1 from here, its kernel 3 to 4).
 * Each gives the call's status, or None where an argument does not pass: heatkv.py then looks again and says which. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>

#include "heatkv.h"

static PyObject *s_data_ptr, *s_stride, *s_dtype, *s_shape, *s_numel, *s_nbytes, *s_is_contiguous, *s_get_device, *s_cuda_stream, *s_addr, *s_addr4, *s_device,
    *s_torch_dtype;
static PyObject *type_int32, *type_float32, *type_uint8, *type_bool;
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
/* a pool's or batch's structure, kept alive by the object that the caller holds (a pool of 4 bits has its address under another name) */
static const void* structure(PyObject* x, PyObject* name, int64_t* device) {
  const int64_t at = number(x, name, 1);
  *device = number(x, s_device, 1);
  return at > 0 && *device >= 0 ? (const void*)(intptr_t)at : NULL;
}
static const void* pool_of(PyObject* x, PyObject* name, int64_t* device, PyObject** type) {
  const void* pool = structure(x, name, device);
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
  if (n_args != 5 || !(pool = pool_of(a[0], s_addr, &device, &type)) || (n = number(a[3], s_numel, 0)) < 0 || n > INT_MAX ||
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
  const void* pool;                                 /* heatkv_paged_pool, or heatkv_paged4_pool */
  int64_t n_kv_heads, d;
  const heatkv_paged_batch* batch;
  int64_t device;
  PyObject* type;
  Rows q;
  void *lists, *stream;
  int64_t n_select;
} Call;
static int call_of(PyObject* pool, PyObject* name, PyObject* batch, PyObject* q, PyObject* sel, PyObject* stream, Call* c) {
  int64_t other, x[3];
  if (!(c->pool = pool_of(pool, name, &c->device, &c->type))) return 0;
  if (name == s_addr) {
    const heatkv_paged_pool* p = c->pool;
    c->n_kv_heads = p->n_kv_heads;
    c->d = p->d;
  } else {
    const heatkv_paged4_pool* p = c->pool;
    c->n_kv_heads = p->n_kv_heads;
    c->d = p->d;
  }
  if (!(c->batch = structure(batch, s_addr, &other)) || other != c->device ||
      !rows(q, c->type, c->device, c->batch->n_tokens, 0, c->d, &c->q) || c->q.heads > INT_MAX || !stream_of(stream, c->device, &c->stream))
    return 0;
  if (!sel) return 1;
  if (!placed(sel, type_int32, c->device, &c->lists) || !extents(sel, s_shape, 0, 3, x) || x[0] != c->batch->n_tokens || x[1] != c->n_kv_heads ||
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
  if (!rows(out, c->type, c->device, c->batch->n_tokens, c->q.heads, c->d, &r->out)) return 0;
  if (lse != Py_None && (!placed(lse, type_float32, c->device, &r->lse) || !extents(lse, s_shape, 0, 2, x) || x[0] != c->batch->n_tokens ||
                         x[1] != c->q.heads || !contiguous(lse)))
    return 0;
  PyObject* type = PyObject_GetAttr(workspace, s_dtype);
  if (!type) PyErr_Clear();
  Py_XDECREF(type);
  return type && placed(workspace, type, c->device, &r->workspace) && (r->bytes = number(workspace, s_nbytes, 1)) >= 0 && contiguous(workspace);
}

/* pool, batch, q, out, lse, ws, causal, scale, stream */
static PyObject* attention(PyObject* const* a, Py_ssize_t n_args, PyObject* name) {
  Call c;
  Results r;
  if (n_args != 9 || !call_of(a[0], name, a[1], a[2], NULL, a[8], &c) || !results_of(&c, a[3], a[4], a[5], &r)) Py_RETURN_NONE;
  const int causal = PyObject_IsTrue(a[6]);
  const double scale = PyFloat_AsDouble(a[7]);
  if (PyErr_Occurred()) return NULL;
  const heatkv_token_strides st = {c.q.tok, c.q.head, r.out.tok, r.out.head};
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = name == s_addr ? heatkv_paged_attention(c.pool, c.batch, (int)c.q.heads, c.q.p, &st, causal, (float)scale, r.out.p, r.lse, r.workspace,
                                               (uint64_t)r.bytes, c.stream)
                      : heatkv_paged4_attention(c.pool, c.batch, (int)c.q.heads, c.q.p, &st, causal, (float)scale, r.out.p, r.lse, r.workspace,
                                                (uint64_t)r.bytes, c.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* py_paged_attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return attention(a, n_args, s_addr); }
static PyObject* py_paged4_attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return attention(a, n_args, s_addr4); }

/* rows of K and V to their slots and back: (pool, k, v, slots, stream) */
static PyObject* rows4(PyObject* const* a, Py_ssize_t n_args, int load) {
  int64_t device, n;
  PyObject* type;
  const heatkv_paged4_pool* pool;
  void *stream, *slots;
  Rows k, v;
  if (n_args != 5 || !(pool = pool_of(a[0], s_addr4, &device, &type)) || (n = number(a[3], s_numel, 0)) < 0 || n > INT_MAX ||
      !rows(a[1], type, device, n, pool->n_kv_heads, pool->d, &k) || !rows(a[2], type, device, n, pool->n_kv_heads, pool->d, &v) ||
      k.tok != v.tok || k.head != v.head || !vector(a[3], n, device, &slots) || !stream_of(a[4], device, &stream))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = load ? heatkv_paged4_load(pool, slots, (int)n, k.p, v.p, k.tok, k.head, stream) : heatkv_paged4_store(pool, k.p, v.p, k.tok, k.head, slots, (int)n, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* py_paged4_store(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return rows4(a, n_args, 0); }
static PyObject* py_paged4_load(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return rows4(a, n_args, 1); }

/* (pool, from, to, stream) */
static PyObject* move(PyObject* const* a, Py_ssize_t n_args, PyObject* name) {
  int64_t device, n;
  PyObject* type;
  const void* pool;
  void *stream, *from, *to;
  if (n_args != 4 || !(pool = pool_of(a[0], name, &device, &type)) || (n = number(a[1], s_numel, 0)) < 0 || n > INT_MAX ||
      !vector(a[1], n, device, &from) || !vector(a[2], n, device, &to) || !stream_of(a[3], device, &stream))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = name == s_addr ? heatkv_paged_move(pool, from, to, (int)n, stream) : heatkv_paged4_move(pool, from, to, (int)n, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* py_paged_move(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return move(a, n_args, s_addr); }
static PyObject* py_paged4_move(PyObject* self, PyObject* const* a, Py_ssize_t n_args) { return move(a, n_args, s_addr4); }

/* what both calls that rearrange rows have: lengths, block_table, free_pages, state, lengths_out, table_out, state_out, move_from, move_to,
 * workspace, stream, from a[0] on; n_moves < 0: any number */
typedef struct {
  int64_t device, n, n_pages, n_moves, bytes, pages, stride, out_stride;
  void *lengths, *table, *free, *state, *lengths_out, *table_out, *state_out, *from, *to, *workspace, *stream;
} Rearranged;
static int table_of(PyObject* t, int64_t n, int64_t device, void** p, int64_t* pages, int64_t* stride) {
  int64_t shape[2], strides[2];
  if (!placed(t, type_int32, device, p) || !extents(t, s_shape, 0, 2, shape) || !extents(t, s_stride, 1, 2, strides) || shape[0] != n ||
      shape[1] > INT_MAX || strides[1] != 1)
    return 0;
  *pages = shape[1];
  *stride = n > 1 ? strides[0] : shape[1];
  return 1;
}
static int rearranged(PyObject* const* a, int by_row, Rearranged* r) {
  int64_t pages;
  r->device = number(a[0], s_get_device, 0);
  r->n = number(a[0], s_numel, 0);
  r->n_pages = number(a[2], s_numel, 0);
  r->n_moves = by_row ? r->n * HEATKV_PAGE_TOKENS : number(a[7], s_numel, 0);
  if (!stream_of(a[10], r->device, &r->stream) || r->n < 0 || r->n > INT_MAX / HEATKV_PAGE_TOKENS || r->n_pages < 0 || r->n_pages > INT_MAX ||
      r->n_moves < 0 || r->n_moves > INT_MAX || !vector(a[0], r->n, r->device, &r->lengths) ||
      !table_of(a[1], r->n, r->device, &r->table, &r->pages, &r->stride) || !vector(a[2], r->n_pages, r->device, &r->free) ||
      !vector(a[3], 4, r->device, &r->state) || !vector(a[4], r->n, r->device, &r->lengths_out) ||
      !table_of(a[5], r->n, r->device, &r->table_out, &pages, &r->out_stride) || pages != r->pages || !vector(a[6], 4, r->device, &r->state_out) ||
      !vector(a[7], r->n_moves, r->device, &r->from) || !vector(a[8], r->n_moves, r->device, &r->to))
    return 0;
  PyObject* type = PyObject_GetAttr(a[9], s_dtype);
  if (!type) PyErr_Clear();
  Py_XDECREF(type);
  return type && placed(a[9], type, r->device, &r->workspace) && (r->bytes = number(a[9], s_nbytes, 1)) >= 0 && contiguous(a[9]);
}

static PyObject* py_paged_fork(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {           /* parents, keep | None, .. */
  Rearranged r;
  void *parents, *keep = NULL;
  if (n_args != 13 || !rearranged(a + 2, 1, &r) || !vector(a[0], r.n, r.device, &parents) || (a[1] != Py_None && !vector(a[1], r.n, r.device, &keep)))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_fork(parents, keep, r.lengths, (int)r.n, r.table, r.stride, (int)r.pages, r.free, (int)r.n_pages, r.state, r.lengths_out, r.table_out,
                         r.out_stride, r.state_out, r.from, r.to, r.workspace, (uint64_t)r.bytes, r.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_paged_compact(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {        /* stays, .. */
  Rearranged r;
  void* stays;
  int64_t shape[2], strides[2];
  if (n_args != 12 || !rearranged(a + 1, 0, &r)) Py_RETURN_NONE;
  if ((!placed(a[0], type_bool, r.device, &stays) && !placed(a[0], type_uint8, r.device, &stays)) || !extents(a[0], s_shape, 0, 2, shape) ||
      !extents(a[0], s_stride, 1, 2, strides) || shape[0] != r.n || shape[1] > INT_MAX || (strides[1] != 1 && shape[1] > 1))
    Py_RETURN_NONE;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = heatkv_paged_compact(stays, r.n > 1 ? strides[0] : shape[1], (int)shape[1], r.lengths, (int)r.n, r.table, r.stride, (int)r.pages, r.free,
                            (int)r.n_pages, r.state, r.lengths_out, r.table_out, r.out_stride, r.state_out, r.from, r.to, (int)r.n_moves, r.workspace,
                            (uint64_t)r.bytes, r.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyObject* py_paged_select(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {         /* pool, batch, q, sel, sink, local, stream */
  Call c;
  if (n_args != 7 || !call_of(a[0], s_addr, a[1], a[2], a[3], a[6], &c)) Py_RETURN_NONE;
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
  if (n_args != 9 || !call_of(a[0], s_addr, a[1], a[2], a[3], a[8], &c) || !results_of(&c, a[4], a[5], a[6], &r)) Py_RETURN_NONE;
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
  PyObject *device, *stream, *i, *f, *u, *o;
  if (!PyArg_ParseTuple(args, "OOOOOO", &device, &stream, &i, &f, &u, &o)) return NULL;
  hook_device = Py_NewRef(device);                              /* (once a process) */
  hook_stream = Py_NewRef(stream);
  type_int32 = Py_NewRef(i);
  type_float32 = Py_NewRef(f);
  type_uint8 = Py_NewRef(u);
  type_bool = Py_NewRef(o);
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
    {"attention4", (PyCFunction)(void (*)(void))py_paged4_attention, METH_FASTCALL,
     "(pool, batch, q, out, lse | None, workspace, causal, sm_scale, stream | None)"},
    {"store4", (PyCFunction)(void (*)(void))py_paged4_store, METH_FASTCALL, "(pool, k_new, v_new, slot_map, stream | None)"},
    {"load4", (PyCFunction)(void (*)(void))py_paged4_load, METH_FASTCALL, "(pool, k_out, v_out, slot_map, stream | None)"},
    {"move", (PyCFunction)(void (*)(void))py_paged_move, METH_FASTCALL, "(pool, move_from, move_to, stream | None)"},
    {"move4", (PyCFunction)(void (*)(void))py_paged4_move, METH_FASTCALL, "(pool, move_from, move_to, stream | None)"},
    {"fork", (PyCFunction)(void (*)(void))py_paged_fork, METH_FASTCALL,
     "(parents, keep_len | None, lengths, block_table, free_pages, state, lengths_out, table_out, state_out, move_from, move_to, workspace, stream | None)"},
    {"compact", (PyCFunction)(void (*)(void))py_paged_compact, METH_FASTCALL,
     "(stays, lengths, block_table, free_pages, state, lengths_out, table_out, state_out, move_from, move_to, workspace, stream | None)"},
    {"set_hooks", py_set_hooks, METH_VARARGS, "(current_device, raw_stream, torch.int32, torch.float32, torch.uint8, torch.bool)"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__paged(void) {
  static const struct {
    PyObject** at;
    const char* name;
  } names[] = {{&s_data_ptr, "data_ptr"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_numel, "numel"}, {&s_nbytes, "nbytes"},
               {&s_is_contiguous, "is_contiguous"}, {&s_get_device, "get_device"}, {&s_cuda_stream, "cuda_stream"}, {&s_addr, "addr"},
               {&s_addr4, "addr4"}, {&s_device, "device"}, {&s_torch_dtype, "torch_dtype"}};
  for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
    if (!(*names[i].at = PyUnicode_InternFromString(names[i].name))) return NULL;
  return PyModule_Create(&module);
}
