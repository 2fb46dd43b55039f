// Argument checks and marshalling, compiled, of the calls that a model's step makes: what binding.py's prefix_prefill_attn
// does with some fifty attribute reads and a ctypes call, 3.6 of the 9.2 us that a call of one launch kept the host busy; the
// operators of a drafted step likewise (small calls, one after another: build_tables 9.3 -> 6.1 us, tree_mask 7.1 -> 4.8,
// tree_attn 11.5 -> 10.7, tree_accept and kv_commit together 17.3 -> 11.4).  Only the ordinary call is taken (no stream or
// tuning argument, every tensor as the entry point wants it); for anything else, and for every error, the answer is None and
// the general path decides, so that there is one place that says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "symph.h"

typedef int32_t (*attn_fn)(const symph_kv_cache*, int32_t, const void*, const void*, const void*, void*, const int32_t*,
                           const int32_t*, const int32_t*, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, float, void*,
                           int64_t, void*);

typedef int32_t (*tables_fn)(const int32_t*, const int32_t*, const int32_t*, int32_t, int32_t*, int32_t, const int32_t*, int32_t,
                             const int32_t*, int32_t, int32_t, int64_t, int32_t*, int64_t*, int64_t*, int32_t*, int32_t*, int32_t*,
                             void*);
typedef int32_t (*mask_fn)(const int32_t*, const int32_t*, const int32_t*, int32_t, int32_t, int32_t, uint64_t*, int32_t, int32_t*,
                           void*);
typedef int32_t (*tree_fn)(const symph_kv_cache*, int32_t, const void*, const void*, const void*, void*, const uint64_t*, int32_t,
                           const int32_t*, const int32_t*, const int32_t*, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t,
                           float, void*, int64_t, void*);
typedef int32_t (*accept_fn)(const int32_t*, const int32_t*, const int32_t*, const int32_t*, const int32_t*, int32_t, int32_t,
                             int32_t*, int32_t*, int32_t*, int32_t*, void*);
typedef int32_t (*commit_fn)(const symph_kv_cache*, const void*, const void*, int32_t, const int32_t*, const int64_t*, int32_t,
                             void*);

// Set once, by bind() and bind_draft()
static attn_fn entry;
static tables_fn tables_entry;
static mask_fn mask_entry;
static tree_fn tree_entry;
static accept_fn accept_entry;
static commit_fn commit_entry;
static PyObject *t_bf16, *t_fp32, *t_int32, *t_int64, *raw_stream, *get_device;
static PyObject *s_dtype, *s_shape, *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_stride, *s_numel, *s_element_size;

static PyObject* bind(PyObject* self, PyObject* args) {
  unsigned long long address;
  PyObject *a, *b, *c, *d, *e;
  (void)self;
  if (!PyArg_ParseTuple(args, "KOOOOO", &address, &a, &b, &c, &d, &e)) return NULL;
  Py_INCREF(a), Py_INCREF(b), Py_INCREF(c), Py_INCREF(d), Py_INCREF(e);
  Py_XDECREF(t_bf16), Py_XDECREF(t_fp32), Py_XDECREF(t_int32), Py_XDECREF(raw_stream), Py_XDECREF(get_device);
  t_bf16 = a, t_fp32 = b, t_int32 = c, raw_stream = d, get_device = e;
  entry = (attn_fn)(uintptr_t)address;
  Py_RETURN_NONE;
}

// (after bind(): the types and the stream's source are the same)
static PyObject* bind_draft(PyObject* self, PyObject* args) {
  unsigned long long a, b, c, d, e;
  PyObject* i64;
  (void)self;
  if (!PyArg_ParseTuple(args, "KKKKKO", &a, &b, &c, &d, &e, &i64)) return NULL;
  Py_INCREF(i64), Py_XDECREF(t_int64);
  t_int64 = i64;
  tables_entry = (tables_fn)(uintptr_t)a, mask_entry = (mask_fn)(uintptr_t)b, tree_entry = (tree_fn)(uintptr_t)c;
  accept_entry = (accept_fn)(uintptr_t)d, commit_entry = (commit_fn)(uintptr_t)e;
  Py_RETURN_NONE;
}

// Each of these returns 1, or 0 where the general path has to look (an exception may be set; the caller clears it).
static int as_int(PyObject* o, int64_t* out) {
  if (!o || !PyLong_CheckExact(o)) return 0;
  *out = PyLong_AsLongLong(o);
  return !(*out == -1 && PyErr_Occurred());
}
static int as_int32(PyObject* o, int32_t* out) {
  int64_t v;
  if (!as_int(o, &v) || v < INT32_MIN || v > INT32_MAX) return 0;
  *out = (int32_t)v;
  return 1;
}
static int method_int(PyObject* t, PyObject* name, int64_t* out) {
  PyObject* r = PyObject_CallMethodNoArgs(t, name);
  const int ok = as_int(r, out);
  Py_XDECREF(r);
  return ok;
}
static int attr_is(PyObject* t, PyObject* name, PyObject* want) {
  PyObject* r = PyObject_GetAttr(t, name);
  const int ok = r == want;
  Py_XDECREF(r);
  return ok;
}
static int dims(PyObject* t, PyObject* name, int call, int n, int64_t* out) {  // the n values of .shape / .stride()
  PyObject* r = call ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
  int ok = r && PyTuple_Check(r) && PyTuple_GET_SIZE(r) == n;
  for (int i = 0; ok && i < n; ++i) ok = as_int(PyTuple_GET_ITEM(r, i), out + i);
  Py_XDECREF(r);
  return ok;
}
// On the device, contiguous, of the element type (NULL: any)
static int dense(PyObject* t, PyObject* dtype, void** ptr) {
  if (!attr_is(t, s_is_cuda, Py_True) || (dtype && !attr_is(t, s_dtype, dtype))) return 0;
  PyObject* r = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  const int ok = r == Py_True;
  Py_XDECREF(r);
  int64_t p;
  if (!ok || !method_int(t, s_data_ptr, &p)) return 0;
  *ptr = (void*)(uintptr_t)p;
  return 1;
}

// (k_pool, v_pool, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table, max_new_len, max_prefix_len, scale,
// workspace) -> status or None
enum { kKPool, kVPool, kLayer, kQ, kKNew, kVNew, kOut, kCu, kLens, kTable, kMaxNew, kMaxPrefix, kScale, kWorkspace, kArgs };

typedef struct {
  symph_kv_cache cache;
  int32_t ints[7];  // layer, table stride, sessions, query heads, tokens, max_new_len, max_prefix_len
  float scale;
  void *ptrs[8], *stream;
  int64_t ws_bytes;
  int64_t q[3], k_new[3], table_rows;
} attn_args;

static int describe(PyObject* k_pool, PyObject* v_pool, PyObject** dtype, symph_kv_cache* c) {
  int64_t pool[5], strides[5], v;
  PyObject* dt = PyObject_GetAttr(k_pool, s_dtype);
  Py_XDECREF(dt);  // (torch's dtypes live as long as the module)
  if (dt != t_bf16 && dt != t_fp32) return 0;
  if (!dims(k_pool, s_shape, 0, 5, pool) || !dims(k_pool, s_stride, 1, 5, strides)) return 0;
  for (int i = 0; i < 5; ++i)
    if (pool[i] > INT32_MAX) return 0;
  if (!method_int(k_pool, s_data_ptr, &v)) return 0;
  c->k_base = (void*)(uintptr_t)v;
  if (!method_int(v_pool, s_data_ptr, &v)) return 0;
  c->v_base = (void*)(uintptr_t)v;
  c->layer_stride = strides[0], c->block_stride = strides[1];
  c->n_layers = (int32_t)pool[0], c->n_blocks = (int32_t)pool[1], c->block_size = (int32_t)pool[2];
  c->n_kv_heads = (int32_t)pool[3], c->head_dim = (int32_t)pool[4];
  c->dtype = dt == t_bf16 ? SYMPH_BF16 : SYMPH_FP32;
  *dtype = dt;
  return 1;
}

// The current stream of the current device
static int current_stream(void** stream) {
  PyObject* device = PyObject_CallNoArgs(get_device);
  PyObject* raw = device ? PyObject_CallOneArg(raw_stream, device) : NULL;
  const int ok = raw && PyLong_Check(raw);
  if (ok) *stream = PyLong_AsVoidPtr(raw);
  Py_XDECREF(raw);
  Py_XDECREF(device);
  return ok && !PyErr_Occurred();
}

static int gather(PyObject* const* a, attn_args* x) {
  int64_t o[3], vn[3], table[2] = {0, 0}, sessions;
  PyObject* dt;
  if (!describe(a[kKPool], a[kVPool], &dt, &x->cache)) return 0;
  if (!dims(a[kQ], s_shape, 0, 3, x->q) || !dims(a[kOut], s_shape, 0, 3, o) || !dims(a[kKNew], s_shape, 0, 3, x->k_new) ||
      !dims(a[kVNew], s_shape, 0, 3, vn))
    return 0;
  for (int i = 0; i < 3; ++i)
    if (x->q[i] != o[i] || x->k_new[i] != vn[i] || x->q[i] > INT32_MAX) return 0;
  void** const ptrs = x->ptrs;
  if (!dense(a[kQ], dt, ptrs + 0) || !dense(a[kKNew], dt, ptrs + 1) || !dense(a[kVNew], dt, ptrs + 2) ||
      !dense(a[kOut], dt, ptrs + 3) || !dense(a[kCu], t_int32, ptrs + 4) || !dense(a[kLens], t_int32, ptrs + 5))
    return 0;
  ptrs[6] = NULL;
  if (a[kTable] != Py_None &&
      (!dims(a[kTable], s_shape, 0, 2, table) || table[1] > INT32_MAX || !dense(a[kTable], t_int32, ptrs + 6)))
    return 0;
  if (!dims(a[kLens], s_shape, 0, 1, &sessions) || sessions > INT32_MAX) return 0;
  int32_t* const ints = x->ints;
  ints[1] = (int32_t)table[1], ints[2] = (int32_t)sessions, ints[3] = (int32_t)x->q[1], ints[4] = (int32_t)x->q[0];
  x->table_rows = table[0];
  if (!as_int32(a[kLayer], ints) || !as_int32(a[kMaxNew], ints + 5) || !as_int32(a[kMaxPrefix], ints + 6)) return 0;
  if (!PyFloat_CheckExact(a[kScale])) return 0;
  x->scale = (float)PyFloat_AS_DOUBLE(a[kScale]);
  ptrs[7] = NULL;
  x->ws_bytes = 0;
  if (a[kWorkspace] != Py_None) {
    int64_t n, e;
    if (!dense(a[kWorkspace], NULL, ptrs + 7) || !method_int(a[kWorkspace], s_numel, &n) ||
        !method_int(a[kWorkspace], s_element_size, &e))
      return 0;
    x->ws_bytes = n * e;
  }
  return current_stream(&x->stream);
}

static PyObject* attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  attn_args x;
  int32_t status;
  if (n != kArgs || !entry || !gather(a, &x)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = entry(&x.cache, x.ints[0], x.ptrs[0], x.ptrs[1], x.ptrs[2], x.ptrs[3], x.ptrs[4], x.ptrs[5], x.ptrs[6], x.ints[1],
                 x.ints[2], x.ints[3], x.ints[4], x.ints[5], x.ints[6], x.scale, x.ptrs[7], x.ws_bytes, x.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// A 1-D tensor of at least `least` entries; None is a null pointer where that is allowed.  `length`: its entries, or NULL
static int vector(PyObject* t, PyObject* dtype, int64_t least, int optional, void** ptr, int64_t* length) {
  int64_t n;
  if (t == Py_None) {
    *ptr = NULL;
    return optional;
  }
  if (!dims(t, s_shape, 0, 1, &n) || n < least || n > INT32_MAX || !dense(t, dtype, ptr)) return 0;
  if (length) *length = n;
  return 1;
}
// The int64 [rows][words] mask
static int words_of(PyObject* t, int64_t rows, void** ptr, int64_t* words) {
  int64_t d[2];
  if (!dims(t, s_shape, 0, 2, d) || d[0] < rows || d[1] > INT32_MAX || !dense(t, t_int64, ptr)) return 0;
  *words = d[1];
  return 1;
}

// (as attn, then tree_mask)
static PyObject* tree(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  (void)self;
  attn_args x;
  int64_t words, n_cu;
  int32_t status;
  void* mask;
  if (n != kArgs + 1 || !tree_entry || !gather(a, &x) || !words_of(a[kArgs], x.q[0], &mask, &words) ||
      x.q[2] != x.cache.head_dim || x.k_new[0] != x.q[0] || x.k_new[1] != x.cache.n_kv_heads || x.k_new[2] != x.q[2] ||
      !dims(a[kCu], s_shape, 0, 1, &n_cu) || n_cu < (int64_t)x.ints[2] + 1 || (x.ptrs[6] && x.table_rows < x.ints[2])) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = tree_entry(&x.cache, x.ints[0], x.ptrs[0], x.ptrs[1], x.ptrs[2], x.ptrs[3], mask, (int32_t)words, x.ptrs[4], x.ptrs[5],
                      x.ptrs[6], x.ints[1], x.ints[2], x.ints[3], x.ints[4], x.ints[5], x.ints[6], x.scale, x.ptrs[7], x.ws_bytes,
                      x.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (prefix_lens, new_lens, block_table, free_blocks, block_size, n_blocks, total_new_tokens, cu_new_lens, token_offsets, slot_map,
// positions, blocks_taken, held_blocks, held_after, free_begin) -> status or None
static PyObject* tables(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  int64_t n, n_free, total, table[2] = {0, 0};
  int32_t block_size, n_blocks, status;
  void *lens, *news, *tab = NULL, *free_list, *cu, *offsets, *slots, *pos, *taken, *held, *after, *begin, *stream;
  if (n_args != 15 || !tables_entry || !vector(a[0], t_int32, 0, 0, &lens, &n) || !vector(a[1], t_int32, n, 0, &news, NULL) ||
      (a[2] != Py_None &&
       (!dims(a[2], s_shape, 0, 2, table) || table[0] < n || table[1] > INT32_MAX || !dense(a[2], t_int32, &tab))) ||
      !vector(a[3], t_int32, 0, 0, &free_list, &n_free) || !as_int32(a[4], &block_size) || !as_int32(a[5], &n_blocks) ||
      !as_int(a[6], &total) || !vector(a[7], t_int32, n + 1, 1, &cu, NULL) || !vector(a[8], t_int64, n + 1, 1, &offsets, NULL) ||
      !vector(a[9], t_int64, total, 1, &slots, NULL) || !vector(a[10], t_int32, total, 1, &pos, NULL) ||
      !vector(a[11], t_int32, 1, 1, &taken, NULL) || !vector(a[12], t_int32, n, 1, &held, NULL) ||
      !vector(a[13], t_int32, n, 1, &after, NULL) || !vector(a[14], t_int32, 1, 1, &begin, NULL) || !current_stream(&stream)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = tables_entry(lens, news, held, (int32_t)n, tab, (int32_t)table[1], free_list, (int32_t)n_free, begin, block_size,
                        n_blocks, total, cu, offsets, slots, pos, taken, after, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (parents, cu_new_lens, max_new_len, mask, prefix_lens, positions) -> status or None
static PyObject* mask(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  int64_t t, n_cu, words;
  int32_t most, status;
  void *parents, *cu, *bits, *lens, *pos, *stream;
  if (n_args != 6 || !mask_entry || !vector(a[0], t_int32, 0, 0, &parents, &t) || !vector(a[1], t_int32, 1, 0, &cu, &n_cu) ||
      !as_int32(a[2], &most) || !words_of(a[3], t, &bits, &words) || !vector(a[4], t_int32, n_cu - 1, 1, &lens, NULL) ||
      !vector(a[5], t_int32, t, 1, &pos, NULL) || !current_stream(&stream)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = mask_entry(parents, cu, lens, (int32_t)(n_cu - 1), (int32_t)t, most, bits, (int32_t)words, pos, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (draft_tokens, parents, target_tokens, cu_new_lens, prefix_lens, rows, n_accepted, next_tokens, new_prefix_lens) -> status
// or None
static PyObject* accept(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  int64_t t, n;
  int32_t status;
  void *draft, *parents, *target, *cu, *lens, *rows, *count, *next, *after, *stream;
  if (n_args != 9 || !accept_entry || !vector(a[0], t_int32, 0, 0, &draft, &t) || !vector(a[1], t_int32, t, 0, &parents, NULL) ||
      !vector(a[2], t_int32, t, 0, &target, NULL) || !vector(a[3], t_int32, 1, 0, &cu, &n) || (n -= 1) < 0 ||
      !vector(a[4], t_int32, n, 1, &lens, NULL) || !vector(a[5], t_int32, t, 0, &rows, NULL) ||
      !vector(a[6], t_int32, n, 0, &count, NULL) || !vector(a[7], t_int32, n, 0, &next, NULL) ||
      !vector(a[8], t_int32, n, 1, &after, NULL) || !current_stream(&stream)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = accept_entry(draft, parents, target, cu, lens, (int32_t)n, (int32_t)t, rows, count, next, after, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (k_pool, v_pool, k_new, v_new, rows, slot_map) -> status or None
static PyObject* commit(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  symph_kv_cache c;
  int64_t kn[4], vn[4], n;
  int32_t status;
  PyObject* dt;
  void *k, *v, *rows, *slots, *stream;
  if (n_args != 6 || !commit_entry || !describe(a[0], a[1], &dt, &c) || !dims(a[2], s_shape, 0, 4, kn) ||
      !dims(a[3], s_shape, 0, 4, vn) || kn[0] != vn[0] || kn[1] != vn[1] || kn[2] != vn[2] || kn[3] != vn[3] ||
      kn[0] != c.n_layers || kn[1] > INT32_MAX || kn[2] != c.n_kv_heads || kn[3] != c.head_dim || !dense(a[2], dt, &k) ||
      !dense(a[3], dt, &v) || !vector(a[4], t_int32, 0, 0, &rows, &n) || !vector(a[5], t_int64, n, 0, &slots, NULL) ||
      !current_stream(&stream)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = commit_entry(&c, k, v, (int32_t)kn[1], rows, slots, (int32_t)n, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "bind(address of the entry point, bfloat16, float32, int32, raw stream of a device, current device)"},
    {"attn", (PyCFunction)(void (*)(void))attn, METH_FASTCALL, "status of the call, or None where the general path has to make it"},
    {"bind_draft", bind_draft, METH_VARARGS, "bind_draft(addresses of build_tables, tree_mask, tree_attn, tree_accept, kv_commit, int64)"},
    {"tree", (PyCFunction)(void (*)(void))tree, METH_FASTCALL, "tree_attn, likewise"},
    {"tables", (PyCFunction)(void (*)(void))tables, METH_FASTCALL, "build_tables, likewise"},
    {"mask", (PyCFunction)(void (*)(void))mask, METH_FASTCALL, "tree_mask, likewise"},
    {"accept", (PyCFunction)(void (*)(void))accept, METH_FASTCALL, "tree_accept, likewise"},
    {"commit", (PyCFunction)(void (*)(void))commit, METH_FASTCALL, "kv_commit, likewise"},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attn_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__attn_call(void) {
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_stride = PyUnicode_InternFromString("stride");
  s_numel = PyUnicode_InternFromString("numel");
  s_element_size = PyUnicode_InternFromString("element_size");
  if (!s_dtype || !s_shape || !s_is_cuda || !s_is_contiguous || !s_data_ptr || !s_stride || !s_numel || !s_element_size)
    return NULL;
  return PyModule_Create(&module);
}
