// Argument checks and marshalling, compiled, of the calls that a model's step makes: what binding.py's prefix_prefill_attn
// does with some fifty attribute reads and a ctypes call, 3.6 of the 9.2 us that a call of one launch kept the host busy; the
// operators of a drafted step likewise (small calls, one after another: build_tables 9.3 -> 6.1 us, tree_mask 7.1 -> 4.8,
// tree_attn 11.5 -> 10.7, tree_accept and kv_commit together 17.3 -> 11.4); and those of a step of beam search (3 to 4 us less
// each).  Only the ordinary call is taken (no stream or
// tuning argument, every tensor as the entry point wants it); for anything else, and for every error, the answer is None and
// the general path decides, so that there is one place that says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "symph.h"

// A tensor's description in one call, where this torch has the exchange interface of DLPack for C (the build passes the folder of its
// header), five attributes else: calls of one small launch, kv_fork with its 16 tensors 7.4 -> 4.7 us, kv_free and kv_compact 6.5 -> 4.5
// and 4.9.
#if defined(SYMPH_DLPACK)
#include <dlpack.h>
#endif

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
typedef int32_t (*select_fn)(const void*, int64_t, int32_t, int32_t, int32_t, const float*, const int32_t*, const int32_t*, int32_t,
                             int32_t, int32_t, int32_t, int32_t*, int32_t*, float*, float*, void*, int64_t, void*);
typedef int32_t (*fork_fn)(const int32_t*, int32_t, const int32_t*, const int32_t*, int32_t, const int32_t*, int32_t, int32_t, int32_t,
                           const int32_t*, const int32_t*, int32_t, const int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*,
                           int32_t*, int32_t*, int32_t*, void*);
typedef int32_t (*copy_fn)(const symph_kv_cache*, const int32_t*, const int32_t*, const int32_t*, int32_t, void*);
typedef int32_t (*free_fn)(const int32_t*, const int32_t*, const int32_t*, int32_t, const int32_t*, int32_t, int32_t, int32_t,
                           const int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, const int32_t*, int32_t, const int32_t*,
                           const int32_t*, void*, int64_t, void*);
typedef int32_t (*compact_fn)(const int32_t*, int32_t, int32_t, const int32_t*, const int32_t*, int32_t, const int32_t*, int32_t, int32_t,
                              int32_t*, int32_t*, int32_t*, int32_t*, int32_t*, int32_t, int32_t*, void*, int64_t, void*);

// Set once, by bind(), bind_draft() and bind_beam()
static attn_fn entry;
static tables_fn tables_entry;
static mask_fn mask_entry;
static tree_fn tree_entry;
static accept_fn accept_entry;
static commit_fn commit_entry;
static select_fn select_entry;
static fork_fn fork_entry;
static copy_fn copy_entry;
static free_fn free_entry;
static compact_fn compact_entry;
#if defined(SYMPH_DLPACK)
static const DLPackExchangeAPI* exchange;  // NULL: by attributes
static PyTypeObject* tensor_type;
#endif
static PyObject *t_bf16, *t_fp32, *t_int32, *t_int64, *raw_stream, *get_device;
static PyObject *s_dtype, *s_shape, *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_stride, *s_numel, *s_element_size, *s_get_device;

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

// (after bind() and bind_draft(), whose types these are)
static PyObject* bind_beam(PyObject* self, PyObject* args) {
  unsigned long long a, b, c, d, e;
  PyObject *tensor, *capsule;
  (void)self;
  if (!PyArg_ParseTuple(args, "KKKKKOO", &a, &b, &c, &d, &e, &tensor, &capsule)) return NULL;
#if defined(SYMPH_DLPACK)
  exchange = NULL;
  if (PyType_Check(tensor) && PyCapsule_IsValid(capsule, "dlpack_exchange_api")) {
    const DLPackExchangeAPI* api = (const DLPackExchangeAPI*)PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
    if (api && api->header.version.major == DLPACK_MAJOR_VERSION && api->dltensor_from_py_object_no_sync) {
      Py_INCREF(tensor), Py_INCREF(capsule);  // (both live as long as torch)
      exchange = api, tensor_type = (PyTypeObject*)tensor;
    }
  }
#endif
  select_entry = (select_fn)(uintptr_t)a, fork_entry = (fork_fn)(uintptr_t)b, copy_entry = (copy_fn)(uintptr_t)c;
  free_entry = (free_fn)(uintptr_t)d, compact_entry = (compact_fn)(uintptr_t)e;
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

// ---- beam search: every tensor has to be on the current device ----
typedef struct {
  int64_t device;
  void* stream;
} place;

static int current_place(place* at) {
  PyObject* device = PyObject_CallNoArgs(get_device);
  PyObject* raw = device ? PyObject_CallOneArg(raw_stream, device) : NULL;
  const int ok = raw && PyLong_Check(raw) && as_int(device, &at->device);
  if (ok) at->stream = PyLong_AsVoidPtr(raw);
  Py_XDECREF(raw);
  Py_XDECREF(device);
  return ok && !PyErr_Occurred();
}
// What a tensor is: its n sizes and strides (n < 0: any number, not written down), whether it is dense
typedef struct {
  int64_t sizes[5], strides[5], bytes;
  void* data;
  int dense;
} tensor_at;

#if defined(SYMPH_DLPACK)
static int exchanged(PyObject* t, PyObject* dtype, int n, const place* at, tensor_at* out) {
  DLTensor d;
  if (!PyObject_TypeCheck(t, tensor_type) || exchange->dltensor_from_py_object_no_sync(t, &d) != 0) return 0;
  if (d.device.device_type != kDLROCM || d.device.device_id != at->device || (n >= 0 && d.ndim != n) || d.dtype.lanes != 1) return 0;
  const int bits = d.dtype.bits;
  if (dtype && !(dtype == t_int32   ? d.dtype.code == kDLInt && bits == 32
                 : dtype == t_int64 ? d.dtype.code == kDLInt && bits == 64
                 : dtype == t_fp32  ? d.dtype.code == kDLFloat && bits == 32
                 : dtype == t_bf16  ? d.dtype.code == kDLBfloat && bits == 16
                                    : 0))
    return 0;
  out->dense = 1;
  int64_t count = 1;
  for (int i = d.ndim - 1; i >= 0; --i) {
    if (d.strides && d.shape[i] > 1 && d.strides[i] != count) out->dense = 0;
    if (n >= 0 && i < 5) out->sizes[i] = d.shape[i], out->strides[i] = d.strides ? d.strides[i] : count;
    count *= d.shape[i];
  }
  if (count == 0) out->dense = 1;
  out->bytes = count * ((bits + 7) / 8);
  out->data = (char*)d.data + d.byte_offset;
  return 1;
}
#endif

static int look(PyObject* t, PyObject* dtype, int n, const place* at, tensor_at* out) {
#if defined(SYMPH_DLPACK)
  if (exchange) return exchanged(t, dtype, n, at, out);
#endif
  int64_t device, p, count, size;
  if (!method_int(t, s_get_device, &device) || device != at->device || (dtype && !attr_is(t, s_dtype, dtype))) return 0;
  if (n >= 0 && (!dims(t, s_shape, 0, n, out->sizes) || !dims(t, s_stride, 1, n, out->strides))) return 0;
  PyObject* r = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  out->dense = r == Py_True;
  Py_XDECREF(r);
  if (!method_int(t, s_data_ptr, &p) || !method_int(t, s_numel, &count) || !method_int(t, s_element_size, &size)) return 0;
  out->bytes = count * size;
  out->data = (void*)(uintptr_t)p;
  return 1;
}
static int vector_at(PyObject* t, PyObject* dtype, int64_t least, int optional, const place* at, void** ptr, int64_t* length) {
  tensor_at x;
  if (t == Py_None) {
    *ptr = NULL;
    return optional;
  }
  if (!look(t, dtype, 1, at, &x) || !x.dense || x.sizes[0] < least || x.sizes[0] > INT32_MAX) return 0;
  *ptr = x.data;
  if (length) *length = x.sizes[0];
  return 1;
}
// An int32 [>= rows][stride] table; stride < 0: any, which becomes it
static int table_at(PyObject* t, int64_t rows, int64_t* stride, const place* at, void** ptr) {
  tensor_at x;
  if (!look(t, t_int32, 2, at, &x) || !x.dense || x.sizes[0] < rows || x.sizes[1] > INT32_MAX || (*stride >= 0 && x.sizes[1] != *stride))
    return 0;
  *stride = x.sizes[1];
  *ptr = x.data;
  return 1;
}
static int scratch_at(PyObject* t, const place* at, void** ptr, int64_t* bytes) {
  tensor_at x;
  *ptr = NULL, *bytes = 0;
  if (t == Py_None) return 1;
  if (!look(t, NULL, -1, at, &x) || !x.dense) return 0;
  *ptr = x.data, *bytes = x.bytes;
  return 1;
}
// The pools of a cache on the current device
static int pools_at(PyObject* k, PyObject* v, const place* at, symph_kv_cache* c) {
  tensor_at x, y;
  const int wide = look(k, t_fp32, 5, at, &x);
  if (!wide) PyErr_Clear();
  if ((!wide && !look(k, t_bf16, 5, at, &x)) || !look(v, wide ? t_fp32 : t_bf16, 5, at, &y)) return 0;
  for (int i = 0; i < 5; ++i)
    if (x.sizes[i] > INT32_MAX) return 0;
  c->k_base = x.data, c->v_base = y.data;
  c->layer_stride = x.strides[0], c->block_stride = x.strides[1];
  c->n_layers = (int32_t)x.sizes[0], c->n_blocks = (int32_t)x.sizes[1], c->block_size = (int32_t)x.sizes[2];
  c->n_kv_heads = (int32_t)x.sizes[3], c->head_dim = (int32_t)x.sizes[4];
  c->dtype = wide ? SYMPH_FP32 : SYMPH_BF16;
  return 1;
}

// (logits, scores, cu_rows, cu_next, max_next, parents, tokens, next_scores, end_token, end_scores, workspace) -> status or None
static PyObject* select_beams(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  place at;
  tensor_at x;
  int64_t n, total, ws_bytes;
  int32_t most, end, status, wide = 0;
  void *scores, *cu, *cu_next, *parents, *tokens, *best, *ends, *ws;
  if (n_args != 11 || !select_entry || !current_place(&at) ||
      (!look(a[0], t_bf16, 2, &at, &x) && (PyErr_Clear(), !(wide = look(a[0], t_fp32, 2, &at, &x)))) || x.sizes[0] > INT32_MAX ||
      x.sizes[1] > INT32_MAX || (x.sizes[1] > 1 && x.strides[1] != 1) || (x.sizes[0] > 1 && x.strides[0] < x.sizes[1]) ||
      !vector_at(a[1], t_fp32, x.sizes[0], 0, &at, &scores, NULL) || !vector_at(a[2], t_int32, 1, 0, &at, &cu, &n) || (n -= 1) < 0 ||
      !vector_at(a[3], t_int32, n + 1, 0, &at, &cu_next, NULL) || !as_int32(a[4], &most) ||
      !vector_at(a[5], t_int32, 0, 0, &at, &parents, &total) || !vector_at(a[6], t_int32, total, 0, &at, &tokens, NULL) ||
      !vector_at(a[7], t_fp32, total, 0, &at, &best, NULL) || !as_int32(a[8], &end) ||
      !vector_at(a[9], t_fp32, x.sizes[0], 1, &at, &ends, NULL) || !scratch_at(a[10], &at, &ws, &ws_bytes)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = select_entry(x.data, x.sizes[0] > 1 ? x.strides[0] : x.sizes[1], wide ? SYMPH_FP32 : SYMPH_BF16, (int32_t)x.sizes[0],
                        (int32_t)x.sizes[1], scores, cu, cu_next, (int32_t)n, (int32_t)total, most, end, parents, tokens, best, ends, ws,
                        ws_bytes, at.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (parents, lens, block_table, refs, free_blocks, block_size, table_out, lens_out, refs_after, copy_src, copy_dst, copy_tokens,
// held_blocks, held_out, free_begin, blocks_taken) -> status or None
static PyObject* fork_rows(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  place at;
  int64_t out, n, blocks, n_free, stride = -1;
  int32_t bs, status;
  void *parents, *lens, *table, *refs, *list, *to, *lens_out, *after, *src, *dst, *count, *held, *held_out, *begin, *taken;
  if (n_args != 16 || !fork_entry || !current_place(&at) || !vector_at(a[0], t_int32, 0, 0, &at, &parents, &out) ||
      !vector_at(a[1], t_int32, 0, 0, &at, &lens, &n) || !table_at(a[2], n, &stride, &at, &table) ||
      !vector_at(a[3], t_int32, 0, 0, &at, &refs, &blocks) || !vector_at(a[4], t_int32, 0, 0, &at, &list, &n_free) ||
      !as_int32(a[5], &bs) || !table_at(a[6], out, &stride, &at, &to) || !vector_at(a[7], t_int32, out, 0, &at, &lens_out, NULL) ||
      !vector_at(a[8], t_int32, blocks, 0, &at, &after, NULL) || !vector_at(a[9], t_int32, out, 0, &at, &src, NULL) ||
      !vector_at(a[10], t_int32, out, 0, &at, &dst, NULL) || !vector_at(a[11], t_int32, out, 0, &at, &count, NULL) ||
      !vector_at(a[12], t_int32, n, 1, &at, &held, NULL) || !vector_at(a[13], t_int32, out, 1, &at, &held_out, NULL) ||
      !vector_at(a[14], t_int32, 1, 1, &at, &begin, NULL) || !vector_at(a[15], t_int32, 1, 1, &at, &taken, NULL)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = fork_entry(parents, (int32_t)out, lens, held, (int32_t)n, table, (int32_t)stride, bs, (int32_t)blocks, refs, list,
                      (int32_t)n_free, begin, to, lens_out, held_out, after, src, dst, count, taken, at.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (k_pool, v_pool, src_blocks, dst_blocks, tokens) -> status or None
static PyObject* copy_blocks(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  place at;
  symph_kv_cache c;
  int64_t n;
  int32_t status;
  void *src, *dst, *count;
  if (n_args != 5 || !copy_entry || !current_place(&at) || !pools_at(a[0], a[1], &at, &c) ||
      !vector_at(a[2], t_int32, 0, 0, &at, &src, &n) || !vector_at(a[3], t_int32, n, 0, &at, &dst, NULL) ||
      !vector_at(a[4], t_int32, n, 1, &at, &count, NULL)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = copy_entry(&c, src, dst, count, (int32_t)n, at.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (drop, lens, block_table, refs, block_size, refs_after, free_blocks, n_free, held_blocks, lens_after, held_after, workspace,
// taken_blocks, taken_begin, taken_end) -> status or None
static PyObject* free_rows(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  place at;
  int64_t n, blocks, ws_bytes, n_taken = 0, stride = -1;
  int32_t bs, status;
  void *taken, *taken_begin, *taken_end;
  void *drop, *lens, *table, *refs, *after, *list, *count, *held, *lens_after, *held_after, *ws;
  if (n_args != 15 || !free_entry || a[0] == Py_None || !current_place(&at) || !vector_at(a[0], t_int32, 1, 0, &at, &drop, &n) ||
      !vector_at(a[1], t_int32, n, 0, &at, &lens, NULL) || !table_at(a[2], n, &stride, &at, &table) ||
      !vector_at(a[3], t_int32, 0, 0, &at, &refs, &blocks) || !as_int32(a[4], &bs) ||
      !vector_at(a[5], t_int32, blocks, 0, &at, &after, NULL) || !vector_at(a[6], t_int32, blocks, 0, &at, &list, NULL) ||
      !vector_at(a[7], t_int32, 1, 0, &at, &count, NULL) || !vector_at(a[8], t_int32, n, 1, &at, &held, NULL) ||
      !vector_at(a[9], t_int32, n, 1, &at, &lens_after, NULL) || !vector_at(a[10], t_int32, n, 1, &at, &held_after, NULL) ||
      !scratch_at(a[11], &at, &ws, &ws_bytes) || !vector_at(a[12], t_int32, 0, 1, &at, &taken, &n_taken) ||
      !vector_at(a[13], t_int32, 1, 1, &at, &taken_begin, NULL) ||
      !vector_at(a[14], t_int32, 1, a[12] == Py_None, &at, &taken_end, NULL)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = free_entry(drop, lens, held, (int32_t)n, table, (int32_t)stride, bs, (int32_t)blocks, refs, after, list, count, lens_after,
                      held_after, taken, (int32_t)n_taken, taken_begin, taken_end, ws, ws_bytes, at.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (refs, n_keep, lens, block_table, block_size, table_out, refs_after, block_map, copy_src, copy_dst, counts, held_blocks, workspace)
// -> status or None
static PyObject* compact_pool(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  place at;
  int64_t n, blocks, pairs, ws_bytes, stride = -1;
  int32_t keep, bs, status;
  void *refs, *lens, *table, *to, *after, *map, *src, *dst, *counts, *held, *ws;
  if (n_args != 13 || !compact_entry || !current_place(&at) || !vector_at(a[0], t_int32, 0, 0, &at, &refs, &blocks) ||
      !as_int32(a[1], &keep) || !vector_at(a[2], t_int32, 0, 0, &at, &lens, &n) || !table_at(a[3], n, &stride, &at, &table) ||
      !as_int32(a[4], &bs) || !table_at(a[5], n, &stride, &at, &to) || !vector_at(a[6], t_int32, blocks, 0, &at, &after, NULL) ||
      !vector_at(a[7], t_int32, blocks, 0, &at, &map, NULL) || !vector_at(a[8], t_int32, 0, 0, &at, &src, &pairs) ||
      !vector_at(a[9], t_int32, pairs, 0, &at, &dst, NULL) || !vector_at(a[10], t_int32, 3, 0, &at, &counts, NULL) ||
      !vector_at(a[11], t_int32, n, 1, &at, &held, NULL) || !scratch_at(a[12], &at, &ws, &ws_bytes)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  Py_BEGIN_ALLOW_THREADS
  status = compact_entry(refs, (int32_t)blocks, keep, lens, held, (int32_t)n, table, (int32_t)stride, bs, to, after, map, src, dst,
                         (int32_t)pairs, counts, ws, ws_bytes, at.stream);
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
    {"bind_beam", bind_beam, METH_VARARGS, "bind_beam(addresses of beam_select, kv_fork, kv_copy_blocks, kv_free, kv_compact, torch.Tensor, its exchange capsule or None)"},
    {"select_beams", (PyCFunction)(void (*)(void))select_beams, METH_FASTCALL, "beam_select, likewise"},
    {"fork_rows", (PyCFunction)(void (*)(void))fork_rows, METH_FASTCALL, "kv_fork, likewise"},
    {"copy_blocks", (PyCFunction)(void (*)(void))copy_blocks, METH_FASTCALL, "kv_copy_blocks, likewise"},
    {"free_rows", (PyCFunction)(void (*)(void))free_rows, METH_FASTCALL, "kv_free, likewise"},
    {"compact_pool", (PyCFunction)(void (*)(void))compact_pool, METH_FASTCALL, "kv_compact, likewise"},
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
  s_get_device = PyUnicode_InternFromString("get_device");
  if (!s_dtype || !s_shape || !s_is_cuda || !s_is_contiguous || !s_data_ptr || !s_stride || !s_numel || !s_element_size || !s_get_device)
    return NULL;
  return PyModule_Create(&module);
}
