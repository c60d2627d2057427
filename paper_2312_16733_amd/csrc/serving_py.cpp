// Python's side of the autoregressive serving operators: checks of tensors, outputs and workspaces from torch's allocator, and
// the C entries of include/subnetact.h on the current stream.  In C++ because a decode step of a few requests is shorter than
// its own marshalling: with ctypes an append took 20 us of the host and an attention 14, of which the launch itself is 4.
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime.h>
#include <structmember.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>

#include <string>

#include "../../include/subnetact.h"

namespace {

PyObject* sna_error = nullptr;             // SnaError of the package

// What the tensors were when the object was made.  A tensor can be given other memory or another shape in place (resize_, set_,
// .data), so every call looks at them again and refuses what has changed.
struct Cache {
  PyObject_HEAD
  PyObject *k_pages, *v_pages;
  at::ScalarType type;
  c10::Device* device;
  sna_paged_cache c;
};
struct Batch {
  PyObject_HEAD
  PyObject *starts, *lens, *page_table;
  c10::Device* device;
  sna_paged_batch c;
};
PyTypeObject *cache_type = nullptr, *batch_type = nullptr;

// ---- refusals: text is made only for one that is refused -----------------------------------------------------------------
#define NEED(ok, ...)                            \
  do {                                           \
    if (!(ok)) {                                 \
      PyErr_Format(PyExc_ValueError, __VA_ARGS__); \
      return 0;                                  \
    }                                            \
  } while (0)

std::string shape_of(const at::Tensor& t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ") of " + c10::toString(t.scalar_type()) + " on " + t.device().str();
}
const at::Tensor* tensor_of(PyObject* o, const char* name) {
  if (!o || !THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: a tensor is needed, got %s", name, o ? Py_TYPE(o)->tp_name : "nothing");
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}
bool none(PyObject* o) { return !o || o == Py_None; }
int status(int64_t st) {                   // 0: an exception is set
  if (st >= 0) return 1;
  PyObject* e = PyObject_CallFunction(sna_error, "is", (int)st, sna_last_error());
  if (e) {
    PyErr_SetObject(sna_error, e);
    Py_DECREF(e);
  }
  return 0;
}
bool whole_number(PyObject* o, int64_t* v) {
  if (none(o)) return true;
  *v = PyLong_AsLongLong(o);
  return !(*v == -1 && PyErr_Occurred());
}
bool real_number(PyObject* o, double* v) {
  if (none(o)) return true;
  *v = PyFloat_AsDouble(o);
  return !(*v == -1.0 && PyErr_Occurred());
}

// Positional and keyword arguments in the order of `names`; false: an exception is set
template <int N>
bool arguments(const char* fn, const char* const (&names)[N], int required, PyObject* const* args, Py_ssize_t n, PyObject* kw, PyObject* (&out)[N]) {
  if (n > N) {
    PyErr_Format(PyExc_TypeError, "%s takes at most %d arguments, got %zd", fn, N, n);
    return false;
  }
  for (int i = 0; i < N; ++i) out[i] = i < n ? args[i] : nullptr;
  for (Py_ssize_t j = 0; kw && j < PyTuple_GET_SIZE(kw); ++j) {
    PyObject* name = PyTuple_GET_ITEM(kw, j);
    int i = 0;
    while (i < N && PyUnicode_CompareWithASCIIString(name, names[i])) ++i;
    if (i == N || out[i]) {
      PyErr_Format(PyExc_TypeError, "%s: %s argument %U", fn, i == N ? "unknown" : "repeated", name);
      return false;
    }
    out[i] = args[n + j];
  }
  for (int i = 0; i < required; ++i)
    if (!out[i]) {
      PyErr_Format(PyExc_TypeError, "%s: argument %s is missing", fn, names[i]);
      return false;
    }
  return true;
}

// The device of the tensors, and the stream that the call is enqueued on and its outputs belong to: the current one, or the
// one that is asked for (a torch stream or a raw handle), made the current one meanwhile.
class On {
 public:
  bool begin(PyObject* stream, c10::DeviceIndex device) {
    int now = 0;
    if (hipGetDevice(&now) == hipSuccess && now != device) {
      was_device_ = now;
      if (hipSetDevice(device) != hipSuccess) {
        PyErr_SetString(PyExc_RuntimeError, "hipSetDevice");
        return false;
      }
    }
    if (!none(stream)) {
      PyObject* handle = PyLong_Check(stream) ? Py_NewRef(stream) : PyObject_GetAttrString(stream, "cuda_stream");
      if (!handle) return false;
      void* raw = PyLong_AsVoidPtr(handle);
      Py_DECREF(handle);
      if (PyErr_Occurred()) return false;
      was_ = c10::hip::getCurrentHIPStream(device);
      c10::hip::setCurrentHIPStream(c10::hip::getStreamFromExternal((hipStream_t)raw, device));
    }
    raw_ = c10::hip::getCurrentHIPStream(device).stream();
    return true;
  }
  void* raw() const { return raw_; }
  ~On() {
    if (was_) c10::hip::setCurrentHIPStream(*was_);
    if (was_device_ >= 0) (void)hipSetDevice(was_device_);
  }

 private:
  int was_device_ = -1;
  std::optional<c10::hip::HIPStream> was_;
  hipStream_t raw_ = nullptr;
};

// ---- PagedCache, PagedBatch ------------------------------------------------------------------------------------------------
int describe_cache(PyObject* ko, PyObject* vo, sna_paged_cache* c) {
  const at::Tensor *k = tensor_of(ko, "k_pages"), *v = k ? tensor_of(vo, "v_pages") : nullptr;
  if (!v) return 0;
  NEED(k->dim() == 4 && v->dim() == 4, "k_pages and v_pages have four dimensions");
  const int64_t n = k->size(0), h = k->size(1), ps = k->size(2), d = k->size(3);
  NEED(v->size(0) == n && v->size(1) == h && v->size(2) == d && v->size(3) == ps, "v_pages: (%lld, %lld, %lld, %lld) is needed, got %s", (long long)n, (long long)h,
       (long long)d, (long long)ps, shape_of(*v).c_str());
  const at::ScalarType t = k->scalar_type();
  NEED((t == at::kBFloat16 || t == at::kHalf) && v->scalar_type() == t, "pages: both bf16 or both fp16 are needed, got %s and %s", c10::toString(t), c10::toString(v->scalar_type()));
  NEED(k->is_cuda() && v->device() == k->device(), "pages on %s and %s: one GPU is needed", k->device().str().c_str(), v->device().str().c_str());
  NEED(n >= 1 && n <= INT32_MAX && h >= 1 && h <= 4096 && ps <= 1024 && d <= 1024, "k_pages: %s is out of range", shape_of(*k).c_str());
  NEED(k->stride(3) == 1 && k->stride(2) == d && (h == 1 || k->stride(1) == ps * d) && v->stride(3) == 1 && v->stride(2) == ps && (h == 1 || v->stride(1) == d * ps), "pages have to be dense");
  const int64_t dense = h * ps * d;
  *c = sna_paged_cache{k->data_ptr(), v->data_ptr(), n > 1 ? k->stride(0) : dense, n > 1 ? v->stride(0) : dense, (int32_t)n, (int32_t)h, (int32_t)ps, (int32_t)d,
                       t == at::kHalf ? SNA_DTYPE_FP16 : SNA_DTYPE_BF16};
  return 1;
}
int fill_cache(Cache* c, PyObject* ko, PyObject* vo) {
  if (!describe_cache(ko, vo, &c->c)) return 0;
  c->type = c->c.dtype == SNA_DTYPE_FP16 ? at::kHalf : at::kBFloat16;
  c->device = new c10::Device(THPVariable_Unpack(ko).device());
  c->k_pages = Py_NewRef(ko);
  c->v_pages = Py_NewRef(vo);
  return 1;
}
int is_current(const Cache* c) {
  sna_paged_cache now;
  if (!describe_cache(c->k_pages, c->v_pages, &now)) return 0;
  const sna_paged_cache& was = c->c;
  NEED(now.k_pages_dev == was.k_pages_dev && now.v_pages_dev == was.v_pages_dev && now.k_page_stride == was.k_page_stride && now.v_page_stride == was.v_page_stride &&
           now.n_pages == was.n_pages && now.kv_heads == was.kv_heads && now.page_size == was.page_size && now.head_dim == was.head_dim && now.dtype == was.dtype &&
           THPVariable_Unpack(c->k_pages).device() == *c->device,
       "the pages were resized or replaced in place: a new PagedCache is needed");
  return 1;
}
PyObject* cache_new(PyTypeObject* type, PyObject* args, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* names[] = {"k_pages", "v_pages", nullptr};
  PyObject *k, *v;
  if (!PyArg_ParseTupleAndKeywords(args, kw, "OO:PagedCache", (char**)names, &k, &v)) return nullptr;
  Cache* c = (Cache*)type->tp_alloc(type, 0);
  if (c && !fill_cache(c, k, v)) Py_CLEAR(c);
  return (PyObject*)c;
  END_HANDLE_TH_ERRORS
}
void cache_free(PyObject* o) {
  Cache* c = (Cache*)o;
  PyTypeObject* type = Py_TYPE(o);
  Py_XDECREF(c->k_pages);
  Py_XDECREF(c->v_pages);
  delete c->device;
  type->tp_free(o);
  Py_DECREF(type);
}
PyObject* cache_dtype(PyObject* o, void*) { return PyObject_GetAttrString(((Cache*)o)->k_pages, "dtype"); }
PyObject* cache_device(PyObject* o, void*) { return PyObject_GetAttrString(((Cache*)o)->k_pages, "device"); }

bool int32_on(const at::Tensor* t, const char* name, c10::Device device) {
  NEED(t->scalar_type() == at::kInt && t->device() == device, "%s: int32 on %s is needed, got %s", name, device.str().c_str(), shape_of(*t).c_str());
  return true;
}
int describe_batch(PyObject* so, PyObject* lo, PyObject* to, int64_t max_new, int64_t max_len, sna_paged_batch* b) {
  const at::Tensor *s = tensor_of(so, "starts"), *l = s ? tensor_of(lo, "lens") : nullptr, *t = l ? tensor_of(to, "page_table") : nullptr;
  if (!t) return 0;
  NEED(l->dim() == 1 && l->is_cuda(), "lens: one dimension on a GPU is needed, got %s", shape_of(*l).c_str());
  const int64_t n = l->size(0);
  if (!int32_on(s, "starts", l->device()) || !int32_on(l, "lens", l->device()) || !int32_on(t, "page_table", l->device())) return 0;
  NEED(s->dim() == 1 && s->size(0) == n + 1, "starts: %lld entries are needed for %lld sequences, got %s", (long long)n + 1, (long long)n, shape_of(*s).c_str());
  NEED(t->dim() == 2 && t->size(0) == n, "page_table: %lld rows are needed, got %s", (long long)n, shape_of(*t).c_str());
  NEED((n <= 1 || l->stride(0) == 1) && (n == 0 || s->stride(0) == 1) && (t->size(1) <= 1 || t->stride(1) == 1), "starts, lens and the rows of page_table have to be dense");
  NEED(n <= INT32_MAX && t->size(1) <= INT32_MAX && max_new >= 0 && max_new <= INT32_MAX && max_len >= 0 && max_len <= INT32_MAX, "the batch is out of range");
  *b = sna_paged_batch{(const int32_t*)s->data_ptr(), (const int32_t*)l->data_ptr(), (const int32_t*)t->data_ptr(), t->stride(0), (int32_t)n, 0, (int32_t)t->size(1),
                       (int32_t)max_new, (int32_t)max_len};
  return 1;
}
int fill_batch(Batch* b, PyObject* so, PyObject* lo, PyObject* to, int64_t max_new, int64_t max_len) {
  if (!describe_batch(so, lo, to, max_new, max_len, &b->c)) return 0;
  b->device = new c10::Device(THPVariable_Unpack(lo).device());
  b->starts = Py_NewRef(so);
  b->lens = Py_NewRef(lo);
  b->page_table = Py_NewRef(to);
  return 1;
}
int is_current(const Batch* b) {
  sna_paged_batch now;
  const sna_paged_batch& was = b->c;
  if (!describe_batch(b->starts, b->lens, b->page_table, was.max_new, was.max_len, &now)) return 0;
  NEED(now.starts_dev == was.starts_dev && now.lens_dev == was.lens_dev && now.page_table_dev == was.page_table_dev && now.table_stride == was.table_stride &&
           now.n_seqs == was.n_seqs && now.table_width == was.table_width && THPVariable_Unpack(b->lens).device() == *b->device,
       "starts, lens or page_table were resized or replaced in place: a new PagedBatch is needed");
  return 1;
}
PyObject* batch_new(PyTypeObject* type, PyObject* args, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* names[] = {"starts", "lens", "page_table", "max_new", "max_len", nullptr};
  PyObject *s, *l, *t;
  long long max_new, max_len;
  if (!PyArg_ParseTupleAndKeywords(args, kw, "OOOLL:PagedBatch", (char**)names, &s, &l, &t, &max_new, &max_len)) return nullptr;
  Batch* b = (Batch*)type->tp_alloc(type, 0);
  if (b && !fill_batch(b, s, l, t, max_new, max_len)) Py_CLEAR(b);
  return (PyObject*)b;
  END_HANDLE_TH_ERRORS
}
void batch_free(PyObject* o) {
  Batch* b = (Batch*)o;
  PyTypeObject* type = Py_TYPE(o);
  Py_XDECREF(b->starts);
  Py_XDECREF(b->lens);
  Py_XDECREF(b->page_table);
  delete b->device;
  type->tp_free(o);
  Py_DECREF(type);
}

PyMemberDef cache_members[] = {{"k_pages", T_OBJECT, offsetof(Cache, k_pages), READONLY, nullptr},
                               {"v_pages", T_OBJECT, offsetof(Cache, v_pages), READONLY, nullptr},
                               {"n_pages", T_INT, offsetof(Cache, c.n_pages), READONLY, nullptr},
                               {"kv_heads", T_INT, offsetof(Cache, c.kv_heads), READONLY, nullptr},
                               {"page_size", T_INT, offsetof(Cache, c.page_size), READONLY, nullptr},
                               {"head_dim", T_INT, offsetof(Cache, c.head_dim), READONLY, nullptr},
                               {nullptr, 0, 0, 0, nullptr}};
PyGetSetDef cache_getters[] = {{"dtype", cache_dtype, nullptr, nullptr, nullptr}, {"device", cache_device, nullptr, nullptr, nullptr}, {nullptr, nullptr, nullptr, nullptr, nullptr}};
PyMemberDef batch_members[] = {{"starts", T_OBJECT, offsetof(Batch, starts), READONLY, nullptr},
                               {"lens", T_OBJECT, offsetof(Batch, lens), READONLY, nullptr},
                               {"page_table", T_OBJECT, offsetof(Batch, page_table), READONLY, nullptr},
                               {"n_seqs", T_INT, offsetof(Batch, c.n_seqs), READONLY, nullptr},
                               {"max_new", T_INT, offsetof(Batch, c.max_new), READONLY, nullptr},
                               {"max_len", T_INT, offsetof(Batch, c.max_len), READONLY, nullptr},
                               {nullptr, 0, 0, 0, nullptr}};
PyType_Slot cache_slots[] = {{Py_tp_new, (void*)cache_new}, {Py_tp_dealloc, (void*)cache_free}, {Py_tp_members, cache_members}, {Py_tp_getset, cache_getters}, {0, nullptr}};
PyType_Slot batch_slots[] = {{Py_tp_new, (void*)batch_new}, {Py_tp_dealloc, (void*)batch_free}, {Py_tp_members, batch_members}, {0, nullptr}};
PyType_Spec cache_spec = {"paper_2312_16733_amd._serving.PagedCache", sizeof(Cache), 0, Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE, cache_slots};
PyType_Spec batch_spec = {"paper_2312_16733_amd._serving.PagedBatch", sizeof(Batch), 0, Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE, batch_slots};

// ---- the step's parts --------------------------------------------------------------------------------------------------------
struct Step {
  Cache* cache;
  sna_paged_batch batch;
  const at::Tensor* q;
  at::Tensor out;
  sna_rows q_rows, out_rows;
};
// heads < 0: any number
int rows_of(const at::Tensor& t, const char* name, int64_t heads, const Cache* c, sna_rows* r) {
  NEED(t.dim() == 3 && t.size(2) == c->c.head_dim && (heads < 0 || t.size(1) == heads), "%s: [tokens][%s][%d] is needed, got %s", name,
       heads < 0 ? "heads" : std::to_string(heads).c_str(), c->c.head_dim, shape_of(t).c_str());
  NEED(t.scalar_type() == c->type && t.device() == *c->device, "%s: %s on %s is needed, got %s", name, c10::toString(c->type), c->device->str().c_str(), shape_of(t).c_str());
  NEED(t.stride(2) == 1, "%s: a head's elements have to be dense", name);
  const bool empty = t.numel() == 0;
  *r = sna_rows{t.data_ptr(), t.size(0) > 1 && !empty ? t.stride(0) : 0, t.size(1) > 1 && !empty ? t.stride(1) : 0};
  return 1;
}
int step_of(Step* s, PyObject* cache, PyObject* batch, PyObject* q, PyObject* out) {
  if (!PyObject_TypeCheck(cache, cache_type) || !PyObject_TypeCheck(batch, batch_type)) {
    PyErr_SetString(PyExc_TypeError, "a PagedCache and a PagedBatch are needed");
    return 0;
  }
  s->cache = (Cache*)cache;
  const Batch* b = (Batch*)batch;
  if (!is_current(s->cache) || !is_current(b)) return 0;
  NEED(*b->device == *s->cache->device, "the batch is on %s, the cache on %s", b->device->str().c_str(), s->cache->device->str().c_str());
  if (!(s->q = tensor_of(q, "q")) || !rows_of(*s->q, "q", -1, s->cache, &s->q_rows)) return 0;
  NEED(s->q->size(0) <= INT32_MAX && s->q->size(1) <= INT32_MAX, "q: %s is out of range", shape_of(*s->q).c_str());
  s->batch = b->c;
  s->batch.n_tokens = (int32_t)s->q->size(0);
  // bounds that this step cannot reach say nothing about it: the C entries take the nearest ones that it can
  if (s->batch.n_tokens > 0 && s->batch.max_new > s->batch.n_tokens) s->batch.max_new = s->batch.n_tokens;
  if (s->batch.max_len < s->batch.max_new) s->batch.max_len = s->batch.max_new;
  if (!none(out)) {
    const at::Tensor* t = tensor_of(out, "out");
    if (!t) return 0;
    NEED(t->sizes() == s->q->sizes(), "out: %s is needed, got %s", shape_of(*s->q).c_str(), shape_of(*t).c_str());
    s->out = *t;
  }
  return 1;
}
int out_of(Step* s) {                      // on the call's stream
  if (!s->out.defined()) s->out = at::empty(s->q->sizes(), s->q->options());
  return rows_of(s->out, "out", -1, s->cache, &s->out_rows);
}
int vector_of(PyObject* o, const char* name, int64_t n, const Cache* c, const float** p, int64_t* count) {
  *p = nullptr;
  if (none(o)) return 1;
  const at::Tensor* t = tensor_of(o, name);
  if (!t) return 0;
  NEED(t->scalar_type() == at::kFloat && t->device() == *c->device && t->dim() == 1 && (t->size(0) <= 1 || t->stride(0) == 1) && (n < 0 || t->size(0) == n),
       "%s: a dense fp32 vector%s on %s is needed, got %s", name, n < 0 ? "" : (" of " + std::to_string(n)).c_str(), c->device->str().c_str(), shape_of(*t).c_str());
  *p = (const float*)t->data_ptr();
  *count = t->size(0);
  return 1;
}

// A dense int32 vector of n, or none
int ints_of(PyObject* o, const char* name, int64_t n, c10::Device device, const int32_t** p) {
  *p = nullptr;
  if (none(o)) return 1;
  const at::Tensor* t = tensor_of(o, name);
  if (!t) return 0;
  NEED(t->scalar_type() == at::kInt && t->device() == device && t->dim() == 1 && t->size(0) == n && (n <= 1 || t->stride(0) == 1), "%s: dense int32 [%lld] on %s is needed, got %s", name,
       (long long)n, device.str().c_str(), shape_of(*t).c_str());
  *p = (const int32_t*)t->data_ptr();
  return 1;
}

PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"cache", "batch", "q", "k", "v", "inv_freq", "interleaved", "q_norm", "k_norm", "eps", "out", "stream", "positions"};
  PyObject* a[13];
  if (!arguments("kv_append", names, 5, args, n, kw, a)) return nullptr;
  Step s;
  if (!step_of(&s, a[0], a[1], a[2], a[10])) return nullptr;
  sna_rows k, v;
  const at::Tensor *kt = tensor_of(a[3], "k"), *vt = kt ? tensor_of(a[4], "v") : nullptr;
  if (!vt || !rows_of(*kt, "k", s.cache->c.kv_heads, s.cache, &k) || !rows_of(*vt, "v", s.cache->c.kv_heads, s.cache, &v)) return nullptr;
  NEED(kt->size(0) == s.q->size(0) && vt->size(0) == s.q->size(0), "%lld tokens of q, %lld of k, %lld of v", (long long)s.q->size(0), (long long)kt->size(0), (long long)vt->size(0));
  const float *inv, *qn, *kn;
  int64_t pairs = 0, dim = s.cache->c.head_dim, ignored;
  if (!vector_of(a[5], "inv_freq", -1, s.cache, &inv, &pairs) || !vector_of(a[7], "q_norm", dim, s.cache, &qn, &ignored) || !vector_of(a[8], "k_norm", dim, s.cache, &kn, &ignored)) return nullptr;
  NEED(pairs <= dim, "inv_freq: %lld pairs of a head of %lld", (long long)pairs, (long long)dim);
  const int32_t* positions;
  if (!ints_of(a[12], "positions", s.q->size(0), *s.cache->device, &positions)) return nullptr;
  const int interleaved = none(a[6]) ? 0 : PyObject_IsTrue(a[6]);
  double eps = 1e-6;
  if (interleaved < 0 || !real_number(a[9], &eps)) return nullptr;
  On on;
  if (!on.begin(a[11], s.cache->device->index()) || !out_of(&s)) return nullptr;
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_kv_append_at(&s.cache->c, &s.batch, (int32_t)s.q->size(1), &s.q_rows, &k, &v, &s.out_rows, inv, (int32_t)(2 * pairs), interleaved, qn, kn, (float)eps, positions, on.raw());
  Py_END_ALLOW_THREADS
  if (!status(st)) return nullptr;
  return none(a[10]) ? THPVariable_Wrap(std::move(s.out)) : Py_NewRef(a[10]);
  END_HANDLE_TH_ERRORS
}

// What the caller brought, where it is large enough, or the allocator's, on the call's stream
int workspace_of(PyObject* o, int64_t need, const at::Tensor& like, at::Tensor* workspace) {
  if (need <= 0) return 1;
  const at::Tensor* given = none(o) ? nullptr : tensor_of(o, "workspace");
  if (!none(o) && !given) return 0;
  NEED(!given || (given->scalar_type() == at::kByte && given->device() == like.device() && given->is_contiguous()), "workspace: dense uint8 on %s is needed, got %s",
       like.device().str().c_str(), shape_of(*given).c_str());
  *workspace = given && given->numel() >= need ? *given : at::empty({need}, like.options().dtype(at::kByte));
  return 1;
}

// What both forms of attention share behind their own arguments.  No words: causal
struct Masks {
  const uint64_t* masks;
  int32_t words;
  const int32_t *prefix, *positions;
};
PyObject* attend(Step& s, const Masks& m, PyObject* scale_o, PyObject* window_o, PyObject* out_o, PyObject* workspace_o, PyObject* stream_o) {
  double scale = 1.0 / std::sqrt((double)s.cache->c.head_dim);
  int64_t window = 0;
  if (!real_number(scale_o, &scale) || !whole_number(window_o, &window)) return nullptr;
  NEED(window >= 0 && window <= INT32_MAX, "window: %lld is out of range", (long long)window);
  const int32_t heads = (int32_t)s.q->size(1);
  const int64_t need = m.words ? sna_tree_attention_workspace_bytes(&s.cache->c, &s.batch, heads, m.words, (int32_t)window)
                               : sna_paged_attention_workspace_bytes(&s.cache->c, &s.batch, heads, (int32_t)window);
  if (!status(need)) return nullptr;
  On on;
  if (!on.begin(stream_o, s.cache->device->index()) || !out_of(&s)) return nullptr;
  at::Tensor workspace;
  if (!workspace_of(workspace_o, need, *s.q, &workspace)) return nullptr;
  void* ws = need > 0 ? workspace.data_ptr() : nullptr;
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = m.words ? sna_tree_attention(&s.cache->c, &s.batch, heads, &s.q_rows, &s.out_rows, m.masks, m.words, m.prefix, m.positions, (float)scale, (int32_t)window, ws, (size_t)need, on.raw())
               : sna_paged_attention(&s.cache->c, &s.batch, heads, &s.q_rows, &s.out_rows, (float)scale, (int32_t)window, ws, (size_t)need, on.raw());
  Py_END_ALLOW_THREADS
  if (!status(st)) return nullptr;
  return none(out_o) ? THPVariable_Wrap(std::move(s.out)) : Py_NewRef(out_o);
}

PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"cache", "batch", "q", "scale", "window", "out", "workspace", "stream"};
  PyObject* a[8];
  if (!arguments("paged_attention", names, 3, args, n, kw, a)) return nullptr;
  Step s;
  if (!step_of(&s, a[0], a[1], a[2], a[5])) return nullptr;
  return attend(s, Masks{}, a[3], a[4], a[5], a[6], a[7]);
  END_HANDLE_TH_ERRORS
}

PyObject* tree_attention(PyObject*, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"cache", "batch", "q", "masks", "prefix", "positions", "scale", "window", "out", "workspace", "stream"};
  PyObject* a[11];
  if (!arguments("tree_attention", names, 4, args, n, kw, a)) return nullptr;
  Step s;
  if (!step_of(&s, a[0], a[1], a[2], a[8])) return nullptr;
  const at::Tensor* t = tensor_of(a[3], "masks");
  if (!t) return nullptr;
  NEED(t->dim() == 2 && t->size(0) == s.q->size(0) && t->size(1) >= 1 && t->size(1) <= 64 && t->scalar_type() == at::kLong && t->device() == *s.cache->device && t->is_contiguous(),
       "masks: dense int64 [%lld][words], 1 to 64 words, on %s is needed, got %s", (long long)s.q->size(0), s.cache->device->str().c_str(), shape_of(*t).c_str());
  Masks m = {};
  m.words = (int32_t)t->size(1);
  m.masks = (const uint64_t*)t->data_ptr();
  if (!ints_of(a[4], "prefix", s.batch.n_seqs, *s.cache->device, &m.prefix) || !ints_of(a[5], "positions", s.q->size(0), *s.cache->device, &m.positions)) return nullptr;
  return attend(s, m, a[6], a[7], a[8], a[9], a[10]);
  END_HANDLE_TH_ERRORS
}

PyObject* verify_draft(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"target", "tokens", "uniforms", "draft_probs", "n_draft", "stream"};
  PyObject* a[6];
  if (!arguments("verify_draft", names, 3, args, nargs, kw, a)) return nullptr;
  const at::Tensor *p = tensor_of(a[0], "target"), *t = p ? tensor_of(a[1], "tokens") : nullptr, *u = t ? tensor_of(a[2], "uniforms") : nullptr;
  if (!u) return nullptr;
  NEED(p->dim() == 3 && p->scalar_type() == at::kFloat && p->is_cuda() && p->size(1) >= 1 && (p->size(2) <= 1 || p->stride(2) == 1),
       "target: fp32 [sequences][drafts + 1][vocabulary], dense rows on a GPU are needed, got %s", shape_of(*p).c_str());
  const int64_t n = p->size(0), K = p->size(1) - 1, V = p->size(2);
  const c10::Device device = p->device();
  NEED(n <= INT32_MAX && K <= INT32_MAX && V <= INT32_MAX, "target: %s is out of range", shape_of(*p).c_str());
  NEED(t->dim() == 2 && t->size(0) == n && t->size(1) == K && (t->scalar_type() == at::kInt || t->scalar_type() == at::kLong) && t->device() == device && t->is_contiguous(),
       "tokens: dense int32 or int64 [%lld][%lld] on %s is needed, got %s", (long long)n, (long long)K, device.str().c_str(), shape_of(*t).c_str());
  NEED(u->dim() == 2 && u->size(0) == n && u->size(1) == K + 1 && u->scalar_type() == at::kFloat && u->device() == device && u->is_contiguous(),
       "uniforms: dense fp32 [%lld][%lld] on %s is needed, got %s", (long long)n, (long long)K + 1, device.str().c_str(), shape_of(*u).c_str());
  const at::Tensor *q = nullptr, *c = nullptr;
  if (!none(a[3])) {
    if (!(q = tensor_of(a[3], "draft_probs"))) return nullptr;
    NEED(q->dim() == 3 && q->size(0) == n && q->size(1) == K && q->size(2) == V && q->scalar_type() == at::kFloat && q->device() == device && (V <= 1 || q->stride(2) == 1),
         "draft_probs: fp32 [%lld][%lld][%lld], dense rows on %s are needed, got %s", (long long)n, (long long)K, (long long)V, device.str().c_str(), shape_of(*q).c_str());
  }
  if (!none(a[4])) {
    if (!(c = tensor_of(a[4], "n_draft"))) return nullptr;
    NEED(c->dim() == 1 && c->size(0) == n && c->scalar_type() == at::kInt && c->device() == device && c->is_contiguous(), "n_draft: dense int32 [%lld] on %s is needed, got %s", (long long)n,
         device.str().c_str(), shape_of(*c).c_str());
  }
  On on;
  if (!on.begin(a[5], device.index())) return nullptr;
  at::Tensor out = at::empty({n, K + 1}, p->options().dtype(at::kInt)), accepted = at::empty({n}, out.options());
  const bool has_q = q && q->numel();
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_verify_draft((const float*)p->data_ptr(), p->stride(0), p->stride(1), has_q ? (const float*)q->data_ptr() : nullptr, has_q ? q->stride(0) : 0, has_q ? q->stride(1) : 0, t->data_ptr(),
                        (int32_t)t->element_size(), (const float*)u->data_ptr(), c ? (const int32_t*)c->data_ptr() : nullptr, (int32_t)n, (int32_t)K, (int32_t)V, (int32_t*)out.data_ptr(),
                        (int32_t*)accepted.data_ptr(), on.raw());
  Py_END_ALLOW_THREADS
  if (!status(st)) return nullptr;
  PyObject *x = THPVariable_Wrap(std::move(out)), *y = x ? THPVariable_Wrap(std::move(accepted)) : nullptr, *r = y ? PyTuple_Pack(2, x, y) : nullptr;
  Py_XDECREF(x);
  Py_XDECREF(y);
  return r;
  END_HANDLE_TH_ERRORS
}

PyObject* wrapped(std::initializer_list<at::Tensor> tensors) {
  PyObject* r = PyTuple_New((Py_ssize_t)tensors.size());
  Py_ssize_t i = 0;
  for (const at::Tensor& t : tensors) {
    PyObject* x = r ? THPVariable_Wrap(t) : nullptr;
    if (!x) {
      Py_XDECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, x);
  }
  return r;
}
const Batch* batch_of(PyObject* o) {
  if (!PyObject_TypeCheck(o, batch_type)) {
    PyErr_SetString(PyExc_TypeError, "a PagedBatch is needed");
    return nullptr;
  }
  return is_current((Batch*)o) ? (Batch*)o : nullptr;
}
const Cache* cache_of(PyObject* o) {
  if (!PyObject_TypeCheck(o, cache_type)) {
    PyErr_SetString(PyExc_TypeError, "a PagedCache is needed");
    return nullptr;
  }
  return is_current((Cache*)o) ? (Cache*)o : nullptr;
}

// Dense tokens [n], int32 or int64
const at::Tensor* tokens_of(PyObject* o, const char* name, int64_t n, c10::Device device) {
  const at::Tensor* t = tensor_of(o, name);
  if (!t) return nullptr;
  NEED(t->dim() == 1 && (n < 0 || t->size(0) == n) && (t->scalar_type() == at::kInt || t->scalar_type() == at::kLong) && t->device() == device && t->is_contiguous(),
       "%s: dense int32 or int64 [%s] on %s is needed, got %s", name, n < 0 ? "tokens" : std::to_string(n).c_str(), device.str().c_str(), shape_of(*t).c_str());
  return t;
}

PyObject* verify_tree(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"batch", "sampled", "tokens", "parents", "stream"};
  PyObject* a[5];
  if (!arguments("verify_tree", names, 4, args, nargs, kw, a)) return nullptr;
  const Batch* b = batch_of(a[0]);
  if (!b) return nullptr;
  const c10::Device device = *b->device;
  const at::Tensor *sampled = tokens_of(a[1], "sampled", -1, device), *tokens = sampled ? tokens_of(a[2], "tokens", sampled->size(0), device) : nullptr;
  if (!tokens) return nullptr;
  const int64_t n = tokens->size(0);
  NEED(n <= INT32_MAX, "tokens: %s is out of range", shape_of(*tokens).c_str());
  const at::Tensor* p = tensor_of(a[3], "parents");
  const int32_t* parents;
  if (!p || !ints_of(a[3], "parents", n, device, &parents)) return nullptr;
  sna_paged_batch c = b->c;
  c.n_tokens = (int32_t)n;
  On on;
  if (!on.begin(a[4], device.index())) return nullptr;
  const auto options = THPVariable_Unpack(b->lens).options();
  at::Tensor kept = at::empty({c.n_seqs, c.max_new}, options), counts = at::empty({c.n_seqs}, options), next = at::empty({c.n_seqs}, options);
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_verify_tree(&c, sampled->data_ptr(), (int32_t)sampled->element_size(), tokens->data_ptr(), (int32_t)tokens->element_size(), parents, (int32_t*)kept.data_ptr(), (int32_t*)counts.data_ptr(),
                       (int32_t*)next.data_ptr(), on.raw());
  Py_END_ALLOW_THREADS
  return status(st) ? wrapped({kept, counts, next}) : nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* kv_compact(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"cache", "batch", "kept", "counts", "stream"};
  PyObject* a[5];
  if (!arguments("kv_compact", names, 4, args, nargs, kw, a)) return nullptr;
  const Cache* c = cache_of(a[0]);
  const Batch* b = c ? batch_of(a[1]) : nullptr;
  if (!b) return nullptr;
  NEED(*b->device == *c->device, "the batch is on %s, the cache on %s", b->device->str().c_str(), c->device->str().c_str());
  const at::Tensor* kept = tensor_of(a[2], "kept");
  if (!kept) return nullptr;
  NEED(kept->dim() == 2 && kept->size(0) == b->c.n_seqs && kept->size(1) <= INT32_MAX && kept->scalar_type() == at::kInt && kept->device() == *c->device && kept->is_contiguous(),
       "kept: dense int32 [%d][tokens] on %s is needed, got %s", b->c.n_seqs, c->device->str().c_str(), shape_of(*kept).c_str());
  const int32_t* counts;
  if (!tensor_of(a[3], "counts") || !ints_of(a[3], "counts", b->c.n_seqs, *c->device, &counts)) return nullptr;
  On on;
  if (!on.begin(a[4], c->device->index())) return nullptr;
  at::Tensor lens = at::empty({b->c.n_seqs}, THPVariable_Unpack(b->lens).options());
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_kv_compact(&c->c, &b->c, (const int32_t*)kept->data_ptr(), (int32_t)kept->size(1), counts, (int32_t*)lens.data_ptr(), on.raw());
  Py_END_ALLOW_THREADS
  return status(st) ? THPVariable_Wrap(std::move(lens)) : nullptr;
  END_HANDLE_TH_ERRORS
}

PyObject* copy_pages(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"cache", "source", "target", "stream"};
  PyObject* a[4];
  if (!arguments("copy_pages", names, 3, args, nargs, kw, a)) return nullptr;
  const Cache* c = cache_of(a[0]);
  const at::Tensor* from = c ? tensor_of(a[1], "source") : nullptr;
  if (!from || !tensor_of(a[2], "target")) return nullptr;
  const int64_t n = from->dim() == 1 ? from->size(0) : 0;
  const int32_t *source, *target;
  if (!ints_of(a[1], "source", n, *c->device, &source) || !ints_of(a[2], "target", n, *c->device, &target)) return nullptr;
  NEED(n <= INT32_MAX, "source: %s is out of range", shape_of(*from).c_str());
  On on;
  if (!on.begin(a[3], c->device->index())) return nullptr;
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_copy_pages(&c->c, source, target, (int32_t)n, on.raw());
  Py_END_ALLOW_THREADS
  if (!status(st)) return nullptr;
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// A number for all rows, or a dense vector of one for each
int setting(PyObject* o, const char* name, int64_t n, at::ScalarType type, c10::Device device, const void** of, double* all) {
  *of = nullptr;
  if (none(o)) return 1;
  if (!THPVariable_Check(o)) return real_number(o, all);
  const at::Tensor& t = THPVariable_Unpack(o);
  NEED(t.dim() == 1 && t.size(0) == n && t.scalar_type() == type && t.device() == device && (n <= 1 || t.stride(0) == 1), "%s: a number or dense %s [%lld] on %s is needed, got %s", name,
       c10::toString(type), (long long)n, device.str().c_str(), shape_of(t).c_str());
  *of = t.data_ptr();
  return 1;
}

PyObject* sample_tokens(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kw) {
  HANDLE_TH_ERRORS
  static const char* const names[] = {"logits", "uniforms", "temperature", "top_k", "top_p", "min_p", "probs", "out", "workspace", "stream"};
  PyObject* a[10];
  if (!arguments("sample_tokens", names, 2, args, nargs, kw, a)) return nullptr;
  const at::Tensor *l = tensor_of(a[0], "logits"), *u = l ? tensor_of(a[1], "uniforms") : nullptr;
  if (!u) return nullptr;
  const at::ScalarType type = l->scalar_type();
  NEED(l->dim() == 2 && (type == at::kFloat || type == at::kBFloat16 || type == at::kHalf) && l->is_cuda() && l->size(1) >= 1 && (l->size(1) == 1 || l->stride(1) == 1),
       "logits: fp32, bf16 or fp16 [rows][vocabulary], dense rows on a GPU are needed, got %s", shape_of(*l).c_str());
  const int64_t n = l->size(0), V = l->size(1);
  const c10::Device device = l->device();
  NEED(n <= INT32_MAX && V <= INT32_MAX, "logits: %s is out of range", shape_of(*l).c_str());
  NEED(u->dim() == 1 && u->size(0) == n && u->scalar_type() == at::kFloat && u->device() == device && (n <= 1 || u->stride(0) == 1), "uniforms: dense fp32 [%lld] on %s is needed, got %s", (long long)n,
       device.str().c_str(), shape_of(*u).c_str());
  double temperature = 1.0, top_k = 0.0, top_p = 1.0, min_p = 0.0;
  sna_sampling s = {};
  if (!setting(a[2], "temperature", n, at::kFloat, device, (const void**)&s.temperature_dev, &temperature) || !setting(a[3], "top_k", n, at::kInt, device, (const void**)&s.top_k_dev, &top_k) ||
      !setting(a[4], "top_p", n, at::kFloat, device, (const void**)&s.top_p_dev, &top_p) || !setting(a[5], "min_p", n, at::kFloat, device, (const void**)&s.min_p_dev, &min_p))
    return nullptr;
  NEED(top_k >= 0.0 && top_k <= INT32_MAX && top_k == std::floor(top_k), "top_k: %s is no count", std::to_string(top_k).c_str());
  s.logits_dev = l->data_ptr();
  s.row_stride = n > 1 ? l->stride(0) : 0;
  s.n_rows = (int32_t)n;
  s.vocab = (int32_t)V;
  s.dtype = type == at::kFloat ? SNA_DTYPE_FP32 : type == at::kHalf ? SNA_DTYPE_FP16 : SNA_DTYPE_BF16;
  s.top_k = (int32_t)top_k;
  s.temperature = (float)temperature;
  s.top_p = (float)top_p;
  s.min_p = (float)min_p;
  s.uniforms_dev = (const float*)u->data_ptr();
  const int64_t need = sna_sample_tokens_workspace_bytes(&s);
  if (!status(need)) return nullptr;
  const at::Tensor *given_probs = !none(a[6]) && THPVariable_Check(a[6]) ? &THPVariable_Unpack(a[6]) : nullptr, *given_out = none(a[7]) ? nullptr : tensor_of(a[7], "out");
  if (!none(a[7]) && !given_out) return nullptr;
  NEED(!given_probs || (given_probs->dim() == 2 && given_probs->sizes() == l->sizes() && given_probs->scalar_type() == at::kFloat && given_probs->device() == device &&
                        (V == 1 || given_probs->stride(1) == 1)),
       "probs: fp32 (%lld, %lld), dense rows on %s are needed, got %s", (long long)n, (long long)V, device.str().c_str(), shape_of(*given_probs).c_str());
  NEED(!given_out || (given_out->dim() == 1 && given_out->size(0) == n && given_out->scalar_type() == at::kInt && given_out->device() == device && (n <= 1 || given_out->stride(0) == 1)),
       "out: dense int32 [%lld] on %s is needed, got %s", (long long)n, device.str().c_str(), shape_of(*given_out).c_str());
  const int want_probs = given_probs ? 1 : none(a[6]) ? 0 : PyObject_IsTrue(a[6]);
  if (want_probs < 0) return nullptr;
  On on;
  if (!on.begin(a[9], device.index())) return nullptr;
  at::Tensor workspace, tokens = given_out ? *given_out : at::empty({n}, l->options().dtype(at::kInt)), probs;
  if (want_probs) probs = given_probs ? *given_probs : at::empty({n, V}, l->options().dtype(at::kFloat));
  if (!workspace_of(a[8], need, *l, &workspace)) return nullptr;
  void* ws = need > 0 ? workspace.data_ptr() : nullptr;
  float* p = want_probs && n ? (float*)probs.data_ptr() : nullptr;
  sna_status st;
  Py_BEGIN_ALLOW_THREADS
  st = sna_sample_tokens(&s, (int32_t*)tokens.data_ptr(), p, p && n > 1 ? probs.stride(0) : V, ws, (size_t)need, on.raw());
  Py_END_ALLOW_THREADS
  if (!status(st)) return nullptr;
  return want_probs ? wrapped({tokens, probs}) : THPVariable_Wrap(std::move(tokens));
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"kv_append", (PyCFunction)(void*)kv_append, METH_FASTCALL | METH_KEYWORDS,
     "kv_append(cache, batch, q, k, v, inv_freq=None, interleaved=False, q_norm=None, k_norm=None, eps=1e-6, out=None, stream=None, positions=None)\n\n"
     "Stores the step's k and v [tokens][kv_heads][head_dim] in the cache and returns its q [tokens][heads][head_dim], q and k\n"
     "normalised per head (fp32 q_norm and k_norm [head_dim], both or neither) and rotated (fp32 inv_freq [rot_dim / 2]; pairs\n"
     "i and i + rot_dim / 2, or 2 i and 2 i + 1 where `interleaved`).  Strided q, k and v are read in place.  `out` may be q.\n"
     "positions int32 [tokens]: what the rotation goes by where it is not the slot's number, as in trees."},
    {"paged_attention", (PyCFunction)(void*)paged_attention, METH_FASTCALL | METH_KEYWORDS,
     "paged_attention(cache, batch, q, scale=None, window=0, out=None, workspace=None, stream=None)\n\n"
     "Causal attention of the step's q [tokens][heads][head_dim] over the cached keys and values, these tokens' own among them\n"
     "(after kv_append).  heads is a multiple of kv_heads.  scale: 1 / sqrt(head_dim).  window: keys that a token sees, its own\n"
     "among them; 0: all.  workspace: a dense uint8 tensor that is used where it is large enough, instead of the allocator's."},
    {"verify_draft", (PyCFunction)(void*)verify_draft, METH_FASTCALL | METH_KEYWORDS,
     "verify_draft(target, tokens, uniforms, draft_probs=None, n_draft=None, stream=None)\n\n"
     "Which drafted tokens stand, and the token after them.  target fp32 [n][K + 1][V]: the target's probabilities at every\n"
     "drafted place and at the one after the last; tokens [n][K] (int32 or int64); uniforms fp32 [n][K + 1] from [0, 1): one for\n"
     "each draft, the last for the draw; draft_probs fp32 [n][K][V] that the drafts were drawn from, or None where they were\n"
     "chosen without chance; n_draft int32 [n]: how many of the K each sequence has (all).  Returns (out int32 [n][K + 1],\n"
     "accepted int32 [n]): the accepted drafts, the drawn token, -1 behind it."},
    {"tree_attention", (PyCFunction)(void*)tree_attention, METH_FASTCALL | METH_KEYWORDS,
     "tree_attention(cache, batch, q, masks, prefix=None, positions=None, scale=None, window=0, out=None, workspace=None, stream=None)\n\n"
     "Attention of the tokens of drafted trees q [tokens][heads][head_dim] over the cached keys and values, theirs among them (after\n"
     "kv_append).  A sequence's tree begins behind its first prefix[b] slots (int32 [n]; None: all but the step's own tokens).  A token\n"
     "sees what lies before the tree, and slot prefix + 64 w + j where bit j of masks[token][w] is set (int64 [tokens][words], up\n"
     "to 64 words; see tree_masks).  window: how far back it sees before the tree, from its position (int32 [tokens]; None: its\n"
     "slot); 0: all.  The rest is as for paged_attention."},
    {"verify_tree", (PyCFunction)(void*)verify_tree, METH_FASTCALL | METH_KEYWORDS,
     "verify_tree(batch, sampled, tokens, parents, stream=None)\n\n"
     "Which tokens of the step's trees stand.  A sequence's first token is its root and stands; behind one that stands its first child\n"
     "(parents int32 [tokens]: a number within the sequence) whose token is sampled[parent] does, too.  sampled, tokens [tokens]\n"
     "int32 or int64.  Returns (kept int32 [n][max_new]: their numbers within the sequence, then -1; counts int32 [n]; next int32\n"
     "[n]: the token sampled behind the last)."},
    {"kv_compact", (PyCFunction)(void*)kv_compact, METH_FASTCALL | METH_KEYWORDS,
     "kv_compact(cache, batch, kept, counts, stream=None)\n\n"
     "Moves the keys and values of the kept ones of the step's tokens (kept int32 [n][any], rising, counts[b] of them) up to the first\n"
     "slots of the step, and returns the new lengths int32 [n].  A pool whose layers lie next to each other within a page goes in\n"
     "one call, as a PagedCache of layers * kv_heads heads."},
    {"copy_pages", (PyCFunction)(void*)copy_pages, METH_FASTCALL | METH_KEYWORDS,
     "copy_pages(cache, source, target, stream=None)\n\n"
     "Copies page source[i] over page target[i] (int32 [n]), keys and values.  No target is another's target or source."},
    {"sample_tokens", (PyCFunction)(void*)sample_tokens, METH_FASTCALL | METH_KEYWORDS,
     "sample_tokens(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, probs=False, out=None, workspace=None, stream=None)\n\n"
     "A token int32 [n] of each row of logits [n][V] (fp32, bf16 or fp16) by uniforms fp32 [n] from [0, 1): of the top_k largest (0:\n"
     "all; ties go to the lower token) the fewest that make top_p of their weights exp(logit / temperature), of these the ones with\n"
     "at least min_p of the largest's; drawn by running sums in token order.  Temperature 0: the largest.  -1 where no logit is more\n"
     "than -inf (NaN counts as that).  Each setting is a number or a tensor [n] (top_k int32, the others fp32).  probs: True, or an\n"
     "fp32 [n][V] to write to: (tokens, probs) is returned, the probabilities that the token was drawn by.  What is written to, out\n"
     "(int32 [n]) or probs, is none of what is read."},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() {
  PyObject* binding = PyImport_ImportModule("paper_2312_16733_amd.binding");
  if (!binding) return nullptr;
  sna_error = PyObject_GetAttrString(binding, "SnaError");
  Py_DECREF(binding);
  PyObject* m = sna_error ? PyModule_Create(&module) : nullptr;
  if (!m) return nullptr;
  cache_type = (PyTypeObject*)PyType_FromSpec(&cache_spec);
  batch_type = (PyTypeObject*)PyType_FromSpec(&batch_spec);
  if (!cache_type || !batch_type || PyModule_AddObject(m, "PagedCache", Py_NewRef((PyObject*)cache_type)) < 0 ||
      PyModule_AddObject(m, "PagedBatch", Py_NewRef((PyObject*)batch_type)) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
