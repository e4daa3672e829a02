// The operators for many requests about one long video without Python between the arguments and the library: mrope_append8, page_gather,
// chunk_attn8 and prefix_attn for arguments as programs pass them.  Each function returns NotImplemented where an argument is anything else (a
// tensor subclass, another dtype, shape or stride than the library takes, a tensor that is not on the current GPU, a stream of its own, ...) or a
// torch function mode is active; serve.py's own code then takes the call, converts what can be converted and raises what has to be raised.
// Nothing is kept between calls.
//
// us a call and its kernels in an unbroken row of them, ctypes / here: mrope_append8 of 13 rows and their page_gather 24.9 / 7.3 (two calls), page_gather of
// seven tails 10.0 / 3.5, prefix_attn of five tokens 16.8 / 10.7.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstring>

#include "../../../include/sparrow_serve.h"

namespace {

PyObject *g_check, *g_stream_of, *g_ndarray;             // serve._check, paged._stream_of, numpy.ndarray

// The library's functions, in the copy of the library that serve.py has loaded.
#define SPARROW_FUNCTIONS(f) f(mrope_append8) f(page_gather) f(prefix_attn_workspace) f(chunk_attn8) f(prefix_attn)
struct Library {
#define SPARROW_MEMBER(n) decltype(&sparrow_##n) n;
  SPARROW_FUNCTIONS(SPARROW_MEMBER)
} lib;
#define SPARROW_STRING_OF(x) #x
#define SPARROW_STRING(x) SPARROW_STRING_OF(x)
#define SPARROW_NAME(n) "sparrow_" #n,
constexpr const char *kFunctions[] = {SPARROW_FUNCTIONS(SPARROW_NAME)};
// Code compiled against the headers of one torch and one Python reads another's objects wrongly, without an error:
// serve.py takes this part only where it runs under the same ones.
constexpr char kBuiltFor[] = "torch " TORCH_VERSION ", Python " SPARROW_STRING(PY_MAJOR_VERSION) "." SPARROW_STRING(PY_MINOR_VERSION);
constexpr int kNumFunctions = sizeof(kFunctions) / sizeof(kFunctions[0]);
static_assert(sizeof(Library) == kNumFunctions * sizeof(void *), "one address after the other");

struct NotHere {};                                       // the general code takes the call
struct Raised {};                                        // a Python exception is set
void need(bool ok) {
  if (!ok) throw NotHere{};
}
bool none(PyObject *o) { return o == Py_None; }

class Object {                                           // an owned reference
 public:
  explicit Object(PyObject *o) : o_(o) {}
  ~Object() { Py_XDECREF(o_); }
  Object(const Object &) = delete;
  Object &operator=(const Object &) = delete;
  PyObject *get() const { return o_; }

 private:
  PyObject *o_;
};

// The tensors of a call, all on one GPU
class Call {
 public:
  const at::Tensor &tensor(PyObject *o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor &t = THPVariable_Unpack(o);
    need(t.is_cuda() && (device_ < 0 || t.get_device() == device_));
    device_ = t.get_device();
    return t;
  }
  const int32_t *ints(PyObject *o, at::IntArrayRef shape) {
    const at::Tensor &t = tensor(o);
    need(t.scalar_type() == at::kInt && t.sizes() == shape && t.is_contiguous());
    return (const int32_t *)t.data_ptr();
  }
  // The device's current stream, where the device is the current one and the call names no stream
  void *stream(PyObject *named) {
    need(none(named));
    Object index(PyLong_FromLong(device_));
    if (index.get() == nullptr) throw Raised{};
    Object p(PyObject_CallOneArg(g_stream_of, index.get()));
    if (p.get() == nullptr) throw Raised{};
    need(!none(p.get()));
    void *s = PyLong_AsVoidPtr(p.get());
    if (s == nullptr && PyErr_Occurred()) throw Raised{};
    return s;
  }

 private:
  int device_ = -1;
};

int32_t int_arg(PyObject *o) {
  need(PyLong_CheckExact(o));
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    need(false);
  }
  need(x >= INT32_MIN && x <= INT32_MAX);
  return (int32_t)x;
}
float float_arg(PyObject *o) {
  need(PyFloat_CheckExact(o));
  return (float)PyFloat_AS_DOUBLE(o);
}
bool truth(PyObject *o) {
  need(PyBool_Check(o));
  return o == Py_True;
}
// A one-dimensional contiguous numpy array of one element type, held for the call.
class HostArray {
 public:
  HostArray(PyObject *o, char format, int itemsize) {
    need(Py_TYPE(o) == (PyTypeObject *)g_ndarray);
    if (PyObject_GetBuffer(o, &buf_, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
      PyErr_Clear();
      need(false);
    }
    if (!(buf_.ndim == 1 && buf_.itemsize == itemsize && buf_.format != nullptr && buf_.format[0] == format && buf_.format[1] == 0)) {
      PyBuffer_Release(&buf_);
      need(false);
    }
  }
  ~HostArray() { PyBuffer_Release(&buf_); }              // (not run where the constructor threw)
  HostArray(const HostArray &) = delete;
  HostArray &operator=(const HostArray &) = delete;
  const void *data() const { return buf_.buf; }
  int64_t size() const { return buf_.shape[0]; }

 private:
  Py_buffer buf_;
};

template <class F> void call(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  if (rc == SPARROW_OK) return;
  Object code(PyLong_FromLong(rc));
  if (code.get() != nullptr) Object(PyObject_CallOneArg(g_check, code.get()));
  throw Raised{};                                        // (_check raises SparrowError for every other status)
}
PyObject *tuple(std::initializer_list<at::Tensor> items) {      // an undefined tensor: None
  Object r(PyTuple_New((Py_ssize_t)items.size()));
  if (r.get() == nullptr) throw Raised{};
  Py_ssize_t i = 0;
  for (const at::Tensor &t : items) {
    PyObject *o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    if (o == nullptr) throw Raised{};
    PyTuple_SET_ITEM(r.get(), i++, o);
  }
  return Py_NewRef(r.get());
}

struct Table { int32_t *at; int32_t width; int64_t stride; };
Table table(Call &c, PyObject *o, int64_t B) {
  const at::Tensor &t = c.tensor(o);
  need(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == B && t.size(1) > 0 && t.size(1) <= INT32_MAX &&
       (t.size(1) == 1 || t.stride(1) == 1));
  return {(int32_t *)t.data_ptr(), (int32_t)t.size(1), B > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1))};
}
// [N, heads, d] with contiguous rows: elements between them
int64_t rows(const at::Tensor &t, int64_t heads, int64_t d, at::ScalarType type) {
  need(t.dim() == 3 && t.scalar_type() == type && t.size(1) == heads && t.size(2) == d && t.stride(2) == 1 && (heads == 1 || t.stride(1) == d));
  return t.size(0) > 1 ? t.stride(0) : heads * d;
}
// A cache of 8 bits with exponents, of `type` without; the exponents' address
struct Cache { sparrow_paged_desc desc; uint8_t *exponents; };
Cache cache_of(Call &c, PyObject *ko, PyObject *vo, PyObject *eo, at::ScalarType type, int64_t n_q_heads, float scale) {
  const at::Tensor &k = c.tensor(ko), &v = c.tensor(vo);
  need(k.dim() == 4 && k.stride(3) == 1 && v.strides() == k.strides() && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type());
  for (int i = 0; i < 4; ++i) need(k.size(i) > 0 && k.size(i) <= INT32_MAX);
  need(n_q_heads > 0 && n_q_heads <= INT32_MAX && (type == at::kBFloat16 || type == at::kFloat));
  Cache r;
  r.exponents = nullptr;
  if (none(eo)) {
    need(k.scalar_type() == type);
  } else {
    const at::Tensor &e = c.tensor(eo);
    need(k.scalar_type() == at::kFloat8_e4m3fn && e.scalar_type() == at::kByte && e.dim() == 4 && e.size(0) == k.size(0) && e.size(1) == k.size(2) &&
         e.size(2) == k.size(1) && e.size(3) == 2 && e.is_contiguous());
    r.exponents = (uint8_t *)e.data_ptr();
  }
  sparrow_paged_desc &d = r.desc;
  d.dtype = type == at::kBFloat16 ? SPARROW_BF16 : SPARROW_F32;
  d.n_q_heads = (int32_t)n_q_heads;
  d.n_kv_heads = (int32_t)k.size(2);
  d.head_dim = (int32_t)k.size(3);
  d.scale = scale;
  d.page_size = (int32_t)k.size(1);
  d.n_pages = (int32_t)k.size(0);
  d.kv_stride_page = k.size(0) > 1 ? k.stride(0) : std::max(k.stride(0), k.size(3));
  d.kv_stride_token = k.stride(1);
  d.kv_stride_head = k.size(2) > 1 ? k.stride(2) : k.size(3);
  d.q_stride_row = d.kv_stride_row = 0;
  return r;
}
struct Positions { const int32_t *at; int32_t axes; int64_t stride; };
Positions positions(const at::Tensor &t, int64_t N) {
  need(t.scalar_type() == at::kInt && (t.dim() == 1 || t.dim() == 2) && t.size(-1) == N && (N == 1 || t.stride(-1) == 1));
  if (t.dim() == 1) return {(const int32_t *)t.data_ptr(), 1, 0};
  need(t.size(0) <= INT32_MAX);
  return {(const int32_t *)t.data_ptr(), (int32_t)t.size(0), t.stride(0)};
}

// (q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, exponents, q_out, stream)
PyObject *mrope_append8(PyObject *const *a) {
  Call c;
  const at::Tensor &q = c.tensor(a[0]), &k = c.tensor(a[1]), &v = c.tensor(a[2]);
  need(q.dim() == 3 && k.dim() == 3 && v.dim() == 3 && q.size(0) > 0 && q.size(0) < 1 << 24 && !none(a[9]));
  const int64_t N = q.size(0), Hq = q.size(1);
  Cache cache = cache_of(c, a[7], a[8], a[9], q.scalar_type(), Hq, 0.f);
  sparrow_paged_desc &d = cache.desc;
  d.q_stride_row = rows(q, Hq, d.head_dim, q.scalar_type());
  d.kv_stride_row = rows(k, d.n_kv_heads, d.head_dim, q.scalar_type());
  need(rows(v, d.n_kv_heads, d.head_dim, q.scalar_type()) == d.kv_stride_row && k.size(0) == N && v.size(0) == N);
  const Positions p = positions(c.tensor(a[3]), N);
  const HostArray inv(a[4], 'd', 8), axis(a[5], 'i', 4);
  need(2 * inv.size() == d.head_dim && axis.size() == inv.size());
  const int32_t *slots = c.ints(a[6], {N});
  at::Tensor out;
  if (none(a[10])) {
    out = at::empty({N, Hq, q.size(2)}, q.options());
  } else {
    out = c.tensor(a[10]);
    need(out.scalar_type() == q.scalar_type() && out.sizes() == q.sizes() && out.is_contiguous());
  }
  void *const st = c.stream(a[11]);
  void *const pq = q.data_ptr(), *const pk = k.data_ptr(), *const pv = v.data_ptr(), *const po = out.data_ptr(),
             *const pkc = THPVariable_Unpack(a[7]).data_ptr(), *const pvc = THPVariable_Unpack(a[8]).data_ptr();
  call([&] {
    return lib.mrope_append8(&d, pq, pk, pv, p.at, p.stride, p.axes, (const double *)inv.data(), (const int32_t *)axis.data(), slots, (int32_t)N,
                             po, pkc, pvc, cache.exponents, st);
  });
  return none(a[10]) ? THPVariable_Wrap(out) : Py_NewRef(a[10]);
}

// (k_cache, v_cache, block_table, cu_rows, k_out, v_out, exponents, first, stream)
PyObject *page_gather(PyObject *const *a) {
  Call c;
  const at::Tensor &ko = c.tensor(a[4]), &vo = c.tensor(a[5]), &cu = c.tensor(a[3]);
  need(cu.dim() == 1 && cu.size(0) > 1 && cu.size(0) <= SPARROW_MAX_PAGED_BATCH + 1);
  const int64_t B = cu.size(0) - 1;
  const int32_t *pcu = c.ints(a[3], {B + 1}), *first = none(a[7]) ? nullptr : c.ints(a[7], {B});
  need(ko.dim() == 3 && ko.stride(2) == 1 && vo.strides() == ko.strides() && vo.sizes() == ko.sizes() && vo.scalar_type() == ko.scalar_type());
  const int64_t n = ko.size(0), heads = ko.size(1), d = ko.size(2);
  need(n > 0 && n <= INT32_MAX);
  const Cache cache = cache_of(c, a[0], a[1], a[6], ko.scalar_type(), heads, 0.f);
  need(heads == cache.desc.n_kv_heads && d == cache.desc.head_dim);
  const Table t = table(c, a[2], B);
  const int64_t row = n > 1 ? ko.stride(0) : d, head = heads > 1 ? ko.stride(1) : d;
  need(n == 1 || heads == 1 || row >= heads * head || head >= n * row);
  void *const st = c.stream(a[8]);
  void *const pk = THPVariable_Unpack(a[0]).data_ptr(), *const pv = THPVariable_Unpack(a[1]).data_ptr(), *const pko = ko.data_ptr(), *const pvo = vo.data_ptr();
  call([&] {
    return lib.page_gather(&cache.desc, pk, pv, cache.exponents, t.at, t.width, t.stride, first, pcu, (int32_t)B, (int32_t)n, pko, pvo, row, head, st);
  });
  return tuple({ko, vo});
}

// Of both attentions; eight: without groups, an 8-bit cache
struct AttnArguments {
  PyObject *q, *k, *v, *exponents, *table, *cu, *len, *start, *prefix, *max_new, *scale, *out, *lse, *want, *workspace, *stream;
};
PyObject *attention(const AttnArguments &a, bool eight) {
  Call c;
  const at::Tensor &q = c.tensor(a.q), &len = c.tensor(a.len);
  need(q.dim() == 3 && len.dim() == 1 && len.size(0) > 0 && len.size(0) <= SPARROW_MAX_PAGED_BATCH && q.size(0) > 0 && q.size(0) <= INT32_MAX);
  const int64_t N = q.size(0), Hq = q.size(1), B = len.size(0);
  Cache cache = cache_of(c, a.k, a.v, a.exponents, q.scalar_type(), Hq, float_arg(a.scale));
  sparrow_paged_desc &d = cache.desc;
  d.q_stride_row = rows(q, Hq, d.head_dim, q.scalar_type());
  const Table t = table(c, a.table, B);
  const int32_t *cu = c.ints(a.cu, {B + 1}), *kv = c.ints(a.len, {B}), *start = nullptr, *prefix = nullptr;
  int64_t G = 0;
  if (!none(a.start)) {
    const at::Tensor &gs = c.tensor(a.start);
    need(gs.dim() == 1 && gs.size(0) > 0 && gs.size(0) <= SPARROW_MAX_PREFIX_GROUPS + 1);
    G = gs.size(0) - 1;
    start = c.ints(a.start, {G + 1});
    prefix = c.ints(a.prefix, {G});
  }
  const int32_t max_new = int_arg(a.max_new);
  at::Tensor out, lse, ws;
  if (none(a.out)) {
    out = at::empty({N, Hq, q.size(2)}, q.options());
  } else {
    out = c.tensor(a.out);
    need(out.scalar_type() == q.scalar_type() && out.sizes() == q.sizes() && out.is_contiguous());
  }
  const bool want = truth(a.want);
  if (none(a.lse)) {
    if (want) lse = at::empty({N, Hq}, q.options().dtype(at::kFloat));
  } else {
    lse = c.tensor(a.lse);
    need(lse.scalar_type() == at::kFloat && lse.dim() == 2 && lse.size(0) == N && lse.size(1) == Hq && lse.is_contiguous());
  }
  if (none(a.workspace)) {
    const size_t bytes = lib.prefix_attn_workspace(&d, (int32_t)B, (int32_t)G, (int32_t)N, max_new);
    if (bytes > 0) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
  } else {
    ws = c.tensor(a.workspace);
    need(ws.is_contiguous());
  }
  void *const st = c.stream(a.stream);
  void *const pq = q.data_ptr(), *const pk = THPVariable_Unpack(a.k).data_ptr(), *const pv = THPVariable_Unpack(a.v).data_ptr(), *const po = out.data_ptr(),
             *const pl = lse.defined() ? lse.data_ptr() : nullptr, *const pw = ws.defined() ? ws.data_ptr() : nullptr;
  const size_t ws_bytes = ws.defined() ? (size_t)(ws.numel() * ws.element_size()) : 0;
  call([&] {
    return eight ? lib.chunk_attn8(&d, pq, pk, pv, cache.exponents, t.at, t.width, t.stride, cu, kv, (int32_t)B, (int32_t)N, max_new, po, (float *)pl, pw,
                                   ws_bytes, st)
                 : lib.prefix_attn(&d, pq, pk, pv, cache.exponents, t.at, t.width, t.stride, cu, kv, (int32_t)B, start, prefix, (int32_t)G, (int32_t)N,
                                   max_new, po, (float *)pl, pw, ws_bytes, st);
  });
  return tuple({out, lse});
}

// (q, k_cache, v_cache, exponents, block_table, cu_new, kv_len, max_new, scale, out, lse, want_lse, workspace, stream)
PyObject *chunk_attn8(PyObject *const *a) {
  need(!none(a[3]));
  return attention({a[0], a[1], a[2], a[3], a[4], a[5], a[6], Py_None, Py_None, a[7], a[8], a[9], a[10], a[11], a[12], a[13]}, true);
}
// (q, k_cache, v_cache, block_table, cu_new, kv_len, group_start, prefix_len, max_new, exponents, scale, out, lse, want_lse, workspace, stream)
PyObject *prefix_attn(PyObject *const *a) {
  return attention({a[0], a[1], a[2], a[9], a[3], a[4], a[5], a[6], a[7], a[8], a[10], a[11], a[12], a[13], a[14], a[15]}, false);
}

template <PyObject *(*kCall)(PyObject *const *), int kArgs>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  if (g_check == nullptr || at::impl::torch_function_mode_enabled()) return Py_NewRef(Py_NotImplemented);
  try {
    return kCall(args);
  } catch (const NotHere &) {
    return Py_NewRef(Py_NotImplemented);
  } catch (const Raised &) {
    return nullptr;
  } catch (const std::exception &) {                     // torch refused (no memory, no data pointer): let it say so in Python
    return Py_NewRef(Py_NotImplemented);
  }
}

// setup(check, stream_of, ndarray, addresses of FUNCTIONS...)
PyObject *setup(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 3 + kNumFunctions) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  void *at[kNumFunctions];
  for (int i = 0; i < kNumFunctions; ++i) {
    at[i] = PyLong_AsVoidPtr(args[3 + i]);
    if (at[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s has no address", kFunctions[i]);
      return nullptr;
    }
  }
  std::memcpy(&lib, at, sizeof(lib));
  g_check = Py_NewRef(args[0]);
  g_stream_of = Py_NewRef(args[1]);
  g_ndarray = Py_NewRef(args[2]);
  Py_RETURN_NONE;
}

#define SPARROW_ENTRY(f, n) {#f, (PyCFunction)(void (*)())entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SPARROW_ENTRY(mrope_append8, 12), SPARROW_ENTRY(page_gather, 9), SPARROW_ENTRY(chunk_attn8, 14),
                         SPARROW_ENTRY(prefix_attn, 16), {"setup", (PyCFunction)(void (*)())setup, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_serve", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_serve(void) {
  Object m(PyModule_Create(&module)), names(PyTuple_New(kNumFunctions));
  if (m.get() == nullptr || names.get() == nullptr) return nullptr;
  for (int i = 0; i < kNumFunctions; ++i) {
    PyObject *s = PyUnicode_FromString(kFunctions[i]);
    if (s == nullptr) return nullptr;
    PyTuple_SET_ITEM(names.get(), i, s);
  }
  if (PyObject_SetAttrString(m.get(), "FUNCTIONS", names.get()) != 0 || PyModule_AddStringConstant(m.get(), "BUILT_FOR", kBuiltFor) != 0)
    return nullptr;
  return Py_NewRef(m.get());
}
