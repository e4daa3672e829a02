// The paged-cache operators without Python between the arguments and the library: page_update, mrope_table, mrope_append and chunk_attn for
// arguments as programs pass them.  Each function returns NotImplemented where an argument is anything else (a tensor subclass, another
// dtype, shape or stride than the library takes, a tensor that is not on the current GPU, a stream of its own, ...) or a torch function mode
// is active; paged.py's own code then takes the call, converts what can be converted and raises what has to be raised.  Nothing is
// kept between calls.
//
// us a call and its kernel in an unbroken row of them, ctypes / here (by machine): mrope_table of six rows 8.0 / 3.8 to 4.4, mrope_append of 13 rows
// 11.9 / 4.4 to 4.5, two calls of page_update and a copy 30 / 14.7 to 16.6.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstring>

#include "../../../include/sparrow_paged.h"

namespace {

PyObject *g_check, *g_stream_of, *g_ndarray;             // paged._check, paged._stream_of, numpy.ndarray

// The library's functions, in the copy of the library that paged.py has loaded.
#define SPARROW_FUNCTIONS(f) f(page_update) f(mrope_table) f(mrope_append) f(chunk_attn_workspace) f(chunk_attn)
struct Library {
#define SPARROW_MEMBER(n) decltype(&sparrow_##n) n;
  SPARROW_FUNCTIONS(SPARROW_MEMBER)
} lib;
#define SPARROW_STRING_OF(x) #x
#define SPARROW_STRING(x) SPARROW_STRING_OF(x)
#define SPARROW_NAME(n) "sparrow_" #n,
constexpr const char *kFunctions[] = {SPARROW_FUNCTIONS(SPARROW_NAME)};
// Code compiled against the headers of one torch and one Python reads another's objects wrongly, without an error:
// paged.py takes this part only where it runs under the same ones.
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
int32_t dtype_code(const at::Tensor &t) {
  if (t.scalar_type() == at::kBFloat16) return SPARROW_BF16;
  need(t.scalar_type() == at::kFloat);
  return SPARROW_F32;
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

// The part of a one-dimensional tensor from `first` on: an allocation of its own costs the host more.
at::Tensor part(const at::Tensor &whole, int64_t first, int64_t n) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(first);
  t.unsafeGetTensorImpl()->set_sizes_contiguous({n});
  return t;
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
sparrow_paged_desc desc_of(const at::Tensor &k, const at::Tensor &v, int64_t n_q_heads, float scale) {
  need(k.dim() == 4 && k.stride(3) == 1 && v.strides() == k.strides() && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type());
  for (int i = 0; i < 4; ++i) need(k.size(i) > 0 && k.size(i) <= INT32_MAX);
  need(n_q_heads > 0 && n_q_heads <= INT32_MAX);
  sparrow_paged_desc d;
  d.dtype = dtype_code(k);
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
  return d;
}
struct Positions { const int32_t *at; int32_t axes; int64_t stride; };
Positions positions(const at::Tensor &t, int64_t N) {
  need(t.scalar_type() == at::kInt && (t.dim() == 1 || t.dim() == 2) && t.size(-1) == N && (N == 1 || t.stride(-1) == 1));
  if (t.dim() == 1) return {(const int32_t *)t.data_ptr(), 1, 0};
  need(t.size(0) <= INT32_MAX);
  return {(const int32_t *)t.data_ptr(), (int32_t)t.size(0), t.stride(0)};
}

// (old_len, new_len, block_table, free_pages, n_free, page_size, n_rows, pos_offset, outputs, stream)
PyObject *page_update(PyObject *const *a) {
  Call c;
  const at::Tensor &old = c.tensor(a[0]);
  need(old.dim() == 1 && old.size(0) > 0 && old.size(0) <= SPARROW_MAX_PAGED_BATCH);
  const int64_t B = old.size(0);
  const int32_t *po = c.ints(a[0], {B}), *pn = c.ints(a[1], {B});
  const Table t = table(c, a[2], B);
  const at::Tensor &free = c.tensor(a[3]);
  need(free.dim() == 1 && free.scalar_type() == at::kInt && free.is_contiguous() && free.size(0) <= INT32_MAX);
  int32_t *n_free = (int32_t *)c.ints(a[4], {1});
  const int32_t page = int_arg(a[5]), n = int_arg(a[6]);
  need(n >= 0);
  const int32_t *off = none(a[7]) ? nullptr : c.ints(a[7], {B});
  at::Tensor out[4];
  const int64_t sizes[4] = {n, B + 1, n, 1};
  if (none(a[8])) {
    const at::Tensor whole = at::empty({sizes[0] + sizes[1] + sizes[2] + sizes[3]}, old.options());
    int64_t first = 0;
    for (int i = 0; i < 4; ++i) {
      out[i] = part(whole, first, sizes[i]);
      first += sizes[i];
    }
  } else {
    need(PyTuple_CheckExact(a[8]) && PyTuple_GET_SIZE(a[8]) == 4);
    for (int i = 0; i < 4; ++i) {
      c.ints(PyTuple_GET_ITEM(a[8], i), {sizes[i]});
      out[i] = c.tensor(PyTuple_GET_ITEM(a[8], i));
    }
  }
  void *const st = c.stream(a[9]), *const pf = free.data_ptr();
  int32_t *p[4];
  for (int i = 0; i < 4; ++i) p[i] = (int32_t *)out[i].data_ptr();
  const int32_t capacity = (int32_t)free.size(0);
  call([&] {
    return lib.page_update(po, pn, (int32_t)B, page, t.at, t.width, t.stride, (int32_t *)pf, capacity, n_free, off, n, p[0], p[2], p[1], p[3], st);
  });
  return tuple({out[0], out[1], out[2], out[3]});
}

// (positions, inv_freq, freq_axis, cos, sin, stream)
PyObject *mrope_table(PyObject *const *a) {
  Call c;
  const at::Tensor &pos = c.tensor(a[0]);
  need((pos.dim() == 1 || pos.dim() == 2) && pos.size(-1) > 0 && pos.size(-1) < 1 << 24);
  const int64_t N = pos.size(-1);
  const Positions p = positions(pos, N);
  const HostArray inv(a[1], 'd', 8), axis(a[2], 'i', 4);
  const int64_t half = inv.size();
  need((half == 32 || half == 64) && axis.size() == half);
  at::Tensor out[2];
  for (int i = 0; i < 2; ++i) {
    if (none(a[3 + i])) {
      out[i] = at::empty({N, half}, pos.options().dtype(at::kFloat));
    } else {
      out[i] = c.tensor(a[3 + i]);
      need(out[i].scalar_type() == at::kFloat && out[i].dim() == 2 && out[i].size(0) == N && out[i].size(1) == half && out[i].is_contiguous());
    }
  }
  void *const st = c.stream(a[5]);
  float *const pc = (float *)out[0].data_ptr(), *const ps = (float *)out[1].data_ptr();
  call([&] {
    return lib.mrope_table(p.at, p.stride, p.axes, (const double *)inv.data(), (const int32_t *)axis.data(), (int32_t)(2 * half), (int32_t)N, pc, ps, st);
  });
  return tuple({out[0], out[1]});
}

// (q, k, v, positions, inv_freq, freq_axis, slots, k_cache, v_cache, q_out, stream)
PyObject *mrope_append(PyObject *const *a) {
  Call c;
  const at::Tensor &q = c.tensor(a[0]), &k = c.tensor(a[1]), &v = c.tensor(a[2]), &kc = c.tensor(a[7]), &vc = c.tensor(a[8]);
  need(q.dim() == 3 && k.dim() == 3 && v.dim() == 3 && q.size(0) > 0 && q.size(0) < 1 << 24);
  const int64_t N = q.size(0), Hq = q.size(1);
  sparrow_paged_desc d = desc_of(kc, vc, Hq, 0.f);
  d.q_stride_row = rows(q, Hq, d.head_dim, kc.scalar_type());
  d.kv_stride_row = rows(k, d.n_kv_heads, d.head_dim, kc.scalar_type());
  need(rows(v, d.n_kv_heads, d.head_dim, kc.scalar_type()) == d.kv_stride_row && k.size(0) == N && v.size(0) == N);
  const Positions p = positions(c.tensor(a[3]), N);
  const HostArray inv(a[4], 'd', 8), axis(a[5], 'i', 4);
  need(2 * inv.size() == d.head_dim && axis.size() == inv.size());
  const int32_t *slots = c.ints(a[6], {N});
  at::Tensor out;
  if (none(a[9])) {
    out = at::empty({N, Hq, q.size(2)}, q.options());
  } else {
    out = c.tensor(a[9]);
    need(out.scalar_type() == q.scalar_type() && out.sizes() == q.sizes() && out.is_contiguous());
  }
  void *const st = c.stream(a[10]);
  void *const pq = q.data_ptr(), *const pk = k.data_ptr(), *const pv = v.data_ptr(), *const po = out.data_ptr(), *const pkc = kc.data_ptr(),
             *const pvc = vc.data_ptr();
  call([&] {
    return lib.mrope_append(&d, pq, pk, pv, p.at, p.stride, p.axes, (const double *)inv.data(), (const int32_t *)axis.data(), slots, (int32_t)N,
                            po, pkc, pvc, st);
  });
  return none(a[9]) ? THPVariable_Wrap(out) : Py_NewRef(a[9]);
}

// (q, k_cache, v_cache, block_table, cu_new, kv_len, max_new, scale, out, lse, want_lse, workspace, stream)
PyObject *chunk_attn(PyObject *const *a) {
  Call c;
  const at::Tensor &q = c.tensor(a[0]), &k = c.tensor(a[1]), &v = c.tensor(a[2]), &len = c.tensor(a[5]);
  need(q.dim() == 3 && len.dim() == 1 && len.size(0) > 0 && len.size(0) <= SPARROW_MAX_PAGED_BATCH && q.size(0) > 0 && q.size(0) <= INT32_MAX);
  const int64_t N = q.size(0), Hq = q.size(1), B = len.size(0);
  sparrow_paged_desc d = desc_of(k, v, Hq, float_arg(a[7]));
  d.q_stride_row = rows(q, Hq, d.head_dim, k.scalar_type());
  const Table t = table(c, a[3], B);
  const int32_t *cu = c.ints(a[4], {B + 1}), *kv = c.ints(a[5], {B});
  const int32_t max_new = int_arg(a[6]);
  at::Tensor out, lse, ws;
  if (none(a[8])) {
    out = at::empty({N, Hq, q.size(2)}, q.options());
  } else {
    out = c.tensor(a[8]);
    need(out.scalar_type() == q.scalar_type() && out.sizes() == q.sizes() && out.is_contiguous());
  }
  const bool want = truth(a[10]);
  if (none(a[9])) {
    if (want) lse = at::empty({N, Hq}, q.options().dtype(at::kFloat));
  } else {
    lse = c.tensor(a[9]);
    need(lse.scalar_type() == at::kFloat && lse.dim() == 2 && lse.size(0) == N && lse.size(1) == Hq && lse.is_contiguous());
  }
  if (none(a[11])) {
    const size_t bytes = lib.chunk_attn_workspace(&d, (int32_t)B, (int32_t)N, max_new);
    if (bytes > 0) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
  } else {
    ws = c.tensor(a[11]);
    need(ws.is_contiguous());
  }
  void *const st = c.stream(a[12]);
  void *const pq = q.data_ptr(), *const pk = k.data_ptr(), *const pv = v.data_ptr(), *const po = out.data_ptr(),
             *const pl = lse.defined() ? lse.data_ptr() : nullptr, *const pw = ws.defined() ? ws.data_ptr() : nullptr;
  const size_t ws_bytes = ws.defined() ? (size_t)(ws.numel() * ws.element_size()) : 0;
  call([&] {
    return lib.chunk_attn(&d, pq, pk, pv, t.at, t.width, t.stride, cu, kv, (int32_t)B, (int32_t)N, max_new, po, (float *)pl, pw, ws_bytes, st);
  });
  return tuple({out, lse});
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
PyMethodDef methods[] = {SPARROW_ENTRY(page_update, 10), SPARROW_ENTRY(mrope_table, 6), SPARROW_ENTRY(mrope_append, 11),
                         SPARROW_ENTRY(chunk_attn, 13), {"setup", (PyCFunction)(void (*)())setup, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native_paged", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_paged(void) {
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
