// The Python entry of the serving operators (paper_2002_12798_b200/ops.py): checks of tensors, allocation of outputs and the
// C call (amap_serve.h), for steps of small kernels whose time would otherwise be the interpreter's.  PyTorch gives
// device memory and streams, nothing else.
//
// Functions take positional arguments only and are called by ops.py, which documents them.  Plans, caches and attention's
// fixed arguments arrive as addresses of the C structs that ops.py keeps alive.
#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/core/AutogradState.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/VariableTypeUtils.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "amap_serve.h"

namespace {

PyObject *g_refusal = nullptr;  // binding.AmapError(code, where)

// thrown with a Python error set
struct Raised {};

[[noreturn]] void refuse_value(const char *why) {
  PyErr_SetString(PyExc_ValueError, why);
  throw Raised();
}
[[noreturn]] void refuse_value(const char *name, const char *why) {
  PyErr_Format(PyExc_ValueError, "%s: %s", name, why);
  throw Raised();
}
inline void require(bool ok, const char *why) {
  if (C10_UNLIKELY(!ok)) refuse_value(why);
}
void check(int rc, const char *where) {
  if (C10_LIKELY(rc == AMAP_OK)) return;
  const char *why = amap_serve_error();
  PyObject *text = PyUnicode_FromFormat(*why ? "%s (%s)" : "%s", where, why);
  PyObject *error = text ? PyObject_CallFunction(g_refusal, "iN", rc, text) : nullptr;
  if (error) {
    PyErr_SetObject(g_refusal, error);
    Py_DECREF(error);
  }
  throw Raised();
}

inline const at::Tensor &tensor(PyObject *o, const char *name) {
  if (C10_UNLIKELY(!THPVariable_Check(o))) refuse_value(name, "not a tensor");
  return THPVariable_Unpack(o);
}
inline int64_t integer(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
inline int32_t integer32(PyObject *o) {
  const int64_t v = integer(o);
  require(v >= INT32_MIN && v <= INT32_MAX, "a number beyond 32 bits");
  return (int32_t)v;
}
template <typename T> inline T *address(PyObject *o) { return reinterpret_cast<T *>((uintptr_t)integer(o)); }

// the current stream of the tensors' device, which has to be the current device: kernels are launched there
inline void *stream_of(int device) {
  if (C10_UNLIKELY(device < 0)) refuse_value("the tensors are on the CPU");
  if (C10_UNLIKELY(device != c10::cuda::current_device())) refuse_value("the tensors are not on the current device (torch.cuda.device)");
  return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
}
inline int cuda_of(const at::Tensor &t) { return t.is_cuda() ? t.get_device() : -1; }

// address of n int32 numbers that lie side by side on the device
inline int32_t *ints(PyObject *o, const char *name, int64_t n, int device) {
  const at::Tensor &t = tensor(o, name);
  if (C10_UNLIKELY(t.scalar_type() != at::kInt || cuda_of(t) != device || t.numel() != n || !t.is_contiguous()))
    refuse_value(name, "contiguous int32 numbers, as many as the other tensors say, on their device");
  return static_cast<int32_t *>(t.data_ptr());
}

struct Table {
  int32_t *at;
  int32_t rows, entries;
  int64_t stride;
  int device;
};
inline Table table_of(PyObject *o) {
  const at::Tensor &t = tensor(o, "block_table");
  if (C10_UNLIKELY(t.scalar_type() != at::kInt || !t.is_cuda() || t.dim() != 2 || (t.stride(1) != 1 && t.size(1) > 1) || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX))
    refuse_value("block_table: an int32 CUDA tensor [requests, pages] with contiguous rows");
  const int64_t stride = t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
  return {static_cast<int32_t *>(t.data_ptr()), (int32_t)t.size(0), (int32_t)t.size(1), stride, cuda_of(t)};
}

inline void heads_of(const at::Tensor &t, const char *name, int64_t dim, int device) {
  if (C10_UNLIKELY(t.dim() != 3 || t.size(2) != dim || (t.stride(2) != 1 && dim > 1) || cuda_of(t) != device || t.size(1) > INT32_MAX))
    refuse_value(name, "a CUDA tensor [tokens, heads, head_dim] whose heads are contiguous, on the device of the other tensors");
}
inline int32_t type_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return AMAP_BF16;
    case at::kHalf: return AMAP_FP16;
    case at::kFloat: return AMAP_FP32;
    default: return 0;  // refused by the C call
  }
}

// an output: given, or made like its input
inline at::Tensor output(PyObject *given, const at::Tensor &like, int64_t dim, int device) {
  if (given == Py_None) return at::empty_like(like);
  const at::Tensor &t = tensor(given, "out");
  heads_of(t, "out", dim, device);
  require(t.scalar_type() == like.scalar_type() && t.sizes() == like.sizes(), "out: of its input's shape and type");
  return t;
}

struct Positions {
  const void *at;
  int64_t axis, row;
  int32_t bits;
};
inline Positions positions_of(PyObject *o, int64_t tokens, int64_t axes, int device) {
  const at::Tensor &t = tensor(o, "positions");
  const int64_t d = t.dim();
  if (C10_UNLIKELY((d != 1 && d != 2) || t.size(d - 1) != tokens || (d == 2 ? t.size(0) : 1) < axes || cuda_of(t) != device))
    refuse_value("positions: [tokens] or [axes, tokens], one per token and axis, on the device of the other tensors");
  const int bits = t.scalar_type() == at::kInt ? 32 : t.scalar_type() == at::kLong ? 64 : 0;
  require(bits != 0, "positions: int32 or int64");
  return {t.data_ptr(), d == 2 ? t.stride(0) : 0, t.stride(d - 1), bits};
}

// whether autograd, backward or forward, follows a tensor at this call (a view's tangent is asked for only where there can be
// one: looking for it costs 0.1 us)
template <typename... T>
inline bool tracked(const T &...t) {
  if ((t.requires_grad() || ...) && at::GradMode::is_enabled()) return true;
  return c10::AutogradState::get_tls_state().get_fw_grad_mode() && torch::autograd::ForwardADLevel::try_get_by_idx(0) &&
         (torch::autograd::isFwGradDefined(t) || ...);
}

inline PyObject *wrap(at::Tensor t) {
  PyObject *o = THPVariable_Wrap(std::move(t));
  if (!o) throw Raised();
  return o;
}
PyObject *wrap_all(const at::Tensor *t, int n) {
  PyObject *all = PyTuple_New(n);
  if (!all) throw Raised();
  for (int i = 0; i < n; ++i) {
    PyObject *o = THPVariable_Wrap(t[i]);
    if (!o) {
      Py_DECREF(all);
      throw Raised();
    }
    PyTuple_SET_ITEM(all, i, o);
  }
  return all;
}

// nothing thrown passes into the interpreter
template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens, n_pages (None), out (None) -> the seven
PyObject *extend(PyObject *const *a) {
  const Table t = table_of(a[2]);
  void *stream = stream_of(t.device);
  amap_pages_extend_args g;
  memset(&g, 0, sizeof g);
  const at::Tensor &free_pages = tensor(a[3], "free_pages");
  require(free_pages.numel() <= INT32_MAX, "free_pages: too many");
  g.n_requests = t.rows, g.max_pages = t.entries, g.page_size = integer32(a[5]), g.max_tokens = integer32(a[6]);
  g.free_capacity = (int32_t)free_pages.numel(), g.n_pages = a[7] == Py_None ? g.free_capacity : integer32(a[7]);
  g.table_stride = t.stride, g.block_table = t.at;
  g.new_lens = ints(a[0], "new_lens", t.rows, t.device), g.seq_lens = ints(a[1], "seq_lens", t.rows, t.device);
  g.free_pages = ints(a[3], "free_pages", g.free_capacity, t.device), g.free_count = ints(a[4], "free_count", 1, t.device);
  const int64_t n = t.rows, m = std::max(g.max_tokens, 0), sizes[7] = {n + 1, m, m, m, n, 1, n};
  int32_t **const to[7] = {&g.query_start, &g.slots, &g.positions, &g.requests, &g.seq_lens_out, &g.free_count_out, &g.status};
  at::Tensor out[7];
  if (a[8] == Py_None) {
    at::AutoDispatchBelowADInplaceOrView plain;
    const at::Tensor whole = at::empty({3 * n + 2 + 3 * m}, free_pages.options());
    int64_t at = 0;
    for (int i = 0; i < 7; at += sizes[i++]) {
      out[i] = whole.narrow(0, at, sizes[i]);
      *to[i] = static_cast<int32_t *>(whole.data_ptr()) + at;
    }
    check(amap_pages_extend(&g, stream), "amap_pages_extend");
    return wrap_all(out, 7);
  }
  static const char *const names[7] = {"query_start", "slots", "positions", "requests", "seq_lens", "free_count", "status"};
  require(PyTuple_Check(a[8]) && PyTuple_GET_SIZE(a[8]) == 7, "out: a PagesStep");
  for (int i = 0; i < 7; ++i) *to[i] = ints(PyTuple_GET_ITEM(a[8], i), names[i], sizes[i], t.device);
  check(amap_pages_extend(&g, stream), "amap_pages_extend");
  Py_INCREF(a[8]);
  return a[8];
}

// done, seq_lens, block_table, free_pages, free_count, page_size, n_pages (None) -> seq_lens, free_count
PyObject *release(PyObject *const *a) {
  const Table t = table_of(a[2]);
  void *stream = stream_of(t.device);
  const at::Tensor &done = tensor(a[0], "done"), &free_pages = tensor(a[3], "free_pages");
  if ((done.scalar_type() != at::kBool && done.scalar_type() != at::kByte) || cuda_of(done) != t.device || done.numel() != t.rows || !done.is_contiguous())
    refuse_value("done: contiguous bool or uint8 values, one per request, on the device of the other tensors");
  require(free_pages.numel() <= INT32_MAX, "free_pages: too many");
  amap_pages_release_args g;
  memset(&g, 0, sizeof g);
  g.n_requests = t.rows, g.max_pages = t.entries, g.page_size = integer32(a[5]), g.free_capacity = (int32_t)free_pages.numel();
  g.table_stride = t.stride, g.block_table = t.at, g.done = static_cast<const uint8_t *>(done.data_ptr());
  g.seq_lens = ints(a[1], "seq_lens", t.rows, t.device), g.free_pages = ints(a[3], "free_pages", g.free_capacity, t.device);
  g.free_count = ints(a[4], "free_count", 1, t.device);
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor whole = at::empty({(int64_t)t.rows + 1}, free_pages.options());
  g.seq_lens_out = static_cast<int32_t *>(whole.data_ptr()), g.free_count_out = g.seq_lens_out + t.rows;
  check(amap_pages_release_within(&g, a[6] == Py_None ? INT32_MAX : integer32(a[6]), stream), "amap_pages_release");
  const at::Tensor out[2] = {whole.narrow(0, 0, t.rows), whole.narrow(0, t.rows, 1)};
  return wrap_all(out, 2);
}

// plan, head_dim, axes, xs, positions, inverse, outs (None) -> outs
PyObject *rotate(PyObject *const *a) {
  const int64_t dim = integer(a[1]);
  PyObject *const xs = a[3], *const ys = a[6];
  require((PyList_Check(xs) || PyTuple_Check(xs)) && (ys == Py_None || PyList_Check(ys) || PyTuple_Check(ys)), "rotate: lists of tensors");
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(xs);
  require(n >= 1 && n <= 4, "rotate takes 1 to 4 tensors");
  require(ys == Py_None || PySequence_Fast_GET_SIZE(ys) == n, "outs: one per tensor");
  amap_rope_args g;
  memset(&g, 0, sizeof g);
  at::Tensor out[4];
  const at::Tensor &first = tensor(PySequence_Fast_GET_ITEM(xs, 0), "x");
  const int device = cuda_of(first);
  void *stream = stream_of(device);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor &x = tensor(PySequence_Fast_GET_ITEM(xs, i), "x");
    heads_of(x, "x", dim, device);
    require(x.scalar_type() == first.scalar_type() && x.size(0) == first.size(0), "rotate: tensors of one type and token count");
    out[i] = output(ys == Py_None ? Py_None : PySequence_Fast_GET_ITEM(ys, i), x, dim, device);
    g.part[i] = {x.data_ptr(), out[i].data_ptr(), x.stride(0), x.stride(1), out[i].stride(0), out[i].stride(1), (int32_t)x.size(1), 0};
  }
  const Positions p = positions_of(a[4], first.size(0), integer(a[2]), device);
  g.n_parts = (int32_t)n, g.dtype = type_of(first), g.rows = first.size(0), g.positions = p.at, g.position_axis = p.axis, g.position_row = p.row;
  g.position_bits = p.bits, g.inverse = PyObject_IsTrue(a[5]);
  if (g.rows) check(amap_rope_rotate(address<const amap_rope_t>(a[0]), &g, stream), "amap_rope_rotate");
  PyObject *all = PyList_New(n);
  if (!all) throw Raised();
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *o = THPVariable_Wrap(out[i]);
    if (!o) {
      Py_DECREF(all);
      throw Raised();
    }
    PyList_SET_ITEM(all, i, o);
  }
  return all;
}

// plan, head_dim, axes, q, k, v, positions, slots, cache, its device, out (None) -> out; NotImplemented, and nothing done, where
// autograd follows an input
PyObject *append(PyObject *const *a) {
  const int64_t dim = integer(a[1]);
  const at::Tensor &q = tensor(a[3], "q"), &k = tensor(a[4], "k"), &v = tensor(a[5], "v");
  if (C10_UNLIKELY(tracked(q, k, v))) Py_RETURN_NOTIMPLEMENTED;
  const int device = cuda_of(q);
  void *stream = stream_of(device);
  heads_of(q, "q", dim, device);
  heads_of(k, "k", dim, device);
  heads_of(v, "v", dim, device);
  amap_append_args g;
  memset(&g, 0, sizeof g);
  memcpy(&g.cache, address<const amap_cache>(a[8]), sizeof g.cache);
  require(k.sizes() == v.sizes() && k.size(0) == q.size(0) && k.size(1) == g.cache.heads && k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type(),
          "append: q, k and v of one type and token count, k and v with the cache's heads");
  require(integer(a[9]) == device, "append: the cache is on another device");
  const Positions p = positions_of(a[6], q.size(0), integer(a[2]), device);
  g.slots = ints(a[7], "slots", q.size(0), device);
  at::Tensor out = output(a[10], q, dim, device);
  g.rows = q.size(0), g.dtype = type_of(q), g.q_heads = (int32_t)q.size(1);
  g.q = q.data_ptr(), g.k = k.data_ptr(), g.v = v.data_ptr(), g.q_out = out.data_ptr();
  g.q_row = q.stride(0), g.q_head = q.stride(1), g.k_row = k.stride(0), g.k_head = k.stride(1), g.v_row = v.stride(0), g.v_head = v.stride(1);
  g.q_out_row = out.stride(0), g.q_out_head = out.stride(1);
  g.positions = p.at, g.position_axis = p.axis, g.position_row = p.row, g.position_bits = p.bits;
  if (g.rows) check(amap_rope_append(address<const amap_rope_t>(a[0]), &g, stream), "amap_rope_append");
  return wrap(std::move(out));
}

// the plan's fixed arguments, its device, most requests, head_dim, q, cache, maps, the cache's device, block_table, seq_lens, out (None), lse (bool)
// -> out, or (out, lse); NotImplemented, and nothing done, where autograd follows q
PyObject *attend(PyObject *const *a) {
  amap_attend_args g;
  memcpy(&g, address<const amap_attend_args>(a[0]), sizeof g);  // q_heads, cache.heads, scale, softcap, window, workspace
  const int device = (int)integer(a[1]);
  void *stream = stream_of(device);
  const int64_t dim = integer(a[3]);
  const at::Tensor &q = tensor(a[4], "q");
  if (C10_UNLIKELY(tracked(q))) Py_RETURN_NOTIMPLEMENTED;
  heads_of(q, "q", dim, device);
  const Table t = table_of(a[8]);
  const int32_t kv_heads = g.cache.heads;
  memcpy(&g.cache, address<const amap_cache>(a[5]), sizeof g.cache);
  require(q.size(0) <= integer(a[2]) && t.rows == q.size(0), "attend: no more requests than the plan is for, each with a row of the block table");
  require(q.size(1) == g.q_heads && g.cache.heads == kv_heads && g.cache.head_dim == dim, "attend: the plan is for other heads");
  require(integer(a[7]) == device && t.device == device, "attend: plan, q, block_table and cache on one device");
  g.maps = address<const amap_cache_maps>(a[6]);
  g.seq_lens = ints(a[9], "seq_lens", t.rows, device);
  at::Tensor out[2];
  out[0] = output(a[10], q, dim, device);
  const bool lse = PyObject_IsTrue(a[11]) == 1;
  if (lse) {
    out[1] = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
    g.lse = static_cast<float *>(out[1].data_ptr()), g.lse_row = g.q_heads;
  }
  g.n_requests = t.rows, g.dtype = type_of(q), g.max_pages = t.entries, g.block_table = t.at, g.table_stride = t.stride;
  g.q = q.data_ptr(), g.out = out[0].data_ptr();
  g.q_row = q.stride(0), g.q_head = q.stride(1), g.out_row = out[0].stride(0), g.out_head = out[0].stride(1);
  if (t.rows) check(amap_attend(&g, stream), "amap_attend");
  return lse ? wrap_all(out, 2) : wrap(std::move(out[0]));
}

PyObject *refuse_with(PyObject *, PyObject *error) {
  Py_INCREF(error);
  Py_XSETREF(g_refusal, error);
  Py_RETURN_NONE;
}

#define ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&guarded<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {ENTRY(extend, 9), ENTRY(release, 7), ENTRY(rotate, 7), ENTRY(append, 11), ENTRY(attend, 12),
                          {"refuse_with", refuse_with, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
// the build looks for this text in the library (build.py)
const char kBuiltAgainst[] = SERVE_BUILT_AGAINST;
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_serve_torch", kBuiltAgainst, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__serve_torch(void) { return PyModule_Create(&kModule); }
