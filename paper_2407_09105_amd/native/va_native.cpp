// The calls of `binding` that a training or a decoding step makes per layer, without their Python: the checks, the output
// allocations and the library call of one pass in one C++ call each.
//
// A pass over 16 tokens (boundaries, forward, backward: four kernels of 3 to 6 us) took 38 us of host time: 14 us for the
// launches themselves, the rest in Python checks, seven torch.empty of 1.3 us and ctypes calls of up to 21 arguments.
//
// Each function handles the plain case - exact torch.Tensor arguments that satisfy every check of its counterpart in
// binding.py, outputs not given - and returns None for anything else before it has done anything; the caller then goes on
// in Python, where every error is raised.  Tensors are allocated in the same order, by the same operators, and the library is
// reached through the addresses of the C functions that binding.py loaded.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/python_headers.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/VirtualGuardImpl.h>

#include <algorithm>

#include "varlen_attn.h"

namespace {

struct Library {
  decltype(&va_plan_bytes) plan_bytes;
  decltype(&va_segments_bind) segments_bind;
  decltype(&va_pack_to_cu_seqlens) pack;
  decltype(&va_attn_workspace_bytes) workspace_bytes;
  decltype(&va_varlen_attn_fwd) fwd;
  decltype(&va_varlen_attn_bwd) bwd;
  decltype(&va_cache_write) cache_write;
  decltype(&va_cache_read) cache_read;
  decltype(&va_paged_attn_workspace_bytes) paged_workspace_bytes;
  decltype(&va_paged_attn_fwd) paged;
};
Library lib = {};

// Other Python threads run while a tensor is allocated (which can wait for the GPU) and kernels are launched (which can wait
// for room in their queue), as they do around torch's own allocations and around ctypes calls.  A 16-token pass takes 23.0 us
// with it and without.
struct WithoutGil {
  PyThreadState *state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};

template <class F> void set_address(F &f, PyObject *address) { f = (F)PyLong_AsVoidPtr(address); }

// The tensor behind `x`, or nullptr where it is no plain one that lives contiguously on the GPU, or where a mode asks to see
// the Python calls that create tensors.
const at::Tensor *plain(PyObject *x) {
  if (!THPVariable_CheckExact(x) || at::impl::torch_function_mode_enabled()) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(x);
  return t.layout() == at::kStrided && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

int element_type(at::ScalarType t) {
  return t == at::kFloat ? VA_F32 : t == at::kBFloat16 ? VA_BF16 : t == at::kHalf ? VA_F16 : -1;
}

struct Sizes {
  int64_t n, hq, hkv, d;
};
// Q [N, Hq, d], K and V [N, Hkv, d] of one element type the library has, for a stream of rows * T tokens
bool sizes(const at::Tensor *q, const at::Tensor *k, const at::Tensor *v, int64_t tokens, Sizes &s) {
  if (!q || !k || !v || q->dim() != 3 || k->dim() != 3 || v->sizes() != k->sizes()) return false;
  s = {q->size(0), q->size(1), k->size(1), q->size(2)};
  return k->size(0) == s.n && k->size(2) == s.d && s.n == tokens && q->scalar_type() == k->scalar_type() &&
         q->scalar_type() == v->scalar_type() && element_type(q->scalar_type()) >= 0;
}

// connect(plan_bytes, segments_bind, pack, workspace_bytes, fwd, bwd): addresses of the library's functions
PyObject *connect(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "connect takes 6 addresses");
  set_address(lib.plan_bytes, a[0]);
  set_address(lib.segments_bind, a[1]);
  set_address(lib.pack, a[2]);
  set_address(lib.workspace_bytes, a[3]);
  set_address(lib.fwd, a[4]);
  set_address(lib.bwd, a[5]);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// pack(position_ids, address of a va_segments, stream) -> (rows, tokens_per_row, plan) | status | None
PyObject *pack(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *pos = n == 3 ? plain(a[0]) : nullptr;
  if (!pos || pos->dim() != 2 || (pos->scalar_type() != at::kLong && pos->scalar_type() != at::kInt)) Py_RETURN_NONE;
  const int64_t rows = pos->size(0), T = pos->size(1);
  if (rows <= 0 || T <= 0 || rows >= INT32_MAX || T >= INT32_MAX) Py_RETURN_NONE;
  va_segments *seg = (va_segments *)PyLong_AsVoidPtr(a[1]);
  void *stream = PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return nullptr;
  const size_t bytes = lib.plan_bytes((int32_t)rows, (int32_t)T);
  if (bytes == 0) Py_RETURN_NONE;
  at::Tensor plan;
  va_status bound, s = VA_OK;
  {
    WithoutGil free;
    plan = at::empty({(int64_t)(bytes / 4)}, pos->options().dtype(at::kInt));
    bound = lib.segments_bind(plan.data_ptr(), bytes, (int32_t)rows, (int32_t)T, seg);
    if (bound == VA_OK)
      s = lib.pack(pos->data_ptr(), pos->scalar_type() == at::kLong ? VA_I64 : VA_I32, (int32_t)rows, (int32_t)T, seg, stream);
  }
  if (bound != VA_OK) Py_RETURN_NONE;
  if (s != VA_OK) return PyLong_FromLong(s);
  return Py_BuildValue("LLN", (long long)rows, (long long)T, THPVariable_Wrap(std::move(plan)));
  END_HANDLE_TH_ERRORS
}

// fwd(q, k, v, address of the va_segments, rows, tokens_per_row, softmax_scale, stream) -> (o, lse) | status | None
PyObject *fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) Py_RETURN_NONE;
  const va_segments *seg = (const va_segments *)PyLong_AsVoidPtr(a[3]);
  const int64_t rows = PyLong_AsLongLong(a[4]), T = PyLong_AsLongLong(a[5]);
  const float scale = (float)PyFloat_AsDouble(a[6]);
  void *stream = PyLong_AsVoidPtr(a[7]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *q = plain(a[0]), *k = plain(a[1]), *v = plain(a[2]);
  Sizes s;
  if (!sizes(q, k, v, rows * T, s)) Py_RETURN_NONE;
  at::Tensor o, lse;
  va_status status;
  {
    WithoutGil free;
    o = at::empty_like(*q), lse = at::empty({s.hq, s.n}, q->options().dtype(at::kFloat));
    status = lib.fwd(q->data_ptr(), k->data_ptr(), v->data_ptr(), o.data_ptr(), (float *)lse.data_ptr(), seg, (int32_t)rows,
                     (int32_t)T, (int32_t)s.hq, (int32_t)s.hkv, (int32_t)s.d, (va_dtype)element_type(q->scalar_type()), scale, nullptr,
                     0, stream);
  }
  if (status != VA_OK) return PyLong_FromLong(status);
  return Py_BuildValue("NN", THPVariable_Wrap(std::move(o)), THPVariable_Wrap(std::move(lse)));
  END_HANDLE_TH_ERRORS
}

// bwd(do, q, k, v, o, lse, address of the va_segments, rows, tokens_per_row, softmax_scale, gradients in float32, stream)
// -> (dq, dk, dv) | status | None.  Gradients in float32, or else in the inputs' type.
PyObject *bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 12) Py_RETURN_NONE;
  const va_segments *seg = (const va_segments *)PyLong_AsVoidPtr(a[6]);
  const int64_t rows = PyLong_AsLongLong(a[7]), T = PyLong_AsLongLong(a[8]);
  const float scale = (float)PyFloat_AsDouble(a[9]);
  const bool f32_grads = a[10] == Py_True;
  void *stream = PyLong_AsVoidPtr(a[11]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *g = plain(a[0]), *q = plain(a[1]), *k = plain(a[2]), *v = plain(a[3]), *o = plain(a[4]), *lse = plain(a[5]);
  Sizes s;
  if (!g || !o || !lse || !sizes(q, k, v, rows * T, s) || g->scalar_type() != q->scalar_type() || o->scalar_type() != q->scalar_type() ||
      lse->scalar_type() != at::kFloat || lse->sizes() != at::IntArrayRef({s.hq, s.n}) || g->numel() < q->numel() || o->numel() < q->numel())
    Py_RETURN_NONE;
  const at::TensorOptions like = q->options(), grads = f32_grads ? like.dtype(at::kFloat) : like;
  at::Tensor dq, dk, dv;
  va_status status;
  {
    WithoutGil free;
    dq = at::empty(q->sizes(), grads), dk = at::empty(k->sizes(), grads), dv = at::empty(v->sizes(), grads);
    const size_t bytes = lib.workspace_bytes((int32_t)s.n, (int32_t)s.hq, (int32_t)s.hkv, (int32_t)s.d, 1);
    const int64_t floats = (int64_t)(std::max<size_t>(bytes, 4) / 4);
    at::Tensor ws = at::empty({floats}, like.dtype(at::kFloat));
    status = lib.bwd(g->data_ptr(), q->data_ptr(), k->data_ptr(), v->data_ptr(), o->data_ptr(), (const float *)lse->data_ptr(),
                     dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), f32_grads ? VA_F32 : (va_dtype)element_type(q->scalar_type()), seg,
                     (int32_t)rows, (int32_t)T, (int32_t)s.hq, (int32_t)s.hkv, (int32_t)s.d, (va_dtype)element_type(q->scalar_type()),
                     scale, ws.data_ptr(), (size_t)floats * 4, stream);
  }
  if (status != VA_OK) return PyLong_FromLong(status);
  return Py_BuildValue("NNN", THPVariable_Wrap(std::move(dq)), THPVariable_Wrap(std::move(dk)), THPVariable_Wrap(std::move(dv)));
  END_HANDLE_TH_ERRORS
}

// connect_cache(cache_write, cache_read, paged_workspace_bytes, paged): addresses of the library's functions
PyObject *connect_cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "connect_cache takes 4 addresses");
  set_address(lib.cache_write, a[0]);
  set_address(lib.cache_read, a[1]);
  set_address(lib.paged_workspace_bytes, a[2]);
  set_address(lib.paged, a[3]);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

int64_t current_device() { return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index(); }

// A cache (tuple of k, v and their scales or None) and a page table, for rows of type `rows`, all on `device`: the library's view
// of them, or false where they are not what binding.py asks for.
bool cache_view(PyObject *cache, PyObject *page_table, at::ScalarType rows, int64_t device, va_kv_cache &c) {
  if (!PyTuple_Check(cache) || PyTuple_GET_SIZE(cache) != 4) return false;
  const at::Tensor *k = plain(PyTuple_GET_ITEM(cache, 0)), *v = plain(PyTuple_GET_ITEM(cache, 1));
  if (!k || !v || k->dim() != 4 || v->sizes() != k->sizes() || v->scalar_type() != k->scalar_type()) return false;
  if (k->get_device() != device || v->get_device() != device) return false;
  const at::ScalarType t = k->scalar_type();
  c.format = t == at::kChar ? VA_CACHE_I8 : t == at::kFloat8_e4m3fn ? VA_CACHE_E4M3 : VA_CACHE_PLAIN;
  if (c.format == VA_CACHE_PLAIN && (t != rows || element_type(t) < 0)) return false;
  c.k_scale = c.v_scale = nullptr;
  if (c.format != VA_CACHE_PLAIN) {
    float **to[2] = {&c.k_scale, &c.v_scale};
    for (int i = 0; i < 2; ++i) {
      const at::Tensor *s = plain(PyTuple_GET_ITEM(cache, 2 + i));
      if (!s || s->scalar_type() != at::kFloat || s->sizes() != k->sizes().slice(0, 3) || s->get_device() != device) return false;
      *to[i] = (float *)s->data_ptr();
    }
  }
  if (!THPVariable_CheckExact(page_table)) return false;
  const at::Tensor &table = THPVariable_Unpack(page_table);
  if (table.layout() != at::kStrided || !table.is_cuda() || table.dim() != 2 || table.scalar_type() != at::kInt || table.get_device() != device)
    return false;
  const int64_t seqs = table.size(0), width = table.size(1), stride = seqs > 1 ? table.stride(0) : width;
  if ((width > 1 && table.stride(1) != 1) || stride < width) return false;
  if (k->size(0) > INT32_MAX || k->size(1) > INT32_MAX || k->size(2) > INT32_MAX || k->size(3) > INT32_MAX || seqs > INT32_MAX || width > INT32_MAX)
    return false;
  c.k = k->data_ptr(), c.v = v->data_ptr();
  c.n_pages = (int32_t)k->size(0), c.hkv = (int32_t)k->size(1), c.page_size = (int32_t)k->size(2), c.d = (int32_t)k->size(3);
  c.n_seqs = (int32_t)seqs, c.max_pages = (int32_t)width, c.table_stride = stride;
  c.page_table = (const int32_t *)table.data_ptr();
  return true;
}

// Position ids and sequence ids (or None) of `tokens` tokens
bool token_ids(PyObject *position_ids, PyObject *seq_ids, int64_t tokens, int64_t device, const at::Tensor *&pos, const at::Tensor *&seq) {
  pos = plain(position_ids);
  if (!pos || pos->numel() != tokens || (pos->scalar_type() != at::kLong && pos->scalar_type() != at::kInt) || pos->get_device() != device) return false;
  seq = nullptr;
  if (seq_ids == Py_None) return true;
  seq = plain(seq_ids);
  return seq && seq->numel() == tokens && seq->scalar_type() == at::kInt && seq->get_device() == device;
}

// cache_write(k, v, cache, page_table, position_ids, seq_ids or None, stream) -> status | None
PyObject *cache_write(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) Py_RETURN_NONE;
  void *stream = PyLong_AsVoidPtr(a[6]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *k = plain(a[0]), *v = plain(a[1]), *pos, *seq;
  if (!k || !v) Py_RETURN_NONE;
  const int64_t device = current_device();
  va_kv_cache c;
  if ( k->dim() != 3 || v->sizes() != k->sizes() || v->scalar_type() != k->scalar_type() || element_type(k->scalar_type()) < 0 ||
      k->get_device() != device || v->get_device() != device || !cache_view(a[2], a[3], k->scalar_type(), device, c) ||
      k->size(1) != c.hkv || k->size(2) != c.d || k->size(0) > INT32_MAX || !token_ids(a[4], a[5], k->size(0), device, pos, seq))
    Py_RETURN_NONE;
  va_status status;
  {
    WithoutGil free;
    status = lib.cache_write(k->data_ptr(), v->data_ptr(), (va_dtype)element_type(k->scalar_type()), &c,
                             seq ? (const int32_t *)seq->data_ptr() : nullptr, pos->data_ptr(),
                             pos->scalar_type() == at::kLong ? VA_I64 : VA_I32, (int32_t)k->size(0), stream);
  }
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}

// cache_read(cache, page_table, position_ids, seq_ids or None, type of the rows, stream) -> (k, v) | status | None.  The rows
// have the pages' type; out of an 8-bit cache VA_F32, VA_BF16 or VA_F16 as told.
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6) Py_RETURN_NONE;
  const int64_t type = PyLong_AsLongLong(a[4]);
  void *stream = PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  const at::ScalarType rows = type == VA_F32 ? at::kFloat : type == VA_BF16 ? at::kBFloat16 : at::kHalf;
  const at::Tensor *pos = plain(a[2]), *seq;
  if (!pos) Py_RETURN_NONE;
  const int64_t device = current_device();
  va_kv_cache c;
  if (pos->numel() > INT32_MAX || !cache_view(a[0], a[1], rows, device, c) || !token_ids(a[2], a[3], pos->numel(), device, pos, seq))
    Py_RETURN_NONE;
  at::Tensor k, v;
  va_status status;
  {
    WithoutGil free;
    const at::TensorOptions like = pos->options().dtype(rows);
    k = at::empty({pos->numel(), c.hkv, c.d}, like), v = at::empty({pos->numel(), c.hkv, c.d}, like);
    status = lib.cache_read(k.data_ptr(), v.data_ptr(), (va_dtype)element_type(rows), &c, seq ? (const int32_t *)seq->data_ptr() : nullptr,
                            pos->data_ptr(), pos->scalar_type() == at::kLong ? VA_I64 : VA_I32, (int32_t)pos->numel(), stream);
  }
  if (status != VA_OK) return PyLong_FromLong(status);
  return Py_BuildValue("NN", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
  END_HANDLE_TH_ERRORS
}

// paged(q, cache, page_table, context_lens, softmax_scale, stream) -> (o, lse) | status | None
PyObject *paged(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AsDouble(a[4]);
  void *stream = PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *q = plain(a[0]), *lens = plain(a[3]);
  if (!q || !lens) Py_RETURN_NONE;
  const int64_t device = current_device();
  va_kv_cache c;
  if (q->dim() != 3 || lens->dim() != 1 || element_type(q->scalar_type()) < 0 || lens->scalar_type() != at::kInt ||
      q->get_device() != device || lens->get_device() != device || !cache_view(a[1], a[2], q->scalar_type(), device, c) ||
      q->size(0) != c.n_seqs || lens->size(0) != c.n_seqs || q->size(2) != c.d || c.hkv <= 0 || q->size(1) % c.hkv != 0 || q->size(1) > INT32_MAX)
    Py_RETURN_NONE;
  at::Tensor o, lse, ws;
  va_status status;
  {
    WithoutGil free;
    const int32_t hq = (int32_t)q->size(1);
    o = at::empty_like(*q), lse = at::empty({q->size(1), q->size(0)}, q->options().dtype(at::kFloat));
    const size_t bytes = lib.paged_workspace_bytes(c.n_seqs, c.max_pages, c.page_size, hq, c.hkv, c.d);
    if (bytes > 0) ws = at::empty({(int64_t)(bytes / 4)}, q->options().dtype(at::kFloat));
    status = lib.paged(q->data_ptr(), o.data_ptr(), (float *)lse.data_ptr(), (va_dtype)element_type(q->scalar_type()), &c, hq,
                       (const int32_t *)lens->data_ptr(), scale, bytes > 0 ? ws.data_ptr() : nullptr, bytes, stream);
  }
  if (status != VA_OK) return PyLong_FromLong(status);
  return Py_BuildValue("NN", THPVariable_Wrap(std::move(o)), THPVariable_Wrap(std::move(lse)));
  END_HANDLE_TH_ERRORS
}

#define VA_METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {VA_METHOD(connect), VA_METHOD(pack), VA_METHOD(fwd), VA_METHOD(bwd), VA_METHOD(connect_cache), VA_METHOD(cache_write),
                         VA_METHOD(cache_read), VA_METHOD(paged), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_va_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__va_native() {
  PyObject *m = PyModule_Create(&module);
  // the torch whose headers this was compiled with: objects of another one may lie differently in memory
  if (m && PyModule_AddStringConstant(m, "torch_version", VA_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
