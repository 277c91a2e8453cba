// Native argument marshalling between torch tensors and the C ABI (mea.h): the
// ordinary case of attention.py's calls -- plain GPU tensors whose layout the
// kernels read in place -- as one call each.  Every function returns None for
// anything else, and for what the library refuses, before anything is launched;
// attention.py then takes its general path, which copies or raises.  A launch
// that fails is raised here, and not tried again.
//
// Why it exists: a training step on a small problem is bound by the host.
// Autograd runs the backward on a thread of its own, and each hand-over leaves
// the interpreter's working set cold, so the marshalling in Python, 52 us in a
// loop on one thread, took 178 us of every 1x1x256x256 forward + backward.
// The functions are found by address (init), so this module links to torch
// only and uses the library that _lib.load() loaded; errors are raised by
// _lib.check.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <memory>
#include <optional>
#include <vector>

#include "../../include/mea.h"

namespace {

decltype(&mea_attention_fwd_workspace_size) g_fwd_ws;
decltype(&mea_attention_bwd_workspace_size) g_bwd_ws;
decltype(&mea_attention_fwd) g_fwd;
decltype(&mea_attention_bwd) g_bwd;
decltype(&mea_scored_attention_fwd_workspace_size) g_scored_fwd_ws;
decltype(&mea_scored_attention_bwd_workspace_size) g_scored_bwd_ws;
decltype(&mea_scored_attention_fwd) g_scored_fwd;
decltype(&mea_scored_attention_bwd) g_scored_bwd;
decltype(&mea_prefix_attention_fwd_workspace_size) g_prefix_ws;
decltype(&mea_prefix_attention_fwd) g_prefix_fwd;
PyObject* g_check;  // check(name, status): raises what a status means

// A plain torch.Tensor or Parameter with storage on a GPU (no subclass, no
// functorch wrapper), or null.
const at::Tensor* gpu_tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.device().is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}

int dtype_code(at::ScalarType t) {
  return t == at::kFloat ? MEA_F32 : t == at::kHalf ? MEA_F16 : t == at::kBFloat16 ? MEA_BF16 : -1;
}

// Whether the kernels can read or write t ([B, H, n, features]) in place.
bool in_place(const at::Tensor& t) {
  if (t.dim() != 4 || t.stride(3) != 1 || reinterpret_cast<uintptr_t>(t.const_data_ptr()) % 16) return false;
  const int64_t unit = 16 / t.element_size();
  return t.stride(0) % unit == 0 && t.stride(1) % unit == 0 && t.stride(2) % unit == 0;
}

bool like(const at::Tensor& t, const at::Tensor& ref, at::ScalarType dtype) {
  return t.device() == ref.device() && t.scalar_type() == dtype && in_place(t);
}

mea_tensor_strides strides_of(const at::Tensor& t) { return {t.stride(0), t.stride(1), t.stride(2)}; }

// None, or an int32 [B] vector on q's device: its address in *out.
bool kv_len_ok(PyObject* o, const at::Device& dev, int64_t B, const int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = gpu_tensor(o);
  if (!t || t->scalar_type() != at::kInt || t->device() != dev || t->dim() != 1 || t->size(0) != B ||
      !t->is_contiguous())
    return false;
  *out = static_cast<const int32_t*>(t->const_data_ptr());
  return true;
}

// Sizes, dtype, mask, scale and padding of a call; false: not the ordinary case.
bool problem(mea_problem* p, int64_t B, int64_t H, int64_t n_q, int64_t n_k, int64_t d, int64_t d_v, int dtype,
             PyObject* causal, PyObject* scale, PyObject* kv_len, const at::Device& dev, bool out_f32) {
  *p = mea_problem{};
  p->batch = B;
  p->heads = H;
  p->n_q = n_q;
  p->n_k = n_k;
  p->d = d;
  p->d_v = d_v == d ? 0 : d_v;
  p->dtype = dtype;
  const int c = PyObject_IsTrue(causal);
  p->causal = c;
  double s = d > 0 ? 1.0 / std::sqrt((double)d) : 0.0;
  if (scale != Py_None && c >= 0) s = PyFloat_AsDouble(scale);
  if (c < 0 || PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  p->scale = (float)s;
  p->out_f32 = out_f32 && dtype != MEA_F32;
  return kv_len_ok(kv_len, dev, B, &p->kv_len);
}

// Same-shape checks of [B, H, n_q, d], [B, H, n_k, d], [B, H, n_k, d_v].
bool qkv_shapes(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v) {
  return q.size(0) == k.size(0) && q.size(1) == k.size(1) && q.size(3) == k.size(3) && k.size(0) == v.size(0) &&
         k.size(1) == v.size(1) && k.size(2) == v.size(2);
}

hipStream_t stream_of(const at::Device& dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

at::Tensor workspace(size_t bytes, const at::Device& dev) {
  return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(dev));
}

PyObject* none() { Py_RETURN_NONE; }

// The result of a call whose status is not MEA_OK: None where the library
// refused the arguments (it launches nothing then), else the error.
PyObject* failed(const char* name, mea_status st) {
  if (st == MEA_ERR_INVALID_ARG || st == MEA_ERR_UNSUPPORTED) return none();
  return PyObject_CallFunction(g_check, "si", name, (int)st);
}

// A new tuple of tensors; undefined ones are None.
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// Allocates lse, o_lo and the workspace, and launches the forward (without the
// interpreter lock).  Returns the status.
mea_status launch_fwd(const mea_problem& p, const at::Tensor& q, const void* k, const void* v, void* o,
                      at::Tensor* lse, at::Tensor* o_lo, at::IntArrayRef lse_shape, at::IntArrayRef o_shape,
                      at::ScalarType out_dtype) {
  size_t bytes = 0;
  mea_status st = g_fwd_ws(&p, &bytes);
  if (st != MEA_OK) return st;
  const at::Device dev = q.device();
  if (lse) *lse = at::empty(lse_shape, at::TensorOptions().dtype(at::kFloat).device(dev));
  if (o_lo) *o_lo = at::empty(o_shape, at::TensorOptions().dtype(out_dtype).device(dev));
  at::Tensor ws;
  if (bytes) ws = workspace(bytes, dev);
  return g_fwd(&p, q.const_data_ptr(), k, v, o, lse ? static_cast<float*>(lse->mutable_data_ptr()) : nullptr,
               o_lo ? o_lo->mutable_data_ptr() : nullptr, bytes ? ws.mutable_data_ptr() : nullptr, bytes,
               stream_of(dev));
}

// fwd(q, k, v, causal, scale, need_lse, out, out_dtype, kv_len, residual):
// attention_fwd's result, or None.
PyObject* ext_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]);
  if (!q || !k || !v) return none();
  const at::ScalarType dt = q->scalar_type();
  if (dtype_code(dt) < 0 || !in_place(*q) || !like(*k, *q, dt) || !like(*v, *q, dt) || !qkv_shapes(*q, *k, *v))
    return none();
  at::ScalarType out_dt = dt;
  if (a[7] != Py_None) {
    if (!THPDtype_Check(a[7])) return none();
    out_dt = reinterpret_cast<THPDtype*>(a[7])->scalar_type;
    if (out_dt != dt && out_dt != at::kFloat) return none();
  }
  const int64_t shape[4] = {q->size(0), q->size(1), q->size(2), v->size(3)};
  const at::Tensor* out = nullptr;
  if (a[6] != Py_None) {
    out = gpu_tensor(a[6]);
    if (!out || !like(*out, *q, out_dt) || out->sizes() != at::IntArrayRef(shape, 4)) return none();
  }
  const int need_lse = PyObject_IsTrue(a[5]), residual = PyObject_IsTrue(a[9]);
  mea_problem p;
  if (need_lse < 0 || residual < 0 ||
      !problem(&p, shape[0], shape[1], shape[2], k->size(2), q->size(3), shape[3], dtype_code(dt), a[3], a[4], a[8],
               q->device(), out_dt == at::kFloat)) {
    PyErr_Clear();
    return none();
  }
  at::Tensor o, lse, o_lo;
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    o = out ? *out : at::empty(at::IntArrayRef(shape, 4), at::TensorOptions().dtype(out_dt).device(q->device()));
    mea_strides ms = {};
    if (!q->is_contiguous() || !k->is_contiguous() || !v->is_contiguous() || !o.is_contiguous()) {
      ms.q = strides_of(*q);
      ms.k = strides_of(*k);
      ms.v = strides_of(*v);
      ms.o = strides_of(o);
      p.strides = &ms;
    }
    st = launch_fwd(p, *q, k->const_data_ptr(), v->const_data_ptr(), o.mutable_data_ptr(), need_lse ? &lse : nullptr,
                    residual && out_dt != at::kFloat ? &o_lo : nullptr, at::IntArrayRef(shape, 3),
                    at::IntArrayRef(shape, 4), out_dt);
  }
  if (st != MEA_OK) return failed("mea_attention_fwd", st);
  return residual ? tuple_of({o, lse, o_lo}) : tuple_of({o, lse});
  END_HANDLE_TH_ERRORS
}

mea_status launch_bwd(const mea_problem& p, const at::Tensor& q, const void* k, const void* v, const void* o,
                      const void* o_lo, const void* d_o, const at::Tensor& lse, void* dq, void* dk, void* dv) {
  size_t bytes = 0;
  const mea_status st = g_bwd_ws(&p, &bytes);
  if (st != MEA_OK) return st;
  at::Tensor ws = workspace(bytes, q.device());
  return g_bwd(&p, q.const_data_ptr(), k, v, o, o_lo, d_o, static_cast<const float*>(lse.const_data_ptr()), dq, dk, dv,
               ws.mutable_data_ptr(), bytes, stream_of(q.device()));
}

// The log-sum-exp of n_q rows per (batch, head).
bool lse_ok(const at::Tensor* t, const at::Device& dev, int64_t B, int64_t H, int64_t n_q) {
  return t && t->device() == dev && t->scalar_type() == at::kFloat && t->is_contiguous() && t->dim() == 3 &&
         t->size(0) == B && t->size(1) == H && t->size(2) == n_q;
}

// bwd(q, k, v, o, lse, do, causal, scale, need_dq, need_dkdv, out, kv_len,
// o_lo): attention_bwd's result, or None.
PyObject* ext_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 13) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]), *o = gpu_tensor(a[3]),
                   *lse = gpu_tensor(a[4]), *d_o = gpu_tensor(a[5]);
  if (!q || !k || !v || !o || !lse || !d_o) return none();
  const at::ScalarType dt = q->scalar_type(), out_dt = o->scalar_type();
  if (dtype_code(dt) < 0 || (out_dt != dt && out_dt != at::kFloat) || !in_place(*q) || !like(*k, *q, dt) ||
      !like(*v, *q, dt) || !like(*o, *q, out_dt) || !like(*d_o, *q, out_dt) || !qkv_shapes(*q, *k, *v) ||
      !lse_ok(lse, q->device(), q->size(0), q->size(1), q->size(2)))
    return none();
  const int64_t shape[4] = {q->size(0), q->size(1), q->size(2), v->size(3)};
  const at::IntArrayRef o_shape(shape, 4);
  if (o->sizes() != o_shape || d_o->sizes() != o_shape) return none();
  const at::Tensor* o_lo = nullptr;
  if (a[12] != Py_None) {
    o_lo = gpu_tensor(a[12]);
    if (!o_lo || !like(*o_lo, *q, out_dt) || o_lo->sizes() != o_shape || !o_lo->is_contiguous()) return none();
  }
  const int need[2] = {PyObject_IsTrue(a[8]), PyObject_IsTrue(a[9])};
  // The gradients: given ones are checked, the others allocated.
  const at::Tensor* src[3] = {q, k, v};
  const at::Tensor* given[3] = {nullptr, nullptr, nullptr};
  if (a[10] != Py_None) {
    if (!PyTuple_CheckExact(a[10]) || PyTuple_GET_SIZE(a[10]) != 3) return none();
    for (int i = 0; i < 3; ++i) {
      PyObject* g = PyTuple_GET_ITEM(a[10], i);
      if (g == Py_None || need[i > 0] <= 0) continue;
      given[i] = gpu_tensor(g);
      if (!given[i] || !like(*given[i], *q, dt) || given[i]->sizes() != src[i]->sizes()) return none();
    }
  }
  mea_problem p;
  if (need[0] < 0 || need[1] < 0 || !(need[0] || need[1]) ||
      !problem(&p, shape[0], shape[1], shape[2], k->size(2), q->size(3), shape[3], dtype_code(dt), a[6], a[7], a[11],
               q->device(), out_dt == at::kFloat)) {
    PyErr_Clear();
    return none();
  }
  at::Tensor g[3];
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    bool contiguous = q->is_contiguous() && k->is_contiguous() && v->is_contiguous() && o->is_contiguous() &&
                      d_o->is_contiguous();
    for (int i = 0; i < 3; ++i) {
      if (!need[i > 0]) continue;
      g[i] = given[i] ? *given[i]
                      : at::empty(src[i]->sizes(), at::TensorOptions().dtype(dt).device(q->device()));
      contiguous = contiguous && g[i].is_contiguous();
    }
    mea_strides ms = {};
    if (!contiguous) {
      mea_tensor_strides* gs[3] = {&ms.dq, &ms.dk, &ms.dv};
      ms.q = strides_of(*q);
      ms.k = strides_of(*k);
      ms.v = strides_of(*v);
      ms.o = strides_of(*o);
      ms.d_o = strides_of(*d_o);
      for (int i = 0; i < 3; ++i)
        if (g[i].defined()) *gs[i] = strides_of(g[i]);
      p.strides = &ms;
    }
    auto ptr = [](at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; };
    st = launch_bwd(p, *q, k->const_data_ptr(), v->const_data_ptr(), o->const_data_ptr(),
                    o_lo ? o_lo->const_data_ptr() : nullptr, d_o->const_data_ptr(), *lse, ptr(g[0]), ptr(g[1]),
                    ptr(g[2]));
  }
  if (st != MEA_OK) return failed("mea_attention_bwd", st);
  return tuple_of({g[0], g[1], g[2]});
  END_HANDLE_TH_ERRORS
}

// A contiguous packed projection [B, n, 3, H, d], or null.
const at::Tensor* packed_qkv(PyObject* o) {
  const at::Tensor* t = gpu_tensor(o);
  return t && t->dim() == 5 && t->size(2) == 3 && t->is_contiguous() && dtype_code(t->scalar_type()) >= 0 &&
                 t->size(4) % 16 == 0 && reinterpret_cast<uintptr_t>(t->const_data_ptr()) % 16 == 0
             ? t
             : nullptr;
}

// Address of q (0), k (1) or v (2) inside a packed projection.
char* packed_part(const at::Tensor& t, int i) {
  return static_cast<char*>(const_cast<void*>(t.const_data_ptr())) + i * t.size(3) * t.size(4) * t.element_size();
}

// packed_fwd(qkv, causal, scale, kv_len): (o [B, n, H, d], lse, o_lo), or None.
PyObject* ext_packed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor* t = n_args == 4 ? packed_qkv(a[0]) : nullptr;
  if (!t) return none();
  const int64_t B = t->size(0), n = t->size(1), H = t->size(3), d = t->size(4);
  const at::ScalarType dt = t->scalar_type();
  mea_problem p;
  if (!problem(&p, B, H, n, n, d, d, dtype_code(dt), a[1], a[2], a[3], t->device(), false)) return none();
  mea_strides ms = {};
  ms.q = ms.k = ms.v = mea_tensor_strides{n * 3 * H * d, d, 3 * H * d};
  ms.o = mea_tensor_strides{n * H * d, d, H * d};
  p.strides = &ms;
  at::Tensor o, lse, o_lo;
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    o = at::empty({B, n, H, d}, at::TensorOptions().dtype(dt).device(t->device()));
    st = launch_fwd(p, *t, packed_part(*t, 1), packed_part(*t, 2), o.mutable_data_ptr(), &lse,
                    dt != at::kFloat ? &o_lo : nullptr, {B, H, n}, {B, H, n, d}, dt);
  }
  if (st != MEA_OK) return failed("mea_attention_fwd", st);
  return tuple_of({o, lse, o_lo});
  END_HANDLE_TH_ERRORS
}

// packed_bwd(qkv, o, lse, o_lo, do, causal, scale, kv_len): the packed
// gradient, or None.  o and do are [B, n, H, d].
PyObject* ext_packed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor* t = n_args == 8 ? packed_qkv(a[0]) : nullptr;
  if (!t) return none();
  const at::Tensor *o = gpu_tensor(a[1]), *lse = gpu_tensor(a[2]), *d_o = gpu_tensor(a[4]);
  if (!o || !lse || !d_o) return none();
  const int64_t B = t->size(0), n = t->size(1), H = t->size(3), d = t->size(4);
  const at::ScalarType dt = t->scalar_type();
  const int64_t shape[4] = {B, n, H, d};
  const at::IntArrayRef o_shape(shape, 4);
  if (!like(*o, *t, dt) || !like(*d_o, *t, dt) || o->sizes() != o_shape || d_o->sizes() != o_shape ||
      !lse_ok(lse, t->device(), B, H, n))
    return none();
  const at::Tensor* o_lo = nullptr;
  if (a[3] != Py_None) {
    o_lo = gpu_tensor(a[3]);
    if (!o_lo || !like(*o_lo, *t, dt) || !o_lo->is_contiguous() || o_lo->numel() != o->numel()) return none();
  }
  mea_problem p;
  if (!problem(&p, B, H, n, n, d, d, dtype_code(dt), a[5], a[6], a[7], t->device(), false)) return none();
  auto bnh = [](const at::Tensor& x) { return mea_tensor_strides{x.stride(0), x.stride(2), x.stride(1)}; };
  mea_strides ms = {};
  ms.q = ms.k = ms.v = ms.dq = ms.dk = ms.dv = mea_tensor_strides{n * 3 * H * d, d, 3 * H * d};
  ms.o = bnh(*o);
  ms.d_o = bnh(*d_o);
  p.strides = &ms;
  at::Tensor g;
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    g = at::empty_like(*t);
    st = launch_bwd(p, *t, packed_part(*t, 1), packed_part(*t, 2), o->const_data_ptr(),
                    o_lo ? o_lo->const_data_ptr() : nullptr, d_o->const_data_ptr(), *lse, packed_part(g, 0),
                    packed_part(g, 1), packed_part(g, 2));
  }
  if (st != MEA_OK) return failed("mea_attention_bwd", st);
  return THPVariable_Wrap(g);
  END_HANDLE_TH_ERRORS
}

// ---- attention with modified scores and over a shared prefix

// None, or a contiguous tensor of a type and shape on a device: its address in *out.
bool vector_ok(PyObject* o, const at::Device& dev, at::ScalarType type, at::IntArrayRef shape, const void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = gpu_tensor(o);
  if (!t || t->scalar_type() != type || t->device() != dev || t->sizes() != shape || !t->is_contiguous()) return false;
  *out = t->const_data_ptr();
  return true;
}

// Shapes of q, k, v with grouped key heads.
bool grouped_shapes(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v) {
  return q.size(0) == k.size(0) && q.size(3) == k.size(3) && k.sizes() == v.sizes() && k.size(1) > 0 &&
         q.size(1) % k.size(1) == 0;
}

// softcap, slopes, bias, edges (None, or (address, number, two-sided)), q_doc,
// k_doc, prefix_len, q_pos: a[0] .. a[7].  *bias: the bias or null.
bool score(mea_score* s, PyObject* const* a, const at::Tensor& q, const at::Tensor& k, const at::Tensor** bias) {
  *s = mea_score{};
  *bias = nullptr;
  const at::Device dev = q.device();
  const int64_t B = q.size(0), H = q.size(1);
  s->kv_heads = k.size(1);
  if (a[0] != Py_None) {
    const double cap = PyFloat_AsDouble(a[0]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      return false;
    }
    s->softcap = (float)cap;
    if (!(s->softcap > 0.0f)) return false;
  }
  const void* p;
  if (!vector_ok(a[1], dev, at::kFloat, {H}, &p)) return false;
  s->slopes = static_cast<const float*>(p);
  if (a[2] != Py_None) {
    const at::Tensor* t = gpu_tensor(a[2]);
    if (!t || !PyTuple_CheckExact(a[3]) || PyTuple_GET_SIZE(a[3]) != 3) return false;
    s->edges = static_cast<const int32_t*>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[3], 0)));
    s->n_edges = (int32_t)PyLong_AsLong(PyTuple_GET_ITEM(a[3], 1));
    s->two_sided = PyObject_IsTrue(PyTuple_GET_ITEM(a[3], 2));
    if (PyErr_Occurred()) {
      PyErr_Clear();
      return false;
    }
    if (t->device() != dev || (t->scalar_type() != at::kFloat && t->scalar_type() != q.scalar_type()) || t->dim() != 2 ||
        t->size(1) != H || t->size(0) != (int64_t)s->n_edges * (s->two_sided ? 2 : 1) || !t->is_contiguous())
      return false;
    s->table = t->const_data_ptr();
    s->table_dtype = dtype_code(t->scalar_type());
    *bias = t;
  }
  if (!vector_ok(a[4], dev, at::kInt, {B, q.size(2)}, &p)) return false;
  s->q_doc = static_cast<const int32_t*>(p);
  if (!vector_ok(a[5], dev, at::kInt, {B, k.size(2)}, &p)) return false;
  s->k_doc = static_cast<const int32_t*>(p);
  if (!vector_ok(a[6], dev, at::kInt, {B}, &p)) return false;
  s->prefix_len = static_cast<const int32_t*>(p);
  if (!vector_ok(a[7], dev, at::kInt, {B}, &p)) return false;
  s->q_pos = static_cast<const int32_t*>(p);
  return true;
}

// The forward into *o (allocated if undefined), *lse and *o_lo as wanted.
mea_status run_scored_fwd(mea_problem& p, const mea_score& s, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v,
                          bool need_lse, bool residual, at::Tensor* o, at::Tensor* lse, at::Tensor* o_lo) {
  const c10::DeviceGuard on(q.device());
  const auto opts = at::TensorOptions().dtype(q.scalar_type()).device(q.device());
  size_t bytes = 0;
  const mea_status st = g_scored_fwd_ws(&p, &s, &bytes);
  if (st != MEA_OK) return st;
  if (!o->defined()) *o = at::empty(q.sizes(), opts);
  mea_strides ms = {};
  p.strides = nullptr;
  if (!q.is_contiguous() || !k.is_contiguous() || !v.is_contiguous() || !o->is_contiguous()) {
    ms.q = strides_of(q);
    ms.k = strides_of(k);
    ms.v = strides_of(v);
    ms.o = strides_of(*o);
    p.strides = &ms;
  }
  if (need_lse) *lse = at::empty(q.sizes().slice(0, 3), opts.dtype(at::kFloat));
  if (residual && q.scalar_type() != at::kFloat) *o_lo = at::empty(q.sizes(), opts);
  at::Tensor ws;
  if (bytes) ws = workspace(bytes, q.device());
  return g_scored_fwd(&p, &s, q.const_data_ptr(), k.const_data_ptr(), v.const_data_ptr(), o->mutable_data_ptr(),
                      need_lse ? static_cast<float*>(lse->mutable_data_ptr()) : nullptr,
                      o_lo->defined() ? o_lo->mutable_data_ptr() : nullptr, bytes ? ws.mutable_data_ptr() : nullptr, bytes,
                      stream_of(q.device()));
}

// The backward into g: dq, dk, dv and the bias's gradient, need[] of (dq, dk and dv, the bias's).
mea_status run_scored_bwd(mea_problem& p, const mea_score& s, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v,
                          const at::Tensor& o, const at::Tensor& o_lo, const at::Tensor& lse, const at::Tensor& d_o,
                          const at::Tensor* bias, const int (&need)[3], at::Tensor (&g)[4]) {
  const c10::DeviceGuard on(q.device());
  const auto opts = at::TensorOptions().dtype(q.scalar_type()).device(q.device());
  size_t bytes = 0;
  mea_status st = g_scored_bwd_ws(&p, &s, &bytes);
  if (st != MEA_OK) return st;
  if (need[0] || need[2]) g[0] = at::empty(q.sizes(), opts);
  if (need[1]) {
    g[1] = at::empty(k.sizes(), opts);
    g[2] = at::empty(k.sizes(), opts);
  }
  if (need[2]) g[3] = at::empty(bias->sizes(), opts.dtype(bias->scalar_type()));
  mea_strides ms = {};
  p.strides = nullptr;
  if (!q.is_contiguous() || !k.is_contiguous() || !v.is_contiguous() || !o.is_contiguous() || !d_o.is_contiguous()) {
    ms.q = strides_of(q);
    ms.k = strides_of(k);
    ms.v = strides_of(v);
    ms.o = strides_of(o);
    ms.d_o = strides_of(d_o);
    if (g[0].defined()) ms.dq = strides_of(g[0]);
    if (g[1].defined()) ms.dk = ms.dv = strides_of(g[1]);
    p.strides = &ms;
  }
  at::Tensor ws = workspace(bytes, q.device());
  auto ptr = [](at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; };
  st = g_scored_bwd(&p, &s, q.const_data_ptr(), k.const_data_ptr(), v.const_data_ptr(), o.const_data_ptr(),
                    o_lo.defined() ? o_lo.const_data_ptr() : nullptr, d_o.const_data_ptr(),
                    static_cast<const float*>(lse.const_data_ptr()), ptr(g[0]), ptr(g[1]), ptr(g[2]), ptr(g[3]),
                    ws.mutable_data_ptr(), bytes, stream_of(q.device()));
  if (!need[0]) g[0] = at::Tensor();
  return st;
}

// scored_fwd(q, k, v, causal, scale, need_lse, out, kv_len, residual, <score>):
// attention_scored_fwd's result, or None.
PyObject* ext_scored_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 17) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]), *bias;
  if (!q || !k || !v) return none();
  const at::ScalarType dt = q->scalar_type();
  if (dtype_code(dt) < 0 || !in_place(*q) || !like(*k, *q, dt) || !like(*v, *q, dt) || !grouped_shapes(*q, *k, *v))
    return none();
  const at::Tensor* out = nullptr;
  if (a[6] != Py_None) {
    out = gpu_tensor(a[6]);
    if (!out || !like(*out, *q, dt) || out->sizes() != q->sizes()) return none();
  }
  const int need_lse = PyObject_IsTrue(a[5]), residual = PyObject_IsTrue(a[8]);
  mea_problem p;
  mea_score s;
  if (need_lse < 0 || residual < 0 ||
      !problem(&p, q->size(0), q->size(1), q->size(2), k->size(2), q->size(3), q->size(3), dtype_code(dt), a[3], a[4], a[7],
               q->device(), false) ||
      !score(&s, a + 9, *q, *k, &bias)) {
    PyErr_Clear();
    return none();
  }
  at::Tensor o, lse, o_lo;
  if (out) o = *out;
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    st = run_scored_fwd(p, s, *q, *k, *v, need_lse, residual, &o, &lse, &o_lo);
  }
  if (st != MEA_OK) return failed("mea_scored_attention_fwd", st);
  return residual ? tuple_of({o, lse, o_lo}) : tuple_of({o, lse});
  END_HANDLE_TH_ERRORS
}

// scored_bwd(q, k, v, o, lse, do, causal, scale, need_dq, need_dkdv, need_dbias,
// kv_len, o_lo, <score>): attention_scored_bwd's result, or None.
PyObject* ext_scored_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 21) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]), *o = gpu_tensor(a[3]),
                   *lse = gpu_tensor(a[4]), *d_o = gpu_tensor(a[5]), *bias;
  if (!q || !k || !v || !o || !lse || !d_o) return none();
  const at::ScalarType dt = q->scalar_type();
  if (dtype_code(dt) < 0 || !in_place(*q) || !like(*k, *q, dt) || !like(*v, *q, dt) || !like(*o, *q, dt) ||
      !like(*d_o, *q, dt) || !grouped_shapes(*q, *k, *v) || o->sizes() != q->sizes() || d_o->sizes() != q->sizes() ||
      !lse_ok(lse, q->device(), q->size(0), q->size(1), q->size(2)))
    return none();
  const at::Tensor* o_lo = nullptr;
  if (a[12] != Py_None) {
    o_lo = gpu_tensor(a[12]);
    if (!o_lo || !like(*o_lo, *q, dt) || o_lo->sizes() != q->sizes() || !o_lo->is_contiguous()) return none();
  }
  int need[3];
  for (int i = 0; i < 3; ++i)
    if ((need[i] = PyObject_IsTrue(a[8 + i])) < 0) {
      PyErr_Clear();
      return none();
    }
  mea_problem p;
  mea_score s;
  if (!problem(&p, q->size(0), q->size(1), q->size(2), k->size(2), q->size(3), q->size(3), dtype_code(dt), a[6], a[7], a[11],
               q->device(), false) ||
      !score(&s, a + 13, *q, *k, &bias)) {
    PyErr_Clear();
    return none();
  }
  if (!bias) need[2] = 0;
  if (!(need[0] || need[1] || need[2])) return none();
  at::Tensor g[4];
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    st = run_scored_bwd(p, s, *q, *k, *v, *o, o_lo ? *o_lo : at::Tensor(), *lse, *d_o, bias, need, g);
  }
  if (st != MEA_OK) return failed("mea_scored_attention_bwd", st);
  return tuple_of({g[0], g[1], g[2], g[3]});
  END_HANDLE_TH_ERRORS
}

// The differentiable call without Python in it: a backward that autograd's thread runs
// on its own (a training step on a small problem is bound by the host, and by the
// hand-over of the interpreter between the two threads).
struct Refused {
  mea_status st;
};
struct ScoredNode : public torch::autograd::Function<ScoredNode> {
  // extra: kv_len, slopes, q_doc, k_doc, prefix_len, q_pos, where given.
  static at::Tensor forward(torch::autograd::AutogradContext* ctx, at::Tensor q, at::Tensor k, at::Tensor v,
                            std::optional<at::Tensor> bias, mea_problem p, mea_score s, std::vector<at::Tensor> extra) {
    at::Tensor o, lse, o_lo;
    const mea_status st = run_scored_fwd(p, s, q, k, v, true, true, &o, &lse, &o_lo);
    if (st != MEA_OK) throw Refused{st};
    torch::autograd::variable_list saved = {q, k, v, bias ? *bias : at::Tensor(), o, lse, o_lo};
    for (const at::Tensor& t : extra) saved.push_back(t);
    ctx->save_for_backward(std::move(saved));
    ctx->saved_data["i"] = std::vector<int64_t>{p.causal, (int64_t)reinterpret_cast<uintptr_t>(s.edges), s.n_edges, s.two_sided};
    ctx->saved_data["f"] = std::vector<double>{p.scale, s.softcap};
    return o;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
    torch::autograd::variable_list none(7);
    if (!grads[0].defined()) return none;
    const auto t = ctx->get_saved_variables();
    const at::Tensor &q = t[0], &k = t[1], &v = t[2], &bias = t[3], &o = t[4], &lse = t[5], &o_lo = t[6];
    at::Tensor g[4];
    mea_status st;
    {
      const at::AutoGradMode no_grad(false);
      at::Tensor d_o = grads[0];
      if (d_o.scalar_type() != q.scalar_type()) d_o = d_o.to(q.scalar_type());
      if (!in_place(d_o)) d_o = d_o.contiguous();
      const auto i = ctx->saved_data["i"].toIntVector();
      const auto f = ctx->saved_data["f"].toDoubleVector();
      auto ptr = [&](int at) { return t[at].defined() ? t[at].const_data_ptr() : nullptr; };
      mea_problem p = {};
      p.batch = q.size(0);
      p.heads = q.size(1);
      p.n_q = q.size(2);
      p.n_k = k.size(2);
      p.d = q.size(3);
      p.dtype = dtype_code(q.scalar_type());
      p.causal = (int32_t)i[0];
      p.scale = (float)f[0];
      p.kv_len = static_cast<const int32_t*>(ptr(7));
      mea_score s = {};
      s.kv_heads = k.size(1);
      s.softcap = (float)f[1];
      s.edges = reinterpret_cast<const int32_t*>((uintptr_t)i[1]);
      s.n_edges = (int32_t)i[2];
      s.two_sided = (int32_t)i[3];
      if (bias.defined()) {
        s.table = bias.const_data_ptr();
        s.table_dtype = dtype_code(bias.scalar_type());
      }
      s.slopes = static_cast<const float*>(ptr(8));
      s.q_doc = static_cast<const int32_t*>(ptr(9));
      s.k_doc = static_cast<const int32_t*>(ptr(10));
      s.prefix_len = static_cast<const int32_t*>(ptr(11));
      s.q_pos = static_cast<const int32_t*>(ptr(12));
      const int need[3] = {ctx->needs_input_grad(0), ctx->needs_input_grad(1) || ctx->needs_input_grad(2),
                           bias.defined() && ctx->needs_input_grad(3)};
      if (!(need[0] || need[1] || need[2])) return none;
      st = run_scored_bwd(p, s, q, k, v, o, o_lo, lse, d_o, &bias, need, g);
    }
    if (st != MEA_OK) {
      pybind11::gil_scoped_acquire gil;
      Py_XDECREF(PyObject_CallFunction(g_check, "si", "mea_scored_attention_bwd", (int)st));
      python_error e;
      e.persist();
      throw e;
    }
    torch::autograd::variable_list r = {g[0], g[1], g[2], g[3]};
    if (at::GradMode::is_enabled()) {  // create_graph: the gradient cannot be differentiated again
      auto error = std::make_shared<torch::autograd::DelayedError>("scored attention cannot be differentiated twice", 4);
      r = (*error)(std::move(r));
    }
    r.resize(7);
    return r;
  }
};

// Whether the current stream is being captured into a graph while t is a leaf of a
// graph recorded on another stream that still lives: autograd would run the leaf's end of
// the captured backward on that stream, which ends the capture and often the process.
bool leaf_of_other_stream(const at::Tensor& t) {
  if (!t.requires_grad() || !t.is_leaf()) return false;
  const auto end = torch::autograd::impl::try_get_grad_accumulator(t);
  if (!end) return false;
  const auto stream = end->stream();
  return stream && *stream != c10::hip::getCurrentHIPStream(t.device().index()).unwrap();
}

// scored_apply(q, k, v, causal, scale, kv_len, <score>): o, with its gradient, or None.
PyObject* ext_scored_apply(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 14) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]), *bias;
  if (!q || !k || !v) return none();
  if (at::GradMode::is_enabled() && c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None)
    for (PyObject* o : {a[0], a[1], a[2], a[8]}) {
      const at::Tensor* t = gpu_tensor(o);
      if (t && leaf_of_other_stream(*t)) {
        PyErr_SetString(PyExc_RuntimeError,
                        "attention_scored: a leaf of this captured call belongs to a graph recorded on another stream that "
                        "still lives; free that graph's outputs before the capture, or record it on the capture's stream");
        return nullptr;
      }
    }
  const at::ScalarType dt = q->scalar_type();
  if (dtype_code(dt) < 0 || !in_place(*q) || !like(*k, *q, dt) || !like(*v, *q, dt) || !grouped_shapes(*q, *k, *v))
    return none();
  mea_problem p;
  mea_score s;
  if (!problem(&p, q->size(0), q->size(1), q->size(2), k->size(2), q->size(3), q->size(3), dtype_code(dt), a[3], a[4], a[5],
               q->device(), false) ||
      !score(&s, a + 6, *q, *k, &bias)) {
    PyErr_Clear();
    return none();
  }
  const bool grad = at::GradMode::is_enabled() &&
                    (q->requires_grad() || k->requires_grad() || v->requires_grad() || (bias && bias->requires_grad()));
  // (checked above: a tensor or None)
  std::vector<at::Tensor> extra;
  for (PyObject* o : {a[5], a[7], a[10], a[11], a[12], a[13]}) extra.push_back(o == Py_None ? at::Tensor() : *gpu_tensor(o));
  at::Tensor o, lse, o_lo;
  mea_status st = MEA_OK;
  {
    pybind11::gil_scoped_release no_gil;
    if (grad) {
      try {
        o = ScoredNode::apply(*q, *k, *v, bias ? std::optional<at::Tensor>(*bias) : std::nullopt, p, s, std::move(extra));
      } catch (const Refused& r) {
        st = r.st;
      }
    } else {
      st = run_scored_fwd(p, s, *q, *k, *v, false, false, &o, &lse, &o_lo);
    }
  }
  if (st != MEA_OK) return failed("mea_scored_attention_fwd", st);
  return THPVariable_Wrap(o);
  END_HANDLE_TH_ERRORS
}

// prefix_fwd(q, k_prefix, v_prefix, k, v, causal, scale, kv_len, q_pos, out,
// need_lse): (o, lse), or None.
PyObject* ext_prefix_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11) return none();
  const at::Tensor *q = gpu_tensor(a[0]), *kp = gpu_tensor(a[1]), *vp = gpu_tensor(a[2]), *k = gpu_tensor(a[3]),
                   *v = gpu_tensor(a[4]);
  if (!q || !kp || !vp || !k || !v) return none();
  const at::ScalarType dt = q->scalar_type();
  if (dtype_code(dt) < 0 || !in_place(*q) || !like(*k, *q, dt) || !like(*v, *q, dt) || !grouped_shapes(*q, *k, *v))
    return none();
  const int64_t unit = 16 / q->element_size();
  for (const at::Tensor* t : {kp, vp})
    if (t->device() != q->device() || t->scalar_type() != dt || t->dim() != 3 || t->stride(2) != 1 ||
        reinterpret_cast<uintptr_t>(t->const_data_ptr()) % 16 || t->stride(0) % unit || t->stride(1) % unit ||
        t->size(0) != k->size(1) || t->size(2) != q->size(3) || t->size(1) != kp->size(1) ||
        t->stride(1) < t->size(2))  // (a row stride of 0 would be read as contiguous)
      return none();
  const at::Tensor* out = nullptr;
  if (a[9] != Py_None) {
    out = gpu_tensor(a[9]);
    if (!out || !like(*out, *q, dt) || out->sizes() != q->sizes()) return none();
  }
  const int need_lse = PyObject_IsTrue(a[10]);
  mea_problem p;
  mea_shared_prefix x = {};
  const void* pos;
  if (need_lse < 0 ||
      !problem(&p, q->size(0), q->size(1), q->size(2), k->size(2), q->size(3), q->size(3), dtype_code(dt), a[5], a[6], a[7],
               q->device(), false) ||
      !vector_ok(a[8], q->device(), at::kInt, {q->size(0)}, &pos)) {
    PyErr_Clear();
    return none();
  }
  x.kv_heads = k->size(1);
  x.n_p = kp->size(1);
  x.k = kp->const_data_ptr();
  x.v = vp->const_data_ptr();
  x.k_strides = mea_tensor_strides{0, kp->stride(0), kp->stride(1)};
  x.v_strides = mea_tensor_strides{0, vp->stride(0), vp->stride(1)};
  x.q_pos = static_cast<const int32_t*>(pos);
  at::Tensor o, lse;
  mea_status st;
  {
    pybind11::gil_scoped_release no_gil;
    const c10::DeviceGuard on(q->device());
    size_t bytes = 0;
    st = g_prefix_ws(&p, &x, &bytes);
    if (st == MEA_OK) {
      o = out ? *out : at::empty(q->sizes(), at::TensorOptions().dtype(dt).device(q->device()));
      if (need_lse) lse = at::empty(q->sizes().slice(0, 3), at::TensorOptions().dtype(at::kFloat).device(q->device()));
      mea_strides ms = {};
      if (!q->is_contiguous() || !k->is_contiguous() || !v->is_contiguous() || !o.is_contiguous()) {
        ms.q = strides_of(*q);
        ms.k = strides_of(*k);
        ms.v = strides_of(*v);
        ms.o = strides_of(o);
        p.strides = &ms;
      }
      at::Tensor ws = workspace(bytes, q->device());
      st = g_prefix_fwd(&p, &x, q->const_data_ptr(), k->const_data_ptr(), v->const_data_ptr(), o.mutable_data_ptr(),
                        need_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr, ws.mutable_data_ptr(), bytes,
                        stream_of(q->device()));
    }
  }
  if (st != MEA_OK) return failed("mea_prefix_attention_fwd", st);
  return tuple_of({o, lse});
  END_HANDLE_TH_ERRORS
}

// init_scored(<addresses in the order of _lib.NATIVE_SCORED_CALLS>).
PyObject* ext_init_scored(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "init_scored takes six addresses");
    return nullptr;
  }
  void* f[6];
  for (int i = 0; i < 6; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_scored_fwd_ws = reinterpret_cast<decltype(g_scored_fwd_ws)>(f[0]);
  g_scored_bwd_ws = reinterpret_cast<decltype(g_scored_bwd_ws)>(f[1]);
  g_scored_fwd = reinterpret_cast<decltype(g_scored_fwd)>(f[2]);
  g_scored_bwd = reinterpret_cast<decltype(g_scored_bwd)>(f[3]);
  g_prefix_ws = reinterpret_cast<decltype(g_prefix_ws)>(f[4]);
  g_prefix_fwd = reinterpret_cast<decltype(g_prefix_fwd)>(f[5]);
  Py_RETURN_NONE;
}

// init(check, fwd_workspace_size, bwd_workspace_size, fwd, bwd): _lib.check and
// the addresses of the library's entry points.
PyObject* ext_init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "init takes a function and four addresses");
    return nullptr;
  }
  void* f[4];
  for (int i = 0; i < 4; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i + 1]);
    if (PyErr_Occurred()) return nullptr;
  }
  PyObject* old = g_check;
  g_check = Py_NewRef(a[0]);
  Py_XDECREF(old);
  g_fwd_ws = reinterpret_cast<decltype(g_fwd_ws)>(f[0]);
  g_bwd_ws = reinterpret_cast<decltype(g_bwd_ws)>(f[1]);
  g_fwd = reinterpret_cast<decltype(g_fwd)>(f[2]);
  g_bwd = reinterpret_cast<decltype(g_bwd)>(f[3]);
  Py_RETURN_NONE;
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {
    {"init", fast(ext_init), METH_FASTCALL, nullptr},
    {"fwd", fast(ext_fwd), METH_FASTCALL, nullptr},
    {"bwd", fast(ext_bwd), METH_FASTCALL, nullptr},
    {"packed_fwd", fast(ext_packed_fwd), METH_FASTCALL, nullptr},
    {"packed_bwd", fast(ext_packed_bwd), METH_FASTCALL, nullptr},
    {"init_scored", fast(ext_init_scored), METH_FASTCALL, nullptr},
    {"scored_fwd", fast(ext_scored_fwd), METH_FASTCALL, nullptr},
    {"scored_bwd", fast(ext_scored_bwd), METH_FASTCALL, nullptr},
    {"scored_apply", fast(ext_scored_apply), METH_FASTCALL, nullptr},
    {"prefix_fwd", fast(ext_prefix_fwd), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_ext", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_ext() { return PyModule_Create(&module); }
