// The calls that a program makes at every layer and step, from Python objects straight to the C ABI: what runner.py's methods check
// and pass on, without a Python object for every look at a tensor.  Small calls are bound by the host (a launch alone takes 2.6
// us).  Host time of a call, through ctypes and here: a linear map 5.2 and 3.3 us, a cache write 7.1 and 3.9, a rotation 5.1 and
// 3.8, attention on rotated queries 5.1 and 3.5, on raw ones 8.6 and 7.2 (its launches take most of that); the smallest
// rollout step in fp32 18 to 20 -> 15.1 us, a linear map of 257 x 768 x 1024 5.76 -> 5.53.
//
// A function here takes a call only if everything is as it should be (plain tensors, exact integers, lists or tuples, shapes and
// strides that fit); otherwise it returns None and has done nothing, and the Python code does what it does: checks one by one and
// raises.  It returns the result, or the library's code where that is not CA_OK.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <initializer_list>

#include "cascade_attn.h"

namespace {

// the library's entry points, as the module that loaded it hands them over
decltype(&kv_cache_append_batch) append_batch_fn = nullptr;
decltype(&rope3d_apply_strided) rope_fn = nullptr;
decltype(&cascade_attn_forward) forward_fn = nullptr;
decltype(&cascade_attn_forward_share) share_fn = nullptr;
decltype(&cascade_attn_forward_rope) forward_rope_fn = nullptr;
decltype(&layer_qkv_publish) publish_fn = nullptr;
decltype(&layer_linear_bf16) linear_fn = nullptr;
decltype(&layer_qk_norm_rope) norm_fn = nullptr;
decltype(&layer_qk_norm_rope_workspace) norm_workspace_fn = nullptr;
decltype(&layer_qk_norm_rope_backward) norm_backward_fn = nullptr;
decltype(&kv_cache_append_batch_norm) append_norm_fn = nullptr;
decltype(&layer_linear_i8_workspace) i8_workspace_fn = nullptr;
decltype(&layer_linear_i8_values) i8_fn = nullptr;
decltype(&layer_gated_bf16) gated_fn = nullptr;
decltype(&layer_gated_saved_bytes) gated_saved_fn = nullptr;
decltype(&layer_gated_backward_workspace) gated_workspace_fn = nullptr;
decltype(&layer_gated_backward_bf16) gated_backward_fn = nullptr;

decltype(&layer_norm) row_norm_fn = nullptr;
decltype(&layer_norm_backward_workspace) row_norm_workspace_fn = nullptr;
decltype(&layer_norm_backward) row_norm_backward_fn = nullptr;
decltype(&layer_linear_adapted_workspace) adapted_room_fn = nullptr;
decltype(&layer_linear_adapted_bf16) adapted_fn = nullptr;
decltype(&layer_linear_adapted_backward_workspace) adapted_workspace_fn = nullptr;
decltype(&layer_linear_adapted_backward_bf16) adapted_backward_fn = nullptr;
decltype(&layer_adamw) adamw_fn = nullptr;

constexpr int kMaxBlocks = 64;                    // of a call taken here

PyObject* not_taken() { Py_RETURN_NONE; }

// a tensor that is nothing but one: no subclass, no wrapper without memory of its own
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckTypeExact(Py_TYPE(o))) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.has_storage() && t.layout() == at::kStrided ? &t : nullptr;
}

bool whole(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}
bool whole32(PyObject* o, int32_t* v) {
  int64_t x;
  if (!whole(o, &x) || x != int32_t(x)) return false;
  *v = int32_t(x);
  return true;
}

// items of a list or tuple, or -1
Py_ssize_t items(PyObject* o, PyObject*** first) {
  if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return -1;
  *first = PySequence_Fast_ITEMS(o);
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
  return n <= kMaxBlocks ? n : -1;
}

template <typename T, bool (*read)(PyObject*, T*)>
int all(PyObject* o, T* out) {
  PyObject** at;
  const Py_ssize_t n = items(o, &at);
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!read(at[i], out + i)) return -1;
  return int(n);
}

struct Pool {                                     // a CascadePool: its context, and what its tensors have to look like
  ca_ctx* ctx;
  int64_t heads, head_dim, block_tokens, f32, device;
  at::ScalarType dtype() const { return f32 ? at::kFloat : at::kBFloat16; }
  void* stream() const {
    return c10::hip::getCurrentHIPStream(device < 0 ? c10::hip::current_device() : c10::DeviceIndex(device)).stream();
  }
};

bool pool_of(PyObject* handle, PyObject* shape, Pool* p) {
  int64_t h;
  if (!whole(handle, &h) || h == 0 || !PyTuple_CheckExact(shape) || PyTuple_GET_SIZE(shape) != 5) return false;
  p->ctx = reinterpret_cast<ca_ctx*>(h);
  int64_t* const to[] = {&p->heads, &p->head_dim, &p->block_tokens, &p->f32, &p->device};
  for (int i = 0; i < 5; ++i)
    if (!whole(PyTuple_GET_ITEM(shape, i), to[i])) return false;
  return true;
}

// [n, heads, head_dim] with any token and head strides
bool fits(const Pool& p, const at::Tensor* t) {
  return t && t->is_cuda() && t->scalar_type() == p.dtype() && t->dim() == 3 && t->stride(2) == 1 && t->size(1) == p.heads && t->size(2) == p.head_dim;
}

// memory of the device that `like` is on (pinned host memory, which kernels reach too, is left to the Python code)
bool beside(const at::Tensor& t, const at::Tensor& like) { return t.is_cuda() && t.device() == like.device(); }

template <typename F>
int32_t released(const F& call) {
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// None, or a result given by the caller, or a new tensor
struct Result {
  at::Tensor made;
  const at::Tensor* t = nullptr;
  PyObject* given = nullptr;
  bool take(PyObject* o) {
    if (o == Py_None) return true;
    given = o;
    t = plain(o);
    return t != nullptr;
  }
  const at::Tensor& or_empty(at::IntArrayRef sizes, const at::Tensor& like) { return or_empty(sizes, like.options()); }
  const at::Tensor& or_empty(at::IntArrayRef sizes, const at::TensorOptions& options) {
    if (!t) {
      made = at::empty(sizes, options);
      t = &made;
    }
    return *t;
  }
  PyObject* give(int32_t rc) {
    if (rc != CA_OK) return PyLong_FromLong(rc);
    if (given) {
      Py_INCREF(given);
      return given;
    }
    return THPVariable_Wrap(made);
  }
};

// Anything that throws (a tensor whose memory cannot be looked at, no memory for a result) is left to the Python code, but for
// what Python code raised in here (a dispatch mode around the allocation), which is the caller's to see.
template <PyObject* (*call)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return call(a, n);
  } catch (python_error& e) {
    e.restore();
  } catch (...) {
  }
  return PyErr_Occurred() ? nullptr : not_taken();
}

// linear(x, w, out)
PyObject* linear(PyObject* const* a, Py_ssize_t n) {
  if (n != 3) return not_taken();
  const at::Tensor *x = plain(a[0]), *w = plain(a[1]);
  Result r;
  if (!x || !w || !r.take(a[2]) || !x->is_cuda() || !w->is_cuda() || x->scalar_type() != at::kBFloat16 || w->scalar_type() != at::kBFloat16 ||
      x->dim() != 2 || w->dim() != 2 || x->size(1) != w->size(1) || x->stride(1) != 1 || w->stride(1) != 1)
    return not_taken();
  const int64_t m = x->size(0), cols = w->size(0), k = x->size(1);
  if (cols != int32_t(cols) || k != int32_t(k)) return not_taken();
  const at::Tensor& y = r.or_empty({m, cols}, *x);
  if (y.dim() != 2 || y.size(0) != m || y.size(1) != cols || y.stride(1) != 1 || y.scalar_type() != at::kBFloat16 || !beside(y, *x)) return not_taken();
  void* const stream = c10::hip::getCurrentHIPStream(x->device().index()).stream();
  const void *xp = x->data_ptr(), *wp = w->data_ptr();
  void* const yp = y.data_ptr();
  const int64_t ldx = x->stride(0), ldw = w->stride(0), ldy = y.stride(0);
  return r.give(released([&] { return linear_fn(xp, wp, yp, m, int32_t(cols), int32_t(k), ldx, ldw, ldy, stream); }));
}

bool real(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = float(PyFloat_AS_DOUBLE(o));
  return true;
}

// a norm's weight: head_dim values of the pool's type, in one piece
bool weighs(const Pool& p, const at::Tensor* w) {
  return w && w->is_cuda() && w->scalar_type() == p.dtype() && w->dim() == 1 && w->size(0) == p.head_dim && w->stride(0) == 1;
}

// append_batch(handle, shape, block_ids, timesteps, epoch, ks, vs) -> slots; append_batch_norm(..., k_weight, eps)
PyObject* append(PyObject* const* a, bool norm) {
  Pool p;
  int64_t ids[kMaxBlocks];
  int32_t ts[kMaxBlocks], slots[kMaxBlocks], epoch;
  const void *ks[kMaxBlocks], *vs[kMaxBlocks], *weight = nullptr;
  float eps = 0.f;
  if (!pool_of(a[0], a[1], &p) || !whole32(a[4], &epoch)) return not_taken();
  const int blocks = all<int64_t, whole>(a[2], ids);
  PyObject **k, **v;
  if (blocks < 1 || all<int32_t, whole32>(a[3], ts) != blocks || items(a[5], &k) != blocks || items(a[6], &v) != blocks) return not_taken();
  int64_t tok = 0, head = 0;
  for (int i = 0; i < blocks; ++i) {
    const at::Tensor *kt = plain(k[i]), *vt = plain(v[i]);
    if (!fits(p, kt) || !fits(p, vt) || kt->size(0) != p.block_tokens || vt->size(0) != p.block_tokens) return not_taken();
    if (i == 0) tok = kt->stride(0), head = kt->stride(1);
    if (kt->stride(0) != tok || kt->stride(1) != head || vt->stride(0) != tok || vt->stride(1) != head) return not_taken();
    ks[i] = kt->data_ptr();
    vs[i] = vt->data_ptr();
  }
  if (norm) {
    const at::Tensor* w = plain(a[7]);
    if (!weighs(p, w) || !real(a[8], &eps)) return not_taken();
    weight = w->data_ptr();
  }
  void* const stream = p.stream();
  const int32_t rc = released([&] {
    return norm ? append_norm_fn(p.ctx, blocks, ids, ts, epoch, ks, vs, tok, head, weight, eps, stream, slots)
                : append_batch_fn(p.ctx, blocks, ids, ts, epoch, ks, vs, tok, head, stream, slots);
  });
  if (rc != CA_OK) return PyLong_FromLong(rc);
  PyObject* const out = PyList_New(blocks);
  for (int i = 0; out && i < blocks; ++i) PyList_SET_ITEM(out, i, PyLong_FromLong(slots[i]));
  return out;
}
PyObject* append_batch(PyObject* const* a, Py_ssize_t n) { return n == 7 ? append(a, false) : not_taken(); }
PyObject* append_batch_norm(PyObject* const* a, Py_ssize_t n) { return n == 9 ? append(a, true) : not_taken(); }

// of a single token or head the stride is free
ca_heads view(const Pool& p, const at::Tensor& t) {
  return ca_heads{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : p.heads * p.head_dim, p.heads > 1 ? t.stride(1) : p.head_dim};
}

PyObject* tuple(std::initializer_list<PyObject*> of) {       // (takes the references)
  PyObject* const t = PyTuple_New(Py_ssize_t(of.size()));
  Py_ssize_t i = 0;
  for (PyObject* o : of) {
    if (t)
      PyTuple_SET_ITEM(t, i++, o);
    else
      Py_XDECREF(o);
  }
  return t;
}
PyObject* none() { Py_RETURN_NONE; }

// norm_rope(handle, shape, q, k, q_weight, k_weight, first_frame, eps, q_out, k_out) -> (q', k'); backward: norm_rope_backward(handle,
// shape, dq_out, dk_out, q, k, q_weight, k_weight, first_frame, eps, dq, dk) -> (dq, dk, dq_weight, dk_weight).  q or k may be None.
PyObject* norm(PyObject* const* a, bool backward) {
  Pool p;
  int64_t first, rows = -1;
  float eps;
  PyObject* const* const of = a + (backward ? 4 : 2);          // q, k, their weights, first_frame, eps, results
  if (!pool_of(a[0], a[1], &p) || !whole(of[4], &first) || !real(of[5], &eps)) return not_taken();
  Result r[2];
  ca_heads x[2], y[2], dz[2];
  const void* w[2] = {};
  at::Tensor dw[2];
  bool there[2];
  const at::Tensor* like = nullptr;
  for (int s = 0; s < 2; ++s) {
    there[s] = of[s] != Py_None;
    if (!there[s]) {
      if (of[2 + s] != Py_None || of[6 + s] != Py_None || (backward && a[2 + s] != Py_None)) return not_taken();
      continue;
    }
    const at::Tensor *t = plain(of[s]), *wt = plain(of[2 + s]);
    if (!fits(p, t) || !weighs(p, wt) || !r[s].take(of[6 + s]) || (rows >= 0 && t->size(0) != rows)) return not_taken();
    rows = t->size(0);
    like = t;
    const at::Tensor& out = r[s].or_empty(t->sizes(), *t);
    if (!fits(p, &out) || out.size(0) != rows) return not_taken();
    if (backward) {
      const at::Tensor* d = plain(a[2 + s]);
      if (!fits(p, d) || d->size(0) != rows) return not_taken();
      dz[s] = view(p, *d);
      dw[s] = at::empty({p.head_dim}, t->options().dtype(at::kFloat));
    }
    x[s] = view(p, *t);
    y[s] = view(p, out);
    w[s] = wt->data_ptr();
  }
  if (!like) return not_taken();
  void* const stream = p.stream();
  auto at_side = [&](ca_heads* v, int s) { return there[s] ? v + s : nullptr; };
  int32_t rc;
  if (backward) {
    const size_t bytes = norm_workspace_fn(p.ctx);
    const at::Tensor work = at::empty({int64_t(bytes)}, like->options().dtype(at::kByte));
    float* const grads[] = {there[0] ? dw[0].data_ptr<float>() : nullptr, there[1] ? dw[1].data_ptr<float>() : nullptr};
    void* const wp = work.data_ptr();
    rc = released([&] {
      return norm_backward_fn(p.ctx, at_side(dz, 0), at_side(dz, 1), at_side(x, 0), at_side(x, 1), w[0], w[1], eps, at_side(y, 0), at_side(y, 1),
                              grads[0], grads[1], rows, first, wp, bytes, stream);
    });
  } else {
    rc = released([&] {
      return norm_fn(p.ctx, at_side(x, 0), at_side(x, 1), w[0], w[1], eps, at_side(y, 0), at_side(y, 1), rows, first, stream);
    });
  }
  if (rc != CA_OK) return PyLong_FromLong(rc);
  PyObject* const out[] = {there[0] ? r[0].give(CA_OK) : none(), there[1] ? r[1].give(CA_OK) : none()};
  if (!backward) return tuple({out[0], out[1]});
  return tuple({out[0], out[1], there[0] ? THPVariable_Wrap(dw[0]) : none(), there[1] ? THPVariable_Wrap(dw[1]) : none()});
}
PyObject* norm_rope(PyObject* const* a, Py_ssize_t n) { return n == 10 ? norm(a, false) : not_taken(); }
PyObject* norm_rope_backward(PyObject* const* a, Py_ssize_t n) { return n == 12 ? norm(a, true) : not_taken(); }

// a [rows, cols] matrix with unit stride along its rows in memory of the device that `like` is on, and its row stride (of a single row
// it is free: whole steps of 16)
bool matrix(const at::Tensor* t, at::ScalarType type, int64_t rows, int64_t cols, const at::Tensor& like, int64_t* ld) {
  if (!t || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || (cols > 1 && t->stride(1) != 1) || !beside(*t, like))
    return false;
  *ld = rows > 1 ? t->stride(0) : (cols + 15) / 16 * 16;
  return true;
}

// linear_i8(x, w_codes, w_scales, k, out): of values x; codes and scales are a QuantizedRows'
PyObject* linear_i8(PyObject* const* a, Py_ssize_t n) {
  int32_t k;
  Result r;
  if (n != 5 || !whole32(a[3], &k) || k < 1 || !r.take(a[4])) return not_taken();
  const at::Tensor *x = plain(a[0]), *w = plain(a[1]), *scales = plain(a[2]);
  if (!x || !w || !scales || !x->is_cuda() || x->dim() != 2 || (x->scalar_type() != at::kBFloat16 && x->scalar_type() != at::kFloat) || w->dim() != 2)
    return not_taken();
  const int64_t m = x->size(0), cols = w->size(0);
  int64_t ldx, ldw, ldy;
  if (cols != int32_t(cols) || !matrix(x, x->scalar_type(), m, k, *x, &ldx) || !matrix(w, at::kChar, cols, (int64_t(k) + 255) / 256 * 256, *x, &ldw) ||
      scales->scalar_type() != at::kFloat || scales->dim() != 1 || scales->size(0) != cols || !scales->is_contiguous() || !beside(*scales, *x))
    return not_taken();
  const at::Tensor& y = r.or_empty({m, cols}, x->scalar_type() == at::kFloat ? x->options().dtype(at::kBFloat16) : x->options());
  if (!matrix(&y, at::kBFloat16, m, cols, *x, &ldy)) return not_taken();
  const size_t bytes = i8_workspace_fn(m, k);
  const at::Tensor work = at::empty({int64_t(bytes)}, x->options().dtype(at::kByte));
  void* const stream = c10::hip::getCurrentHIPStream(x->device().index()).stream();
  const int32_t dtype = x->scalar_type() == at::kFloat ? CA_F32 : CA_BF16;
  const void* const xp = x->data_ptr();
  const int8_t* const wp = w->data_ptr<int8_t>();
  const float* const sp = scales->data_ptr<float>();
  void *const yp = y.data_ptr(), *const workp = work.data_ptr();
  return r.give(released([&] { return i8_fn(xp, dtype, wp, sp, yp, m, int32_t(cols), k, ldx, ldw, ldy, workp, bytes, stream); }));
}

struct GatedCall {
  const at::Tensor *x, *wg, *wu;
  int64_t m, f, k, ldx, ldg, ldu;
  bool take(PyObject* const* a) {
    x = plain(a[0]), wg = plain(a[1]), wu = plain(a[2]);
    if (!x || !wg || !wu || !x->is_cuda() || x->dim() != 2 || wg->dim() != 2) return false;
    m = x->size(0), k = x->size(1), f = wg->size(0);
    return k == int32_t(k) && f == int32_t(f) && matrix(x, at::kBFloat16, m, k, *x, &ldx) && matrix(wg, at::kBFloat16, f, k, *x, &ldg) &&
           matrix(wu, at::kBFloat16, f, k, *x, &ldu);
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(x->device().index()).stream(); }
};

// gated(x, w_gate, w_up, activation, out, train) -> h, or (h, saved)
PyObject* gated(PyObject* const* a, Py_ssize_t n) {
  GatedCall c;
  Result r;
  int32_t act;
  if (n != 6 || !c.take(a) || !whole32(a[3], &act) || !r.take(a[4])) return not_taken();
  const bool train = a[5] == Py_True;
  const at::Tensor& h = r.or_empty({c.m, c.f}, *c.x);
  int64_t ldh;
  if (!matrix(&h, at::kBFloat16, c.m, c.f, *c.x, &ldh)) return not_taken();
  at::Tensor saved;
  float* kept = nullptr;
  if (train) {
    saved = at::empty({int64_t(gated_saved_fn(c.m, int32_t(c.f)) / 4)}, c.x->options().dtype(at::kFloat));
    kept = saved.data_ptr<float>();
  }
  const void *xp = c.x->data_ptr(), *gp = c.wg->data_ptr(), *up = c.wu->data_ptr();
  void *const hp = h.data_ptr(), *const stream = c.stream();
  const int32_t rc = released([&] {
    return gated_fn(xp, gp, up, hp, kept, act, c.m, int32_t(c.f), int32_t(c.k), c.ldx, c.ldg, c.ldu, ldh, stream);
  });
  if (!train || rc != CA_OK) return r.give(rc);
  return tuple({r.give(rc), THPVariable_Wrap(saved)});
}

// gated_backward(x, w_gate, w_up, dh, saved, activation) -> (dx, dw_gate, dw_up)
PyObject* gated_backward(PyObject* const* a, Py_ssize_t n) {
  GatedCall c;
  int32_t act;
  int64_t lddh;
  if (n != 6 || !c.take(a) || !whole32(a[5], &act)) return not_taken();
  const at::Tensor *dh = plain(a[3]), *saved = plain(a[4]);
  if (!matrix(dh, at::kBFloat16, c.m, c.f, *c.x, &lddh) || !saved || saved->scalar_type() != at::kFloat || 
      uint64_t(saved->numel()) * 4 != gated_saved_fn(c.m, int32_t(c.f)) || !saved->is_contiguous() || !beside(*saved, *c.x))
    return not_taken();
  const size_t bytes = gated_workspace_fn(c.m, int32_t(c.f), int32_t(c.k));
  const at::Tensor dx = at::empty({c.m, c.k}, c.x->options()), dw = at::empty({2, c.f, c.k}, c.x->options()),
                   work = at::empty({int64_t(bytes)}, c.x->options().dtype(at::kByte));
  const float* const kept = saved->data_ptr<float>();
  const void *xp = c.x->data_ptr(), *gp = c.wg->data_ptr(), *up = c.wu->data_ptr(), *dhp = dh->data_ptr();
  void *const dxp = dx.data_ptr(), *const dwp = dw.data_ptr(), *const workp = work.data_ptr(), *const stream = c.stream();
  const int32_t rc = released([&] {
    return gated_backward_fn(dhp, xp, gp, up, kept, act, dxp, dwp, static_cast<char*>(dwp) + c.f * c.k * 2, c.m, int32_t(c.f), int32_t(c.k), lddh, c.ldx,
                             c.ldg, c.ldu, c.k, c.k, workp, bytes, stream);
  });
  if (rc != CA_OK) return PyLong_FromLong(rc);
  return tuple({THPVariable_Wrap(dx), THPVariable_Wrap(dw[0]), THPVariable_Wrap(dw[1])});
}

// a [rows, cols] matrix of any alignment and row stride
bool rows_of(const at::Tensor* t, at::ScalarType type, int64_t rows, int64_t cols, const at::Tensor& like, int64_t* ld) {
  if (!t || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || (cols > 1 && t->stride(1) != 1) || !beside(*t, like))
    return false;
  *ld = rows > 1 ? t->stride(0) : cols;
  return true;
}
bool stored(const at::Tensor& t, int32_t* dtype) {
  *dtype = t.scalar_type() == at::kFloat ? CA_F32 : CA_BF16;
  return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16;
}
// launches go to the current device: other ones are left to the Python code
bool here(const at::Tensor& t) { return t.is_cuda() && t.device().index() == c10::hip::current_device(); }

struct RowNormCall {                              // x, weight, bias
  const at::Tensor *x, *w[2] = {nullptr, nullptr};
  int64_t rows, width, groups = 1, ldx, ldw;
  int32_t dtype, w_dtype = CA_F32;
  bool take(PyObject* const* a) {
    x = plain(a[0]);
    if (!x || x->dim() != 2 || !here(*x) || !stored(*x, &dtype)) return false;
    rows = x->size(0), width = ldw = x->size(1);
    if (width != int32_t(width) || width < 1 || !rows_of(x, x->scalar_type(), rows, width, *x, &ldx)) return false;
    const at::Tensor* like = nullptr;
    for (int i = 0; i < 2; ++i) {
      if (a[1 + i] == Py_None) continue;
      const at::Tensor* t = w[i] = plain(a[1 + i]);
      if (!t || !beside(*t, *x) || !stored(*t, &w_dtype) || (t->scalar_type() != at::kFloat && t->scalar_type() != x->scalar_type()) || t->dim() < 1 ||
          t->dim() > 2 || t->size(-1) != width || (width > 1 && t->stride(-1) != 1) ||
          (like && (t->scalar_type() != like->scalar_type() || t->sizes() != like->sizes() || t->strides() != like->strides())))
        return false;
      like = t;
      groups = t->dim() == 2 ? t->size(0) : 1;
      ldw = groups > 1 ? t->stride(0) : width;
    }
    return groups >= 1 && rows % groups == 0;
  }
  const void* weight(int i) const { return w[i] ? w[i]->data_ptr() : nullptr; }
  void* stream() const { return c10::hip::getCurrentHIPStream(x->device().index()).stream(); }
};

// layer_norm(x, weight, bias, eps, out)
PyObject* layer_norm_(PyObject* const* a, Py_ssize_t n) {
  RowNormCall c;
  Result r;
  float eps;
  int64_t ldy;
  if (n != 5 || !c.take(a) || !real(a[3], &eps) || !r.take(a[4])) return not_taken();
  const at::Tensor& y = r.or_empty({c.rows, c.width}, *c.x);
  if (!rows_of(&y, c.x->scalar_type(), c.rows, c.width, *c.x, &ldy)) return not_taken();
  const void *const xp = c.x->data_ptr(), *const wp = c.weight(0), *const bp = c.weight(1);
  void *const yp = y.data_ptr(), *const stream = c.stream();
  return r.give(released([&] { return row_norm_fn(xp, c.dtype, wp, bp, c.w_dtype, eps, yp, c.rows, int32_t(c.width), c.groups, c.ldx, c.ldw, ldy, stream); }));
}

// layer_norm_backward(x, weight, bias, dy, eps, dx) -> (dx, dweight, dbias)
PyObject* layer_norm_backward_(PyObject* const* a, Py_ssize_t n) {
  RowNormCall c;
  Result r;
  float eps;
  int64_t lddy, lddx;
  if (n != 6 || !c.take(a) || !real(a[4], &eps) || !r.take(a[5])) return not_taken();
  const at::Tensor* dy = plain(a[3]);
  if (!rows_of(dy, c.x->scalar_type(), c.rows, c.width, *c.x, &lddy)) return not_taken();
  const at::Tensor& dx = r.or_empty({c.rows, c.width}, *c.x);
  if (!rows_of(&dx, c.x->scalar_type(), c.rows, c.width, *c.x, &lddx)) return not_taken();
  const auto single = c.x->options().dtype(at::kFloat);
  at::Tensor grads[2], work;
  float* to[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (c.w[i]) {
      grads[i] = at::empty(c.w[i]->sizes(), single);
      to[i] = grads[i].data_ptr<float>();
    }
  const size_t bytes = row_norm_workspace_fn(c.rows, int32_t(c.width), c.groups);
  work = at::empty({int64_t(bytes)}, c.x->options().dtype(at::kByte));
  const void *const xp = c.x->data_ptr(), *const wp = c.weight(0), *const dyp = dy->data_ptr();
  void *const dxp = dx.data_ptr(), *const workp = work.data_ptr(), *const stream = c.stream();
  const int32_t rc = released([&] {
    return row_norm_backward_fn(dyp, xp, c.dtype, wp, c.w_dtype, eps, dxp, to[0], to[1], c.rows, int32_t(c.width), c.groups, lddy, c.ldx, c.ldw, lddx, workp, bytes,
                                stream);
  });
  if (rc != CA_OK) return PyLong_FromLong(rc);
  return tuple({r.give(rc), c.w[0] ? THPVariable_Wrap(grads[0]) : none(), c.w[1] ? THPVariable_Wrap(grads[1]) : none()});
}

struct AdaptedCall {                              // x, down, up, scales, index
  const at::Tensor *x, *down, *up, *scales, *index;
  int64_t m, n, k, adapters, rank, ldx;
  bool take(PyObject* const* a) {
    const at::Tensor** const to[] = {&x, &down, &up, &scales, &index};
    for (int i = 0; i < 5; ++i)
      if (!(*to[i] = plain(a[i]))) return false;
    if (!here(*x) || x->dim() != 2 || down->dim() != 3 || up->dim() != 3) return false;
    m = x->size(0), k = x->size(1), n = up->size(1), adapters = down->size(0), rank = down->size(1);
    for (const at::Tensor* t : {down, up, scales, index})
      if (!beside(*t, *x) || !t->is_contiguous()) return false;
    return n == int32_t(n) && k == int32_t(k) && adapters == int32_t(adapters) && rank == int32_t(rank) && matrix(x, at::kBFloat16, m, k, *x, &ldx) &&
           down->scalar_type() == at::kBFloat16 && up->scalar_type() == at::kBFloat16 && down->size(2) == k && up->size(0) == adapters && up->size(2) == rank &&
           scales->scalar_type() == at::kFloat && scales->dim() == 1 && scales->size(0) == adapters && index->scalar_type() == at::kInt && index->dim() == 1 &&
           index->size(0) == m;
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(x->device().index()).stream(); }
};

// linear_adapted(x, down, up, scales, index, w, out) -> (y, low)
PyObject* linear_adapted(PyObject* const* a, Py_ssize_t n) {
  AdaptedCall c;
  Result r;
  int64_t ldw, ldy;
  if (n != 7 || !c.take(a) || !r.take(a[6])) return not_taken();
  const at::Tensor* w = plain(a[5]);
  if (!matrix(w, at::kBFloat16, c.n, c.k, *c.x, &ldw)) return not_taken();
  const at::Tensor& y = r.or_empty({c.m, c.n}, *c.x);
  if (!matrix(&y, at::kBFloat16, c.m, c.n, *c.x, &ldy)) return not_taken();
  const at::Tensor low = at::empty({2, c.m, c.rank}, c.x->options());
  const size_t bytes = adapted_room_fn(c.m, int32_t(c.rank));
  at::Tensor work;
  if (bytes > 0) work = at::empty({int64_t(bytes)}, c.x->options().dtype(at::kByte));
  void* const workp = bytes > 0 ? work.data_ptr() : nullptr;
  const void *const xp = c.x->data_ptr(), *const wp = w->data_ptr(), *const dp = c.down->data_ptr(), *const up = c.up->data_ptr();
  const float* const sp = c.scales->data_ptr<float>();
  const int32_t* const ip = c.index->data_ptr<int32_t>();
  void *const lp = low.data_ptr(), *const yp = y.data_ptr(), *const stream = c.stream();
  const int32_t rc = released([&] {
    return adapted_fn(xp, wp, dp, up, sp, ip, lp, yp, c.m, int32_t(c.n), int32_t(c.k), int32_t(c.adapters), int32_t(c.rank), c.ldx, ldw, ldy, workp, bytes,
                      stream);
  });
  return rc != CA_OK ? PyLong_FromLong(rc) : tuple({r.give(rc), THPVariable_Wrap(low)});
}

// linear_adapted_backward(x, down, up, scales, index, dy, w_t, saved, rank) -> (dx, d_down, d_up)
PyObject* linear_adapted_backward(PyObject* const* a, Py_ssize_t n) {
  AdaptedCall c;
  int64_t lddy, ldw, used;
  if (n != 9 || !c.take(a) || !whole(a[8], &used) || used < 1 || used > c.rank) return not_taken();
  const at::Tensor *dy = plain(a[5]), *w = a[6] == Py_None ? nullptr : plain(a[6]), *saved = plain(a[7]);
  ldw = c.n;
  if (!matrix(dy, at::kBFloat16, c.m, c.n, *c.x, &lddy) || (a[6] != Py_None && !matrix(w, at::kBFloat16, c.k, c.n, *c.x, &ldw)) || !saved ||
      saved->scalar_type() != at::kBFloat16 || saved->dim() != 3 || saved->size(0) != 2 || saved->size(1) != c.m || saved->size(2) != c.rank || !saved->is_contiguous() ||
      !beside(*saved, *c.x))
    return not_taken();
  const size_t bytes = adapted_workspace_fn(c.m, int32_t(c.n), int32_t(c.k), int32_t(c.adapters), int32_t(c.rank));
  at::Tensor dx;
  if (w) dx = at::empty({c.m, c.k}, c.x->options());
  const at::Tensor d_down = at::empty({c.adapters, used, c.k}, c.x->options()), d_up = at::empty({c.adapters, c.n, used}, c.x->options()),
                   work = at::empty({int64_t(bytes)}, c.x->options().dtype(at::kByte));
  const void *const xp = c.x->data_ptr(), *const wp = w ? w->data_ptr() : nullptr, *const dp = c.down->data_ptr(), *const up = c.up->data_ptr(),
             *const dyp = dy->data_ptr(), *const lp = saved->data_ptr();
  const float* const sp = c.scales->data_ptr<float>();
  const int32_t* const ip = c.index->data_ptr<int32_t>();
  void *const dxp = w ? dx.data_ptr() : nullptr, *const ddp = d_down.data_ptr(), *const dup = d_up.data_ptr(), *const workp = work.data_ptr(), *const stream = c.stream();
  const int32_t rc = released([&] {
    return adapted_backward_fn(dyp, xp, wp, dp, up, sp, ip, lp, dxp, ddp, dup, c.m, int32_t(c.n), int32_t(c.k), int32_t(c.adapters), int32_t(c.rank), int32_t(used),
                               lddy, c.ldx, ldw, c.k, workp, bytes, stream);
  });
  if (rc != CA_OK) return PyLong_FromLong(rc);
  return tuple({w ? THPVariable_Wrap(dx) : none(), THPVariable_Wrap(d_down), THPVariable_Wrap(d_up)});
}

// adamw(address of the tensors, their table on the device, params, grads, state_bits, lr, (beta1, beta2), eps, weight_decay, grad_scale)
PyObject* adamw(PyObject* const* a, Py_ssize_t n) {
  int64_t at_host;
  int32_t bits;
  double v[4], betas[2];
  if (n != 10 || !whole(a[0], &at_host) || at_host == 0 || !whole32(a[4], &bits) || !PyTuple_CheckExact(a[6]) || PyTuple_GET_SIZE(a[6]) != 2) return not_taken();
  PyObject* const numbers[] = {a[5], a[7], a[8], a[9]};
  for (int i = 0; i < 4; ++i) {
    if (!PyFloat_CheckExact(numbers[i])) return not_taken();
    v[i] = PyFloat_AS_DOUBLE(numbers[i]);
  }
  for (int i = 0; i < 2; ++i) {
    PyObject* const o = PyTuple_GET_ITEM(a[6], i);
    if (!PyFloat_CheckExact(o)) return not_taken();
    betas[i] = PyFloat_AS_DOUBLE(o);
  }
  const at::Tensor* table = plain(a[1]);
  if (!table || !here(*table) || !PyList_CheckExact(a[2]) || (!PyList_CheckExact(a[3]) && !PyTuple_CheckExact(a[3]))) return not_taken();
  const Py_ssize_t count = PyList_GET_SIZE(a[2]);
  if (PySequence_Fast_GET_SIZE(a[3]) != count || size_t(table->numel()) != size_t(count) * sizeof(ca_adamw_tensor)) return not_taken();
  ca_adamw_tensor* const tensors = reinterpret_cast<ca_adamw_tensor*>(at_host);
  PyObject** const grads = PySequence_Fast_ITEMS(a[3]);
  for (Py_ssize_t i = 0; i < count; ++i) {
    const at::Tensor* p = plain(PyList_GET_ITEM(a[2], i));
    if (!p || p->data_ptr() != tensors[i].param) return not_taken();
    if (grads[i] == Py_None) {
      tensors[i].grad = nullptr;
      continue;
    }
    const at::Tensor* g = plain(grads[i]);
    if (!g || !beside(*g, *p) || g->sizes() != p->sizes() || !g->is_contiguous() || !stored(*g, &tensors[i].grad_dtype)) return not_taken();
    tensors[i].grad = g->data_ptr();
  }
  const ca_adamw_tensor* const on_device = static_cast<const ca_adamw_tensor*>(table->data_ptr());
  void* const stream = c10::hip::getCurrentHIPStream(table->device().index()).stream();
  // (the lock is held: the tensors are the optimizer's, and another thread's call would write them)
  return PyLong_FromLong(adamw_fn(tensors, on_device, int32_t(count), bits, v[0], betas[0], betas[1], v[1], v[2], v[3], stream));
}

// rope(handle, shape, x, first_frame, out)
PyObject* rope(PyObject* const* a, Py_ssize_t n) {
  Pool p;
  Result r;
  int64_t first;
  if (n != 5 || !pool_of(a[0], a[1], &p) || !whole(a[3], &first) || !r.take(a[4])) return not_taken();
  const at::Tensor* x = plain(a[2]);
  if (!fits(p, x)) return not_taken();
  const at::Tensor& y = r.or_empty(x->sizes(), *x);
  if (!fits(p, &y) || y.size(0) != x->size(0)) return not_taken();
  void *const stream = p.stream(), *const yp = y.data_ptr();
  const void* const xp = x->data_ptr();
  const int64_t s[] = {x->stride(0), x->stride(1), y.stride(0), y.stride(1)}, rows = x->size(0);
  return r.give(released([&] { return rope_fn(p.ctx, xp, s[0], s[1], yp, s[2], s[3], rows, first, stream); }));
}

// forward(handle, shape, q_rot, inflight, mode, out, share) with share None or (first, count)
PyObject* forward(PyObject* const* a, Py_ssize_t n) {
  Pool p;
  Result r;
  int64_t ids[kMaxBlocks];
  int32_t mode, share[2];
  if (n != 7 || !pool_of(a[0], a[1], &p) || !whole32(a[4], &mode) || !r.take(a[5])) return not_taken();
  const int blocks = all<int64_t, whole>(a[3], ids);
  const bool part = a[6] != Py_None;
  PyObject** of_share;
  if (blocks < 1 || (part && (items(a[6], &of_share) != 2 || !whole32(of_share[0], share) || !whole32(of_share[1], share + 1)))) return not_taken();
  const at::Tensor* q = plain(a[2]);
  if (!fits(p, q) || !q->is_contiguous() || q->size(0) != (part ? share[1] : blocks) * p.block_tokens) return not_taken();
  const at::Tensor& o = r.or_empty(q->sizes(), *q);
  if (!o.is_contiguous() || o.sizes() != q->sizes() || !fits(p, &o) || !beside(o, *q)) return not_taken();
  void *const stream = p.stream(), *const op = o.data_ptr();
  const void* const qp = q->data_ptr();
  return r.give(released([&] {
    return part ? share_fn(p.ctx, qp, ids, blocks, share[0], share[1], mode, op, stream) : forward_fn(p.ctx, qp, ids, blocks, mode, op, stream);
  }));
}

// forward_rope(handle, shape, q, inflight, mode, out)
PyObject* forward_rope(PyObject* const* a, Py_ssize_t n) {
  Pool p;
  Result r;
  int64_t ids[kMaxBlocks];
  int32_t mode;
  if (n != 6 || !pool_of(a[0], a[1], &p) || !whole32(a[4], &mode) || !r.take(a[5])) return not_taken();
  const int blocks = all<int64_t, whole>(a[3], ids);
  const at::Tensor* q = plain(a[2]);
  if (blocks < 1 || !fits(p, q) || q->size(0) != blocks * p.block_tokens) return not_taken();
  const at::Tensor& o = r.or_empty(q->sizes(), *q);
  if (!o.is_contiguous() || o.sizes() != q->sizes() || !fits(p, &o) || !beside(o, *q)) return not_taken();
  void *const stream = p.stream(), *const op = o.data_ptr();
  const void* const qp = q->data_ptr();
  const int64_t tok = q->stride(0), head = q->stride(1);
  return r.give(released([&] { return forward_rope_fn(p.ctx, qp, tok, head, ids, blocks, mode, op, stream); }));
}

// qkv_publish(handle, shape, x, w_qkv, block_ids, timesteps, epoch, q_out)
PyObject* qkv_publish(PyObject* const* a, Py_ssize_t n) {
  Pool p;
  Result r;
  int64_t ids[kMaxBlocks];
  int32_t ts[kMaxBlocks], slots[kMaxBlocks], epoch;
  if (n != 8 || !pool_of(a[0], a[1], &p) || !whole32(a[6], &epoch) || !r.take(a[7])) return not_taken();
  const int blocks = all<int64_t, whole>(a[4], ids);
  const at::Tensor *x = plain(a[2]), *w = plain(a[3]);
  const int64_t rows = blocks * p.block_tokens, width = p.heads * p.head_dim;
  if (blocks < 1 || all<int32_t, whole32>(a[5], ts) != blocks || !x || !w || !x->is_cuda() || x->scalar_type() != at::kBFloat16 || x->dim() != 2 ||
      x->size(0) != rows || x->stride(1) != 1 || x->size(1) != int32_t(x->size(1)) || w->dim() != 2 || w->size(0) != 3 * width ||
      w->size(1) != x->size(1) || w->stride(1) != 1 || w->scalar_type() != at::kBFloat16 || !beside(*w, *x))
    return not_taken();
  const at::Tensor& q = r.or_empty({rows, p.heads, p.head_dim}, *x);
  if (q.dim() != 3 || !q.is_contiguous() || q.size(0) != rows || q.size(1) != p.heads || q.size(2) != p.head_dim || q.scalar_type() != at::kBFloat16 ||
      !beside(q, *x))
    return not_taken();
  void *const stream = p.stream(), *const qp = q.data_ptr();
  const void *const xp = x->data_ptr(), *const wp = w->data_ptr();
  const int64_t ldx = x->stride(0), ldw = w->stride(0);
  const int32_t k = int32_t(x->size(1));
  return r.give(released([&] { return publish_fn(p.ctx, blocks, ids, ts, epoch, xp, ldx, wp, ldw, k, qp, stream, slots); }));
}

// bind(addresses of the seven entry points in the order above)
PyObject* bind(PyObject* const* a, Py_ssize_t n) {
  int64_t f[7];
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "seven addresses");
    return nullptr;
  }
  for (int i = 0; i < 7; ++i)
    if (!whole(a[i], f + i) || f[i] == 0) {
      PyErr_SetString(PyExc_TypeError, "an address is an int");
      return nullptr;
    }
  append_batch_fn = reinterpret_cast<decltype(append_batch_fn)>(f[0]);
  rope_fn = reinterpret_cast<decltype(rope_fn)>(f[1]);
  forward_fn = reinterpret_cast<decltype(forward_fn)>(f[2]);
  share_fn = reinterpret_cast<decltype(share_fn)>(f[3]);
  forward_rope_fn = reinterpret_cast<decltype(forward_rope_fn)>(f[4]);
  publish_fn = reinterpret_cast<decltype(publish_fn)>(f[5]);
  linear_fn = reinterpret_cast<decltype(linear_fn)>(f[6]);
  Py_RETURN_NONE;
}

// bind_layer(addresses of the ten entry points of the rest of a layer in the order above)
PyObject* bind_layer(PyObject* const* a, Py_ssize_t n) {
  int64_t f[10];
  if (n != 10) {
    PyErr_SetString(PyExc_TypeError, "ten addresses");
    return nullptr;
  }
  for (int i = 0; i < 10; ++i)
    if (!whole(a[i], f + i) || f[i] == 0) {
      PyErr_SetString(PyExc_TypeError, "an address is an int");
      return nullptr;
    }
  norm_fn = reinterpret_cast<decltype(norm_fn)>(f[0]);
  norm_workspace_fn = reinterpret_cast<decltype(norm_workspace_fn)>(f[1]);
  norm_backward_fn = reinterpret_cast<decltype(norm_backward_fn)>(f[2]);
  append_norm_fn = reinterpret_cast<decltype(append_norm_fn)>(f[3]);
  i8_workspace_fn = reinterpret_cast<decltype(i8_workspace_fn)>(f[4]);
  i8_fn = reinterpret_cast<decltype(i8_fn)>(f[5]);
  gated_fn = reinterpret_cast<decltype(gated_fn)>(f[6]);
  gated_saved_fn = reinterpret_cast<decltype(gated_saved_fn)>(f[7]);
  gated_workspace_fn = reinterpret_cast<decltype(gated_workspace_fn)>(f[8]);
  gated_backward_fn = reinterpret_cast<decltype(gated_backward_fn)>(f[9]);
  Py_RETURN_NONE;
}

// bind_adapt(addresses of the eight entry points of the operators that a layer is adapted with in the order above)
PyObject* bind_adapt(PyObject* const* a, Py_ssize_t n) {
  int64_t f[8];
  if (n != 8) {
    PyErr_SetString(PyExc_TypeError, "eight addresses");
    return nullptr;
  }
  for (int i = 0; i < 8; ++i)
    if (!whole(a[i], f + i) || f[i] == 0) {
      PyErr_SetString(PyExc_TypeError, "an address is an int");
      return nullptr;
    }
  row_norm_fn = reinterpret_cast<decltype(row_norm_fn)>(f[0]);
  row_norm_workspace_fn = reinterpret_cast<decltype(row_norm_workspace_fn)>(f[1]);
  row_norm_backward_fn = reinterpret_cast<decltype(row_norm_backward_fn)>(f[2]);
  adapted_room_fn = reinterpret_cast<decltype(adapted_room_fn)>(f[3]);
  adapted_fn = reinterpret_cast<decltype(adapted_fn)>(f[4]);
  adapted_workspace_fn = reinterpret_cast<decltype(adapted_workspace_fn)>(f[5]);
  adapted_backward_fn = reinterpret_cast<decltype(adapted_backward_fn)>(f[6]);
  adamw_fn = reinterpret_cast<decltype(adamw_fn)>(f[7]);
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(linear), METHOD(append_batch), METHOD(rope), METHOD(forward), METHOD(forward_rope), METHOD(qkv_publish),
                         METHOD(append_batch_norm), METHOD(norm_rope), METHOD(norm_rope_backward), METHOD(linear_i8), METHOD(gated),
                         METHOD(gated_backward), METHOD(linear_adapted), METHOD(linear_adapted_backward), METHOD(adamw),
                         {"layer_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<layer_norm_>)), METH_FASTCALL, nullptr},
                         {"layer_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<layer_norm_backward_>)), METH_FASTCALL, nullptr},
                         METHOD(bind), METHOD(bind_layer), METHOD(bind_adapt), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
