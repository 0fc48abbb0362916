// Native call path of the Python binding.
//
// Each function takes the tensors of one library call, checks what the Python
// binding checks (type, shape, contiguity, device, with the same rules) and
// makes the call on torch's current stream.  It answers None, having done
// nothing, wherever anything is out of the ordinary: a wrong shape, another
// current device, a tensor subclass, an active torch mode.  The binding then goes
// its general way, which accepts or refuses the call with its own messages.  A
// call that the library has seen is never made again: a status other than MOA_OK
// raises the binding's error (after a failed launch part of the work may be
// enqueued).  What it saves is host time: about 13 us of interpreted checks per
// call become about 2.
#include <Python.h>

#include <algorithm>
#include <cstring>
#include <new>

#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/PythonTorchFunctionTLS.h>

#include "moa.h"

namespace {

// Entry points of the loaded library, in the order of the binding's table.
struct Api {
  decltype(&moa_prefill) prefill;
  decltype(&moa_kv_append) kv_append;
  decltype(&moa_decode) decode;
  decltype(&moa_decode_noalloc) decode_noalloc;
  decltype(&moa_kv_append_ragged) kv_append_ragged;
  decltype(&moa_decode_ragged) decode_ragged;
  decltype(&moa_influence) influence;
  decltype(&moa_rule_loss) rule_loss;
  decltype(&moa_paged_append) paged_append;
  decltype(&moa_paged_prefill) paged_prefill;
  decltype(&moa_paged_decode) paged_decode;
  decltype(&moa_paged_decode_shared) paged_decode_shared;
  decltype(&moa_paged_assign) paged_assign;
  decltype(&moa_quant_append) quant_append;
  decltype(&moa_quant_prefill) quant_prefill;
  decltype(&moa_quant_decode) quant_decode;
  decltype(&moa_quant_decode_shared) quant_decode_shared;
  decltype(&moa_paged_assign_state) paged_assign_state;
};

// What the checks need of a library and a plan; held by a capsule.
struct Bound {
  Api api;
  const moa_plan_t* plan;       // null: for the calls that take no plan
  int64_t hq, hkv, d, rows;
  at::ScalarType dtype;
  PyObject* check;              // the binding's function that raises for a status
  ~Bound() { Py_XDECREF(check); }
};
constexpr const char* kName = "moa.bound";

Bound* bound_of(PyObject* o) {
  return PyCapsule_IsValid(o, kName) ? static_cast<Bound*>(PyCapsule_GetPointer(o, kName)) : nullptr;
}

// A plain strided GPU tensor that no torch transform wraps.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) return nullptr;
  using K = c10::DispatchKey;
  const c10::DispatchKeySet odd({K::Python, K::PythonTLSSnapshot, K::Functionalize, K::FuncTorchBatched,
                                 K::FuncTorchGradWrapper, K::Conjugate, K::Negative, K::ZeroTensor});
  return t.key_set().has_any(odd) ? nullptr : &t;
}

bool modes_active() {
  return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled();
}

// The shape, type and device of one call's tensors.
struct Check {
  bool ok = true;
  c10::DeviceIndex device = -1;
  const at::Tensor* any(PyObject* o) {
    const at::Tensor* t = ok ? plain(o) : nullptr;
    if (!t || (device >= 0 && t->device().index() != device) || !t->is_contiguous()) {
      ok = false;
      return nullptr;
    }
    device = t->device().index();
    return t;
  }
  const at::Tensor* operator()(PyObject* o, at::ScalarType type, at::IntArrayRef shape) {
    const at::Tensor* t = any(o);
    if (t && (t->scalar_type() != type || t->sizes() != shape)) ok = false;
    return ok ? t : nullptr;
  }
  // Packed tokens [n, heads, d], contiguous but for the tokens; null where they are
  // not of this kind.
  const at::Tensor* tokens(PyObject* o, at::ScalarType type, at::IntArrayRef shape, int64_t* stride) {
    const at::Tensor* t = ok ? plain(o) : nullptr;
    if (!t || (device >= 0 && t->device().index() != device) || t->scalar_type() != type || t->sizes() != shape ||
        t->stride(2) != 1 || (shape[1] > 1 && t->stride(1) != shape[2])) {
      ok = false;
      return nullptr;
    }
    device = t->device().index();
    *stride = shape[0] > 1 ? t->stride(0) : shape[1] * shape[2];
    return t;
  }
  // Tensors checked and the call's device current.
  bool done() const { return ok && device >= 0 && c10::hip::current_device() == device; }
  void* stream() const { return c10::hip::getCurrentHIPStream(device).stream(); }
};

// Makes the call while other Python threads run; false with a Python exception
// set where it was not MOA_OK.
template <class F>
bool call(const Bound& b, F&& f) {
  moa_status_t st = MOA_OK;
  bool no_memory = false;
  Py_BEGIN_ALLOW_THREADS
  try {
    st = f();
  } catch (...) {                 // of a message's string: nothing else in the library throws
    no_memory = true;
  }
  Py_END_ALLOW_THREADS
  if (no_memory) return PyErr_NoMemory(), false;
  if (st == MOA_OK) return true;
  PyObject* r = PyObject_CallFunction(b.check, "i", static_cast<int>(st));
  if (r) PyErr_Format(PyExc_RuntimeError, "moa status %d", static_cast<int>(st));
  Py_XDECREF(r);
  return false;
}

bool as_int(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}

PyObject* none() { Py_RETURN_NONE; }
PyObject* same(PyObject* o) {
  Py_INCREF(o);
  return o;
}

// The output: `given`, or a new tensor like q where it is None.
struct Out {
  at::Tensor fresh;
  const at::Tensor* t = nullptr;
  PyObject* given;
  Out(PyObject* o, const at::Tensor* q, Check& c) : given(o) {
    if (!c.ok) return;
    if (o != Py_None) {
      t = c(o, q->scalar_type(), q->sizes());
    } else if (c.done()) {
      fresh = at::empty_like(*q);
      t = &fresh;
    }
  }
  PyObject* answer() { return given != Py_None ? same(given) : THPVariable_Wrap(fresh); }
};

#define MOA_ENTER(n)                                   \
  Bound* b = nargs == (n) ? bound_of(args[0]) : nullptr; \
  if (!b || modes_active()) return none();             \
  try {                                                \
    Check c;
#define MOA_LEAVE            \
  }                          \
  catch (...) {              \
    PyErr_Clear();           \
    return none();           \
  }

// prefill(bound, q, k, v, o)
PyObject* prefill(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(5)
  const at::Tensor* q = c.any(args[1]);
  if (!b->plan || !q || q->dim() != 4) return none();
  const int64_t bsz = q->size(0), n = q->size(1);
  c(args[1], b->dtype, {bsz, n, b->hq, b->d});
  const at::Tensor* k = c(args[2], b->dtype, {bsz, n, b->hkv, b->d});
  const at::Tensor* v = c(args[3], b->dtype, {bsz, n, b->hkv, b->d});
  Out o(args[4], q, c);
  if (!c.done() || !o.t || bsz > INT32_MAX) return none();
  void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *po = o.t->data_ptr(), *s = c.stream();
  if (!call(*b, [&] { return b->api.prefill(b->plan, pq, pk, pv, po, static_cast<int32_t>(bsz), n, s); })) return nullptr;
  return o.answer();
  MOA_LEAVE
}

// kv_append(bound, k_cache, v_cache, pos_cache, k_new, v_new, start_pos)
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  int64_t start;
  const at::Tensor* kn = c.any(args[4]);
  if (!b->plan || !kn || kn->dim() != 4 || !as_int(args[6], &start)) return none();
  const int64_t bsz = kn->size(0), n = kn->size(1);
  c(args[4], b->dtype, {bsz, n, b->hkv, b->d});
  const at::Tensor* vn = c(args[5], b->dtype, {bsz, n, b->hkv, b->d});
  const at::Tensor* kc = c(args[1], b->dtype, {bsz, b->rows, b->d});
  const at::Tensor* vc = c(args[2], b->dtype, {bsz, b->rows, b->d});
  const at::Tensor* pc = c(args[3], at::kInt, {bsz, b->rows});
  if (!c.done() || bsz > INT32_MAX) return none();
  void *pkc = kc->data_ptr(), *pvc = vc->data_ptr(), *pkn = kn->data_ptr(), *pvn = vn->data_ptr(), *s = c.stream();
  int32_t* pp = static_cast<int32_t*>(pc->data_ptr());
  if (!call(*b, [&] { return b->api.kv_append(b->plan, pkc, pvc, pp, pkn, pvn, static_cast<int32_t>(bsz), start, n, s); }))
    return nullptr;
  Py_RETURN_TRUE;
  MOA_LEAVE
}

// kv_append_ragged(bound, k_cache, v_cache, pos_cache, k_new, v_new, positions)
PyObject* kv_append_ragged(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  const at::Tensor* kn = c.any(args[4]);
  if (!b->plan || !kn || kn->dim() != 4) return none();
  const int64_t bsz = kn->size(0);
  c(args[4], b->dtype, {bsz, 1, b->hkv, b->d});
  const at::Tensor* vn = c(args[5], b->dtype, {bsz, 1, b->hkv, b->d});
  const at::Tensor* kc = c(args[1], b->dtype, {bsz, b->rows, b->d});
  const at::Tensor* vc = c(args[2], b->dtype, {bsz, b->rows, b->d});
  const at::Tensor* pc = c(args[3], at::kInt, {bsz, b->rows});
  const at::Tensor* ps = c(args[6], at::kInt, {bsz});
  if (!c.done() || bsz > INT32_MAX) return none();
  void *pkc = kc->data_ptr(), *pvc = vc->data_ptr(), *pkn = kn->data_ptr(), *pvn = vn->data_ptr(), *s = c.stream();
  int32_t* pp = static_cast<int32_t*>(pc->data_ptr());
  const int32_t* at_ = static_cast<const int32_t*>(ps->data_ptr());
  if (!call(*b, [&] { return b->api.kv_append_ragged(b->plan, pkc, pvc, pp, pkn, pvn, at_, static_cast<int32_t>(bsz), s); }))
    return nullptr;
  Py_RETURN_TRUE;
  MOA_LEAVE
}

// q, k_cache, v_cache of a decode call
struct DecodeTensors {
  const at::Tensor *q, *kc = nullptr, *vc = nullptr;
  int64_t bsz = 0;
  DecodeTensors(const Bound& b, PyObject* const* args, Check& c) : q(c.any(args[1])) {
    if (!b.plan || !q || q->dim() != 3) {
      c.ok = false;
      return;
    }
    bsz = q->size(0);
    c(args[1], b.dtype, {bsz, b.hq, b.d});
    kc = c(args[2], b.dtype, {bsz, b.rows, b.d});
    vc = c(args[3], b.dtype, {bsz, b.rows, b.d});
    if (bsz > INT32_MAX) c.ok = false;
  }
};

// decode(bound, q, k_cache, v_cache, pos, workspace, o)
PyObject* decode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  int64_t pos;
  if (!as_int(args[4], &pos)) return none();
  const DecodeTensors t(*b, args, c);
  const at::Tensor* w = c.any(args[5]);
  Out o(args[6], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *pk = t.kc->data_ptr(), *pv = t.vc->data_ptr(), *po = o.t->data_ptr();
  void *pw = w->data_ptr(), *s = c.stream();
  const size_t nw = w->nbytes();
  if (!call(*b, [&] { return b->api.decode(b->plan, pq, pk, pv, po, static_cast<int32_t>(t.bsz), pos, pw, nw, s); }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}

// decode_noalloc(bound, q, k_cache, v_cache, pos, o)
PyObject* decode_noalloc(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(6)
  int64_t pos;
  if (!as_int(args[4], &pos) || args[5] == Py_None) return none();
  const DecodeTensors t(*b, args, c);
  Out o(args[5], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *pk = t.kc->data_ptr(), *pv = t.vc->data_ptr(), *po = o.t->data_ptr(), *s = c.stream();
  if (!call(*b, [&] { return b->api.decode_noalloc(b->plan, pq, pk, pv, po, static_cast<int32_t>(t.bsz), pos, s); }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}

// decode_ragged(bound, q, k_cache, v_cache, positions, workspace, o)
PyObject* decode_ragged(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  const DecodeTensors t(*b, args, c);
  const at::Tensor* ps = c(args[4], at::kInt, {t.bsz});
  const at::Tensor* w = c.any(args[5]);
  Out o(args[6], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *pk = t.kc->data_ptr(), *pv = t.vc->data_ptr(), *po = o.t->data_ptr();
  void *pw = w->data_ptr(), *s = c.stream();
  const int32_t* at_ = static_cast<const int32_t*>(ps->data_ptr());
  const size_t nw = w->nbytes();
  if (!call(*b, [&] { return b->api.decode_ragged(b->plan, pq, pk, pv, po, at_, static_cast<int32_t>(t.bsz), pw, nw, s); }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}

// influence(bound, q, k, v, dout, ebar, softmax_scale)
PyObject* influence(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  const at::Tensor* q = c.any(args[1]);
  const at::Tensor* k = c.any(args[2]);
  if (!q || !k || q->dim() != 4 || k->dim() != 4 || !PyFloat_CheckExact(args[6])) return none();
  const int64_t bsz = q->size(0), n = q->size(1), hq = q->size(2), d = q->size(3), hkv = k->size(2);
  c(args[1], at::kBFloat16, {bsz, n, hq, d});
  c(args[2], at::kBFloat16, {bsz, n, hkv, d});
  const at::Tensor* v = c(args[3], at::kBFloat16, {bsz, n, hkv, d});
  const at::Tensor* g = c(args[4], at::kBFloat16, {bsz, n, hq, d});
  if (!c.done() || std::max({bsz, n, hq, hkv, d}) > INT32_MAX) return none();
  const int64_t nb = (n + 63) / 64;
  at::Tensor fresh;
  const at::Tensor* e = &fresh;
  if (args[5] == Py_None) fresh = at::empty({hq, nb, nb}, q->options().dtype(at::kFloat));
  else e = c(args[5], at::kFloat, {hq, nb, nb});
  if (!c.done()) return none();
  moa_desc_t desc = {};
  desc.num_q_heads = static_cast<int32_t>(hq);
  desc.num_kv_heads = static_cast<int32_t>(hkv);
  desc.head_dim = static_cast<int32_t>(d);
  desc.n = n;
  desc.dtype = MOA_BF16;
  desc.softmax_scale = static_cast<float>(PyFloat_AS_DOUBLE(args[6]));
  void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *pg = g->data_ptr(), *s = c.stream();
  float* pe = static_cast<float*>(e->data_ptr());
  if (!call(*b, [&] { return b->api.influence(&desc, pq, pk, pv, pg, pe, static_cast<int32_t>(bsz), n, s); })) return nullptr;
  return args[5] == Py_None ? THPVariable_Wrap(fresh) : same(args[5]);
  MOA_LEAVE
}

// A one-dimensional contiguous float64 buffer.
struct Doubles {
  Py_buffer v;
  bool held = false, ok = false;
  explicit Doubles(PyObject* o) {
    if (!PyObject_CheckBuffer(o)) return;
    held = PyObject_GetBuffer(o, &v, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) == 0;
    if (!held) PyErr_Clear();
    ok = held && v.ndim == 1 && v.itemsize == 8 && v.format && v.format[0] == 'd' && v.format[1] == 0 && v.len > 0;
  }
  ~Doubles() {
    if (held) PyBuffer_Release(&v);
  }
  Doubles(const Doubles&) = delete;
};

// rule_loss(bound, ebar, n, num_sink, alpha, beta, flags) -> (dl, density)
PyObject* rule_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(7)
  int64_t n, sink, flags;
  const at::Tensor* e = c.any(args[1]);
  if (!e || e->dim() != 3 || !as_int(args[2], &n) || !as_int(args[3], &sink) || !as_int(args[6], &flags)) return none();
  const int64_t h = e->size(0), nb = (n + 63) / 64;
  if (n < 1 || sink < 0 || sink > INT32_MAX || flags < 0 || flags > 3 || h > INT32_MAX) return none();
  c(args[1], at::kFloat, {h, nb, nb});
  const Doubles al(args[4]), be(args[5]);
  if (!al.ok || !be.ok || al.v.len != be.v.len || !c.done()) return none();
  const int64_t r = al.v.len / 8;
  if (r > INT32_MAX) return none();
  at::Tensor dl = at::empty({h, r}, e->options().dtype(at::kDouble));
  at::Tensor dens = at::empty({r}, e->options().dtype(at::kDouble));
  const float* pe = static_cast<const float*>(e->data_ptr());
  double *pd = static_cast<double*>(dl.data_ptr()), *pn = static_cast<double*>(dens.data_ptr());
  void* s = c.stream();
  if (!call(*b, [&] {
        return b->api.rule_loss(pe, static_cast<int32_t>(h), n, static_cast<int32_t>(sink), static_cast<uint32_t>(flags),
                                static_cast<const double*>(al.v.buf), static_cast<const double*>(be.v.buf),
                                static_cast<int32_t>(r), pd, pn, s);
      }))
    return nullptr;
  PyObject* pair = PyTuple_New(2);
  if (!pair) return nullptr;
  PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(dl));
  PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(dens));
  return pair;
  MOA_LEAVE
}

// k_pages, v_pages and table of a paged call of `bsz` sequences: of the plan's type, or, with scales, in 8 bits.
struct Pages {
  moa_pages_t p = {};
  float* scales = nullptr;
  moa_quant_pages_t quant() const {
    return {p.k_pages, p.v_pages, scales, p.table, p.num_pages, p.page_size, p.max_pages};
  }
};
Pages pages_of(const Bound& b, Check& c, PyObject* kp, PyObject* vp, PyObject* sc, PyObject* table, int64_t bsz) {
  Pages r;
  moa_pages_t& p = r.p;
  const at::Tensor* k = c.any(kp);
  const at::Tensor* t = c.any(table);
  if (!b.plan || !k || !t || k->dim() != 3 || t->dim() != 3) {
    c.ok = false;
    return r;
  }
  const int64_t np = k->size(0), ps = k->size(1), mp = t->size(2);
  const at::ScalarType type = sc ? at::kFloat8_e4m3fn : b.dtype;
  c(kp, type, {np, ps, b.d});
  const at::Tensor* v = c(vp, type, {np, ps, b.d});
  const at::Tensor* s = sc ? c(sc, at::kFloat, {np, ps / MOA_QUANT_BLOCK, 2}) : nullptr;
  c(table, at::kInt, {bsz, b.hkv, mp});
  if (!c.ok || ps > INT32_MAX || mp > INT32_MAX || bsz > INT32_MAX) {
    c.ok = false;
    return r;
  }
  p.k_pages = k->data_ptr();
  p.v_pages = v->data_ptr();
  if (s) r.scales = static_cast<float*>(s->data_ptr());
  p.table = static_cast<const int32_t*>(t->data_ptr());
  p.num_pages = np;
  p.page_size = static_cast<int32_t>(ps);
  p.max_pages = static_cast<int32_t>(mp);
  return r;
}

// (bound, k_pages, v_pages, [scales,] table, q, k_new, v_new, positions, seq_start, inv_freq, interleaved, q_out)
template <bool kQuant>
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(kQuant ? 13 : 12)
  PyObject* const sc = kQuant ? args[3] : nullptr;
  PyObject* const* a = args + (kQuant ? 4 : 3);           // from the table on
  const at::Tensor* at_ = c.any(a[4]);
  const at::Tensor* k0 = plain(a[2]);
  if (!b->plan || !at_ || at_->dim() != 1 || !k0 || k0->dim() != 3 || !PyBool_Check(a[7])) return none();
  const int64_t bsz = at_->size(0), n = k0->size(0);
  c(a[4], at::kInt, {bsz});
  const Pages pages = pages_of(*b, c, args[1], args[2], sc, a[0], bsz);
  int64_t qs = 0, ks = 0, vs = 0;
  const at::Tensor* k = c.tokens(a[2], b->dtype, {n, b->hkv, b->d}, &ks);
  const at::Tensor* v = c.tokens(a[3], b->dtype, {n, b->hkv, b->d}, &vs);
  const bool with_q = a[1] != Py_None;
  const at::Tensor* q = with_q ? c.tokens(a[1], b->dtype, {n, b->hq, b->d}, &qs) : nullptr;
  const at::Tensor* ss = a[5] != Py_None ? c(a[5], at::kInt, {bsz + 1}) : nullptr;
  const at::Tensor* f = a[6] != Py_None ? c.any(a[6]) : nullptr;
  if (!c.done() || (f && (f->dim() != 1 || f->scalar_type() != at::kFloat || f->size(0) > INT32_MAX / 2)))
    return none();
  at::Tensor fresh;
  const at::Tensor* out = &fresh;
  if (!with_q) {
    if (a[8] != Py_None) return none();
  } else if (a[8] == Py_None) {
    fresh = at::empty({n, b->hq, b->d}, q->options());
  } else {
    out = c(a[8], b->dtype, {n, b->hq, b->d});
  }
  if (!c.done()) return none();
  moa_rope_t rope = {};
  if (f) {
    rope.inv_freq = static_cast<const float*>(f->data_ptr());
    rope.rotary_dim = static_cast<int32_t>(2 * f->size(0));
    rope.interleaved = a[7] == Py_True;
  }
  void *pq = with_q ? q->data_ptr() : nullptr, *po = with_q ? out->data_ptr() : nullptr;
  void *pk = k->data_ptr(), *pv = v->data_ptr(), *s = c.stream();
  const int32_t* pp = static_cast<const int32_t*>(at_->data_ptr());
  const int32_t* ps = ss ? static_cast<const int32_t*>(ss->data_ptr()) : nullptr;
  const moa_quant_pages_t quant = pages.quant();
  if (!call(*b, [&] {
        const int32_t batch = static_cast<int32_t>(bsz);
        if constexpr (kQuant)
          return b->api.quant_append(b->plan, &quant, pq, qs, pk, ks, pv, vs, po, f ? &rope : nullptr, pp, ps, batch, n, s);
        else
          return b->api.paged_append(b->plan, &pages.p, pq, qs, pk, ks, pv, vs, po, f ? &rope : nullptr, pp, ps, batch, n, s);
      }))
    return nullptr;
  if (!with_q) Py_RETURN_TRUE;
  return a[8] == Py_None ? THPVariable_Wrap(fresh) : same(a[8]);
  MOA_LEAVE
}
constexpr auto paged_append = append<false>, quant_append = append<true>;

// q, pages, positions, workspace and o of a paged attention call
struct PagedTensors {
  const at::Tensor *q, *ps = nullptr, *w = nullptr;
  Pages pages;
  moa_quant_pages_t quant = {};
  int64_t n = 0, bsz = 0;
  // one_each: one token per sequence
  PagedTensors(const Bound& b, Check& c, PyObject* oq, PyObject* kp, PyObject* vp, PyObject* sc, PyObject* table,
               PyObject* pos, PyObject* work, bool one_each)
      : q(c.any(oq)) {
    ps = c.any(pos);
    if (!b.plan || !q || !ps || q->dim() != 3 || ps->dim() != 1) {
      c.ok = false;
      return;
    }
    n = q->size(0);
    bsz = ps->size(0);
    c(oq, b.dtype, {one_each ? bsz : n, b.hq, b.d});
    c(pos, at::kInt, {bsz});
    pages = pages_of(b, c, kp, vp, sc, table, bsz);
    quant = pages.quant();
    w = c.any(work);
  }
  const int32_t* positions() const { return static_cast<const int32_t*>(ps->data_ptr()); }
};

// (bound, q, k_pages, v_pages, [scales,] table, positions, seq_start, workspace, o)
template <bool kQuant>
PyObject* packed_prefill(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(kQuant ? 10 : 9)
  PyObject* const* a = args + (kQuant ? 5 : 4);           // from the table on
  const PagedTensors t(*b, c, args[1], args[2], args[3], kQuant ? args[4] : nullptr, a[0], a[1], a[3], false);
  const at::Tensor* ss = c(a[2], at::kInt, {t.bsz + 1});
  Out o(a[4], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *po = o.t->data_ptr(), *pw = t.w->data_ptr(), *s = c.stream();
  const int32_t* ps = static_cast<const int32_t*>(ss->data_ptr());
  const size_t nw = t.w->nbytes();
  if (!call(*b, [&] {
        const int32_t batch = static_cast<int32_t>(t.bsz);
        if constexpr (kQuant)
          return b->api.quant_prefill(b->plan, &t.quant, pq, po, t.positions(), ps, batch, t.n, pw, nw, s);
        else
          return b->api.paged_prefill(b->plan, &t.pages.p, pq, po, t.positions(), ps, batch, t.n, pw, nw, s);
      }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}
constexpr auto paged_prefill = packed_prefill<false>, quant_prefill = packed_prefill<true>;

// (bound, q, k_pages, v_pages, [scales,] table, positions, workspace, o)
template <bool kQuant>
PyObject* pages_decode(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(kQuant ? 9 : 8)
  PyObject* const* a = args + (kQuant ? 5 : 4);           // from the table on
  const PagedTensors t(*b, c, args[1], args[2], args[3], kQuant ? args[4] : nullptr, a[0], a[1], a[2], true);
  Out o(a[3], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *po = o.t->data_ptr(), *pw = t.w->data_ptr(), *s = c.stream();
  const size_t nw = t.w->nbytes();
  if (!call(*b, [&] {
        const int32_t batch = static_cast<int32_t>(t.bsz);
        if constexpr (kQuant) return b->api.quant_decode(b->plan, &t.quant, pq, po, t.positions(), batch, pw, nw, s);
        else return b->api.paged_decode(b->plan, &t.pages.p, pq, po, t.positions(), batch, pw, nw, s);
      }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}
constexpr auto paged_decode = pages_decode<false>, quant_decode = pages_decode<true>;

// (bound, q, k_pages, v_pages, [scales,] prefix_table, prefix_len, table, positions, workspace, o)
template <bool kQuant>
PyObject* pages_decode_shared(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(kQuant ? 11 : 10)
  PyObject* const* a = args + (kQuant ? 5 : 4);           // from the prefix's table on
  int64_t len;
  if (!as_int(a[1], &len)) return none();
  const PagedTensors t(*b, c, args[1], args[2], args[3], kQuant ? args[4] : nullptr, a[2], a[3], a[4], true);
  const at::Tensor* pre = c(a[0], at::kInt, {b->hkv, int64_t(t.pages.p.max_pages)});
  Out o(a[5], t.q, c);
  if (!c.done() || !o.t) return none();
  void *pq = t.q->data_ptr(), *po = o.t->data_ptr(), *pw = t.w->data_ptr(), *s = c.stream();
  const int32_t* pp = static_cast<const int32_t*>(pre->data_ptr());
  const size_t nw = t.w->nbytes();
  if (!call(*b, [&] {
        const int32_t batch = static_cast<int32_t>(t.bsz);
        if constexpr (kQuant)
          return b->api.quant_decode_shared(b->plan, &t.quant, pp, len, pq, po, t.positions(), batch, pw, nw, s);
        else
          return b->api.paged_decode_shared(b->plan, &t.pages.p, pp, len, pq, po, t.positions(), batch, pw, nw, s);
      }))
    return nullptr;
  return o.answer();
  MOA_LEAVE
}
constexpr auto paged_decode_shared = pages_decode_shared<false>, quant_decode_shared = pages_decode_shared<true>;

// (bound, table, free_pages, counts, page_size, positions, workspace, seq_start, fresh, slots[, scales, lacked, n_tokens])
template <bool kState>
PyObject* assign(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  MOA_ENTER(kState ? 13 : 10)
  int64_t page;
  const at::Tensor* t = c.any(args[1]);
  const at::Tensor* f = c.any(args[2]);
  const at::Tensor* ps = c.any(args[5]);
  if (!b->plan || !t || !f || !ps || t->dim() != 3 || f->dim() != 1 || ps->dim() != 1 || !as_int(args[4], &page) ||
      page < 0 || page > INT32_MAX)
    return none();
  const int64_t bsz = ps->size(0), mp = t->size(2);
  c(args[1], at::kInt, {bsz, b->hkv, mp});
  c(args[2], at::kInt, {f->size(0)});
  const at::Tensor* n2 = c(args[3], at::kInt, {2});
  c(args[5], at::kInt, {bsz});
  const at::Tensor* w = c.any(args[6]);
  const at::Tensor* ss = args[7] != Py_None ? c(args[7], at::kInt, {bsz + 1}) : nullptr;
  const at::Tensor* fr = args[8] != Py_None ? c(args[8], at::kInt, {bsz}) : nullptr;
  const at::Tensor* sl = args[9] != Py_None ? c.any(args[9]) : nullptr;
  if (sl && (sl->dim() != 2 || sl->scalar_type() != at::kInt || sl->size(1) != b->hkv || (!ss && sl->size(0) != bsz)))
    return none();
  const at::Tensor *sc = nullptr, *la = nullptr;
  int64_t n = sl ? sl->size(0) : (int64_t(1) << 30) - 1;
  if constexpr (kState) {
    if (args[12] != Py_None && (sl || !as_int(args[12], &n))) return none();
    la = args[11] != Py_None ? c(args[11], at::kInt, {bsz}) : nullptr;
    sc = args[10] != Py_None ? c.any(args[10]) : nullptr;
    if (sc && (sc->dim() != 3 || sc->scalar_type() != at::kFloat || sc->size(0) < f->size(0) ||
               sc->size(1) != page / MOA_QUANT_BLOCK || sc->size(2) != 2))
      return none();
  }
  if (!c.done() || bsz > INT32_MAX || mp > INT32_MAX) return none();
  auto at_ = [](const at::Tensor* x) { return x ? static_cast<int32_t*>(x->data_ptr()) : nullptr; };
  const moa_page_tables_t tables = {at_(t), at_(f), at_(n2), f->size(0), static_cast<int32_t>(page), static_cast<int32_t>(mp)};
  void *pw = w->data_ptr(), *s = c.stream();
  const size_t nw = w->nbytes();
  const int32_t *pp = at_(ps), *pss = at_(ss), *pf = at_(fr);
  int32_t* psl = at_(sl);
  const moa_page_state_t state = {sc ? static_cast<float*>(sc->data_ptr()) : nullptr, at_(la)};
  if (!call(*b, [&] {
        const int32_t batch = static_cast<int32_t>(bsz);
        if constexpr (kState)
          return b->api.paged_assign_state(b->plan, &tables, &state, pp, pss, pf, psl, batch, n, pw, nw, s);
        else
          return b->api.paged_assign(b->plan, &tables, pp, pss, pf, psl, batch, n, pw, nw, s);
      }))
    return nullptr;
  Py_RETURN_TRUE;
  MOA_LEAVE
}
constexpr auto paged_assign = assign<false>, paged_assign_state = assign<true>;

// bind(addresses of the entry points, plan address or 0, num_q_heads, num_kv_heads, head_dim, cache rows, is bf16,
//      function that raises for a status)
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *table, *check;
  unsigned long long plan;
  long long hq, hkv, d, rows;
  int bf16;
  if (!PyArg_ParseTuple(args, "O!KLLLLpO", &PyTuple_Type, &table, &plan, &hq, &hkv, &d, &rows, &bf16, &check))
    return nullptr;
  constexpr Py_ssize_t kEntries = sizeof(Api) / sizeof(void*);
  void* at_[kEntries];
  if (PyTuple_GET_SIZE(table) != kEntries) {
    PyErr_SetString(PyExc_ValueError, "entry point table of the wrong length");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < kEntries; ++i) {
    at_[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(table, i));
    if (!at_[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
      return nullptr;
    }
  }
  Bound* b = new (std::nothrow) Bound{};
  if (!b) return PyErr_NoMemory();
  memcpy(&b->api, at_, sizeof(b->api));
  b->plan = reinterpret_cast<const moa_plan_t*>(static_cast<uintptr_t>(plan));
  b->hq = hq;
  b->hkv = hkv;
  b->d = d;
  b->rows = rows;
  b->dtype = bf16 ? at::kBFloat16 : at::kFloat;
  b->check = same(check);
  PyObject* o = PyCapsule_New(b, kName, [](PyObject* x) { delete static_cast<Bound*>(PyCapsule_GetPointer(x, kName)); });
  if (!o) delete b;
  return o;
}

#define MOA_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    MOA_FAST(prefill), MOA_FAST(kv_append), MOA_FAST(kv_append_ragged), MOA_FAST(decode), MOA_FAST(decode_noalloc),
    MOA_FAST(decode_ragged), MOA_FAST(influence), MOA_FAST(rule_loss), MOA_FAST(paged_append), MOA_FAST(paged_prefill),
    MOA_FAST(paged_decode), MOA_FAST(paged_decode_shared), MOA_FAST(paged_assign), MOA_FAST(quant_append),
    MOA_FAST(quant_prefill), MOA_FAST(quant_decode), MOA_FAST(quant_decode_shared), MOA_FAST(paged_assign_state),
    {"bind", bind, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&kModule); }
