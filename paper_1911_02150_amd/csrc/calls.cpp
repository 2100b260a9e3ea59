// The calls of a decoding loop from Python without the interpreter's share of them: checks of the tensors, their addresses,
// the current stream and the call into libmqa_decode.so in one native function each (a CPython extension over torch's own tensor
// type).  They take what the binding's general path takes in its plainest form only, torch tensors on the current GPU, contiguous, of the
// right types and shapes, with no mode of torch active; for anything else they return None, nothing has happened, and the general path accepts it or says
// what is wrong.
// Measured (us a call among others, general path through ctypes / here; GPU alone, from a graph): one attention 7.1 / 4.5 (4.3), a layer's
// three calls 21.7 / 17.3 (16.9), a memory and its step 15.3 / 9.4 (9.0), a beam step and its reorder 18.8 / 12.7 (11.5).  The launch
// itself is 3.2 of a call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mqa.h"

namespace {

// Addresses of the library's functions (binding.py loads the library and hands them over), and the error to raise.
struct Functions {
  decltype(&mqa_decode_step) mqa_decode, mha_decode;
  decltype(&mqa_decode_step_window) mqa_window, mha_window;
  decltype(&mqa_project_append_qkv) append_qkv;
  decltype(&mqa_project_qkvo_ex) project;
  decltype(&mqa_project_add_layernorm) add_layernorm;
  decltype(&mqa_project_memory_kv) memory_kv;
  decltype(&mqa_project_memory_kv_ws) memory_kv_ws;
  decltype(&mqa_memory_decode_step) memory_decode;
  decltype(&mqa_decode_step_beams) beams;
  decltype(&mqa_beam_reorder_kv) reorder;
  decltype(&mqa_prefill_attention) mqa_prefill, mha_prefill;
  decltype(&mqa_paged_append_kv_rows) paged_append;
  decltype(&mqa_paged_decode_workspace_bytes) paged_workspace;
  decltype(&mqa_paged_decode_step) paged_decode;
  decltype(&mqa_paged_evict_kv) paged_evict;
  decltype(&mqa_stack_verify_workspace_bytes) verify_workspace;
  decltype(&mqa_stack_verify_drafts) verify;
  decltype(&mqa_paged_scaled_append_kv_rows) scaled_append;
  decltype(&mqa_paged_scaled_decode_workspace_bytes) scaled_workspace;
  decltype(&mqa_paged_scaled_decode_step) scaled_decode;
  decltype(&mqa_paged_fork_pages) fork_pages;
  decltype(&mqa_paged_free_pages) free_pages;
  decltype(&mqa_paged_reserve_workspace_bytes) reserve_workspace;
  decltype(&mqa_paged_reserve_pages) reserve_pages;
  decltype(&mqa_paged_compact_workspace_bytes) compact_workspace;
  decltype(&mqa_paged_compact_pages) compact_pages;
  decltype(&mqa_paged_copy_pages) copy_pages;
  decltype(&mqa_stack_adjust_logits) adjust_logits;
} fn;
PyObject* error_class = nullptr;
PyObject* parameter_class = nullptr;

const uint64_t kPlainKeys = (c10::DispatchKeySet(c10::DispatchKey::CUDA) | c10::DispatchKeySet(c10::DispatchKey::AutogradCUDA) |
                             c10::DispatchKeySet(c10::DispatchKey::ADInplaceOrView) | c10::DispatchKeySet(c10::DispatchKey::AutocastCUDA)).raw_repr();

// Nobody looks on: the output is made without a word to a function mode or a dispatch mode.
bool no_modes() { return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set(); }

thread_local c10::DeviceIndex device = 0;      // the current one, of a call

// A tensor that is no more than memory on that GPU (no subclass, no wrapper of a transform), contiguous, of this type; else null.
const at::Tensor* plain(PyObject* o) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != THPVariableClass && reinterpret_cast<PyObject*>(Py_TYPE(o)) != parameter_class) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || (t.unsafeGetTensorImpl()->key_set().raw_repr() & ~kPlainKeys) || !t.is_cuda() || t.device().index() != device || !t.is_contiguous()) return nullptr;
  return &t;
}
const at::Tensor* plain(PyObject* o, at::ScalarType type) {
  const at::Tensor* t = plain(o);
  return t && t->scalar_type() == type ? t : nullptr;
}
const at::Tensor* f32(PyObject* o) { return plain(o, at::kFloat); }
const at::Tensor* i32(PyObject* o) { return plain(o, at::kInt); }

bool shape_is(const at::Tensor& t, std::initializer_list<int64_t> s) { return t.sizes() == at::IntArrayRef(s); }
bool fits(const at::Tensor& t) {               // sizes as the library's ints
  for (int64_t s : t.sizes())
    if (s > INT32_MAX) return false;
  return true;
}
int cache_type(const at::Tensor& K) { return K.scalar_type() == at::kBFloat16 ? MQA_BF16 : K.scalar_type() == at::kFloat ? MQA_F32 : -1; }
size_t bytes_of(const at::Tensor& t) { return (size_t)t.numel() * t.element_size(); }
void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }      // (of the current device)

template <typename T> T* at_of(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

// The output: the caller's, or a new one of this shape like `like`.  Returns a new reference, or null.
PyObject* output(PyObject* given, const at::Tensor& like, std::initializer_list<int64_t> shape, const at::Tensor** t, at::Tensor* own) {
  if (given == Py_None) {
    *own = at::empty(at::IntArrayRef(shape), like.options().requires_grad(false));
    *t = own;
    return THPVariable_Wrap(*own);
  }
  *t = f32(given);
  if (!*t || !shape_is(**t, shape)) return nullptr;
  Py_INCREF(given);
  return given;
}

PyObject* result(int status, const char* name, PyObject* value) {
  if (status == MQA_OK) return value;
  Py_DECREF(value);
  PyObject* e = PyObject_CallFunction(error_class, "si", name, status);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return nullptr;
}

struct Held {                                  // a reference that goes with an exception
  PyObject* p;
  ~Held() { Py_XDECREF(p); }
  PyObject* take() { PyObject* const q = p; p = nullptr; return q; }
};

#define NOT_HERE return PyErr_Occurred() ? nullptr : (Py_INCREF(Py_None), Py_None)
// C++ exceptions (an allocation that fails, memory that a tensor does not have) stay here: the general path meets them again
#define MQA_CALL(NAME, COUNT)                                                             \
  PyObject* NAME##_body(PyObject* const* a);                                              \
  PyObject* NAME(PyObject*, PyObject* const* a, Py_ssize_t n) {                           \
    if (n != COUNT) { PyErr_SetString(PyExc_TypeError, #NAME ": " #COUNT " arguments"); return nullptr; } \
    try { if (!no_modes()) NOT_HERE; device = c10::hip::current_device(); return NAME##_body(a); } catch (const std::exception&) { NOT_HERE; }            \
  }                                                                                       \
  PyObject* NAME##_body(PyObject* const* a)
#define WITHOUT_GIL(EXPR) [&] { int rc_; Py_BEGIN_ALLOW_THREADS rc_ = (EXPR); Py_END_ALLOW_THREADS return rc_; }()

bool number(PyObject* o, float* x) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  *x = (float)v;
  return true;
}
bool integer(PyObject* o, int* x) {
  if (!PyLong_Check(o)) return false;
  const long v = PyLong_AsLong(o);
  if ((v == -1 && PyErr_Occurred()) || v < INT32_MIN || v > INT32_MAX) { PyErr_Clear(); return false; }
  *x = (int)v;
  return true;
}

// (multi_head, q, K, V, lens, o, scale, workspace, window or None)
MQA_CALL(decode, 9) {
  const bool mh = a[0] == Py_True;
  const at::Tensor *q = f32(a[1]), *K = plain(a[2]), *V = plain(a[3]), *lens = i32(a[4]), *ws = plain(a[7]), *o;
  float scale;
  int window = 0;
  if (!q || !K || !V || !lens || !ws || q->dim() != 3 || V->dim() < 2 || !number(a[6], &scale) || (a[8] != Py_None && !integer(a[8], &window))) NOT_HERE;
  const int64_t b = q->size(0), h = q->size(1), k = q->size(2), cap = V->size(-2), v = V->size(-1);
  const int dt = cache_type(*K);
  if (dt < 0 || K->scalar_type() != V->scalar_type() || lens->numel() != b || !fits(*q) || !fits(*V) ||
      !(mh ? shape_is(*K, {b, h, cap, k}) && shape_is(*V, {b, h, cap, v}) : shape_is(*K, {b, cap, k}) && shape_is(*V, {b, cap, v})))
    NOT_HERE;
  at::Tensor own;
  Held out{output(a[5], *q, {b, h, v}, &o, &own)};
  if (!out.p) NOT_HERE;
  const float *qp = at_of<float>(q);
  const void *Kp = K->data_ptr(), *Vp = V->data_ptr();
  const int32_t* lp = at_of<int32_t>(lens);
  float* op = at_of<float>(o);
  void *wp = ws->data_ptr(), *st = current_stream();
  const size_t nbytes = bytes_of(*ws);
  if (a[8] == Py_None)
    return result(WITHOUT_GIL((mh ? fn.mha_decode : fn.mqa_decode)(qp, Kp, Vp, lp, op, b, h, cap, k, v, (mqa_dtype)dt, scale, wp, nbytes, st)),
                  mh ? "mha_decode_step" : "mqa_decode_step", out.take());
  return result(WITHOUT_GIL((mh ? fn.mha_window : fn.mqa_window)(qp, Kp, Vp, lp, op, b, h, cap, k, v, (mqa_dtype)dt, scale, window, wp, nbytes, st)),
                mh ? "mha_decode_step_window" : "mqa_decode_step_window", out.take());
}

// (x, P_q, P_k, P_v, K, V, lens_in, lens_out, q)
MQA_CALL(append_qkv, 9) {
  const at::Tensor *x = f32(a[0]), *Pq = f32(a[1]), *Pk = f32(a[2]), *Pv = f32(a[3]), *K = plain(a[4]), *V = plain(a[5]), *in = i32(a[6]), *out = i32(a[7]), *q;
  if (!x || !Pq || !Pk || !Pv || !K || !V || !in || !out || x->dim() != 2 || Pq->dim() != 3 || Pk->dim() < 2 || Pk->dim() > 3 || Pv->dim() != Pk->dim() ||
      K->dim() < 2)
    NOT_HERE;
  const int64_t b = x->size(0), d = x->size(1), h = Pq->size(0), k = Pq->size(2), v = Pv->size(-1), cap = K->size(-2);
  const bool one = Pk->dim() == 2;
  const int64_t h_kv = one ? 1 : Pk->size(0);
  const int dt = cache_type(*K);
  if (dt < 0 || K->scalar_type() != V->scalar_type() || Pq->size(1) != d || Pk->size(-2) != d || Pk->size(-1) != k || Pv->size(-2) != d ||
      (!one && Pv->size(0) != h_kv) || in->numel() != b || out->numel() != b || !fits(*x) || !fits(*Pq) || !fits(*Pv) || !fits(*K) ||
      !(one ? shape_is(*K, {b, cap, k}) && shape_is(*V, {b, cap, v}) : shape_is(*K, {b, h_kv, cap, k}) && shape_is(*V, {b, h_kv, cap, v})))
    NOT_HERE;
  at::Tensor own;
  Held res{output(a[8], *x, {b, h, k}, &q, &own)};
  if (!res.p) NOT_HERE;
  const float *xp = at_of<float>(x), *Pqp = at_of<float>(Pq), *Pkp = at_of<float>(Pk), *Pvp = at_of<float>(Pv);
  float* qp = at_of<float>(q);
  void *Kp = K->data_ptr(), *Vp = V->data_ptr(), *st = current_stream();
  int32_t *ip = at_of<int32_t>(in), *lp = at_of<int32_t>(out);
  return result(WITHOUT_GIL(fn.append_qkv(xp, Pqp, Pkp, Pvp, qp, Kp, Vp, ip, lp, b, d, h, h_kv, cap, k, v, (mqa_dtype)dt, st)), "mqa_project_append_qkv", res.take());
}

// The sizes of a projection; false: not these
struct Product { int64_t rows, d, h, kv; };
bool product_of(int mode, const at::Tensor& x, const at::Tensor& P, Product* s) {
  const bool two = mode == MQA_PROJ_KV || mode == MQA_PROJ_LINEAR;
  if (mode < 0 || mode > 4 || P.dim() != (two ? 2 : 3) || x.dim() != (mode == MQA_PROJ_O ? 3 : 2) || !fits(x) || !fits(P)) return false;
  *s = Product{x.size(0), P.size(-2), two ? 1 : P.size(0), P.size(-1)};
  return mode == MQA_PROJ_O ? x.size(1) == s->h && x.size(2) == s->kv : x.size(1) == s->d;
}

// (mode, x, P, out, epilogue or None)
MQA_CALL(project, 5) {
  int mode, epilogue = MQA_EPI_STORE;
  const at::Tensor *x = f32(a[1]), *P = f32(a[2]), *out;
  Product s;
  if (!x || !P || !integer(a[0], &mode) || (a[4] != Py_None && !integer(a[4], &epilogue)) || !product_of(mode, *x, *P, &s) || (epilogue == MQA_EPI_ADD && a[3] == Py_None)) NOT_HERE;
  at::Tensor own;
  Held res{mode == MQA_PROJ_O ? output(a[3], *x, {s.rows, s.d}, &out, &own)
                              : mode == MQA_PROJ_Q || mode == MQA_PROJ_KV_MH ? output(a[3], *x, {s.rows, s.h, s.kv}, &out, &own)
                                                                             : output(a[3], *x, {s.rows, s.kv}, &out, &own)};
  if (!res.p) NOT_HERE;
  const float *xp = at_of<float>(x), *Pp = at_of<float>(P);
  float* op = at_of<float>(out);
  void* st = current_stream();
  return result(WITHOUT_GIL(fn.project((mqa_proj_mode)mode, xp, Pp, op, s.rows, s.d, s.h, s.kv, (mqa_proj_epilogue)epilogue, st)),
                a[4] == Py_None ? "mqa_project_qkvo" : "mqa_project_qkvo_ex", res.take());
}

// (mode, x, P, acc, out, eps, workspace)
MQA_CALL(add_layernorm, 7) {
  int mode;
  float eps;
  const at::Tensor *x = f32(a[1]), *P = f32(a[2]), *acc = f32(a[3]), *ws = plain(a[6]), *out;
  Product s;
  if (!x || !P || !acc || !ws || !integer(a[0], &mode) || (mode != MQA_PROJ_O && mode != MQA_PROJ_LINEAR) || !number(a[5], &eps) || !product_of(mode, *x, *P, &s) ||
      !shape_is(*acc, {s.rows, mode == MQA_PROJ_O ? s.d : s.kv}))
    NOT_HERE;
  at::Tensor own;
  Held res{output(a[4], *acc, {acc->size(0), acc->size(1)}, &out, &own)};
  if (!res.p) NOT_HERE;
  const float *xp = at_of<float>(x), *Pp = at_of<float>(P);
  float *ap = at_of<float>(acc), *op = at_of<float>(out);
  void *wp = ws->data_ptr(), *st = current_stream();
  const size_t nbytes = bytes_of(*ws);
  return result(WITHOUT_GIL(fn.add_layernorm((mqa_proj_mode)mode, xp, Pp, ap, op, s.rows, s.d, s.h, s.kv, eps, wp, nbytes, st)), "mqa_project_add_layernorm", res.take());
}

// (M, P_k, P_v, K, V, lens, mem_lens, workspace, products from which a call asks for a workspace)
MQA_CALL(memory_kv, 9) {
  const at::Tensor *M = f32(a[0]), *Pk = f32(a[1]), *Pv = f32(a[2]), *K = plain(a[3]), *V = plain(a[4]), *lens = i32(a[5]);
  const at::Tensor *valid = a[6] == Py_None ? nullptr : i32(a[6]), *ws = a[7] == Py_None ? nullptr : plain(a[7]);
  if (!M || !Pk || !Pv || !K || !V || !lens || (a[6] != Py_None && !valid) || (a[7] != Py_None && !ws) || M->dim() != 3 || Pk->dim() < 2 || Pk->dim() > 3 ||
      Pv->dim() != Pk->dim() || K->dim() != Pk->dim() + 1)
    NOT_HERE;
  const int64_t b = M->size(0), m = M->size(1), d = M->size(2), k = Pk->size(-1), v = Pv->size(-1), cap = K->size(-2);
  const bool one = Pk->dim() == 2;
  const int64_t h_kv = one ? 1 : Pk->size(0);
  const int dt = cache_type(*K);
  int small;
  if (!integer(a[8], &small) || (!ws && (double)b * m * d * h_kv * (k + v) >= small)) NOT_HERE;
  if (dt < 0 || K->scalar_type() != V->scalar_type() || Pk->size(-2) != d || Pv->size(-2) != d || (!one && Pv->size(0) != h_kv) || lens->numel() != b ||
      (valid && valid->numel() != b) || !fits(*M) || !fits(*Pk) || !fits(*Pv) || !fits(*K) ||
      !(one ? shape_is(*K, {b, cap, k}) && shape_is(*V, {b, cap, v}) : shape_is(*K, {b, h_kv, cap, k}) && shape_is(*V, {b, h_kv, cap, v})))
    NOT_HERE;
  const float *Mp = at_of<float>(M), *Pkp = at_of<float>(Pk), *Pvp = at_of<float>(Pv);
  void *Kp = K->data_ptr(), *Vp = V->data_ptr(), *wp = at_of<void>(ws), *st = current_stream();
  int32_t *vp = at_of<int32_t>(valid), *lp = at_of<int32_t>(lens);
  const size_t nbytes = ws ? bytes_of(*ws) : 0;
  Py_INCREF(Py_True);
  return result(WITHOUT_GIL(ws ? fn.memory_kv_ws(Mp, Pkp, Pvp, Kp, Vp, vp, lp, b, m, d, h_kv, cap, k, v, (mqa_dtype)dt, wp, nbytes, st)
                               : fn.memory_kv(Mp, Pkp, Pvp, Kp, Vp, vp, lp, b, m, d, h_kv, cap, k, v, (mqa_dtype)dt, st)),
                "mqa_project_memory_kv", Py_True);
}

// (which: 0 a memory's step, q [b,queries,h,k]; 1 a prompt, q [b,n,h,k]; 2 a multi-head one, q [b,h,n,k]; q, K, V, lens, o, scale, workspace)
MQA_CALL(attend_rows, 8) {
  int which;
  float scale;
  const at::Tensor *q = f32(a[1]), *K = plain(a[2]), *V = plain(a[3]), *lens = i32(a[4]), *ws = plain(a[7]), *o;
  if (!q || !K || !V || !lens || !ws || q->dim() != 4 || V->dim() < 2 || !integer(a[0], &which) || !number(a[6], &scale)) NOT_HERE;
  const bool mh = which == 2;
  const int64_t b = q->size(0), n = q->size(mh ? 2 : 1), h = q->size(mh ? 1 : 2), k = q->size(3), cap = V->size(-2), v = V->size(-1);
  const int dt = cache_type(*K);
  if (dt < 0 || K->scalar_type() != V->scalar_type() || lens->numel() != b || !fits(*q) || !fits(*V) ||
      !(mh ? shape_is(*K, {b, h, cap, k}) && shape_is(*V, {b, h, cap, v}) : shape_is(*K, {b, cap, k}) && shape_is(*V, {b, cap, v})))
    NOT_HERE;
  at::Tensor own;
  Held out{output(a[5], *q, {b, q->size(1), q->size(2), v}, &o, &own)};
  if (!out.p) NOT_HERE;
  const float* qp = at_of<float>(q);
  const void *Kp = K->data_ptr(), *Vp = V->data_ptr();
  const int32_t* lp = at_of<int32_t>(lens);
  float* op = at_of<float>(o);
  void *wp = ws->data_ptr(), *st = current_stream();
  const size_t nbytes = bytes_of(*ws);
  static const char* const names[] = {"mqa_memory_decode_step", "mqa_prefill_attention", "mha_prefill_attention"};
  const auto call = which == 0 ? fn.memory_decode : which == 1 ? fn.mqa_prefill : fn.mha_prefill;
  return result(WITHOUT_GIL(call(qp, Kp, Vp, lp, op, b, n, h, cap, k, v, (mqa_dtype)dt, scale, wp, nbytes, st)), names[which], out.take());
}

// (q, K_src, V_src, lens_src, K_own, V_own, lens_own, o, scale, workspace)
MQA_CALL(beams, 10) {
  float scale;
  const at::Tensor *q = f32(a[0]), *Ks = plain(a[1]), *Vs = plain(a[2]), *ls = i32(a[3]), *Ko = plain(a[4]), *Vo = plain(a[5]), *lo = i32(a[6]), *ws = plain(a[9]), *o;
  if (!q || !Ks || !Vs || !ls || !Ko || !Vo || !lo || !ws || q->dim() != 4 || Vs->dim() != 3 || Vo->dim() != 4 || !number(a[8], &scale)) NOT_HERE;
  const int64_t b = q->size(0), e = q->size(1), h = q->size(2), k = q->size(3), cs = Vs->size(1), co = Vo->size(2), v = Vs->size(2);
  const int dt = cache_type(*Ks);
  if (dt < 0 || Ks->scalar_type() != Ko->scalar_type() || Ks->scalar_type() != Vs->scalar_type() || Ks->scalar_type() != Vo->scalar_type() ||
      !shape_is(*Ks, {b, cs, k}) || !shape_is(*Vs, {b, cs, v}) || !shape_is(*Ko, {b, e, co, k}) || !shape_is(*Vo, {b, e, co, v}) || ls->numel() != b ||
      lo->numel() != b * e || !fits(*q) || !fits(*Vs) || !fits(*Vo))
    NOT_HERE;
  at::Tensor own;
  Held out{output(a[7], *q, {b, e, h, v}, &o, &own)};
  if (!out.p) NOT_HERE;
  const float* qp = at_of<float>(q);
  const void *Ksp = Ks->data_ptr(), *Vsp = Vs->data_ptr(), *Kop = Ko->data_ptr(), *Vop = Vo->data_ptr();
  const int32_t *lsp = at_of<int32_t>(ls), *lop = at_of<int32_t>(lo);
  float* op = at_of<float>(o);
  void *wp = ws->data_ptr(), *st = current_stream();
  const size_t nbytes = bytes_of(*ws);
  return result(WITHOUT_GIL(fn.beams(qp, Ksp, Vsp, lsp, Kop, Vop, lop, op, b, e, h, cs, co, k, v, (mqa_dtype)dt, scale, wp, nbytes, st)), "mqa_decode_step_beams", out.take());
}

// (K_src, V_src, lens_src, parent, K_dst, V_dst, lens_dst)
MQA_CALL(reorder, 7) {
  const at::Tensor *Ks = plain(a[0]), *Vs = plain(a[1]), *ls = i32(a[2]), *parent = i32(a[3]), *Kd = plain(a[4]), *Vd = plain(a[5]), *ld = i32(a[6]);
  if (!Ks || !Vs || !ls || !parent || !Kd || !Vd || !ld || Ks->dim() < 3 || Ks->dim() > 4 || Vs->dim() != Ks->dim()) NOT_HERE;
  const int64_t n = Ks->size(0), cap = Ks->size(-2), k = Ks->size(-1), v = Vs->size(-1), h_kv = Ks->dim() == 4 ? Ks->size(1) : 1;
  const int dt = cache_type(*Ks);
  if (dt < 0 || Vs->scalar_type() != Ks->scalar_type() || Kd->scalar_type() != Ks->scalar_type() || Vd->scalar_type() != Ks->scalar_type() ||
      Kd->sizes() != Ks->sizes() || Vd->sizes() != Vs->sizes() || Vs->sizes().slice(0, Vs->dim() - 1) != Ks->sizes().slice(0, Ks->dim() - 1) ||
      ls->numel() != n || parent->numel() != n || ld->numel() != n || !fits(*Ks) || !fits(*Vs))
    NOT_HERE;
  const void *Ksp = Ks->data_ptr(), *Vsp = Vs->data_ptr();
  void *Kdp = Kd->data_ptr(), *Vdp = Vd->data_ptr(), *st = current_stream();
  const int32_t *lsp = at_of<int32_t>(ls), *pp = at_of<int32_t>(parent);
  int32_t* ldp = at_of<int32_t>(ld);
  Py_INCREF(Py_True);
  return result(WITHOUT_GIL(fn.reorder(Ksp, Vsp, lsp, pp, Kdp, Vdp, ldp, n, h_kv, cap, k, v, (mqa_dtype)dt, st)), "mqa_beam_reorder_kv", Py_True);
}

// A tensor of this type or None; false: neither.
bool maybe(PyObject* o, at::ScalarType type, const at::Tensor** t) {
  *t = nullptr;
  return o == Py_None || (*t = plain(o, type)) != nullptr;
}

// The sizes of a paged cache; false: not these
struct Paged { int64_t h_kv, pages, size, each, k, v; int dt; };
bool paged_of(const at::Tensor* K, const at::Tensor* V, const at::Tensor* table, int64_t b, Paged* c) {
  if (!K || !V || !table || K->dim() < 3 || K->dim() > 4 || V->dim() != K->dim() || table->dim() != 2 || table->size(0) != b || V->scalar_type() != K->scalar_type() ||
      V->sizes().slice(0, V->dim() - 1) != K->sizes().slice(0, K->dim() - 1) || !fits(*K) || !fits(*V) || !fits(*table))
    return false;
  *c = Paged{K->dim() == 4 ? K->size(1) : 1, K->size(0), K->size(-2), table->size(1), K->size(-1), V->size(-1), cache_type(*K)};
  return c->dt >= 0 && c->size > 0;
}
// [b, (h_kv,) last], as the cache has its heads
bool per_head(const at::Tensor& t, const at::Tensor& K, int64_t b, int64_t last) {
  return K.dim() == 4 ? shape_is(t, {b, K.size(1), last}) : shape_is(t, {b, last});
}

// Scratch memory for a call: the caller's (held until the call has been made), or a block of the allocator, the current stream's.  false: the general path's matter
// (a stream that is captured, another kind of memory).
struct Scratch { at::Tensor own; void* at = nullptr; size_t bytes = 0; };
bool scratch(PyObject* given, size_t need, const at::Tensor& like, Scratch* s) {
  if (given != Py_None) {
    const at::Tensor* t = plain(given);
    if (!t) return false;
    s->at = t->data_ptr();
    s->bytes = bytes_of(*t);
    return true;
  }
  if (need == 0) return true;
  if (c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) return false;
  s->own = at::empty({(int64_t)need}, like.options().dtype(at::kByte).requires_grad(false));
  s->at = s->own.data_ptr();
  s->bytes = need;
  return true;
}

// (K_pages, V_pages, table, k_new, v_new, lens, lens_out, counts)
MQA_CALL(paged_append, 8) {
  const at::Tensor *K = plain(a[0]), *V = plain(a[1]), *table = i32(a[2]), *kn = f32(a[3]), *vn = f32(a[4]), *lens = i32(a[5]), *out = i32(a[6]), *counts;
  Paged c;
  if (!kn || !vn || !lens || !out || !maybe(a[7], at::kInt, &counts) || kn->dim() < 3 || !fits(*kn) || !paged_of(K, V, table, kn->size(0), &c)) NOT_HERE;
  const int64_t b = kn->size(0), n = kn->size(1);
  if (!(K->dim() == 4 ? shape_is(*kn, {b, n, c.h_kv, c.k}) && shape_is(*vn, {b, n, c.h_kv, c.v}) : shape_is(*kn, {b, n, c.k}) && shape_is(*vn, {b, n, c.v})) ||
      lens->numel() != b || out->numel() != b || (counts && counts->numel() != b))
    NOT_HERE;
  const float *kp = at_of<float>(kn), *vp = at_of<float>(vn);
  const int32_t *cp = at_of<int32_t>(counts), *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens);
  int32_t* op = at_of<int32_t>(out);
  void *Kp = K->data_ptr(), *Vp = V->data_ptr(), *st = current_stream();
  Py_INCREF(a[6]);
  return result(WITHOUT_GIL(fn.paged_append(kp, vp, cp, Kp, Vp, tp, lp, op, b, n, c.h_kv, c.pages, c.size, c.each, c.k, c.v, (mqa_dtype)c.dt, st)),
                "mqa_paged_append_kv_rows", a[6]);
}

// (q, K_pages, V_pages, table, lens, o, scale, scores, scores_out, workspace)
MQA_CALL(paged_decode, 10) {
  const at::Tensor *q = f32(a[0]), *K = plain(a[1]), *V = plain(a[2]), *table = i32(a[3]), *lens = i32(a[4]), *in, *out, *o;
  float scale;
  Paged c;
  if (!q || !lens || q->dim() < 3 || q->dim() > 4 || !fits(*q) || !number(a[6], &scale) || !maybe(a[7], at::kFloat, &in) || !maybe(a[8], at::kFloat, &out) ||
      !paged_of(K, V, table, q->size(0), &c))
    NOT_HERE;
  const int64_t b = q->size(0), n = q->dim() == 4 ? q->size(1) : 1, h = q->size(-2);
  if (!out) out = in;
  if (q->size(-1) != c.k || lens->numel() != b || c.each > INT32_MAX / c.size || (in && !per_head(*in, *K, b, c.each * c.size)) ||
      (out && !per_head(*out, *K, b, c.each * c.size)))
    NOT_HERE;
  at::Tensor own;
  Held res{q->dim() == 4 ? output(a[5], *q, {b, n, h, c.v}, &o, &own) : output(a[5], *q, {b, h, c.v}, &o, &own)};
  if (!res.p) NOT_HERE;
  Scratch ws;
  if (!scratch(a[9], a[9] == Py_None ? fn.paged_workspace(b, n, h, c.h_kv, c.size, c.each, c.k, c.v, (mqa_dtype)c.dt, out != nullptr) : 0, *q, &ws)) NOT_HERE;
  const float *qp = at_of<float>(q), *ip = at_of<float>(in);
  float *op = at_of<float>(o), *sp = at_of<float>(out);
  const int32_t *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens);
  const void *Kp = K->data_ptr(), *Vp = V->data_ptr();
  void* st = current_stream();
  return result(WITHOUT_GIL(fn.paged_decode(qp, Kp, Vp, tp, lp, op, ip, sp, b, n, h, c.h_kv, c.pages, c.size, c.each, c.k, c.v, (mqa_dtype)c.dt, scale, ws.at, ws.bytes, st)),
                "mqa_paged_decode_step", res.take());
}

// (K_pages, V_pages, table, lens, scores, table_out, lens_out, scores_out, kept, recent)
MQA_CALL(paged_evict, 10) {
  const at::Tensor *K = plain(a[0]), *V = plain(a[1]), *table = i32(a[2]), *lens = i32(a[3]), *scores = f32(a[4]), *table_out = i32(a[5]), *lens_out = i32(a[6]),
                   *scores_out = f32(a[7]), *kept = i32(a[8]);
  int recent;
  Paged c, d;
  if (!lens || !scores || !lens_out || !scores_out || !kept || kept->dim() < 1 || !fits(*kept) || !integer(a[9], &recent) || !paged_of(K, V, table, lens->numel(), &c) ||
      !paged_of(K, V, table_out, lens->numel(), &d))
    NOT_HERE;
  const int64_t b = lens->numel(), budget = kept->size(-1);
  if (c.each > INT32_MAX / c.size || d.each > INT32_MAX / c.size || !per_head(*scores, *K, b, c.each * c.size) || !per_head(*scores_out, *K, b, d.each * c.size) ||
      !per_head(*kept, *K, b, budget) || lens_out->numel() != b)
    NOT_HERE;
  void *Kp = K->data_ptr(), *Vp = V->data_ptr(), *st = current_stream();
  const int32_t *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens), *up = at_of<int32_t>(table_out);
  const float* sp = at_of<float>(scores);
  int32_t *mp = at_of<int32_t>(lens_out), *kp = at_of<int32_t>(kept);
  float* rp = at_of<float>(scores_out);
  Py_INCREF(a[8]);
  return result(WITHOUT_GIL(fn.paged_evict(Kp, Vp, tp, lp, sp, up, mp, rp, kp, b, c.h_kv, c.pages, c.size, c.each, d.each, c.k, c.v, (mqa_dtype)c.dt, budget, recent, st)),
                "mqa_paged_evict_kv", a[8]);
}

// (logits, drafts, u, draft_logits, counts, temperature, tokens, accepted, workspace)
MQA_CALL(verify, 9) {
  const at::Tensor *logits = f32(a[0]), *drafts, *u, *draft_logits, *counts, *tokens, *accepted;
  float temperature;
  if (!logits || logits->dim() != 3 || !fits(*logits) || !maybe(a[1], at::kInt, &drafts) || !maybe(a[2], at::kFloat, &u) || !maybe(a[3], at::kFloat, &draft_logits) ||
      !maybe(a[4], at::kInt, &counts) || !number(a[5], &temperature) || !maybe(a[6], at::kInt, &tokens) || !maybe(a[7], at::kInt, &accepted))
    NOT_HERE;
  const int64_t b = logits->size(0), n = logits->size(1) - 1, vocab = logits->size(2);
  if (n < 0 || (drafts && !shape_is(*drafts, {b, n})) || (u && !shape_is(*u, {b, n + 1})) || (draft_logits && !shape_is(*draft_logits, {b, n, vocab})) ||
      (counts && !shape_is(*counts, {b})) || (tokens && !shape_is(*tokens, {b, n + 1})) || (accepted && !shape_is(*accepted, {b})))
    NOT_HERE;
  Scratch ws;
  if (!scratch(a[8], a[8] == Py_None ? fn.verify_workspace(b, n, vocab) : 0, *logits, &ws)) NOT_HERE;
  const auto ints = logits->options().dtype(at::kInt).requires_grad(false);
  at::Tensor new_tokens, new_accepted;
  Held t{nullptr}, c{nullptr};
  if (tokens) Py_INCREF(a[6]), t.p = a[6];
  else new_tokens = at::empty({b, n + 1}, ints), tokens = &new_tokens, t.p = THPVariable_Wrap(new_tokens);
  if (accepted) Py_INCREF(a[7]), c.p = a[7];
  else new_accepted = at::empty({b}, ints), accepted = &new_accepted, c.p = THPVariable_Wrap(new_accepted);
  if (!t.p || !c.p) NOT_HERE;
  const float *lp = at_of<float>(logits), *qp = at_of<float>(draft_logits), *up = at_of<float>(u);
  const int32_t *dp = at_of<int32_t>(drafts), *np = at_of<int32_t>(counts);
  int32_t *tp = at_of<int32_t>(tokens), *ap = at_of<int32_t>(accepted);
  void* st = current_stream();
  PyObject* both = PyTuple_Pack(2, t.p, c.p);
  if (!both) NOT_HERE;
  return result(WITHOUT_GIL(fn.verify(lp, qp, dp, np, up, tp, ap, b, n, vocab, temperature, ws.at, ws.bytes, st)), "mqa_stack_verify_drafts", both);
}

// ---------------------------------------------------------------- caches of 8 bits
// Their sizes and positions of a scale; false: not these
bool scaled_of(const at::Tensor* K, const at::Tensor* Ks, const at::Tensor* V, const at::Tensor* Vs, const at::Tensor* table, int64_t b, Paged* c, int* block) {
  if (!K || !Ks || !V || !Vs || !table || K->dim() < 3 || K->dim() > 4 || V->dim() != K->dim() || table->dim() != 2 || table->size(0) != b || V->scalar_type() != K->scalar_type() ||
      V->sizes().slice(0, V->dim() - 1) != K->sizes().slice(0, K->dim() - 1) || Ks->dim() != K->dim() - 1 || Ks->sizes() != Vs->sizes() ||
      Ks->sizes().slice(0, Ks->dim() - 1) != K->sizes().slice(0, K->dim() - 2) || !fits(*K) || !fits(*V) || !fits(*table))
    return false;
  const int dt = K->scalar_type() == at::kFloat8_e4m3fn ? MQA_E4M3 : K->scalar_type() == at::kChar ? MQA_INT8 : -1;
  *c = Paged{K->dim() == 4 ? K->size(1) : 1, K->size(0), K->size(-2), table->size(1), K->size(-1), V->size(-1), dt};
  const int64_t blocks = Ks->size(-1);
  if (dt < 0 || c->size <= 0 || blocks <= 0 || c->size % blocks) return false;
  *block = (int)(c->size / blocks);
  return true;
}

// (K_pages, K_scales, V_pages, V_scales, table, k_new, v_new, lens, lens_out, counts)
MQA_CALL(scaled_append, 10) {
  const at::Tensor *K = plain(a[0]), *Ks = f32(a[1]), *V = plain(a[2]), *Vs = f32(a[3]), *table = i32(a[4]), *kn = f32(a[5]), *vn = f32(a[6]), *lens = i32(a[7]),
                   *out = i32(a[8]), *counts;
  Paged c;
  int block;
  if (!kn || !vn || !lens || !out || !maybe(a[9], at::kInt, &counts) || kn->dim() < 3 || !fits(*kn) || !scaled_of(K, Ks, V, Vs, table, kn->size(0), &c, &block)) NOT_HERE;
  const int64_t b = kn->size(0), n = kn->size(1);
  if (!(K->dim() == 4 ? shape_is(*kn, {b, n, c.h_kv, c.k}) && shape_is(*vn, {b, n, c.h_kv, c.v}) : shape_is(*kn, {b, n, c.k}) && shape_is(*vn, {b, n, c.v})) ||
      lens->numel() != b || out->numel() != b || (counts && counts->numel() != b))
    NOT_HERE;
  const float *kp = at_of<float>(kn), *vp = at_of<float>(vn);
  const int32_t *cp = at_of<int32_t>(counts), *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens);
  int32_t* op = at_of<int32_t>(out);
  float *sk = at_of<float>(Ks), *sv = at_of<float>(Vs);
  void *Kp = K->data_ptr(), *Vp = V->data_ptr(), *st = current_stream();
  Py_INCREF(a[8]);
  return result(WITHOUT_GIL(fn.scaled_append(kp, vp, cp, Kp, sk, Vp, sv, tp, lp, op, b, n, c.h_kv, c.pages, c.size, block, c.each, c.k, c.v, (mqa_dtype)c.dt, st)),
                "mqa_paged_scaled_append_kv_rows", a[8]);
}

// (q, K_pages, K_scales, V_pages, V_scales, table, lens, o, scale, workspace)
MQA_CALL(scaled_decode, 10) {
  const at::Tensor *q = f32(a[0]), *K = plain(a[1]), *Ks = f32(a[2]), *V = plain(a[3]), *Vs = f32(a[4]), *table = i32(a[5]), *lens = i32(a[6]), *o;
  float scale;
  Paged c;
  int block;
  if (!q || !lens || q->dim() < 3 || q->dim() > 4 || !fits(*q) || !number(a[8], &scale) || !scaled_of(K, Ks, V, Vs, table, q->size(0), &c, &block)) NOT_HERE;
  const int64_t b = q->size(0), n = q->dim() == 4 ? q->size(1) : 1, h = q->size(-2);
  if (q->size(-1) != c.k || lens->numel() != b) NOT_HERE;
  at::Tensor own;
  Held res{q->dim() == 4 ? output(a[7], *q, {b, n, h, c.v}, &o, &own) : output(a[7], *q, {b, h, c.v}, &o, &own)};
  if (!res.p) NOT_HERE;
  Scratch ws;
  if (!scratch(a[9], a[9] == Py_None ? fn.scaled_workspace(b, n, h, c.h_kv, c.size, c.each, c.k, c.v, (mqa_dtype)c.dt) : 0, *q, &ws)) NOT_HERE;
  const float *qp = at_of<float>(q), *sk = at_of<float>(Ks), *sv = at_of<float>(Vs);
  float* op = at_of<float>(o);
  const int32_t *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens);
  const void *Kp = K->data_ptr(), *Vp = V->data_ptr();
  void* st = current_stream();
  return result(WITHOUT_GIL(fn.scaled_decode(qp, Kp, sk, Vp, sv, tp, lp, op, b, n, h, c.h_kv, c.pages, c.size, block, c.each, c.k, c.v, (mqa_dtype)c.dt, scale, ws.at, ws.bytes, st)),
                "mqa_paged_scaled_decode_step", res.take());
}

// ---------------------------------------------------------------- pages
// (table, lens, parents, table_out, lens_out, refs, page_size)
MQA_CALL(fork_pages, 7) {
  const at::Tensor *table = i32(a[0]), *lens = i32(a[1]), *parents = i32(a[2]), *to = i32(a[3]), *out = i32(a[4]), *refs = i32(a[5]);
  int size;
  if (!table || !lens || !parents || !to || !out || !refs || table->dim() != 2 || parents->dim() != 1 || refs->dim() != 1 || !fits(*table) || !fits(*parents) || !fits(*refs) ||
      !integer(a[6], &size))
    NOT_HERE;
  const int64_t b = table->size(0), each = table->size(1), n = parents->size(0), pages = refs->size(0);
  if (!shape_is(*lens, {b}) || !shape_is(*to, {n, each}) || !shape_is(*out, {n})) NOT_HERE;
  const int32_t *tp = at_of<int32_t>(table), *lp = at_of<int32_t>(lens), *pp = at_of<int32_t>(parents);
  int32_t *op = at_of<int32_t>(to), *np = at_of<int32_t>(out), *rp = at_of<int32_t>(refs);
  void* st = current_stream();
  Py_INCREF(a[3]);
  return result(WITHOUT_GIL(fn.fork_pages(tp, lp, pp, op, np, rp, b, n, pages, size, each, st)), "mqa_paged_fork_pages", a[3]);
}

// (table, lens, refs, page_size)
MQA_CALL(free_pages, 4) {
  const at::Tensor *table = i32(a[0]), *lens = i32(a[1]), *refs = i32(a[2]);
  int size;
  if (!table || !lens || !refs || table->dim() != 2 || refs->dim() != 1 || !fits(*table) || !fits(*refs) || !integer(a[3], &size) || !shape_is(*lens, {table->size(0)})) NOT_HERE;
  const int64_t b = table->size(0), each = table->size(1), pages = refs->size(0);
  int32_t *tp = at_of<int32_t>(table), *rp = at_of<int32_t>(refs);
  const int32_t* lp = at_of<int32_t>(lens);
  void* st = current_stream();
  Py_INCREF(a[0]);
  return result(WITHOUT_GIL(fn.free_pages(tp, lp, rp, b, pages, size, each, st)), "mqa_paged_free_pages", a[0]);
}

// (table, lens, refs, page_size, n, counts, granted, moves, workspace)
MQA_CALL(reserve_pages, 9) {
  const at::Tensor *table = i32(a[0]), *lens = i32(a[1]), *refs = i32(a[2]), *counts, *granted, *moves;
  int size, n;
  if (!table || !lens || !refs || table->dim() != 2 || refs->dim() != 1 || !fits(*table) || !fits(*refs) || !integer(a[3], &size) || !integer(a[4], &n) ||
      !maybe(a[5], at::kInt, &counts) || !maybe(a[6], at::kInt, &granted) || !maybe(a[7], at::kInt, &moves))
    NOT_HERE;
  const int64_t b = table->size(0), each = table->size(1), pages = refs->size(0);
  if (!shape_is(*lens, {b}) || (counts && !shape_is(*counts, {b})) || (granted && !shape_is(*granted, {b})) || (moves && !shape_is(*moves, {b, 2}))) NOT_HERE;
  Scratch ws;
  if (!scratch(a[8], a[8] == Py_None ? fn.reserve_workspace(b, n, pages, size, each) : 0, *table, &ws)) NOT_HERE;
  const auto ints = table->options().requires_grad(false);
  at::Tensor new_granted, new_moves;
  Held g{nullptr}, m{nullptr};
  if (granted) Py_INCREF(a[6]), g.p = a[6];
  else new_granted = at::empty({b}, ints), granted = &new_granted, g.p = THPVariable_Wrap(new_granted);
  if (moves) Py_INCREF(a[7]), m.p = a[7];
  else new_moves = at::empty({b, 2}, ints), moves = &new_moves, m.p = THPVariable_Wrap(new_moves);
  if (!g.p || !m.p) NOT_HERE;
  int32_t *tp = at_of<int32_t>(table), *rp = at_of<int32_t>(refs), *gp = at_of<int32_t>(granted), *mp = at_of<int32_t>(moves);
  const int32_t *lp = at_of<int32_t>(lens), *cp = at_of<int32_t>(counts);
  void* st = current_stream();
  PyObject* both = PyTuple_Pack(2, g.p, m.p);
  if (!both) NOT_HERE;
  return result(WITHOUT_GIL(fn.reserve_pages(tp, lp, cp, rp, gp, mp, b, n, pages, size, each, ws.at, ws.bytes, st)), "mqa_paged_reserve_pages", both);
}

// (table, refs, table_out, refs_out, moves, used, workspace)
MQA_CALL(compact_pages, 7) {
  const at::Tensor *table = i32(a[0]), *refs = i32(a[1]), *to = i32(a[2]), *refs_out = i32(a[3]), *moves = i32(a[4]), *used = i32(a[5]);
  if (!table || !refs || !to || !refs_out || !moves || !used || table->dim() != 2 || refs->dim() != 1 || !fits(*table) || !fits(*refs)) NOT_HERE;
  const int64_t b = table->size(0), each = table->size(1), pages = refs->size(0);
  if (!shape_is(*to, {b, each}) || !shape_is(*refs_out, {pages}) || !shape_is(*moves, {pages / 2 > 1 ? pages / 2 : 1, 2}) || !shape_is(*used, {1})) NOT_HERE;
  Scratch ws;
  if (!scratch(a[6], a[6] == Py_None ? fn.compact_workspace(b, pages, each) : 0, *table, &ws)) NOT_HERE;
  const int32_t *tp = at_of<int32_t>(table), *rp = at_of<int32_t>(refs);
  int32_t *op = at_of<int32_t>(to), *np = at_of<int32_t>(refs_out), *mp = at_of<int32_t>(moves), *up = at_of<int32_t>(used);
  void* st = current_stream();
  Py_INCREF(a[4]);
  return result(WITHOUT_GIL(fn.compact_pages(tp, rp, op, np, mp, up, b, pages, each, ws.at, ws.bytes, st)), "mqa_paged_compact_pages", a[4]);
}

// (pools, moves)
MQA_CALL(copy_pages, 2) {
  constexpr Py_ssize_t most = 64;
  const at::Tensor* moves = i32(a[1]);
  if (!moves || moves->dim() != 2 || moves->size(1) != 2 || !fits(*moves) || !(PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0]))) NOT_HERE;
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[0]);
  if (count < 1 || count > most) NOT_HERE;
  void* at[most];
  size_t sizes[most];
  int64_t pages = 0;
  for (Py_ssize_t i = 0; i < count; ++i) {
    const at::Tensor* t = plain(PySequence_Fast_GET_ITEM(a[0], i));
    if (!t || t->dim() < 2 || !fits(*t) || (i > 0 && t->size(0) != pages) || t->size(0) <= 0) NOT_HERE;
    pages = t->size(0);
    at[i] = t->data_ptr();
    sizes[i] = bytes_of(*t) / (size_t)pages;
  }
  const int32_t* mp = at_of<int32_t>(moves);
  const int64_t m = moves->size(0);
  void* st = current_stream();
  Py_INCREF(Py_True);
  return result(WITHOUT_GIL(fn.copy_pages(at, sizes, (int)count, mp, m, pages, st)), "mqa_paged_copy_pages", Py_True);
}

// (logits, history, lens, drafts, prompts, repetition, frequency, presence, bias_tokens, biases, allowed, out)
MQA_CALL(adjust_logits, 12) {
  const at::Tensor *logits = f32(a[0]), *history = i32(a[1]), *lens = i32(a[2]), *drafts, *prompts, *repetition, *frequency, *presence, *tokens, *biases, *allowed, *out;
  if (!logits || !history || !lens || logits->dim() < 2 || logits->dim() > 3 || history->dim() != 2 || !fits(*logits) || !fits(*history) || !maybe(a[3], at::kInt, &drafts) ||
      !maybe(a[4], at::kInt, &prompts) || !maybe(a[5], at::kFloat, &repetition) || !maybe(a[6], at::kFloat, &frequency) || !maybe(a[7], at::kFloat, &presence) ||
      !maybe(a[8], at::kInt, &tokens) || !maybe(a[9], at::kFloat, &biases) || !maybe(a[10], at::kInt, &allowed))
    NOT_HERE;
  const bool flat = logits->dim() == 2;
  const int64_t b = logits->size(0), n = flat ? 0 : logits->size(1) - 1, vocab = logits->size(-1), words = (vocab + 31) / 32;
  if (history->size(0) != b || !shape_is(*lens, {b}) || (drafts && !shape_is(*drafts, {b, n})) || (prompts && !shape_is(*prompts, {b})) ||
      (repetition && !shape_is(*repetition, {b})) || (frequency && !shape_is(*frequency, {b})) || (presence && !shape_is(*presence, {b})) || !tokens != !biases ||
      (allowed && !(flat ? shape_is(*allowed, {b, words}) : shape_is(*allowed, {b, n + 1, words}))))
    NOT_HERE;
  int64_t m = 0;
  if (biases) {
    if (biases->dim() != 2 || biases->size(0) != b || !fits(*biases) || tokens->sizes() != biases->sizes()) NOT_HERE;
    m = biases->size(1);
  }
  at::Tensor own;
  Held res{flat ? output(a[11], *logits, {b, vocab}, &out, &own) : output(a[11], *logits, {b, n + 1, vocab}, &out, &own)};
  if (!res.p) NOT_HERE;
  const float *lp = at_of<float>(logits), *rp = at_of<float>(repetition), *fp = at_of<float>(frequency), *pp = at_of<float>(presence), *vp = at_of<float>(biases);
  const int32_t *hp = at_of<int32_t>(history), *np = at_of<int32_t>(lens), *dp = at_of<int32_t>(drafts), *mp = at_of<int32_t>(prompts), *tp = at_of<int32_t>(tokens);
  const uint32_t* ap = at_of<uint32_t>(allowed);
  float* op = at_of<float>(out);
  const int64_t cap = history->size(1);
  void* st = current_stream();
  return result(WITHOUT_GIL(fn.adjust_logits(lp, op, hp, np, mp, dp, rp, fp, pp, tp, vp, ap, b, n, vocab, cap, m, st)), "mqa_stack_adjust_logits", res.take());
}

// (the error's class, torch.nn.Parameter, addresses in the order of Functions)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr Py_ssize_t count = sizeof(Functions) / sizeof(void*);
  if (n != 2 + count) { PyErr_SetString(PyExc_TypeError, "init: a class, a class and the functions' addresses"); return nullptr; }
  void* at[count];
  for (Py_ssize_t i = 0; i < count; ++i) {
    at[i] = PyLong_AsVoidPtr(a[2 + i]);
    if (!at[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "init: no address");
      return nullptr;
    }
  }
  memcpy(&fn, at, sizeof fn);
  Py_INCREF(a[0]), Py_INCREF(a[1]);
  Py_XSETREF(error_class, a[0]);
  Py_XSETREF(parameter_class, a[1]);
  Py_RETURN_NONE;
}

// of the torch whose tensors these functions know from within
PyObject* torch_version(PyObject*, PyObject* const*, Py_ssize_t) { return PyUnicode_FromString(MQA_TORCH_VERSION); }

#define ENTRY(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(init), ENTRY(torch_version), ENTRY(decode), ENTRY(append_qkv), ENTRY(project), ENTRY(add_layernorm), ENTRY(memory_kv), ENTRY(attend_rows), ENTRY(beams),
                         ENTRY(reorder), ENTRY(paged_append), ENTRY(paged_decode), ENTRY(paged_evict), ENTRY(verify), ENTRY(scaled_append), ENTRY(scaled_decode),
                         ENTRY(fork_pages), ENTRY(free_pages), ENTRY(reserve_pages), ENTRY(compact_pages), ENTRY(copy_pages), ENTRY(adjust_logits), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Native argument marshalling of binding.py", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
