// The per-call part of the Python binding for encode, decode, attention, the
// serving operators and the paged 8-bit cache:
// argument checks, output allocation and the library call, without the Python
// interpreter between them (14 us of checks around a 7 us kernel before, about
// 2 us here).  Every function returns None, having done nothing, for any
// argument that it does not recognise as valid; the Python code then goes
// through its own checks, which name what is wrong.  Once the library has been
// entered, its status is final: anything but FIBQ_OK raises FibqError.
//
// The library is reached through the entry points that bind() is given (the
// loaded library's own), so this module does not load it.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/python_arg_parser.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>

#include <cmath>
#include <cstdint>

#include "fibq.h"

namespace {

decltype(&fibq_encode) g_encode;
decltype(&fibq_decode) g_decode;
decltype(&fibq_attn_decode) g_attn;
decltype(&fibq_attn_workspace_bytes) g_ws;
decltype(&fibq_payload_bytes) g_payload;
PyObject* g_check;  // the package's _check(status, where): raises FibqError

using at::Tensor;

// A plain dense device tensor (no subclass, no wrapper without storage).
const Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() ||
      t.is_conj() || t.is_neg())
    return nullptr;
  return &t;
}
bool int_arg(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0 && *v >= -1 && *v < (1LL << 62);
}
bool shaped(const Tensor* t, at::ScalarType ty, std::initializer_list<int64_t> s) {
  if (!t || t->scalar_type() != ty || t->dim() != (int64_t)s.size() || !t->is_contiguous())
    return false;
  int64_t i = 0;
  for (int64_t v : s)
    if (t->size(i++) != v) return false;
  return true;
}
bool norm_type(const Tensor* t) {
  return t && (t->scalar_type() == at::kShort || t->scalar_type() == at::kUInt16);
}
int dtype_code(const Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return FIBQ_F32;
    case at::kHalf: return FIBQ_F16;
    case at::kBFloat16: return FIBQ_BF16;
    default: return -1;
  }
}
const void* ptr(const Tensor& t) { return t.const_data_ptr(); }

// d, k, N of the call: R [d, d] and C [N, k] float32 on x's device
bool codec(const Tensor* R, const Tensor* C, int64_t d, int64_t k, int64_t N, at::Device dev,
           int64_t* P, double* rate) {
  if (d < 1 || d > 4096 || k < 1 || k > d || N < 2 || N > 65536) return false;
  if (!shaped(R, at::kFloat, {d, d}) || !shaped(C, at::kFloat, {N, k})) return false;
  if (R->device() != dev || C->device() != dev) return false;
  *P = g_payload((int)d, (int)k, (int)N);
  *rate = std::log2((double)N) / (double)k;
  return *P > 0;
}

// Raises FibqError for a status of the library.  (Not None: the Python code
// would enter the library a second time, and a HIP error is reported once.)
PyObject* raise_status(int rc, const char* where) {
  PyObject* r = PyObject_CallFunction(g_check, "is", rc, where);
  if (r) {  // (_check returned)
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, where);
  }
  return nullptr;
}

// Other Python threads run while this lives: an allocation may wait for the
// allocator, and a launch for a free place in the queue or, the first time,
// for the kernels to be loaded.  Raw pointers are taken before.
struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};

#define FIBQ_NONE return Py_NewRef_(Py_None)
PyObject* Py_NewRef_(PyObject* o) {
  Py_INCREF(o);
  return o;
}
PyObject* keep(PyObject* given, const Tensor& t) {
  return given != Py_None ? Py_NewRef_(given) : THPVariable_Wrap(t);
}

// encode(x, k, N, R, C, payload, norms, stream) -> (payload, norms)
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_encode || n_args != 8) FIBQ_NONE;
  const Tensor* x = tensor(a[0]);
  int64_t k, N, st, P;
  double rate;
  if (!x || x->dim() != 2 || !int_arg(a[1], &k) || !int_arg(a[2], &N) || !int_arg(a[7], &st)) FIBQ_NONE;
  const int64_t n = x->size(0), d = x->size(1);
  const int dt = dtype_code(*x);
  if (dt < 0 || x->stride(1) != 1 || (n > 1 && x->stride(0) < d)) FIBQ_NONE;
  const Tensor *R = tensor(a[3]), *C = tensor(a[4]);
  if (!codec(R, C, d, k, N, x->device(), &P, &rate)) FIBQ_NONE;
  Tensor payload, norms;
  if (a[5] != Py_None) {
    const Tensor* t = tensor(a[5]);
    if (!shaped(t, at::kByte, {n, P}) || t->device() != x->device()) FIBQ_NONE;
    payload = *t;
  }
  if (a[6] != Py_None) {
    const Tensor* t = tensor(a[6]);
    if (!norm_type(t) || !shaped(t, t->scalar_type(), {n}) || t->device() != x->device()) FIBQ_NONE;
    norms = *t;
  }
  const auto opt = at::TensorOptions().device(x->device());
  const void* px = ptr(*x);
  const int64_t stride = x->stride(0);
  const float *pR = static_cast<const float*>(ptr(*R)), *pC = static_cast<const float*>(ptr(*C));
  int rc;
  {
    NoGil no_gil;
    if (!payload.defined()) payload = at::empty({n, P}, opt.dtype(at::kByte));
    if (!norms.defined()) norms = at::empty({n}, opt.dtype(at::kShort));
    rc = g_encode(px, dt, n, stride, (int)d, (int)k, rate, (int)N, pR, pC,
                  static_cast<uint8_t*>(payload.data_ptr()),
                  static_cast<uint16_t*>(norms.data_ptr()), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_encode");
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, keep(a[5], payload));
  PyTuple_SET_ITEM(r, 1, keep(a[6], norms));
  return r;
  END_HANDLE_TH_ERRORS
}

// decode(payload, norms, d, k, N, R, C, token_ids, out, stream) -> out
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_decode || n_args != 10) FIBQ_NONE;
  const Tensor *p = tensor(a[0]), *h = tensor(a[1]);
  int64_t d, k, N, st, P;
  double rate;
  if (!p || !h || !int_arg(a[2], &d) || !int_arg(a[3], &k) || !int_arg(a[4], &N) ||
      !int_arg(a[9], &st) || p->dim() != 2)
    FIBQ_NONE;
  const at::Device dev = p->device();
  const Tensor *R = tensor(a[5]), *C = tensor(a[6]);
  if (!codec(R, C, d, k, N, dev, &P, &rate)) FIBQ_NONE;
  const int64_t cache = p->size(0);
  if (!shaped(p, at::kByte, {cache, P}) || !norm_type(h) || !shaped(h, h->scalar_type(), {cache}) ||
      h->device() != dev)
    FIBQ_NONE;
  const int64_t* ids = nullptr;
  int64_t n = cache;
  if (a[7] != Py_None) {
    const Tensor* t = tensor(a[7]);
    if (!t || t->dim() != 1 || !shaped(t, at::kLong, {t->size(0)}) || t->device() != dev) FIBQ_NONE;
    n = t->size(0);
    ids = static_cast<const int64_t*>(ptr(*t));
  }
  Tensor out;
  if (a[8] != Py_None) {
    const Tensor* t = tensor(a[8]);
    if (!shaped(t, at::kFloat, {n, d}) || t->device() != dev) FIBQ_NONE;
    out = *t;
  }
  const uint8_t* pp = static_cast<const uint8_t*>(ptr(*p));
  const uint16_t* ph = static_cast<const uint16_t*>(ptr(*h));
  const float *pR = static_cast<const float*>(ptr(*R)), *pC = static_cast<const float*>(ptr(*C));
  int rc;
  {
    NoGil no_gil;
    if (!out.defined()) out = at::empty({n, d}, at::TensorOptions().device(dev).dtype(at::kFloat));
    rc = g_decode(pp, ph, ids, n, cache, (int)d, (int)k, rate, (int)N, pR, pC,
                  static_cast<float*>(out.data_ptr()), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_decode");
  return keep(a[8], out);
  END_HANDLE_TH_ERRORS
}

// attn(q, k_payload, k_norms, v_payload, v_norms, T, k, N, R, C, scale,
//      workspace, out, stream) -> out
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_attn || n_args != 14) FIBQ_NONE;
  const Tensor *q = tensor(a[0]), *kp = tensor(a[1]), *kn = tensor(a[2]), *vp = tensor(a[3]),
               *vn = tensor(a[4]);
  int64_t T, k, N, st, P;
  double rate;
  if (!q || !kp || q->dim() != 3 || kp->dim() != 3 || !q->is_contiguous() || !int_arg(a[5], &T) ||
      !int_arg(a[6], &k) || !int_arg(a[7], &N) || !PyFloat_CheckExact(a[10]) || !int_arg(a[13], &st))
    FIBQ_NONE;
  const int64_t ng = q->size(0), G = q->size(1), d = q->size(2), Ts = kp->size(1);
  const at::Device dev = q->device();
  const int dt = dtype_code(*q);
  const Tensor *R = tensor(a[8]), *C = tensor(a[9]);
  if (dt < 0 || G < 1 || G > 16 || T < 0 || T > Ts || !codec(R, C, d, k, N, dev, &P, &rate)) FIBQ_NONE;
  if (!shaped(kp, at::kByte, {ng, Ts, P}) || !shaped(vp, at::kByte, {ng, Ts, P}) ||
      !norm_type(kn) || !norm_type(vn) || !shaped(kn, kn->scalar_type(), {ng, Ts}) ||
      !shaped(vn, vn->scalar_type(), {ng, Ts}))
    FIBQ_NONE;
  if (kp->device() != dev || vp->device() != dev || kn->device() != dev || vn->device() != dev)
    FIBQ_NONE;
  Tensor out, ws;
  const auto opt = at::TensorOptions().device(dev);
  const int64_t need = (int64_t)g_ws(ng, (int)G, T, (int)d, (int)k, (int)N);
  if (a[11] != Py_None) {
    const Tensor* t = tensor(a[11]);
    if (!t || t->dim() != 1 || !shaped(t, at::kByte, {t->size(0)}) || t->size(0) < need ||
        t->device() != dev)
      FIBQ_NONE;
    ws = *t;
  }
  if (a[12] != Py_None) {
    const Tensor* t = tensor(a[12]);
    if (!shaped(t, at::kFloat, {ng, G, d}) || t->device() != dev) FIBQ_NONE;
    out = *t;
  }
  const void* pq = ptr(*q);
  const uint8_t *pkp = static_cast<const uint8_t*>(ptr(*kp)), *pvp = static_cast<const uint8_t*>(ptr(*vp));
  const uint16_t *pkn = static_cast<const uint16_t*>(ptr(*kn)), *pvn = static_cast<const uint16_t*>(ptr(*vn));
  const float *pR = static_cast<const float*>(ptr(*R)), *pC = static_cast<const float*>(ptr(*C));
  const float scale = (float)PyFloat_AS_DOUBLE(a[10]);
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined()) ws = at::empty({need > 1 ? need : 1}, opt.dtype(at::kByte));
    if (!out.defined()) out = at::empty({ng, G, d}, opt.dtype(at::kFloat));
    rc = g_attn(pq, dt, pkp, pkn, pvp, pvn, ng, (int)G, T, Ts, (int)d, (int)k, rate, (int)N, pR, pC,
                scale, static_cast<float*>(out.data_ptr()), ws.data_ptr(), (size_t)ws.numel(),
                reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_attn_decode");
  return keep(a[12], out);
  END_HANDLE_TH_ERRORS
}

// ----------------------------------------------------------------- serving --
decltype(&fibq_attn_tree) g_tree;
decltype(&fibq_attn_tree_workspace_bytes) g_tree_ws;
decltype(&fibq_attn_decode_accum) g_accum;
decltype(&fibq_attn_decode_accum_workspace_bytes) g_accum_ws;
decltype(&fibq_accept_draft) g_accept;
decltype(&fibq_evict) g_evict;
decltype(&fibq_evict_workspace_bytes) g_evict_ws;

// k_payload, k_norms, v_payload, v_norms, at a[0] .. a[3], on the device `index`
struct Rows {
  const uint8_t *kp, *vp;
  const uint16_t *kn, *vn;
  int64_t n, T, P;
  at::Device dev = at::kCPU;
};
bool rows(PyObject* const* a, int64_t index, Rows* r) {
  const Tensor *kp = tensor(a[0]), *kn = tensor(a[1]), *vp = tensor(a[2]), *vn = tensor(a[3]);
  if (!kp || kp->dim() != 3 || kp->device().index() != index) return false;
  r->n = kp->size(0), r->T = kp->size(1), r->P = kp->size(2), r->dev = kp->device();
  if (!shaped(kp, at::kByte, {r->n, r->T, r->P}) || !shaped(vp, at::kByte, {r->n, r->T, r->P}) ||
      !norm_type(kn) || !norm_type(vn) || !shaped(kn, kn->scalar_type(), {r->n, r->T}) ||
      !shaped(vn, vn->scalar_type(), {r->n, r->T}) || kn->device() != r->dev ||
      vp->device() != r->dev || vn->device() != r->dev)
    return false;
  r->kp = static_cast<const uint8_t*>(ptr(*kp)), r->kn = static_cast<const uint16_t*>(ptr(*kn));
  r->vp = static_cast<const uint8_t*>(ptr(*vp)), r->vn = static_cast<const uint16_t*>(ptr(*vn));
  return true;
}
// a tensor of this type and shape on dev, or null
const Tensor* given(PyObject* o, at::ScalarType ty, std::initializer_list<int64_t> s, at::Device dev) {
  const Tensor* t = tensor(o);
  return shaped(t, ty, s) && t->device() == dev ? t : nullptr;
}
bool shared(const Tensor* x, const Tensor* y) {  // any memory
  const char *px = static_cast<const char*>(ptr(*x)), *py = static_cast<const char*>(ptr(*y));
  return px < py + y->nbytes() && py < px + x->nbytes();
}
// an optional workspace of at least `need` bytes; false: not a valid one
bool workspace(PyObject* o, int64_t need, at::Device dev, Tensor* ws) {
  if (o == Py_None) return true;
  const Tensor* t = tensor(o);
  if (!t || t->dim() != 1 || !shaped(t, at::kByte, {t->size(0)}) || t->size(0) < need ||
      t->device() != dev)
    return false;
  *ws = *t;
  return true;
}
Tensor empty(at::Device dev, at::ScalarType ty, at::IntArrayRef s) {
  return at::empty(s, at::TensorOptions().device(dev).dtype(ty));
}

// attn_tree(q, k_payload, k_norms, v_payload, v_norms, lens, masks, k, N, R, C,
//           scale, workspace, out, stream, device) -> out
PyObject* attn_tree(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_tree || n_args != 16) FIBQ_NONE;
  const Tensor *q = tensor(a[0]), *masks = tensor(a[6]);
  int64_t k, N, st, index, P;
  double rate;
  Rows r;
  if (!q || q->dim() != 4 || !q->is_contiguous() || !masks || !int_arg(a[7], &k) ||
      !int_arg(a[8], &N) || !PyFloat_CheckExact(a[11]) || !int_arg(a[14], &st) ||
      !int_arg(a[15], &index) || !rows(a + 1, index, &r))
    FIBQ_NONE;
  const int64_t M = q->size(1), G = q->size(2), d = q->size(3);
  const int dt = dtype_code(*q);
  const Tensor *R = tensor(a[9]), *C = tensor(a[10]);
  if (dt < 0 || q->size(0) != r.n || q->device() != r.dev || M < 1 || M > 64 || G < 1 || G > 16 ||
      !codec(R, C, d, k, N, r.dev, &P, &rate) || P != r.P)
    FIBQ_NONE;
  const Tensor* lens = given(a[5], at::kInt, {r.n}, r.dev);
  const bool shared = masks->dim() == 1;
  if (!lens || masks->device() != r.dev ||
      !(shared ? shaped(masks, at::kLong, {M}) : shaped(masks, at::kLong, {r.n, M})))
    FIBQ_NONE;
  const int64_t need = (int64_t)g_tree_ws(r.n, (int)M, (int)G, (int)d, (int)k, (int)N);
  Tensor ws, out;
  if (!workspace(a[12], need, r.dev, &ws)) FIBQ_NONE;
  if (a[13] != Py_None) {
    const Tensor* t = given(a[13], at::kFloat, {r.n, M, G, d}, r.dev);
    if (!t) FIBQ_NONE;
    out = *t;
  }
  const void* pq = ptr(*q);
  const int32_t* pl = static_cast<const int32_t*>(ptr(*lens));
  const uint64_t* pm = static_cast<const uint64_t*>(ptr(*masks));
  const float *pR = static_cast<const float*>(ptr(*R)), *pC = static_cast<const float*>(ptr(*C));
  const float scale = (float)PyFloat_AS_DOUBLE(a[11]);
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined()) ws = empty(r.dev, at::kByte, {need > 1 ? need : 1});
    if (!out.defined()) out = empty(r.dev, at::kFloat, {r.n, M, G, d});
    rc = g_tree(pq, dt, r.kp, r.kn, r.vp, r.vn, pl, pm, shared ? 0 : M, r.n, (int)M, (int)G, r.T,
                (int)d, (int)k, rate, (int)N, pR, pC, scale, static_cast<float*>(out.data_ptr()),
                ws.data_ptr(), (size_t)ws.numel(), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_attn_tree");
  return keep(a[13], out);
  END_HANDLE_TH_ERRORS
}

// attn_accum(q, k_payload, k_norms, v_payload, v_norms, lens, acc, k, N, R, C,
//            scale, workspace, out, stream, device) -> out
PyObject* attn_accum(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_accum || n_args != 16) FIBQ_NONE;
  const Tensor* q = tensor(a[0]);
  int64_t k, N, st, index, P;
  double rate;
  Rows r;
  if (!q || q->dim() != 3 || !q->is_contiguous() || !int_arg(a[7], &k) || !int_arg(a[8], &N) ||
      !PyFloat_CheckExact(a[11]) || !int_arg(a[14], &st) || !int_arg(a[15], &index) ||
      !rows(a + 1, index, &r))
    FIBQ_NONE;
  const int64_t G = q->size(1), d = q->size(2);
  const int dt = dtype_code(*q);
  const Tensor *R = tensor(a[9]), *C = tensor(a[10]);
  if (dt < 0 || q->size(0) != r.n || q->device() != r.dev || G < 1 || G > 16 ||
      !codec(R, C, d, k, N, r.dev, &P, &rate) || P != r.P)
    FIBQ_NONE;
  const Tensor *lens = given(a[5], at::kInt, {r.n}, r.dev), *acc = given(a[6], at::kFloat, {r.n, r.T}, r.dev);
  if (!lens || !acc) FIBQ_NONE;
  const int64_t need = (int64_t)g_accum_ws(r.n, (int)G, (int)d, (int)k, (int)N);
  Tensor ws, out;
  if (!workspace(a[12], need, r.dev, &ws)) FIBQ_NONE;
  if (a[13] != Py_None) {
    const Tensor* t = given(a[13], at::kFloat, {r.n, G, d}, r.dev);
    if (!t) FIBQ_NONE;
    out = *t;
  }
  const void* pq = ptr(*q);
  const int32_t* pl = static_cast<const int32_t*>(ptr(*lens));
  float* pa = static_cast<float*>(acc->data_ptr());
  const float *pR = static_cast<const float*>(ptr(*R)), *pC = static_cast<const float*>(ptr(*C));
  const float scale = (float)PyFloat_AS_DOUBLE(a[11]);
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined()) ws = empty(r.dev, at::kByte, {need > 1 ? need : 1});
    if (!out.defined()) out = empty(r.dev, at::kFloat, {r.n, G, d});
    rc = g_accum(pq, dt, r.kp, r.kn, r.vp, r.vn, pl, pa, r.n, (int)G, r.T, (int)d, (int)k, rate,
                 (int)N, pR, pC, scale, static_cast<float*>(out.data_ptr()), ws.data_ptr(),
                 (size_t)ws.numel(), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_attn_decode_accum");
  return keep(a[13], out);
  END_HANDLE_TH_ERRORS
}

// accept(k_payload, k_norms, v_payload, v_norms, lens, M, path, n_acc, new_lens,
//        stream, device) -> new_lens
PyObject* accept(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_accept || n_args != 11) FIBQ_NONE;
  int64_t M, st, index;
  Rows r;
  const Tensor* path = tensor(a[6]);
  if (!int_arg(a[5], &M) || M < 1 || M > 64 || !int_arg(a[9], &st) || !int_arg(a[10], &index) ||
      !path || path->dim() != 2 || !rows(a, index, &r))
    FIBQ_NONE;
  const int64_t A = path->size(1);
  const Tensor *lens = given(a[4], at::kInt, {r.n}, r.dev), *n_acc = given(a[7], at::kInt, {r.n}, r.dev);
  if (!lens || !n_acc || A < 1 || A > 64 || !shaped(path, at::kInt, {r.n, A}) || path->device() != r.dev)
    FIBQ_NONE;
  Tensor out;
  if (a[8] != Py_None) {
    const Tensor* t = given(a[8], at::kInt, {r.n}, r.dev);
    if (!t) FIBQ_NONE;
    for (const Tensor* x : {lens, n_acc, path})  // (lens or n_acc itself is fine)
      if (shared(x, t) && (x == path || ptr(*x) != ptr(*t))) FIBQ_NONE;
    out = *t;
  }
  const int32_t *pl = static_cast<const int32_t*>(ptr(*lens)), *pp = static_cast<const int32_t*>(ptr(*path)),
                *pn = static_cast<const int32_t*>(ptr(*n_acc));
  int rc;
  {
    NoGil no_gil;
    if (!out.defined()) out = empty(r.dev, at::kInt, {r.n});
    rc = g_accept(const_cast<uint8_t*>(r.kp), const_cast<uint16_t*>(r.kn), const_cast<uint8_t*>(r.vp),
                  const_cast<uint16_t*>(r.vn), pl, r.n, r.T, (int)r.P, (int)M, pp, (int)A, pn,
                  static_cast<int32_t*>(out.data_ptr()), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_accept_draft");
  return keep(a[8], out);
  END_HANDLE_TH_ERRORS
}

// evict(k_payload, k_norms, v_payload, v_norms, acc, lens, keep, recent, out,
//       workspace, stream, device) -> out; out: a tuple of seven tensors
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_evict || n_args != 12 || !PyTuple_CheckExact(a[8]) || PyTuple_GET_SIZE(a[8]) != 7) FIBQ_NONE;
  int64_t n_keep, recent, st, index;
  Rows r, o;
  PyObject* outs[7];
  for (int i = 0; i < 7; ++i) outs[i] = PyTuple_GET_ITEM(a[8], i);
  if (!int_arg(a[6], &n_keep) || !int_arg(a[7], &recent) || n_keep < 1 || n_keep >= (1LL << 30) ||
      !int_arg(a[10], &st) || !int_arg(a[11], &index) || !rows(a, index, &r) ||
      !rows(outs, index, &o) || o.n != r.n || o.P != r.P)
    FIBQ_NONE;
  const Tensor* in[] = {tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]),
                        given(a[4], at::kFloat, {r.n, r.T}, r.dev), given(a[5], at::kInt, {r.n}, r.dev)};
  const Tensor* to[] = {tensor(outs[0]), tensor(outs[1]), tensor(outs[2]), tensor(outs[3]),
                        given(outs[4], at::kFloat, {r.n, o.T}, r.dev), given(outs[5], at::kInt, {r.n}, r.dev),
                        given(outs[6], at::kInt, {r.n, n_keep}, r.dev)};
  if (!in[4] || !in[5] || !to[4] || !to[5] || !to[6]) FIBQ_NONE;
  for (const Tensor*& y : to) {  // (no output may share memory with an input or another output)
    for (const Tensor* x : in)
      if (shared(x, y)) FIBQ_NONE;
    for (const Tensor** x = to; x != &y; ++x)
      if (shared(*x, y)) FIBQ_NONE;
  }
  const int64_t need = (int64_t)g_evict_ws(r.n, r.T);
  Tensor ws;
  if (!workspace(a[9], need, r.dev, &ws)) FIBQ_NONE;
  const float* pa = static_cast<const float*>(ptr(*in[4]));
  const int32_t* pl = static_cast<const int32_t*>(ptr(*in[5]));
  float* qa = static_cast<float*>(to[4]->data_ptr());
  int32_t *ql = static_cast<int32_t*>(to[5]->data_ptr()), *qi = static_cast<int32_t*>(to[6]->data_ptr());
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined() && need > 0) ws = empty(r.dev, at::kByte, {need});
    rc = g_evict(r.kp, r.kn, r.vp, r.vn, pa, pl, r.n, r.T, (int)r.P, n_keep, recent, o.T,
                 const_cast<uint8_t*>(o.kp), const_cast<uint16_t*>(o.kn), const_cast<uint8_t*>(o.vp),
                 const_cast<uint16_t*>(o.vn), qa, ql, qi, ws.defined() ? ws.data_ptr() : nullptr,
                 ws.defined() ? (size_t)ws.numel() : 0, reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_evict");
  return Py_NewRef_(a[8]);
  END_HANDLE_TH_ERRORS
}

// bind_serving(attn_tree, its workspace_bytes, attn_decode_accum, its
// workspace_bytes, accept_draft, evict, its workspace_bytes): addresses
PyObject* bind_serving(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 7) {
    PyErr_SetString(PyExc_TypeError, "bind_serving takes seven addresses");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_tree = reinterpret_cast<decltype(g_tree)>(p[0]);
  g_tree_ws = reinterpret_cast<decltype(g_tree_ws)>(p[1]);
  g_accum = reinterpret_cast<decltype(g_accum)>(p[2]);
  g_accum_ws = reinterpret_cast<decltype(g_accum_ws)>(p[3]);
  g_accept = reinterpret_cast<decltype(g_accept)>(p[4]);
  g_evict = reinterpret_cast<decltype(g_evict)>(p[5]);
  g_evict_ws = reinterpret_cast<decltype(g_evict_ws)>(p[6]);
  Py_RETURN_NONE;
}

// ------------------------------------------------------- paged 8-bit cache --
decltype(&fibq_rope) g_rope;
decltype(&fibq_page_resize) g_resize;
decltype(&fibq_page_resize_workspace_bytes) g_resize_ws;
decltype(&fibq_cache8_write) g_write8;
decltype(&fibq_attn_cache8) g_attn8;
decltype(&fibq_attn_cache8_workspace_bytes) g_attn8_ws;

// Rows of heads [n, H, d] of type ty on dev, dense heads at any strides
struct HeadRows {
  const char *begin, *end;
  int64_t n, H, d, row, head, size;
};
bool head_rows(const Tensor* t, at::ScalarType ty, at::Device dev, HeadRows* r) {
  if (!t || t->scalar_type() != ty || t->dim() != 3 || t->device() != dev) return false;
  r->n = t->size(0), r->H = t->size(1), r->d = t->size(2), r->size = t->element_size();
  if (t->stride(2) != 1 && r->d > 1) return false;
  r->head = r->H > 1 ? t->stride(1) : r->d;
  r->row = r->n > 1 ? t->stride(0) : (r->H - 1) * r->head + r->d;
  r->begin = r->end = static_cast<const char*>(ptr(*t));
  if (t->numel() > 0) r->end += ((r->n - 1) * r->row + (r->H - 1) * r->head + r->d) * r->size;
  return true;
}
// no memory in common: extents that do not meet, or columns of one matrix that do not
bool apart(const HeadRows& a, const HeadRows& b) {
  if (a.end <= b.begin || b.end <= a.begin) return true;
  const int64_t row = a.row * a.size;
  if (row != b.row * b.size || row == 0 || a.n < 2) return false;
  const int64_t wide_a = ((a.H - 1) * a.head + a.d) * a.size,
                wide_b = ((b.H - 1) * b.head + b.d) * b.size;
  const int64_t at = ((b.begin - a.begin) % row + row) % row;
  return wide_a <= at && at + wide_b <= row;
}
bool once(const HeadRows& a) {  // (no element twice)
  return (a.head >= a.d && a.row >= (a.H - 1) * a.head + a.d) ||
         (a.row >= a.d && a.head >= (a.n - 1) * a.row + a.d);
}
bool meets(const HeadRows& a, const Tensor* t) {
  const char* p = static_cast<const char*>(ptr(*t));
  return a.begin < p + t->nbytes() && p < a.end;
}

// rope(q, k, positions, freqs, layout, scale, inverse, out, stream, device) -> (q, k);
// out: None or (q, k) themselves.  Calls that torch would record a gradient of are left
// to the Python code.
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_rope || n_args != 10) FIBQ_NONE;
  const Tensor *q = tensor(a[0]), *k = a[1] == Py_None ? nullptr : tensor(a[1]), *at_ = tensor(a[2]),
               *freqs = tensor(a[3]);
  int64_t st, index;
  const bool has_k = a[1] != Py_None;
  if (!q || (has_k && !k) || !at_ || !freqs || !PyFloat_CheckExact(a[5]) || !PyBool_Check(a[6]) ||
      !PyBool_Check(a[4]) || !int_arg(a[8], &st) || !int_arg(a[9], &index) ||
      q->device().index() != index || freqs->dim() != 1)
    FIBQ_NONE;
  if (c10::GradMode::is_enabled() && (q->requires_grad() || (has_k && k->requires_grad()) || freqs->requires_grad()))
    FIBQ_NONE;
  const at::Device dev = q->device();
  const int dt = dtype_code(*q);
  HeadRows rq, rk{};
  if (dt < 0 || !head_rows(q, q->scalar_type(), dev, &rq) ||
      (has_k && (!head_rows(k, q->scalar_type(), dev, &rk) || rk.n != rq.n || rk.d != rq.d)) ||
      !shaped(at_, at::kInt, {rq.n}) || !shaped(freqs, at::kDouble, {freqs->size(0)}) ||
      at_->device() != dev || freqs->device() != dev || rq.H > 2048 || rk.H > 2048)
    FIBQ_NONE;
  const int64_t rot = 2 * freqs->size(0);
  if (rq.d > 512 || rot < 2 || rot > rq.d) FIBQ_NONE;
  const bool in_place = a[7] != Py_None;
  if (in_place) {
    if (!PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) != 2 || PyTuple_GET_ITEM(a[7], 0) != a[0] ||
        PyTuple_GET_ITEM(a[7], 1) != a[1])
      FIBQ_NONE;
    if (!once(rq) || meets(rq, at_) || meets(rq, freqs)) FIBQ_NONE;
    if (has_k && (!once(rk) || !apart(rq, rk) || meets(rk, at_) || meets(rk, freqs))) FIBQ_NONE;
  }
  const void *pq = ptr(*q), *pk = has_k ? ptr(*k) : nullptr;
  const int32_t* pp = static_cast<const int32_t*>(ptr(*at_));
  const double* pf = static_cast<const double*>(ptr(*freqs));
  const at::ScalarType ty = q->scalar_type();
  const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
  const bool interleaved = a[4] == Py_True, inverse = a[6] == Py_True;
  Tensor qo, ko;
  int64_t qs[2] = {rq.row, rq.head}, ks[2] = {rk.row, rk.head};
  int rc;
  {
    NoGil no_gil;
    void *to_q = const_cast<void*>(pq), *to_k = const_cast<void*>(pk);
    if (!in_place) {
      qo = empty(dev, ty, {rq.n, rq.H, rq.d});
      to_q = qo.data_ptr(), qs[0] = rq.H * rq.d, qs[1] = rq.d;
      if (has_k) {
        ko = empty(dev, ty, {rk.n, rk.H, rk.d});
        to_k = ko.data_ptr(), ks[0] = rk.H * rk.d, ks[1] = rk.d;
      }
    }
    rc = g_rope(pq, pk, dt, rq.n, (int)rq.H, (int)rk.H, (int)rq.d, rq.row, rq.head, rk.row, rk.head,
                pp, pf, (int)rot, interleaved ? FIBQ_ROPE_INTERLEAVED : FIBQ_ROPE_HALF, scale, inverse,
                to_q, to_k, qs[0], qs[1], ks[0], ks[1], reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_rope");
  if (in_place) return Py_NewRef_(a[7]);
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(qo));
  PyTuple_SET_ITEM(r, 1, has_k ? THPVariable_Wrap(ko) : Py_NewRef_(Py_None));
  return r;
  END_HANDLE_TH_ERRORS
}

// page_resize(table, lens, grow, page, n_pages, free, n_free, n_rows, out, workspace,
//             stream, device) -> out; out: a tuple of five tensors or None
PyObject* page_resize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_resize || n_args != 12) FIBQ_NONE;
  const Tensor *table = tensor(a[0]), *stack = tensor(a[5]);
  int64_t page, n_pages, n_rows, st, index;
  if (!table || table->dim() != 2 || !stack || stack->dim() != 1 || !int_arg(a[3], &page) ||
      !int_arg(a[4], &n_pages) || !int_arg(a[7], &n_rows) || !int_arg(a[10], &st) ||
      !int_arg(a[11], &index) || table->device().index() != index || page < 1 || page > 65536 ||
      n_rows < 0 || n_rows >= (1LL << 31))
    FIBQ_NONE;
  const at::Device dev = table->device();
  const int64_t n = table->size(0), max_pages = table->size(1), cap = stack->size(0);
  const Tensor* in[] = {given(a[0], at::kInt, {n, max_pages}, dev), given(a[5], at::kInt, {cap}, dev),
                        given(a[1], at::kInt, {n}, dev), given(a[2], at::kInt, {n}, dev),
                        given(a[6], at::kInt, {1}, dev)};
  for (const Tensor* x : in)
    if (!x) FIBQ_NONE;
  for (int w = 0; w < 2; ++w)  // the table and the stack are written
    for (int i = w + 1; i < 5; ++i)
      if (shared(in[w], in[i])) FIBQ_NONE;
  const int64_t sizes[5] = {n, n + 1, n_rows, n_rows, 1};
  Tensor out[5], ws;
  const int64_t need = (int64_t)g_resize_ws(n);
  if (!workspace(a[9], need, dev, &ws)) FIBQ_NONE;
  if (ws.defined())
    for (const Tensor* x : in)
      if (shared(x, &ws)) FIBQ_NONE;
  if (a[8] != Py_None) {
    if (!PyTuple_CheckExact(a[8]) || PyTuple_GET_SIZE(a[8]) != 5) FIBQ_NONE;
    for (int i = 0; i < 5; ++i) {
      const Tensor* t = given(PyTuple_GET_ITEM(a[8], i), i == 2 ? at::kLong : at::kInt, {sizes[i]}, dev);
      if (!t) FIBQ_NONE;
      const Tensor* same = i == 0 ? in[2] : i == 4 ? in[4] : nullptr;  // (may be this input)
      for (const Tensor* x : in)
        if (shared(x, t) && !(x == same && ptr(*x) == ptr(*t))) FIBQ_NONE;
      for (int j = 0; j < i; ++j)
        if (shared(&out[j], t)) FIBQ_NONE;
      if (ws.defined() && shared(&ws, t)) FIBQ_NONE;
      out[i] = *t;
    }
  }
  const int32_t *pl = static_cast<const int32_t*>(ptr(*in[2])), *pg = static_cast<const int32_t*>(ptr(*in[3])),
                *pn = static_cast<const int32_t*>(ptr(*in[4]));
  int32_t *pt = static_cast<int32_t*>(table->data_ptr()), *pf = static_cast<int32_t*>(stack->data_ptr());
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined()) ws = empty(dev, at::kByte, {need > 1 ? need : 1});
    for (int i = 0; i < 5; ++i)
      if (!out[i].defined()) out[i] = empty(dev, i == 2 ? at::kLong : at::kInt, {sizes[i]});
    rc = g_resize(pt, pl, pg, n, max_pages, (int)page, n_pages, pf, cap, pn, n_rows,
                  static_cast<int32_t*>(out[0].data_ptr()), static_cast<int32_t*>(out[1].data_ptr()),
                  static_cast<int64_t*>(out[2].data_ptr()), static_cast<int32_t*>(out[3].data_ptr()),
                  static_cast<int32_t*>(out[4].data_ptr()), ws.data_ptr(), (size_t)ws.numel(),
                  reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_page_resize");
  if (a[8] != Py_None) return Py_NewRef_(a[8]);
  PyObject* r = PyTuple_New(5);
  if (!r) return nullptr;
  for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(out[i]));
  return r;
  END_HANDLE_TH_ERRORS
}

// k_pages, k_scales, v_pages, v_scales at a[0] .. a[3], on the device `index`
struct Pools {
  const Tensor* t[4];
  int64_t n_pages, H, page, d;
  int codes;
  at::Device dev = at::kCPU;
};
bool pools(PyObject* const* a, int64_t index, Pools* p) {
  for (int i = 0; i < 4; ++i) p->t[i] = tensor(a[i]);
  const Tensor* k = p->t[0];
  if (!k || k->dim() != 4 || k->device().index() != index) return false;
  p->n_pages = k->size(0), p->H = k->size(1), p->page = k->size(2), p->d = k->size(3);
  p->dev = k->device();
  const at::ScalarType ty = k->scalar_type();
  if (ty != at::kChar && ty != at::kFloat8_e4m3fn) return false;
  p->codes = ty == at::kChar ? FIBQ_INT8 : FIBQ_E4M3;
  for (int i = 0; i < 4; ++i)
    if (!p->t[i] || p->t[i]->device() != p->dev ||
        !(i % 2 ? shaped(p->t[i], at::kFloat, {p->n_pages, p->H})
                : shaped(p->t[i], ty, {p->n_pages, p->H, p->page, p->d})))
      return false;
  return p->H > 0 && p->H <= 1024 && p->page <= 128 && p->d <= 256;
}

// cache8_write(k, v, slots, k_pages, k_scales, v_pages, v_scales, stream, device) -> True
PyObject* cache8_write(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_write8 || n_args != 9) FIBQ_NONE;
  const Tensor *k = tensor(a[0]), *v = tensor(a[1]), *slots = tensor(a[2]);
  int64_t st, index;
  Pools p;
  HeadRows rk, rv;
  if (!k || !v || !slots || !int_arg(a[7], &st) || !int_arg(a[8], &index) || !pools(a + 3, index, &p))
    FIBQ_NONE;
  const int dt = dtype_code(*k);
  if (dt < 0 || !head_rows(k, k->scalar_type(), p.dev, &rk) || !head_rows(v, k->scalar_type(), p.dev, &rv) ||
      rv.n != rk.n || rk.H != p.H || rv.H != p.H || rk.d != p.d || rv.d != p.d ||
      !shaped(slots, at::kLong, {rk.n}) || slots->device() != p.dev)
    FIBQ_NONE;
  for (int i = 0; i < 4; ++i) {
    if (meets(rk, p.t[i]) || meets(rv, p.t[i]) || shared(slots, p.t[i])) FIBQ_NONE;
    for (int j = 0; j < i; ++j)
      if (shared(p.t[i], p.t[j])) FIBQ_NONE;
  }
  void* to[4];
  for (int i = 0; i < 4; ++i) to[i] = p.t[i]->data_ptr();
  const int64_t* ps = static_cast<const int64_t*>(ptr(*slots));
  int rc;
  {
    NoGil no_gil;
    rc = g_write8(rk.begin, rv.begin, dt, rk.n, rk.row, rk.head, rv.row, rv.head, ps, (int)p.H, (int)p.d,
                  (int)p.page, p.n_pages, p.codes, to[0], static_cast<float*>(to[1]), to[2],
                  static_cast<float*>(to[3]), reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_cache8_write");
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// attn_cache8(q, k_pages, k_scales, v_pages, v_scales, table, lens, starts, causal, scale,
//             workspace, out, stream, device) -> out
PyObject* attn_cache8(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_attn8 || n_args != 14) FIBQ_NONE;
  const Tensor *q = tensor(a[0]), *table = tensor(a[5]);
  int64_t st, index;
  Pools p;
  if (!q || q->dim() != 3 || !q->is_contiguous() || !table || table->dim() != 2 || !PyBool_Check(a[8]) ||
      !PyFloat_CheckExact(a[9]) || !int_arg(a[12], &st) || !int_arg(a[13], &index) ||
      !pools(a + 1, index, &p))
    FIBQ_NONE;
  const int64_t n_rows = q->size(0), Hq = q->size(1), n = table->size(0), max_pages = table->size(1);
  const int dt = dtype_code(*q);
  if (dt < 0 || q->device() != p.dev || q->size(2) != p.d || Hq < 1 || Hq % p.H != 0 || Hq / p.H > 16 ||
      max_pages >= (1LL << 30))
    FIBQ_NONE;
  const bool has_starts = a[7] != Py_None;
  const Tensor *cells = given(a[5], at::kInt, {n, max_pages}, p.dev), *lens = given(a[6], at::kInt, {n}, p.dev),
               *starts = has_starts ? given(a[7], at::kInt, {n + 1}, p.dev) : nullptr;
  if (!cells || !lens || (has_starts ? !starts : n_rows != n)) FIBQ_NONE;
  const int G = (int)(Hq / p.H);
  const int64_t need =
      (int64_t)g_attn8_ws(n, n_rows, (int)p.H, G, max_pages, (int)p.page, (int)p.d);
  Tensor ws, out;
  if (!workspace(a[10], need, p.dev, &ws)) FIBQ_NONE;
  if (a[11] != Py_None) {
    const Tensor* t = given(a[11], at::kFloat, {n_rows, Hq, p.d}, p.dev);
    if (!t) FIBQ_NONE;
    out = *t;
  }
  const Tensor* in[] = {q, p.t[0], p.t[1], p.t[2], p.t[3], cells, lens, starts};
  for (const Tensor* x : in)
    if (x && ((out.defined() && shared(x, &out)) || (ws.defined() && shared(x, &ws)))) FIBQ_NONE;
  if (out.defined() && ws.defined() && shared(&out, &ws)) FIBQ_NONE;
  const void *pq = ptr(*q), *kp = ptr(*p.t[0]), *vp = ptr(*p.t[2]);
  const float *ks = static_cast<const float*>(ptr(*p.t[1])), *vs = static_cast<const float*>(ptr(*p.t[3]));
  const int32_t *pt = static_cast<const int32_t*>(ptr(*cells)), *pl = static_cast<const int32_t*>(ptr(*lens)),
                *ps = starts ? static_cast<const int32_t*>(ptr(*starts)) : nullptr;
  const float scale = (float)PyFloat_AS_DOUBLE(a[9]);
  const bool causal = a[8] == Py_True;
  int rc;
  {
    NoGil no_gil;
    if (!ws.defined() && need > 0) ws = empty(p.dev, at::kByte, {need});
    if (!out.defined()) out = empty(p.dev, at::kFloat, {n_rows, Hq, p.d});
    rc = g_attn8(pq, dt, kp, ks, vp, vs, p.codes, pt, pl, ps, n, n_rows, (int)p.H, G, max_pages, (int)p.page,
                 p.n_pages, (int)p.d, causal, scale, static_cast<float*>(out.data_ptr()),
                 ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (size_t)ws.numel() : 0,
                 reinterpret_cast<void*>(st));
  }
  if (rc != FIBQ_OK) return raise_status(rc, "fibq_attn_cache8");
  return keep(a[11], out);
  END_HANDLE_TH_ERRORS
}

// bind_paged(rope, page_resize, its workspace_bytes, cache8_write, attn_cache8, its
// workspace_bytes): addresses
PyObject* bind_paged(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) {
    PyErr_SetString(PyExc_TypeError, "bind_paged takes six addresses");
    return nullptr;
  }
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_rope = reinterpret_cast<decltype(g_rope)>(p[0]);
  g_resize = reinterpret_cast<decltype(g_resize)>(p[1]);
  g_resize_ws = reinterpret_cast<decltype(g_resize_ws)>(p[2]);
  g_write8 = reinterpret_cast<decltype(g_write8)>(p[3]);
  g_attn8 = reinterpret_cast<decltype(g_attn8)>(p[4]);
  g_attn8_ws = reinterpret_cast<decltype(g_attn8_ws)>(p[5]);
  Py_RETURN_NONE;
}

// bind(encode, decode, attn_decode, attn_workspace_bytes, payload_bytes,
// check): addresses of the loaded library's entry points, and _check
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) {
    PyErr_SetString(PyExc_TypeError, "bind takes five addresses and a callable");
    return nullptr;
  }
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g_encode = reinterpret_cast<decltype(g_encode)>(p[0]);
  g_decode = reinterpret_cast<decltype(g_decode)>(p[1]);
  g_attn = reinterpret_cast<decltype(g_attn)>(p[2]);
  g_ws = reinterpret_cast<decltype(g_ws)>(p[3]);
  g_payload = reinterpret_cast<decltype(g_payload)>(p[4]);
  Py_INCREF(a[5]);
  Py_XSETREF(g_check, a[5]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
    {"encode", (PyCFunction)(void*)encode, METH_FASTCALL, nullptr},
    {"decode", (PyCFunction)(void*)decode, METH_FASTCALL, nullptr},
    {"attn", (PyCFunction)(void*)attn, METH_FASTCALL, nullptr},
    {"bind_serving", (PyCFunction)(void*)bind_serving, METH_FASTCALL, nullptr},
    {"attn_tree", (PyCFunction)(void*)attn_tree, METH_FASTCALL, nullptr},
    {"attn_accum", (PyCFunction)(void*)attn_accum, METH_FASTCALL, nullptr},
    {"accept", (PyCFunction)(void*)accept, METH_FASTCALL, nullptr},
    {"evict", (PyCFunction)(void*)evict, METH_FASTCALL, nullptr},
    {"bind_paged", (PyCFunction)(void*)bind_paged, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void*)rope, METH_FASTCALL, nullptr},
    {"page_resize", (PyCFunction)(void*)page_resize, METH_FASTCALL, nullptr},
    {"cache8_write", (PyCFunction)(void*)cache8_write, METH_FASTCALL, nullptr},
    {"attn_cache8", (PyCFunction)(void*)attn_cache8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr,
                      nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
