// Python module _pda_torch: the calls of include/pda_ops.h from torch tensors.
//
// A small call's kernels take 3 - 8 us, and reading the shapes, strides and
// pointers of up to 14 tensors from Python took 5 - 7 us of host time before each
// launch; from here it takes below 1 us. A function gets the entry's address, the stream, and
// the arguments of the binding's function of the same name. It returns the
// entry's status code, or None for arguments that it does not accept as they
// are: the binding's own checks then say what is wrong with them. It accepts only
// what these checks accept.

#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>
#include <initializer_list>

#include "pda_ops.h"

namespace {

struct Refused {};

struct Pointer {
  void* p = nullptr;
  c10::ScalarType type = c10::ScalarType::Undefined;
};

class Args {
 public:
  Args(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) : a_(a) { need(n == want); }

  static void need(bool ok) {
    if (!ok) throw Refused();
  }
  static int32_t int32(int64_t x) {
    need(x >= 0 && x <= INT_MAX);
    return (int32_t)x;
  }

  // Argument i, on the first tensor's device.
  const at::Tensor& tensor(int i) {
    need(THPVariable_CheckExact(a_[i]));
    const at::Tensor& t = THPVariable_Unpack(a_[i]);
    need(t.is_cuda() && t.layout() == c10::kStrided);
    if (index_ < 0) index_ = t.get_device();
    need(t.get_device() == index_);
    return t;
  }
  bool none(int i) const { return a_[i] == Py_None; }

  Pointer contiguous(int i, c10::IntArrayRef shape) {
    const at::Tensor& t = tensor(i);
    need(t.sizes() == shape && t.is_contiguous());
    return {t.mutable_data_ptr(), t.scalar_type()};
  }
  template <typename T = void>
  T* array(int i, c10::ScalarType type, std::initializer_list<int64_t> shape) {
    const Pointer x = contiguous(i, shape);
    need(x.type == type);
    return static_cast<T*>(x.p);
  }
  template <typename T = void>
  T* optional(int i, c10::ScalarType type, std::initializer_list<int64_t> shape) {
    return none(i) ? nullptr : array<T>(i, type, shape);
  }

  // [T, H, D], a token's heads contiguous; *stride: elements between tokens (0: one token).
  Pointer heads(int i, c10::IntArrayRef shape, int64_t* stride) {
    const at::Tensor& t = tensor(i);
    const auto n = t.sizes(), s = t.strides();
    need(n == shape && n.size() == 3 && s[2] == 1 && (s[1] == n[2] || n[1] == 1));
    need(n[0] <= 1 || s[0] >= n[1] * n[2]);
    *stride = n[0] <= 1 ? 0 : s[0];
    return {t.mutable_data_ptr(), t.scalar_type()};
  }
  // [T, V], a row's words contiguous.
  Pointer rows(int i, c10::IntArrayRef shape, int64_t* stride) {
    const at::Tensor& t = tensor(i);
    const auto n = t.sizes(), s = t.strides();
    need(n == shape && n.size() == 2 && (s[1] == 1 || n[1] <= 1) && (n[0] <= 1 || s[0] >= n[1]));
    *stride = n[0] <= 1 ? 0 : s[0];
    return {t.mutable_data_ptr(), t.scalar_type()};
  }

  void* address(int i) {
    void* p = PyLong_AsVoidPtr(a_[i]);
    clear();
    return p;
  }
  float number(int i) {
    const double x = PyFloat_AsDouble(a_[i]);
    clear();
    return (float)x;
  }
  int32_t integer(int i) {
    const long x = PyLong_AsLong(a_[i]);
    clear();
    need(x >= INT_MIN && x <= INT_MAX);
    return (int32_t)x;
  }
  bool truth(int i) {
    const int x = PyObject_IsTrue(a_[i]);
    clear();
    return x == 1;
  }

 private:
  static void clear() {
    if (!PyErr_Occurred()) return;
    PyErr_Clear();
    throw Refused();
  }
  PyObject* const* a_;
  int64_t index_ = -1;
};

int32_t float_code(c10::ScalarType t) {
  if (t == c10::kFloat) return PDA_DTYPE_F32;
  Args::need(t == c10::kBFloat16);
  return PDA_DTYPE_BF16;
}
int32_t cache_code(c10::ScalarType t) {
  return t == c10::kByte || t == c10::kFloat8_e4m3fn ? (int32_t)PDA_DTYPE_FP8_E4M3 : float_code(t);
}

// What the three calls of the norm and rotation share: q, k, weights, cos_sin,
// positions (arguments at .. at + 5, with v at `v` or none).
struct Rope {
  pdaops_rope_problem pr = {};
  int64_t T, hq, hkv, d;
  Pointer q, k, v, wq, wk;
  const float* table;

  Rope(Args& a, int iq, int ik, int iv, int iw, int itable) {
    const auto n = a.tensor(iq).sizes(), m = a.tensor(ik).sizes();
    Args::need(n.size() == 3 && m.size() == 3 && m[0] == n[0] && m[2] == n[2]);
    T = n[0], hq = n[1], hkv = m[1], d = n[2];
    q = a.heads(iq, n, &pr.q_stride);
    k = a.heads(ik, m, &pr.k_stride);
    Args::need(k.type == q.type);
    if (iv >= 0) {
      v = a.heads(iv, m, &pr.v_stride);
      Args::need(v.type == q.type);
    }
    Args::need(a.none(iw) == a.none(iw + 1));
    pr.weight_dtype = PDA_DTYPE_F32;
    if (!a.none(iw)) {
      wq = a.contiguous(iw, {d});
      wk = a.contiguous(iw + 1, {d});
      Args::need(wq.type == wk.type);
      pr.weight_dtype = float_code(wq.type);
    }
    const auto p = a.tensor(itable).sizes();
    Args::need(p.size() == 2);
    table = a.array<float>(itable, c10::kFloat, {p[0], p[1]});
    pr.num_tokens = Args::int32(T);
    pr.num_q_heads = Args::int32(hq);
    pr.num_kv_heads = Args::int32(hkv);
    pr.head_dim = Args::int32(d);
    pr.rotary_dim = Args::int32(p[1]);
    pr.max_positions = Args::int32(p[0]);
    pr.dtype = pr.out_dtype = float_code(q.type);
  }
};

// The entry, without the interpreter's lock (a workspace that grows waits for its stream).
template <typename F, typename... A>
int enter(void* entry, A... a) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<F>(entry)(a...);
  Py_END_ALLOW_THREADS
  return rc;
}

int append(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 19);
  enum { ENTRY, STREAM, Q, K, V, WQ, WK, TABLE, OFFSETS, KC, VC, SCALES, BLOCKS, LENS, OUT, EPS, INTER, POS, MOST };
  Rope r(a, Q, K, V, WQ, TABLE);
  r.pr.out_dtype = float_code(a.heads(OUT, {r.T, r.hq, r.d}, &r.pr.q_out_stride).type);
  r.pr.eps = a.number(EPS);
  r.pr.interleaved = a.truth(INTER);
  const auto c = a.tensor(KC).sizes(), b = a.tensor(BLOCKS).sizes();
  Args::need(c.size() == 4 && c[1] == r.hkv && c[3] == r.d && b.size() == 2);
  const Pointer kc = a.contiguous(KC, c), vc = a.contiguous(VC, {c[0], c[1], c[3], c[2]});
  pdaops_cache ca = {Args::int32(b[0]), Args::int32(c[2]), Args::int32(b[1]), a.integer(MOST), c[0], cache_code(kc.type)};
  Args::need(cache_code(vc.type) == ca.kv_dtype && (ca.kv_dtype != PDA_DTYPE_FP8_E4M3 || !a.none(SCALES)));
  float* scales = a.optional<float>(SCALES, c10::kFloat, {2, c[0], c[1]});
  const auto* blocks = a.array<int32_t>(BLOCKS, c10::kInt, {b[0], b[1]});
  const auto* lens = a.array<int32_t>(LENS, c10::kInt, {b[0]});
  const auto* offsets = a.optional<int32_t>(OFFSETS, c10::kInt, {b[0] + 1});
  const auto* pos = a.optional<int32_t>(POS, c10::kInt, {r.T});
  int64_t ignored;
  return enter<decltype(&pdaops_paged_qk_norm_rope_append)>(
      a.address(ENTRY), r.q.p, r.k.p, r.v.p, r.wq.p, r.wk.p, r.table, pos, offsets, a.heads(OUT, {r.T, r.hq, r.d}, &ignored).p,
      kc.p, vc.p, scales, blocks, lens, &r.pr, &ca, static_cast<hipStream_t>(a.address(STREAM)));
}

int forward(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 12);
  enum { ENTRY, STREAM, Q, K, WQ, WK, TABLE, POS, QOUT, KOUT, EPS, INTER };
  Rope r(a, Q, K, -1, WQ, TABLE);
  const Pointer qo = a.heads(QOUT, {r.T, r.hq, r.d}, &r.pr.q_out_stride), ko = a.heads(KOUT, {r.T, r.hkv, r.d}, &r.pr.k_out_stride);
  r.pr.out_dtype = float_code(qo.type);
  Args::need(ko.type == qo.type);
  r.pr.eps = a.number(EPS);
  r.pr.interleaved = a.truth(INTER);
  const auto* pos = a.array<int32_t>(POS, c10::kInt, {r.T});
  return enter<decltype(&pdaops_qk_norm_rope)>(a.address(ENTRY), r.q.p, r.k.p, r.wq.p, r.wk.p, r.table, pos, qo.p, ko.p, &r.pr,
                                               static_cast<hipStream_t>(a.address(STREAM)));
}

int backward(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 16);
  enum { ENTRY, STREAM, Q, K, WQ, WK, TABLE, POS, GQ, GK, DQ, DK, DWQ, DWK, EPS, INTER };
  Rope r(a, Q, K, -1, WQ, TABLE);
  const Pointer gq = a.heads(GQ, {r.T, r.hq, r.d}, &r.pr.q_out_stride), gk = a.heads(GK, {r.T, r.hkv, r.d}, &r.pr.k_out_stride);
  const Pointer dq = a.heads(DQ, {r.T, r.hq, r.d}, &r.pr.grad_q_stride), dk = a.heads(DK, {r.T, r.hkv, r.d}, &r.pr.grad_k_stride);
  Args::need(gq.type == r.q.type && gk.type == r.q.type && dq.type == r.q.type && dk.type == r.q.type);
  r.pr.eps = a.number(EPS);
  r.pr.interleaved = a.truth(INTER);
  Args::need(!r.wq.p || (!a.none(DWQ) && !a.none(DWK)));
  float* dwq = a.optional<float>(DWQ, c10::kFloat, {r.d});
  float* dwk = a.optional<float>(DWK, c10::kFloat, {r.d});
  const auto* pos = a.array<int32_t>(POS, c10::kInt, {r.T});
  return enter<decltype(&pdaops_qk_norm_rope_backward)>(a.address(ENTRY), r.q.p, r.k.p, r.wq.p, r.wk.p, r.table, pos, gq.p, gk.p,
                                                        dq.p, dk.p, dwq, dwk, &r.pr, static_cast<hipStream_t>(a.address(STREAM)));
}

struct Logits {
  pdaops_logits_problem pr = {};
  int64_t T, V;
  Pointer z, y;

  Logits(Args& a, int iz, int iy) {
    const auto n = a.tensor(iz).sizes();
    Args::need(n.size() == 2);
    T = n[0], V = n[1];
    z = a.rows(iz, n, &pr.row_stride);
    y = a.contiguous(iy, {T});
    Args::need(y.type == c10::kLong || y.type == c10::kInt);
    pr.num_tokens = Args::int32(T);
    pr.vocab = Args::int32(V);
    pr.dtype = float_code(z.type);
    pr.targets_int64 = y.type == c10::kLong;
  }
};

int logprobs(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 7);
  enum { ENTRY, STREAM, LOGITS, TARGETS, LOGP, ENT, TEMP };
  Logits l(a, LOGITS, TARGETS);
  l.pr.temperature = a.number(TEMP);
  float* lp = a.array<float>(LOGP, c10::kFloat, {l.T});
  float* ent = a.optional<float>(ENT, c10::kFloat, {l.T});
  return enter<decltype(&pdaops_token_logprobs)>(a.address(ENTRY), l.z.p, l.y.p, lp, ent, &l.pr,
                                                 static_cast<hipStream_t>(a.address(STREAM)));
}

int policy(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 19);
  enum { ENTRY, STREAM, LOGITS, TARGETS, OLD, ADV, WEIGHT, STATS, GRAD, LOGP, ENT, REF, LOW, HIGH, DUAL, KL, ENTC, TEMP, SCALE };
  Logits l(a, LOGITS, TARGETS);
  l.pr.temperature = a.number(TEMP);
  pdaops_policy_options op = {a.number(LOW), a.number(HIGH), a.number(DUAL), a.number(KL), a.number(ENTC), a.number(SCALE), 0};
  const auto f = c10::kFloat;
  const float* old = a.array<float>(OLD, f, {l.T});
  const float* adv = a.array<float>(ADV, f, {l.T});
  const float* w = a.array<float>(WEIGHT, f, {l.T});
  float* stats = a.array<float>(STATS, f, {8});
  Pointer g;
  if (!a.none(GRAD)) {
    g = a.rows(GRAD, {l.T, l.V}, &op.dlogits_stride);
    Args::need(g.type == l.z.type);
  }
  float* lp = a.optional<float>(LOGP, f, {l.T});
  float* ent = a.optional<float>(ENT, f, {l.T});
  const float* ref = a.optional<float>(REF, f, {l.T});
  return enter<decltype(&pdaops_policy_loss)>(a.address(ENTRY), l.z.p, l.y.p, old, ref, adv, w, stats, g.p, lp, ent, &l.pr, &op,
                                              static_cast<hipStream_t>(a.address(STREAM)));
}

template <int (*F)(PyObject* const*, Py_ssize_t)>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int rc;
  try {
    rc = F(args, n);
  } catch (...) {  // refused, or torch could not give a tensor's memory
    Py_RETURN_NONE;
  }
  return PyLong_FromLong(rc);
}

template <int (*F)(PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<append>("paged_qk_norm_rope_append"), method<forward>("qk_norm_rope"),
                         method<backward>("qk_norm_rope_backward"), method<logprobs>("token_logprobs"),
                         method<policy>("policy_loss"), {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pda_torch", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__pda_torch() { return PyModule_Create(&module); }
