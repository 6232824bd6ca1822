// Argument marshalling of the rotary calls, the cache reads and prompts over an e4m3 cache as a CPython extension: checks, output tensors and the call of the C ABI in one step.  A decode
// step's device work takes 4 us, and a call through ctypes with the same checks 18; here it takes 7.  Raises AssertionError for what the wrappers check, and
// returns the library's code (a negative int) where a call is refused.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "../../include/mala.h"

namespace {

struct Refused : std::exception {
  const char* what_;
  explicit Refused(const char* w) : what_(w) {}
  const char* what() const noexcept override { return what_; }
};
struct PythonError {};
void require(bool ok, const char* what) {
  if (!ok) throw Refused(what);
}

// One of a call's arguments; None: no tensor
struct Arg {
  const at::Tensor* t = nullptr;
  explicit Arg(PyObject* o) {
    if (o == Py_None) return;
    require(THPVariable_Check(o), "expects a tensor");
    t = &THPVariable_Unpack(o);
  }
  explicit operator bool() const { return t != nullptr; }
  const at::Tensor* operator->() const { return t; }
  const at::Tensor& operator*() const { return *t; }
  void* data() const { return t ? t->data_ptr() : nullptr; }
};
const at::Tensor& tensor(PyObject* o) {
  Arg a(o);
  require((bool)a, "expects a tensor");
  return *a.t;
}

double number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw PythonError();
  return x;
}
bool truth(PyObject* o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw PythonError();
  return x != 0;
}
int whole(PyObject* o) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) throw PythonError();
  require(x >= INT32_MIN && x <= INT32_MAX, "expects a 32-bit number");
  return (int)x;
}

// The current stream of the current device, on which all tensors have to lie (a kernel given another one's memory faults)
struct Here {
  int device;
  Here() : device(c10::cuda::current_device()) {}
  void on(const at::Tensor& t) const { require(t.is_cuda() && t.get_device() == device, "expects tensors on the current device"); }
  void on(const Arg& a) const {
    if (a) on(*a);
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(device).stream(); }
};

int size(const at::Tensor& t, int dim) {
  const int64_t n = t.size(dim);
  require(n <= INT32_MAX, "sizes count in 32 bits");
  return (int)n;
}

// bf16 (or 8-bit) views [B,N,H,d] and rows [rows,H,d], last dim contiguous
void check_rows(const at::Tensor& t, int dims, bool fp8) {
  const bool type = fp8 ? t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e4m3fn : t.scalar_type() == at::kBFloat16;
  require(type && t.dim() == dims && t.stride(dims - 1) == 1, fp8 ? "expects 8-bit [B,N,H,d], last dim contiguous" : "expects bf16 [B,N,H,d] or [rows,H,d], last dim contiguous");
}
mala_tin in4(const at::Tensor& t, bool fp8 = false) {
  check_rows(t, 4, fp8);
  return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}
mala_tout out4(const at::Tensor& t, bool fp8 = false) {
  check_rows(t, 4, fp8);
  return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}
mala_tin in3(const at::Tensor& t) {
  check_rows(t, 3, false);
  return {t.data_ptr(), 0, t.stride(0), t.stride(1)};
}
mala_tout out3(const at::Tensor& t) {
  check_rows(t, 3, false);
  return {t.data_ptr(), 0, t.stride(0), t.stride(1)};
}

void ints(const at::Tensor& t) { require(t.scalar_type() == at::kInt && t.is_contiguous(), "expects contiguous int32 tensors"); }
void check_scales(const at::Tensor& t, int64_t num_pages, int64_t Hkv, int64_t page_size) {
  require(t.scalar_type() == at::kFloat && t.is_contiguous() && t.dim() == 3 && t.size(0) == num_pages && t.size(1) == Hkv && t.size(2) == (page_size < 128 ? 1 : page_size / 128),
          "expects fp32 scales [num_pages, Hkv, max(1, page_size/128)]");
}

// A new tensor for rotated rows (dense, whatever wider tensor x is a part of), or the given one
at::Tensor like(const at::Tensor& x, const Arg& out) {
  if (!out) return at::empty_like(x);
  require(out->sizes() == x.sizes(), "expects an output of its input's shape");
  return *out;
}

// inv_freq, interleaved, magnitude, eps (None: no norm), q_weight, k_weight
struct Rule {
  mala_rotary rotary;
  mala_head_norm norm;
  bool normed;
  Arg q_weight, k_weight;
  static constexpr int kArgs = 6;
  Rule(PyObject* const* a, int64_t d, const Here& here) : normed(a[3] != Py_None), q_weight(a[4]), k_weight(a[5]) {
    const at::Tensor& f = tensor(a[0]);
    require(f.scalar_type() == at::kDouble && f.dim() == 1 && f.is_contiguous(), "expects frequencies in fp64");
    require(!q_weight || !k_weight || q_weight->scalar_type() == k_weight->scalar_type(), "expects weights of one type");
    here.on(f);
    rotary = {f.data_ptr<double>(), 2 * size(f, 0), truth(a[1]), (float)number(a[2])};
    norm = {};
    if (!normed) return;
    for (const Arg* w : {&q_weight, &k_weight}) {
      if (!*w) continue;
      here.on(*w);
      require((*w)->dim() == 1 && (*w)->size(0) == d && (*w)->is_contiguous() && ((*w)->scalar_type() == at::kBFloat16 || (*w)->scalar_type() == at::kFloat), "a weight per column of a head");
      norm.weights_fp32 = (*w)->scalar_type() == at::kFloat;
    }
    norm.q_weight = q_weight.data();
    norm.k_weight = k_weight.data();
    norm.eps = (float)number(a[3]);
  }
  const mala_head_norm* head_norm() const { return normed ? &norm : nullptr; }
};

const mala_tin kNoIn = {nullptr, 0, 0, 0};
const mala_tout kNoOut = {nullptr, 0, 0, 0};

// Sizes that q [B,Nq,Hq,d], k [B,Nk,Hkv,d] (or none) and their positions or offsets agree on
struct Call {
  int B, Nq, Nk, Hq, Hkv = 0, d, sequences = 0;
  Arg positions, cu_q, cu_k;
  Call(const at::Tensor& q, const Arg& k, PyObject* positions_, PyObject* cu_q_, PyObject* cu_k_, const Here& here) : positions(positions_), cu_q(cu_q_), cu_k(cu_k_) {
    require(q.dim() == 4, "expects q [B,N,H,d]");
    B = size(q, 0); Nq = Nk = size(q, 1); Hq = size(q, 2); d = size(q, 3);
    here.on(q);
    if (k) {
      here.on(k);
      require(k->dim() == 4 && k->size(0) == B && k->size(3) == d, "expects k of q's batch and head size");
      Nk = size(*k, 1);
      Hkv = size(*k, 2);
    }
    if (positions) {
      here.on(positions);
      ints(*positions);
      require(positions->dim() == 2 && positions->size(0) == B && positions->size(1) == Nk && Nk >= Nq, "expects a position per row of k (or of q, without keys)");
    }
    if (cu_q) {
      require((bool)cu_k && B == 1, "packed sequences: [1,total,H,d] and offsets of both");
      here.on(cu_q);
      here.on(cu_k);
      ints(*cu_q);
      ints(*cu_k);
      require(cu_q->dim() == 1 && cu_k->dim() == 1 && cu_q->size(0) == cu_k->size(0) && cu_q->size(0) >= 1, "expects offsets of as many sequences");
      sequences = size(*cu_q, 0) - 1;
    }
  }
};

PyObject* code(int rc) { return PyLong_FromLong(rc); }
PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
template <int N>
PyObject* tuple(const at::Tensor (&t)[N]) {
  PyObject* r = PyTuple_New(N);
  if (!r) throw PythonError();
  for (int i = 0; i < N; ++i) {
    PyObject* x = wrap(t[i]);
    if (!x) {
      Py_DECREF(r);
      throw PythonError();
    }
    PyTuple_SET_ITEM(r, i, x);
  }
  return r;
}

template <PyObject* (*F)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_Format(PyExc_TypeError, "expects %d arguments, got %zd", kArgs, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_AssertionError, e.what());
  } catch (const PythonError&) {
  } catch (...) {                          // (torch's own: no memory left, ...)
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

// q, k, rule, positions, cu_q, cu_k, q_out, k_out
PyObject* rotary(PyObject* const* a) {
  const Here here;
  const at::Tensor& q = tensor(a[0]);
  const Arg k(a[1]), q_out(a[11]), k_out(a[12]);
  const Call c(q, k, a[8], a[9], a[10], here);
  const Rule r(a + 2, c.d, here);
  here.on(q_out);
  here.on(k_out);
  at::Tensor out[2] = {like(q, q_out), k ? like(*k, k_out) : at::Tensor()};
  const mala_tin ki = k ? in4(*k) : kNoIn;
  const mala_tout ko = k ? out4(out[1]) : kNoOut;
  const int rc = c.cu_q ? mala_rotary_fwd_varlen(in4(q), ki, (const int32_t*)c.cu_q.data(), (const int32_t*)c.cu_k.data(), &r.rotary, r.head_norm(), out4(out[0]), ko, c.sequences,
                                                 c.Hq, c.Hkv, c.Nq, c.Nk, c.d, here.stream())
                        : mala_rotary_fwd(in4(q), ki, (const int32_t*)c.positions.data(), &r.rotary, r.head_norm(), out4(out[0]), ko, c.B, c.Nq, c.Nk, c.Hq, c.Hkv, c.d, here.stream());
  return rc != MALA_OK ? code(rc) : tuple(out);
}

// dq, dk, rule, positions, cu_q, cu_k, q, k, dq_out, dk_out, weights
PyObject* rotary_bwd(PyObject* const* a) {
  const Here here;
  const at::Tensor& dq = tensor(a[0]);
  const Arg dk(a[1]), q(a[11]), k(a[12]), dq_out(a[13]), dk_out(a[14]);
  const bool weights = truth(a[15]);
  const Call c(dq, dk, a[8], a[9], a[10], here);
  const Rule r(a + 2, c.d, here);
  if (r.normed) {
    require(q && q->sizes() == dq.sizes() && (!dk || (k && k->sizes() == dk->sizes())), "with a norm: q and k");
    here.on(q);
    if (dk) here.on(k);
  }
  here.on(dq_out);
  here.on(dk_out);
  at::Tensor out[4] = {like(dq, dq_out), dk ? like(*dk, dk_out) : at::Tensor(), at::Tensor(), at::Tensor()}, ws;
  const auto fp32 = dq.options().dtype(at::kFloat);
  if (r.normed && weights && r.q_weight) out[2] = at::empty({c.d}, fp32);
  if (r.normed && weights && r.k_weight && dk) out[3] = at::empty({c.d}, fp32);
  size_t bytes = 0;
  if (out[2].defined() || out[3].defined()) {
    bytes = mala_rotary_workspace_bytes(c.d);
    bytes = bytes < 256 ? 256 : bytes;
    ws = at::empty({(int64_t)bytes}, dq.options().dtype(at::kByte));
  }
  float* const dwq = out[2].defined() ? out[2].data_ptr<float>() : nullptr;
  float* const dwk = out[3].defined() ? out[3].data_ptr<float>() : nullptr;
  void* const wsp = ws.defined() ? ws.data_ptr() : nullptr;
  const mala_tin qi = r.normed ? in4(*q) : kNoIn, ki = r.normed && dk ? in4(*k) : kNoIn, dki = dk ? in4(*dk) : kNoIn;
  const mala_tout dko = dk ? out4(out[1]) : kNoOut;
  const int rc = c.cu_q ? mala_rotary_bwd_varlen(in4(dq), dki, qi, ki, (const int32_t*)c.cu_q.data(), (const int32_t*)c.cu_k.data(), &r.rotary, r.head_norm(), out4(out[0]), dko, dwq,
                                                 dwk, c.sequences, c.Hq, c.Hkv, c.Nq, c.Nk, c.d, wsp, bytes, here.stream())
                        : mala_rotary_bwd(in4(dq), dki, qi, ki, (const int32_t*)c.positions.data(), &r.rotary, r.head_norm(), out4(out[0]), dko, dwq, dwk, c.B, c.Nq, c.Nk, c.Hq, c.Hkv,
                                          c.d, wsp, bytes, here.stream());
  return rc != MALA_OK ? code(rc) : tuple(out);
}

// q, k, v, positions, slots, kpages, vpages, kscale, vscale (None: bf16 pages), rule, q_out
PyObject* rotary_write(PyObject* const* a) {
  const Here here;
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &positions = tensor(a[3]), &slots = tensor(a[4]), &kp = tensor(a[5]), &vp = tensor(a[6]);
  const Arg ks(a[7]), vs(a[8]), q_out(a[15]);
  const bool fp8 = (bool)ks;
  require(q.dim() == 3 && k.dim() == 3 && kp.dim() == 4, "expects rows [rows,H,d] and pages [num_pages, page_size, Hkv, d]");
  const int rows = size(q, 0), Hq = size(q, 1), d = size(q, 2), Hkv = size(k, 1), num_pages = size(kp, 0), page_size = size(kp, 1);
  require(k.sizes() == v.sizes() && k.size(0) == rows && k.size(2) == d, "expects k, v [rows,Hkv,d]");
  require(slots.scalar_type() == at::kLong && slots.is_contiguous() && slots.dim() == 1 && slots.size(0) == rows, "expects slots int64 [rows]");
  ints(positions);
  require(positions.dim() == 1 && positions.size(0) == rows, "expects positions int32 [rows]");
  require(kp.sizes() == vp.sizes() && kp.size(2) == Hkv && kp.size(3) == d, "expects pages [num_pages, page_size, Hkv, d]");
  const Rule r(a + 9, d, here);
  for (const at::Tensor* t : {&q, &k, &v, &positions, &slots, &kp, &vp}) here.on(*t);
  here.on(q_out);
  if (fp8) {
    require((bool)vs, "expects scales of keys and of values");
    check_scales(*ks, num_pages, Hkv, page_size);
    check_scales(*vs, num_pages, Hkv, page_size);
    here.on(ks);
    here.on(vs);
  }
  const at::Tensor qo = like(q, q_out);
  const int rc = fp8 ? mala_rotary_write_fp8(in3(q), in3(k), in3(v), positions.data_ptr<int32_t>(), slots.data_ptr<int64_t>(), &r.rotary, r.head_norm(), out3(qo), out4(kp, true),
                                             out4(vp, true), ks->data_ptr<float>(), vs->data_ptr<float>(), rows, Hq, Hkv, num_pages, page_size, d, here.stream())
                     : mala_rotary_write(in3(q), in3(k), in3(v), positions.data_ptr<int32_t>(), slots.data_ptr<int64_t>(), &r.rotary, r.head_norm(), out3(qo), out4(kp), out4(vp), rows,
                                         Hq, Hkv, num_pages, page_size, d, here.stream());
  return rc != MALA_OK ? code(rc) : wrap(qo);
}

// kpages, vpages, kscale, vscale (None: bf16 pages), block_table, seqlens, rows
PyObject* cache_read(PyObject* const* a) {
  const Here here;
  const at::Tensor &kp = tensor(a[0]), &vp = tensor(a[1]), &table = tensor(a[4]), &lens = tensor(a[5]);
  const Arg ks(a[2]), vs(a[3]);
  const int rows = whole(a[6]);
  const bool fp8 = (bool)ks;
  require(kp.dim() == 4 && kp.sizes() == vp.sizes() && table.dim() == 2 && lens.dim() == 1 && rows >= 0, "expects pages [num_pages, page_size, Hkv, d], a block table and lengths");
  const int num_pages = size(kp, 0), page_size = size(kp, 1), Hkv = size(kp, 2), d = size(kp, 3), B = size(table, 0), width = size(table, 1);
  require(lens.size(0) == B, "expects a length per row of the block table");
  ints(table);
  ints(lens);
  for (const at::Tensor* t : {&kp, &vp, &table, &lens}) here.on(*t);
  if (fp8) {
    require((bool)vs, "expects scales of keys and of values");
    check_scales(*ks, num_pages, Hkv, page_size);
    check_scales(*vs, num_pages, Hkv, page_size);
    here.on(ks);
    here.on(vs);
  }
  const auto bf16 = kp.options().dtype(at::kBFloat16);
  const at::Tensor out[3] = {at::empty({1, rows, Hkv, d}, bf16), at::empty({1, rows, Hkv, d}, bf16), at::empty({B + 1}, lens.options())};
  const int rc = fp8 ? mala_cache_read_fp8(in4(kp, true), in4(vp, true), ks->data_ptr<float>(), vs->data_ptr<float>(), table.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), out4(out[0]),
                                           out4(out[1]), out[2].data_ptr<int32_t>(), B, Hkv, num_pages, page_size, width, rows, d, here.stream())
                     : mala_cache_read(in4(kp), in4(vp), table.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), out4(out[0]), out4(out[1]), out[2].data_ptr<int32_t>(), B, Hkv, num_pages,
                                       page_size, width, rows, d, here.stream());
  return rc != MALA_OK ? code(rc) : tuple(out);
}

// q, kpages8, vpages8, kscale, vscale, cu_seqlens_q, block_table, seqlens_k, max_seqlen_q, total_k, scale, tau, causal, num_splits (None: see the wrapper), ws, and the
// telemetry's three tensors (None: no telemetry)
PyObject* fwd_paged_fp8(PyObject* const* a) {
  const Here here;
  const at::Tensor &q = tensor(a[0]), &kp = tensor(a[1]), &vp = tensor(a[2]), &ks = tensor(a[3]), &vs = tensor(a[4]), &cu = tensor(a[5]), &table = tensor(a[6]), &lens = tensor(a[7]);
  const int max_q = whole(a[8]), total_k = whole(a[9]), causal = truth(a[12]);
  const float scale = (float)number(a[10]), tau = (float)number(a[11]);
  const Arg ws_given(a[14]), retained(a[15]), bitmask(a[16]), totals(a[17]);
  require(q.dim() == 4 && q.size(0) == 1 && kp.dim() == 4 && table.dim() == 2, "expects q [1,total_q,Hq,d], pages [num_pages, page_size, Hkv, d] and a block table");
  const int total_q = size(q, 1), Hq = size(q, 2), d = size(q, 3), num_pages = size(kp, 0), page_size = size(kp, 1), Hkv = size(kp, 2), B = size(table, 0), width = size(table, 1);
  ints(cu);
  ints(table);
  ints(lens);
  require(cu.dim() == 1 && cu.size(0) == B + 1 && lens.dim() == 1 && lens.size(0) == B, "expects offsets and lengths of the block table's sequences");
  require(kp.sizes() == vp.sizes() && kp.size(3) == d, "expects pages of q's head size");
  check_scales(ks, num_pages, Hkv, page_size);
  check_scales(vs, num_pages, Hkv, page_size);
  for (const at::Tensor* t : {&q, &kp, &vp, &ks, &vs, &cu, &table, &lens}) here.on(*t);
  here.on(ws_given);
  require(!ws_given || (ws_given->scalar_type() == at::kByte && ws_given->is_contiguous()), "expects a workspace of bytes");
  int splits = 1;
  if (a[13] != Py_None) {
    splits = whole(a[13]);
  } else if (tau == 0.f && !ws_given) {
    const int64_t room = (int64_t)width * page_size;
    splits = mala_paged_fp8_suggest_splits(B, Hq, max_q, (int)(room < total_k ? room : total_k), total_k, 0);
    if (splits < 1) splits = 1;            // (lengths that the call refuses)
  }
  const mala_tin qi = in4(q), ki = in4(kp, true), vi = in4(vp, true);
  const at::Tensor o = at::empty_like(q), lse = at::empty({Hq, total_q}, q.options().dtype(at::kFloat));
  at::Tensor ws;
  if (!ws_given) {
    const size_t need = mala_paged_fp8_split_workspace_bytes(B, Hq, Hkv, max_q, total_k, d, splits);
    ws = at::empty({(int64_t)(need < 256 ? 256 : need)}, q.options().dtype(at::kByte));
  } else {
    ws = *ws_given;
  }
  const mala_stats st = {(uint32_t*)retained.data(), (uint32_t*)bitmask.data(), (uint64_t*)totals.data()};
  const int rc = mala_fwd_paged_fp8_split(qi, ki, vi, ks.data_ptr<float>(), vs.data_ptr<float>(), cu.data_ptr<int32_t>(), table.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), out4(o),
                                          lse.data_ptr<float>(), totals ? &st : nullptr, B, Hq, Hkv, total_q, max_q, total_k, num_pages, page_size, width, d, causal, scale, tau, splits,
                                          ws.data_ptr(), (size_t)ws.numel(), here.stream());
  const at::Tensor out[2] = {o, lse};
  return rc != MALA_OK ? code(rc) : tuple(out);
}

PyMethodDef methods[] = {{"rotary", (PyCFunction)(void*)entry<rotary, 13>, METH_FASTCALL, nullptr},
                         {"rotary_bwd", (PyCFunction)(void*)entry<rotary_bwd, 16>, METH_FASTCALL, nullptr},
                         {"rotary_write", (PyCFunction)(void*)entry<rotary_write, 16>, METH_FASTCALL, nullptr},
                         {"cache_read", (PyCFunction)(void*)entry<cache_read, 7>, METH_FASTCALL, nullptr},
                         {"fwd_paged_fp8", (PyCFunction)(void*)entry<fwd_paged_fp8, 18>, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of the rotary calls, the cache reads and prompts over an e4m3 cache.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
