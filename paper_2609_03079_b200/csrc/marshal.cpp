// Argument marshalling of the per-token calls for Python: takes tensors as they are, checks them, reads their pointers, strides
// and the current stream, and calls the C ABI.  The same through ctypes costs 8 to 10 microseconds a call, several times what
// the smallest kernels behind these calls take; here it is under one.  Holds no state and no arithmetic.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/leanstream.h"

namespace {

decltype(&ls_paged_kv_append) f_append = nullptr;
decltype(&ls_paged_kv_attend) f_attend = nullptr;
decltype(&ls_block_norm) f_norm = nullptr;
decltype(&ls_paged_kv4_append) f_append4 = nullptr;
decltype(&ls_paged_kv4_attend) f_attend4 = nullptr;
decltype(&ls_paged_kv4_read) f_read4 = nullptr;

struct Plan {  // what the checks need to know of a paged cache
  void* handle;  // ls_paged_kv or ls_paged_kv4, by the capsule's name
  int device;
  at::ScalarType dtype;
  int64_t heads, kv_heads, dim, page;
};

struct Refusal { const char* what; };  // thrown and caught in this file only

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refusal{what};
  return THPVariable_Unpack(o);
}
void need(bool ok, const char* what) {
  if (!ok) throw Refusal{what};
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refusal{nullptr};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refusal{nullptr};
  return v;
}
int32_t as32(long long v) {
  need(v >= INT32_MIN && v <= INT32_MAX, "a size does not fit 32 bits");
  return (int32_t)v;
}
void* stream_of(PyObject* o, int device) {
  if (o == Py_None) return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  return (void*)(uintptr_t)integer(o);
}
// A dense int32 tensor on the device.
const int32_t* ids(const at::Tensor& t, int device, const char* what) {
  need(t.scalar_type() == at::kInt && t.is_cuda() && t.get_device() == device && t.is_contiguous(), what);
  return static_cast<const int32_t*>(t.data_ptr());
}
// [tokens, heads, dim] or [sequences, tokens, heads, dim] with heads and components side by side: its token stride.
int64_t token_stride(const Plan& p, const at::Tensor& t, int64_t heads, const char* what) {
  const auto sz = t.sizes(), st = t.strides();
  const int64_t n = t.dim();
  need(t.scalar_type() == p.dtype && t.is_cuda() && t.get_device() == p.device && (n == 3 || n == 4) && sz[n - 1] == p.dim && sz[n - 2] == heads &&
           st[n - 1] == 1 && (heads == 1 || st[n - 2] == p.dim),
       what);
  if (n == 4 && sz[1] > 1) {
    need(sz[0] <= 1 || st[0] == sz[1] * st[1], what);
    return st[1];
  }
  return sz[0] > 1 ? st[0] : heads * p.dim;  // (a single token has no stride)
}
struct Table { const int32_t* at; int32_t rows, width; int64_t stride; };
Table table_of(const Plan& p, const at::Tensor& t) {
  need(t.scalar_type() == at::kInt && t.is_cuda() && t.get_device() == p.device && t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1),
       "table: int32 [sequences, pages] on the cache's device, pages side by side");
  return {static_cast<const int32_t*>(t.data_ptr()), as32(t.size(0)), as32(t.size(1)), t.size(0) > 1 ? t.stride(0) : t.size(1)};
}
// [rows, d] or [d] with elements side by side: its row stride.
int64_t row_stride(const at::Tensor& t, int64_t n, int64_t d, int device, const char* what) {
  const auto sz = t.sizes(), st = t.strides();
  const int64_t k = t.dim();
  need(t.is_cuda() && t.get_device() == device && (k == 1 || k == 2) && sz[k - 1] == d && (k == 2 ? sz[0] == n : n == 1) && (d == 1 || st[k - 1] == 1), what);
  return n > 1 ? st[0] : d;
}
int32_t dtype_code(at::ScalarType t) {
  if (t == at::kBFloat16) return LS_WDTYPE_BF16;
  if (t == at::kHalf) return LS_WDTYPE_FP16;
  need(t == at::kFloat, "dtype: bfloat16, float16 or float32");
  return LS_DTYPE_F32;
}
const float* gain(PyObject* o, int64_t d, int device, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& w = tensor(o, what);
  need(w.scalar_type() == at::kFloat && w.is_cuda() && w.get_device() == device && w.is_contiguous() && w.numel() == d, what);
  return static_cast<const float*>(w.data_ptr());
}

template <class F>
PyObject* guarded(F f) {
  try {
    return PyLong_FromLong(f());
  } catch (const Refusal& r) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.what);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}
constexpr const char *kPlan = "ls_paged_kv", *kPlan4 = "ls_paged_kv4";
Plan* plan_of(PyObject* o, const char* name) {
  Plan* p = static_cast<Plan*>(PyCapsule_GetPointer(o, name));
  if (!p) throw Refusal{nullptr};
  return p;
}
bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, want);
  return false;
}

// bind(append, attend, norm, append4, attend4, read4): addresses of the C functions
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return guarded([&] {
    f_append4 = reinterpret_cast<decltype(f_append4)>((uintptr_t)integer(a[3]));
    f_attend4 = reinterpret_cast<decltype(f_attend4)>((uintptr_t)integer(a[4]));
    f_read4 = reinterpret_cast<decltype(f_read4)>((uintptr_t)integer(a[5]));
    f_append = reinterpret_cast<decltype(f_append)>((uintptr_t)integer(a[0]));
    f_attend = reinterpret_cast<decltype(f_attend)>((uintptr_t)integer(a[1]));
    f_norm = reinterpret_cast<decltype(f_norm)>((uintptr_t)integer(a[2]));
    return 0;
  });
}

template <class F>
PyObject* new_plan(const char* name, F make) {
  try {
    Plan* p = new Plan(make());
    PyObject* c = PyCapsule_New(p, name, [](PyObject* c) { delete static_cast<Plan*>(PyCapsule_GetPointer(c, PyCapsule_GetName(c))); });
    if (!c) delete p;
    return c;
  } catch (const Refusal& r) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.what);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// plan(handle, k_pages, n_q_heads) -> capsule
PyObject* py_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  return new_plan(kPlan, [&] {
    const at::Tensor& k = tensor(a[1], "k_pages: a tensor");
    return Plan{reinterpret_cast<void*>((uintptr_t)integer(a[0])), (int)k.get_device(), k.scalar_type(), integer(a[2]), k.size(2), k.size(3), k.size(1)};
  });
}

// plan4(handle, pages, like, n_q_heads, head_dim, page_size) -> capsule; `like`: a tensor of the cache's 16-bit type
PyObject* py_plan4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 6)) return nullptr;
  return new_plan(kPlan4, [&] {
    const at::Tensor &k = tensor(a[1], "pages: a tensor"), &like = tensor(a[2], "like: a tensor");
    return Plan{reinterpret_cast<void*>((uintptr_t)integer(a[0])), (int)k.get_device(), like.scalar_type(), integer(a[3]), k.size(1), integer(a[4]), integer(a[5])};
  });
}

// append(plan, q, k, v, q_out, seq, pos, table, stream), for either cache
template <class H, class F>
PyObject* append_to(const char* name, F call, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  return guarded([&] {
    const Plan& p = *plan_of(a[0], name);
    const at::Tensor &k = tensor(a[2], "k: a tensor"), &v = tensor(a[3], "v: a tensor"), &seq = tensor(a[5], "seq: a tensor"), &pos = tensor(a[6], "pos: a tensor");
    const int64_t T = k.dim() == 3 ? k.size(0) : -1;
    need(T >= 0, "k: [tokens, kv_heads, head_dim]");
    need(v.dim() == 3 && v.size(0) == T && seq.numel() == T && pos.numel() == T, "k, v, seq and pos disagree about the number of tokens");
    const int64_t sk = token_stride(p, k, p.kv_heads, "k: [tokens, kv_heads, head_dim] of the cache's type and device"),
                  sv = token_stride(p, v, p.kv_heads, "v: [tokens, kv_heads, head_dim] of the cache's type and device");
    const void* q = nullptr;
    void* qo = nullptr;
    int64_t sq = 0, so = 0;
    need((a[1] == Py_None) == (a[4] == Py_None), "q and q_out go together");
    if (a[1] != Py_None) {
      const at::Tensor &tq = tensor(a[1], "q: a tensor"), &to = tensor(a[4], "q_out: a tensor");
      need(tq.dim() == 3 && to.dim() == 3 && tq.size(0) == T && to.size(0) == T, "q and q_out: [tokens, heads, head_dim] of as many tokens as k");
      sq = token_stride(p, tq, p.heads, "q: [tokens, heads, head_dim] of the cache's type and device");
      so = token_stride(p, to, p.heads, "q_out: [tokens, heads, head_dim] of the cache's type and device");
      q = tq.data_ptr();
      qo = to.data_ptr();
    }
    const Table t = table_of(p, tensor(a[7], "table: a tensor"));
    return call(static_cast<H*>(p.handle), q, sq, qo, so, k.data_ptr(), sk, v.data_ptr(), sv, as32(T), ids(seq, p.device, "seq: int32 [tokens] on the cache's device"),
                    ids(pos, p.device, "pos: int32 [tokens] on the cache's device"), t.at, t.rows, t.width, t.stride, stream_of(a[8], p.device));
  });
}

PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return append_to<ls_paged_kv>(kPlan, f_append, a, n); }
PyObject* py_append4(PyObject*, PyObject* const* a, Py_ssize_t n) { return append_to<ls_paged_kv4>(kPlan4, f_append4, a, n); }

// The operands that both attentions have.
struct Rows {
  const void* q;
  void* out;
  int64_t sq, so, B, m;
  const int32_t* len;
  Table t;
  float* lse;
  Rows(const Plan& p, PyObject* oq, PyObject* oo, PyObject* ol, PyObject* ot, PyObject* olse) {
    const at::Tensor &q = tensor(oq, "q: a tensor"), &out = tensor(oo, "out: a tensor"), &len = tensor(ol, "seq_len: a tensor");
    need(q.dim() == 3 || q.dim() == 4, "q: [sequences, heads, head_dim] or [sequences, q_len, heads, head_dim]");
    need(out.sizes() == q.sizes(), "out: of q's shape");
    B = q.size(0);
    m = q.dim() == 4 ? q.size(1) : 1;
    sq = token_stride(p, q, p.heads, "q: heads and components side by side, evenly spaced tokens, of the cache's type and device");
    so = token_stride(p, out, p.heads, "out: heads and components side by side, evenly spaced tokens, of the cache's type and device");
    t = table_of(p, tensor(ot, "table: a tensor"));
    need(len.numel() == B && t.rows == B, "seq_len and table: one row per sequence");
    this->len = ids(len, p.device, "seq_len: int32 on the cache's device");
    lse = nullptr;
    if (olse != Py_None) {
      const at::Tensor& tl = tensor(olse, "lse: a tensor");
      need(tl.scalar_type() == at::kFloat && tl.is_cuda() && tl.get_device() == p.device && tl.is_contiguous() && tl.numel() == B * m * p.heads,
           "lse: dense float32, one value per row of q");
      lse = static_cast<float*>(tl.data_ptr());
    }
    this->q = q.data_ptr();
    this->out = out.data_ptr();
  }
};

// attend(plan, q, out, seq_len, table, prefix_pages, prefix_len, window, scale, lse, stream)
PyObject* py_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 11)) return nullptr;
  return guarded([&] {
    const Plan& p = *plan_of(a[0], kPlan);
    const Rows r(p, a[1], a[2], a[3], a[4], a[9]);
    const long long prefix = integer(a[6]);
    const int32_t* pages = nullptr;
    if (prefix > 0) {
      const at::Tensor& tp = tensor(a[5], "prefix_pages: a tensor");
      pages = ids(tp, p.device, "prefix_pages: int32 on the cache's device");
      need(tp.numel() * p.page >= prefix, "prefix_pages: too few for prefix_len");
    }
    return f_attend(static_cast<ls_paged_kv*>(p.handle), r.q, r.sq, r.out, r.so, r.lse, as32(r.B), as32(r.m), r.len, r.t.at, r.t.width, r.t.stride, pages,
                    as32(prefix), as32(integer(a[7])), (float)real(a[8]), stream_of(a[10], p.device));
  });
}

// attend4(plan, q, out, seq_len, table, window, scale, lse, stream)
PyObject* py_attend4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  return guarded([&] {
    const Plan& p = *plan_of(a[0], kPlan4);
    const Rows r(p, a[1], a[2], a[3], a[4], a[7]);
    return f_attend4(static_cast<ls_paged_kv4*>(p.handle), r.q, r.sq, r.out, r.so, r.lse, as32(r.B), as32(r.m), r.len, r.t.at, r.t.width, r.t.stride,
                     as32(integer(a[5])), (float)real(a[6]), stream_of(a[8], p.device));
  });
}

// read4(plan, k_out, v_out, seq, pos, table, stream)
PyObject* py_read4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 7)) return nullptr;
  return guarded([&] {
    const Plan& p = *plan_of(a[0], kPlan4);
    const at::Tensor &seq = tensor(a[3], "seq: a tensor"), &pos = tensor(a[4], "pos: a tensor");
    const int64_t T = seq.numel();
    need(pos.numel() == T, "seq and pos disagree about the number of tokens");
    auto rows = [&](PyObject* o, const char* what, int64_t& stride) -> void* {
      stride = 0;
      if (o == Py_None) return nullptr;
      const at::Tensor& x = tensor(o, what);
      need(x.dim() == 3 && x.size(0) == T, what);
      stride = token_stride(p, x, p.kv_heads, what);
      return x.data_ptr();
    };
    int64_t sk, sv;
    void *k = rows(a[1], "k_out: [tokens, kv_heads, head_dim] of the cache's type and device", sk),
         *v = rows(a[2], "v_out: [tokens, kv_heads, head_dim] of the cache's type and device", sv);
    const Table t = table_of(p, tensor(a[5], "table: a tensor"));
    return f_read4(static_cast<ls_paged_kv4*>(p.handle), k, sk, v, sv, as32(T), ids(seq, p.device, "seq: int32 [tokens] on the cache's device"),
                   ids(pos, p.device, "pos: int32 [tokens] on the cache's device"), t.at, t.rows, t.width, t.stride, stream_of(a[6], p.device));
  });
}

// norm(x, y, x_out, h, post_norm, w_post, gate, scale, pre_norm, w_pre, eps, stream)
PyObject* py_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  return guarded([&] {
    const at::Tensor& x = tensor(a[0], "x: a tensor");
    need(x.dim() == 1 || x.dim() == 2, "x: [rows, d] or [d]");
    need(x.is_cuda(), "x: on a CUDA device");
    const int64_t d = x.size(-1), rows = x.dim() == 2 ? x.size(0) : 1;
    const int dev = (int)x.get_device();
    const int64_t sx = row_stride(x, rows, d, dev, "x: elements side by side");
    at::ScalarType kind = x.scalar_type();
    bool known = false;
    auto block = [&](PyObject* o, const char* what, int64_t& stride) -> void* {
      stride = 0;
      if (o == Py_None) return nullptr;
      const at::Tensor& t = tensor(o, what);
      need(!known || t.scalar_type() == kind, "y, h and gate: of one type");
      kind = t.scalar_type();
      known = true;
      stride = row_stride(t, rows, d, dev, what);
      return t.data_ptr();
    };
    int64_t sy, sh, so = 0, sg = 0;
    void *y = block(a[1], "y: of x's shape and device, elements side by side", sy), *h = block(a[3], "h: of x's shape and device, elements side by side", sh);
    void* xo = nullptr;
    if (a[2] != Py_None) {
      const at::Tensor& t = tensor(a[2], "x_out: a tensor");
      need(t.scalar_type() == x.scalar_type(), "x_out: of x's type");
      so = row_stride(t, rows, d, dev, "x_out: of x's shape and device, elements side by side");
      xo = t.data_ptr();
    }
    const void* g = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor& t = tensor(a[6], "gate: a tensor");
      need(!known || t.scalar_type() == kind, "y, h and gate: of one type");
      if (t.dim() == 2) sg = row_stride(t, rows, d, dev, "gate: [d] or of x's shape, elements side by side");
      else row_stride(t, 1, d, dev, "gate: [d] or of x's shape, elements side by side");
      g = t.data_ptr();
    }
    const int post = PyObject_IsTrue(a[4]), pre = PyObject_IsTrue(a[8]);
    if (post < 0 || pre < 0) throw Refusal{nullptr};
    return f_norm(x.data_ptr(), sx, dtype_code(x.scalar_type()), y, sy, dtype_code(kind), xo, so, h, sh, as32(rows), as32(d), post ? LS_NORM_RMS : LS_NORM_NONE,
                  gain(a[5], d, dev, "w_post: dense float32 [d] on x's device"), g, sg, (float)real(a[7]), pre ? LS_NORM_RMS : LS_NORM_NONE,
                  gain(a[9], d, dev, "w_pre: dense float32 [d] on x's device"), (float)real(a[10]), stream_of(a[11], dev));
  });
}

#define LS_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"bind", LS_FAST(py_bind), nullptr},     {"plan", LS_FAST(py_plan), nullptr}, {"append", LS_FAST(py_append), nullptr},
                         {"attend", LS_FAST(py_attend), nullptr}, {"norm", LS_FAST(py_norm), nullptr},
                         {"plan4", LS_FAST(py_plan4), nullptr},   {"append4", LS_FAST(py_append4), nullptr},
                         {"attend4", LS_FAST(py_attend4), nullptr}, {"read4", LS_FAST(py_read4), nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "ls_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ls_marshal(void) { return PyModule_Create(&module); }
