// Python side of the serving calls: takes tensors, checks them, calls the C entry points.
//
// These calls take three to ten microseconds on the GPU and are made once or more per layer and generated token.  Marshalling
// thirty arguments through ctypes and testing a dozen tensors in Python took ten; here it takes about one, so that a loop of
// them without a CUDA graph is bounded by the launches.  The entry points are those of libt5b200.so, whose addresses
// bind() receives; nothing is computed here.
//
// A call returns None, the library's negative code, or a text that says which tensor does not fit; the Python wrappers
// turn the latter two into T5Error.
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/t5_b200.h"

namespace {

decltype(&t5_paged_kv_append) g_append = nullptr;
decltype(&t5_paged_attention) g_attention = nullptr;
decltype(&t5_verify_draft) g_verify = nullptr;

struct Refusal { std::string what; };
[[noreturn]] void refuse(const std::string& what) { throw Refusal{what}; }

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": want a tensor");
  return THPVariable_Unpack(o);
}
std::string describe(const at::Tensor& t) {
  std::string s = std::string(c10::toString(t.scalar_type())) + " [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += "] strides [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  return s + "] on " + t.device().str();
}
[[noreturn]] void wrong(const char* name, const std::string& want, const at::Tensor& t) {
  refuse(std::string(name) + ": want " + want + " on the current device, got " + describe(t));
}

// What every tensor of a call has to share
struct Call {
  int64_t device;
  at::ScalarType type;
  int code;
  void* stream;
  Call(const at::Tensor& t, const char* name) : device(t.is_cuda() ? t.get_device() : -1), type(t.scalar_type()) {
    if (device < 0 || device != c10::cuda::current_device()) wrong(name, "a CUDA tensor", t);
    if (type != at::kFloat && type != at::kBFloat16) wrong(name, "a float32 or bfloat16 tensor", t);
    code = type == at::kFloat ? 0 : 1;
    stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  }
  bool here(const at::Tensor& t, at::ScalarType ty) const { return t.scalar_type() == ty && t.is_cuda() && t.get_device() == device; }
};

std::string shape(std::initializer_list<int64_t> s) {
  std::string r = "[";
  for (int64_t v : s) r += (r.size() > 1 ? ", " : "") + std::to_string(v);
  return r + "]";
}
// [rows, heads, d] with adjacent heads; rows may be slices of wider ones
int64_t heads(const Call& c, const at::Tensor& t, const char* name, int64_t n, int64_t h, int64_t d) {
  if (!c.here(t, c.type) || t.dim() != 3 || t.size(0) != n || t.size(1) != h || t.size(2) != d || t.stride(2) != 1 ||
      (h > 1 && t.stride(1) != d))
    wrong(name, shape({n, h, d}) + " of the type of the first argument, heads adjacent columns,", t);
  return n > 1 ? t.stride(0) : h * d;
}
void* vec(const Call& c, const at::Tensor& t, const char* name, at::ScalarType ty, int64_t n) {
  if (!c.here(t, ty) || t.numel() != n || !t.is_contiguous())
    wrong(name, std::string(c10::toString(ty)) + ", " + std::to_string(n) + " contiguous entries,", t);
  return t.data_ptr();
}
struct Pools {
  void *k, *v, *table;
  int64_t n, ps, g, d, st[3], seqs, max_pages, ld;
  Pools(const Call& c, const at::Tensor& kp, const at::Tensor& vp, const at::Tensor& tb) {
    if (!c.here(kp, c.type) || kp.dim() != 4 || kp.stride(3) != 1) wrong("k_pages", "[n_pages, page_size, kv_heads, d_kv] of the type of the first argument", kp);
    if (!c.here(vp, c.type) || vp.sizes() != kp.sizes() || vp.stride(3) != 1) wrong("v_pages", "a pool like k_pages", vp);
    n = kp.size(0); ps = kp.size(1); g = kp.size(2); d = kp.size(3);
    const int64_t size[3] = {n, ps, g};
    for (int i = 0; i < 3; ++i) {
      st[i] = size[i] > 1 ? kp.stride(i) : ps * g * d;      // a dimension of one entry has no stride
      if (size[i] > 1 && vp.stride(i) != st[i]) wrong("v_pages", "the strides of k_pages", vp);
    }
    if (!c.here(tb, at::kInt) || tb.dim() != 2 || (tb.size(1) > 1 && tb.stride(1) != 1)) wrong("page_table", "int32 [sequences, pages] with contiguous rows", tb);
    seqs = tb.size(0); max_pages = tb.size(1);
    ld = seqs > 1 ? tb.stride(0) : max_pages;
    k = kp.data_ptr(); v = vp.data_ptr(); table = tb.data_ptr();
    if (n > INT32_MAX || ps > INT32_MAX || g > INT32_MAX || d > INT32_MAX || seqs > INT32_MAX || max_pages > INT32_MAX) refuse("pools: sizes beyond 2^31");
  }
};
int64_t integer(PyObject* o, const char* name) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); refuse(std::string(name) + ": want an integer"); }
  if (v > INT32_MAX || v < INT32_MIN) refuse(std::string(name) + ": out of range");
  return v;
}
double number(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); refuse(std::string(name) + ": want a number"); }
  return v;
}
void fits32(int64_t v, const char* what) { if (v > INT32_MAX) refuse(std::string(what) + ": beyond 2^31"); }

PyObject* done(int rc) {
  if (rc == 0) Py_RETURN_NONE;
  return PyLong_FromLong(rc);
}
// Runs f (returns the library's code), turning refusals and C++ exceptions into Python values and errors
template <typename F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return done(f());
  } catch (const Refusal& r) {
    return PyUnicode_FromString(r.what.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&] {
    g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[0]));
    g_attention = reinterpret_cast<decltype(g_attention)>(PyLong_AsVoidPtr(a[1]));
    g_verify = reinterpret_cast<decltype(g_verify)>(PyLong_AsVoidPtr(a[2]));
    return 0;
  });
}

// k, v, k_pages, v_pages, page_table, seq_of_token, positions, q, q_out, rot_dim, rot_base, rot_interleaved
PyObject* paged_kv_append(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded(na, 12, [&] {
    const at::Tensor& k = tensor(a[0], "k");
    const Call c(k, "k");
    const Pools p(c, tensor(a[2], "k_pages"), tensor(a[3], "v_pages"), tensor(a[4], "page_table"));
    if (k.dim() != 3) wrong("k", "[tokens, kv_heads, d_kv]", k);
    const int64_t n = k.size(0);
    fits32(n, "tokens");
    const int64_t ldk = heads(c, k, "k", n, p.g, p.d), ldv = heads(c, tensor(a[1], "v"), "v", n, p.g, p.d);
    void* seq = vec(c, tensor(a[5], "seq_of_token"), "seq_of_token", at::kInt, n);
    void* pos = vec(c, tensor(a[6], "positions"), "positions", at::kInt, n);
    int64_t h = 0, ldq = 0, ldqo = 0;
    void *q = nullptr, *qo = nullptr;
    if ((a[7] == Py_None) != (a[8] == Py_None)) refuse("q and q_out: want both or neither");
    if (a[7] != Py_None) {
      const at::Tensor &tq = tensor(a[7], "q"), &to = tensor(a[8], "q_out");
      if (tq.dim() != 3) wrong("q", "[tokens, heads, d_kv]", tq);
      h = tq.size(1);
      ldq = heads(c, tq, "q", n, h, p.d);
      ldqo = heads(c, to, "q_out", n, h, p.d);
      q = tq.data_ptr(); qo = to.data_ptr();
      fits32(h, "heads");
    }
    const int rot = (int)integer(a[9], "rot_dim"), inter = PyObject_IsTrue(a[11]) ? 1 : 0;
    const double base = number(a[10], "rot_base");
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_append(c.code, (int)n, (int)h, (int)p.g, (int)p.d, q, ldq, k.data_ptr(), ldk, THPVariable_Unpack(a[1]).data_ptr(),
                  ldv, qo, ldqo, (const int32_t*)seq, (const int32_t*)pos, rot, base, inter, p.k, p.v, (int)p.n, (int)p.ps,
                  p.st[0], p.st[1], p.st[2], (const int32_t*)p.table, (int)p.seqs, (int)p.max_pages, p.ld, c.stream);
    Py_END_ALLOW_THREADS
    return rc;
  });
}

// q, k_pages, v_pages, page_table, lens, out, workspace, scale, n_q, bias, lse
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded(na, 11, [&] {
    const at::Tensor& q = tensor(a[0], "q");
    const Call c(q, "q");
    const Pools p(c, tensor(a[1], "k_pages"), tensor(a[2], "v_pages"), tensor(a[3], "page_table"));
    if (q.dim() != 3) wrong("q", "[rows, heads, d_kv]", q);
    const int64_t r = q.size(0), h = q.size(1), n_q = integer(a[8], "n_q");
    fits32(r, "rows");
    fits32(h, "heads");
    const at::Tensor& out = tensor(a[5], "out");
    const int64_t ldq = heads(c, q, "q", r, h, p.d), ldo = heads(c, out, "out", r, h, p.d);
    if (p.seqs * n_q != r) refuse("page_table: want a row for every n_q rows of q");
    void* lens = vec(c, tensor(a[4], "lens"), "lens", at::kInt, r);
    const at::Tensor& ws = tensor(a[6], "workspace");
    if (!ws.is_cuda() || ws.get_device() != c.device || !ws.is_contiguous()) wrong("workspace", "a contiguous tensor", ws);
    const double scale = number(a[7], "scale");
    const float* bias = nullptr;
    float* lse = nullptr;
    int64_t n_bias = 0;
    if (a[9] != Py_None) {
      const at::Tensor& b = tensor(a[9], "bias");
      if (b.dim() != 2 || b.size(0) != h) wrong("bias", "float32 [heads, distances]", b);
      n_bias = b.size(1);
      fits32(n_bias, "bias");
      bias = (const float*)vec(c, b, "bias", at::kFloat, h * n_bias);
    }
    if (a[10] != Py_None) lse = (float*)vec(c, tensor(a[10], "lse"), "lse", at::kFloat, r * h);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_attention(c.code, (int)r, (int)n_q, (int)h, (int)p.g, (int)p.d, (float)scale, q.data_ptr(), ldq, p.k, p.v,
                     (int)p.n, (int)p.ps, p.st[0], p.st[1], p.st[2], (const int32_t*)p.table, (int)p.max_pages, p.ld,
                     (const int32_t*)lens, bias, (int)n_bias, out.data_ptr(), ldo, lse, ws.data_ptr(), (int64_t)ws.nbytes(),
                     c.stream);
    Py_END_ALLOW_THREADS
    return rc;
  });
}

// target, draft, draft_tokens, n_draft, u_accept, u_sample, out_tokens, n_accepted
PyObject* verify_draft(PyObject*, PyObject* const* a, Py_ssize_t na) {
  return guarded(na, 8, [&] {
    const at::Tensor& t = tensor(a[0], "target");
    const Call c(t, "target");
    if (t.dim() != 3 || t.size(1) < 1 || (t.size(2) > 1 && t.stride(2) != 1)) wrong("target", "[sequences, drafts + 1, vocab]", t);
    const int64_t s = t.size(0), k = t.size(1) - 1, v = t.size(2);
    fits32(s, "sequences");
    fits32(v, "vocab");
    fits32(k, "drafts");
    // [s, width] with contiguous rows; returns the row stride
    auto rows = [&](PyObject* o, const char* name, at::ScalarType ty, int64_t width, void*& ptr) -> int64_t {
      const at::Tensor& x = tensor(o, name);
      if (!c.here(x, ty) || x.dim() != 2 || x.size(0) != s || x.size(1) != width || (width > 1 && x.stride(1) != 1))
        wrong(name, std::string(c10::toString(ty)) + " " + shape({s, width}) + " with contiguous rows", x);
      ptr = x.data_ptr();
      return s > 1 ? x.stride(0) : width;
    };
    void *x, *u, *out, *d = nullptr, *nd = nullptr;
    const int64_t ldx = rows(a[2], "draft_tokens", at::kInt, k, x), ldu = rows(a[4], "u_accept", at::kFloat, k, u);
    const int64_t ldo = rows(a[6], "out_tokens", at::kInt, k + 1, out);
    int64_t ds = 0, dr = v;
    if (a[1] != Py_None && k > 0) {
      const at::Tensor& y = tensor(a[1], "draft");
      if (!c.here(y, c.type) || y.dim() != 3 || y.size(0) != s || y.size(1) != k || y.size(2) != v || (v > 1 && y.stride(2) != 1))
        wrong("draft", shape({s, k, v}) + " of the target's type", y);
      d = y.data_ptr();
      ds = s > 1 ? y.stride(0) : 0;
      dr = k > 1 ? y.stride(1) : v;
    }
    if (a[3] != Py_None) nd = vec(c, tensor(a[3], "n_draft"), "n_draft", at::kInt, s);
    void* us = vec(c, tensor(a[5], "u_sample"), "u_sample", at::kFloat, s);
    void* acc = vec(c, tensor(a[7], "n_accepted"), "n_accepted", at::kInt, s);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_verify(c.code, (int)s, (int)k, (int)v, t.data_ptr(), s > 1 ? t.stride(0) : 0, k > 0 ? t.stride(1) : v, d, ds, dr,
                  (const int32_t*)x, ldx, (const int32_t*)nd, (const float*)u, ldu, (const float*)us, (int32_t*)out, ldo,
                  (int32_t*)acc, c.stream);
    Py_END_ALLOW_THREADS
    return rc;
  });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "addresses of the library's entry points"},
    {"paged_kv_append", (PyCFunction)(void (*)(void))paged_kv_append, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {"verify_draft", (PyCFunction)(void (*)(void))verify_draft, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__serving() { return PyModule_Create(&module); }
