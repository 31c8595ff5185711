// Python calls of the operators on torch tensors (CPython module _operators): argument checks and one call of the C ABI.
//
// These operators take microseconds.  The same checks written in Python over ctypes take 4.0 us a call beside the 2.7 us
// of the launch; a write of one token goes from 7.4 us to 3.3 with them here.  A call goes to the current stream of its tensors' device and
// returns the C ABI's code.  Wrong arguments raise TypeError or ValueError; no C++ exception leaves an entry.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>

#include <initializer_list>
#include <optional>
#include <sstream>
#include <string>

#include "sara.h"

namespace {

struct Refusal { PyObject* type; std::string text; };
[[noreturn]] void value_error(const std::string& text) { throw Refusal{PyExc_ValueError, text}; }
[[noreturn]] void type_error(const std::string& text) { throw Refusal{PyExc_TypeError, text}; }
struct PythonError {};   // an exception is set already

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) type_error(std::string(what) + " must be a tensor");
  return THPVariable_Unpack(o);
}
int32_t size32(int64_t n, const char* what) {
  if (n > INT32_MAX) value_error(std::string(what) + ": a size above 2^31 - 1");
  return (int32_t)n;
}
int32_t float_type(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kBFloat16) return SARA_BF16;
  if (t.scalar_type() == at::kFloat) return SARA_F32;
  type_error(std::string(what) + " must be bfloat16 or float32, not " + toString(t.scalar_type()));
}
float number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw PythonError{};
  return (float)x;
}

// The device of a call's tensors, the current one for as long as the call lasts, and its current stream.
struct Place {
  c10::DeviceIndex index;
  std::optional<c10::DeviceGuard> guard;
  explicit Place(const at::Tensor& t) {
    if (!t.is_cuda()) value_error("tensors must be on the GPU");
    index = t.get_device();
    guard.emplace(t.device());
  }
  void check(const at::Tensor& t, const char* what) const {
    if (!t.is_cuda() || t.get_device() != index) value_error(std::string(what) + " must be on the GPU, all tensors on one");
  }
  void* stream() const {
    static PyObject* current = nullptr;   // torch's own lookup of the raw handle
    if (!current) {
      PyObject* c = PyImport_ImportModule("torch._C");
      if (c) current = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
      Py_XDECREF(c);
      if (!current) throw PythonError{};
    }
    PyObject* device = PyLong_FromLong(index);
    PyObject* handle = device ? PyObject_CallOneArg(current, device) : nullptr;
    Py_XDECREF(device);
    if (!handle) throw PythonError{};
    void* s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!s && PyErr_Occurred()) throw PythonError{};
    return s;
  }
};

// codes [n_pages, n_kv_heads, 16, head_dim] (int8 or float8_e4m3fn) and exponents [n_pages, n_kv_heads] (uint8)
sara_kv8_cache kv8_cache(PyObject* const* a, const Place& at) {
  const at::Tensor &k = tensor(a[0], "codes"), &v = tensor(a[1], "codes"), &ke = tensor(a[2], "exponents"),
                   &ve = tensor(a[3], "exponents");
  const auto type = k.scalar_type();
  if (type != at::kChar && type != at::kFloat8_e4m3fn)
    type_error(std::string("codes must be int8 or float8_e4m3fn, not ") + toString(type));
  if (k.dim() != 4 || k.size(2) != 16 || v.sizes() != k.sizes() || v.scalar_type() != type)
    value_error("codes must be [n_pages, n_kv_heads, 16, head_dim], alike for K and V");
  const auto pages = k.sizes().slice(0, 2);
  if (ke.scalar_type() != at::kByte || ve.scalar_type() != at::kByte || ke.sizes() != pages || ve.sizes() != pages)
    value_error("exponents must be uint8 [n_pages, n_kv_heads]");
  for (const at::Tensor* t : {&k, &v, &ke, &ve}) {
    at.check(*t, "the cache");
    if (!t->is_contiguous()) value_error("codes and exponents must be contiguous");
  }
  return sara_kv8_cache{k.data_ptr(), v.data_ptr(), (uint8_t*)ke.data_ptr(), (uint8_t*)ve.data_ptr(), size32(k.size(0), "pages"),
                        size32(k.size(1), "KV heads"), size32(k.size(3), "head_dim"),
                        type == at::kChar ? SARA_KV8_INT8 : SARA_KV8_E4M3};
}

// the stride of an axis; of one that holds a single element torch's may be anything
int64_t stride_of(const at::Tensor& t, int64_t axis, int64_t single) { return t.size(axis) > 1 ? t.stride(axis) : single; }

// a [rows, heads, dim] tensor whose last dimension is contiguous
struct Rows { void* p; int64_t row, head; };
Rows rows3(const at::Tensor& t, int64_t rows, int64_t heads, int64_t dim, const Place& at, const char* what) {
  if (t.dim() != 3 || t.size(0) != rows || t.size(1) != heads || t.size(2) != dim) {
    std::ostringstream s;
    s << what << " must be [" << rows << ", " << heads << ", " << dim << "], not " << t.sizes();
    value_error(s.str());
  }
  at.check(t, what);
  if (t.stride(2) != 1 && t.numel()) value_error(std::string(what) + " must have a contiguous last dimension");
  return Rows{t.data_ptr(), stride_of(t, 0, 0), stride_of(t, 1, 0)};
}

// a page table and its per-sequence arrays
struct Seqs { const int32_t *pages, *seq, *off; int32_t n, width; };
Seqs sequences(PyObject* o_pages, PyObject* o_seq, PyObject* o_off, int64_t n_rows, const Place& at) {
  const at::Tensor &pages = tensor(o_pages, "page table"), &seq = tensor(o_seq, "per-sequence array");
  if (pages.dim() != 2 || pages.scalar_type() != at::kInt || seq.scalar_type() != at::kInt || seq.numel() != pages.size(0))
    value_error("page table [n_seqs, max_pages] and per-sequence array [n_seqs] must be int32");
  at.check(pages, "page table");
  at.check(seq, "per-sequence array");
  if (!pages.is_contiguous() || !seq.is_contiguous()) value_error("page table and per-sequence array must be contiguous");
  Seqs s = {pages.data_ptr<int32_t>(), seq.data_ptr<int32_t>(), nullptr, size32(pages.size(0), "sequences"),
            size32(pages.size(1), "pages of a sequence")};
  if (o_off == Py_None) {
    if (n_rows != s.n) value_error(std::to_string(n_rows) + " rows for " + std::to_string(s.n) + " sequences: give d_off");
    return s;
  }
  const at::Tensor& off = tensor(o_off, "d_off");
  if (off.scalar_type() != at::kInt || off.numel() != (int64_t)s.n + 1 || !off.is_contiguous())
    value_error("d_off must be contiguous int32 [n_seqs + 1]");
  at.check(off, "d_off");
  s.off = off.data_ptr<int32_t>();
  return s;
}

// n contiguous elements, or None
template <typename T> T* per_row(PyObject* o, int64_t n, at::ScalarType type, const Place& at, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous())
    value_error(std::string(what) + " must hold " + std::to_string(n) + " contiguous elements of " + toString(type));
  at.check(t, what);
  return (T*)t.data_ptr();
}

// the caller's workspace, or one of torch's allocator, which ties it to the current stream
struct Workspace { at::Tensor keep; void* p; int64_t bytes; };
Workspace workspace(PyObject* o, int64_t need, const at::Tensor& like, const Place& at) {
  if (need == 0) return {};
  Workspace w;
  if (o == Py_None) {
    w.keep = at::empty({need}, like.options().dtype(at::kByte));
  } else {
    w.keep = tensor(o, "workspace");
    at.check(w.keep, "workspace");
    if (!w.keep.is_contiguous()) value_error("the workspace must be contiguous");
  }
  w.p = w.keep.data_ptr();
  w.bytes = (int64_t)w.keep.nbytes();
  return w;
}

// A call that has written to tensors raises their version, so that autograd notices where one was saved for a backward pass.
int written(int rc, std::initializer_list<PyObject*> outputs) {
  if (rc == SARA_OK)
    for (PyObject* o : outputs)
      if (o != Py_None && !THPVariable_Unpack(o).is_inference()) THPVariable_Unpack(o).unsafeGetTensorImpl()->bump_version();
  return rc;
}

template <typename F> int without_gil(F&& call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call();
  Py_END_ALLOW_THREADS;
  return rc;
}

// Runs an entry of `want` arguments; its result is the code of the C ABI.
template <typename F> PyObject* entry(Py_ssize_t n, Py_ssize_t want, F&& body) {
  try {
    if (n != want) type_error("wrong number of arguments");
    return PyLong_FromLong(body());
  } catch (const Refusal& r) {
    PyErr_SetString(r.type, r.text.c_str());
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// (k_cache, v_cache, k_exp, v_exp, d_k, d_v, d_pages, d_start, d_off)
template <bool WRITE> PyObject* kv8_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 9, [&] {
    const at::Tensor &k = tensor(a[4], "K"), &v = tensor(a[5], "V");
    const int32_t type = float_type(k, "K and V");
    if (v.scalar_type() != k.scalar_type()) value_error("K and V must have the same dtype");
    const Place at(k);
    const sara_kv8_cache c = kv8_cache(a, at);
    const int64_t rows = k.dim() ? k.size(0) : 0;
    const Rows rk = rows3(k, rows, c.n_kv_heads, c.head_dim, at, "K"), rv = rows3(v, rows, c.n_kv_heads, c.head_dim, at, "V");
    const Seqs s = sequences(a[6], a[7], a[8], rows, at);
    const int32_t n_rows = size32(rows, "rows");
    void* st = at.stream();
    const int rc = without_gil([&] {
      if (WRITE)
        return sara_kv8_write(&c, rk.p, rk.row, rk.head, rv.p, rv.row, rv.head, type, n_rows, s.pages, s.width, s.seq, s.off,
                              s.n, st);
      return sara_kv8_read(&c, rk.p, rk.row, rk.head, rv.p, rv.row, rv.head, type, n_rows, s.pages, s.width, s.seq, s.off, s.n,
                           st);
    });
    return WRITE ? written(rc, {a[0], a[1], a[2], a[3]}) : written(rc, {a[4], a[5]});
  });
}

// (k_cache, v_cache, k_exp, v_exp, d_q, d_out, d_pages, d_ctx, d_off, scale, max_ctx, workspace); None: the defaults
PyObject* kv8_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 12, [&] {
    const at::Tensor &q = tensor(a[4], "q"), &out = tensor(a[5], "out");
    const int32_t type = float_type(q, "q");
    if (out.scalar_type() != q.scalar_type()) value_error("out must have q's dtype");
    const Place at(q);
    const sara_kv8_cache c = kv8_cache(a, at);
    if (q.dim() != 3) value_error("q must be [rows, n_heads, head_dim]");
    const int32_t n_rows = size32(q.size(0), "rows"), heads = size32(q.size(1), "heads");
    const Rows rq = rows3(q, n_rows, heads, c.head_dim, at, "q"), ro = rows3(out, n_rows, heads, c.head_dim, at, "out");
    const Seqs s = sequences(a[6], a[7], a[8], n_rows, at);
    const float scale = a[9] == Py_None ? (c.head_dim == 64 ? 0.125f : 0.08838834764831845f) : number(a[9]);
    int64_t max_ctx = 16 * (int64_t)s.width;
    if (a[10] != Py_None) {
      max_ctx = PyLong_AsLongLong(a[10]);
      if (max_ctx == -1 && PyErr_Occurred()) throw PythonError{};
    }
    if (max_ctx != (int32_t)max_ctx) value_error("max_ctx must be below 2^31");
    int64_t need = 0;
    int rc = sara_kv8_attention_workspace(c.n_kv_heads, c.head_dim, n_rows, heads, s.n, s.off != nullptr, (int32_t)max_ctx, &need);
    if (rc) return rc;
    const Workspace ws = workspace(a[11], need, q, at);
    void* st = at.stream();
    rc = without_gil([&] {
      return sara_kv8_attention(&c, rq.p, rq.row, rq.head, ro.p, ro.row, ro.head, type, n_rows, heads, s.pages, s.width, s.seq,
                                s.off, s.n, (int32_t)max_ctx, scale, ws.p, ws.bytes, st);
    });
    return written(rc, {a[5]});
  });
}

// [rows, vocab] with contiguous rows
void check_logits(const at::Tensor& t, const Place& at, const char* what) {
  if (t.dim() != 2 || (stride_of(t, 1, 1) != 1 && t.numel())) value_error(std::string(what) + " must be [rows, vocab] with contiguous rows");
  at.check(t, what);
}

// (d_logits, d_tok, d_logp, d_entropy, d_stats, d_top_id, d_top_logp, temperature, workspace)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 9, [&] {
    const at::Tensor& x = tensor(a[0], "logits");
    const int32_t type = float_type(x, "logits");
    const Place at(x);
    check_logits(x, at, "logits");
    const int32_t rows = size32(x.size(0), "rows"), V = size32(x.size(1), "vocab");
    if ((a[5] == Py_None) != (a[6] == Py_None)) value_error("give both of d_top_id and d_top_logp");
    int32_t k = 0;
    if (a[5] != Py_None) {
      const at::Tensor& id = tensor(a[5], "top ids");
      if (id.dim() != 2) value_error("top ids must be [rows, n_top]");
      k = size32(id.size(1), "top ids");
    }
    const float temp = number(a[7]);
    int64_t need = 0;
    int rc = sara_token_logprobs_workspace(rows, V, k, &need);
    if (rc) return rc;
    const int32_t* tok = per_row<int32_t>(a[1], rows, at::kInt, at, "tokens");
    float* logp = per_row<float>(a[2], rows, at::kFloat, at, "logp");
    float* ent = per_row<float>(a[3], rows, at::kFloat, at, "entropy");
    float* stats = per_row<float>(a[4], 2 * (int64_t)rows, at::kFloat, at, "stats");
    int32_t* id = per_row<int32_t>(a[5], (int64_t)rows * k, at::kInt, at, "top ids");
    float* lp = per_row<float>(a[6], (int64_t)rows * k, at::kFloat, at, "top logp");
    const Workspace ws = workspace(a[8], need, x, at);
    void* st = at.stream();
    rc = without_gil([&] {
      return sara_token_logprobs(x.data_ptr(), type, stride_of(x, 0, V), rows, V, tok, temp, k, logp, ent, stats, id, lp, ws.p, ws.bytes,
                                 st);
    });
    return written(rc, {a[2], a[3], a[4], a[5], a[6]});
  });
}

// (d_logits, d_tok, d_stats, d_entropy, d_g_logp, d_g_entropy, d_grad, temperature)
PyObject* token_logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 8, [&] {
    const at::Tensor &x = tensor(a[0], "logits"), &y = tensor(a[6], "gradient");
    const int32_t type = float_type(x, "logits");
    float_type(y, "gradient");
    const Place at(x);
    check_logits(x, at, "logits");
    check_logits(y, at, "gradient");
    if (y.sizes() != x.sizes() || y.scalar_type() != x.scalar_type()) value_error("the gradient must have the logits' shape and dtype");
    const int32_t rows = size32(x.size(0), "rows"), V = size32(x.size(1), "vocab");
    const int32_t* tok = per_row<int32_t>(a[1], rows, at::kInt, at, "tokens");
    const float* stats = per_row<float>(a[2], 2 * (int64_t)rows, at::kFloat, at, "stats");
    const float* ent = per_row<float>(a[3], rows, at::kFloat, at, "entropy");
    const float* g = per_row<float>(a[4], rows, at::kFloat, at, "g_logp");
    const float* h = per_row<float>(a[5], rows, at::kFloat, at, "g_entropy");
    const float temp = number(a[7]);
    void* st = at.stream();
    const int rc = without_gil([&] {
      return sara_token_logprobs_grad(x.data_ptr(), type, stride_of(x, 0, V), rows, V, tok, temp, stats, ent, g, h, y.data_ptr(),
                                      stride_of(y, 0, V), st);
    });
    return written(rc, {a[6]});
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyCFunction fast() { return (PyCFunction)(void (*)())F; }

PyMethodDef methods[] = {{"kv8_write", fast<kv8_rows<true>>(), METH_FASTCALL, nullptr},
                         {"kv8_read", fast<kv8_rows<false>>(), METH_FASTCALL, nullptr},
                         {"kv8_attention", fast<kv8_attention>(), METH_FASTCALL, nullptr},
                         {"token_logprobs", fast<token_logprobs>(), METH_FASTCALL, nullptr},
                         {"token_logprobs_grad", fast<token_logprobs_grad>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators(void) { return PyModule_Create(&module); }
