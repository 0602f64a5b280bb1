// The Python calls over a paged cache (cache.py, select_blocks of binding.py) down to the C ABI: checks of the tensors, outputs and workspace, one call.
// A decoding loop makes these calls a few times a layer with a few tokens, and what a call costs on the host is then what it costs: with the checks
// in Python an append of one token took 10.1 us, its attention 14.7 and its selection 8.4, of which a launch is 3.7; from here 5.6, 10.3 and 5.2.
// The library knows nothing of this file or of torch.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../../include/nsa_sel.h"

namespace {

constexpr int64_t kD = 128;
PyObject* g_error = nullptr;  // NsaSelError

struct Refused {
  std::string why;
};

std::string text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused{std::string(name) + " must be a torch.Tensor"};
  return THPVariable_Unpack(o);
}
const at::Tensor& dims(PyObject* o, const char* name, int64_t n) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != n) throw Refused{std::string(name) + " must have " + std::to_string(n) + " dimensions, got " + text(t.sizes())};
  return t;
}

void expect_kind(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev) {
  if (t.scalar_type() != type) throw Refused{std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type())};
  if (t.sizes() != shape) throw Refused{std::string(name) + " must have shape " + text(shape) + ", got " + text(t.sizes())};
  if (t.device() != dev) throw Refused{std::string(name) + " must live on " + dev.str() + ", got " + t.device().str()};
  if (t.requires_grad() && at::GradMode::is_enabled())
    throw Refused{std::string(name) + " requires grad, and the calls over a cache have no backward: call under torch.no_grad(), or detach it"};
}
// A contiguous tensor; its address.
void* expect(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev) {
  expect_kind(t, name, type, shape, dev);
  if (!t.is_contiguous()) throw Refused{std::string(name) + " must be contiguous"};
  return t.data_ptr();
}
// bf16 [tokens, heads, 128] whose tokens may lie apart (a slice of one projection) and whose heads may not; the values between tokens.
int64_t expect_rows(const at::Tensor& t, const char* name, at::IntArrayRef shape, const at::Device& dev) {
  expect_kind(t, name, at::kBFloat16, shape, dev);
  if (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) throw Refused{std::string(name) + " must be 16-byte aligned"};
  const int64_t tokens = shape[0], heads = shape[1];
  if (tokens == 0 || t.is_contiguous()) return heads * kD;
  if (t.stride(2) != 1 || (heads > 1 && t.stride(1) != kD)) throw Refused{std::string("the heads of a token of ") + name + " must be contiguous"};
  if (tokens == 1) return heads * kD;
  if (t.stride(0) < heads * kD || (t.stride(0) & 7))
    throw Refused{std::string("the tokens of ") + name + " must be a multiple of 8 values apart, and not overlap"};
  return t.stride(0);
}

int32_t small(PyObject* o, const char* name) {
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (PyErr_Occurred()) throw python_error();
  if (over || v < INT32_MIN || v > INT32_MAX) throw Refused{std::string(name) + " is out of range"};
  return (int32_t)v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}

// Other Python threads run while torch allocates and the library launches: the allocator may wait, and so may a full queue.
struct WithoutGil {
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};
template <class F>
auto without_gil(F&& f) {
  const WithoutGil w;
  return f();
}
at::Tensor empty(at::IntArrayRef shape, at::TensorOptions options) {
  return without_gil([&] { return at::empty(shape, options); });
}

void done(int rc, const char* what) {
  if (rc != NSA_SEL_OK) throw Refused{std::string(what) + ": " + nsa_sel_strerror(rc) + " (" + std::to_string(rc) + ")"};
}
void on_gpu(const at::Device& dev) {
  if (!dev.is_cuda()) throw Refused{"tensors must be contiguous device tensors"};
}
void count(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) throw Refused{"internal: wrong number of arguments"};
}

// ---- a cache: its tensors and sizes ----------------------------------------------------------------------------------------------
struct CacheInfo {
  at::Tensor t[4];  // K and V pages and, in 8 bits, their scales
  at::ScalarType type;
  int32_t n_pages, hkv, page, dtype;
  at::Device device = at::kCPU;
};
constexpr char kCapsule[] = "nsa_sel_cache";
void free_info(PyObject* o) { delete static_cast<CacheInfo*>(PyCapsule_GetPointer(o, kCapsule)); }
const CacheInfo& info(PyObject* o) {
  auto* p = static_cast<CacheInfo*>(PyCapsule_GetPointer(o, kCapsule));
  if (!p) throw python_error();
  return *p;
}

// Where they lie at this call: their owner may have given them other storage since the last one, or none.
struct Pages {
  void *k, *v;
  float *ks = nullptr, *vs = nullptr;
};
void* address(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev) {
  if (t.has_storage() && t.storage().nbytes() < (size_t)(t.storage_offset() + t.numel()) * t.itemsize()) throw Refused{std::string(name) + " has lost its storage"};
  return expect(t, name, type, shape, dev);
}
Pages pages(const CacheInfo& c) {
  const int64_t shape[4] = {c.n_pages, c.hkv, c.page, kD};
  const at::IntArrayRef scales(shape, 2);
  Pages p;
  p.k = address(c.t[0], "k_pages", c.type, shape, c.device);
  p.v = address(c.t[1], "v_pages", c.type, shape, c.device);
  if (c.dtype == NSA_SEL_CACHE_E4M3) {
    p.ks = (float*)address(c.t[2], "k_scale", at::kFloat, scales, c.device);
    p.vs = (float*)address(c.t[3], "v_scale", at::kFloat, scales, c.device);
  }
  return p;
}

PyObject* describe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 4);
    const at::Tensor& k = dims(a[0], "k_pages", 4);
    const at::ScalarType type = k.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat8_e4m3fn) throw Refused{"pages must be bfloat16 or float8_e4m3fn [n_pages, hkv, page, 128]"};
    const auto s = k.sizes();
    const int64_t p = s[2];
    if (s[3] != kD || s[1] < 1 || p < 16 || p > 256 || (p & (p - 1)) || s[0] > INT32_MAX || s[1] > INT32_MAX)
      throw Refused{"pages must be [n_pages, hkv, page, 128] with 16, 32, 64, 128 or 256 tokens a page, got " + text(s)};
    auto c = std::make_unique<CacheInfo>();
    c->device = k.device();
    c->type = type;
    c->n_pages = (int32_t)s[0];
    c->hkv = (int32_t)s[1];
    c->page = (int32_t)p;
    c->dtype = type == at::kBFloat16 ? NSA_SEL_CACHE_BF16 : NSA_SEL_CACHE_E4M3;
    c->t[0] = k;
    c->t[1] = dims(a[1], "v_pages", 4);
    if (c->dtype == NSA_SEL_CACHE_E4M3) {
      c->t[2] = dims(a[2], "k_scale", 2);
      c->t[3] = dims(a[3], "v_scale", 2);
    } else if (a[2] != Py_None || a[3] != Py_None) {
      throw Refused{"bfloat16 pages have no scales"};
    }
    pages(*c);
    PyObject* o = PyCapsule_New(c.get(), kCapsule, free_info);
    if (o) c.release();
    return o;
  } catch (const Refused& r) {
    PyErr_SetString(g_error, r.why.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// What all calls have: table, lengths, starts.
struct Batch {
  const int32_t *table, *kv_len, *cu;
  int64_t nseq, max_pages;
};
const int32_t* starts(PyObject* o, int64_t nseq, int64_t tokens, const at::Device& dev) {
  if (o != Py_None) return (const int32_t*)expect(dims(o, "cu_seqlens", 1), "cu_seqlens", at::kInt, {nseq + 1}, dev);
  if (nseq != tokens)
    throw Refused{"without cu_seqlens every sequence has one new token: " + std::to_string(nseq) + " sequences for " + std::to_string(tokens) + " tokens"};
  return nullptr;
}
Batch batch(PyObject* table, PyObject* kv_len, PyObject* cu, int64_t tokens, const at::Device& dev) {
  const at::Tensor& t = dims(table, "table", 2);
  Batch b;
  b.nseq = t.size(0);
  b.max_pages = t.size(1);
  if (b.nseq > INT32_MAX || b.max_pages > INT32_MAX) throw Refused{"table is too large"};
  b.table = (const int32_t*)expect(t, "table", at::kInt, {b.nseq, b.max_pages}, dev);
  b.kv_len = (const int32_t*)expect(tensor(kv_len, "kv_len"), "kv_len", at::kInt, {b.nseq}, dev);
  b.cu = starts(cu, b.nseq, tokens, dev);
  return b;
}
nsa_sel_cache_shape shape_of(const CacheInfo& c, const Batch& b, int64_t tokens, int64_t hq) {
  if (tokens > INT32_MAX || hq > INT32_MAX) throw Refused{"too many tokens or heads"};
  nsa_sel_cache_shape s = {};
  s.n_tokens = (int32_t)tokens;
  s.nseq = (int32_t)b.nseq;
  s.hq = (int32_t)hq;
  s.hkv = c.hkv;
  s.d = kD;
  s.dtype = c.dtype;
  s.page = c.page;
  s.n_pages = c.n_pages;
  s.max_pages = (int32_t)b.max_pages;
  s.block = 64;
  return s;
}
PyObject* given(PyObject* o) {
  Py_INCREF(o);
  return o;
}

// (info, k, v, table, kv_len, cu, q, inv_freq, interleaved, rotated_k, q_out, k_out, stream) -> (rotated q or None, rotated k or None)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 13);
    const CacheInfo& c = info(a[0]);
    const Pages p = pages(c);
    const at::Tensor &k = dims(a[1], "k", 3), &v = dims(a[2], "v", 3);
    const int64_t T = k.size(0);
    const int64_t kv_rows[3] = {T, c.hkv, kD};
    const int64_t k_stride = expect_rows(k, "k", kv_rows, c.device), v_stride = expect_rows(v, "v", kv_rows, c.device);
    const Batch b = batch(a[3], a[4], a[5], T, c.device);
    int64_t hq = c.hkv, q_stride = 0;
    void *q_ptr = nullptr, *q_out = nullptr, *k_out = nullptr;
    at::Tensor new_q, new_k;
    const auto options = at::TensorOptions().dtype(at::kBFloat16).device(c.device);
    if (a[6] != Py_None) {
      const at::Tensor& q = dims(a[6], "q", 3);
      hq = q.size(1);
      const int64_t rows[3] = {T, hq, kD};
      q_stride = expect_rows(q, "q", rows, c.device);
      q_ptr = q.data_ptr();
      if (a[10] != Py_None) {
        q_out = expect(tensor(a[10], "q_out"), "q_out", at::kBFloat16, rows, c.device);
      } else {
        new_q = empty(rows, options);
        q_out = new_q.data_ptr();
      }
    } else if (a[10] != Py_None) {
      throw Refused{"q_out without q"};
    }
    if (a[11] != Py_None) {
      k_out = expect(tensor(a[11], "k_out"), "k_out", at::kBFloat16, kv_rows, c.device);
    } else if (truth(a[9])) {
      new_k = empty(kv_rows, options);
      k_out = new_k.data_ptr();
    }
    const double* freq = nullptr;
    int64_t pairs = 0;
    if (a[7] != Py_None) {
      const at::Tensor& f = dims(a[7], "inv_freq", 1);
      pairs = f.size(0);
      freq = (const double*)expect(f, "inv_freq", at::kDouble, {pairs}, c.device);
      if (pairs > kD) throw Refused{"inv_freq must be float64 [rot / 2], rot a multiple of 16 up to 128"};
    }
    const nsa_sel_cache_shape s = shape_of(c, b, T, hq);
    on_gpu(c.device);
    const bool interleaved = truth(a[8]);
    void* const stream = PyLong_AsVoidPtr(a[12]);
    done(without_gil([&] {
           return nsa_sel_cache_append(&s, q_ptr, q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, b.cu, b.kv_len, b.table, freq,
                                       (int32_t)(2 * pairs), interleaved, p.k, p.v, p.ks, p.vs, q_out, k_out, stream);
         }),
         "nsa_sel_cache_append");
    PyObject* r = PyTuple_New(2);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, new_q.defined() ? THPVariable_Wrap(std::move(new_q)) : given(a[6] == Py_None ? Py_None : a[10]));
    PyTuple_SET_ITEM(r, 1, new_k.defined() ? THPVariable_Wrap(std::move(new_k)) : given(a[11]));
    return r;
  } catch (const Refused& r) {
    PyErr_SetString(g_error, r.why.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (info, q, table, kv_len, cu, idx, block, window, scale, gate, o_acc, out, lse, ws, stream) -> (O, LSE)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 15);
    const CacheInfo& c = info(a[0]);
    const Pages p = pages(c);
    const at::Tensor& q = dims(a[1], "q", 3);
    const int64_t T = q.size(0), hq = q.size(1);
    const int64_t rows[3] = {T, hq, kD}, per_row[2] = {T, hq};
    const void* q_ptr = expect(q, "q", at::kBFloat16, rows, c.device);
    const Batch b = batch(a[2], a[3], a[4], T, c.device);
    nsa_sel_cache_shape s = shape_of(c, b, T, hq);
    const int32_t* idx = nullptr;
    if (a[5] != Py_None) {
      const at::Tensor& x = dims(a[5], "idx", 3);
      if (x.size(2) < 1 || x.size(2) > INT32_MAX) throw Refused{"idx must be int32 [tokens, hkv, topk], topk at least 1"};
      s.topk = (int32_t)x.size(2);
      idx = (const int32_t*)expect(x, "idx", at::kInt, {T, c.hkv, x.size(2)}, c.device);
    }
    s.block = small(a[6], "block");
    s.window = small(a[7], "window");
    s.scale = number(a[8]);
    const float* gate = nullptr;
    const void* acc = nullptr;
    if (a[9] != Py_None) {
      gate = (const float*)expect(tensor(a[9], "gate"), "gate", at::kFloat, per_row, c.device);
      if (a[10] != Py_None) acc = expect(tensor(a[10], "o_acc"), "o_acc", at::kBFloat16, rows, c.device);
    } else if (a[10] != Py_None) {
      throw Refused{"o_acc without gate"};
    }
    const auto options = at::TensorOptions().device(c.device);
    at::Tensor new_o, new_l, new_ws;
    void *out, *lse, *ws = nullptr;
    size_t need = 0;
    done(nsa_sel_cache_workspace_bytes(&s, &need), "nsa_sel_cache_workspace_bytes");
    if (a[13] != Py_None) {
      const at::Tensor& w = tensor(a[13], "ws");
      if (w.device() != c.device || !w.is_contiguous()) throw Refused{"ws must be a contiguous tensor on " + c.device.str()};
      if (w.nbytes() < need) throw Refused{"ws holds " + std::to_string(w.nbytes()) + " bytes, " + std::to_string(need) + " are needed"};
      ws = w.data_ptr();
    } else if (need > 0) {
      new_ws = empty({(int64_t)need}, options.dtype(at::kByte));
      ws = new_ws.data_ptr();
    }
    if (a[11] != Py_None) {
      out = expect(tensor(a[11], "out"), "out", at::kBFloat16, rows, c.device);
    } else {
      new_o = empty(rows, options.dtype(at::kBFloat16));
      out = new_o.data_ptr();
    }
    if (a[12] != Py_None) {
      lse = expect(tensor(a[12], "lse"), "lse", at::kFloat, per_row, c.device);
    } else {
      new_l = empty(per_row, options.dtype(at::kFloat));
      lse = new_l.data_ptr();
    }
    on_gpu(c.device);
    void* const stream = PyLong_AsVoidPtr(a[14]);
    done(without_gil([&] {
           return nsa_sel_cache_attention(&s, q_ptr, idx, b.cu, b.kv_len, b.table, p.k, p.v, p.ks, p.vs, gate, acc, out, (float*)lse, ws, need, stream);
         }),
         "nsa_sel_cache_attention");
    PyObject* r = PyTuple_New(2);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, new_o.defined() ? THPVariable_Wrap(std::move(new_o)) : given(a[11]));
    PyTuple_SET_ITEM(r, 1, new_l.defined() ? THPVariable_Wrap(std::move(new_l)) : given(a[12]));
    return r;
  } catch (const Refused& r) {
    PyErr_SetString(g_error, r.why.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (scores, kv_len, cu, topk, block, n_sink, n_local, out, stream) -> idx
PyObject* select_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    count(n, 9);
    const at::Tensor& x = dims(a[0], "scores", 3);
    const at::Device dev = x.device();
    const int64_t T = x.size(0), hkv = x.size(1), stride = x.size(2);
    const void* scores = expect(x.requires_grad() ? x.detach() : x, "scores", at::kFloat, x.sizes(), dev);  // block ids have no gradient
    const at::Tensor& lengths = dims(a[1], "kv_len", 1);
    const int64_t nseq = lengths.size(0);
    if (T > INT32_MAX || hkv > INT32_MAX || nseq > INT32_MAX) throw Refused{"too many tokens, heads or sequences"};
    const void* kv_len = expect(lengths, "kv_len", at::kInt, {nseq}, dev);
    const int32_t* cu = starts(a[2], nseq, T, dev);
    nsa_sel_cache_shape s = {};
    s.n_tokens = (int32_t)T;
    s.nseq = (int32_t)nseq;
    s.hq = s.hkv = (int32_t)hkv;
    s.d = kD;
    s.page = 64;
    s.topk = small(a[3], "topk");
    s.block = small(a[4], "block");
    if (s.topk < 0) throw Refused{"topk must not be negative"};
    at::Tensor made;
    void* out;
    const int64_t rows[3] = {T, hkv, s.topk};
    if (a[7] != Py_None) {
      out = expect(tensor(a[7], "out"), "out", at::kInt, rows, dev);
    } else {
      const auto options = at::TensorOptions().dtype(at::kInt).device(dev);
      made = cu ? without_gil([&] { return at::full(rows, -1, options); }) : empty(rows, options);  // rows of no sequence stay -1
      out = made.data_ptr();
    }
    on_gpu(dev);
    const int32_t n_sink = small(a[5], "n_sink"), n_local = small(a[6], "n_local");
    void* const queue = PyLong_AsVoidPtr(a[8]);
    done(without_gil([&] {
           return nsa_sel_select_blocks_cached(&s, (const float*)scores, stride, cu, (const int32_t*)kv_len, n_sink, n_local, (int32_t*)out, queue);
         }),
         "nsa_sel_select_blocks_cached");
    return made.defined() ? THPVariable_Wrap(std::move(made)) : given(a[7]);
  } catch (const Refused& r) {
    PyErr_SetString(g_error, r.why.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XINCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {{"describe", (PyCFunction)(void (*)(void))describe, METH_FASTCALL, nullptr},
                          {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
                          {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, nullptr},
                          {"select_blocks", (PyCFunction)(void (*)(void))select_blocks, METH_FASTCALL, nullptr},
                          {"set_error", set_error, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_cache_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache_native() { return PyModule_Create(&kModule); }
