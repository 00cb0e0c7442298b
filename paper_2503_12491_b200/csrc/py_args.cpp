// Argument marshalling of the Python binding in native code: tensors to device pointers, the current
// CUDA stream, the call.  Every function takes the address of the context (0 after destroy) and
// returns the library's status; a tensor that the library cannot take raises ValueError.
//
// The entry points of the path are called once per layer or per layer and token: through ctypes a
// decode step cost 11 us on the host, of which 8 us were attribute look-ups and argument conversion.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <dlfcn.h>

#include <exception>
#include <stdexcept>
#include <string>
#include <vector>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cake.h"

namespace {

struct Lib {
  decltype(&cake_begin) begin;
  decltype(&cake_score_layer) score_layer;
  decltype(&cake_allocate) allocate;
  decltype(&cake_evict) evict;
  decltype(&cake_compact) compact;
  decltype(&cake_compact_int4) compact_int4;
  decltype(&cake_clear_unused) clear_unused;
  decltype(&cake_decode_step) decode_step;
  decltype(&cake_decode_get_state) decode_get_state;
  decltype(&cake_select_positions_static) select_positions_static;
  decltype(&cake_attend_prompt) attend_prompt;
  decltype(&cake_accumulate_attention) accumulate_attention;
  decltype(&cake_attend_workspace_bytes) attend_workspace_bytes;
  decltype(&cake_attend_cache) attend_cache;
  decltype(&cake_attend_int4) attend_int4;
} lib;

// The current CUDA stream; false with a Python error set if there is none (no usable device).
bool stream(void** st) {
  try {
    *st = (void*)c10::cuda::getCurrentCUDAStream().stream();
    return true;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
}

cake_ctx* ctx_of(PyObject* h) { return (cake_ctx*)PyLong_AsVoidPtr(h); }

constexpr at::ScalarType kAny = at::ScalarType::Undefined;
at::ScalarType element(PyObject* is_fp32) {
  return PyObject_IsTrue(is_fp32) ? at::ScalarType::Float : at::ScalarType::BFloat16;
}

// Device pointer of a tensor (null for None); false with a Python error set if the library cannot
// take it.
bool ptr(PyObject* o, at::ScalarType want, void** out, bool pinned_ok = false) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor or None");
    return false;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  try {
    if (!t.is_cuda() && !(pinned_ok && t.is_pinned())) {
      PyErr_SetString(PyExc_ValueError, pinned_ok ? "libcake takes CUDA tensors only (or pinned host tensors here)"
                                                  : "libcake takes CUDA tensors only");
      return false;
    }
    if (!t.is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "tensor must be contiguous");
      return false;
    }
    if (want != kAny && t.scalar_type() != want) {
      PyErr_Format(PyExc_ValueError, "expected torch.%s, got torch.%s",
                   want == at::ScalarType::Float ? "float32" : want == at::ScalarType::BFloat16 ? "bfloat16"
                   : want == at::ScalarType::Long ? "int64" : "int32",
                   c10::toString(t.scalar_type()));
      return false;
    }
    *out = t.data_ptr();
    return true;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return false;
  }
}

// The pointers of a sequence of tensors.
bool ptrs(PyObject* seq, at::ScalarType want, bool pinned_ok, std::vector<const void*>& out) {
  PyObject* fast = PySequence_Fast(seq, "expected a sequence of tensors");
  if (!fast) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
  out.resize((size_t)n);
  bool ok = true;
  for (Py_ssize_t i = 0; ok && i < n; ++i) {
    void* p;
    ok = ptr(PySequence_Fast_GET_ITEM(fast, i), want, &p, pinned_ok);
    out[(size_t)i] = p;
  }
  Py_DECREF(fast);
  return ok;
}

// One pointer per layer in both arrays; missing ones are null.
bool per_layer(std::vector<const void*>& k, std::vector<const void*>& v, long layers) {
  if (PyErr_Occurred()) return false;               // `layers` was not a number
  if (layers < 0 || layers > CAKE_MAX_LAYERS) {
    PyErr_SetString(PyExc_ValueError, "no such number of layers");
    return false;
  }
  if (k.size() > (size_t)layers || v.size() > (size_t)layers) {
    PyErr_SetString(PyExc_IndexError, "more tensors than layers");
    return false;
  }
  k.resize((size_t)layers, nullptr);
  v.resize((size_t)layers, nullptr);
  return true;
}

bool integers(PyObject* seq, std::vector<int64_t>& out) {
  PyObject* fast = PySequence_Fast(seq, "expected a sequence of integers");
  if (!fast) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
  out.resize((size_t)n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* v = PyNumber_Long(PySequence_Fast_GET_ITEM(fast, i));
    out[(size_t)i] = v ? PyLong_AsLongLong(v) : -1;
    Py_XDECREF(v);
    if (PyErr_Occurred()) break;
  }
  Py_DECREF(fast);
  return !PyErr_Occurred();
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

#define INT(i) ((int32_t)PyLong_AsLong(a[i]))
// Makes the call on the current stream, `st` in its arguments, without the interpreter lock (it may
// wait for room in the launch queue).
#define DONE(call)                            \
  do {                                        \
    if (PyErr_Occurred()) return nullptr;     \
    int32_t rc_;                              \
    void* st;                                 \
    if (!stream(&st)) return nullptr;         \
    Py_BEGIN_ALLOW_THREADS                    \
    rc_ = (call);                             \
    Py_END_ALLOW_THREADS                      \
    return PyLong_FromLong((long)rc_);        \
  } while (0)

// init(path of libcake.so)
PyObject* init(PyObject*, PyObject* path) {
  const char* p = PyUnicode_AsUTF8(path);
  if (!p) return nullptr;
  void* h = dlopen(p, RTLD_NOW | RTLD_LOCAL);
  if (!h) {
    PyErr_SetString(PyExc_ImportError, dlerror());
    return nullptr;
  }
#define SYM(name)                                                  \
  lib.name = (decltype(lib.name))dlsym(h, "cake_" #name);          \
  if (!lib.name) {                                                 \
    PyErr_SetString(PyExc_ImportError, "libcake lacks cake_" #name); \
    return nullptr;                                                \
  }
  SYM(begin) SYM(score_layer) SYM(allocate) SYM(evict) SYM(compact) SYM(compact_int4) SYM(clear_unused)
  SYM(decode_step) SYM(decode_get_state) SYM(select_positions_static)
  SYM(attend_prompt) SYM(accumulate_attention) SYM(attend_workspace_bytes) SYM(attend_cache) SYM(attend_int4)
#undef SYM
  Py_RETURN_NONE;
}

// begin(ctx, cu_seqlens)
PyObject* begin(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 2)) return nullptr;
  std::vector<int64_t> cu;
  if (!integers(a[1], cu)) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  DONE(lib.begin(c, (int32_t)cu.size() - 1, cu.data(), st));
}

// score_layer(ctx, layer, is_fp32, q_win, k, lse)
PyObject* score_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *q, *k, *lse;
  if (!arity(n, 6)) return nullptr;
  const at::ScalarType e = element(a[2]);
  if (!ptr(a[3], e, &q) || !ptr(a[4], e, &k) || !ptr(a[5], at::ScalarType::Float, &lse)) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t layer = INT(1);
  DONE(lib.score_layer(c, layer, q, k, (const float*)lse, st));
}

PyObject* allocate(PyObject*, PyObject* const* a, Py_ssize_t n) {      // (ctx, stage)
  if (!arity(n, 2)) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t stage = INT(1);
  DONE(lib.allocate(c, stage, st));
}

PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {         // (ctx, stage)
  if (!arity(n, 2)) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t stage = INT(1);
  DONE(lib.evict(c, stage, st));
}

// prefill(ctx, n_layers, is_fp32, q_layers, k_layers): score, allocate and evict of every layer
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  const at::ScalarType e = element(a[2]);
  const int32_t layers = INT(1);
  std::vector<const void*> q, k;
  if (!ptrs(a[3], e, false, q) || !ptrs(a[4], e, false, k) || PyErr_Occurred()) return nullptr;
  if ((int64_t)q.size() < layers || (int64_t)k.size() < layers) {
    PyErr_SetString(PyExc_IndexError, "fewer tensors than layers");
    return nullptr;
  }
  cake_ctx* c = ctx_of(a[0]);
  auto all = [&](void* st) {
    int32_t rc = CAKE_OK;
    for (int32_t l = 0; l < layers && rc == CAKE_OK; ++l) {
      rc = lib.score_layer(c, l, q[l], k[l], nullptr, st);
      if (rc == CAKE_OK) rc = lib.allocate(c, l, st);
      if (rc == CAKE_OK) rc = lib.evict(c, l, st);
    }
    return rc;
  };
  DONE(all(st));
}

// compact(ctx, n_layers, is_fp32, lo, hi, k_layers, v_layers, k_out, v_out, row_offsets, positions)
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  const at::ScalarType e = element(a[2]);
  std::vector<const void*> k, v;
  void *ko, *vo, *off, *pos;
  // K/V of a layer may also live in pinned host memory: the gather then fetches only the retained
  // rows over the bus
  if (!ptrs(a[5], e, true, k) || !ptrs(a[6], e, true, v) || !ptr(a[7], kAny, &ko) || !ptr(a[8], kAny, &vo) ||
      !ptr(a[9], at::ScalarType::Long, &off) || !ptr(a[10], at::ScalarType::Int, &pos)) return nullptr;
  if (!per_layer(k, v, PyLong_AsLong(a[1]))) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t lo = INT(3), hi = INT(4);
  DONE(lib.compact(c, lo, hi, k.data(), v.data(), ko, vo, (int64_t*)off, (int32_t*)pos, st));
}

// compact_int4(ctx, n_layers, is_fp32, group, k_layers, v_layers, k_codes, k_scale, k_zero, v_codes,
//              v_scale, v_zero, row_offsets, kgroup_offsets, positions)
PyObject* compact_int4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 15)) return nullptr;
  const at::ScalarType e = element(a[2]);
  std::vector<const void*> k, v;
  void* o[9];
  if (!ptrs(a[4], e, false, k) || !ptrs(a[5], e, false, v)) return nullptr;
  for (int i = 0; i < 9; ++i)
    if (!ptr(a[6 + i], kAny, &o[i])) return nullptr;
  if (!per_layer(k, v, PyLong_AsLong(a[1]))) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t layers = INT(1), group = INT(3);
  DONE(lib.compact_int4(c, 0, layers, k.data(), v.data(), group, (uint8_t*)o[0], (float*)o[1], (float*)o[2], (uint8_t*)o[3],
                        (float*)o[4], (float*)o[5], (int64_t*)o[6], (int64_t*)o[7], (int32_t*)o[8], st));
}

// clear_unused(tensors, offsets): zeroes the rows of every tensor beyond the last entry of its offsets
PyObject* clear_unused(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 2)) return nullptr;
  void* bufs[CAKE_CLEAR_MAX];
  const int64_t* used[CAKE_CLEAR_MAX];
  int64_t bytes[CAKE_CLEAR_MAX], rows[CAKE_CLEAR_MAX];
  int32_t m = 0;
  auto fill = [&](PyObject* tensors, PyObject* offsets) {
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(tensors);
    if (count > CAKE_CLEAR_MAX || PySequence_Fast_GET_SIZE(offsets) != count) {
      PyErr_SetString(PyExc_ValueError, "clear_unused: too many tensors, or not an offsets tensor for each");
      return false;
    }
    for (; m < (int32_t)count; ++m) {
      PyObject *x = PySequence_Fast_GET_ITEM(tensors, m), *o = PySequence_Fast_GET_ITEM(offsets, m);
      void* off;
      if (!THPVariable_Check(x) || !THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a torch.Tensor");
        return false;
      }
      if (!ptr(x, kAny, &bufs[m]) || !ptr(o, at::ScalarType::Long, &off)) return false;
      const at::Tensor &t = THPVariable_Unpack(x), &u = THPVariable_Unpack(o);
      if (t.dim() < 1 || u.numel() < 1) {
        PyErr_SetString(PyExc_ValueError, "clear_unused: a tensor without rows, or empty offsets");
        return false;
      }
      rows[m] = t.size(0);
      bytes[m] = rows[m] > 0 ? (int64_t)t.nbytes() / rows[m] : 0;
      used[m] = (const int64_t*)off + (u.numel() - 1);
    }
    return true;
  };
  PyObject* tensors = PySequence_Fast(a[0], "expected a sequence of tensors");
  PyObject* offsets = tensors ? PySequence_Fast(a[1], "expected a sequence of tensors") : nullptr;
  const bool ok = offsets && fill(tensors, offsets);
  Py_XDECREF(tensors);
  Py_XDECREF(offsets);
  if (!ok) return nullptr;
  DONE(lib.clear_unused(m, bufs, bytes, rows, used, st));
}

// decode_step(ctx, layer, is_fp32, q_new, k_new, v_new, k_cache, v_cache)
PyObject* decode_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *q, *k, *v, *kc, *vc;
  if (!arity(n, 8)) return nullptr;
  const at::ScalarType e = element(a[2]);
  if (!ptr(a[3], e, &q) || !ptr(a[4], e, &k) || !ptr(a[5], e, &v) || !ptr(a[6], kAny, &kc) || !ptr(a[7], kAny, &vc))
    return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t layer = INT(1);
  DONE(lib.decode_step(c, layer, q, k, v, kc, vc, st));
}

// decode_get_state(ctx, req, layer, positions, scores, slots)
PyObject* decode_get_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *p, *s, *sl;
  if (!arity(n, 6)) return nullptr;
  if (!ptr(a[3], kAny, &p) || !ptr(a[4], kAny, &s) || !ptr(a[5], kAny, &sl)) return nullptr;
  cake_ctx* c = ctx_of(a[0]);
  const int32_t req = INT(1), layer = INT(2);
  DONE(lib.decode_get_state(c, req, layer, (int32_t*)p, (float*)s, (int32_t*)sl, st));
}

// select(values, n_heads, n, keep, out)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void *v, *o;
  if (!arity(n, 5)) return nullptr;
  if (!ptr(a[0], at::ScalarType::Float, &v) || !ptr(a[4], at::ScalarType::Int, &o)) return nullptr;
  const int32_t heads = INT(1), len = INT(2), keep = INT(3);
  DONE(lib.select_positions_static((const float*)v, heads, len, keep, (int32_t*)o, st));
}

// ---- attention over prompts and caches: shapes are checked here, outputs allocated where none are given

// The tensor of an argument, on the current device and of the wanted type and shape (-1: any size); `strided`: only its
// channels have to be contiguous.  Throws what becomes a Python error.
const at::Tensor& tensor(PyObject* o, const char* name, at::ScalarType want, at::IntArrayRef shape, bool strided = false) {
  if (!THPVariable_Check(o)) throw std::invalid_argument(std::string(name) + ": expected a torch.Tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  auto fail = [&](const std::string& why) { throw std::invalid_argument(std::string(name) + ": " + why); };
  if (!t.is_cuda()) fail("libcake takes CUDA tensors only");
  if (t.get_device() != c10::cuda::current_device()) fail("tensor is not on the current device");
  if (t.scalar_type() != want) fail(std::string("expected ") + c10::toString(want) + ", got " + c10::toString(t.scalar_type()));
  bool same = t.dim() == (int64_t)shape.size();
  for (size_t i = 0; same && i < shape.size(); ++i) same = shape[i] < 0 || t.size((int64_t)i) == shape[i];
  if (!same) {
    std::string w;
    for (int64_t x : shape) w += (w.empty() ? "[" : ", ") + (x < 0 ? std::string("*") : std::to_string(x));
    fail("expected shape " + w + "]");
  }
  if (strided ? t.size(-1) > 1 && t.stride(-1) != 1 : !t.is_contiguous()) fail("tensor must be contiguous");
  return t;
}
at::Tensor tensor_or_new(PyObject* o, const char* name, at::ScalarType want, at::IntArrayRef shape, const at::Tensor& like) {
  return o != Py_None ? tensor(o, name, want, shape) : at::empty(shape, like.options().dtype(want));
}
// Strides between heads and tokens of [head][token][channel]; what one head or token alone has is not its tensor's.
void strides(const at::Tensor& t, int64_t& head, int64_t& token) {
  token = t.size(1) > 1 ? t.stride(1) : t.size(2);
  head = t.size(0) > 1 ? t.stride(0) : t.size(1) * token;
}
int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw std::invalid_argument("");
  return v;
}
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::invalid_argument& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// (status, tensor or None, tensor or None)
PyObject* answer(int32_t rc, const at::Tensor& a, const at::Tensor& b) {
  PyObject* x = a.defined() ? THPVariable_Wrap(a) : Py_NewRef(Py_None);
  PyObject* y = b.defined() ? THPVariable_Wrap(b) : Py_NewRef(Py_None);
  return Py_BuildValue("iNN", (int)rc, x, y);
}
template <typename F>
int32_t released(F f) {
  void* st = (void*)c10::cuda::getCurrentCUDAStream().stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f(st);
  Py_END_ALLOW_THREADS
  return rc;
}

// attend_prompt(ctx, is_fp32, n_req, tokens, q_heads, kv_heads, head_dim, window, q, k, v, out, lse, lse_window)
PyObject* attend_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 14)) return nullptr;
  return guarded([&] {
    const at::ScalarType e = element(a[1]), f = at::ScalarType::Float;
    const int64_t R = integer(a[2]), T = integer(a[3]), hq = integer(a[4]), hkv = integer(a[5]), d = integer(a[6]), w = integer(a[7]);
    const at::Tensor &q = tensor(a[8], "q", e, {hq, T, d}, true), &k = tensor(a[9], "k", e, {hkv, T, d}),
                     &v = tensor(a[10], "v", e, {hkv, T, d});
    const at::Tensor out = a[11] != Py_None ? tensor(a[11], "out", e, {hq, T, d}, true) : at::empty_like(q);
    const at::Tensor lse = tensor_or_new(a[12], "lse", f, {hq, T}, q);
    float* lw = a[13] != Py_None ? (float*)tensor(a[13], "lse_window", f, {R, hq, w}).data_ptr() : nullptr;
    int64_t qh, qt, oh, ot;
    strides(q, qh, qt);
    strides(out, oh, ot);
    cake_ctx* c = ctx_of(a[0]);
    const int32_t rc = released([&](void* st) {
      return lib.attend_prompt(c, q.data_ptr(), qh, qt, k.data_ptr(), v.data_ptr(), out.data_ptr(), oh, ot, (float*)lse.data_ptr(),
                               lw, st);
    });
    return answer(rc, out, lse);
  });
}

// accumulate_attention(ctx, is_fp32, tokens, q_heads, kv_heads, head_dim, q, k, lse, out)
PyObject* accumulate_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 10)) return nullptr;
  return guarded([&] {
    const at::ScalarType e = element(a[1]), f = at::ScalarType::Float;
    const int64_t T = integer(a[2]), hq = integer(a[3]), hkv = integer(a[4]), d = integer(a[5]);
    const at::Tensor &q = tensor(a[6], "q", e, {hq, T, d}, true), &k = tensor(a[7], "k", e, {hkv, T, d}),
                     &lse = tensor(a[8], "lse", f, {hq, T});
    const at::Tensor out = tensor_or_new(a[9], "out", f, {hkv, T}, q);
    int64_t qh, qt;
    strides(q, qh, qt);
    cake_ctx* c = ctx_of(a[0]);
    const int32_t rc = released([&](void* st) {
      return lib.accumulate_attention(c, q.data_ptr(), qh, qt, k.data_ptr(), (const float*)lse.data_ptr(), (float*)out.data_ptr(), st);
    });
    return answer(rc, out, at::Tensor());
  });
}

struct Tail {
  const void *k = nullptr, *v = nullptr;
  const int32_t* len = nullptr;
  int64_t cap = 0;
};
Tail tail_of(PyObject* const* a, at::ScalarType e, int64_t n_req, int64_t hkv, int64_t d) {     // k_tail, v_tail, tail_len
  Tail t;
  if (a[0] == Py_None && a[1] == Py_None && a[2] == Py_None) return t;
  const at::Tensor& k = tensor(a[0], "k_tail", e, {n_req, hkv, -1, d});
  t.cap = k.size(2);
  t.k = k.data_ptr();
  t.v = tensor(a[1], "v_tail", e, {n_req, hkv, t.cap, d}).data_ptr();
  t.len = (const int32_t*)tensor(a[2], "tail_len", at::ScalarType::Int, {n_req}).data_ptr();
  return t;
}

// Start of a part of a cache.  One without rows (all requests have tails alone) has no memory: it is never read, and anything
// stands for it.
const void* rows_of(const at::Tensor& t, const at::Tensor& stand_in) { return t.numel() ? t.data_ptr() : stand_in.data_ptr(); }

// attend_cache(ctx, is_fp32, layer, n_layers, q_heads, kv_heads, head_dim, q, row_offsets, k_tail, v_tail, tail_len, out, lse,
//              k_cache, v_cache)
// attend_int4(the same up to lse, k_codes, k_scale, k_zero, v_codes, v_scale, v_zero, kgroup_offsets)
PyObject* attend_cached(PyObject* const* a, bool int4) {
  return guarded([&] {
    const at::ScalarType e = element(a[1]), f = at::ScalarType::Float, u8 = at::ScalarType::Byte, i64 = at::ScalarType::Long;
    const int64_t layer = integer(a[2]), L = integer(a[3]), hq = integer(a[4]), hkv = integer(a[5]), d = integer(a[6]);
    const at::Tensor& q = tensor(a[7], "q", e, {-1, hq, d});
    const int64_t R = q.size(0);
    const int64_t* off = (const int64_t*)tensor(a[8], "row_offsets", i64, {R * L + 1}).data_ptr();
    const Tail t = tail_of(a + 9, e, R, hkv, d);
    if (R > INT32_MAX || layer != (int32_t)layer) throw std::invalid_argument("no such layer, or too many requests");
    const at::Tensor out = a[12] != Py_None ? tensor(a[12], "out", e, {R, hq, d}) : at::empty_like(q);
    const at::Tensor lse = tensor_or_new(a[13], "lse", f, {R, hq}, q);
    cake_ctx* c = ctx_of(a[0]);
    const int64_t bytes = lib.attend_workspace_bytes(c, (int32_t)R);
    if (bytes < 0) return answer((int32_t)bytes, out, lse);
    const at::Tensor ws = at::empty({bytes}, q.options().dtype(u8));
    int32_t rc;
    if (!int4) {
      const at::Tensor &k = tensor(a[14], "k_cache", e, {-1, d}), &v = tensor(a[15], "v_cache", e, {k.size(0), d});
      rc = released([&](void* st) {
        return lib.attend_cache(c, (int32_t)R, (int32_t)layer, q.data_ptr(), rows_of(k, ws), rows_of(v, ws), off, t.k, t.v, t.len, t.cap,
                                out.data_ptr(), (float*)lse.data_ptr(), ws.data_ptr(), bytes, st);
      });
    } else {
      const at::Tensor &kc = tensor(a[14], "k_codes", u8, {-1, d / 2}), &ks = tensor(a[15], "k_scale", f, {-1, d}),
                       &kz = tensor(a[16], "k_zero", f, {ks.size(0), d}), &vc = tensor(a[17], "v_codes", u8, {kc.size(0), d / 2}),
                       &vs = tensor(a[18], "v_scale", f, {kc.size(0), -1}), &vz = tensor(a[19], "v_zero", f, {kc.size(0), vs.size(1)});
      const int64_t* koff = (const int64_t*)tensor(a[20], "kgroup_offsets", i64, {R * L + 1}).data_ptr();
      if (vs.size(1) < 1 || d % vs.size(1)) throw std::invalid_argument("v_scale: no such group");
      rc = released([&](void* st) {
        return lib.attend_int4(c, (int32_t)R, (int32_t)layer, q.data_ptr(), (const uint8_t*)rows_of(kc, ws), (const float*)rows_of(ks, ws),
                               (const float*)rows_of(kz, ws), (const uint8_t*)rows_of(vc, ws), (const float*)rows_of(vs, ws),
                               (const float*)rows_of(vz, ws), (int32_t)(d / vs.size(1)), off, koff, t.k, t.v, t.len, t.cap,
                               out.data_ptr(), (float*)lse.data_ptr(), ws.data_ptr(), bytes, st);
      });
    }
    return answer(rc, out, lse);
  });
}
PyObject* attend_cache(PyObject*, PyObject* const* a, Py_ssize_t n) { return arity(n, 16) ? attend_cached(a, false) : nullptr; }
PyObject* attend_int4(PyObject*, PyObject* const* a, Py_ssize_t n) { return arity(n, 21) ? attend_cached(a, true) : nullptr; }

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", init, METH_O, nullptr},
                         FAST(begin), FAST(score_layer), FAST(allocate), FAST(evict), FAST(prefill), FAST(compact),
                         FAST(compact_int4), FAST(clear_unused), FAST(decode_step), FAST(decode_get_state), FAST(select),
                         FAST(attend_prompt), FAST(accumulate_attention), FAST(attend_cache), FAST(attend_int4),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cake_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cake_py() { return PyModule_Create(&module); }
