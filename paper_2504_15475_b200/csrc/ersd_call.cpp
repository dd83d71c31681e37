// The calling side of binding.py: checks of the tensors a call is given, their addresses, the current
// stream, and the call itself, in one step of native code.  (Through ctypes and torch's Python
// attributes the same steps cost 6 us per call, more than the device needs for a small one: a drafted
// token went from 11.0 to 6.2 us.)  The library's functions come as addresses from binding.py,
// which loads it; nothing here computes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "ersd.h"

namespace {

decltype(&ersd_race_sample) f_race_sample;
decltype(&ersd_verify) f_verify;
decltype(&ersd_verify_noalloc) f_verify_noalloc;
decltype(&ersd_verify_tokens) f_verify_tokens;
decltype(&ersd_verify_tree) f_verify_tree;
decltype(&ersd_gsd_verify) f_gsd_verify;
decltype(&ersd_gsd_verify_tree) f_gsd_verify_tree;
decltype(&ersd_chunk_attention) f_chunk_attention;
decltype(&ersd_cache_append) f_cache_append;
decltype(&ersd_cache_commit) f_cache_commit;
decltype(&ersd_process_logits) f_process_logits;

PyObject* options_type;  // binding.py's ErsdOpts

struct Failed {};  // a Python exception is set

const char* dtype_name(at::ScalarType t) {
  switch (t) {
    case at::kInt: return "torch.int32";
    case at::kLong: return "torch.int64";
    case at::kFloat: return "torch.float32";
    case at::kBFloat16: return "torch.bfloat16";
    case at::kHalf: return "torch.float16";
    case at::kDouble: return "torch.float64";
    default: return c10::toString(t);
  }
}

// A contiguous CUDA tensor (of type `want` unless that is Undefined).
const at::Tensor& tensor(PyObject* o, at::ScalarType want, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
    throw Failed();
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) {
    PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
    throw Failed();
  }
  if (want != at::ScalarType::Undefined && t.scalar_type() != want) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, dtype_name(want));
    throw Failed();
  }
  if (!t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
    throw Failed();
  }
  return t;
}
const void* optional_tensor(PyObject* o, at::ScalarType want, const char* name) {
  return o == Py_None ? nullptr : tensor(o, want, name).data_ptr();
}

struct Logits {
  const void* data;
  at::ScalarType type;
  ersd_dtype code;
  int B, rows, V;
};
// Logits [B, rows, ld]; V (None: ld) is the vocabulary's size.
Logits logits(PyObject* o, PyObject* v, const char* name) {
  const at::Tensor& t = tensor(o, at::ScalarType::Undefined, name);
  Logits l;
  l.data = t.data_ptr();
  l.type = t.scalar_type();
  if (t.dim() != 3) {
    PyErr_Format(PyExc_ValueError, "%s must have three dimensions, got %d", name, (int)t.dim());
    throw Failed();
  }
  const int64_t ld = t.size(2);
  int64_t V = ld;
  if (v != Py_None) {
    PyObject* n = PyNumber_Long(v);
    if (!n) throw Failed();
    V = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (V == -1 && PyErr_Occurred()) throw Failed();
    if (V < 1 || V > ld) {
      PyErr_SetString(PyExc_ValueError, "V must be between 1 and the row length of the tensor");
      throw Failed();
    }
  }
  if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || V > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s has too many rows or columns", name);
    throw Failed();
  }
  l.B = (int)t.size(0);
  l.rows = (int)t.size(1);
  l.V = (int)V;
  return l;
}
void logits_code(Logits& l) {
  if (l.type == at::kFloat) l.code = ERSD_F32;
  else if (l.type == at::kBFloat16) l.code = ERSD_BF16;
  else {
    PyErr_Format(PyExc_TypeError, "logits must be float32 or bfloat16, got %s", dtype_name(l.type));
    throw Failed();
  }
}

float number(PyObject* o) {
  PyObject* f = PyNumber_Float(o);
  if (!f) throw Failed();
  const double v = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return (float)v;
}

void* stream_of(PyObject* o) {
  if (o == Py_None) return (void*)c10::cuda::getCurrentCUDAStream().stream();
  PyObject* a = PyObject_GetAttrString(o, "cuda_stream");
  if (!a) throw Failed();
  void* p = PyLong_AsVoidPtr(a);
  Py_DECREF(a);
  if (!p && PyErr_Occurred()) throw Failed();
  return p;
}

// The options structure (an ErsdOpts, which lends its memory), or none.  Nothing else is taken: the
// library copies the whole structure, addresses and all.
struct Options {
  Py_buffer view;
  const ersd_opts* ptr = nullptr;
  explicit Options(PyObject* o) {
    if (o == Py_None) return;
    const int is_options = PyObject_IsInstance(o, options_type);
    if (is_options < 0) throw Failed();
    if (!is_options) {
      PyErr_Format(PyExc_TypeError, "opts must be an ErsdOpts (see make_opts), got %s", Py_TYPE(o)->tp_name);
      throw Failed();
    }
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
    if (view.len < (Py_ssize_t)sizeof(ersd_opts)) {
      PyBuffer_Release(&view);
      PyErr_Format(PyExc_TypeError, "opts has %d bytes, the library's options %d", (int)view.len, (int)sizeof(ersd_opts));
      throw Failed();
    }
    ptr = (const ersd_opts*)view.buf;
  }
  ~Options() {
    if (ptr) PyBuffer_Release(&view);
  }
  Options(const Options&) = delete;
};

std::vector<int32_t> parents(PyObject* o, int nodes) {
  PyObject* seq = PySequence_Fast(o, "parent must be a sequence of integers");
  if (!seq) throw Failed();
  std::vector<int32_t> p((size_t)PySequence_Fast_GET_SIZE(seq));
  for (size_t i = 0; i < p.size(); ++i) {
    PyObject* n = PyNumber_Long(PySequence_Fast_GET_ITEM(seq, (Py_ssize_t)i));
    const long v = n ? PyLong_AsLong(n) : -1;
    Py_XDECREF(n);
    if (v == -1 && PyErr_Occurred()) {
      Py_DECREF(seq);
      throw Failed();
    }
    if (v < INT32_MIN || v > INT32_MAX) {
      Py_DECREF(seq);
      PyErr_SetString(PyExc_ValueError, "parent has an entry that is no 32-bit number");
      throw Failed();
    }
    p[i] = (int32_t)v;
  }
  Py_DECREF(seq);
  if (p.size() < (size_t)nodes) {
    PyErr_Format(PyExc_ValueError, "parent must have an entry for each of the %d nodes", nodes);
    throw Failed();
  }
  return p;
}

// Runs the call without the interpreter's lock; its status as a Python number.
template <typename F>
PyObject* status_of(F&& call) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

template <int N, typename F>
PyObject* guarded(Py_ssize_t n, F&& body) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments wanted, got %d", N, (int)n);
    return nullptr;
  }
  try {
    return body();
  } catch (const Failed&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// race_sample(logits, seeds, T, out_tok, opts, stream, V)
PyObject* race_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(n, [&]() {
    const Options o(a[4]);
    tensor(a[0], at::ScalarType::Undefined, "logits");
    const void* seeds = tensor(a[1], at::kLong, "seeds").data_ptr();
    int32_t* out = (int32_t*)tensor(a[3], at::kInt, "out_tok").data_ptr();
    Logits l = logits(a[0], a[6], "logits");
    logits_code(l);
    const float T = number(a[2]);
    void* st = stream_of(a[5]);
    return status_of([&] { return f_race_sample(l.data, l.code, (const uint64_t*)seeds, l.B, l.rows, l.V, T, out, o.ptr, st); });
  });
}

// verify(target, draft, seeds, T, out_tokens, out_accept_len, opts, stream, V)
template <typename Fn>
PyObject* verify_with(PyObject* const* a, Py_ssize_t n, Fn fn) {
  return guarded<9>(n, [&]() {
    const Options o(a[6]);
    Logits l = logits(a[0], a[8], "target_logits");
    const void* draft = optional_tensor(a[1], l.type, "draft_logits");
    const void* seeds = tensor(a[2], at::kLong, "seeds").data_ptr();
    int32_t* tok = (int32_t*)tensor(a[4], at::kInt, "out_tokens").data_ptr();
    int32_t* acc = (int32_t*)tensor(a[5], at::kInt, "out_accept_len").data_ptr();
    logits_code(l);
    const float T = number(a[3]);
    void* st = stream_of(a[7]);
    return status_of([&] { return fn(l.data, draft, l.code, (const uint64_t*)seeds, l.B, l.rows - 1, l.V, T, tok, acc, o.ptr, st); });
  });
}
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) { return verify_with(a, n, f_verify); }
PyObject* verify_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n) { return verify_with(a, n, f_verify_noalloc); }

// verify_tokens(target, draft_tokens, seeds, T, out_tokens, out_accept_len, opts, stream, V)
PyObject* verify_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<9>(n, [&]() {
    const Options o(a[6]);
    Logits l = logits(a[0], a[8], "target_logits");
    const void* given = optional_tensor(a[1], at::kInt, "draft_tokens");
    const void* seeds = tensor(a[2], at::kLong, "seeds").data_ptr();
    int32_t* tok = (int32_t*)tensor(a[4], at::kInt, "out_tokens").data_ptr();
    int32_t* acc = (int32_t*)tensor(a[5], at::kInt, "out_accept_len").data_ptr();
    logits_code(l);
    const float T = number(a[3]);
    void* st = stream_of(a[7]);
    return status_of([&] {
      return f_verify_tokens(l.data, (const int32_t*)given, l.code, (const uint64_t*)seeds, l.B, l.rows - 1, l.V, T, tok, acc, o.ptr, st);
    });
  });
}

// verify_tree(target, draft, parent, seeds, T, out_tokens, out_accept_len, opts, stream, V)
PyObject* verify_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<10>(n, [&]() {
    const Options o(a[7]);
    Logits l = logits(a[0], a[9], "target_logits");
    const void* draft = optional_tensor(a[1], l.type, "draft_logits");
    const void* seeds = tensor(a[3], at::kLong, "seeds").data_ptr();
    int32_t* tok = (int32_t*)tensor(a[5], at::kInt, "out_tokens").data_ptr();
    int32_t* acc = (int32_t*)tensor(a[6], at::kInt, "out_accept_len").data_ptr();
    const std::vector<int32_t> parent = parents(a[2], l.rows);
    logits_code(l);
    const float T = number(a[4]);
    void* st = stream_of(a[8]);
    return status_of([&] {
      return f_verify_tree(l.data, draft, l.code, parent.data(), (const uint64_t*)seeds, l.B, l.rows - 1, l.V, T, tok, acc, o.ptr, st);
    });
  });
}

// gsd_verify(target, draft, draft_tokens, seeds, T, out_tokens, out_accept_len, opts, stream, V)
PyObject* gsd_verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<10>(n, [&]() {
    const Options o(a[7]);
    Logits l = logits(a[0], a[9], "target_logits");
    const void* draft = optional_tensor(a[1], l.type, "draft_logits");
    const void* given = optional_tensor(a[2], at::kInt, "draft_tokens");
    const void* seeds = tensor(a[3], at::kLong, "seeds").data_ptr();
    int32_t* tok = (int32_t*)tensor(a[5], at::kInt, "out_tokens").data_ptr();
    int32_t* acc = (int32_t*)tensor(a[6], at::kInt, "out_accept_len").data_ptr();
    logits_code(l);
    const float T = number(a[4]);
    void* st = stream_of(a[8]);
    return status_of([&] {
      return f_gsd_verify(l.data, draft, (const int32_t*)given, l.code, (const uint64_t*)seeds, l.B, l.rows - 1, l.V, T, tok, acc, o.ptr, st);
    });
  });
}

// gsd_verify_tree(target, draft, draft_tokens, parent, seeds, T, out_tokens, out_accept_len, opts, stream, V)
PyObject* gsd_verify_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<11>(n, [&]() {
    const Options o(a[8]);
    Logits l = logits(a[0], a[10], "target_logits");
    const void* draft = optional_tensor(a[1], l.type, "draft_logits");
    const void* given = optional_tensor(a[2], at::kInt, "draft_tokens");
    const void* seeds = tensor(a[4], at::kLong, "seeds").data_ptr();
    int32_t* tok = (int32_t*)tensor(a[6], at::kInt, "out_tokens").data_ptr();
    int32_t* acc = (int32_t*)tensor(a[7], at::kInt, "out_accept_len").data_ptr();
    const std::vector<int32_t> parent = parents(a[3], l.rows);
    logits_code(l);
    const float T = number(a[5]);
    void* st = stream_of(a[9]);
    return status_of([&] {
      return f_gsd_verify_tree(l.data, draft, (const int32_t*)given, l.code, parent.data(), (const uint64_t*)seeds, l.B, l.rows - 1, l.V, T,
                               tok, acc, o.ptr, st);
    });
  });
}

// ---- calls over a cache and on logits: tensors of any strides whose innermost dimension is contiguous, all on
// one device, which is made the current one for the call (the stream is its current one unless one is given).

[[noreturn]] void refuse(PyObject* type, const char* format, const char* name) {
  PyErr_Format(type, format, name);
  throw Failed();
}

// A CUDA tensor of `dims` dimensions (0: any number) on `device`, its innermost dimension contiguous.
const at::Tensor& strided(PyObject* o, at::ScalarType want, int dims, const at::Tensor* with, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse(PyExc_ValueError, "%s must be a CUDA tensor", name);
  if (with && t.device() != with->device()) refuse(PyExc_ValueError, "%s must be on the same device as the other tensors", name);
  if (want != at::ScalarType::Undefined && t.scalar_type() != want) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, dtype_name(want));
    throw Failed();
  }
  if (dims && t.dim() != dims) {
    PyErr_Format(PyExc_ValueError, "%s must have %d dimensions, got %d", name, dims, (int)t.dim());
    throw Failed();
  }
  if (t.dim() && t.size(t.dim() - 1) > 1 && t.stride(t.dim() - 1) != 1)
    refuse(PyExc_ValueError, "the innermost dimension of %s must be contiguous", name);
  for (int64_t n : t.sizes())
    if (n > INT32_MAX) refuse(PyExc_ValueError, "%s has a dimension that is too long", name);
  return t;
}
// The addresses of a contiguous int32 or float tensor of the sizes wanted, or of none.
template <typename T>
const T* small(PyObject* o, std::initializer_list<int64_t> sizes, const at::Tensor& with, const char* name) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = strided(o, std::is_same<T, float>::value ? at::kFloat : at::kInt, 0, &with, name);
  if (t.sizes() != at::IntArrayRef(sizes.begin(), sizes.size())) refuse(PyExc_ValueError, "%s does not have the shape that goes with the call", name);
  if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", name);
  return (const T*)t.data_ptr();
}
int integer(PyObject* o, const char* name) {
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Failed();
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw Failed();
  if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, "%s is out of range", name);
  return (int)v;
}
ersd_dtype code_of(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kFloat) return ERSD_F32;
  if (t.scalar_type() != at::kBFloat16) {
    PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %s", name, dtype_name(t.scalar_type()));
    throw Failed();
  }
  return ERSD_BF16;
}

// k_cache, v_cache [pages, page, heads, dim] (commit: also [layers, ...]), block_table [B, entries].
ersd_cache cache_of(PyObject* k, PyObject* v, PyObject* table, bool layers, int64_t* B) {
  const at::Tensor& kc = strided(k, at::ScalarType::Undefined, 0, nullptr, "k_cache");
  const at::Tensor& vc = strided(v, kc.scalar_type(), 0, &kc, "v_cache");
  const at::Tensor& bt = strided(table, at::kInt, 2, &kc, "block_table");
  const int at = (int)kc.dim() - 4;
  if (at != 0 && !(layers && at == 1))
    refuse(PyExc_ValueError, "%s must have the dimensions [pages, positions of a page, heads, head_dim], with one for the layers "
           "before them where a call takes several layers", "k_cache");
  if (kc.sizes() != vc.sizes()) refuse(PyExc_ValueError, "%s must have the shape of k_cache", "v_cache");
  ersd_cache c;
  memset(&c, 0, sizeof c);
  c.struct_size = sizeof c;
  c.dtype = code_of(kc, "k_cache");
  c.k = kc.data_ptr();
  c.v = vc.data_ptr();
  c.layers = at ? (int)kc.size(0) : 1;
  c.num_pages = (int)kc.size(at);
  c.page_size = (int)kc.size(at + 1);
  c.heads = (int)kc.size(at + 2);
  c.head_dim = (int)kc.size(at + 3);
  c.k_stride_layer = at ? kc.stride(0) : 0;
  c.k_stride_page = kc.stride(at);
  c.k_stride_token = kc.stride(at + 1);
  c.k_stride_head = kc.stride(at + 2);
  c.v_stride_layer = at ? vc.stride(0) : 0;
  c.v_stride_page = vc.stride(at);
  c.v_stride_token = vc.stride(at + 1);
  c.v_stride_head = vc.stride(at + 2);
  c.block_table = (const int32_t*)bt.data_ptr();
  c.table_stride = bt.stride(0);
  c.max_pages = (int)bt.size(1);
  *B = bt.size(0);
  return c;
}
// Tensor [B, R, heads, dim] of the cache's type beside the cache.
const at::Tensor& rows_of(PyObject* o, const at::Tensor& kc, int64_t B, const char* name) {
  const at::Tensor& t = strided(o, kc.scalar_type(), 4, &kc, name);
  if (t.size(0) != B) refuse(PyExc_ValueError, "%s must have as many sequences as block_table", name);
  if (t.size(3) != kc.size(3)) refuse(PyExc_ValueError, "%s must have the cache's head_dim", name);
  return t;
}
// (strides that are all 0 mean contiguous: an expanded tensor of one row each is that)
void strides_of(const at::Tensor& t, int64_t* b, int64_t* r, int64_t* h) {
  *b = t.stride(0);
  *r = t.stride(1);
  *h = t.stride(2);
}
bool no_strides(const at::Tensor& t) { return !t.stride(0) && !t.stride(1) && !t.stride(2) && t.numel() > t.size(3); }

// chunk_attention(q, k_cache, v_cache, block_table, context_lens, out, scale, parent, row_counts, window, sinks,
//                 max_context, split, kernel_path, stream)
PyObject* chunk_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<15>(n, [&]() {
    int64_t B;
    const ersd_cache c = cache_of(a[1], a[2], a[3], false, &B);
    const at::Tensor& kc = THPVariable_Unpack(a[1]);
    const at::Tensor& q = rows_of(a[0], kc, B, "q");
    const at::Tensor& out = rows_of(a[5], kc, B, "out");
    if (out.sizes() != q.sizes()) refuse(PyExc_ValueError, "%s must have the shape of q", "out");
    if (no_strides(q) || no_strides(out)) refuse(PyExc_ValueError, "%s must not be one row expanded to all", "q or out");
    ersd_chunk_opts o;
    memset(&o, 0, sizeof o);
    o.struct_size = sizeof o;
    const int32_t* lens = small<int32_t>(a[4], {B}, kc, "context_lens");
    o.scale = a[6] == Py_None ? 0.0f : number(a[6]);
    if (a[6] != Py_None && o.scale == 0.0f) refuse(PyExc_ValueError, "%s must not be 0", "scale");  // (the library's sign for none given)
    std::vector<int32_t> parent;
    if (a[7] != Py_None) {
      parent = parents(a[7], (int)q.size(1));
      o.parent = parent.data();
    }
    o.row_counts = small<int32_t>(a[8], {B}, kc, "row_counts");
    o.window = integer(a[9], "window");
    o.sinks = integer(a[10], "sinks");
    o.max_context = integer(a[11], "max_context");
    o.split = integer(a[12], "split");
    o.kernel_path = (uint32_t)integer(a[13], "kernel_path");
    strides_of(q, &o.a_stride_b, &o.a_stride_r, &o.a_stride_h);
    strides_of(out, &o.b_stride_b, &o.b_stride_r, &o.b_stride_h);
    const c10::cuda::CUDAGuard guard(kc.device());
    void* st = stream_of(a[14]);
    return status_of([&] { return f_chunk_attention(&c, q.data_ptr(), out.data_ptr(), lens, (int)B, (int)q.size(1), (int)q.size(2), &o, st); });
  });
}

// cache_append(k_new, v_new, k_cache, v_cache, block_table, context_lens, row_counts, stream)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(n, [&]() {
    int64_t B;
    const ersd_cache c = cache_of(a[2], a[3], a[4], false, &B);
    const at::Tensor& kc = THPVariable_Unpack(a[2]);
    const at::Tensor& k = rows_of(a[0], kc, B, "k_new");
    const at::Tensor& v = rows_of(a[1], kc, B, "v_new");
    if (k.sizes() != v.sizes()) refuse(PyExc_ValueError, "%s must have the shape of k_new", "v_new");
    if (k.size(2) != kc.size(2)) refuse(PyExc_ValueError, "%s must have the cache's heads", "k_new");
    if (no_strides(k) || no_strides(v)) refuse(PyExc_ValueError, "%s must not be one row expanded to all", "k_new or v_new");
    ersd_chunk_opts o;
    memset(&o, 0, sizeof o);
    o.struct_size = sizeof o;
    const int32_t* lens = small<int32_t>(a[5], {B}, kc, "context_lens");
    o.row_counts = small<int32_t>(a[6], {B}, kc, "row_counts");
    strides_of(k, &o.a_stride_b, &o.a_stride_r, &o.a_stride_h);
    strides_of(v, &o.b_stride_b, &o.b_stride_r, &o.b_stride_h);
    const c10::cuda::CUDAGuard guard(kc.device());
    void* st = stream_of(a[7]);
    return status_of([&] { return f_cache_append(&c, k.data_ptr(), v.data_ptr(), lens, (int)B, (int)k.size(1), &o, st); });
  });
}

// cache_commit(k_cache, v_cache, block_table, context_lens, path, accept_len, out_context_lens, stream)
PyObject* cache_commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<8>(n, [&]() {
    int64_t B;
    const ersd_cache c = cache_of(a[0], a[1], a[2], true, &B);
    const at::Tensor& kc = THPVariable_Unpack(a[0]);
    const int32_t* lens = small<int32_t>(a[3], {B}, kc, "context_lens");
    const at::Tensor& path = strided(a[4], at::kInt, 2, &kc, "path");
    if (path.size(0) != B || path.size(1) < 1 || !path.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous [B, D+1]", "path");
    const int32_t* accept = small<int32_t>(a[5], {B}, kc, "accept_len");
    int32_t* out = (int32_t*)small<int32_t>(a[6], {B}, kc, "out_context_lens");
    const c10::cuda::CUDAGuard guard(kc.device());
    void* st = stream_of(a[7]);
    return status_of([&] { return f_cache_commit(&c, lens, (const int32_t*)path.data_ptr(), accept, (int)B, (int)path.size(1) - 1, out, st); });
  });
}

// process_logits(logits, out, history, history_lens, prompt_lens, draft_tokens, parent, repetition, presence,
//                frequency, bias_tokens, bias_values, mask, V, stream)
PyObject* process_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<15>(n, [&]() {
    const at::Tensor& x = strided(a[0], at::ScalarType::Undefined, 3, nullptr, "logits");
    const ersd_dtype code = code_of(x, "logits");
    const at::Tensor& y = strided(a[1], x.scalar_type(), 3, &x, "out");
    const int64_t B = x.size(0), R = x.size(1);
    if (y.sizes() != x.sizes()) refuse(PyExc_ValueError, "%s must have the shape of logits", "out");
    ersd_logit_opts o;
    memset(&o, 0, sizeof o);
    o.struct_size = sizeof o;
    // rows at equal distances: [B, R] can be walked as one
    auto row_stride = [&](const at::Tensor& t, const char* name) {
      if (R > 1 && B > 1 && t.stride(0) != R * t.stride(1)) refuse(PyExc_ValueError, "the rows of %s must be at equal distances", name);
      return R > 1 ? t.stride(1) : B > 1 ? t.stride(0) : t.size(2);
    };
    int64_t V = x.size(2);
    if (a[13] != Py_None) {
      V = integer(a[13], "V");
      if (V < 1 || V > x.size(2)) refuse(PyExc_ValueError, "%s must be between 1 and the row length of the tensor", "V");
    }
    o.ld_in = row_stride(x, "logits");
    o.ld_out = row_stride(y, "out");
    if (o.ld_in < V || o.ld_out < V) refuse(PyExc_ValueError, "the rows of %s must not overlap", "logits or out");
    if (a[2] != Py_None) {
      const at::Tensor& h = strided(a[2], at::kInt, 2, &x, "history");
      if (h.size(0) != B || !h.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous [B, width]", "history");
      o.history_width = (int)h.size(1);
      o.history = o.history_width ? (const int32_t*)h.data_ptr() : nullptr;  // (none yet: no lengths to look at either)
    }
    if (a[2] == Py_None || o.history) {
      o.history_lens = small<int32_t>(a[3], {B}, x, "history_lens");
      o.prompt_lens = small<int32_t>(a[4], {B}, x, "prompt_lens");
    }
    std::vector<int32_t> parent;
    if (a[6] != Py_None && a[5] != Py_None) {
      parent = parents(a[6], (int)R);
      o.parent = parent.data();
    }
    o.draft_tokens = small<int32_t>(a[5], {B, o.parent ? R : R - 1}, x, "draft_tokens");
    if (!o.draft_tokens) o.parent = nullptr;  // (a chain's single row: an empty tensor)
    o.repetition = small<float>(a[7], {B}, x, "repetition");
    o.presence = small<float>(a[8], {B}, x, "presence");
    o.frequency = small<float>(a[9], {B}, x, "frequency");
    if ((a[10] == Py_None) != (a[11] == Py_None)) refuse(PyExc_ValueError, "%s go together", "bias_tokens and bias_values");
    if (a[10] != Py_None) {
      const at::Tensor& t = strided(a[10], at::kInt, 2, &x, "bias_tokens");
      const at::Tensor& f = strided(a[11], at::kFloat, 2, &x, "bias_values");
      if ((t.size(0) != B && t.size(0) != 1) || t.sizes() != f.sizes() || !t.is_contiguous() || !f.is_contiguous())
        refuse(PyExc_ValueError, "%s must be contiguous, both [B, n] or [1, n]", "bias_tokens and bias_values");
      o.bias_count = (int)t.size(1);
      o.bias_stride = t.size(0) == 1 ? 0 : o.bias_count;
      o.bias_tokens = o.bias_count ? (const int32_t*)t.data_ptr() : nullptr;
      o.bias_values = o.bias_count ? (const float*)f.data_ptr() : nullptr;
    }
    if (a[12] != Py_None) {
      const at::Tensor& m = strided(a[12], at::kInt, 3, &x, "mask");
      if ((m.size(0) != B && m.size(0) != 1) || (m.size(1) != R && m.size(1) != 1) || m.size(2) < (V + 31) / 32)
        refuse(PyExc_ValueError, "%s must be [B or 1, R or 1, words] with a bit for each token", "mask");
      o.mask = (const uint32_t*)m.data_ptr();
      o.mask_stride_b = m.size(0) == 1 ? 0 : m.stride(0);
      o.mask_stride_r = m.size(1) == 1 ? 0 : m.stride(1);
    }
    const c10::cuda::CUDAGuard guard(x.device());
    void* st = stream_of(a[14]);
    return status_of([&] { return f_process_logits(x.data_ptr(), y.data_ptr(), code, (int)B, (int)R, (int)V, &o, st); });
  });
}

// use(race_sample, verify, verify_noalloc, verify_tokens, verify_tree, gsd_verify, gsd_verify_tree,
// chunk_attention, cache_append, cache_commit, process_logits, opts): the library's functions, as addresses, and the type of the options structure
PyObject* use(PyObject*, PyObject* args) {
  unsigned long long f[11];
  PyObject* type;
  if (!PyArg_ParseTuple(args, "KKKKKKKKKKKO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &f[9], &f[10], &type)) return nullptr;
  if (!PyType_Check(type)) {
    PyErr_SetString(PyExc_TypeError, "the type of the options structure is wanted");
    return nullptr;
  }
  Py_INCREF(type);
  Py_XDECREF(options_type);
  options_type = type;
  f_race_sample = (decltype(f_race_sample))(uintptr_t)f[0];
  f_verify = (decltype(f_verify))(uintptr_t)f[1];
  f_verify_noalloc = (decltype(f_verify_noalloc))(uintptr_t)f[2];
  f_verify_tokens = (decltype(f_verify_tokens))(uintptr_t)f[3];
  f_verify_tree = (decltype(f_verify_tree))(uintptr_t)f[4];
  f_gsd_verify = (decltype(f_gsd_verify))(uintptr_t)f[5];
  f_gsd_verify_tree = (decltype(f_gsd_verify_tree))(uintptr_t)f[6];
  f_chunk_attention = (decltype(f_chunk_attention))(uintptr_t)f[7];
  f_cache_append = (decltype(f_cache_append))(uintptr_t)f[8];
  f_cache_commit = (decltype(f_cache_commit))(uintptr_t)f[9];
  f_process_logits = (decltype(f_process_logits))(uintptr_t)f[10];
  Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"use", use, METH_VARARGS, nullptr}, FAST(race_sample), FAST(verify), FAST(verify_noalloc), FAST(verify_tokens),
                         FAST(verify_tree), FAST(gsd_verify), FAST(gsd_verify_tree), FAST(chunk_attention), FAST(cache_append),
                         FAST(cache_commit), FAST(process_logits), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ersd_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (torch_version: the torch this was built against, whose tensors alone it can take apart)
PyMODINIT_FUNC PyInit__ersd_call() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", ERSD_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
