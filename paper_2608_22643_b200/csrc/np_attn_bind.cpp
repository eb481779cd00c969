// The calls of the paged cache and its attention for Python: tensors in, pointers and structures out (marshalling and checks only;
// the work is in libnp.so).  The other entry points go through ctypes; here a decode step makes two calls per layer whose
// kernels take a few microseconds, and what the interpreter needs to look at ten tensors is as much.  A call of np_kv_append in
// a stream of them takes 7.0 us with these checks compiled and took 12.4 with the same in Python; its kernel takes 4.0.
//
// Functions take their arguments by position (binding.py has the signatures).  A tensor that is not what a call takes, and an
// error of the library, raise the exception type handed to setup(), made from (code, text).
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <cstring>
#include <sstream>
#include <string>

#include "np.h"

namespace {

PyObject* g_error = nullptr;                                    // the exception type
PyObject *g_room = nullptr, *g_cuda_stream = nullptr;           // names of attributes

struct Refused {
  std::string text;
};
struct Raised {};  // a Python error is set

[[noreturn]] void refuse(const std::string& text) { throw Refused{text}; }

int current_device() {
  try {
    return c10::cuda::current_device();
  } catch (...) {
    return -2;  // no device: no tensor's either
  }
}

std::string describe(const at::Tensor& t) {
  std::ostringstream s;
  s << t.scalar_type() << " " << t.sizes() << " with strides " << t.strides() << " on " << t.device();
  return s.str();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a tensor");
  return THPVariable_Unpack(o);
}

int as_int(int64_t n, const char* name) {
  if (n < INT_MIN || n > INT_MAX) refuse(std::string(name) + ": does not fit in 32 bits");
  return (int)n;
}

int int_of(PyObject* o, const char* name) {
  const long long n = PyLong_AsLongLong(o);
  if (n == -1 && PyErr_Occurred()) throw Raised{};
  return as_int(n, name);
}

void* stream_of(PyObject* o) {
  if (o == Py_None) return nullptr;
  PyObject* held = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttr(o, g_cuda_stream);
  if (!held) throw Raised{};
  void* s = PyLong_AsVoidPtr(held);
  Py_DECREF(held);
  if (PyErr_Occurred()) throw Raised{};
  return s;
}

double scale_of(PyObject* o, int64_t head_dim) {
  if (o == Py_None) return head_dim > 0 ? 1.0 / std::sqrt((double)head_dim) : 1.0;
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Raised{};
  return x;
}

// The bytes of a ctypes structure.
template <class T>
T structure(PyObject* o, const char* name) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Raised{};
  T out;
  const bool fits = b.len == (Py_ssize_t)sizeof out;
  if (fits) std::memcpy(&out, b.buf, sizeof out);
  PyBuffer_Release(&b);
  if (!fits) refuse(std::string(name) + ": another structure");
  return out;
}

// Address of a contiguous tensor of the device that holds at least `least` elements; None is NULL.
template <class T = int32_t>
T* array(PyObject* o, at::ScalarType type, int device, int64_t least, const char* name) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.get_device() != device || t.scalar_type() != type || !t.is_contiguous() || t.numel() < least) {
    std::ostringstream s;
    s << name << ": expected a contiguous " << type << " tensor of at least " << least << " elements on the current CUDA device, got " << describe(t);
    refuse(s.str());
  }
  return static_cast<T*>(t.data_ptr());
}
int32_t* ints(PyObject* o, int device, int64_t least, const char* name) { return array(o, at::kInt, device, least, name); }

// Rows of heads: a tensor [tokens][heads][head_dim] with any strides between tokens and heads.  A stride that nobody steps along
// may be anything in torch.
np_rows rows(PyObject* o, at::ScalarType type, int device, int64_t tokens, int64_t heads, int64_t head_dim, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.get_device() != device || t.scalar_type() != type || t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != head_dim ||
      t.stride(2) != 1) {
    std::ostringstream s;
    s << name << ": expected rows [" << tokens << "][" << heads << "][" << head_dim << "] of " << type
      << ", the last dimension contiguous, on the current CUDA device, got " << describe(t);
    refuse(s.str());
  }
  return np_rows{t.data_ptr(), tokens > 1 ? t.stride(0) : 0, heads > 1 ? t.stride(1) : 0};
}

at::ScalarType type_of(const np_kv_desc& d) {
  const int type = d.dtype & ~NP_KV_E4M3;
  if (type != NP_T_BF16 && type != NP_T_FP16) refuse("desc: dtype must be NP_T_BF16 or NP_T_FP16, or one of them and NP_KV_E4M3");
  return type == NP_T_BF16 ? at::kBFloat16 : at::kHalf;
}

void* cache_of(PyObject* o, const np_kv_desc& d, int device, const char* name) {
  const at::Tensor& t = tensor(o, name);
  const at::ScalarType type = type_of(d);
  if (d.dtype & NP_KV_E4M3) {
    const int64_t page = (int64_t)2 * d.n_kv_heads * d.page_tokens * (d.head_dim + 1);
    if (t.get_device() != device || t.scalar_type() != at::kByte || !t.is_contiguous() || t.dim() != 3 || t.size(0) != d.n_layers || t.size(1) != d.n_pages ||
        t.size(2) != page) {
      std::ostringstream s;
      s << name << ": expected a contiguous cache [" << d.n_layers << "][" << d.n_pages << "][" << page << "] of bytes on the current CUDA device, got " << describe(t);
      refuse(s.str());
    }
    return t.data_ptr();
  }
  if (t.get_device() != device || t.scalar_type() != type || !t.is_contiguous() || t.dim() != 6 || t.size(0) != d.n_layers || t.size(1) != d.n_pages ||
      t.size(2) != 2 || t.size(3) != d.n_kv_heads || t.size(4) != d.page_tokens || t.size(5) != d.head_dim) {
    std::ostringstream s;
    s << name << ": expected a contiguous cache [" << d.n_layers << "][" << d.n_pages << "][2][" << d.n_kv_heads << "][" << d.page_tokens << "]["
      << d.head_dim << "] of " << type << " on the current CUDA device, got " << describe(t);
    refuse(s.str());
  }
  return t.data_ptr();
}

// A table structure whose tensors (if make_kv_tables made it: (device, elements of page_table, lens, refs, scratch or -1)) are of the
// device and serve the description.
np_kv_tables tables_of(PyObject* o, const np_kv_desc& d, int device, const char* name) {
  const np_kv_tables t = structure<np_kv_tables>(o, name);
  PyObject* room = PyObject_GetAttr(o, g_room);
  if (!room) throw Raised{};
  long long has[5] = {0};
  const bool known = PyTuple_Check(room) && PyTuple_GET_SIZE(room) == 5;
  if (known)
    for (int i = 0; i < 5; ++i) has[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(room, i));
  Py_DECREF(room);
  if (PyErr_Occurred()) throw Raised{};
  np_kv_sizes_out sizes;
  if (known && np_kv_sizes(&d, &sizes) == NP_OK &&
      (has[0] != device || has[1] * 4 < (long long)sizes.table_bytes || has[2] < d.max_seqs || has[3] < d.n_pages ||
       (has[4] >= 0 && has[4] * 4 < (long long)sizes.scratch_bytes))) {
    std::ostringstream s;
    s << name << ": tables on device " << has[0] << " of " << has[1] << ", " << has[2] << ", " << has[3] << " and " << has[4]
      << " elements do not serve max_seqs " << d.max_seqs << ", max_pages " << d.max_pages << ", n_pages " << d.n_pages << " on device " << device;
    refuse(s.str());
  }
  return t;
}

void raise(int code, const char* text) {
  PyObject* e = PyObject_CallFunction(g_error ? g_error : PyExc_RuntimeError, "is", code, text);
  if (!e) return;
  PyErr_SetObject((PyObject*)Py_TYPE(e), e);
  Py_DECREF(e);
}

// `call` gives the library's code; what it throws becomes a Python error.
template <class Call>
PyObject* answer(Py_ssize_t given, Py_ssize_t wanted, Call call) {
  if (given != wanted) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    const int rc = call();
    if (rc < 0) {
      raise(rc, np_attn_last_error());
      return nullptr;
    }
    return PyLong_FromLong(rc);
  } catch (const Refused& r) {
    raise(NP_E_INVAL, r.text.c_str());
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// Other threads run while the library queues the kernel (which waits where the queue is full).
template <class Call>
int outside(Call call) {
  PyThreadState* s = PyEval_SaveThread();
  const int rc = call();
  PyEval_RestoreThread(s);
  return rc;
}

typedef PyObject* const* Args;

PyObject* kv_reset(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 3, [&] {
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const np_kv_tables t = tables_of(a[1], d, current_device(), "tables");
    void* s = stream_of(a[2]);
    return outside([&] { return np_kv_reset(&d, &t, s); });
  });
}

PyObject* kv_reserve(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 6, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const np_kv_tables t = tables_of(a[1], d, dev, "tables");
    const int m = as_int(tensor(a[3], "n_new").numel(), "n_new");
    const int32_t *seqs = ints(a[2], dev, m, "seqs"), *add = ints(a[3], dev, m, "n_new");
    int32_t* start = ints(a[4], dev, m, "start_out");
    void* s = stream_of(a[5]);
    return outside([&] { return np_kv_reserve(&d, &t, seqs, add, m, start, s); });
  });
}

PyObject* kv_append(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 10, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    void* cache = cache_of(a[1], d, dev, "cache");
    const int layer = int_of(a[2], "layer");
    const np_kv_tables t = tables_of(a[3], d, dev, "tables");
    const at::Tensor& kt = tensor(a[4], "k");
    const int tokens = kt.dim() > 0 ? as_int(kt.size(0), "k") : 0, m = as_int(tensor(a[8], "start").numel(), "start");
    const np_rows k = rows(a[4], type_of(d), dev, tokens, d.n_kv_heads, d.head_dim, "k"), v = rows(a[5], type_of(d), dev, tokens, d.n_kv_heads, d.head_dim, "v");
    const int32_t *seqs = ints(a[6], dev, m, "seqs"), *cu = ints(a[7], dev, (int64_t)m + 1, "cu"), *start = ints(a[8], dev, m, "start");
    void* s = stream_of(a[9]);
    return outside([&] { return np_kv_append(&d, cache, layer, &t, &k, &v, tokens, seqs, cu, start, m, s); });
  });
}

PyObject* kv_fork(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 6, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    void* cache = cache_of(a[1], d, dev, "cache");
    const np_kv_tables t = tables_of(a[2], d, dev, "tables");
    const int m = as_int(tensor(a[3], "src").numel(), "src");
    const int32_t *src = ints(a[3], dev, m, "src"), *dst = ints(a[4], dev, m, "dst");
    void* s = stream_of(a[5]);
    return outside([&] { return np_kv_fork(&d, cache, &t, src, dst, m, s); });
  });
}

PyObject* kv_free(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 5, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const np_kv_tables t = tables_of(a[1], d, dev, "tables");
    const int m = a[3] != Py_None ? int_of(a[3], "n") : a[2] != Py_None ? as_int(tensor(a[2], "seqs").numel(), "seqs") : d.max_seqs;
    const int32_t* seqs = ints(a[2], dev, m, "seqs");
    void* s = stream_of(a[4]);
    return outside([&] { return np_kv_free(&d, &t, seqs, m, s); });
  });
}

PyObject* kv_compact(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 6, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    void* cache = cache_of(a[1], d, dev, "cache");
    const np_kv_tables in = tables_of(a[2], d, dev, "tables"), out = tables_of(a[3], d, dev, "out_tables");
    int32_t* live = ints(a[4], dev, 1, "n_live");
    void* s = stream_of(a[5]);
    return outside([&] { return np_kv_compact(&d, cache, &in, &out, live, s); });
  });
}

PyObject* kv_copy_pages(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 7, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    void *to = cache_of(a[1], d, dev, "dst_cache"), *from = cache_of(a[2], d, dev, "src_cache");
    const int m = as_int(tensor(a[3], "src").numel(), "src");
    const int32_t *src = ints(a[3], dev, m, "src"), *dst = ints(a[4], dev, m, "dst");
    int32_t* status = ints(a[5], dev, 1, "status");
    void* s = stream_of(a[6]);
    return outside([&] { return np_kv_copy_pages(&d, to, from, src, dst, m, status, s); });
  });
}

PyObject* attn_decode(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 11, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const void* cache = cache_of(a[1], d, dev, "cache");
    const int layer = int_of(a[2], "layer");
    const np_kv_tables t = tables_of(a[3], d, dev, "tables");
    const at::Tensor &qt = tensor(a[4], "q"), &wt = tensor(a[6], "workspace");
    if (qt.dim() != 3) refuse("q: expected rows [sequences][heads][head_dim], got " + describe(qt));
    const int m = as_int(qt.size(0), "q"), heads = as_int(qt.size(1), "q");
    const np_rows q = rows(a[4], type_of(d), dev, m, heads, d.head_dim, "q"), out = rows(a[5], type_of(d), dev, m, heads, d.head_dim, "out");
    void* space = array<void>(a[6], at::kByte, dev, 0, "workspace");
    const uint64_t bytes = wt.numel();
    const int32_t* seqs = ints(a[7], dev, m, "seqs");
    const float scale = (float)scale_of(a[8], d.head_dim);
    float* lse = array<float>(a[9], at::kFloat, dev, (int64_t)m * heads, "lse");
    void* s = stream_of(a[10]);
    return outside([&] { return np_attn_decode(&d, cache, layer, &t, &q, heads, seqs, m, scale, &out, lse, space, bytes, s); });
  });
}

PyObject* attn_prompt(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 9, [&] {
    const int dev = current_device();
    const at::Tensor &qt = tensor(a[0], "q"), &kt = tensor(a[1], "k");
    if (qt.dim() != 3 || kt.dim() != 3) refuse("q and k: expected rows [tokens][heads][head_dim], got " + describe(qt) + " and " + describe(kt));
    const at::ScalarType type = qt.scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf) refuse("q: expected bfloat16 or float16, got " + describe(qt));
    const int tokens = as_int(qt.size(0), "q"), heads = as_int(qt.size(1), "q"), kv = as_int(kt.size(1), "k"), hd = as_int(qt.size(2), "q");
    const np_rows q = rows(a[0], type, dev, tokens, heads, hd, "q"), k = rows(a[1], type, dev, tokens, kv, hd, "k"),
                  v = rows(a[2], type, dev, tokens, kv, hd, "v"), out = rows(a[4], type, dev, tokens, heads, hd, "out");
    const int32_t* cu = ints(a[3], dev, 2, "cu");
    const int m = cu || a[3] != Py_None ? as_int(tensor(a[3], "cu").numel() - 1, "cu") : 0;
    int32_t* status = ints(a[5], dev, 1, "status");
    const float scale = (float)scale_of(a[6], hd);
    float* lse = array<float>(a[7], at::kFloat, dev, (int64_t)tokens * heads, "lse");
    void* s = stream_of(a[8]);
    const np_attn_shape shape = {type == at::kBFloat16 ? NP_T_BF16 : NP_T_FP16, heads, kv, hd, {0, 0, 0, 0}};
    return outside([&] { return np_attn_prompt(&shape, &q, &k, &v, cu, m, tokens, scale, &out, lse, status, s); });
  });
}

// A rotation whose tensors (if make_rotation made it: (device, head_dim of its gains or -1)) serve the call.
np_rotation rotation_of(PyObject* o, int64_t head_dim, int device) {
  const np_rotation r = structure<np_rotation>(o, "rotation");
  PyObject* room = PyObject_GetAttr(o, g_room);
  if (!room) throw Raised{};
  long long has[2] = {0};
  const bool known = PyTuple_Check(room) && PyTuple_GET_SIZE(room) == 2;
  if (known)
    for (int i = 0; i < 2; ++i) has[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(room, i));
  Py_DECREF(room);
  if (PyErr_Occurred()) throw Raised{};
  if (known && (has[0] != device || (has[1] >= 0 && has[1] != head_dim))) {
    std::ostringstream s;
    s << "rotation: tensors on device " << has[0] << " with gains of " << has[1] << " values do not serve heads of " << head_dim << " on device " << device;
    refuse(s.str());
  }
  return r;
}

// The sequences' starts, and the rows that they say where to put.
struct Tokens {
  int n;
  const int32_t *seqs, *cu, *start;
  Tokens(PyObject* seqs_, PyObject* cu_, PyObject* start_, int dev)
      : n(as_int(tensor(start_, "start").numel(), "start")),
        seqs(ints(seqs_, dev, n, "seqs")),
        cu(ints(cu_, dev, (int64_t)n + 1, "cu")),
        start(ints(start_, dev, n, "start")) {}
};

PyObject* attn_rotate(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 8, [&] {
    const int dev = current_device();
    const at::Tensor &qt = tensor(a[1], "q"), &kt = tensor(a[2], "k");
    if (qt.dim() != 3 || kt.dim() != 3) refuse("q and k: expected rows [tokens][heads][head_dim], got " + describe(qt) + " and " + describe(kt));
    const at::ScalarType type = qt.scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf) refuse("q: expected bfloat16 or float16, got " + describe(qt));
    const int tokens = as_int(qt.size(0), "q"), heads = as_int(qt.size(1), "q"), kv = as_int(kt.size(1), "k"), hd = as_int(qt.size(2), "q");
    const np_rotation r = rotation_of(a[0], hd, dev);
    const np_rows q = rows(a[1], type, dev, tokens, heads, hd, "q"), k = rows(a[2], type, dev, tokens, kv, hd, "k"),
                  qo = rows(a[3], type, dev, tokens, heads, hd, "q_out"), ko = rows(a[4], type, dev, tokens, kv, hd, "k_out");
    const Tokens w(Py_None, a[5], a[6], dev);
    void* s = stream_of(a[7]);
    const np_attn_shape shape = {type == at::kBFloat16 ? NP_T_BF16 : NP_T_FP16, heads, kv, hd, {0, 0, 0, 0}};
    return outside([&] { return np_attn_rotate(&shape, &r, &q, &k, &qo, &ko, tokens, w.cu, w.start, w.n, s); });
  });
}

PyObject* kv_append_rotated(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 13, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    void* cache = cache_of(a[1], d, dev, "cache");
    const int layer = int_of(a[2], "layer");
    const np_kv_tables t = tables_of(a[3], d, dev, "tables");
    const np_rotation r = rotation_of(a[4], d.head_dim, dev);
    const at::Tensor& qt = tensor(a[5], "q");
    if (qt.dim() != 3) refuse("q: expected rows [tokens][heads][head_dim], got " + describe(qt));
    const int tokens = as_int(qt.size(0), "q"), heads = as_int(qt.size(1), "q");
    const at::ScalarType type = type_of(d);
    const np_rows q = rows(a[5], type, dev, tokens, heads, d.head_dim, "q"), k = rows(a[6], type, dev, tokens, d.n_kv_heads, d.head_dim, "k"),
                  v = rows(a[7], type, dev, tokens, d.n_kv_heads, d.head_dim, "v"), qo = rows(a[8], type, dev, tokens, heads, d.head_dim, "q_out");
    const Tokens w(a[9], a[10], a[11], dev);
    void* s = stream_of(a[12]);
    return outside([&] { return np_kv_append_rotated(&d, cache, layer, &t, &r, &q, heads, &k, &v, &qo, tokens, w.seqs, w.cu, w.start, w.n, s); });
  });
}

PyObject* kv_read(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 10, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const void* cache = cache_of(a[1], d, dev, "cache");
    const int layer = int_of(a[2], "layer");
    const np_kv_tables t = tables_of(a[3], d, dev, "tables");
    const at::Tensor& kt = tensor(a[4], "k");
    const int tokens = kt.dim() > 0 ? as_int(kt.size(0), "k") : 0;
    const np_rows k = rows(a[4], type_of(d), dev, tokens, d.n_kv_heads, d.head_dim, "k"), v = rows(a[5], type_of(d), dev, tokens, d.n_kv_heads, d.head_dim, "v");
    const Tokens w(a[6], a[7], a[8], dev);
    void* s = stream_of(a[9]);
    return outside([&] { return np_kv_read(&d, cache, layer, &t, &k, &v, tokens, w.seqs, w.cu, w.start, w.n, s); });
  });
}

PyObject* kv_shared(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 7, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const np_kv_tables t = tables_of(a[1], d, dev, "tables");
    const int groups = as_int(tensor(a[4], "shared").numel(), "shared");
    const int m = a[5] != Py_None ? int_of(a[5], "n") : a[2] != Py_None ? as_int(tensor(a[2], "seqs").numel(), "seqs") : d.max_seqs;
    const int32_t *seqs = ints(a[2], dev, m, "seqs"), *cu = ints(a[3], dev, (int64_t)groups + 1, "cu");
    int32_t* shared = ints(a[4], dev, groups, "shared");
    void* s = stream_of(a[6]);
    return outside([&] { return np_kv_shared(&d, &t, seqs, m, cu, groups, shared, s); });
  });
}

PyObject* attn_decode_shared(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 13, [&] {
    const int dev = current_device();
    const np_kv_desc d = structure<np_kv_desc>(a[0], "desc");
    const void* cache = cache_of(a[1], d, dev, "cache");
    const int layer = int_of(a[2], "layer");
    const np_kv_tables t = tables_of(a[3], d, dev, "tables");
    const at::Tensor &qt = tensor(a[4], "q"), &wt = tensor(a[6], "workspace");
    if (qt.dim() != 3) refuse("q: expected rows [sequences][heads][head_dim], got " + describe(qt));
    const int m = as_int(qt.size(0), "q"), heads = as_int(qt.size(1), "q");
    const np_rows q = rows(a[4], type_of(d), dev, m, heads, d.head_dim, "q"), out = rows(a[5], type_of(d), dev, m, heads, d.head_dim, "out");
    void* space = array<void>(a[6], at::kByte, dev, 0, "workspace");
    const uint64_t bytes = wt.numel();
    const int groups = as_int(tensor(a[8], "shared").numel(), "shared");
    const int32_t *cu = ints(a[7], dev, (int64_t)groups + 1, "cu"), *shared = ints(a[8], dev, groups, "shared"), *seqs = ints(a[9], dev, m, "seqs");
    const float scale = (float)scale_of(a[10], d.head_dim);
    float* lse = array<float>(a[11], at::kFloat, dev, (int64_t)m * heads, "lse");
    void* s = stream_of(a[12]);
    return outside([&] { return np_attn_decode_shared(&d, cache, layer, &t, &q, heads, seqs, m, cu, shared, groups, scale, &out, lse, space, bytes, s); });
  });
}

PyObject* attn_check(PyObject*, Args a, Py_ssize_t n) {
  return answer(n, 2, [&] {
    const int32_t* status = ints(a[0], current_device(), 1, "status");
    void* s = stream_of(a[1]);
    return outside([&] { return np_attn_check(status, s); });
  });
}

PyObject* setup(PyObject*, PyObject* type) {
  Py_XSETREF(g_error, Py_NewRef(type));
  Py_RETURN_NONE;
}

#define NP_CALL(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {NP_CALL(kv_reset),   NP_CALL(kv_reserve),    NP_CALL(kv_append),   NP_CALL(kv_fork),     NP_CALL(kv_free),
                           NP_CALL(kv_compact), NP_CALL(kv_copy_pages), NP_CALL(attn_decode), NP_CALL(attn_prompt), NP_CALL(attn_check),
                           NP_CALL(attn_rotate), NP_CALL(kv_append_rotated), NP_CALL(kv_read), NP_CALL(kv_shared), NP_CALL(attn_decode_shared),
                           {"setup", setup, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "np_attn_bind", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_np_attn_bind(void) {
  g_room = PyUnicode_InternFromString("room");
  g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  PyObject* m = g_room && g_cuda_stream ? PyModule_Create(&g_module) : nullptr;
  if (m && PyModule_AddStringConstant(m, "built_for", NP_BUILT_FOR) != 0) Py_CLEAR(m);  // binding.py compares
  return m;
}
