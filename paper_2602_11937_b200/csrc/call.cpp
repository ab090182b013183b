// The Python binding's way into the entry points that a decode step or a prompt chunk calls: tensors to pointers, sizes and
// strides, checked, and the current stream.  A small call costs the GPU 2 to 6 us; the same marshalling through ctypes took
// 4 to 5 us of host time beside the launch's own 3, this takes about half a microsecond.  The entry points themselves stay
// plain C and know nothing of torch: this module is given their addresses.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>
#include <string>

#include "puzzle_attn.h"

namespace {

struct Entries {
  decltype(&puzzle_kv_append) kv_append;
  decltype(&puzzle_kv_append_tokens) kv_append_tokens;
  decltype(&puzzle_kv_append_rope) kv_append_rope;
  decltype(&puzzle_kv_read_tokens) kv_read_tokens;
  decltype(&puzzle_decode_attn) decode_attn;
  decltype(&puzzle_decode_attn_tcgen05) decode_attn_tcgen05;
  decltype(&puzzle_decode_attn_tokens) decode_attn_tokens;
  decltype(&puzzle_kv_append_packed) kv_append_packed;
  decltype(&puzzle_prompt_attn) prompt_attn;
  decltype(&puzzle_chunk_attn) chunk_attn;
} entry;
constexpr Py_ssize_t kEntries = sizeof(Entries) / sizeof(void*);

struct PythonError {};   // an exception is set

[[noreturn]] void refuse(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw PythonError();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_CheckExact(o) && !THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor, got %s", name, Py_TYPE(o)->tp_name);
    throw PythonError();
  }
  return THPVariable_Unpack(o);
}

const char* type_name(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return "torch.bfloat16";
    case at::kFloat: return "torch.float32";
    case at::kInt: return "torch.int32";
    default: return c10::toString(t);
  }
}

std::string shape_text(at::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + (s.size() == 1 ? ",)" : ")");
}

// Kernels are launched on the current device, so everything they are given has to lie there.
void check_place(const char* name, int64_t device, int64_t current) {
  if (device != current)
    refuse(std::string(name) + " is on cuda:" + std::to_string(device) + ", the current device is cuda:" + std::to_string(current));
}
// The current device, asked for once in a call (a call whose arguments are no CUDA tensors never asks).
struct Here {
  int device = -1;
  int get() {
    if (device < 0) device = c10::cuda::current_device();
    return device;
  }
  void check(const char* name, const at::Tensor& t) { check_place(name, t.get_device(), get()); }
};

void check_contiguous(const char* name, const at::Tensor& t) {
  if (!t.is_contiguous()) refuse(std::string(name) + " must be contiguous");
}

// Device pointer of a contiguous CUDA tensor (None: NULL) of at least `need` elements: what the call reads or writes.
void* pointer(Here& here, PyObject* o, const char* name, at::ScalarType type, int64_t need) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) refuse(std::string(name) + " must be a CUDA tensor");
  here.check(name, t);
  check_contiguous(name, t);
  if (type != at::kByte && t.scalar_type() != type)   // kByte: any type
    refuse(std::string(name) + " must be " + type_name(type) + ", got " + type_name(t.scalar_type()));
  if (t.numel() < need)
    refuse(std::string(name) + " has " + std::to_string(t.numel()) + " elements, the call needs " + std::to_string(need));
  return t.data_ptr();
}
template <typename T>
T* pointer_to(Here& here, PyObject* o, const char* name, at::ScalarType type, int64_t need) {
  return static_cast<T*>(pointer(here, o, name, type, need));
}
// Elements of a token, for descriptors that the library takes; others need nothing here, because it refuses them itself with
// a code that says why.
bool taken(const puzzle_layer_desc& d) {
  return d.num_kv_heads > 0 && d.head_dim == 64 && d.num_q_heads == 8 * (int64_t)d.num_kv_heads;
}
int64_t q_heads(const puzzle_layer_desc& d) { return taken(d) ? d.num_q_heads : 0; }
int64_t q_row(const puzzle_layer_desc& d) { return q_heads(d) * d.head_dim; }
int64_t kv_row(const puzzle_layer_desc& d) { return taken(d) ? (int64_t)d.num_kv_heads * d.head_dim : 0; }

// A ctypes structure's bytes.
template <typename T>
T structure(PyObject* o) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PythonError();
  T v;
  const bool fits = b.len == (Py_ssize_t)sizeof(T);
  if (fits) std::memcpy(&v, b.buf, sizeof(T));
  PyBuffer_Release(&b);
  if (!fits) refuse("a descriptor has the wrong size");
  return v;
}

// The numbers that the binding notes on a descriptor it made from tensors (attribute _held: a tuple, or None on a descriptor
// that was filled in by hand): what the tensors hold, which the pointers in the structure do not say.
template <size_t N>
bool held(PyObject* o, int64_t (&v)[N]) {
  static PyObject* const name = PyUnicode_InternFromString("_held");
  PyObject* t = PyObject_GetAttr(o, name);
  if (!t) {
    PyErr_Clear();
    return false;
  }
  bool known = PyTuple_Check(t) && PyTuple_GET_SIZE(t) == (Py_ssize_t)N;
  for (size_t i = 0; known && i < N; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
  Py_DECREF(t);
  if (PyErr_Occurred()) throw PythonError();
  return known;
}

int64_t block_bytes(const puzzle_layer_desc& d) {   // of one (block, KV head), K or V
  return d.kv_dtype == PUZZLE_KV_FP4_E2M1 ? PUZZLE_FP4_BLOCK_BYTES : d.kv_dtype == PUZZLE_KV_BF16 ? 16 * 64 * 2 : 16 * 64;
}
// Whether what a view points to has room for this descriptor and this many sequences.  type_taken: the entry point has this
// cache type (others it refuses itself, with a code that says why).
void check_view(Here& here, PyObject* view, const puzzle_layer_desc& d, const puzzle_kv_view& v, int batch,
                bool type_taken = true) {
  int64_t h[4];   // device, sequences, scales, bytes of the smaller cache
  if (!held(view, h)) return;
  if (h[1] < batch)
    refuse("the cache view has " + std::to_string(h[1]) + " sequences, the call needs " + std::to_string(batch));
  if (taken(d) && h[2] < d.num_kv_heads && d.kv_dtype != PUZZLE_KV_BF16)
    refuse("the cache view has " + std::to_string(h[2]) + " scales, the call needs " + std::to_string(d.num_kv_heads));
  const int64_t need = taken(d) && type_taken ? v.num_blocks * d.num_kv_heads * block_bytes(d) : 0;
  if (h[3] < need)
    refuse("the cache has " + std::to_string(h[3]) + " bytes, the descriptor's " + std::to_string(v.num_blocks) + " blocks need " +
           std::to_string(need));
  check_place("the cache view", h[0], here.get());
}
void check_rope(Here& here, PyObject* rope, int batch) {
  int64_t h[2];   // device, sequences that have an offset
  if (!held(rope, h)) return;
  if (h[1] < batch)
    refuse("the rotation has offsets for " + std::to_string(h[1]) + " sequences, the call needs " + std::to_string(batch));
  check_place("the rotation", h[0], here.get());
}

// The stream's handle (None: the current one).
void* stream_of(Here& here, PyObject* stream) {
  if (stream == Py_None) return c10::cuda::getCurrentCUDAStream(here.get()).stream();
  PyObject* h = PyObject_GetAttrString(stream, "cuda_stream");
  if (!h) throw PythonError();
  void* s = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (PyErr_Occurred()) throw PythonError();
  return s;
}

int integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  if (v < INT_MIN || v > INT_MAX) refuse("an integer argument does not fit 32 bits");
  return (int)v;
}

// Batches and token counts are 32-bit in the C interface.
int extent(const at::Tensor& t, int dim) {
  const int64_t n = t.size(dim);
  if (n > INT_MAX) refuse("a dimension does not fit 32 bits");
  return (int)n;
}

template <typename F>
PyObject* call(const char* name, Py_ssize_t given, Py_ssize_t wanted, F&& body) {
  HANDLE_TH_ERRORS
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, wanted, given);
    return nullptr;
  }
  if (!entry.kv_append) {
    PyErr_SetString(PyExc_RuntimeError, "the entry points have not been bound");
    return nullptr;
  }
  try {
    Here here;
    return PyLong_FromLong(body(here));
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// The C call itself, without Python's lock.
template <typename F>
int unlocked(F&& f) {
  PyThreadState* ts = PyEval_SaveThread();
  const int code = f();
  PyEval_RestoreThread(ts);
  return code;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != kEntries) {
    PyErr_Format(PyExc_TypeError, "bind takes %zd addresses", kEntries);
    return nullptr;
  }
  void* p[kEntries];
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  std::memcpy(&entry, p, sizeof entry);
  Py_RETURN_NONE;
}

// desc, view, k_new, v_new, dev_status, stream
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("kv_append", n, 6, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor& t = tensor(a[2], "k_new");
    const int batch = extent(t, 0);
    check_contiguous("k_new", t);   // or its first dimension need not be the batch
    check_view(here, a[1], desc, view, batch);
    void* k = pointer(here, a[2], "k_new", at::kBFloat16, batch * kv_row(desc));
    void* v = pointer(here, a[3], "v_new", at::kBFloat16, batch * kv_row(desc));
    int32_t* status = pointer_to<int32_t>(here, a[4], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[5]);
    return unlocked([&] { return entry.kv_append(&desc, &view, k, v, batch, status, s); });
  });
}

// desc, view, k_new, v_new, new_lens, dev_status, stream
PyObject* kv_append_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("kv_append_tokens", n, 7, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor& t = tensor(a[2], "k_new");
    const int batch = extent(t, 0), n_new = extent(t, 1);
    check_contiguous("k_new", t);
    check_view(here, a[1], desc, view, batch);
    void* k = pointer(here, a[2], "k_new", at::kBFloat16, (int64_t)batch * n_new * kv_row(desc));
    void* v = pointer(here, a[3], "v_new", at::kBFloat16, (int64_t)batch * n_new * kv_row(desc));
    int32_t* lens = pointer_to<int32_t>(here, a[4], "new_lens", at::kInt, batch);
    int32_t* status = pointer_to<int32_t>(here, a[5], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[6]);
    return unlocked([&] { return entry.kv_append_tokens(&desc, &view, k, v, lens, batch, n_new, status, s); });
  });
}

// Rows [batch][n_new][heads][D] or [batch][heads][D] of new tokens: every dimension as expected.
void check_rows(const at::Tensor& t, const char* name, const at::Tensor& like, int heads, int row) {
  const auto s = t.sizes(), l = like.sizes();
  const size_t d = l.size();
  if (s.size() == d && s[0] == l[0] && (d == 3 || s[1] == l[1]) && s[d - 2] == heads && s[d - 1] == row) return;
  auto want = l.vec();
  want[d - 2] = heads;
  want[d - 1] = row;
  refuse(std::string(name) + " must be " + shape_text(want) + ", got " + shape_text(s));
}
struct Rows {
  void* p;
  int64_t seq_stride, token_stride;
};
Rows rows(Here& here, const at::Tensor& t, const char* name, int row) {
  if (!t.is_cuda() || t.scalar_type() != at::kBFloat16) refuse(std::string(name) + " must be a bf16 CUDA tensor");
  here.check(name, t);
  const auto st = t.strides();
  const size_t d = st.size();
  if (st[d - 1] != 1 || (st[d - 2] != row && t.size(d - 2) > 1))
    refuse("the heads of a token of " + std::string(name) + " must be contiguous");
  return {t.data_ptr(), st[0], d == 4 ? st[1] : 0};
}

// desc, view, rope, q, k_new, v_new, q_out, new_lens, dev_status, stream
PyObject* kv_append_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("kv_append_rope", n, 10, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const auto rope = structure<puzzle_rope>(a[2]);
    const bool with_q = a[3] != Py_None;
    if (with_q != (a[6] != Py_None)) refuse("q and q_out go together");
    const at::Tensor &k = tensor(a[4], "k_new"), &v = tensor(a[5], "v_new");
    if (k.dim() != 3 && k.dim() != 4) refuse("k_new must be [batch][n_new][heads][D] or [batch][heads][D]");
    const int batch = extent(k, 0), n_new = k.dim() == 4 ? extent(k, 1) : 1;
    check_view(here, a[1], desc, view, batch);
    check_rope(here, a[2], batch);
    check_rows(k, "k_new", k, desc.num_kv_heads, desc.head_dim);
    check_rows(v, "v_new", k, desc.num_kv_heads, desc.head_dim);
    if (with_q) {
      check_rows(tensor(a[3], "q"), "q", k, desc.num_q_heads, desc.head_dim);
      check_rows(tensor(a[6], "q_out"), "q_out", k, desc.num_q_heads, desc.head_dim);
    }
    const Rows kr = rows(here, k, "k_new", desc.head_dim), vr = rows(here, v, "v_new", desc.head_dim);
    const Rows qr = with_q ? rows(here, tensor(a[3], "q"), "q", desc.head_dim) : Rows{nullptr, 0, 0};
    const puzzle_qkv qkv = {qr.p,          kr.p,            vr.p,          qr.seq_stride,  qr.token_stride,
                            kr.seq_stride, kr.token_stride, vr.seq_stride, vr.token_stride};
    void* q_out = pointer(here, a[6], "q_out", at::kBFloat16, 0);   // its shape has been checked
    int32_t* lens = pointer_to<int32_t>(here, a[7], "new_lens", at::kInt, batch);
    int32_t* status = pointer_to<int32_t>(here, a[8], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[9]);
    return unlocked([&] {
      return entry.kv_append_rope(&desc, &view, &rope, &qkv, q_out, lens, batch, n_new, status, s);
    });
  });
}

// desc, view, k_out, v_out, read_lens, dev_status, stream
PyObject* kv_read_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("kv_read_tokens", n, 7, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor &k = tensor(a[2], "k_out"), &v = tensor(a[3], "v_out");
    if (k.dim() != 4 || k.size(2) != desc.num_kv_heads || k.size(3) != desc.head_dim || v.sizes() != k.sizes())
      refuse("k_out and v_out must be [batch][n_read][" + std::to_string(desc.num_kv_heads) + "][" +
             std::to_string(desc.head_dim) + "], got " + shape_text(k.sizes()) + " and " + shape_text(v.sizes()));
    const int batch = extent(k, 0), n_read = extent(k, 1);
    check_view(here, a[1], desc, view, batch);
    void* kp = pointer(here, a[2], "k_out", at::kBFloat16, 0);   // their shapes have been checked
    void* vp = pointer(here, a[3], "v_out", at::kBFloat16, 0);
    int32_t* lens = pointer_to<int32_t>(here, a[4], "read_lens", at::kInt, batch);
    int32_t* status = pointer_to<int32_t>(here, a[5], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[6]);
    return unlocked([&] { return entry.kv_read_tokens(&desc, &view, kp, vp, lens, batch, n_read, status, s); });
  });
}

// desc, view, q, sinks, out, lse_out, num_splits, workspace, dev_status, stream
PyObject* decode(const char* name, decltype(&puzzle_decode_attn) f, bool fp8_only, PyObject* const* a, Py_ssize_t n) {
  return call(name, n, 10, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor &t = tensor(a[2], "q"), &w = tensor(a[7], "workspace");
    const int batch = extent(t, 0);
    check_contiguous("q", t);   // or its first dimension need not be the batch
    check_view(here, a[1], desc, view, batch, !fp8_only || desc.kv_dtype == PUZZLE_KV_FP8_E4M3);
    void* q = pointer(here, a[2], "q", at::kBFloat16, batch * q_row(desc));
    const float* sinks = pointer_to<float>(here, a[3], "sinks", at::kFloat, q_heads(desc));
    void* out = pointer(here, a[4], "out", at::kBFloat16, batch * q_row(desc));
    float* lse = pointer_to<float>(here, a[5], "lse_out", at::kFloat, batch * q_heads(desc));
    const int splits = integer(a[6]);
    void* workspace = pointer(here, a[7], "workspace", at::kByte, 0);   // the library checks its size
    const size_t bytes = w.nbytes();
    int32_t* status = pointer_to<int32_t>(here, a[8], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[9]);
    return unlocked([&] { return f(&desc, &view, q, sinks, out, lse, batch, splits, workspace, bytes, status, s); });
  });
}
PyObject* decode_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return decode("decode_attn", entry.decode_attn, false, a, n);
}
PyObject* decode_attn_tcgen05(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return decode("decode_attn_tcgen05", entry.decode_attn_tcgen05, true, a, n);
}

// desc, view, q, q_lens, sinks, out, lse_out, workspace, dev_status, stream
PyObject* decode_attn_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("decode_attn_tokens", n, 10, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor &t = tensor(a[2], "q"), &w = tensor(a[7], "workspace");
    const int batch = extent(t, 0), n_q = extent(t, 1);
    const int64_t tokens = (int64_t)batch * n_q;
    check_contiguous("q", t);
    check_view(here, a[1], desc, view, batch, desc.kv_dtype != PUZZLE_KV_BF16);
    void* q = pointer(here, a[2], "q", at::kBFloat16, tokens * q_row(desc));
    const int32_t* lens = pointer_to<int32_t>(here, a[3], "q_lens", at::kInt, batch);
    const float* sinks = pointer_to<float>(here, a[4], "sinks", at::kFloat, q_heads(desc));
    void* out = pointer(here, a[5], "out", at::kBFloat16, tokens * q_row(desc));
    float* lse = pointer_to<float>(here, a[6], "lse_out", at::kFloat, tokens * q_heads(desc));
    void* workspace = pointer(here, a[7], "workspace", at::kByte, 0);   // the library checks its size
    const size_t bytes = w.nbytes();
    int32_t* status = pointer_to<int32_t>(here, a[8], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[9]);
    return unlocked([&] {
      return entry.decode_attn_tokens(&desc, &view, q, lens, sinks, out, lse, batch, n_q, workspace, bytes, status, s);
    });
  });
}

// Packed rows [tokens][heads][D]: every dimension as expected (all inputs of a call before any pointer is taken).
void check_packed(PyObject* o, const char* name, int64_t tokens, int heads, int row) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != row)
    refuse(std::string(name) + " must be " + shape_text({tokens, heads, row}) + ", got " + shape_text(t.sizes()));
}
// Pointer and token stride of an input's packed rows.
Rows packed_rows(Here& here, PyObject* o, const char* name, int row) {
  Rows r = rows(here, tensor(o, name), name, row);
  r.token_stride = r.seq_stride;
  r.seq_stride = 0;
  return r;
}
// A contiguous packed array [tokens][heads][D].
void* packed_out(Here& here, PyObject* o, const char* name, int64_t tokens, int heads, int row) {
  if (o == Py_None) return nullptr;
  check_packed(o, name, tokens, heads, row);
  return pointer(here, o, name, at::kBFloat16, 0);
}
int packed_batch(const at::Tensor& starts) {
  if (starts.dim() != 1 || starts.size(0) < 2) refuse("starts must have one element more than there are sequences");
  if (starts.size(0) - 1 > INT_MAX) refuse("a dimension does not fit 32 bits");
  return (int)(starts.size(0) - 1);
}

// desc, view, rope, q, k_new, v_new, starts, q_out, k_out, keep_last, dev_status, stream
PyObject* kv_append_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("kv_append_packed", n, 12, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    puzzle_rope rope = {};
    const bool rotate = a[2] != Py_None, with_q = a[3] != Py_None;
    if (rotate) rope = structure<puzzle_rope>(a[2]);
    if (with_q != (a[7] != Py_None)) refuse("q and q_out go together");
    const at::Tensor& k = tensor(a[4], "k_new");
    if (k.dim() != 3) refuse("k_new must be [tokens][heads][D]");
    const int tokens = extent(k, 0), batch = packed_batch(tensor(a[6], "starts"));
    check_view(here, a[1], desc, view, batch);
    if (rotate) check_rope(here, a[2], batch);
    check_packed(a[4], "k_new", tokens, desc.num_kv_heads, desc.head_dim);
    check_packed(a[5], "v_new", tokens, desc.num_kv_heads, desc.head_dim);
    if (with_q) check_packed(a[3], "q", tokens, desc.num_q_heads, desc.head_dim);
    const Rows kr = packed_rows(here, a[4], "k_new", desc.head_dim), vr = packed_rows(here, a[5], "v_new", desc.head_dim);
    const Rows qr = with_q ? packed_rows(here, a[3], "q", desc.head_dim) : Rows{nullptr, 0, 0};
    const puzzle_qkv qkv = {qr.p, kr.p, vr.p, 0, qr.token_stride, 0, kr.token_stride, 0, vr.token_stride};
    const int32_t* starts = pointer_to<int32_t>(here, a[6], "starts", at::kInt, 2);
    void* q_out = packed_out(here, a[7], "q_out", tokens, desc.num_q_heads, desc.head_dim);
    void* k_out = packed_out(here, a[8], "k_out", tokens, desc.num_kv_heads, desc.head_dim);
    const int keep = integer(a[9]);
    int32_t* status = pointer_to<int32_t>(here, a[10], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[11]);
    return unlocked([&] {
      return entry.kv_append_packed(&desc, &view, rotate ? &rope : nullptr, &qkv, q_out, k_out, starts, batch, tokens, keep, status,
                                    s);
    });
  });
}

// desc, q, k, v, starts, sinks, out, lse_out, dev_status, stream
PyObject* prompt_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("prompt_attn", n, 10, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const at::Tensor& t = tensor(a[1], "q");
    if (t.dim() != 3) refuse("q must be [tokens][heads][D]");
    const int tokens = extent(t, 0), batch = packed_batch(tensor(a[4], "starts"));
    check_packed(a[1], "q", tokens, desc.num_q_heads, desc.head_dim);
    check_packed(a[2], "k", tokens, desc.num_kv_heads, desc.head_dim);
    check_packed(a[3], "v", tokens, desc.num_kv_heads, desc.head_dim);
    const Rows qr = packed_rows(here, a[1], "q", desc.head_dim), kr = packed_rows(here, a[2], "k", desc.head_dim);
    const Rows vr = packed_rows(here, a[3], "v", desc.head_dim);
    const puzzle_qkv qkv = {qr.p, kr.p, vr.p, 0, qr.token_stride, 0, kr.token_stride, 0, vr.token_stride};
    const int32_t* starts = pointer_to<int32_t>(here, a[4], "starts", at::kInt, 2);
    const float* sinks = pointer_to<float>(here, a[5], "sinks", at::kFloat, q_heads(desc));
    if (a[6] == Py_None) refuse("out is required");
    void* out = packed_out(here, a[6], "out", tokens, desc.num_q_heads, desc.head_dim);
    float* lse = pointer_to<float>(here, a[7], "lse_out", at::kFloat, tokens * q_heads(desc));
    int32_t* status = pointer_to<int32_t>(here, a[8], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[9]);
    return unlocked([&] { return entry.prompt_attn(&desc, &qkv, starts, sinks, out, lse, batch, tokens, status, s); });
  });
}

// desc, view, q, starts, sinks, out, lse_out, workspace, dev_status, stream
PyObject* chunk_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("chunk_attn", n, 10, [&](Here& here) {
    const auto desc = structure<puzzle_layer_desc>(a[0]);
    const auto view = structure<puzzle_kv_view>(a[1]);
    const at::Tensor &t = tensor(a[2], "q"), &w = tensor(a[7], "workspace");
    if (t.dim() != 3) refuse("q must be [tokens][heads][D]");
    const int tokens = extent(t, 0), batch = packed_batch(tensor(a[3], "starts"));
    check_view(here, a[1], desc, view, batch);
    check_packed(a[2], "q", tokens, desc.num_q_heads, desc.head_dim);
    const Rows qr = packed_rows(here, a[2], "q", desc.head_dim);
    const int32_t* starts = pointer_to<int32_t>(here, a[3], "starts", at::kInt, 2);
    const float* sinks = pointer_to<float>(here, a[4], "sinks", at::kFloat, q_heads(desc));
    if (a[5] == Py_None) refuse("out is required");
    void* out = packed_out(here, a[5], "out", tokens, desc.num_q_heads, desc.head_dim);
    float* lse = pointer_to<float>(here, a[6], "lse_out", at::kFloat, tokens * q_heads(desc));
    void* workspace = pointer(here, a[7], "workspace", at::kByte, 0);   // the library checks its size
    const size_t bytes = w.nbytes();
    int32_t* status = pointer_to<int32_t>(here, a[8], "dev_status", at::kInt, 1);
    void* s = stream_of(here, a[9]);
    return unlocked([&] {
      return entry.chunk_attn(&desc, &view, qr.p, qr.token_stride, starts, sinks, out, lse, batch, tokens, workspace, bytes,
                              status, s);
    });
  });
}

// name, device of a tensor, current device: the check every tensor of every call goes through, for tests without two GPUs.
PyObject* check_device(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call("check_device", n, 3, [&](Here&) {
    const char* name = PyUnicode_AsUTF8(a[0]);
    if (!name) throw PythonError();
    check_place(name, integer(a[1]), integer(a[2]));
    return 0;
  });
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(static_cast<Fast>(name))), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),           METHOD(kv_append),   METHOD(kv_append_tokens),    METHOD(kv_append_rope),
                         METHOD(kv_read_tokens), METHOD(decode_attn), METHOD(decode_attn_tcgen05), METHOD(decode_attn_tokens),
                         METHOD(kv_append_packed), METHOD(prompt_attn), METHOD(chunk_attn), METHOD(check_device),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_puzzle_call", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__puzzle_call() {
  PyObject* m = PyModule_Create(&module);
  // the binding compares it with what it runs in: the interfaces used here change between versions
  if (m && PyModule_AddStringConstant(m, "built_for", PUZZLE_BUILT_FOR) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
