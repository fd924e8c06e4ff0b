// Argument marshalling of a serving step's calls: checks tensors and passes their addresses,
// sizes and strides to the library's C entry points (include/ebd.h), whose addresses
// bind() is given.  The same checks in Python with ctypes cost 10 to 16 us of host time
// a call, more than most of these kernels run: an append step of 32 sequences took 18.5
// us a call, its kernel 4.2; this way calls follow one another every 3.9 us.
//
// Every function returns the entry point's status; what it refuses itself is raised as the
// TypeError or ValueError that the Python helpers raise.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <string>

#include "../../include/ebd.h"

namespace {

using at::ScalarType;

struct Refusal {
  PyObject* type;
  std::string text;
};
[[noreturn]] void bad_type(const std::string& s) { throw Refusal{PyExc_TypeError, s}; }
[[noreturn]] void bad_value(const std::string& s) { throw Refusal{PyExc_ValueError, s}; }

std::string dtype_name(ScalarType t) {
  switch (t) {
    case at::kFloat: return "torch.float32";
    case at::kBFloat16: return "torch.bfloat16";
    case at::kHalf: return "torch.float16";
    case at::kDouble: return "torch.float64";
    case at::kInt: return "torch.int32";
    case at::kLong: return "torch.int64";
    case at::kByte: return "torch.uint8";
    case at::kBool: return "torch.bool";
    default: return std::string("torch.") + c10::toString(t);
  }
}

template <typename Sizes>
std::string shape_name(const Sizes& s) {
  std::string out = "(";
  size_t n = 0;
  for (int64_t v : s) out += (n++ ? ", " : "") + std::to_string(v);
  return out + (n == 1 ? ",)" : ")");
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) bad_type(std::string(name) + " must be a torch.Tensor");
  return THPVariable_Unpack(o);
}

void check_dtype(const at::Tensor& t, ScalarType dtype, const char* name) {
  if (t.scalar_type() != dtype)
    bad_type(std::string(name) + " has dtype " + dtype_name(t.scalar_type()) + ", expected " +
             dtype_name(dtype));
}

ebd_dtype dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return EBD_F32;
  if (t.scalar_type() == at::kBFloat16) return EBD_BF16;
  bad_type("unsupported dtype " + dtype_name(t.scalar_type()) + "; expected float32 or bfloat16");
}

// Address of a contiguous CUDA tensor of this type and shape; None: null.
template <typename T>
T* address(PyObject* o, ScalarType dtype, std::initializer_list<int64_t> shape, const char* name) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) bad_value(std::string(name) + " must be a CUDA tensor");
  if (!t.is_contiguous()) bad_value(std::string(name) + " must be contiguous");
  check_dtype(t, dtype, name);
  if (t.sizes() != at::IntArrayRef(shape))
    bad_value(std::string(name) + " has shape " + shape_name(t.sizes()) + ", expected " +
              shape_name(shape));
  return static_cast<T*>(t.data_ptr());
}
int32_t* ints(PyObject* o, std::initializer_list<int64_t> shape, const char* name) {
  return address<int32_t>(o, at::kInt, shape, name);
}

// A [T, H, d] tensor with any token and head strides.
struct Rows {
  void* p = nullptr;
  int64_t ts = 0, hs = 0;
};
Rows rows(PyObject* o, ScalarType dtype, int64_t n_tokens, int64_t n_heads, int64_t head_dim,
          const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) bad_value(std::string(name) + " must be a CUDA tensor");
  check_dtype(t, dtype, name);
  if (t.dim() != 3 || t.size(0) != n_tokens || t.size(1) != n_heads || t.size(2) != head_dim)
    bad_value(std::string(name) + " has shape " + shape_name(t.sizes()) + ", expected " +
              shape_name(std::initializer_list<int64_t>{n_tokens, n_heads, head_dim}));
  if (t.stride(2) != 1 && head_dim > 1)
    bad_value("the last dimension of " + std::string(name) + " must be contiguous");
  return Rows{t.data_ptr(), t.stride(0), t.stride(1)};
}
const at::Tensor& three(PyObject* o, const char* name, const char* shape) {
  if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != 3)
    bad_value(std::string(name) + " must be " + shape);
  return THPVariable_Unpack(o);
}

int32_t int32_of(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) bad_value(std::string(name) + " is out of range");
  return (int32_t)v;
}
int32_t integer(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refusal{nullptr, ""};
  return int32_of(v, name);
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refusal{nullptr, ""};
  return (float)v;
}

// The stream of a call, torch's current one for None, and its device.
struct Stream {
  void* raw;
  int device;
  bool given;

  explicit Stream(PyObject* o) : given(o != Py_None) {
    if (!given) {
      const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
      raw = s.stream();
      device = s.device_index();
      return;
    }
    raw = (void*)(uintptr_t)attribute(o, "cuda_stream");
    device = (int)attribute(o, "device_index");
    if (device != c10::cuda::current_device())
      bad_value("the call's stream is on cuda:" + std::to_string(device) +
                ", which is not the current device");
  }
  static unsigned long long attribute(PyObject* o, const char* name) {
    PyObject* v = PyObject_GetAttrString(o, name);
    if (!v) throw Refusal{nullptr, ""};
    const unsigned long long x = PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) throw Refusal{nullptr, ""};
    return x;
  }
  // Refuses a tensor (and with it all of the call's) of another device than the one that the
  // call launches on.
  void check(const at::Tensor& t, const char* name) const {
    if (t.is_cuda() && t.device().index() != device)
      bad_value(std::string(name) + " is on cuda:" + std::to_string(t.device().index()) +
                ", the call's stream on cuda:" + std::to_string(device));
  }
};

// A call's workspace: the given one, or a buffer from the pool of the call's stream, which
// gets it back in stream order when the call returns.
struct Workspace {
  void *p = nullptr, *own = nullptr;
  size_t bytes = 0;

  Workspace(size_t need, PyObject* given, const Stream& s) {
    if (need == 0) return;
    if (given == Py_None) {
      p = own = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(need, (cudaStream_t)s.raw);
      bytes = need;
      return;
    }
    const at::Tensor& t = tensor(given, "workspace");
    if (!t.is_cuda()) bad_value("workspace must be a CUDA tensor");
    if (!t.is_contiguous()) bad_value("workspace must be contiguous");
    if ((size_t)t.nbytes() < need)
      bad_value("workspace too small: " + std::to_string(t.nbytes()) + " < " +
                std::to_string(need));
    p = t.data_ptr();
    bytes = t.nbytes();
  }
  Workspace(const Workspace&) = delete;
  ~Workspace() {
    if (own) c10::cuda::CUDACachingAllocator::raw_delete(own);
  }
};

ebd_paged_cache paged(PyObject* Ko, PyObject* Vo, PyObject* bto, PyObject* no) {
  const at::Tensor &K = tensor(Ko, "K_pages"), &V = tensor(Vo, "V_pages");
  const at::Tensor &bt = tensor(bto, "block_table"), &n = tensor(no, "seq_len");
  if (K.dim() != 4 || V.sizes() != K.sizes() || V.strides() != K.strides())
    bad_value("K_pages and V_pages must be [n_pages, Hkv, page_size, d] tensors of equal shapes "
              "and strides");
  if (!K.is_cuda() || !V.is_cuda() || !bt.is_cuda() || !n.is_cuda())
    bad_value("a paged cache's tensors must be CUDA tensors");
  check_dtype(V, K.scalar_type(), "V_pages");
  if (bt.scalar_type() != at::kInt || n.scalar_type() != at::kInt)
    bad_type("block_table and seq_len must be int32");
  if (bt.dim() != 2 || n.dim() != 1 || bt.size(0) != n.size(0) || !bt.is_contiguous() ||
      !n.is_contiguous())
    bad_value("block_table must be a contiguous [B, max_blocks] and seq_len a contiguous [B] "
              "tensor");
  if (K.stride(3) != 1)
    bad_value("the last dimension of K_pages and V_pages must be contiguous");
  ebd_paged_cache c = {};
  c.dtype = dtype_code(K);
  c.batch = int32_of(bt.size(0), "batch");
  c.n_kv_heads = int32_of(K.size(1), "n_kv_heads");
  c.head_dim = int32_of(K.size(3), "head_dim");
  c.page_size = int32_of(K.size(2), "page_size");
  c.n_pages = int32_of(K.size(0), "n_pages");
  c.max_blocks = int32_of(bt.size(1), "max_blocks");
  c.page_stride = K.stride(0);
  c.head_stride = K.stride(1);
  c.row_stride = K.stride(2);
  c.K_pages = K.data_ptr();
  c.V_pages = V.data_ptr();
  c.block_table = (const int32_t*)bt.data_ptr();
  c.seq_len = (const int32_t*)n.data_ptr();
  return c;
}

// A norm's weight, [d] or [heads, d], in x's type or float32; None: none.
struct Weight {
  void* p = nullptr;
  ebd_dtype dtype = EBD_F32;
  int64_t hs = 0;
};
Weight norm_weight(PyObject* o, ScalarType dtype, int64_t heads, int64_t d, const char* name) {
  Weight w;
  if (o == Py_None) return w;
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) bad_value(std::string(name) + " must be a CUDA tensor");
  if (t.scalar_type() != at::kFloat && t.scalar_type() != dtype)
    bad_type(std::string(name) + " has dtype " + dtype_name(t.scalar_type()) + ", expected " +
             dtype_name(dtype) + " or float32");
  const bool one = t.dim() == 1 && t.size(0) == d;
  if (!one && !(t.dim() == 2 && t.size(0) == heads && t.size(1) == d))
    bad_value(std::string(name) + " has shape " + shape_name(t.sizes()) + ", expected " +
              shape_name(std::initializer_list<int64_t>{d}) + " or " +
              shape_name(std::initializer_list<int64_t>{heads, d}));
  if (d > 1 && t.stride(-1) != 1)
    bad_value("the last dimension of " + std::string(name) + " must be contiguous");
  w.p = t.data_ptr();
  w.dtype = dtype_code(t);
  if (!one) {
    w.hs = t.stride(0);
    if (w.hs < 1) bad_value(std::string(name) + " must have a row of its own for every head");
  }
  return w;
}

struct Table {
  const float* p = nullptr;
  int32_t n_pos = 0, rot = 0;
};
Table rotary_table(PyObject* o) {
  Table r;
  if (o == Py_None) return r;
  const at::Tensor& t = tensor(o, "table");
  if (t.dim() != 3 || t.size(2) != 2)
    bad_value("table has shape " + shape_name(t.sizes()) + ", expected [n_pos, rotary_dim / 2, 2]");
  if (!t.is_cuda()) bad_value("table must be a CUDA tensor");
  if (!t.is_contiguous()) bad_value("table must be contiguous");
  check_dtype(t, at::kFloat, "table");
  r.p = (const float*)t.data_ptr();
  r.n_pos = int32_of(t.size(0), "n_pos");
  r.rot = int32_of(2 * t.size(1), "rotary_dim");
  return r;
}

// ---------------------------------------------------------------- the entry points
#define EBD_CALLS(X)                            \
  X(ebd_paged_deal)                             \
  X(ebd_norm_rotary)                            \
  X(ebd_norm_rotary_backward)                   \
  X(ebd_norm_rotary_backward_workspace_bytes)   \
  X(ebd_paged_append_norm)                      \
  X(ebd_tree_masks)                             \
  X(ebd_paged_attention_workspace_bytes)        \
  X(ebd_paged_tree_attention)                   \
  X(ebd_paged_keep)

struct {
#define X(f) decltype(&f) f = nullptr;
  EBD_CALLS(X)
#undef X
} L;

// A call's tensors are all on one GPU (the kernels take their addresses as they are).
void check_devices(PyObject* const* a, Py_ssize_t n, const char* const* names) {
  int device = -1, first = 0;
  for (int i = 0; i < n; ++i) {
    // (asked whether it is a tensor, a number takes 60 ns)
    if (a[i] == Py_None || PyLong_Check(a[i]) || PyFloat_Check(a[i])) continue;
    if (!THPVariable_Check(a[i])) continue;
    const c10::Device d = THPVariable_Unpack(a[i]).device();
    if (!d.is_cuda()) continue;
    const int at = d.index();
    if (device < 0) device = at, first = i;
    if (at != device)
      bad_value(std::string(names[i]) + " is on cuda:" + std::to_string(at) + ", " + names[first] +
                " on cuda:" + std::to_string(device));
  }
}

// Runs body() on the arguments of these names, its refusals and C++ exceptions raised as
// Python's.
template <size_t N, typename F>
PyObject* guarded(PyObject* const* a, Py_ssize_t n, const char* const (&names)[N], F body) {
  if (n != (Py_ssize_t)N) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, (Py_ssize_t)N);
    return nullptr;
  }
  if (!L.ebd_paged_keep) {
    PyErr_SetString(PyExc_RuntimeError, "the library is not bound");
    return nullptr;
  }
  try {
    check_devices(a, n, names);
    return PyLong_FromLong(body());
  } catch (const Refusal& r) {
    if (r.type) PyErr_SetString(r.type, r.text.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// The call itself, without the interpreter's lock: a full launch queue makes it wait.
template <typename F>
long launched(F call) {
  struct Unlocked {  // (an exception takes the lock again too)
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  } unlocked;
  return call();
}

PyObject* bind(PyObject*, PyObject* addresses) {  // {name: address}
#define X(f)                                                                     \
  {                                                                              \
    PyObject* v = PyDict_GetItemString(addresses, #f);                           \
    const unsigned long long p = v ? PyLong_AsUnsignedLongLong(v) : 0;           \
    if (PyErr_Occurred()) return nullptr;                                        \
    if (!p) {                                                                    \
      PyErr_SetString(PyExc_RuntimeError, "bind: no address of " #f);            \
      return nullptr;                                                            \
    }                                                                            \
    L.f = reinterpret_cast<decltype(L.f)>((uintptr_t)p);                         \
  }
  EBD_CALLS(X)
#undef X
  Py_RETURN_NONE;
}

PyObject* deal(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"free_pages", "n_free", "held", "K_pages", "V_pages",
      "block_table", "seq_len", "dev_status", "n_new", "n_tokens", "window", "cu_new", "positions",
      "slots", "served", "seq_len_out", "held_out", "n_free_out", "stream"};
  return guarded(a, n, names, [&] {
    const ebd_paged_cache c = paged(a[3], a[4], a[5], a[6]);
    const int64_t B = c.batch;
    const int32_t T = integer(a[9], "n_tokens"), window = integer(a[10], "window");
    const int32_t* n_new = ints(a[8], {B}, "n_new");
    const int32_t *held = ints(a[2], {B, 2}, "held"), *n_free = ints(a[1], {1}, "n_free");
    int32_t* free_pages = ints(a[0], {c.n_pages}, "free_pages");
    int32_t* seq_len_out = ints(a[15], {B}, "seq_len_out");
    int32_t* held_out = ints(a[16], {B, 2}, "held_out");
    int32_t* n_free_out = ints(a[17], {1}, "n_free_out");
    int32_t *cu = ints(a[11], {B + 1}, "cu_new"), *served = ints(a[14], {B}, "served");
    int32_t* pos = ints(a[12], {T}, "positions");
    int64_t* slots = address<int64_t>(a[13], at::kLong, {T}, "slots");
    int32_t* status = ints(a[7], {1}, "dev_status");
    const Stream s(a[18]);
    s.check(tensor(a[6], "seq_len"), "seq_len");
    return launched([&] {
      return L.ebd_paged_deal(c.batch, c.page_size, c.n_pages, c.max_blocks, T, window, n_new,
                              c.seq_len, held, n_free, free_pages, (int32_t*)c.block_table,
                              seq_len_out, held_out, n_free_out, cu, served, pos, slots, status,
                              s.raw);
    });
  });
}

const int32_t* norm_positions(PyObject* o, const Table& t, int64_t T) {
  if (!t.p) return nullptr;
  if (o == Py_None) bad_value("a rotation needs positions");
  return ints(o, {T}, "positions");
}

PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"x", "weight", "positions", "table", "out", "layout", "eps",
      "dev_status", "stream"};
  return guarded(a, n, names, [&] {
    const at::Tensor& xt = three(a[0], "x", "[T, H, d]");
    const int32_t T = int32_of(xt.size(0), "T"), H = int32_of(xt.size(1), "H");
    const int32_t d = int32_of(xt.size(2), "d");
    const ScalarType dt = xt.scalar_type();
    const Rows x = rows(a[0], dt, T, H, d, "x"), y = rows(a[4], dt, T, H, d, "out");
    if (a[1] == Py_None) bad_type("weight must be a torch.Tensor");
    const Weight w = norm_weight(a[1], dt, H, d, "weight");
    const Table t = rotary_table(a[3]);
    const int32_t* pos = norm_positions(a[2], t, T);
    const int32_t layout = integer(a[5], "layout");
    const float eps = real(a[6]);
    int32_t* status = ints(a[7], {1}, "dev_status");
    const ebd_dtype code = dtype_code(xt);
    const Stream s(a[8]);
    s.check(xt, "x");
    return launched([&] {
      return L.ebd_norm_rotary(code, T, H, d, x.p, x.ts, x.hs, w.p, w.dtype, w.hs, eps, pos, t.p,
                               t.n_pos, t.rot, (ebd_rotary_layout)layout, y.p, y.ts, y.hs, status,
                               s.raw);
    });
  });
}

PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"dy", "x", "weight", "positions", "table", "dx", "dweight",
      "layout", "eps", "workspace", "dev_status", "stream"};
  return guarded(a, n, names, [&] {
    const at::Tensor& xt = three(a[1], "x", "[T, H, d]");
    const int32_t T = int32_of(xt.size(0), "T"), H = int32_of(xt.size(1), "H");
    const int32_t d = int32_of(xt.size(2), "d");
    const ScalarType dt = xt.scalar_type();
    const Rows x = rows(a[1], dt, T, H, d, "x"), dy = rows(a[0], dt, T, H, d, "dy");
    const Rows dx = rows(a[5], dt, T, H, d, "dx");
    if (a[2] == Py_None) bad_type("weight must be a torch.Tensor");
    const Weight w = norm_weight(a[2], dt, H, d, "weight");
    float* dw = w.hs ? address<float>(a[6], at::kFloat, {H, d}, "dweight")
                     : address<float>(a[6], at::kFloat, {d}, "dweight");
    const Table t = rotary_table(a[4]);
    const int32_t* pos = norm_positions(a[3], t, T);
    const int32_t layout = integer(a[7], "layout");
    const float eps = real(a[8]);
    int32_t* status = ints(a[10], {1}, "dev_status");
    const ebd_dtype code = dtype_code(xt);
    const Stream s(a[11]);
    s.check(xt, "x");
    const Workspace ws(L.ebd_norm_rotary_backward_workspace_bytes(H, d, w.hs != 0), a[9], s);
    return launched([&] {
      return L.ebd_norm_rotary_backward(code, T, H, d, dy.p, dy.ts, dy.hs, x.p, x.ts, x.hs,
                                        w.p, w.dtype, w.hs, eps, pos, t.p, t.n_pos, t.rot,
                                        (ebd_rotary_layout)layout, dx.p, dx.ts, dx.hs, dw, status,
                                        ws.p, ws.bytes, s.raw);
    });
  });
}

PyObject* append_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"K_pages", "V_pages", "block_table", "seq_len", "dev_status",
      "k_new", "v_new", "k_weight", "q", "q_weight", "q_out", "cu_new", "slots", "positions",
      "table", "layout", "eps", "stream"};
  return guarded(a, n, names, [&] {
    if (a[8] == Py_None && (a[9] != Py_None || a[10] != Py_None))
      bad_value("q_weight or q_out without q");
    const ebd_paged_cache c = paged(a[0], a[1], a[2], a[3]);
    const at::Tensor& Kt = THPVariable_Unpack(a[0]);
    const ScalarType dt = Kt.scalar_type();
    const int64_t T = three(a[5], "k_new", "[T, Hkv, d]").size(0), H = c.n_kv_heads, d = c.head_dim;
    const Rows k = rows(a[5], dt, T, H, d, "k_new"), v = rows(a[6], dt, T, H, d, "v_new");
    if ((a[11] == Py_None) == (a[12] == Py_None))
      bad_value("tokens are placed by cu_new or by slots, one of the two");
    const Table t = rotary_table(a[14]);
    if (t.p && a[13] == Py_None && a[11] == Py_None)
      bad_value("slots tell no positions: a rotation needs them");
    const Weight kw = norm_weight(a[7], dt, H, d, "k_weight");
    Weight qw;
    Rows q, o;
    int64_t hq = 0;
    if (a[8] != Py_None) {
      if (a[10] == Py_None) bad_value("q must be [T, Hq, d] and come with q_out");
      hq = three(a[8], "q", "[T, Hq, d] and come with q_out").size(1);
      q = rows(a[8], dt, T, hq, d, "q");
      o = rows(a[10], dt, T, hq, d, "q_out");
      qw = norm_weight(a[9], dt, hq, d, "q_weight");
      if (kw.p && qw.p && kw.dtype != qw.dtype)
        bad_type("k_weight and q_weight must have one dtype");
    }
    const int32_t* cu = ints(a[11], {c.batch + 1}, "cu_new");
    const int64_t* slots = address<int64_t>(a[12], at::kLong, {T}, "slots");
    const int32_t* pos = ints(a[13], {T}, "positions");
    const int32_t layout = integer(a[15], "layout");
    const float eps = real(a[16]);
    int32_t* status = ints(a[4], {1}, "dev_status");
    const int32_t T32 = int32_of(T, "T"), hq32 = int32_of(hq, "Hq");
    const Stream s(a[17]);
    s.check(Kt, "K_pages");
    return launched([&] {
      return L.ebd_paged_append_norm(&c, T32, cu, slots, pos, k.p, k.ts, k.hs, v.p, v.ts, v.hs,
                                     kw.p, kw.hs, qw.p, qw.hs, qw.p ? qw.dtype : kw.dtype, eps, t.p,
                                     t.n_pos, t.rot, (ebd_rotary_layout)layout, hq32, q.p, q.ts,
                                     q.hs, o.p, o.ts, o.hs, status, s.raw);
    });
  });
}

PyObject* tree_masks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"parents", "cu_new", "seq_len", "max_new", "window", "mask",
      "positions", "dev_status", "stream"};
  return guarded(a, n, names, [&] {
    const at::Tensor &pt = tensor(a[0], "parents"), &st = tensor(a[2], "seq_len");
    if (pt.dim() != 1 || st.dim() != 1) bad_value("parents must be [T] and seq_len [B]");
    const int64_t T = pt.size(0), B = st.size(0);
    const int32_t most = integer(a[3], "max_new"), window = integer(a[4], "window");
    const int64_t words = ((int64_t)most + 31) / 32;
    const int32_t *parents = ints(a[0], {T}, "parents"), *cu = ints(a[1], {B + 1}, "cu_new");
    const int32_t* seq_len = ints(a[2], {B}, "seq_len");
    int32_t *mask = ints(a[5], {T, words}, "mask"), *pos = ints(a[6], {T}, "positions");
    int32_t* status = ints(a[7], {1}, "dev_status");
    const int32_t T32 = int32_of(T, "T"), B32 = int32_of(B, "B");
    const Stream s(a[8]);
    s.check(pt, "parents");
    return launched([&] {
      return L.ebd_tree_masks(B32, T32, most, parents, cu, seq_len, window, (uint32_t*)mask,
                              (int32_t)words, pos, status, s.raw);
    });
  });
}

PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"K_pages", "V_pages", "block_table", "seq_len", "dev_status",
      "q", "cu_new", "max_new", "mask", "positions", "y", "lse", "scale", "window", "workspace",
      "stream"};
  return guarded(a, n, names, [&] {
    const ebd_paged_cache c = paged(a[0], a[1], a[2], a[3]);
    const at::Tensor& qt = three(a[5], "q", "[T, Hq, d]");
    const ScalarType dt = THPVariable_Unpack(a[0]).scalar_type();
    const int64_t T = qt.size(0), hq = qt.size(1), d = c.head_dim;
    const Rows q = rows(a[5], dt, T, hq, d, "q");
    int64_t words = 0;  // (no mask: causal)
    if (a[8] != Py_None) {
      const at::Tensor& mt = tensor(a[8], "mask");
      if (mt.dim() != 2) bad_value("mask must be [T, W]");
      words = mt.size(1);
      if (words < 1 && T > 0) bad_value("mask must have a word per 32 new tokens");
    }
    const int32_t most = integer(a[7], "max_new"), window = integer(a[13], "window");
    const int32_t* cu = ints(a[6], {c.batch + 1}, "cu_new");
    const int32_t *mask = ints(a[8], {T, words}, "mask"), *pos = ints(a[9], {T}, "positions");
    const Rows y = rows(a[10], dt, T, hq, d, "y");
    if (!THPVariable_Unpack(a[10]).is_contiguous()) bad_value("y must be contiguous");
    float* lse = address<float>(a[11], at::kFloat, {T, hq}, "lse");
    const float scale = a[12] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : real(a[12]);
    int32_t* status = ints(a[4], {1}, "dev_status");
    const int32_t T32 = int32_of(T, "T"), hq32 = int32_of(hq, "Hq");
    const int32_t words32 = int32_of(words, "W");
    const Stream s(a[15]);
    s.check(qt, "q");
    const Workspace ws(L.ebd_paged_attention_workspace_bytes(&c, hq32, most), a[14], s);
    return launched([&] {
      return L.ebd_paged_tree_attention(&c, T32, most, hq32, cu, q.p, q.ts, q.hs, scale, window,
                                        (const uint32_t*)mask, words32, pos, y.p, lse, status,
                                        ws.p, ws.bytes, s.raw);
    });
  });
}

PyObject* keep(PyObject*, PyObject* const* a, Py_ssize_t n) {
  static const char* const names[] = {"K_pages", "V_pages", "block_table", "seq_len", "dev_status",
      "cu_new", "path", "n_accepted", "seq_len_out", "K_layers", "V_layers", "stream"};
  return guarded(a, n, names, [&] {
    const ebd_paged_cache c = paged(a[0], a[1], a[2], a[3]);
    int64_t layers = 1, stride = 0;
    if ((a[9] == Py_None) != (a[10] == Py_None))
      bad_value("K_layers and V_layers come together");
    if (a[9] != Py_None) {
      const char* names[2] = {"K_layers", "V_layers"};
      for (int i = 0; i < 2; ++i) {
        const at::Tensor &t = tensor(a[9 + i], names[i]), &first = THPVariable_Unpack(a[i]);
        check_dtype(t, first.scalar_type(), names[i]);
        if (t.dim() != 5 || t.sizes().slice(1) != first.sizes() ||
            t.strides().slice(1) != first.strides())
          bad_value(std::string(names[i]) + " must be [L, n_pages, Hkv, page_size, d] with the "
                                            "strides of the cache's pools");
        if (t.data_ptr() != first.data_ptr())
          bad_value(std::string("the cache's pool must be the first of ") + names[i]);
        if (i == 1 && (t.size(0) != layers || t.stride(0) != stride))
          bad_value("K_layers and V_layers must have one shape and one layer stride");
        layers = t.size(0);
        stride = t.stride(0);
      }
    }
    const at::Tensor& pt = tensor(a[6], "path");
    if (pt.dim() != 2) bad_value("path must be [B, max_path]");
    const int64_t B = c.batch, most = pt.size(1);
    const int32_t *cu = ints(a[5], {B + 1}, "cu_new"), *path = ints(a[6], {B, most}, "path");
    const int32_t* accepted = ints(a[7], {B}, "n_accepted");
    int32_t* len = ints(a[8], {B}, "seq_len_out");
    int32_t* status = ints(a[4], {1}, "dev_status");
    const int32_t layers32 = int32_of(layers, "L"), most32 = int32_of(most, "max_path");
    const Stream s(a[11]);
    s.check(THPVariable_Unpack(a[0]), "K_pages");
    return launched([&] {
      return L.ebd_paged_keep(&c, layers32, stride, cu, path, most32, accepted, len, status, s.raw);
    });
  });
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_O, nullptr}, FAST(deal), FAST(norm),
                         FAST(norm_backward), FAST(append_norm), FAST(tree_masks),
                         FAST(tree_attention), FAST(keep), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "ebd_call", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ebd_call() { return PyModule_Create(&module); }
