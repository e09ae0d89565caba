// The hot entry points of libtrdq.so for plain torch tensors: what trdq.py does for a call (checks, outputs, pointers, strides, current
// stream) in one native function.  A small layer is bound by this host work, not by the GPU: through ctypes a call took about 9 us,
// 2 us of it for each output, 1.5 for the conversion of the arguments and 1 for the tensors' attributes, and a linear layer of 256 x 1024
// (two calls, 7 us on the GPU) 19.3 us, now 10.3; three calls for two ragged row segments 37.4, now 22.6.
//
// Every function returns None for arguments it does not handle: tensor subclasses, tensors of other devices or layouts, wrapped tensors
// (functorch, functional, fake), numbers that are not Python ints, an active function or dispatch mode (torch.set_default_device is one).  The caller
// then goes its general way, which costs what it did and 0.15 us for the question, and is where wrong arguments are reported.  A status other than
// TRDQ_OK is returned as an int.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <limits>

#include "../../include/trdq.h"

namespace {

// Addresses in the library that trdq.py has loaded.
struct Entry {
  decltype(&trdq_rotate_quantize) rotate_quantize;
  decltype(&trdq_norm_rotate_quantize) norm_rotate_quantize;
  decltype(&trdq_rotate_quantize_asym) rotate_quantize_asym;
  decltype(&trdq_linear_act) linear_act;
  decltype(&trdq_linear_cfg) linear_cfg;
  decltype(&trdq_linear_asym) linear_asym;
  decltype(&trdq_linear_splitk_workspace) splitk_workspace;
  decltype(&trdq_linear_splitk) linear_splitk;
} entry;

struct BlockEntry {
  decltype(&trdq_fp8_quantize) fp8_quantize;
  decltype(&trdq_fp8_quantize_weights) fp8_quantize_weights;
  decltype(&trdq_fp8_linear) fp8_linear;
  decltype(&trdq_gated_norm) gated_norm;
  decltype(&trdq_gated_norm_fp8) gated_norm_fp8;
  decltype(&trdq_gated_norm_backward_workspace) gated_norm_backward_workspace;
  decltype(&trdq_gated_norm_backward) gated_norm_backward;
} block_entry;

bool no_modes() { return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// A strided CUDA tensor that is nothing but that.
bool plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  static const c10::DispatchKeySet ordinary = c10::DispatchKeySet({c10::DispatchKey::Dense, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutogradFunctionality,
                                                                   c10::DispatchKey::AutocastCUDA}) |
                                              c10::DispatchKeySet(c10::BackendComponent::CUDABit);
  return t.defined() && t.is_cuda() && (t.key_set().raw_repr() & ~ordinary.raw_repr()) == 0 && t.has_storage();
}
bool plain_or_none(PyObject* o) { return o == Py_None || plain(o); }
void* pointer(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).data_ptr(); }

// an exact Python int that fits T
template <typename T>
bool number(PyObject* o, T* out) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow || v < static_cast<long long>(std::numeric_limits<T>::min()) || v > static_cast<long long>(std::numeric_limits<T>::max())) return false;
  *out = static_cast<T>(v);
  return true;
}
bool handle(PyObject* o, void** out) {
  if (!PyLong_CheckExact(o)) return false;
  *out = PyLong_AsVoidPtr(o);
  return true;
}

// X of a rotate + quantize call: two-dimensional, 16-bit elements, columns side by side
bool activations(PyObject* o, int64_t K, int32_t* M, int64_t* ldx) {
  if (!plain(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (x.dim() != 2 || x.element_size() != 2 || x.stride(1) != 1 || x.size(0) > std::numeric_limits<int32_t>::max()) return false;
  *M = static_cast<int32_t>(x.size(0));
  *ldx = *M > 1 ? x.stride(0) : K;
  return true;
}
// codes of a linear call: the rows
bool rows(PyObject* o, int32_t* M) {
  if (!plain(o)) return false;
  const at::Tensor& c = THPVariable_Unpack(o);
  if (c.dim() < 1 || c.size(0) > std::numeric_limits<int32_t>::max()) return false;
  *M = static_cast<int32_t>(c.size(0));
  return true;
}
bool output(PyObject* o, int32_t M, int64_t N, int64_t* ld) {
  *ld = N;
  if (o == Py_None) return true;
  if (!plain(o) || THPVariable_Unpack(o).dim() < 1) return false;
  if (M > 1) *ld = THPVariable_Unpack(o).stride(0);
  return true;
}

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// A new CUDA tensor from the allocator's own entry: what torch.empty gives, without the dispatch (no_modes() has been asked).
at::Tensor new_tensor(at::IntArrayRef sizes, at::ScalarType type, at::Device device) { return at::detail::empty_cuda(sizes, type, device, c10::nullopt); }

struct WithoutGil {
  PyThreadState* const state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};

// The outputs of a call: given by the caller or new tensors on the device of `like`.
class Outputs {
 public:
  explicit Outputs(PyObject* like) : options_(THPVariable_Unpack(like).options()) {}
  void add(PyObject* given, int32_t rows, int64_t columns, at::ScalarType type) { put(given, rows, columns, 2, type); }
  void add(PyObject* given, int32_t rows, at::ScalarType type) { put(given, rows, 0, 1, type); }

  // Makes the new ones, runs the library call (it gets the pointers) and returns the outputs in a tuple, a list or alone, or the status.  All
  // of it without the GIL: an allocation may wait for the device, and for other threads' work on it.
  template <typename Call>
  PyObject* run(Call&& call, bool list = false) {
    trdq_status st;
    {
      WithoutGil released;
      void* pointers[kMost];
      for (int i = 0; i < n_; ++i) {
        Item& o = item_[i];
        if (!o.given) o.made = new_tensor(at::IntArrayRef(o.sizes, o.dims), o.type, options_.device());
        pointers[i] = o.given ? o.pointer : o.made.data_ptr();
      }
      st = call(pointers);
    }
    if (st != TRDQ_OK) return PyLong_FromLong(st);
    if (n_ == 1) return wrap(item_[0]);
    PyObject* const r = list ? PyList_New(n_) : PyTuple_New(n_);
    if (!r) return nullptr;
    for (int i = 0; i < n_; ++i) {
      PyObject* const o = wrap(item_[i]);
      if (!o) {
        Py_DECREF(r);
        return nullptr;
      }
      if (list) {
        PyList_SET_ITEM(r, i, o);
      } else {
        PyTuple_SET_ITEM(r, i, o);
      }
    }
    return r;
  }

 private:
  static constexpr int kMost = 3;
  struct Item {
    PyObject* given;  // borrowed from the caller's arguments
    void* pointer;    // of the given one
    int64_t sizes[2];
    int dims;
    at::ScalarType type;
    at::Tensor made;
  };
  void put(PyObject* given, int64_t rows, int64_t columns, int dims, at::ScalarType type) {
    Item& o = item_[n_++];
    o.given = given == Py_None ? nullptr : given;
    o.pointer = pointer(given);
    o.sizes[0] = rows;
    o.sizes[1] = columns;
    o.dims = dims;
    o.type = type;
  }
  static PyObject* wrap(Item& o) {
    if (!o.given) return THPVariable_Wrap(std::move(o.made));
    Py_INCREF(o.given);
    return o.given;
  }

  at::TensorOptions options_;
  Item item_[kMost];
  int n_ = 0;
};

#define GENERAL_WAY_UNLESS(condition) \
  if (!(condition)) Py_RETURN_NONE

// (rot, K, t, X, codes, scales)
PyObject* rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* rot;
  int64_t K, ldx;
  int32_t t, M;
  GENERAL_WAY_UNLESS(n == 6 && handle(a[0], &rot) && number(a[1], &K) && number(a[2], &t) && activations(a[3], K, &M, &ldx) &&
                     plain_or_none(a[4]) && plain_or_none(a[5]) && no_modes());
  Outputs out(a[3]);
  out.add(a[4], M, K, at::kChar);
  out.add(a[5], M, at::kFloat);
  void* const x = pointer(a[3]);
  void* const s = stream();
  return out.run([&](void** o) { return entry.rotate_quantize(static_cast<trdq_rotation*>(rot), t, x, ldx, M, static_cast<int8_t*>(o[0]), static_cast<float*>(o[1]), s); });
  END_HANDLE_TH_ERRORS
}

// (rot, K, t, X, shift, scale, rows_per_sample, eps, codes, scales)
PyObject* norm_rotate_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* rot;
  int64_t K, ldx;
  int32_t t, M, per_sample;
  GENERAL_WAY_UNLESS(n == 10 && handle(a[0], &rot) && number(a[1], &K) && number(a[2], &t) && activations(a[3], K, &M, &ldx) &&
                     plain_or_none(a[4]) && plain_or_none(a[5]) && PyFloat_CheckExact(a[7]) && plain_or_none(a[8]) && plain_or_none(a[9]) && no_modes());
  if (a[6] == Py_None) {
    per_sample = M > 1 ? M : 1;
  } else {
    GENERAL_WAY_UNLESS(number(a[6], &per_sample));
  }
  const float eps = static_cast<float>(PyFloat_AS_DOUBLE(a[7]));
  Outputs out(a[3]);
  out.add(a[8], M, K, at::kChar);
  out.add(a[9], M, at::kFloat);
  void *const x = pointer(a[3]), *const shift = pointer(a[4]), *const scale = pointer(a[5]);
  void* const s = stream();
  return out.run([&](void** o) {
    return entry.norm_rotate_quantize(static_cast<trdq_rotation*>(rot), t, x, ldx, M, shift, scale, per_sample, eps, static_cast<int8_t*>(o[0]),
                                      static_cast<float*>(o[1]), s);
  });
  END_HANDLE_TH_ERRORS
}

// (rot, K, t, X)
PyObject* rotate_quantize_asym(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* rot;
  int64_t K, ldx;
  int32_t t, M;
  GENERAL_WAY_UNLESS(n == 4 && handle(a[0], &rot) && number(a[1], &K) && number(a[2], &t) && activations(a[3], K, &M, &ldx) && no_modes());
  Outputs out(a[3]);
  out.add(Py_None, M, K, at::kByte);
  out.add(Py_None, M, at::kFloat);
  out.add(Py_None, M, at::kInt);
  void* const x = pointer(a[3]);
  void* const s = stream();
  return out.run([&](void** o) {
    return entry.rotate_quantize_asym(static_cast<trdq_rotation*>(rot), t, x, ldx, M, static_cast<uint8_t*>(o[0]), static_cast<float*>(o[1]),
                                      static_cast<int32_t*>(o[2]), s);
  });
  END_HANDLE_TH_ERRORS
}

// (w, N, t, codes, scales, bias, out, act)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* w;
  int64_t N, ldy;
  int32_t t, M, act;
  GENERAL_WAY_UNLESS(n == 8 && handle(a[0], &w) && number(a[1], &N) && number(a[2], &t) && rows(a[3], &M) && plain(a[4]) && plain_or_none(a[5]) &&
                     output(a[6], M, N, &ldy) && number(a[7], &act) && no_modes());
  Outputs out(a[3]);
  out.add(a[6], M, N, at::kBFloat16);
  void *const codes = pointer(a[3]), *const scales = pointer(a[4]), *const bias = pointer(a[5]);
  void* const s = stream();
  return out.run([&](void** o) {
    return entry.linear_act(static_cast<trdq_weights*>(w), t, static_cast<int8_t*>(codes), static_cast<float*>(scales), M, bias, o[0], ldy, act, s);
  });
  END_HANDLE_TH_ERRORS
}

// (w, N, t, codes, scales, zero_points, bias, out)
PyObject* linear_asym(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* w;
  int64_t N, ldy;
  int32_t t, M;
  GENERAL_WAY_UNLESS(n == 8 && handle(a[0], &w) && number(a[1], &N) && number(a[2], &t) && rows(a[3], &M) && plain(a[4]) && plain(a[5]) &&
                     plain_or_none(a[6]) && output(a[7], M, N, &ldy) && no_modes());
  Outputs out(a[3]);
  out.add(a[7], M, N, at::kBFloat16);
  void *const codes = pointer(a[3]), *const scales = pointer(a[4]), *const zero = pointer(a[5]), *const bias = pointer(a[6]);
  void* const s = stream();
  return out.run([&](void** o) {
    return entry.linear_asym(static_cast<trdq_weights*>(w), t, static_cast<uint8_t*>(codes), static_cast<float*>(scales), static_cast<int32_t*>(zero), M,
                             bias, o[0], ldy, s);
  });
  END_HANDLE_TH_ERRORS
}

// (w, N, t, codes, scales, bias, out, workspace)
PyObject* linear_splitk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* w;
  int64_t N, ldy;
  int32_t t, M, splits = 0;
  uint64_t bytes = 0;
  GENERAL_WAY_UNLESS(n == 8 && handle(a[0], &w) && number(a[1], &N) && number(a[2], &t) && rows(a[3], &M) && plain(a[4]) && plain_or_none(a[5]) &&
                     output(a[6], M, N, &ldy) && plain_or_none(a[7]) && no_modes() &&
                     entry.splitk_workspace(static_cast<trdq_weights*>(w), M, &splits, &bytes) == TRDQ_OK);
  Outputs out(a[3]);
  out.add(a[6], M, N, at::kBFloat16);
  void *const codes = pointer(a[3]), *const scales = pointer(a[4]), *const bias = pointer(a[5]), *const given = pointer(a[7]);
  const at::TensorOptions options = THPVariable_Unpack(a[3]).options().dtype(at::kByte);
  const bool make = a[7] == Py_None && bytes;
  if (a[7] != Py_None) bytes = static_cast<uint64_t>(THPVariable_Unpack(a[7]).numel() * THPVariable_Unpack(a[7]).element_size());
  void* const s = stream();
  return out.run([&](void** o) {
    at::Tensor made;
    if (make) made = at::empty({static_cast<int64_t>(bytes)}, options);
    return entry.linear_splitk(static_cast<trdq_weights*>(w), t, static_cast<int8_t*>(codes), static_cast<float*>(scales), M, bias, o[0], ldy,
                               make ? made.data_ptr() : given, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// (w, N, t, (codes, codes), (scales, scales), bias): the outputs in a list
PyObject* linear_cfg(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* w;
  int64_t N;
  int32_t t, M[2];
  GENERAL_WAY_UNLESS(n == 6 && handle(a[0], &w) && number(a[1], &N) && number(a[2], &t) && plain_or_none(a[5]) && no_modes());
  PyObject *codes[2], *scales[2];
  auto two = [](PyObject* o, PyObject** items) {
    if (PyList_CheckExact(o) && PyList_GET_SIZE(o) == 2) {
      items[0] = PyList_GET_ITEM(o, 0);
      items[1] = PyList_GET_ITEM(o, 1);
      return true;
    }
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) return false;
    items[0] = PyTuple_GET_ITEM(o, 0);
    items[1] = PyTuple_GET_ITEM(o, 1);
    return true;
  };
  GENERAL_WAY_UNLESS(two(a[3], codes) && two(a[4], scales) && rows(codes[0], &M[0]) && rows(codes[1], &M[1]) && plain(scales[0]) && plain(scales[1]));
  Outputs out(codes[0]);
  at::Tensor held[4];  // the caller's lists may change while the GIL is released
  const int8_t* c[2];
  const float* sx[2];
  const int64_t ldy[2] = {N, N};
  for (int i = 0; i < 2; ++i) {
    held[2 * i] = THPVariable_Unpack(codes[i]);
    held[2 * i + 1] = THPVariable_Unpack(scales[i]);
    c[i] = static_cast<const int8_t*>(held[2 * i].data_ptr());
    sx[i] = static_cast<const float*>(held[2 * i + 1].data_ptr());
    out.add(Py_None, M[i], N, at::kBFloat16);
  }
  void* const bias = pointer(a[5]);
  void* const s = stream();
  return out.run([&](void** y) { return entry.linear_cfg(static_cast<trdq_weights*>(w), t, c, sx, M, bias, y, ldy, s); }, true);
  END_HANDLE_TH_ERRORS
}

// ---- the block-scaled path and the fused norms.  Their tensors have to be on the current device and of the documented shapes and types; anything
// else goes the general way, which says what is wrong with it.

bool on_device(const at::Tensor& t, c10::DeviceIndex device) { return t.device().index() == device; }
bool fp8_codes(const at::Tensor& t) { return t.scalar_type() == at::kFloat8_e4m3fn || t.scalar_type() == at::kByte; }
bool matrix(const at::Tensor& t, int64_t rows, int64_t cols) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && (t.stride(1) == 1 || cols == 1); }
bool whole(const at::Tensor& t, int64_t rows, int64_t cols) { return matrix(t, rows, cols) && t.is_contiguous(); }
int64_t leading(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
const at::Tensor& tensor(PyObject* o) { return THPVariable_Unpack(o); }
bool int32_size(int64_t n) { return n <= std::numeric_limits<int32_t>::max(); }
// None for no rotation, or its handle
bool handle_or_none(PyObject* o, void** out) {
  *out = nullptr;
  return o == Py_None || handle(o, out);
}

// (rot or None, t, X, codes, scales, weights)
PyObject* fp8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  void* rot;
  int32_t t, weights;
  GENERAL_WAY_UNLESS(n == 6 && handle_or_none(a[0], &rot) && number(a[1], &t) && plain(a[2]) && plain_or_none(a[3]) && plain_or_none(a[4]) &&
                     number(a[5], &weights) && no_modes());
  const at::Tensor& x = tensor(a[2]);
  const c10::DeviceIndex device = c10::cuda::current_device();
  GENERAL_WAY_UNLESS(x.dim() == 2 && x.scalar_type() == at::kBFloat16 && on_device(x, device) && int32_size(x.size(0)) && int32_size(x.size(1)));
  const int64_t M = x.size(0), K = x.size(1);
  const int64_t srows = weights ? (M + 127) / 128 : K / 128, scols = weights ? K / 128 : M;
  GENERAL_WAY_UNLESS(int32_size(srows) && (weights ? x.is_contiguous() : matrix(x, M, K)));
  GENERAL_WAY_UNLESS(a[3] == Py_None || (on_device(tensor(a[3]), device) && fp8_codes(tensor(a[3])) && whole(tensor(a[3]), M, K)));
  GENERAL_WAY_UNLESS(a[4] == Py_None || (on_device(tensor(a[4]), device) && tensor(a[4]).scalar_type() == at::kFloat && whole(tensor(a[4]), srows, scols)));
  Outputs out(a[2]);
  out.add(a[3], static_cast<int32_t>(M), K, at::kFloat8_e4m3fn);
  out.add(a[4], static_cast<int32_t>(srows), scols, at::kFloat);
  const int64_t ldx = leading(x);
  void* const px = x.data_ptr();
  void* const s = stream();
  return out.run([&](void** o) {
    return weights ? block_entry.fp8_quantize_weights(static_cast<trdq_rotation*>(rot), t, px, static_cast<int32_t>(M), static_cast<int32_t>(K),
                                                      static_cast<uint8_t*>(o[0]), static_cast<float*>(o[1]), s)
                   : block_entry.fp8_quantize(static_cast<trdq_rotation*>(rot), t, px, ldx, static_cast<int32_t>(M), static_cast<int32_t>(K),
                                              static_cast<uint8_t*>(o[0]), static_cast<float*>(o[1]), s);
  });
  END_HANDLE_TH_ERRORS
}

// (codes, scales, w_codes, w_scales, bias, out, act)
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int32_t act;
  GENERAL_WAY_UNLESS(n == 7 && plain(a[0]) && plain(a[1]) && plain(a[2]) && plain(a[3]) && plain_or_none(a[4]) && plain_or_none(a[5]) &&
                     number(a[6], &act) && no_modes());
  const at::Tensor &q = tensor(a[0]), &sx = tensor(a[1]), &qw = tensor(a[2]), &sw = tensor(a[3]);
  const c10::DeviceIndex device = c10::cuda::current_device();
  GENERAL_WAY_UNLESS(q.dim() == 2 && qw.dim() == 2 && int32_size(q.size(0)) && int32_size(q.size(1)) && int32_size(qw.size(0)));
  const int64_t M = q.size(0), K = q.size(1), N = qw.size(0);
  GENERAL_WAY_UNLESS(fp8_codes(q) && whole(q, M, K) && fp8_codes(qw) && whole(qw, N, K) && sx.scalar_type() == at::kFloat && whole(sx, K / 128, M) &&
                     sw.scalar_type() == at::kFloat && whole(sw, (N + 127) / 128, K / 128));
  GENERAL_WAY_UNLESS(on_device(q, device) && on_device(sx, device) && on_device(qw, device) && on_device(sw, device));
  if (a[4] != Py_None) {
    const at::Tensor& b = tensor(a[4]);
    GENERAL_WAY_UNLESS(on_device(b, device) && b.scalar_type() == at::kBFloat16 && b.dim() == 1 && b.size(0) == N && b.is_contiguous());
  }
  int64_t ldy = N;
  if (a[5] != Py_None) {
    const at::Tensor& y = tensor(a[5]);
    GENERAL_WAY_UNLESS(on_device(y, device) && y.scalar_type() == at::kBFloat16 && matrix(y, M, N));
    ldy = leading(y);
  }
  Outputs out(a[0]);
  out.add(a[5], static_cast<int32_t>(M), N, at::kBFloat16);
  void *const pq = q.data_ptr(), *const psx = sx.data_ptr(), *const pqw = qw.data_ptr(), *const psw = sw.data_ptr(), *const bias = pointer(a[4]);
  void* const s = stream();
  return out.run([&](void** o) {
    return block_entry.fp8_linear(static_cast<uint8_t*>(pq), static_cast<float*>(psx), static_cast<int32_t>(M), static_cast<int32_t>(K),
                                  static_cast<uint8_t*>(pqw), static_cast<float*>(psw), static_cast<int32_t>(N), bias, o[0], ldy, act, s);
  });
  END_HANDLE_TH_ERRORS
}

bool real(PyObject* o, float* out) {
  if (!PyFloat_CheckExact(o)) return false;
  *out = static_cast<float>(PyFloat_AS_DOUBLE(o));
  return true;
}

// The arguments that the three norm calls share: X, branch, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale
constexpr int kNormArgs = 12;
bool norm_op(PyObject* const* a, c10::DeviceIndex* current, trdq_gated_norm_op* op, int64_t* samples) {
  if (!plain(a[0])) return false;
  for (int i = 1; i < 7; ++i)
    if (!plain_or_none(a[i])) return false;
  // (asked for behind the first CUDA tensor: without a device the question itself is an error, and not the one that the general way reports)
  const c10::DeviceIndex device = *current = c10::cuda::current_device();
  const at::Tensor& x = tensor(a[0]);
  if (x.dim() != 2 || (x.scalar_type() != at::kBFloat16 && x.scalar_type() != at::kFloat) || !int32_size(x.size(0)) || !int32_size(x.size(1))) return false;
  const int64_t M = x.size(0), D = x.size(1);
  if (!matrix(x, M, D) || !on_device(x, device)) return false;
  int32_t rows = M > 1 ? static_cast<int32_t>(M) : 1;
  if (a[9] != Py_None && !number(a[9], &rows)) return false;
  if (rows < 1 || !number(a[7], &op->norm) || !number(a[8], &op->post_norm) || !real(a[10], &op->eps) || !real(a[11], &op->res_scale)) return false;
  *samples = (M + rows - 1) / rows;
  op->M = static_cast<int32_t>(M);
  op->D = static_cast<int32_t>(D);
  op->rows_per_sample = rows;
  op->stream_f32 = x.scalar_type() == at::kFloat;
  op->X = x.data_ptr();
  op->ldx = leading(x);
  const void* p[6];
  int64_t ld[6];
  for (int i = 1; i < 7; ++i) {
    p[i - 1] = nullptr;
    ld[i - 1] = 0;
    if (a[i] == Py_None) continue;
    const at::Tensor& t = tensor(a[i]);
    if (t.scalar_type() != at::kBFloat16 || !on_device(t, device)) return false;
    if (i < 5 ? !matrix(t, i == 1 ? M : *samples, D) : t.dim() != 1 || t.size(0) != D || (t.stride(0) != 1 && D > 1)) return false;
    p[i - 1] = t.data_ptr();
    ld[i - 1] = i < 5 ? leading(t) : 0;
  }
  op->branch_bf16 = p[0], op->ldb = ld[0];
  op->gate_bf16 = p[1], op->ld_gate = ld[1];
  op->shift_bf16 = p[2], op->ld_shift = ld[2];
  op->scale_bf16 = p[3], op->ld_scale = ld[3];
  op->weight_bf16 = p[4];
  op->post_weight_bf16 = p[5];
  return true;
}
// an output [M, D] of a norm call that may be given, with its row stride
bool norm_output(PyObject* o, const trdq_gated_norm_op& op, at::ScalarType type, c10::DeviceIndex device, int64_t* ld) {
  *ld = op.D;
  if (o == Py_None) return true;
  if (!plain(o) || !on_device(tensor(o), device) || tensor(o).scalar_type() != type || !matrix(tensor(o), op.M, op.D)) return false;
  *ld = leading(tensor(o));
  return true;
}

// (the shared twelve, resid, out)
PyObject* gated_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  trdq_gated_norm_op op;
  int64_t samples, ldr, ldh;
  c10::DeviceIndex device;
  GENERAL_WAY_UNLESS(n == kNormArgs + 2 && norm_op(a, &device, &op, &samples) && no_modes());
  const at::ScalarType type = op.stream_f32 ? at::kFloat : at::kBFloat16;
  GENERAL_WAY_UNLESS(norm_output(a[12], op, type, device, &ldr) && norm_output(a[13], op, at::kBFloat16, device, &ldh));
  Outputs out(a[0]);
  out.add(a[12], op.M, op.D, type);
  out.add(a[13], op.M, op.D, at::kBFloat16);
  void* const s = stream();
  return out.run([&](void** o) { return block_entry.gated_norm(&op, o[0], ldr, o[1], ldh, s); });
  END_HANDLE_TH_ERRORS
}

// (the shared twelve, rot or None, t, resid, codes, scales)
PyObject* gated_norm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  trdq_gated_norm_op op;
  int64_t samples, ldr, ldc;
  void* rot;
  int32_t t;
  c10::DeviceIndex device;
  GENERAL_WAY_UNLESS(n == kNormArgs + 5 && norm_op(a, &device, &op, &samples) && handle_or_none(a[12], &rot) && number(a[13], &t) && no_modes());
  const at::ScalarType type = op.stream_f32 ? at::kFloat : at::kBFloat16;
  GENERAL_WAY_UNLESS(norm_output(a[14], op, type, device, &ldr) && norm_output(a[15], op, at::kFloat8_e4m3fn, device, &ldc) && ldc == op.D);
  GENERAL_WAY_UNLESS(a[16] == Py_None || (plain(a[16]) && on_device(tensor(a[16]), device) && tensor(a[16]).scalar_type() == at::kFloat &&
                                          whole(tensor(a[16]), op.D / 128, op.M)));
  Outputs out(a[0]);
  out.add(a[14], op.M, op.D, type);
  out.add(a[15], op.M, op.D, at::kFloat8_e4m3fn);
  out.add(a[16], op.D / 128, op.M, at::kFloat);
  void* const s = stream();
  return out.run([&](void** o) {
    return block_entry.gated_norm_fp8(&op, static_cast<trdq_rotation*>(rot), t, o[0], ldr, static_cast<uint8_t*>(o[1]), static_cast<float*>(o[2]), s);
  });
  END_HANDLE_TH_ERRORS
}

// (the shared twelve, dH, dR or None): dx, db, dgate, dshift, dscale, dweight, dpost_weight, None where there is no such input
PyObject* gated_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  trdq_gated_norm_op op;
  int64_t samples, lddh, lddr;
  c10::DeviceIndex device;
  GENERAL_WAY_UNLESS(n == kNormArgs + 2 && norm_op(a, &device, &op, &samples) && no_modes());
  const at::ScalarType type = op.stream_f32 ? at::kFloat : at::kBFloat16;
  GENERAL_WAY_UNLESS(a[12] != Py_None && norm_output(a[12], op, at::kBFloat16, device, &lddh) && norm_output(a[13], op, type, device, &lddr));
  uint64_t bytes = 0;
  bool wanted[7] = {true};  // (a tensor without elements has a null address: what is given decides)
  for (int i = 1; i < 7; ++i) wanted[i] = a[i] != Py_None;
  GENERAL_WAY_UNLESS(block_entry.gated_norm_backward_workspace(&op, &bytes) == TRDQ_OK);
  void *const dh = pointer(a[12]), *const dr = pointer(a[13]);
  const at::Device where = tensor(a[0]).device();
  void* const s = stream();
  at::Tensor made[7];
  trdq_status st;
  {
    WithoutGil released;
    at::Tensor workspace;
    const bool sums = wanted[2] || wanted[3] || wanted[4] || wanted[5] || wanted[6];
    if (sums) workspace = new_tensor({static_cast<int64_t>(bytes > 16 ? bytes : 16)}, at::kByte, where);
    for (int i = 0; i < 7; ++i) {
      if (!wanted[i]) continue;
      const int64_t rows = i < 2 ? op.M : samples;
      const at::ScalarType o = i == 0 ? type : i == 1 ? at::kBFloat16 : at::kFloat;
      made[i] = i < 5 ? new_tensor({rows, op.D}, o, where) : new_tensor({op.D}, o, where);
    }
    auto at_ = [&](int i) { return wanted[i] ? static_cast<float*>(made[i].data_ptr()) : nullptr; };
    st = block_entry.gated_norm_backward(&op, dh, lddh, dr, dr ? lddr : 0, at_(0), op.D, at_(1), op.D, at_(2), at_(3), at_(4), at_(5), at_(6),
                                         sums ? workspace.data_ptr() : nullptr, sums ? static_cast<uint64_t>(workspace.numel()) : 0, s);
  }
  if (st != TRDQ_OK) return PyLong_FromLong(st);
  PyObject* const r = PyTuple_New(7);
  if (!r) return nullptr;
  for (int i = 0; i < 7; ++i) {
    PyObject* o = Py_None;
    if (wanted[i]) {
      o = THPVariable_Wrap(std::move(made[i]));
      if (!o) {
        Py_DECREF(r);
        return nullptr;
      }
    } else {
      Py_INCREF(o);
    }
    PyTuple_SET_ITEM(r, i, o);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// (addresses of the library's functions, in the order of BlockEntry)
PyObject* bind_block(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* address[7];
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "seven addresses");
    return nullptr;
  }
  for (int i = 0; i < 7; ++i) {
    address[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  block_entry = {reinterpret_cast<decltype(block_entry.fp8_quantize)>(address[0]),   reinterpret_cast<decltype(block_entry.fp8_quantize_weights)>(address[1]),
                 reinterpret_cast<decltype(block_entry.fp8_linear)>(address[2]),     reinterpret_cast<decltype(block_entry.gated_norm)>(address[3]),
                 reinterpret_cast<decltype(block_entry.gated_norm_fp8)>(address[4]), reinterpret_cast<decltype(block_entry.gated_norm_backward_workspace)>(address[5]),
                 reinterpret_cast<decltype(block_entry.gated_norm_backward)>(address[6])};
  Py_RETURN_NONE;
}

// (addresses of the library's functions, in the order of Entry)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* address[8];
  if (n != 8) {
    PyErr_SetString(PyExc_TypeError, "eight addresses");
    return nullptr;
  }
  for (int i = 0; i < 8; ++i) {
    address[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  entry = {reinterpret_cast<decltype(entry.rotate_quantize)>(address[0]),      reinterpret_cast<decltype(entry.norm_rotate_quantize)>(address[1]),
           reinterpret_cast<decltype(entry.rotate_quantize_asym)>(address[2]), reinterpret_cast<decltype(entry.linear_act)>(address[3]),
           reinterpret_cast<decltype(entry.linear_cfg)>(address[4]),           reinterpret_cast<decltype(entry.linear_asym)>(address[5]),
           reinterpret_cast<decltype(entry.splitk_workspace)>(address[6]),     reinterpret_cast<decltype(entry.linear_splitk)>(address[7])};
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),        METHOD(rotate_quantize), METHOD(norm_rotate_quantize), METHOD(rotate_quantize_asym), METHOD(linear),
                         METHOD(linear_asym), METHOD(linear_splitk),   METHOD(linear_cfg),           METHOD(bind_block),
                         METHOD(fp8_quantize), METHOD(fp8_linear),      METHOD(gated_norm),           METHOD(gated_norm_fp8),       METHOD(gated_norm_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
