// The Python binding's way into libnvfp4.so: a call takes tensors, rounding descriptors and numbers as they are and makes the
// C entry point's arguments of them.  A small call is bound by the host, and fetching the arguments one by one in Python and
// passing them through ctypes took 2.7 us of its 6 (three calls on kept weights: 18.4 -> 14.2 us, a 256-token step's two 29.1 -> 22.9).
//
// Argument rules, by what the C parameter is:
//   pointer       a tensor or another object with data_ptr(), or None; the FP8 and expert calls take tensors of the current device
//                 only (the kernels run there, on its current stream), the others take their caller's word for it
//   rounding      a Rounding (the class that bind() was given), or None
//   dtype         an int, or a tensor (its dtype as an nvfp4_dtype): the parameters that NVFP4_CALLS lists
//   size_t        an int, or a tensor (its number of elements): the size of the buffer before it
//   int, int64    an int; a tensor in its place is a misplaced argument and refused
// The last parameter of every entry point is the stream: a torch.cuda.Stream, or None for the current stream.
//
// The outputs that a caller of the FP8 and expert calls does not give are made here too: torch.empty and a slice from Python take 2.6 and
// 1.1 us each, which for four of them is more than the launch (quantizing both ways 24 -> 10 us of host time).
//
// Memory for a call that is given a stream is allocated on that stream (OnStream below): the allocator hands a block out again in the
// order of the stream that it was allocated on, so that one of the current stream's could still be written by work queued there
// earlier, or be given away while the call's kernels use it.  Every output that is dropped then costs the host an event on the current
// stream, about 2 us (one output 7.6 -> 9.2 us a call, four 7.1 -> 16.2); a caller who gives the outputs, or makes the stream the current
// one, does not pay that.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <optional>
#include <tuple>
#include <type_traits>
#include <utility>

#include "nvfp4.h"

namespace {

// Thrown with the Python error set.
struct PythonError {};

[[noreturn]] void type_error(const char* expected, PyObject* got) {
  PyErr_Format(PyExc_TypeError, "expected %s, got %s", expected, Py_TYPE(got)->tp_name);
  throw PythonError{};
}

PyTypeObject* rounding_type = nullptr;             // binding.py's Rounding, a ctypes.Structure laid out as nvfp4_rounding

// The struct is read on the host: nothing but a Rounding will do.
const nvfp4_rounding* convert_rounding(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!PyObject_TypeCheck(o, rounding_type)) type_error("a Rounding", o);
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError{};
  void* const p = view.buf;                        // the object outlives the call: the caller holds it
  PyBuffer_Release(&view);
  return static_cast<const nvfp4_rounding*>(p);
}

// HERE: a tensor has to be on the current device.
template <bool HERE, typename T>
T convert_pointer(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (HERE && !(t.is_cuda() && t.device().index() == c10::cuda::current_device())) {
      PyErr_Format(PyExc_ValueError, "expected a tensor on the current CUDA device, got one on %s", t.device().str().c_str());
      throw PythonError{};
    }
    return static_cast<T>(t.data_ptr());
  }
  if (!PyObject_HasAttrString(o, "data_ptr")) type_error("a tensor or None", o);
  PyObject* const address = PyObject_CallMethod(o, "data_ptr", nullptr);   // a storage, say
  if (!address) throw PythonError{};
  void* const p = PyLong_AsVoidPtr(address);
  Py_DECREF(address);
  if (!p && PyErr_Occurred()) throw PythonError{};
  return static_cast<T>(p);
}

template <typename T, bool DTYPE>
T convert_number(PyObject* o) {
  if constexpr (DTYPE || std::is_same_v<T, size_t>) {
    if (THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if constexpr (!DTYPE) return (T)t.numel();
      if (t.scalar_type() == at::kBFloat16) return (T)NVFP4_BF16;
      if (t.scalar_type() == at::kFloat) return (T)NVFP4_FP32;
      PyErr_Format(PyExc_TypeError, "unsupported dtype %s", c10::toString(t.scalar_type()));
      throw PythonError{};
    }
  }
  if (!PyLong_Check(o)) type_error("an int", o);
  if constexpr (std::is_same_v<T, size_t>) {
    const size_t v = PyLong_AsSize_t(o);
    if (v == (size_t)-1 && PyErr_Occurred()) throw PythonError{};
    return v;
  }
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  if constexpr (std::is_same_v<T, int>) {
    if (v != (int)v) {
      PyErr_SetString(PyExc_OverflowError, "argument out of the range of int");
      throw PythonError{};
    }
  }
  return (T)v;
}

void* stream_handle(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* const handle = PyObject_GetAttrString(o, "cuda_stream");
  if (!handle) throw PythonError{};
  void* const p = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (!p && PyErr_Occurred()) throw PythonError{};
  return p;
}

template <size_t... S>
constexpr bool one_of(size_t i) { return ((i == S) || ...); }

// DTYPES: the positions of the dtype parameters.
template <bool HERE, size_t... DTYPES, typename... A, size_t... I>
PyObject* call(int (*f)(A...), PyObject* const* args, std::index_sequence<I...>) {
  constexpr size_t kLast = sizeof...(A) - 1;
  std::tuple<A...> a{[&]() -> A {
    if constexpr (I == kLast) return stream_handle(args[I]);
    else if constexpr (std::is_same_v<A, const nvfp4_rounding*>) return convert_rounding(args[I]);
    else if constexpr (std::is_pointer_v<A>) return convert_pointer<HERE, A>(args[I]);
    else return convert_number<A, one_of<DTYPES...>(I)>(args[I]);
  }()...};
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = std::apply(f, a);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

template <bool HERE, size_t... DTYPES, typename... A>
PyObject* checked_call(int (*f)(A...), PyObject* const* args, Py_ssize_t n) {
  if (!f) {
    PyErr_SetString(PyExc_RuntimeError, "bind() first");
    return nullptr;
  }
  if (n != (Py_ssize_t)sizeof...(A)) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", (Py_ssize_t)sizeof...(A), n);
    return nullptr;
  }
  try {
    return call<HERE, DTYPES...>(f, args, std::index_sequence_for<A...>{});
  } catch (const PythonError&) {
    return nullptr;
  } catch (const std::exception& e) {              // torch's own checks (a tensor without storage, no GPU)
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// The entry points, each with the positions of its dtype parameters.
#define NVFP4_CALLS(X)                                                                                                      \
  X(nvfp4_quantize, 1) X(nvfp4_quantize_dual, 1) X(nvfp4_quantize_mx, 1) X(nvfp4_tensor_amax_scale, 1) X(nvfp4_gemm, 10)    \
  X(nvfp4_gemm_quantized) X(nvfp4_gemm_mx, 10) X(nvfp4_gemm_bf16, 6) X(nvfp4_gemm_bf16_ex, 8) X(nvfp4_linear_fwd, 2, 12)    \
  X(nvfp4_linear_bwd_dx, 2, 12) X(nvfp4_linear_bwd_dw, 2, 12) X(nvfp4_linear_fwd_qout, 2) X(nvfp4_linear_fwd_qin, 4, 12)    \
  X(nvfp4_linear_fwd_save, 2, 14) X(nvfp4_linear_bwd_saved, 1, 12, 14) X(nvfp4_linear_bwd, 3, 16, 18)                       \
  X(nvfp4_linear_bwd_bf16, 7, 9) X(nvfp4_linear_fwd_static, 2, 12)
#define NVFP4_CALLS_HERE(X)                                                                                                 \
  X(nvfp4_quantize_fp8, 1) X(nvfp4_gemm_fp8, 8) X(nvfp4_linear_fp8_fwd, 2, 7) X(nvfp4_linear_fp8_bwd, 3, 8, 10)             \
  X(nvfp4_expert_sort) X(nvfp4_expert_gather, 1, 11) X(nvfp4_expert_combine, 1, 8) X(nvfp4_expert_combine_bwd, 1, 12)       \
  X(nvfp4_quantize_fp8_experts, 1, 11) X(nvfp4_gemm_fp8_experts, 12) X(nvfp4_gemm_fp8_experts_dw, 11)                       \
  X(nvfp4_experts_fp8_fwd, 3, 12) X(nvfp4_experts_fp8_bwd, 3, 7, 16, 18)

#define NVFP4_WRAPPER(name, ...)                                                       \
  decltype(&::name) fn_##name = nullptr;                                               \
  PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t n) { return checked_call<kHere __VA_OPT__(,) __VA_ARGS__>(fn_##name, args, n); }
namespace any_device {
constexpr bool kHere = false;
NVFP4_CALLS(NVFP4_WRAPPER)
}  // namespace any_device
namespace this_device {
constexpr bool kHere = true;
NVFP4_CALLS_HERE(NVFP4_WRAPPER)
}  // namespace this_device
using namespace any_device;
using namespace this_device;

// ---- outputs on the device of a given tensor ----
PyObject* wrap(const at::Tensor& t) {
  PyObject* const o = THPVariable_Wrap(t);
  if (!o) throw PythonError{};
  return o;
}
at::Tensor empty(const at::Tensor& like, at::IntArrayRef size, at::ScalarType type) { return at::empty(size, like.options().dtype(type)); }

// While it lives, memory on the device of `like` is allocated on the given stream (None: on the current one).  leave(t): t goes to the
// caller, who may use it on the stream that is current now, in the order of that stream, and drop it.
class OnStream {
 public:
  OnStream(PyObject* stream, const at::Tensor& like) {
    if (stream == Py_None || !like.is_cuda()) return;
    const c10::DeviceIndex device = like.device().index();
    const c10::cuda::CUDAStream here = c10::cuda::getCurrentCUDAStream(device);
    const cudaStream_t handle = static_cast<cudaStream_t>(stream_handle(stream));
    if (handle == here.stream()) return;
    before_ = here;
    guard_.emplace(handle ? c10::cuda::getStreamFromExternal(handle, device) : c10::cuda::getDefaultCUDAStream(device));
  }
  void leave(const at::Tensor& t) const {
    if (before_ && t.defined()) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), *before_);
  }

 private:
  std::optional<c10::cuda::CUDAStream> before_;
  std::optional<c10::cuda::CUDAStreamGuard> guard_;
};
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) type_error("a tensor", o);
  return THPVariable_Unpack(o);
}
int64_t number(PyObject* o) { return convert_number<int64_t, false>(o); }

// The results of f as a tuple; null with the Python error set.
template <typename F>
PyObject* tuple_of(F&& f) {
  PyObject* made[4] = {};
  int n = 0;
  try {
    n = f(made);
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  PyObject* const t = n ? PyTuple_New(n) : nullptr;
  for (int i = 0; i < 4; ++i) {
    if (t && i < n) PyTuple_SET_ITEM(t, i, made[i] ? made[i] : Py_NewRef(Py_None));
    else Py_XDECREF(made[i]);
  }
  return t;
}

// Codes and scales of both outputs of a quantizer: [batch, rows, cols] and [batch, cols, rows] without the first dimension where batch
// is 0.  Rows of codes take a multiple of 16 bytes.
void make_fp8(const at::Tensor& like, int64_t batch, int64_t rows, int64_t cols, const bool (&wanted)[2], int64_t layout, at::Tensor (&out)[4]) {
  const int64_t size[2] = {rows, cols}, lead = batch ? batch : 1;
  for (int i = 0; i < 2; ++i) {
    if (!wanted[i]) continue;
    const int64_t rq = size[i], kq = size[1 - i], pitch = (kq + 15) / 16 * 16, nb = (kq + 127) / 128;
    const int64_t whole[3] = {lead, rq, pitch}, part[3] = {lead, rq, kq}, strides[3] = {rq * pitch, pitch, 1}, linear[3] = {lead, rq, nb};
    const int skip = batch ? 0 : 1;
    at::Tensor& codes = out[2 * i] = empty(like, at::IntArrayRef(whole).slice(skip), at::kByte);
    if (pitch != kq) codes.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef(part).slice(skip), at::IntArrayRef(strides).slice(skip));
    out[2 * i + 1] = layout == NVFP4_SF_LINEAR ? empty(like, at::IntArrayRef(linear).slice(skip), at::kByte)
                                               : empty(like, {lead * ((rq + 127) / 128) * ((nb + 3) / 4) * 512}, at::kByte);
  }
}
int wrap_all(const at::Tensor (&out)[4], PyObject** made) {
  for (int i = 0; i < 4; ++i)
    if (out[i].defined()) made[i] = wrap(out[i]);
  return 4;
}

// Each of the functions that make outputs takes the stream of the call last, or not at all.
bool has_arguments(Py_ssize_t n, Py_ssize_t expected) {
  if (n == expected || n == expected + 1) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, and a stream or None", expected);
  return false;
}
PyObject* last(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected) { return n > expected ? args[expected] : Py_None; }

// empty_fp8(like, batch, rows, cols, row, transposed, sf_layout): (codes, scales, codes_t, scales_t), None for what is not wanted.
PyObject* py_empty_fp8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!has_arguments(n, 7)) return nullptr;
  return tuple_of([&](PyObject** made) {
    const bool wanted[2] = {number(args[4]) != 0, number(args[5]) != 0};
    at::Tensor out[4];
    const OnStream on(last(args, n, 7), tensor(args[0]));
    make_fp8(tensor(args[0]), number(args[1]), number(args[2]), number(args[3]), wanted, number(args[6]), out);
    for (const at::Tensor& t : out) on.leave(t);
    return wrap_all(out, made);
  });
}
// quantize_fp8(x, block_rows, row, transposed, sf_layout, stream): nvfp4_quantize_fp8 of [rows, cols] or of a dense [batch, rows, cols], with
// outputs as above; or the status that it returned.
PyObject* py_quantize_fp8(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6 || !fn_nvfp4_quantize_fp8) {
    PyErr_SetString(PyExc_TypeError, "expected 6 arguments, after bind()");
    return nullptr;
  }
  int st = 0;
  PyObject* const made = tuple_of([&](PyObject** made) {
    const at::Tensor& x = tensor(args[0]);
    const int64_t d = x.dim();
    const void* const data = convert_pointer<true, const void*>(args[0]);
    if ((d != 2 && d != 3) || x.stride(d - 1) != 1 || (d == 3 && !x.is_contiguous())) {
      PyErr_SetString(PyExc_ValueError, "expected [rows, cols] with dense rows, or a dense [batch, rows, cols]");
      throw PythonError{};
    }
    const int dtype = convert_number<int, true>(args[0]);
    const int64_t batch = d == 3 ? x.size(0) : 0, rows = x.size(d - 2), cols = x.size(d - 1);
    const int block_rows = convert_number<int, false>(args[1]), layout = convert_number<int, false>(args[4]);
    const bool wanted[2] = {number(args[2]) != 0, number(args[3]) != 0};
    // one row alone has no leading dimension to speak of; matrices of one row lie one behind the other
    const int64_t ld = rows * std::max<int64_t>(batch, 1) == 1 ? (cols + 7) / 8 * 8 : d == 3 ? cols : x.stride(0);
    void* const stream = stream_handle(args[5]);
    at::Tensor out[4];
    const OnStream on(args[5], x);
    make_fp8(x, batch, rows, cols, wanted, layout, out);
    for (const at::Tensor& t : out) on.leave(t);
    uint8_t* to[4];
    for (int i = 0; i < 4; ++i) to[i] = out[i].defined() ? static_cast<uint8_t*>(out[i].data_ptr()) : nullptr;
    Py_BEGIN_ALLOW_THREADS
    st = fn_nvfp4_quantize_fp8(data, dtype, d == 3 ? batch : 1, rows, cols, ld, block_rows, to[0], to[1], to[2], to[3], layout, stream);
    Py_END_ALLOW_THREADS
    return wrap_all(out, made);
  });
  if (made && st != 0) {
    Py_DECREF(made);
    return PyLong_FromLong(st);
  }
  return made;
}
// expert_buffers(like, tokens, topk, experts, rows): (counts, offsets, row_of, slot_of)
PyObject* py_expert_buffers(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!has_arguments(n, 5)) return nullptr;
  return tuple_of([&](PyObject** made) {
    const at::Tensor& like = tensor(args[0]);
    const int64_t tokens = number(args[1]), topk = number(args[2]), experts = number(args[3]), rows = number(args[4]);
    const OnStream on(last(args, n, 5), like);
    // one buffer; a tensor of its own for each would cost a microsecond
    const at::Tensor buffer = empty(like, {rows + tokens * topk + 2 * experts + 1}, at::kInt);
    on.leave(buffer);
    int64_t at = 0;
    auto part = [&](std::initializer_list<int64_t> size, int64_t n) {
      at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buffer.storage()), buffer.key_set(), buffer.dtype());
      t.unsafeGetTensorImpl()->set_storage_offset(at);
      t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
      at += n;
      return wrap(t);
    };
    made[3] = part({rows}, rows);
    made[2] = part({tokens, topk}, tokens * topk);
    made[1] = part({experts + 1}, experts + 1);
    made[0] = part({experts}, experts);
    return 4;
  });
}
// matrix(t, rows): (cols, leading dimension) of [rows, cols] whose rows are dense
PyObject* py_matrix(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "expected 2 arguments");
    return nullptr;
  }
  try {
    const at::Tensor& t = tensor(args[0]);
    const int64_t rows = number(args[1]);
    if (t.dim() != 2 || t.stride(1) != 1 || t.size(0) != rows) {
      PyErr_Format(PyExc_ValueError, "expected a matrix of %lld dense rows", (long long)rows);
      return nullptr;
    }
    return Py_BuildValue("(LL)", (long long)t.size(1), (long long)(rows > 1 ? t.stride(0) : (t.size(1) + 7) / 8 * 8));
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// dense(t, like, size...): whether t is contiguous, of that size, and of the dtype of `like` (None: of any)
PyObject* py_dense(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 2) {
    PyErr_SetString(PyExc_TypeError, "expected a tensor, another or None, and sizes");
    return nullptr;
  }
  try {
    const at::Tensor& t = tensor(args[0]);
    bool yes = t.dim() == n - 2 && t.is_contiguous() && (args[1] == Py_None || t.scalar_type() == tensor(args[1]).scalar_type());
    for (Py_ssize_t i = 2; yes && i < n; ++i) yes = t.size(i - 2) == number(args[i]);
    return PyBool_FromLong(yes);
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// empty_rows(like, rows, cols): [rows, cols] of like's dtype
PyObject* py_empty_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (!has_arguments(n, 3)) return nullptr;
  try {
    const at::Tensor& like = tensor(args[0]);
    const OnStream on(last(args, n, 3), like);
    const at::Tensor t = empty(like, {number(args[1]), number(args[2])}, like.scalar_type());
    on.leave(t);
    return wrap(t);
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// empty_on(stream, like, dtype, leaves, size...): on like's device; leaves: it goes to the caller of the call that uses it
PyObject* py_empty_on(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t kFixed = 4, kMostDims = 4;
  if (n <= kFixed || n > kFixed + kMostDims || !THPDtype_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "expected a stream or None, a tensor, a dtype, a number and sizes");
    return nullptr;
  }
  try {
    int64_t size[kMostDims];
    for (Py_ssize_t i = kFixed; i < n; ++i) size[i - kFixed] = number(args[i]);
    const bool leaves = number(args[3]) != 0;
    const at::Tensor& like = tensor(args[1]);
    const OnStream on(args[0], like);
    const at::Tensor t = empty(like, at::IntArrayRef(size, n - kFixed), reinterpret_cast<THPDtype*>(args[2])->scalar_type);
    if (leaves) on.leave(t);
    return wrap(t);
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// fp8_operand(codes, scales): (matrices, Rq, Kq) of codes as the quantizer leaves them, with swizzled scales: flat, or in rows of whole
// tiles.  Buffers that are too small are refused, since the products would read behind them, and so are linear scales, whose rows are a
// byte for each block: they may have just as many bytes.
PyObject* py_fp8_operand(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "expected 2 arguments");
    return nullptr;
  }
  try {
    const at::Tensor &codes = tensor(args[0]), &scales = tensor(args[1]);
    const int64_t d = codes.dim();
    if ((d != 2 && d != 3) || codes.element_size() != 1) {
      PyErr_SetString(PyExc_ValueError, "FP8 codes have one byte each and two or three dimensions");
      return nullptr;
    }
    const int64_t b = d == 3 ? codes.size(0) : 1, rq = codes.size(d - 2), kq = codes.size(d - 1), pitch = (kq + 15) / 16 * 16;
    if (codes.stride(d - 1) != 1 || (rq > 1 && codes.stride(d - 2) != pitch) || (b > 1 && codes.stride(0) != rq * pitch)) {
      PyErr_SetString(PyExc_ValueError, "rows of FP8 codes take a multiple of 16 bytes and lie one behind the other");
      return nullptr;
    }
    const int64_t nb = (kq + 127) / 128, tiles = b * ((rq + 127) / 128) * ((nb + 3) / 4), sd = scales.dim();
    const bool in_tiles = sd == 1 || (sd > 1 && scales.size(sd - 1) % 512 == 0 && scales.size(sd - 1) != nb);
    if (scales.element_size() != 1 || !scales.is_contiguous() || !in_tiles || scales.numel() < tiles * 512) {
      PyErr_SetString(PyExc_ValueError, "FP8 codes come with swizzled scales, in whole tiles of 512 bytes");
      return nullptr;
    }
    return Py_BuildValue("(LLL)", (long long)b, (long long)rq, (long long)kq);
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(path, Rounding): takes the entry points from the library at `path`, and the class of the rounding descriptors.
PyObject* py_bind(PyObject*, PyObject* args) {
  const char* file;
  PyObject* rounding;
  if (!PyArg_ParseTuple(args, "sO!", &file, &PyType_Type, &rounding)) return nullptr;
  if (reinterpret_cast<PyTypeObject*>(rounding) != rounding_type) {
    Py_XDECREF(rounding_type);
    rounding_type = reinterpret_cast<PyTypeObject*>(Py_NewRef(rounding));
  }
  void* const lib = dlopen(file, RTLD_NOW | RTLD_LOCAL);
  if (!lib) {
    PyErr_SetString(PyExc_OSError, dlerror());
    return nullptr;
  }
  bool all = true;
#define NVFP4_BIND(name, ...) all = (fn_##name = reinterpret_cast<decltype(&::name)>(dlsym(lib, #name))) && all;
  NVFP4_CALLS(NVFP4_BIND) NVFP4_CALLS_HERE(NVFP4_BIND)
  if (!all) {
    PyErr_Format(PyExc_OSError, "%s lacks entry points", file);
    return nullptr;
  }
  Py_RETURN_NONE;
}

#define NVFP4_METHOD(name, ...) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr},
#define NVFP4_HELPER(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", py_bind, METH_VARARGS, nullptr}, NVFP4_HELPER(empty_fp8), NVFP4_HELPER(expert_buffers), NVFP4_HELPER(empty_rows),
                         NVFP4_HELPER(empty_on), NVFP4_HELPER(fp8_operand), NVFP4_HELPER(quantize_fp8), NVFP4_HELPER(matrix), NVFP4_HELPER(dense),
                         NVFP4_CALLS(NVFP4_METHOD) NVFP4_CALLS_HERE(NVFP4_METHOD){nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
