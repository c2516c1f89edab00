// The Python side of the calls around the attention (norm, quantising, product, rotary positions) in C++: argument checks,
// outputs, streams, and the call of the C ABI.  An answer makes these calls several times per layer and token, and in Python
// the checks and allocations took three times as long as the kernels.
//
// The module knows libcrisp.so by the addresses that bind() is given; nothing is computed here.
#include <Python.h>

#include <climits>
#include <optional>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/crisp.h"

namespace {

using at::Tensor;

decltype(&crisp_quantize) quantize_fn;
decltype(&crisp_rms_norm) rms_norm_fn;
decltype(&crisp_matmul) matmul_fn;
decltype(&crisp_rotary) rotary_fn;
PyObject* crisp_error;   // called with (status, function) for the exception to raise

constexpr auto kCodes = at::kFloat8_e4m3fn, kScales = at::kFloat8_e8m0fnu, kBf16 = at::kBFloat16, kInt = at::kInt;
constexpr int64_t kHead = 128;

struct Raised {};   // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* format, const char* a = "", const char* b = "") {
  PyErr_Format(type, format, a, b);
  throw Raised();
}

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}

const char* type_name(at::ScalarType t) {
  return t == kCodes ? "float8_e4m3fn" : t == kScales ? "float8_e8m0fnu" : t == kInt ? "int32" : "bfloat16";
}

// Place of a CUDA tensor.
int place(const Tensor& t, const char* name) {
  if (!t.is_cuda()) raise(PyExc_RuntimeError, "%s must be a CUDA tensor (no CPU fallback)", name);
  return t.get_device();
}

// A matrix of that type.
int matrix(const Tensor& t, const char* name, at::ScalarType type) {
  const int index = place(t, name);
  if (t.dim() != 2 || t.scalar_type() != type || !t.is_contiguous())
    raise(PyExc_ValueError, "%s must be a contiguous %s matrix", name, type_name(type));
  return index;
}

// The pointer of a contiguous tensor of that type, place and shape.
void* checked(const Tensor& t, const char* name, at::ScalarType type, int index, at::IntArrayRef shape) {
  if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != index || !t.is_contiguous())
    raise(PyExc_ValueError, "%s must be a contiguous %s tensor on the same device", name, type_name(type));
  if (t.sizes() != shape) raise(PyExc_ValueError, "%s has the wrong shape", name);
  return t.data_ptr();
}

int size32(int64_t n, const char* name) {
  if (n > INT_MAX) raise(PyExc_ValueError, "%s is too large", name);
  return static_cast<int>(n);
}

int int32(PyObject* o, const char* name) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  if (v < INT_MIN || v > INT_MAX) raise(PyExc_ValueError, "%s must be an int32", name);
  return static_cast<int>(v);
}

// The stream of a call: None is the device's current one, an int a handle (0: the default stream), anything else a
// torch.cuda.Stream.  Outputs are allocated on it, and tensors that a call uses are recorded with it (nothing happens where they
// were allocated on it), so that their memory is not handed out again before the call has run.
struct Where {
  c10::cuda::OptionalCUDAGuard device;
  c10::cuda::OptionalCUDAStreamGuard guard;
  std::optional<c10::cuda::CUDAStream> stream;
  cudaStream_t raw;

  Where(PyObject* o, int index) {
    if (o == Py_None) {
      device.set_index(static_cast<c10::DeviceIndex>(index));
      stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(index));
      raw = stream->stream();
      return;
    }
    if (PyLong_Check(o)) {
      void* handle = PyLong_AsVoidPtr(o);
      if (!handle && PyErr_Occurred()) throw Raised();
      stream = handle ? c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), static_cast<c10::DeviceIndex>(index))
                      : c10::cuda::getDefaultCUDAStream(static_cast<c10::DeviceIndex>(index));
    } else {
      const long long id = field(o, "stream_id"), at = field(o, "device_index"), type = field(o, "device_type");
      stream = c10::cuda::CUDAStream::unpack3(id, static_cast<c10::DeviceIndex>(at), static_cast<c10::DeviceType>(type));
    }
    if (stream->device_index() != index) raise(PyExc_ValueError, "the stream must be of the tensors' device");
    guard.reset_stream(*stream);
    raw = stream->stream();
  }
  static long long field(PyObject* stream, const char* name) {
    PyObject* v = PyObject_GetAttrString(stream, name);
    if (!v) throw Raised();
    const long long n = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (n == -1 && PyErr_Occurred()) throw Raised();
    return n;
  }
  void used(std::initializer_list<const Tensor*> tensors) const {
    for (const Tensor* t : tensors)
      if (t && t->defined()) record(*t, *stream);
  }
  static void record(const Tensor& t, c10::cuda::CUDAStream stream) {
    c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), stream);
  }
};

Tensor fresh(at::IntArrayRef shape, at::ScalarType type, int index) {
  return Tensor(at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(index)), std::nullopt));
}

void done(int status, const char* function) {
  if (status == CRISP_OK) return;
  PyObject* e = PyObject_CallFunction(crisp_error, "is", status, function);
  if (e) {
    PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e)), e);
    Py_DECREF(e);
  }
  throw Raised();
}

int64_t scale_cols(int64_t cols) { return (cols + 511) / 512 * 4; }

PyObject* tuple(std::initializer_list<const Tensor*> tensors) {
  PyObject* t = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
  if (!t) throw Raised();
  Py_ssize_t i = 0;
  for (const Tensor* x : tensors) {
    PyObject* o = x && x->defined() ? THPVariable_Wrap(*x) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(t);
      throw Raised();
    }
    PyTuple_SET_ITEM(t, i++, o);
  }
  return t;
}

template <Py_ssize_t kArgs, typename F>
PyObject* guarded(Py_ssize_t n, F body) {
  HANDLE_TH_ERRORS
  if (n != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// quantize(x, stream) -> (codes, scales)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<2>(n, [&] {
    const Tensor& x = tensor(a[0], "x");
    const int index = matrix(x, "x", kBf16);
    const int rows = size32(x.size(0), "x"), cols = size32(x.size(1), "x");
    const Where where(a[1], index);
    const Tensor codes = fresh({rows, cols}, kCodes, index), scales = fresh({rows, scale_cols(cols)}, kScales, index);
    done(quantize_fn(x.data_ptr(), rows, cols, codes.data_ptr(), static_cast<uint8_t*>(scales.data_ptr()), where.raw), "crisp_quantize");
    where.used({&x});
    return tuple({&codes, &scales});
  });
}

// rms_norm(x, weight, residual, eps, sum_out, quantized, stream) -> (y, h) or (codes, scales, h)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(n, [&] {
    const Tensor& x = tensor(a[0], "x");
    const int index = matrix(x, "x", kBf16);
    const int rows = size32(x.size(0), "x"), cols = size32(x.size(1), "x");
    const Tensor none;
    const Tensor& weight = a[1] == Py_None ? none : tensor(a[1], "weight");
    const Tensor& residual = a[2] == Py_None ? none : tensor(a[2], "residual");
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw Raised();
    Tensor h = a[4] == Py_None ? none : tensor(a[4], "sum_out");
    const bool quantized = a[5] == Py_True;
    const void* w = weight.defined() ? checked(weight, "weight", kBf16, index, {cols}) : nullptr;
    const void* r = residual.defined() ? checked(residual, "residual", kBf16, index, x.sizes()) : nullptr;
    if (h.defined()) {
      if (!residual.defined()) raise(PyExc_ValueError, "sum_out belongs to a residual");
      checked(h, "sum_out", kBf16, index, x.sizes());
    }
    const Where where(a[6], index);
    if (residual.defined() && !h.defined()) h = fresh({rows, cols}, kBf16, index);
    const Tensor y = fresh({rows, cols}, quantized ? kCodes : kBf16, index);
    const Tensor scales = quantized ? fresh({rows, scale_cols(cols)}, kScales, index) : none;
    done(rms_norm_fn(x.data_ptr(), r, w, rows, cols, static_cast<float>(eps), h.defined() ? h.data_ptr() : nullptr,
                     quantized ? nullptr : y.data_ptr(), quantized ? y.data_ptr() : nullptr,
                     quantized ? static_cast<uint8_t*>(scales.data_ptr()) : nullptr, where.raw),
         "crisp_rms_norm");
    where.used({&x, &weight, &residual, a[4] != Py_None ? &h : nullptr});
    return quantized ? tuple({&y, &scales, &h}) : tuple({&y, &h});
  });
}

// matmul(codes, scales, w_codes, w_scales, ws, out, stream) -> out; the weights and the workspace are checked already
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(n, [&] {
    const Tensor &codes = tensor(a[0], "codes"), &scales = tensor(a[1], "scales"), &w_codes = tensor(a[2], "w_codes"),
                 &w_scales = tensor(a[3], "w_scales"), &ws = tensor(a[4], "ws");
    const int index = matrix(codes, "codes", kCodes);
    const int rows = size32(codes.size(0), "codes"), cols = size32(codes.size(1), "codes"), n_out = size32(w_codes.size(0), "weights");
    if (cols != w_codes.size(1) || index != w_codes.get_device())
      raise(PyExc_ValueError, "codes must have the weights' columns and be on their device");
    const void* s = checked(scales, "scales", kScales, index, {rows, scale_cols(cols)});
    Tensor out;
    if (a[5] != Py_None) {
      out = tensor(a[5], "out");
      checked(out, "out", kBf16, index, {rows, n_out});
    }
    const Where where(a[6], index);
    if (!out.defined()) out = fresh({rows, n_out}, kBf16, index);
    done(matmul_fn(codes.data_ptr(), static_cast<const uint8_t*>(s), w_codes.data_ptr(), static_cast<const uint8_t*>(w_scales.data_ptr()),
                   rows, n_out, cols, out.data_ptr(), ws.data_ptr(), static_cast<size_t>(ws.numel()), where.raw),
         "crisp_matmul");
    where.used({&codes, &scales, a[5] != Py_None ? &out : nullptr});
    if (a[6] != Py_None) where.used({&w_codes, &w_scales, &ws});   // (the weights' object outlives its calls on the current stream)
    return a[5] != Py_None ? Py_NewRef(a[5]) : THPVariable_Wrap(out);
  });
}

// The positions' pointer, or null.
const int32_t* positions_of(const Tensor& t, int index, int rows) {
  return t.defined() ? static_cast<const int32_t*>(checked(t, "positions", kInt, index, {rows})) : nullptr;
}

// rotary_split(plan, qkv, n_q_heads, n_kv_heads, positions, first_position, stream) -> (q, k, v)
PyObject* rotary_split(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<7>(n, [&] {
    const auto* plan = static_cast<const crisp_rotary_plan*>(PyLong_AsVoidPtr(a[0]));
    const Tensor& qkv = tensor(a[1], "qkv");
    const int index = place(qkv, "qkv"), hq = int32(a[2], "n_q_heads"), hkv = int32(a[3], "n_kv_heads");
    if (hq <= 0 || hkv <= 0 || hq > 65535 || hkv > 65535) raise(PyExc_ValueError, "there must be 1 to 65535 heads");
    const int64_t width = (hq + 2LL * hkv) * kHead;
    if (qkv.dim() != 2 || qkv.scalar_type() != kBf16 || qkv.size(1) != width || qkv.stride(1) != 1)
      raise(PyExc_ValueError, "qkv must be bf16 [tokens, (n_q_heads + 2 n_kv_heads) 128] with contiguous rows");
    const int rows = size32(qkv.size(0), "qkv");
    const Tensor none;
    const Tensor& positions = a[4] == Py_None ? none : tensor(a[4], "positions");
    const int32_t* pos = positions_of(positions, index, rows);
    const int first = int32(a[5], "first_position");
    const Where where(a[6], index);
    const Tensor q = fresh({rows, hq, kHead}, kBf16, index), k = fresh({rows, hkv, kHead}, kBf16, index),
                 v = fresh({rows, hkv, kHead}, kBf16, index);
    if (rows > 0) {
      const int64_t row = rows > 1 ? qkv.stride(0) : width;
      const char* at = static_cast<const char*>(qkv.data_ptr());
      const char *at_k = at + 2 * kHead * hq, *at_v = at_k + 2 * kHead * hkv;
      done(rotary_fn(plan, rows, pos, first, hq, hkv, at, row, at_k, row, at_v, row, q.data_ptr(), k.data_ptr(), v.data_ptr(), where.raw),
           "crisp_rotary");
      where.used({&qkv, &positions});
    }
    return tuple({&q, &k, &v});
  });
}

// rotary_rotate(plan, x, positions, first_position, out, stream) -> out
PyObject* rotary_rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<6>(n, [&] {
    const auto* plan = static_cast<const crisp_rotary_plan*>(PyLong_AsVoidPtr(a[0]));
    const Tensor& x = tensor(a[1], "x");
    const int index = place(x, "x");
    if (x.dim() != 3 || x.scalar_type() != kBf16 || x.size(1) < 1 || x.size(1) > 65535 || x.size(2) != kHead || x.stride(2) != 1 ||
        (x.size(1) > 1 && x.stride(1) != kHead))
      raise(PyExc_ValueError, "x must be bf16 [tokens, heads, 128] with contiguous tokens");
    const int rows = size32(x.size(0), "x"), heads = static_cast<int>(x.size(1));
    const Tensor none;
    const Tensor& positions = a[2] == Py_None ? none : tensor(a[2], "positions");
    const int32_t* pos = positions_of(positions, index, rows);
    const int first = int32(a[3], "first_position");
    Tensor out;
    if (a[4] != Py_None) {
      out = tensor(a[4], "out");
      checked(out, "out", kBf16, index, x.sizes());
    }
    const Where where(a[5], index);
    if (!out.defined()) out = fresh(x.sizes(), kBf16, index);
    if (rows > 0) {
      done(rotary_fn(plan, rows, pos, first, heads, 0, x.data_ptr(), rows > 1 ? x.stride(0) : heads * kHead, nullptr, 0, nullptr, 0,
                     out.data_ptr(), nullptr, nullptr, where.raw),
           "crisp_rotary");
      where.used({&x, &positions, a[4] != Py_None ? &out : nullptr});
    }
    return a[4] != Py_None ? Py_NewRef(a[4]) : THPVariable_Wrap(out);
  });
}

// used(device, tensors...): a call on the device's current stream uses these tensors (or None), as in Where
PyObject* used(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<0>(n > 0 ? 0 : -1, [&] {
    const auto stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(int32(a[0], "device")));
    for (Py_ssize_t i = 1; i < n; ++i)
      if (a[i] != Py_None) Where::record(tensor(a[i], "a tensor given to the call"), stream);
    return Py_NewRef(Py_None);
  });
}

// bind(error, quantize, rms_norm, matmul, rotary): the exception's maker and the addresses of the C calls
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<5>(n, [&] {
    void* at[4];
    for (int i = 0; i < 4; ++i) {
      at[i] = PyLong_AsVoidPtr(a[i + 1]);
      if (!at[i]) raise(PyErr_Occurred() ? PyErr_Occurred() : PyExc_ValueError, "bind: not an address");
    }
    Py_XSETREF(crisp_error, Py_NewRef(a[0]));
    quantize_fn = reinterpret_cast<decltype(quantize_fn)>(at[0]);
    rms_norm_fn = reinterpret_cast<decltype(rms_norm_fn)>(at[1]);
    matmul_fn = reinterpret_cast<decltype(matmul_fn)>(at[2]);
    rotary_fn = reinterpret_cast<decltype(rotary_fn)>(at[3]);
    return Py_NewRef(Py_None);
  });
}

#define CRISP_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CRISP_CALL(bind),   CRISP_CALL(quantize),     CRISP_CALL(rms_norm),
                         CRISP_CALL(matmul), CRISP_CALL(rotary_split), CRISP_CALL(rotary_rotate), CRISP_CALL(used),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "The calls around the attention.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
