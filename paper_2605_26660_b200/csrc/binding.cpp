// Argument marshalling of the feed-forward calls, compiled.  Their kernels for a few tokens take 2 to 15 us, and a call through
// Python's checks, allocations and conversions of a dozen arguments 10 to 12; here it takes 4.5, of which a launch is 2.6.  Nothing is
// computed: every function checks its tensors, allocates the outputs it is not given, and calls the C ABI.
//
// A function takes (handle, device, stream or None, ...) and returns a tuple whose first item is the status; wrong types raise
// TypeError, wrong shapes ValueError, before anything is launched.  The interpreter lock is released while memory is allocated and the
// library runs.
#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "windq.h"

namespace {

using at::Tensor;

int code_of(at::ScalarType t) { return t == at::kHalf ? WINDQ_F16 : t == at::kBFloat16 ? WINDQ_BF16 : -1; }

const Tensor& tensor_of(PyObject* o, const char* name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor");
  return THPVariable_Unpack(o);
}
void on_device(const Tensor& t, int device, const char* name) {
  TORCH_CHECK_TYPE(t.is_cuda(), name, " must be a CUDA tensor");
  TORCH_CHECK_VALUE(t.get_device() == device, name, " is on device ", t.get_device(), ", not on the context's, ", device);
}

struct Rows {
  void* p = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  at::ScalarType type{};
};
int64_t up(int64_t x, int64_t step) { return (x + step - 1) / step * step; }

// A row-major matrix whose rows are `step` elements, or a multiple of that, apart (the library checks that).
Rows rows_of(const Tensor& t, at::ScalarType type, int device, int64_t step, const char* name) {
  TORCH_CHECK_TYPE(t.scalar_type() == type, name, " must be ", type, ", got ", t.scalar_type());
  on_device(t, device, name);
  TORCH_CHECK_VALUE(t.dim() == 2, name, " must have 2 dimensions");
  Rows r;
  r.rows = t.size(0);
  r.cols = t.size(1);
  TORCH_CHECK_VALUE(r.cols <= 1 || t.stride(1) == 1, name, " must be row-major (unit stride along columns)");
  r.ld = r.rows > 1 ? t.stride(0) : up(r.cols, step);  // the stride of a single row means nothing, and torch may report any
  r.p = t.data_ptr();
  r.type = type;
  return r;
}
Rows half_of(const Tensor& t, int device, const char* name) {
  TORCH_CHECK_TYPE(code_of(t.scalar_type()) >= 0, name, " must be torch.float16 or torch.bfloat16, got ", t.scalar_type());
  return rows_of(t, t.scalar_type(), device, 8, name);
}
// Gives the interpreter lock to other threads for as long as it lives: a launch waits where the stream's queue is full, an allocation for
// the device, and what the stream waits for may be another Python thread's to do.  No Python object is touched meanwhile.
class Unlocked {
  PyThreadState* state_ = PyEval_SaveThread();

 public:
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(state_); }
};
template <class F, class... A>
windq_status unlocked(F call, const A&... arguments) {
  const Unlocked others;
  return call(arguments...);
}
struct Call {
  windq_ctx* ctx;
  int device;
  void* stream;
  bool given;  // the stream, by the caller
  Call(PyObject* const* a)
      : ctx(reinterpret_cast<windq_ctx*>(a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]))), device((int)PyLong_AsLong(a[1])), given(a[2] != Py_None) {
    if (!given) {
      stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    } else {  // a torch.cuda.Stream
      PyObject* handle = PyObject_GetAttrString(a[2], "cuda_stream");
      if (!handle) throw python_error();
      stream = PyLong_AsVoidPtr(handle);
      Py_DECREF(handle);
    }
    if (PyErr_Occurred()) throw python_error();
  }
};

// A new tensor in memory of its own, straight from torch's allocator (through the dispatcher, with a view where rows are padded, a call
// takes 1 to 3 us more; through a tensor of bytes 0.1 each), and of the stream that writes it: memory of the current stream's pool may
// still be in use there when another stream comes to it.
Tensor fresh(int64_t bytes, const Call& c, at::ScalarType type, at::IntArrayRef sizes, at::IntArrayRef strides) {
  const Unlocked others;
  const c10::cuda::CUDAGuard on((c10::DeviceIndex)c.device);
  c10::cuda::OptionalCUDAStreamGuard stream;
  if (c.given) stream.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(c.stream), (c10::DeviceIndex)c.device));
  c10::Storage memory(c10::Storage::use_byte_size_t(), bytes, c10::cuda::CUDACachingAllocator::get(), /*resizable=*/true);
  Tensor t = at::detail::make_tensor<c10::TensorImpl>(std::move(memory), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                      c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_sizes_and_strides(sizes, strides);
  return t;
}
int64_t row_length(int64_t cols, int64_t size) { return cols * size % 32 == 0 ? cols : up(cols, 128 / size); }

// A caller's [rows, cols] output, or a new one.  Rows of a new one that are no multiple of 32 bytes are padded to one of 128: copies
// of rows that begin in the middle of 32 bytes take up to a third longer (500 tokens x 2 x 5000 x 5000 70 us, x 5056 57).  A new DENSE
// one is padded only where the library wants its rows apart.
template <bool DENSE = false>
Rows rows_out(PyObject* given, Tensor& t, int64_t rows, int64_t cols, at::ScalarType type, const Call& c, int64_t step, const char* name) {
  if (given == Py_None) {
    const int64_t size = (int64_t)c10::elementSize(type), ld = DENSE && cols % step == 0 ? cols : row_length(cols, size);
    t = fresh(rows * ld * size, c, type, {rows, cols}, {ld, 1});
    return Rows{t.data_ptr(), rows, cols, ld, type};
  }
  t = tensor_of(given, name);
  const Rows r = rows_of(t, type, c.device, step, name);
  TORCH_CHECK_VALUE(r.rows == rows && r.cols == cols, name, " must be a [", rows, ", ", cols, "] tensor");
  return r;
}
float* scales_of(const Tensor& t, int64_t n, int device, const char* name) {
  TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat, name, " must be torch.float32, got ", t.scalar_type());
  on_device(t, device, name);
  TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == n && t.is_contiguous(), name, " must be a contiguous [", n, "] tensor");
  return static_cast<float*>(t.data_ptr());
}
at::ScalarType out_type(PyObject* dtype, PyObject* out) {
  at::ScalarType type;
  if (out != Py_None) {
    type = tensor_of(out, "out").scalar_type();
  } else {
    TORCH_CHECK_TYPE(THPDtype_Check(dtype), "dtype must be a torch.dtype");
    type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
  }
  TORCH_CHECK_TYPE(code_of(type) >= 0, "the output must be torch.float16 or torch.bfloat16, got ", type);
  return type;
}

bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw python_error();
  return t != 0;
}
PyObject* wrapped(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
template <class... T>
PyObject* result(windq_status st, const T&... tensors) {
  PyObject* r = PyTuple_New(1 + sizeof...(tensors));
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, PyLong_FromLong(st));
  Py_ssize_t k = 1;
  (PyTuple_SET_ITEM(r, k++, wrapped(tensors)), ...);
  return r;
}
#define WINDQ_ARGUMENTS(count)                                                  \
  HANDLE_TH_ERRORS                                                              \
  TORCH_CHECK_TYPE(n == (count), "expected ", (count), " arguments, got ", n);  \
  const Call c(a)

// X, want_values, codes, scale, values
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  WINDQ_ARGUMENTS(8);
  const Rows x = half_of(tensor_of(a[3], "X"), c.device, "X");
  Tensor codes, scale, values;
  // Memory of its own for each: who keeps or saves a weight's scales does not keep its codes with them.
  const Rows q = rows_out(a[5], codes, x.rows, x.cols, at::kChar, c, 16, "codes");
  if (a[6] == Py_None) scale = fresh(4 * x.rows, c, at::kFloat, {x.rows}, {1});
  else scale = tensor_of(a[6], "scale");
  Rows v;
  if (truth(a[4])) v = rows_out(a[7], values, x.rows, x.cols, x.type, c, 8, "values");
  return result(unlocked(windq_quantize_rows, c.ctx, code_of(x.type), x.p, x.rows, x.cols, x.ld, static_cast<int8_t*>(q.p), q.ld,
                                    scales_of(scale, x.rows, c.device, "scale"), v.p, v.ld, c.stream),
                codes, scale, values);
  END_HANDLE_TH_ERRORS
}

// codes, scale, w_codes, w_scale, dtype, out
PyObject* int8_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  WINDQ_ARGUMENTS(9);
  const Rows x = rows_of(tensor_of(a[3], "codes"), at::kChar, c.device, 16, "codes");
  const Rows w = rows_of(tensor_of(a[5], "w_codes"), at::kChar, c.device, 16, "w_codes");
  TORCH_CHECK_VALUE(w.cols == x.cols, "codes have ", x.cols, " columns, w_codes ", w.cols);
  const float* sx = scales_of(tensor_of(a[4], "scale"), x.rows, c.device, "scale");
  const float* sw = scales_of(tensor_of(a[6], "w_scale"), w.rows, c.device, "w_scale");
  Tensor out;
  const Rows y = rows_out(a[8], out, x.rows, w.rows, out_type(a[7], a[8]), c, 8, "out");
  return result(unlocked(windq_int8_forward, c.ctx, static_cast<int8_t*>(x.p), x.rows, x.cols, x.ld, sx, static_cast<int8_t*>(w.p), w.rows, w.ld, sw,
                                   code_of(y.type), y.p, y.ld, c.stream),
                out);
  END_HANDLE_TH_ERRORS
}

// codes, scale, wg_codes, wg_scale, wu_codes, wu_scale, activation, dtype, out
PyObject* gated_int8_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  WINDQ_ARGUMENTS(12);
  const Rows x = rows_of(tensor_of(a[3], "codes"), at::kChar, c.device, 16, "codes");
  const Rows g = rows_of(tensor_of(a[5], "wg_codes"), at::kChar, c.device, 16, "wg_codes");
  const Rows u = rows_of(tensor_of(a[7], "wu_codes"), at::kChar, c.device, 16, "wu_codes");
  TORCH_CHECK_VALUE(g.cols == x.cols && u.cols == x.cols && g.rows == u.rows, "shapes do not fit: codes [T, C], wg_codes and wu_codes [F, C]");
  const float* sx = scales_of(tensor_of(a[4], "scale"), x.rows, c.device, "scale");
  const float* sg = scales_of(tensor_of(a[6], "wg_scale"), g.rows, c.device, "wg_scale");
  const float* su = scales_of(tensor_of(a[8], "wu_scale"), g.rows, c.device, "wu_scale");
  const int act = (int)PyLong_AsLong(a[9]);
  if (PyErr_Occurred()) throw python_error();
  Tensor out;
  const Rows h = rows_out(a[11], out, x.rows, g.rows, out_type(a[10], a[11]), c, 8, "out");
  return result(unlocked(windq_gated_int8_forward, c.ctx, act, static_cast<int8_t*>(x.p), x.rows, x.cols, x.ld, sx, static_cast<int8_t*>(g.p), g.ld, sg,
                                         static_cast<int8_t*>(u.p), u.ld, su, g.rows, code_of(h.type), h.p, h.ld, c.stream),
                out);
  END_HANDLE_TH_ERRORS
}

struct Gated {
  Rows x, g, u;
  Gated(PyObject* const* a, int device) : x(half_of(tensor_of(a[0], "X"), device, "X")) {
    g = rows_of(tensor_of(a[1], "Wg"), x.type, device, 8, "Wg");
    u = rows_of(tensor_of(a[2], "Wu"), x.type, device, 8, "Wu");
    TORCH_CHECK_VALUE(g.cols == x.cols && u.cols == x.cols && g.rows == u.rows, "shapes do not fit: X [T, C], Wg and Wu [F, C]");
  }
};

// X, Wg, Wu, activation, want_saved, h, gate, up
PyObject* gated_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  WINDQ_ARGUMENTS(11);
  const Gated q(a + 3, c.device);
  const int act = (int)PyLong_AsLong(a[6]);
  if (PyErr_Occurred()) throw python_error();
  const int64_t T = q.x.rows, F = q.g.rows;
  Tensor h, gate, up_;
  const Rows o = rows_out(a[8], h, T, F, q.x.type, c, 8, "h");
  Rows g, u;
  if (truth(a[7])) {
    g = rows_out(a[9], gate, T, F, q.x.type, c, 8, "gate");
    u = rows_out(a[10], up_, T, F, q.x.type, c, 8, "up");
    TORCH_CHECK_VALUE(g.ld == u.ld, "gate and up must have the same stride between rows");
  }
  return result(unlocked(windq_gated_forward, c.ctx, code_of(q.x.type), act, q.x.p, T, q.x.cols, q.x.ld, q.g.p, q.g.ld, q.u.p, q.u.ld, F, o.p, o.ld, g.p,
                                    u.p, g.ld, c.stream),
                h, gate, up_);
  END_HANDLE_TH_ERRORS
}

// X, Wg, Wu, activation, dH, gate, up, want_dx, want_dw, dx, dWg, dWu
PyObject* gated_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  WINDQ_ARGUMENTS(15);
  const Gated q(a + 3, c.device);
  const int act = (int)PyLong_AsLong(a[6]);
  if (PyErr_Occurred()) throw python_error();
  const int64_t T = q.x.rows, F = q.g.rows, C = q.x.cols;
  const Rows dh = rows_of(tensor_of(a[7], "dH"), q.x.type, c.device, 8, "dH");
  TORCH_CHECK_VALUE(dh.rows == T && dh.cols == F, "dH must be a [", T, ", ", F, "] tensor");
  TORCH_CHECK_VALUE((a[8] == Py_None) == (a[9] == Py_None), "gate and up must be given together");
  Rows g, u, dx, dg, du;
  if (a[8] != Py_None) {
    g = rows_of(tensor_of(a[8], "gate"), q.x.type, c.device, 8, "gate");
    u = rows_of(tensor_of(a[9], "up"), q.x.type, c.device, 8, "up");
    TORCH_CHECK_VALUE(g.rows == T && g.cols == F && u.rows == T && u.cols == F && g.ld == u.ld, "gate and up must be [", T, ", ", F,
                      "] tensors with the same stride between rows");
  }
  Tensor dX, dWg, dWu;
  if (truth(a[10])) dx = rows_out(a[12], dX, T, C, q.x.type, c, 8, "dx");
  if (truth(a[11])) {
    dg = rows_out<true>(a[13], dWg, F, C, q.x.type, c, 8, "dWg");  // the optimiser takes contiguous gradients
    du = rows_out<true>(a[14], dWu, F, C, q.x.type, c, 8, "dWu");
    TORCH_CHECK_VALUE(dg.ld == du.ld, "dWg and dWu must have the same stride between rows");
  }
  return result(unlocked(windq_gated_backward, c.ctx, code_of(q.x.type), act, q.x.p, T, C, q.x.ld, q.g.p, q.g.ld, q.u.p, q.u.ld, F, g.p, u.p, g.ld, dh.p,
                                     dh.ld, dx.p, dx.ld, dg.p, du.p, dg.ld, c.stream),
                dX, dWg, dWu);
  END_HANDLE_TH_ERRORS
}

#define WINDQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {WINDQ_METHOD(quantize_rows),  WINDQ_METHOD(int8_forward),   WINDQ_METHOD(gated_int8_forward),
                         WINDQ_METHOD(gated_forward), WINDQ_METHOD(gated_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
