// The feed-forward operators on torch tensors: checks, results from torch's allocator, and the call of the C ABI, whose
// functions are handed over as addresses by the package's loader (no link between this module and the library).  In C++ because a
// small call's time is the host's: the same steps in Python take 9 to 14 us beside a kernel of 2 to 5.
#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <string>

#include "../../include/xema.h"

namespace {
using at::Tensor;
constexpr auto kBf16 = at::kBFloat16, kF32 = at::kFloat, kI32 = at::kInt, kI16 = at::kShort;
constexpr auto kE4m3 = at::kFloat8_e4m3fn;

struct Functions {
  int (*rms_norm)(const xema_rms_norm_args*, void*);
  int (*gated_ffn)(const xema_gated_ffn_args*, void*, void*);
  int (*gated_ffn_grad)(const xema_gated_ffn_grad_args*, void*, void*);
  int (*lora)(const xema_lora_args*, void*, void*);
  uint64_t (*lora_work_bytes)(int32_t, int32_t, int32_t);
} fn;

[[noreturn]] void refuse(const std::string& what) {
  TORCH_CHECK_VALUE(false, what);
  __builtin_unreachable();
}
void need(bool ok, const char* what) {
  if (!ok) refuse(what);
}
bool given(PyObject* o) { return o && o != Py_None; }

// The tensor behind `o`, on device `index` (or any CUDA device: -1), of this type and rank.  Operators whose results would have to carry
// a gradient on (`recorded`) take none that requires one while gradients are on: the loss would run backward without them.
const Tensor& tensor(PyObject* o, const char* name, at::ScalarType type, int64_t rank, int index, bool recorded = true) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": want a tensor");
  const Tensor& t = THPVariable_Unpack(o);
  if (recorded && t.requires_grad() && c10::GradMode::is_enabled())
    refuse(std::string(name) + ": requires a gradient, which the result would not carry on: call under torch.no_grad() (gated_ffn_backward has gated_ffn's gradients)");
  if (!t.is_cuda() || (index >= 0 && t.get_device() != index))
    refuse(std::string(name) + (index >= 0 ? ": want it on the device of the other tensors" : ": want tensors on a CUDA device (there is no CPU fallback)"));
  if (t.scalar_type() != type) refuse(std::string(name) + ": want " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  if (t.dim() != rank) refuse(std::string(name) + ": want " + std::to_string(rank) + " dimensions");
  if (rank > 0 && t.size(rank - 1) > 1 && t.stride(rank - 1) != 1) refuse(std::string(name) + ": the last dimension has to be contiguous");
  if (t._fw_grad(0).defined()) refuse(std::string(name) + ": carries a forward-mode derivative, which the result would not carry on");
  if (t.numel() > 0 && (!t.has_storage() || !t.storage().data())) refuse(std::string(name) + ": a tensor of this kind has no memory");
  return t;
}
void sized(const Tensor& t, const char* name, at::IntArrayRef want) {
  if (t.sizes() != want) {
    std::string s;
    for (int64_t n : want) s += (s.empty() ? "" : ", ") + std::to_string(n);
    refuse(std::string(name) + ": want shape [" + s + "]");
  }
}
int32_t i32(int64_t v, const char* name) {
  if (v > 0x7fffffff) refuse(std::string(name) + ": too large");
  return (int32_t)v;
}
Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const Tensor& like) {
  return at::empty(sizes, like.options().dtype(type).memory_format(c10::nullopt).requires_grad(false));
}
void* address(const Tensor& t) { return t.data_ptr(); }
void* stream_of(int index) { return c10::cuda::getCurrentCUDAStream(index).stream(); }
PyObject* wrap(const Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
// A tuple of the tensors, or the library's status where it refused.
template <int N>
PyObject* answer(int rc, const Tensor (&t)[N]) {
  if (rc) return PyLong_FromLong(rc);
  if (N == 1) return wrap(t[0]);
  PyObject* out = PyTuple_New(N);
  for (int i = 0; out && i < N; ++i) PyTuple_SET_ITEM(out, i, wrap(t[i]));
  return out;
}
// At the head of each operator.
void argc(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) refuse("wrong number of arguments");
  if (torch::jit::tracer::isTracing() || c10::impl::TorchDispatchModeTLS::get_mode(c10::impl::TorchDispatchModeKey::PROXY).has_value())
    refuse("this operator cannot be traced: the traced program would hold the result of this call");
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();      // (the exception that is set)
  return v;
}
double number(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse(std::string(name) + ": want a number");
  }
  return v;
}

// rms_norm(x, gain, residual, eps, out_is_e4m3, out, residual_out) -> (out, scale, residual_out)
PyObject* rms_norm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  argc(n, 7);
  need(THPVariable_Check(v[0]), "x: want a tensor");
  const bool has_resid = given(v[2]), alone = !has_resid && THPVariable_Unpack(v[0]).scalar_type() == kF32;
  const Tensor& x = tensor(v[0], "x", alone ? kF32 : kBf16, 2, -1);
  const int index = x.get_device();
  const int64_t rows = x.size(0), D = x.size(1);
  xema_rms_norm_args a = {};
  a.rows = i32(rows, "x");
  a.D = i32(D, "x");
  a.eps = (float)number(v[3], "eps");
  if (alone) {
    a.resid = address(x);
    a.ldr = x.stride(0);
    a.resid_is_f32 = 1;
  } else {
    a.x = address(x);
    a.ldx = x.stride(0);
  }
  auto resid_type = kBf16;
  if (has_resid) {
    need(THPVariable_Check(v[2]), "residual: want a tensor");
    if (THPVariable_Unpack(v[2]).scalar_type() == kF32) resid_type = kF32;
    const Tensor& r = tensor(v[2], "residual", resid_type, 2, index);
    sized(r, "residual", {rows, D});
    a.resid = address(r);
    a.ldr = r.stride(0);
    a.resid_is_f32 = resid_type == kF32;
  }
  const Tensor& gain = tensor(v[1], "gain", kBf16, 1, index);
  sized(gain, "gain", {D});
  a.gain = address(gain);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
  a.out_is_e4m3 = truth(v[4]);
  Tensor t[3];
  if (given(v[5])) {
    t[0] = tensor(v[5], "out", a.out_is_e4m3 ? kE4m3 : kBf16, 2, index);
    sized(t[0], "out", {rows, D});
  } else {
    t[0] = fresh({rows, D}, a.out_is_e4m3 ? kE4m3 : kBf16, x);
  }
  a.out = address(t[0]);
  a.ldo = t[0].stride(0);
  if (a.out_is_e4m3) {
    t[1] = fresh({rows}, kF32, x);
    a.out_scale = static_cast<float*>(address(t[1]));
  }
  if (given(v[6])) {
    need(has_resid, "residual_out: there is no residual");
    t[2] = tensor(v[6], "residual_out", resid_type, 2, index);
    sized(t[2], "residual_out", {rows, D});
  } else if (has_resid) {
    t[2] = fresh({rows, D}, resid_type, x);
  }
  if (has_resid) {
    a.resid_out = address(t[2]);
    a.ldro = t[2].stride(0);
  }
  return answer(fn.rms_norm(&a, stream_of(index)), t);
  END_HANDLE_TH_ERRORS
}

struct Weights {
  const void *gate, *up;
  int64_t ffn, ld;
};
Weights weights(PyObject* g, PyObject* u, at::ScalarType type, int64_t width, int index, bool recorded = true) {
  const Tensor &gate = tensor(g, "w_gate", type, 2, index, recorded), &up = tensor(u, "w_up", type, 2, index, recorded);
  sized(gate, "w_gate", {gate.size(0), width});
  sized(up, "w_up", {gate.size(0), width});
  const bool one = gate.size(0) == 1;
  need(one || gate.stride(0) == up.stride(0), "w_gate and w_up: want the same row stride");
  return {address(gate), address(up), gate.size(0), one ? width : gate.stride(0)};
}

// gated_ffn(x, w_gate, w_up, activation, x_scale, gate_scale, up_scale, out, save, status) -> h or (h, saved)
PyObject* gated_ffn(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  argc(n, 10);
  need(THPVariable_Check(v[0]), "x: want a tensor");
  const bool e4m3 = THPVariable_Unpack(v[0]).scalar_type() == kE4m3;
  const auto type = e4m3 ? kE4m3 : kBf16;
  const Tensor& x = tensor(v[0], "x", type, 2, -1);
  const int index = x.get_device();
  const int64_t rows = x.size(0), width = x.size(1);
  const Weights w = weights(v[1], v[2], type, width, index);
  xema_gated_ffn_args a = {};
  a.x = address(x);
  a.ldx = x.stride(0);
  a.w_gate = w.gate;
  a.w_up = w.up;
  a.ldw = w.ld;
  a.rows = i32(rows, "x");
  a.width = i32(width, "x");
  a.ffn = i32(w.ffn, "w_gate");
  a.activation = (int)PyLong_AsLong(v[3]);
  a.is_e4m3 = e4m3;
  const bool save = truth(v[8]);
  if (e4m3) {
    need(!save, "save: gradients are for bf16 operands");
    const Tensor &sx = tensor(v[4], "x_scale", kF32, 1, index), &sg = tensor(v[5], "gate_scale", kF32, 1, index),
                 &su = tensor(v[6], "up_scale", kF32, 1, index);
    sized(sx, "x_scale", {rows});
    sized(sg, "gate_scale", {w.ffn});
    sized(su, "up_scale", {w.ffn});
    a.x_scale = static_cast<const float*>(address(sx));
    a.gate_scale = static_cast<const float*>(address(sg));
    a.up_scale = static_cast<const float*>(address(su));
  } else {
    need(!given(v[4]) && !given(v[5]) && !given(v[6]), "scales: for e4m3 operands only");
  }
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
  Tensor t[2];
  if (given(v[7])) {
    t[0] = tensor(v[7], "out", kBf16, 2, index);
    sized(t[0], "out", {rows, w.ffn});
  } else {
    t[0] = fresh({rows, w.ffn}, kBf16, x);
  }
  a.h = address(t[0]);
  a.ldh = t[0].stride(0);
  if (save) {
    t[1] = fresh({3, rows, w.ffn}, kI16, x);
    a.z = address(t[1]);
  }
  const int rc = fn.gated_ffn(&a, PyLong_AsVoidPtr(v[9]), stream_of(index));
  if (save) return answer(rc, t);
  const Tensor h[1] = {t[0]};
  return answer(rc, h);
  END_HANDLE_TH_ERRORS
}

// gated_ffn_backward(dh, x, w_gate, w_up, saved, activation, want_x, want_weights, reuse_saved, status) -> (dx, dw_gate, dw_up)
PyObject* gated_ffn_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  argc(n, 10);
  const Tensor& x = tensor(v[1], "x", kBf16, 2, -1, false);
  const int index = x.get_device();
  const int64_t rows = x.size(0), width = x.size(1);
  const Weights w = weights(v[2], v[3], kBf16, width, index, false);
  const Tensor& dh = tensor(v[0], "dh", kBf16, 2, index, false);
  sized(dh, "dh", {rows, w.ffn});
  const Tensor& saved = tensor(v[4], "saved", kI16, 3, index, false);
  sized(saved, "saved", {3, rows, w.ffn});
  need(saved.is_contiguous(), "saved: want it as gated_ffn gave it");
  xema_gated_ffn_grad_args a = {};
  a.dh = address(dh);
  a.lddh = dh.stride(0);
  a.x = address(x);
  a.ldx = x.stride(0);
  a.w_gate = w.gate;
  a.w_up = w.up;
  a.ldw = w.ld;
  a.z = address(saved);
  a.rows = i32(rows, "x");
  a.width = i32(width, "x");
  a.ffn = i32(w.ffn, "w_gate");
  a.activation = (int)PyLong_AsLong(v[5]);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
  const Tensor work = truth(v[8]) ? saved : fresh({2, rows, w.ffn}, kBf16, x);
  a.work = address(work);
  Tensor t[3];
  if (truth(v[6])) {
    t[0] = fresh({rows, width}, kBf16, x);
    a.dx = address(t[0]);
    a.lddx = width;
  }
  if (truth(v[7])) {
    t[1] = fresh({w.ffn, width}, kBf16, x);
    t[2] = fresh({w.ffn, width}, kBf16, x);
    a.dw_gate = address(t[1]);
    a.dw_up = address(t[2]);
    a.lddw = width;
  }
  return answer(fn.gated_ffn_grad(&a, PyLong_AsVoidPtr(v[9]), stream_of(index)), t);
  END_HANDLE_TH_ERRORS
}

// row stride, and rows from one batch element to the next, of [batch, rows, features]
void strides_of(const Tensor& t, const char* name, int64_t* ld, int64_t* batch_rows) {
  const int64_t batch = t.size(0), rows = t.size(1);
  *batch_rows = rows;
  *ld = t.size(2);
  if (rows == 1) {
    *batch_rows = 1;
    if (batch > 1) *ld = t.stride(0);
    return;
  }
  *ld = t.stride(1);
  if (batch <= 1) return;
  if (*ld <= 0 || t.stride(0) % *ld) refuse(std::string(name) + ": the batch stride has to be a multiple of the row stride");
  *batch_rows = t.stride(0) / *ld;
}

// lora_linear(x, weight, lora_a, lora_b, scale, adapter, bias, out, status) -> out
PyObject* lora_linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  argc(n, 9);
  const Tensor& x = tensor(v[0], "x", kBf16, 3, -1);
  const int index = x.get_device();
  const int64_t batch = x.size(0), rows = x.size(1), K = x.size(2);
  const Tensor &w = tensor(v[1], "weight", kBf16, 2, index), &la = tensor(v[2], "lora_a", kBf16, 3, index), &lb = tensor(v[3], "lora_b", kBf16, 3, index);
  const int64_t N = w.size(0), adapters = la.size(0), rank = la.size(1);
  sized(w, "weight", {N, K});
  sized(la, "lora_a", {adapters, rank, K});
  sized(lb, "lora_b", {adapters, N, rank});
  need(la.is_contiguous() && lb.is_contiguous(), "lora_a and lora_b: want contiguous tensors");
  const Tensor &scale = tensor(v[4], "scale", kF32, 1, index), &adapter = tensor(v[5], "adapter", kI32, 1, index);
  sized(scale, "scale", {adapters});
  sized(adapter, "adapter", {batch});
  xema_lora_args a = {};
  a.x = address(x);
  strides_of(x, "x", &a.ldx, &a.x_batch_rows);
  a.w = address(w);
  a.ldw = N > 1 ? w.stride(0) : K;
  if (given(v[6])) {
    const Tensor& bias = tensor(v[6], "bias", kBf16, 1, index);
    sized(bias, "bias", {N});
    a.bias = address(bias);
  }
  a.lora_a = address(la);
  a.lora_b = address(lb);
  a.scale = static_cast<const float*>(address(scale));
  a.adapter = static_cast<const int32_t*>(address(adapter));
  a.batch = i32(batch, "x");
  a.rows = i32(rows, "x");
  a.N = i32(N, "weight");
  a.K = i32(K, "x");
  a.rank = i32(rank, "lora_a");
  a.n_adapters = i32(adapters, "lora_a");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
  Tensor t[1];
  if (given(v[7])) {
    t[0] = tensor(v[7], "out", kBf16, 3, index);
    sized(t[0], "out", {batch, rows, N});
  } else {
    t[0] = fresh({batch, rows, N}, kBf16, x);
  }
  a.out = address(t[0]);
  strides_of(t[0], "out", &a.ldo, &a.out_batch_rows);
  const Tensor work = fresh({(int64_t)fn.lora_work_bytes(a.batch, a.rows, a.rank)}, at::kByte, x);
  a.work = address(work);
  return answer(fn.lora(&a, PyLong_AsVoidPtr(v[8]), stream_of(index)), t);
  END_HANDLE_TH_ERRORS
}

// bind(addresses of the C functions, in the order of Functions)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  argc(n, 5);
  fn.rms_norm = reinterpret_cast<decltype(fn.rms_norm)>(PyLong_AsVoidPtr(v[0]));
  fn.gated_ffn = reinterpret_cast<decltype(fn.gated_ffn)>(PyLong_AsVoidPtr(v[1]));
  fn.gated_ffn_grad = reinterpret_cast<decltype(fn.gated_ffn_grad)>(PyLong_AsVoidPtr(v[2]));
  fn.lora = reinterpret_cast<decltype(fn.lora)>(PyLong_AsVoidPtr(v[3]));
  fn.lora_work_bytes = reinterpret_cast<decltype(fn.lora_work_bytes)>(PyLong_AsVoidPtr(v[4]));
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
    {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rms_norm)), METH_FASTCALL, nullptr},
    {"gated_ffn", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gated_ffn)), METH_FASTCALL, nullptr},
    {"gated_ffn_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gated_ffn_backward)), METH_FASTCALL, nullptr},
    {"lora_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(lora_linear)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__torch_ops(void) { return PyModule_Create(&module); }
