// Python entry points of the C ABI for torch tensors: argument marshalling only, in C++ because it is on the path of
// every call. A small layer's two kernels take about 8 us on the device; marshalled in Python (ctypes, one wrapper object
// per pointer, torch.cuda.current_stream()) a call took 13-18 us of host time, so the host set the pace of every layer
// below some 15 us. Each function takes exactly the positional arguments its wrapper in binding.py passes, checks that
// tensors are contiguous CUDA tensors, and returns the sdgp_status as an int.
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <Python.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <algorithm>

#include "../../include/sdgp.h"
#include "torch_autograd.h"

namespace {

// Reads positional arguments in order; after the first failure (a Python exception is set) every read returns zero.
struct Args {
  PyObject* const* a;
  Py_ssize_t left;
  bool ok = true;

  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : a(args), left(n) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
      ok = false;
    }
  }
  int64_t i64() {
    if (!ok) return 0;
    const long long v = PyLong_AsLongLong(*a++);
    if (v == -1 && PyErr_Occurred()) ok = false;
    return v;
  }
  int i32() {
    const int64_t v = i64();
    if (ok && (v > INT32_MAX || v < INT32_MIN)) {
      PyErr_SetString(PyExc_OverflowError, "integer argument does not fit 32 bits");
      ok = false;
    }
    return (int)v;
  }
  uint64_t u64() {  // seeds: any Python int, modulo 2^64
    if (!ok) return 0;
    PyObject* o = *a++;
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) ok = false;
    return v;
  }
  // A contiguous CUDA tensor, or nullptr for None.
  const at::Tensor* tensor(const char* name) {
    if (!ok) return nullptr;
    PyObject* o = *a++;
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "%s must be a torch tensor or None", name);
      ok = false;
      return nullptr;
    }
    const at::Tensor* t = &THPVariable_Unpack(o);
    if (!t->is_cuda() || !t->is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s must be a contiguous CUDA tensor", name);
      ok = false;
      return nullptr;
    }
    (void)t->data_ptr();  // throws here, under the interpreter lock, if there is no memory behind the tensor
    return t;
  }
  void* pointer(const char* name) {
    const at::Tensor* t = tensor(name);
    return t ? t->data_ptr() : nullptr;
  }
  // A tensor whose shape the call reads: None is an error; it has `dims` dimensions (-d: d or more).
  const at::Tensor* shaped(const char* name, int dims) {
    const at::Tensor* t = tensor(name);
    if (ok && !t) {
      PyErr_Format(PyExc_AttributeError, "%s must be a tensor, not None", name);
      ok = false;
    }
    if (ok && (dims > 0 ? t->dim() != dims : t->dim() < -dims)) {
      PyErr_Format(PyExc_ValueError, "%s must have %s%d dimensions, has %d", name, dims > 0 ? "" : "at least ", dims > 0 ? dims : -dims,
                   (int)t->dim());
      ok = false;
      return nullptr;
    }
    return t;
  }
};

struct Workspace {
  void* ptr;
  size_t bytes;
};
Workspace workspace(Args& in) {
  const at::Tensor* t = in.tensor("workspace");
  return t ? Workspace{t->data_ptr(), (size_t)t->nbytes()} : Workspace{nullptr, 0};
}

void* stream() { return (void*)c10::cuda::getCurrentCUDAStream().stream(); }

// K = last dimension, rows = the rest
void rows_and_k(const at::Tensor* t, int64_t& rows, int64_t& K) {
  K = t->dim() ? t->size(-1) : 0;
  rows = K ? t->numel() / K : 0;
}

// Runs the library call without the interpreter lock (a launch may wait for room in the driver's queue).
template <class F>
PyObject* status_of(const Args& in, F call) {
  if (!in.ok) return nullptr;
  void* s = stream();
  sdgp_status st;
  // (`call` only reads sizes and pointers of tensors the caller holds and that Args::tensor has checked: it does not throw)
  Py_BEGIN_ALLOW_THREADS
  st = call(s);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

#define ENTRY(name) PyObject* name(PyObject*, PyObject* const* args, Py_ssize_t nargs)

ENTRY(prune) {  // dO, n, m, scheme, seed, dtype, dense, values, meta, mask
  Args in(args, nargs, 10);
  const at::Tensor* dO = in.shaped("dO", 0);
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  const int dtype = in.i32();
  void *dense = in.pointer("dense"), *values = in.pointer("values"), *meta = in.pointer("meta"), *mask = in.pointer("mask");
  int64_t rows = 0, K = 0;
  if (in.ok) rows_and_k(dO, rows, K);
  return status_of(in, [&](void* s) {
    return sdgp_prune_typed(dO->data_ptr(), rows, K, n, m, (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype, dense, values, meta, mask, s);
  });
}

ENTRY(relu_backward_prune) {  // dY, dSkip, residual, act, n, m, scheme, seed, dtype, grad, dense, values, meta, mask
  Args in(args, nargs, 14);
  const at::Tensor* dY = in.shaped("dY", 0);
  const at::Tensor* skip = in.tensor("dSkip");
  const int residual = in.i32();
  const at::Tensor* act = in.shaped("act", 0);
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  const int dtype = in.i32();
  void *grad = in.pointer("grad"), *dense = in.pointer("dense"), *values = in.pointer("values"), *meta = in.pointer("meta"),
       *mask = in.pointer("mask");
  int64_t rows = 0, K = 0;
  if (in.ok) {
    if (dY->sizes() != act->sizes() || (skip && skip->sizes() != dY->sizes())) {
      PyErr_SetString(PyExc_ValueError, residual ? "dY, dSkip and act must have the same shape" : "dY and act must have the same shape");
      in.ok = false;
    } else {
      rows_and_k(dY, rows, K);
    }
  }
  return status_of(in, [&](void* s) {
    if (residual)
      return sdgp_residual_relu_backward_prune(dY->data_ptr(), skip ? skip->data_ptr() : nullptr, act->data_ptr(), rows, K, n, m,
                                               (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype, grad, dense, values, meta, mask, s);
    return sdgp_relu_backward_prune(dY->data_ptr(), act->data_ptr(), rows, K, n, m, (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype,
                                    grad, dense, values, meta, mask, s);
  });
}

ENTRY(maxpool_relu_backward_prune) {  // dYp, skip, act, n, m, scheme, seed, dtype, grad, dense, values, meta, mask
  Args in(args, nargs, 13);
  const at::Tensor* dY = in.shaped("dYp", 0);
  const at::Tensor* skip = in.tensor("skip");
  const at::Tensor* act = in.shaped("act", 0);
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  const int dtype = in.i32();
  void *grad = in.pointer("grad"), *dense = in.pointer("dense"), *values = in.pointer("values"), *meta = in.pointer("meta"),
       *mask = in.pointer("mask");
  if (in.ok) {
    const char* wrong = nullptr;
    if (skip && skip->sizes() != dY->sizes()) wrong = "skip must have the shape of dYp";
    else if (act->dim() != 4 || dY->dim() != 4) wrong = "dYp and act must be NHWC tensors";
    else if (dY->size(0) != act->size(0) || dY->size(1) != act->size(1) / 2 || dY->size(2) != act->size(2) / 2 ||
             dY->size(3) != act->size(3))
      wrong = "dYp must be [B, H/2, W/2, K]";
    if (wrong) {
      PyErr_SetString(PyExc_ValueError, wrong);
      in.ok = false;
    }
  }
  return status_of(in, [&](void* s) {
    return sdgp_maxpool_relu_backward_prune(dY->data_ptr(), skip ? skip->data_ptr() : nullptr, act->data_ptr(), (int)act->size(0),
                                            (int)act->size(1), (int)act->size(2), act->size(3), n, m, (sdgp_scheme)scheme, seed,
                                            (sdgp_dtype)dtype, grad, dense, values, meta, mask, s);
  });
}

ENTRY(dgrad_linear) {  // dO, W, dD, n, m, scheme, seed, dtype, workspace, flags
  Args in(args, nargs, 10);
  const at::Tensor* dO = in.shaped("dO", 2);
  const at::Tensor* W = in.shaped("W", -2);
  void* dD = in.pointer("dD");
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  const int dtype = in.i32();
  const Workspace ws = workspace(in);
  const uint32_t flags = (uint32_t)in.i32();
  return status_of(in, [&](void* s) {
    return sdgp_dgrad_linear_typed(dO->data_ptr(), W->data_ptr(), dD, dO->size(0), dO->size(1), W->size(1), n, m, (sdgp_scheme)scheme,
                                   seed, (sdgp_dtype)dtype, ws.ptr, ws.bytes, flags, s);
  });
}

ENTRY(dgrad_linear_static) {  // dO, W, dD, n, m, scheme, seed
  Args in(args, nargs, 7);
  const at::Tensor* dO = in.shaped("dO", 2);
  const at::Tensor* W = in.shaped("W", -2);
  void* dD = in.pointer("dD");
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  return status_of(in, [&](void* s) {
    return sdgp_dgrad_linear_static(dO->data_ptr(), W->data_ptr(), dD, dO->size(0), dO->size(1), W->size(1), n, m, (sdgp_scheme)scheme,
                                    seed, s);
  });
}

// dO, W, dD, stride, pad, groups (0: sdgp_dgrad_conv2d), n, m, scheme, seed, dtype, workspace, flags
ENTRY(dgrad_conv2d) {
  Args in(args, nargs, 13);
  void* dO = in.pointer("dO");
  const at::Tensor* W = in.shaped("W", 4);
  const at::Tensor* dD = in.shaped("dD", 4);
  const int stride = in.i32(), pad = in.i32(), groups = in.i32(), n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  const int dtype = in.i32();
  const Workspace ws = workspace(in);
  const uint32_t flags = (uint32_t)in.i32();
  return status_of(in, [&](void* s) {
    const int B = (int)dD->size(0), H = (int)dD->size(1), Wd = (int)dD->size(2), Cin = (int)dD->size(3);
    const int Cout = (int)W->size(0), R = (int)W->size(1), S = (int)W->size(2);
    if (groups)
      return sdgp_dgrad_conv2d_grouped(dO, W->data_ptr(), dD->data_ptr(), B, H, Wd, Cin, Cout, R, S, stride, pad, groups, n, m,
                                       (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype, ws.ptr, ws.bytes, flags, s);
    return sdgp_dgrad_conv2d_typed(dO, W->data_ptr(), dD->data_ptr(), B, H, Wd, Cin, Cout, R, S, stride, pad, n, m,
                                   (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype, ws.ptr, ws.bytes, flags, s);
  });
}

ENTRY(spmm_linear) {  // values, meta, W, dD, dtype
  Args in(args, nargs, 5);
  void *values = in.pointer("values"), *meta = in.pointer("meta");
  const at::Tensor* W = in.shaped("W", -1);
  const at::Tensor* dD = in.shaped("dD", 2);
  const int dtype = in.i32();
  return status_of(in, [&](void* s) {
    return sdgp_spmm_linear_typed(values, meta, W->data_ptr(), dD->data_ptr(), dD->size(0), W->size(0), dD->size(1), (sdgp_dtype)dtype, s);
  });
}

ENTRY(spmm_conv2d) {  // values, meta, W, dD, stride, pad, dtype
  Args in(args, nargs, 7);
  void *values = in.pointer("values"), *meta = in.pointer("meta");
  const at::Tensor* W = in.shaped("W", 4);
  const at::Tensor* dD = in.shaped("dD", 4);
  const int stride = in.i32(), pad = in.i32(), dtype = in.i32();
  return status_of(in, [&](void* s) {
    return sdgp_spmm_conv2d_typed(values, meta, W->data_ptr(), dD->data_ptr(), (int)dD->size(0), (int)dD->size(1), (int)dD->size(2),
                                  (int)dD->size(3), (int)W->size(0), (int)W->size(1), (int)W->size(2), stride, pad, (sdgp_dtype)dtype, s);
  });
}

// ---- operators around a language model's linear layers ----

// Reads arguments like Args; every tensor must lie on the device of the first one and have the element type that it stands for.
struct LmArgs : Args {
  using Args::Args;
  c10::Device device{c10::kCUDA, 0};
  bool any = false;

  PyObject* fail(const char* name, const char* what) {
    if (ok) PyErr_Format(PyExc_ValueError, "%s %s", name, what);
    ok = false;
    return nullptr;
  }
  const at::Tensor* on_device(const char* name) {
    const at::Tensor* t = tensor(name);
    if (!t) return nullptr;
    if (any && t->device() != device) {
      fail(name, "must be on the same device as the other tensors");
      return nullptr;
    }
    device = t->device();
    any = true;
    return t;
  }
  // Elements of `dtype`: its own type, or (16 bits, as elsewhere in this library) integers that hold their bits.
  const at::Tensor* elements(const char* name, int dtype) {
    const at::Tensor* t = on_device(name);
    if (!t) return nullptr;
    const at::ScalarType type = t->scalar_type();
    const bool bits = type == at::kShort || type == at::kUInt16;
    if (dtype == SDGP_FP32   ? type != at::kFloat
        : dtype == SDGP_FP16 ? type != at::kHalf && !bits
        : dtype == SDGP_BF16 ? type != at::kBFloat16 && !bits
                             : t->element_size() != 2) {  // (a dtype that there is not: the call refuses it)
      fail(name, "does not have the elements that dtype names");
      return nullptr;
    }
    return t;
  }
  // The compressed pruned copy: values of `dtype` (which the call refuses if they are fp32) and their 16-bit metadata.
  const at::Tensor* compressed_values(const char* name, int dtype) { return dtype == SDGP_FP32 ? two_bytes(name) : elements(name, dtype); }
  const at::Tensor* two_bytes(const char* name) {
    const at::Tensor* t = on_device(name);
    if (t && t->element_size() != 2) {
      fail(name, "must hold two bytes an element");
      return nullptr;
    }
    return t;
  }
  const at::Tensor* of_type(const char* name, at::ScalarType type, int64_t numel) {
    const at::Tensor* t = on_device(name);
    if (t && t->scalar_type() != type) {
      fail(name, type == at::kFloat ? "must be a float32 tensor" : "must be an int64 tensor");
      return nullptr;
    }
    if (t && numel >= 0 && t->numel() != numel) {
      fail(name, "does not have the number of elements that the other shapes ask for");
      return nullptr;
    }
    return t;
  }
  void same_numel(const char* name, const at::Tensor* t, int64_t numel) {
    if (t && t->numel() != numel) fail(name, "does not have the number of elements that the other shapes ask for");
  }
};

void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
float* floats(const at::Tensor* t) { return (float*)data(t); }

template <class F>
PyObject* status_on(const LmArgs& in, F call) {
  if (!in.ok) return nullptr;
  const c10::cuda::CUDAGuard guard(in.device);
  return status_of(in, call);
}

// An integer, or `otherwise` for None.
int64_t i64_or(Args& in, int64_t otherwise) {
  if (in.ok && *in.a == Py_None) {
    ++in.a;
    return otherwise;
  }
  return in.i64();
}

// A tensor argument that must be there.
const at::Tensor* given(LmArgs& in, const at::Tensor* t, const char* name) {
  if (in.ok && !t) in.fail(name, "must be a tensor, not None");
  return t;
}

float f32(Args& in) {
  if (!in.ok) return 0.0f;
  const double v = PyFloat_AsDouble(*in.a++);
  if (v == -1.0 && PyErr_Occurred()) in.ok = false;
  return (float)v;
}

// The dtype argument (number `at`), read before the tensors whose elements it names.
int dtype_argument(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, Py_ssize_t at) {
  return nargs == want ? (int)PyLong_AsLong(args[at]) : 0;
}

ENTRY(token_logprob) {  // logits, targets, classes, dtype, logprob, entropy, lse, top_logprob, top_token
  LmArgs in(args, nargs, 9);
  const int dtype = dtype_argument(args, nargs, 9, 3);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* logits = given(in, in.elements("logits", dtype), "logits");
  int64_t rows = 0, K = 0;
  if (in.ok) rows_and_k(logits, rows, K);
  const at::Tensor* targets = given(in, in.of_type("targets", at::kLong, rows), "targets");
  const int64_t classes = i64_or(in, K);
  in.i32();
  const at::Tensor* logprob = given(in, in.of_type("logprob", at::kFloat, rows), "logprob");
  const at::Tensor *entropy = in.of_type("entropy", at::kFloat, rows), *lse = in.of_type("lse", at::kFloat, rows),
                   *top_logprob = in.of_type("top_logprob", at::kFloat, -1), *top_token = in.of_type("top_token", at::kLong, -1);
  int64_t top = 0;
  for (const at::Tensor* t : {top_logprob, top_token}) {
    if (!in.ok || !t) continue;
    const int64_t k = t->dim() ? t->size(-1) : 0;
    in.same_numel("top_logprob or top_token", t, rows * k);
    if (in.ok && top != 0 && k != top) in.fail("top_logprob and top_token", "must have the same shape");
    top = k;
  }
  return status_on(in, [&](void* s) {
    return sdgp_token_logprob(data(logits), (const int64_t*)data(targets), rows, K, classes, (sdgp_dtype)dtype,
                              (int)std::min<int64_t>(top, INT32_MAX), floats(logprob), floats(entropy), floats(lse), floats(top_logprob),
                              (int64_t*)data(top_token), s);
  });
}

// logits, targets, lse, entropy, d_logprob, d_entropy, classes, n, m, scheme, seed, dtype, grad, values, meta
ENTRY(token_logprob_backward) {
  LmArgs in(args, nargs, 15);
  const int dtype = dtype_argument(args, nargs, 15, 11);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* logits = given(in, in.elements("logits", dtype), "logits");
  int64_t rows = 0, K = 0;
  if (in.ok) rows_and_k(logits, rows, K);
  const at::Tensor* targets = given(in, in.of_type("targets", at::kLong, rows), "targets");
  const at::Tensor* lse = given(in, in.of_type("lse", at::kFloat, rows), "lse");
  const at::Tensor *entropy = in.of_type("entropy", at::kFloat, rows), *d_logprob = in.of_type("d_logprob", at::kFloat, rows),
                   *d_entropy = in.of_type("d_entropy", at::kFloat, rows);
  const int64_t classes = i64_or(in, K);
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  in.i32();
  const at::Tensor *grad = in.elements("grad", dtype), *values = in.compressed_values("values", dtype), *meta = in.two_bytes("meta");
  in.same_numel("grad", grad, rows * K);
  in.same_numel("values", values, rows * (K / 2));
  in.same_numel("meta", meta, rows * (K / 16));
  return status_on(in, [&](void* s) {
    return sdgp_token_logprob_backward(data(logits), (const int64_t*)data(targets), floats(lse), floats(entropy), floats(d_logprob),
                                       floats(d_entropy), rows, K, classes, n, m, (sdgp_scheme)scheme, seed, (sdgp_dtype)dtype, data(grad),
                                       data(values), data(meta), s);
  });
}

ENTRY(residual_norm) {  // branch, residual, post_weight, gate, pre_weight, alpha, eps, dtype, out, y, post_rstd, pre_rstd
  LmArgs in(args, nargs, 12);
  const int dtype = dtype_argument(args, nargs, 12, 7);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* branch = given(in, in.elements("branch", dtype), "branch");
  int64_t rows = 0, C = 0;
  if (in.ok) rows_and_k(branch, rows, C);
  const at::Tensor* residual = given(in, in.elements("residual", dtype), "residual");
  const at::Tensor *post_weight = in.elements("post_weight", dtype), *gate = in.elements("gate", dtype),
                   *pre_weight = in.elements("pre_weight", dtype);
  const float alpha = f32(in), eps = f32(in);
  in.i32();
  const at::Tensor* out = given(in, in.elements("out", dtype), "out");
  const at::Tensor* y = in.elements("y", dtype);
  const at::Tensor *post_rstd = in.of_type("post_rstd", at::kFloat, rows), *pre_rstd = in.of_type("pre_rstd", at::kFloat, rows);
  in.same_numel("residual", residual, rows * C);
  in.same_numel("out", out, rows * C);
  in.same_numel("y", y, rows * C);
  in.same_numel("post_weight", post_weight, C);
  in.same_numel("pre_weight", pre_weight, C);
  const int64_t groups = gate && C ? gate->numel() / C : 1;
  in.same_numel("gate", gate, groups * C);
  return status_on(in, [&](void* s) {
    return sdgp_residual_norm(data(branch), data(residual), data(post_weight), data(gate), data(pre_weight), rows, C, groups, alpha, eps,
                              (sdgp_dtype)dtype, data(out), data(y), floats(post_rstd), floats(pre_rstd), s);
  });
}

// branch, out, d_out, d_y, post_weight, gate, pre_weight, post_rstd, pre_rstd, alpha, n, m, scheme, seed, dtype, d_residual, d_branch, d_gate,
// d_post_weight, d_pre_weight, values, meta, workspace
ENTRY(residual_norm_backward) {
  LmArgs in(args, nargs, 23);
  const int dtype = dtype_argument(args, nargs, 23, 14);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* branch = given(in, in.elements("branch", dtype), "branch");
  int64_t rows = 0, C = 0;
  if (in.ok) rows_and_k(branch, rows, C);
  const at::Tensor *out = in.elements("out", dtype), *d_out = in.elements("d_out", dtype), *d_y = in.elements("d_y", dtype);
  const at::Tensor *post_weight = in.elements("post_weight", dtype), *gate = in.elements("gate", dtype),
                   *pre_weight = in.elements("pre_weight", dtype);
  const at::Tensor *post_rstd = in.of_type("post_rstd", at::kFloat, rows), *pre_rstd = in.of_type("pre_rstd", at::kFloat, rows);
  const float alpha = f32(in);
  const int n = in.i32(), m = in.i32(), scheme = in.i32();
  const uint64_t seed = in.u64();
  in.i32();
  const at::Tensor *d_residual = in.elements("d_residual", dtype), *d_branch = in.elements("d_branch", dtype);
  const int64_t groups = gate && C ? gate->numel() / C : 1;
  const at::Tensor *d_gate = in.of_type("d_gate", at::kFloat, groups * C), *d_post_weight = in.of_type("d_post_weight", at::kFloat, C),
                   *d_pre_weight = in.of_type("d_pre_weight", at::kFloat, C);
  const at::Tensor *values = in.compressed_values("values", dtype), *meta = in.two_bytes("meta"), *ws = in.on_device("workspace");
  for (const auto& [name, t] : {std::pair<const char*, const at::Tensor*>{"out", out}, {"d_out", d_out}, {"d_y", d_y}, {"d_residual", d_residual},
                                {"d_branch", d_branch}})
    in.same_numel(name, t, rows * C);
  in.same_numel("post_weight", post_weight, C);
  in.same_numel("pre_weight", pre_weight, C);
  in.same_numel("gate", gate, groups * C);
  in.same_numel("values", values, rows * (C / 2));
  in.same_numel("meta", meta, rows * (C / 16));
  const size_t ws_bytes = ws ? (size_t)ws->nbytes() : 0;
  return status_on(in, [&](void* s) {
    return sdgp_residual_norm_backward(data(branch), data(out), data(d_out), data(d_y), data(post_weight), data(gate), data(pre_weight),
                                       floats(post_rstd), floats(pre_rstd), rows, C, groups, alpha, n, m, (sdgp_scheme)scheme, seed,
                                       (sdgp_dtype)dtype, data(d_residual), data(d_branch), floats(d_gate), floats(d_post_weight),
                                       floats(d_pre_weight), data(values), data(meta), data(ws), ws_bytes, s);
  });
}

// A tensor of e4m3 numbers, or of bytes that hold their bits.
const at::Tensor* e4m3(LmArgs& in, const char* name) {
  const at::Tensor* t = given(in, in.on_device(name), name);
  if (t && t->scalar_type() != at::kFloat8_e4m3fn && t->scalar_type() != at::kByte) in.fail(name, "must be a float8_e4m3fn or uint8 tensor");
  return t;
}

ENTRY(fp8_quantize) {  // x, q, scale, block_rows, dtype
  LmArgs in(args, nargs, 5);
  const int dtype = dtype_argument(args, nargs, 5, 4);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* x = given(in, in.elements("x", dtype), "x");
  const at::Tensor* q = e4m3(in, "q");
  const at::Tensor* scale = given(in, in.of_type("scale", at::kFloat, -1), "scale");
  const int block_rows = in.i32();
  in.i32();
  int64_t rows = 0, K = 0;
  if (in.ok) {
    rows_and_k(x, rows, K);
    in.same_numel("q", q, rows * K);
    if (block_rows > 0) in.same_numel("scale", scale, (rows + block_rows - 1) / block_rows * ((K + 127) / 128));
  }
  return status_on(in, [&](void* s) { return sdgp_fp8_quantize(data(x), rows, K, block_rows, (sdgp_dtype)dtype, data(q), floats(scale), s); });
}

ENTRY(fp8_linear) {  // xq, x_scale, wq, w_scale, y, dtype
  LmArgs in(args, nargs, 6);
  const int dtype = dtype_argument(args, nargs, 6, 5);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* xq = e4m3(in, "xq");
  const at::Tensor* x_scale = given(in, in.of_type("x_scale", at::kFloat, -1), "x_scale");
  const at::Tensor* wq = e4m3(in, "wq");
  const at::Tensor* w_scale = given(in, in.of_type("w_scale", at::kFloat, -1), "w_scale");
  const at::Tensor* y = given(in, in.elements("y", dtype), "y");
  in.i32();
  int64_t rows = 0, K = 0, features = 0, wk = 0;
  if (in.ok) {
    rows_and_k(wq, features, wk);
    rows_and_k(xq, rows, K);
    if (wk != K) in.fail("xq and wq", "must have the same last dimension");
    in.same_numel("x_scale", x_scale, rows * ((K + 127) / 128));
    in.same_numel("w_scale", w_scale, (features + 127) / 128 * ((K + 127) / 128));
    in.same_numel("y", y, rows * features);
  }
  return status_on(in, [&](void* s) {
    return sdgp_fp8_linear(data(xq), floats(x_scale), data(wq), floats(w_scale), data(y), rows, features, K, (sdgp_dtype)dtype, s);
  });
}

// Whether the C++ layers take a tensor: what Python hands over is an ordinary tensor (no subclass) in GPU memory of a 16-bit type, and
// nothing watches or transforms the operators that run on it.
bool plain_tensor(PyObject* o, int64_t dims) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && (dims < 0 ? t.dim() >= -dims : t.dim() == dims) &&
         (t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf) && !at::isTensorSubclassLike(t) && !t._fw_grad(0).defined();
}

bool plain_int(PyObject* o) {  // (no bool, no object with __index__: the operators' own argument parser has its rules for those)
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  return overflow == 0 && v >= INT32_MIN && v <= INT32_MAX;
}

// Differentiable layers: x, weight, then `integers` numbers, the last of them a seed. NotImplemented: not a plain call, the caller takes
// the Python form (which also gives the errors of arguments that are none).
template <class F>
PyObject* layer(PyObject* const* args, Py_ssize_t nargs, int integers, int64_t x_dims, int64_t weight_dims, F call) {
  HANDLE_TH_ERRORS
  Args in(args, nargs, 2 + integers);
  if (!in.ok) return nullptr;
  bool plain = !torch::jit::tracer::isTracing() && !at::impl::torch_function_mode_enabled() && plain_tensor(args[0], x_dims) &&
               plain_tensor(args[1], weight_dims) && PyLong_CheckExact(args[1 + integers]);
  for (int k = 2; plain && k < 1 + integers; ++k) plain = plain_int(args[k]);
  at::Tensor t[2];
  for (int k = 0; plain && k < 2; ++k, ++in.a) t[k] = THPVariable_Unpack(*in.a);
  if (!plain || t[0].scalar_type() != t[1].scalar_type() || t[0].device() != t[1].device()) Py_RETURN_NOTIMPLEMENTED;
  std::vector<int64_t> numbers;
  for (int k = 0; k < integers; ++k) numbers.push_back(k + 1 < integers ? (int64_t)in.i32() : (int64_t)in.u64());
  if (!in.ok) return nullptr;
  at::Tensor y;
  {
    struct NoGil {
      PyThreadState* state = PyEval_SaveThread();
      ~NoGil() { PyEval_RestoreThread(state); }
    } no_gil;
    y = call(t[0], t[1], std::move(numbers));
  }
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}
ENTRY(linear_layer) {  // x, weight, n, m, scheme, seed
  return layer(args, nargs, 4, -1, 2, sdgp_torch::linear);
}
ENTRY(conv2d_layer) {  // x, weight, stride, padding, kind, n, m, scheme, seed
  return layer(args, nargs, 7, 4, 4, sdgp_torch::conv2d);
}

ENTRY(workspace_size_linear) {  // rows, K, N, flags
  Args in(args, nargs, 4);
  const int64_t rows = in.i64(), K = in.i64(), N = in.i64();
  const uint32_t flags = (uint32_t)in.i64();
  return in.ok ? PyLong_FromSize_t(sdgp_workspace_size_linear(rows, K, N, flags)) : nullptr;
}

ENTRY(workspace_size_conv2d) {  // B, H, Wd, Cin, Cout, R, S, stride, pad, groups (0: sdgp_workspace_size_conv2d), flags
  Args in(args, nargs, 11);
  int v[10];
  for (int& x : v) x = in.i32();
  const uint32_t flags = (uint32_t)in.i64();
  if (!in.ok) return nullptr;
  return PyLong_FromSize_t(v[9] ? sdgp_workspace_size_conv2d_grouped(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], flags)
                                : sdgp_workspace_size_conv2d(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], flags));
}

ENTRY(workspace_size_residual_norm_backward) {  // rows, C, groups
  Args in(args, nargs, 3);
  const int64_t rows = in.i64(), C = in.i64(), groups = in.i64();
  return in.ok ? PyLong_FromSize_t(sdgp_workspace_size_residual_norm_backward(rows, C, groups)) : nullptr;
}

#undef ENTRY

// A C++ exception (data_ptr() of a tensor without storage, say) becomes a Python one.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
  try {
    return F(self, args, nargs);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))guarded<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(prune), METHOD(relu_backward_prune), METHOD(maxpool_relu_backward_prune), METHOD(dgrad_linear),
                         METHOD(dgrad_linear_static), METHOD(dgrad_conv2d), METHOD(spmm_linear), METHOD(spmm_conv2d),
                         METHOD(token_logprob), METHOD(token_logprob_backward), METHOD(residual_norm), METHOD(residual_norm_backward),
                         METHOD(fp8_quantize), METHOD(fp8_linear), METHOD(workspace_size_residual_norm_backward),
                         METHOD(workspace_size_linear), METHOD(workspace_size_conv2d), METHOD(linear_layer),
                         METHOD(conv2d_layer), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_sdgp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sdgp_torch() { return PyModule_Create(&module_def); }
