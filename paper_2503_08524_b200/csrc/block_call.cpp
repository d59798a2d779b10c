// Python side of the 8-bit block operators and of the constraints on logits: argument checks and marshalling, nothing else.
//
// As for the paged operators, a step of a few rows is bound by the host side of its calls, so the tensors' shapes, strides
// and pointers are read here and not in Python; the library's functions and the error class are handed over once by
// block8.py.
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>
#include <string>

#include "d3.h"

namespace {

decltype(&d3_add_norm) norm_call;
decltype(&d3_matmul8) matmul_call;
decltype(&d3_gated_matmul8) gated_call;
decltype(&d3_constrain_logits) logits_call;
PyObject *error_class;

// Raises D3Error(code, what); always nullptr.
PyObject *fail(int code, const std::string &what) {
  PyObject *e = PyObject_CallFunction(error_class, "is", code, what.c_str());
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return nullptr;
}
PyObject *refuse(const char *call, const std::string &what) { return fail(D3_EINVAL, std::string(call) + ": " + what); }

// The tensor of an argument; nullptr for None.  `ok` is cleared for anything else.
const at::Tensor *tensor(PyObject *o, bool &ok) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) { ok = false; return nullptr; }
  return &THPVariable_Unpack(o);
}
int code_of(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return D3_BF16;
    case at::kHalf: return D3_FP16;
    case at::kFloat: return D3_FP32;
    case at::kFloat8_e4m3fn: return D3_E4M3;
    default: return -1;
  }
}
bool on(const at::Tensor &t, int device) { return device < 0 ? t.is_cpu() : t.is_cuda() && t.get_device() == device; }
bool is_vector(const at::Tensor &t, at::ScalarType type, int64_t n, int device) {
  return t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous() && on(t, device);
}
// [n][width] with contiguous rows; the stride of a single row (which torch leaves arbitrary) counts as its width
struct Rows { void *p; int64_t stride; };
bool rows_of(const at::Tensor &t, int64_t n, int64_t width, at::ScalarType type, int device, Rows &out) {
  if (t.dim() != 2 || t.size(0) != n || t.size(1) != width || t.scalar_type() != type || !on(t, device) || (t.stride(1) != 1 && width > 1))
    return false;
  out.stride = n > 1 ? t.stride(0) : width;
  out.p = t.data_ptr();
  return true;
}
std::string rows_text(const char *name, int64_t n, int64_t width, const char *type) {
  return std::string(name) + " must be " + type + " [" + std::to_string(n) + "][" + std::to_string(width) + "] on the call's device, rows contiguous";
}
// Counts a tensor that the call writes as changed in place: a graph that saved it refuses its backward pass instead of
// computing with other numbers.  (Tensors of inference mode have no count.)
void changed(const at::Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
bool number(PyObject *o, long long &v) {
  v = PyLong_AsLongLong(o);
  return !(v == -1 && PyErr_Occurred());
}
bool type_arg(PyObject *o, at::ScalarType &type) {
  if (!THPDtype_Check(o)) return false;
  type = reinterpret_cast<THPDtype *>(o)->scalar_type;
  return code_of(type) >= 0;
}
int64_t blocks(int64_t n) { return (n + 127) / 128; }
// a new reference to what was given, or to a tensor that the call made
PyObject *result(PyObject *given, const at::Tensor &made) {
  if (made.defined()) return THPVariable_Wrap(made);
  Py_INCREF(given);
  return given;
}
PyObject *pack(PyObject *a, PyObject *b, PyObject *c) {   // takes the references; c may be absent
  PyObject *r = a && b && (c || !PyErr_Occurred()) ? PyTuple_New(c ? 3 : 2) : nullptr;
  if (!r) {
    Py_XDECREF(a); Py_XDECREF(b); Py_XDECREF(c);
    return nullptr;
  }
  PyTuple_SET_ITEM(r, 0, a);
  PyTuple_SET_ITEM(r, 1, b);
  if (c) PyTuple_SET_ITEM(r, 2, c);
  return r;
}

// norm(name of the call, x, gain, add, total, out, scale, dtype, eps) -> (out, scale, total)
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  HANDLE_TH_ERRORS
  if (argc != 9) return refuse("d3_add_norm", "9 arguments");
  const char *call = PyUnicode_AsUTF8(a[0]);
  if (!call) return nullptr;
  bool ok = true;
  const at::Tensor *x = tensor(a[1], ok), *gain = tensor(a[2], ok), *add = tensor(a[3], ok), *total = tensor(a[4], ok), *out = tensor(a[5], ok),
                   *scale = tensor(a[6], ok);
  if (!ok || !x || x->dim() != 2) return refuse(call, "x must be a tensor [rows][dim], the others tensors or None");
  const int64_t n = x->size(0), dim = x->size(1);
  const int device = x->get_device(), code = code_of(x->scalar_type());
  if (code < 0 || code == D3_E4M3) return refuse(call, "x must be bf16, fp16 or fp32");
  if (n > 0x7fffffff || dim < 8 || dim > 65536 || dim % 8) return refuse(call, "fewer than 2^31 rows of 8..65536 numbers, a multiple of 8");
  const double eps = PyFloat_AsDouble(a[8]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  if (!(eps >= 0.0 && eps < 3e38)) return refuse(call, "eps must be finite and not negative");
  d3_add_norm_args args;
  std::memset(&args, 0, sizeof(args));
  args.struct_size = sizeof(args);
  args.n_rows = (int32_t)n; args.dim = (int32_t)dim; args.x_dtype = code; args.eps = (float)eps;
  Rows r;
  if (!rows_of(*x, n, dim, x->scalar_type(), device, r)) return refuse(call, rows_text("x", n, dim, "a matrix"));
  args.x_dev = r.p; args.x_stride = r.stride;
  if (gain) {
    const int gc = code_of(gain->scalar_type());
    if (gc < 0 || gc == D3_E4M3 || !is_vector(*gain, gain->scalar_type(), dim, device))
      return refuse(call, "gain must be a contiguous bf16, fp16 or fp32 vector of " + std::to_string(dim));
    args.gain_dev = gain->data_ptr(); args.gain_dtype = gc;
  }
  at::ScalarType type = at::kFloat8_e4m3fn;
  if (out) {
    type = out->scalar_type();
    if (code_of(type) < 0) return refuse(call, "out must be float8_e4m3fn, bf16, fp16 or fp32");
    at::ScalarType said;
    if (a[7] != Py_None && (!type_arg(a[7], said) || said != type)) return refuse(call, "dtype is not out's");
  } else if (a[7] != Py_None && !type_arg(a[7], type)) {
    return refuse(call, "dtype must be float8_e4m3fn, bf16, fp16 or fp32");
  }
  const bool eight = type == at::kFloat8_e4m3fn;
  if (!eight && scale) return refuse(call, "a scale belongs to results in 8 bits");
  if (add) {
    const at::ScalarType t = add->scalar_type();
    if ((t != x->scalar_type() && t != at::kFloat) || !rows_of(*add, n, dim, t, device, r)) return refuse(call, rows_text("add", n, dim, "of x's type or fp32,"));
    args.add_dev = r.p; args.add_stride = r.stride; args.add_dtype = code_of(t);
  } else if (total) {
    return refuse(call, "total without add");
  }
  if (out && !rows_of(*out, n, dim, type, device, r)) return refuse(call, rows_text("out", n, dim, "a matrix"));
  if (out) { args.out_dev = r.p; args.out_stride = r.stride; }
  if (scale) {
    if (!rows_of(*scale, n, blocks(dim), at::kFloat, device, r)) return refuse(call, rows_text("scale", n, blocks(dim), "fp32"));
    args.scale_dev = static_cast<float *>(r.p); args.scale_stride = r.stride;
  }
  if (total) {
    if (!rows_of(*total, n, dim, add->scalar_type(), device, r)) return refuse(call, rows_text("total", n, dim, "of add's type,"));
    args.total_dev = r.p; args.total_stride = r.stride;
  }
  if (device < 0) return refuse(call, "tensors must be on a CUDA device");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  at::Tensor new_out, new_scale, new_total;
  if (!out) {
    new_out = at::empty({n, dim}, x->options().dtype(type));
    args.out_dev = new_out.data_ptr(); args.out_stride = dim;
  }
  if (eight && !scale) {
    new_scale = at::empty({n, blocks(dim)}, x->options().dtype(at::kFloat));
    args.scale_dev = new_scale.data_ptr<float>(); args.scale_stride = blocks(dim);
  }
  if (add && !total) {
    new_total = at::empty({n, dim}, add->options());
    args.total_dev = new_total.data_ptr(); args.total_stride = dim;
  }
  args.out_dtype = code_of(type);
  if (n > 0) {
    const int rc = norm_call(&args, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
    if (rc != D3_OK) return fail(rc, call);
    if (out) changed(*out);
    if (scale) changed(*scale);
    if (total) changed(*total);
  }
  PyObject *o = result(a[5], new_out), *s = result(a[6], new_scale);
  return pack(o, s, result(a[4], new_total));
  END_HANDLE_TH_ERRORS
}

// product(addresses of the weights (the second 0: no gate), device, a, a_scale, out, scale, dtype, status) -> out, or (out, scale) if gated
PyObject *product(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  HANDLE_TH_ERRORS
  long long w0, w1, dev;
  if (argc != 9) return refuse("d3_matmul8", "9 arguments");
  if (!number(a[0], w0) || !number(a[1], w1) || !number(a[2], dev)) return nullptr;
  const d3_weight8 *w = reinterpret_cast<const d3_weight8 *>(w0), *up = reinterpret_cast<const d3_weight8 *>(w1);
  const char *call = up ? "d3_gated_matmul8" : "d3_matmul8";
  const int device = (int)dev;
  bool ok = true;
  const at::Tensor *x = tensor(a[3], ok), *x_scale = tensor(a[4], ok), *out = tensor(a[5], ok), *scale = tensor(a[6], ok), *status = tensor(a[8], ok);
  if (!ok || !x || !x_scale || x->dim() != 2) return refuse(call, "a and a_scale must be matrices, the others tensors or None");
  const int64_t n = x->size(0), k = w->k, cols = w->n;
  if (n > 0x7fffffff) return refuse(call, "fewer than 2^31 rows");
  d3_matmul8_args args;
  std::memset(&args, 0, sizeof(args));
  args.struct_size = sizeof(args);
  args.n_rows = (int32_t)n;
  Rows r;
  if (!rows_of(*x, n, k, at::kFloat8_e4m3fn, device, r)) return refuse(call, rows_text("a", n, k, "float8_e4m3fn"));
  args.a_dev = r.p; args.a_stride = r.stride;
  if (!rows_of(*x_scale, n, blocks(k), at::kFloat, device, r)) return refuse(call, rows_text("a_scale", n, blocks(k), "fp32"));
  args.a_scale_dev = static_cast<float *>(r.p); args.a_scale_stride = r.stride;
  at::ScalarType type = up ? at::kFloat8_e4m3fn : at::kBFloat16;
  if (out) {
    type = out->scalar_type();
    at::ScalarType said;
    if (a[7] != Py_None && (!type_arg(a[7], said) || said != type)) return refuse(call, "dtype is not out's");
  } else if (a[7] != Py_None && !type_arg(a[7], type)) {
    return refuse(call, "unsupported dtype");
  }
  args.out_dtype = code_of(type);
  const bool eight = type == at::kFloat8_e4m3fn;
  if (args.out_dtype < 0 || (eight && !up)) return refuse(call, up ? "results are float8_e4m3fn, bf16, fp16 or fp32" : "results are bf16, fp16 or fp32");
  if (!eight && scale) return refuse(call, "a scale belongs to results in 8 bits");
  if (out) {
    if (!rows_of(*out, n, cols, type, device, r)) return refuse(call, rows_text("out", n, cols, "a matrix"));
    args.out_dev = r.p; args.out_stride = r.stride;
  }
  if (scale) {
    if (!rows_of(*scale, n, blocks(cols), at::kFloat, device, r)) return refuse(call, rows_text("scale", n, blocks(cols), "fp32"));
    args.scale_dev = static_cast<float *>(r.p); args.scale_stride = r.stride;
  }
  if (status) {
    if (!is_vector(*status, at::kInt, 1, device)) return refuse(call, "status must be an int32 vector of 1");
    args.status_dev = status->data_ptr<int32_t>();
  }
  if (device < 0) return refuse(call, "tensors must be on a CUDA device");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  at::Tensor new_out, new_scale;
  if (!out) {
    new_out = at::empty({n, cols}, x->options().dtype(type));
    args.out_dev = new_out.data_ptr(); args.out_stride = cols;
  }
  if (eight && !scale) {
    new_scale = at::empty({n, blocks(cols)}, x_scale->options());
    args.scale_dev = new_scale.data_ptr<float>(); args.scale_stride = blocks(cols);
  }
  if (n > 0) {
    cudaStream_t st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    const int rc = up ? gated_call(w, up, &args, st) : matmul_call(w, &args, st);
    if (rc != D3_OK) return fail(rc, call);
    if (out) changed(*out);
    if (scale) changed(*scale);
  }
  PyObject *o = result(a[5], new_out);
  if (!up) return o;
  return pack(o, result(a[6], new_scale), nullptr);
  END_HANDLE_TH_ERRORS
}

// logits(logits, history, lengths, prompt, repetition, frequency, presence, bias_ids, bias, masks, mask_of, out, token, status) -> (out, token)
PyObject *logits(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  HANDLE_TH_ERRORS
  static const char *call = "d3_constrain_logits";
  if (argc != 14) return refuse(call, "14 arguments");
  bool ok = true;
  const at::Tensor *t[14];
  for (int i = 0; i < 14; ++i) t[i] = tensor(a[i], ok);
  const at::Tensor *x = t[0], *history = t[1], *ids = t[7], *bias = t[8], *masks = t[9], *mask_of = t[10], *out = t[11], *token = t[12], *status = t[13];
  if (!ok || !x || x->dim() != 2) return refuse(call, "logits must be a matrix, the others tensors or None");
  const int64_t n = x->size(0), vocab = x->size(1);
  const int device = x->get_device(), code = code_of(x->scalar_type());
  if (code < 0 || code == D3_E4M3) return refuse(call, "logits must be bf16, fp16 or fp32");
  if (n > 65535 || vocab < 1 || vocab > (1 << 30)) return refuse(call, "at most 65535 rows of 1..2^30 tokens");
  d3_constrain_logits_args args;
  std::memset(&args, 0, sizeof(args));
  args.struct_size = sizeof(args);
  args.dtype = code; args.n_rows = (int32_t)n; args.vocab = (int32_t)vocab;
  Rows r;
  if (!rows_of(*x, n, vocab, x->scalar_type(), device, r)) return refuse(call, rows_text("logits", n, vocab, "a matrix"));
  args.logits_dev = r.p; args.logits_stride = r.stride;
  if (history) {
    const int64_t m = history->dim() == 2 ? history->size(1) : -1;
    if (m < 0 || m > 0x7fffffff || !rows_of(*history, n, m, at::kInt, device, r)) return refuse(call, rows_text("history", n, m, "int32"));
    args.history_dev = static_cast<int32_t *>(r.p); args.history_stride = r.stride; args.n_history = (int32_t)m;
  }
  static const char *names[] = {"", "", "lengths", "prompt", "repetition", "frequency", "presence"};
  for (int i = 2; i <= 6; ++i) {
    if (!t[i]) continue;
    if (!history) return refuse(call, std::string(names[i]) + " without history");
    if (!is_vector(*t[i], i < 4 ? at::kInt : at::kFloat, n, device))
      return refuse(call, std::string(names[i]) + " must be a contiguous " + (i < 4 ? "int32" : "fp32") + " vector of " + std::to_string(n));
  }
  if (t[2]) args.lengths_dev = t[2]->data_ptr<int32_t>();
  if (t[3]) args.prompt_dev = t[3]->data_ptr<int32_t>();
  if (t[4]) args.repetition_dev = t[4]->data_ptr<float>();
  if (t[5]) args.frequency_dev = t[5]->data_ptr<float>();
  if (t[6]) args.presence_dev = t[6]->data_ptr<float>();
  if ((ids != nullptr) != (bias != nullptr)) return refuse(call, "bias_ids and bias belong together");
  if (ids) {
    const int64_t m = ids->dim() == 2 ? ids->size(1) : -1;
    Rows b;
    if (m < 0 || m > 0x7fffffff || !rows_of(*ids, n, m, at::kInt, device, r)) return refuse(call, rows_text("bias_ids", n, m, "int32"));
    if (!rows_of(*bias, n, m, at::kFloat, device, b) || b.stride != r.stride) return refuse(call, rows_text("bias", n, m, "fp32") + ", of bias_ids' stride");
    args.bias_ids_dev = static_cast<int32_t *>(r.p); args.bias_dev = static_cast<float *>(b.p); args.bias_stride = r.stride; args.n_bias = (int32_t)m;
  }
  if ((masks != nullptr) != (mask_of != nullptr)) return refuse(call, "masks and mask_of belong together");
  if (masks) {
    const int64_t m = masks->dim() == 2 ? masks->size(0) : -1, words = (vocab + 31) / 32;
    if (m < 0 || m > 0x7fffffff || !rows_of(*masks, m, words, at::kInt, device, r)) return refuse(call, rows_text("masks", m, words, "int32"));
    if (!is_vector(*mask_of, at::kInt, n, device)) return refuse(call, "mask_of must be a contiguous int32 vector of " + std::to_string(n));
    // (no masks at all: there is nothing to point at, and every entry of mask_of but -1 is out of range)
    args.masks_dev = m ? static_cast<int32_t *>(r.p) : reinterpret_cast<int32_t *>(mask_of->data_ptr());
    args.mask_stride = r.stride; args.n_masks = (int32_t)m;
    args.mask_of_dev = mask_of->data_ptr<int32_t>();
  }
  if (out) {
    if (!rows_of(*out, n, vocab, x->scalar_type(), device, r)) return refuse(call, rows_text("out", n, vocab, "of logits' type,"));
    args.out_dev = r.p; args.out_stride = r.stride;
  }
  if (token && !is_vector(*token, at::kInt, n, device)) return refuse(call, "token must be a contiguous int32 vector of " + std::to_string(n));
  if (status) {
    if (!is_vector(*status, at::kInt, 1, device)) return refuse(call, "status must be an int32 vector of 1");
    args.status_dev = status->data_ptr<int32_t>();
  }
  if (device < 0) return refuse(call, "tensors must be on a CUDA device");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  at::Tensor new_out, new_token;
  if (!out) {
    new_out = at::empty({n, vocab}, x->options());
    args.out_dev = new_out.data_ptr(); args.out_stride = vocab;
  }
  if (!token) new_token = at::empty({n}, x->options().dtype(at::kInt));
  args.token_dev = token ? token->data_ptr<int32_t>() : new_token.data_ptr<int32_t>();
  if (n > 0) {
    const int rc = logits_call(&args, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
    if (rc != D3_OK) return fail(rc, call);
    if (out) changed(*out);
    if (token) changed(*token);
  }
  PyObject *o = result(a[11], new_out);
  return pack(o, result(a[12], new_token), nullptr);
  END_HANDLE_TH_ERRORS
}

// bind(addresses of d3_add_norm, d3_matmul8, d3_gated_matmul8, d3_constrain_logits, D3Error)
PyObject *bind(PyObject *, PyObject *args) {
  unsigned long long nc, mc, gc, lc;
  PyObject *cls;
  if (!PyArg_ParseTuple(args, "KKKKO", &nc, &mc, &gc, &lc, &cls)) return nullptr;
  norm_call = reinterpret_cast<decltype(norm_call)>(nc);
  matmul_call = reinterpret_cast<decltype(matmul_call)>(mc);
  gated_call = reinterpret_cast<decltype(gated_call)>(gc);
  logits_call = reinterpret_cast<decltype(logits_call)>(lc);
  Py_INCREF(cls);
  Py_XDECREF(error_class);
  error_class = cls;
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_VARARGS, "the library's functions and the error class"},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(norm)), METH_FASTCALL, "d3_add_norm"},
    {"product", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(product)), METH_FASTCALL, "d3_matmul8, d3_gated_matmul8"},
    {"logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(logits)), METH_FASTCALL, "d3_constrain_logits"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_block_call", "calls of the 8-bit block operators", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block_call() { return PyModule_Create(&kModule); }
