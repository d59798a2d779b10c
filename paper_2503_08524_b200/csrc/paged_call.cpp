// Python side of the paged key-value operators: argument checks and marshalling, nothing else.
//
// A decode step of a few rows is bound by the host side of its calls: with the checks in Python an append took 8.4 us
// of host time a call and an attention 10.9, of which the library's own call is 2 to 3.  This module reads the
// tensors' shapes, strides and pointers directly and makes the same C calls (include/d3.h); the library's functions and
// the error class are handed over once by paged.py.
#include <Python.h>

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>
#include <cstring>
#include <string>

#include "d3.h"

namespace {

decltype(&d3_page_plan) plan_call;
decltype(&d3_paged_append) append_call;
decltype(&d3_paged_attention) attention_call;
decltype(&d3_paged_attention_workspace) workspace_call;
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
// a contiguous vector of n entries
bool is_vector(const at::Tensor &t, at::ScalarType type, int64_t n, int device) {
  return t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous() && on(t, device);
}
// [n][heads][dh] with dh contiguous; its strides, those of a dimension of one entry (which torch leaves arbitrary) as if
// the tensor were contiguous there
struct Heads { const void *p; int64_t s0, s1; };
bool heads_of(const at::Tensor &t, int64_t n, int64_t heads, int64_t dh, at::ScalarType type, int device, Heads &out) {
  if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != dh || t.scalar_type() != type || !on(t, device) || t.stride(2) != 1)
    return false;
  out.s1 = heads > 1 ? t.stride(1) : dh;
  out.s0 = n > 1 ? t.stride(0) : heads * out.s1;
  out.p = t.data_ptr();
  return true;
}
std::string shape_text(const char *name, int64_t n, int64_t heads, int64_t dh) {
  return std::string(name) + " must be [" + std::to_string(n) + "][" + std::to_string(heads) + "][" + std::to_string(dh) +
         "] of the call's type and device, last dimension contiguous";
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

// plan(address of the arguments, device, tuple of the tensors written)
PyObject *plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long long at, device;
  if (n != 3 || !PyTuple_Check(a[2])) return refuse("d3_page_plan", "3 arguments");
  if (!number(a[0], at) || !number(a[1], device)) return nullptr;
  if (device < 0) return refuse("d3_page_plan", "tensors must be on a CUDA device");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  const int rc = plan_call(reinterpret_cast<const d3_page_plan_args *>(at), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
  if (rc != D3_OK) return fail(rc, "d3_page_plan");
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[2]); ++i)
    if (THPVariable_Check(PyTuple_GET_ITEM(a[2], i))) changed(THPVariable_Unpack(PyTuple_GET_ITEM(a[2], i)));
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// append(pool, device, k, v, slots, q, q_out, rope, context, status, the pool's K, its V) -> q_out
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  HANDLE_TH_ERRORS
  static const char *call = "d3_paged_append";
  long long pool, dev;
  if (argc != 12) return refuse(call, "12 arguments");
  if (!number(a[0], pool) || !number(a[1], dev)) return nullptr;
  const d3_paged_kv *kv = reinterpret_cast<const d3_paged_kv *>(pool);
  const int device = (int)dev;
  bool ok = true;
  const at::Tensor *k = tensor(a[2], ok), *v = tensor(a[3], ok), *slots = tensor(a[4], ok), *q = tensor(a[5], ok), *q_out = tensor(a[6], ok),
                   *rope = tensor(a[7], ok), *context = tensor(a[8], ok), *status = tensor(a[9], ok), *pool_k = tensor(a[10], ok),
                   *pool_v = tensor(a[11], ok);
  if (!ok || !k || !v || !slots || !pool_k || !pool_v) return refuse(call, "k, v and slots must be tensors, the others tensors or None");
  const int code = code_of(k->scalar_type());
  if (code < 0) return refuse(call, "unsupported type");
  if (slots->dim() != 1 || !is_vector(*slots, at::kLong, slots->size(0), device)) return refuse(call, "slots must be a contiguous int64 vector");
  const int64_t n = slots->size(0), hkv = kv->n_kv_heads, dh = kv->head_dim;
  if (n > 0x7fffffff) return refuse(call, "fewer than 2^31 tokens");
  d3_paged_append_args args;
  std::memset(&args, 0, sizeof(args));
  args.struct_size = sizeof(args);
  args.dtype = code;
  args.n_tokens = (int32_t)n;
  Heads h;
  if (!heads_of(*k, n, hkv, dh, k->scalar_type(), device, h)) return refuse(call, shape_text("k", n, hkv, dh));
  args.k_dev = h.p; args.k_token_stride = h.s0; args.k_head_stride = h.s1;
  if (!heads_of(*v, n, hkv, dh, k->scalar_type(), device, h)) return refuse(call, shape_text("v", n, hkv, dh));
  args.v_dev = h.p; args.v_token_stride = h.s0; args.v_head_stride = h.s1;
  args.slots_dev = slots->data_ptr<int64_t>();
  if (rope) {
    if (rope->scalar_type() != at::kFloat || rope->dim() != 3 || rope->size(1) != dh / 2 || rope->size(2) != 2 || !rope->is_contiguous() ||
        !on(*rope, device) || rope->size(0) > 0x7fffffff)
      return refuse(call, "rope must be contiguous fp32 [positions][" + std::to_string(dh / 2) + "][2]");
    if (!context || !is_vector(*context, at::kInt, n, device)) return refuse(call, "rope needs context, a contiguous int32 vector");
    args.rope_dev = rope->data_ptr<float>();
    args.rope_len = (int32_t)rope->size(0);
    args.context_dev = context->data_ptr<int32_t>();
  }
  at::Tensor fresh;
  if (q) {
    if (!rope) return refuse(call, "q is only rotated, and there is no rope");
    const int64_t hq = q->dim() == 3 ? q->size(1) : -1;
    if (hq < 1 || hq > 0x7fffffff || !heads_of(*q, n, hq, dh, k->scalar_type(), device, h)) return refuse(call, shape_text("q", n, hq, dh));
    args.n_q_heads = (int32_t)hq;
    args.q_dev = h.p; args.q_token_stride = h.s0; args.q_head_stride = h.s1;
    if (!q_out) {
      fresh = at::empty({n, hq, dh}, q->options());
      q_out = &fresh;
    }
    if (!heads_of(*q_out, n, hq, dh, k->scalar_type(), device, h)) return refuse(call, shape_text("q_out", n, hq, dh));
    args.q_out_dev = const_cast<void *>(h.p); args.q_out_token_stride = h.s0; args.q_out_head_stride = h.s1;
  } else if (q_out) {
    return refuse(call, "q_out without q");
  }
  if (status) {
    if (!is_vector(*status, at::kInt, 1, device)) return refuse(call, "status must be an int32 vector of 1");
    args.status_dev = status->data_ptr<int32_t>();
  }
  if (n > 0) {
    if (device < 0) return refuse(call, "tensors must be on a CUDA device");
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    const int rc = append_call(kv, &args, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
    if (rc != D3_OK) return fail(rc, call);
    changed(*pool_k);
    changed(*pool_v);
    if (q_out) changed(*q_out);
  }
  if (fresh.defined()) return THPVariable_Wrap(fresh);
  Py_INCREF(a[6]);
  return a[6];
  END_HANDLE_TH_ERRORS
}

// attention(pool, device, q, table, context, rows, scale, out, lse, with_lse, workspace, status) -> out or (out, lse)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t argc) {
  HANDLE_TH_ERRORS
  static const char *call = "d3_paged_attention";
  long long pool, dev;
  if (argc != 12) return refuse(call, "12 arguments");
  if (!number(a[0], pool) || !number(a[1], dev)) return nullptr;
  const d3_paged_kv *kv = reinterpret_cast<const d3_paged_kv *>(pool);
  const int device = (int)dev;
  bool ok = true;
  const at::Tensor *q = tensor(a[2], ok), *table = tensor(a[3], ok), *context = tensor(a[4], ok), *rows = tensor(a[5], ok), *out = tensor(a[7], ok),
                   *lse = tensor(a[8], ok), *workspace = tensor(a[10], ok), *status = tensor(a[11], ok);
  if (!ok || !q || !table || !context) return refuse(call, "q, table and context must be tensors, the others tensors or None");
  const int code = code_of(q->scalar_type());
  if (code < 0 || q->dim() != 3) return refuse(call, "q must be [n][n_q_heads][head_dim]");
  const int64_t n = q->size(0), hq = q->size(1), dh = kv->head_dim;
  if (n > 0x7fffffff || hq > 0x7fffffff) return refuse(call, "fewer than 2^31 rows and heads");
  d3_paged_attention_args args;
  std::memset(&args, 0, sizeof(args));
  args.struct_size = sizeof(args);
  args.dtype = code;
  args.n_rows = (int32_t)n;
  args.n_q_heads = (int32_t)hq;
  Heads h;
  if (!heads_of(*q, n, hq, dh, q->scalar_type(), device, h)) return refuse(call, shape_text("q", n, hq, dh));
  args.q_dev = h.p; args.q_row_stride = h.s0; args.q_head_stride = h.s1;
  if (table->scalar_type() != at::kInt || table->dim() != 2 || !on(*table, device) || table->size(0) < 1 || table->size(1) < 1 ||
      table->size(0) > 0x7fffffff || table->size(1) > 0x7fffffff || (table->stride(1) != 1 && table->size(1) > 1))
    return refuse(call, "table must be int32 [rows][width] with entries and contiguous rows");
  args.table_dev = table->data_ptr<int32_t>();
  args.table_rows = (int32_t)table->size(0);
  args.table_width = (int32_t)table->size(1);
  args.table_stride = table->size(0) > 1 ? table->stride(0) : table->size(1);
  if (!is_vector(*context, at::kInt, n, device)) return refuse(call, "context must be a contiguous int32 vector of " + std::to_string(n));
  args.context_dev = context->data_ptr<int32_t>();
  if (rows) {
    if (!is_vector(*rows, at::kInt, n, device)) return refuse(call, "rows must be a contiguous int32 vector of " + std::to_string(n));
    args.rows_dev = rows->data_ptr<int32_t>();
  }
  double scale = 1.0 / std::sqrt((double)dh);
  if (a[6] != Py_None) {
    scale = PyFloat_AsDouble(a[6]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
  }
  if (!(std::fabs(scale) < 3e38)) return refuse(call, "scale must be finite");
  args.scale = (float)scale;
  if (status) {
    if (!is_vector(*status, at::kInt, 1, device)) return refuse(call, "status must be an int32 vector of 1");
    args.status_dev = status->data_ptr<int32_t>();
  }
  if (out && !heads_of(*out, n, hq, dh, q->scalar_type(), device, h)) return refuse(call, shape_text("out", n, hq, dh));
  if (lse && (lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != n || lse->size(1) != hq || !lse->is_contiguous() || !on(*lse, device)))
    return refuse(call, "lse must be contiguous fp32 [" + std::to_string(n) + "][" + std::to_string(hq) + "]");
  if (workspace && (!on(*workspace, device) || !workspace->is_contiguous())) return refuse(call, "workspace must be contiguous, on the call's device");
  if (device < 0) return refuse(call, "tensors must be on a CUDA device");
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  at::Tensor new_out, new_lse, new_space;
  if (!out) {
    new_out = at::empty({n, hq, dh}, q->options());
    h = Heads{new_out.data_ptr(), hq * dh, dh};
  }
  args.out_dev = const_cast<void *>(h.p); args.out_row_stride = h.s0; args.out_head_stride = h.s1;
  const int want_lse = lse ? 1 : PyObject_IsTrue(a[9]);
  if (want_lse < 0) return nullptr;
  if (!lse && want_lse) {
    new_lse = at::empty({n, hq}, q->options().dtype(at::kFloat));
    lse = &new_lse;
  }
  if (lse) args.lse_dev = lse->data_ptr<float>();
  if (!workspace) {
    size_t bytes = 0;
    const int rc = workspace_call(kv, args.n_q_heads, &bytes);
    if (rc != D3_OK) return fail(rc, call);
    new_space = at::empty({(int64_t)bytes}, q->options().dtype(at::kByte));
    workspace = &new_space;
  }
  args.workspace_dev = workspace->data_ptr();
  args.workspace_bytes = workspace->nbytes();
  if (n > 0) {
    const int rc = attention_call(kv, &args, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream());
    if (rc != D3_OK) return fail(rc, call);
    if (out) changed(*out);
    if (lse) changed(*lse);
  }
  PyObject *o = new_out.defined() ? THPVariable_Wrap(new_out) : a[7];
  if (!o) return nullptr;
  if (!new_out.defined()) Py_INCREF(o);
  if (!want_lse) return o;
  PyObject *l = new_lse.defined() ? THPVariable_Wrap(new_lse) : a[8];
  if (!l) { Py_DECREF(o); return nullptr; }
  if (!new_lse.defined()) Py_INCREF(l);
  PyObject *both = PyTuple_New(2);
  if (!both) { Py_DECREF(o); Py_DECREF(l); return nullptr; }
  PyTuple_SET_ITEM(both, 0, o);
  PyTuple_SET_ITEM(both, 1, l);
  return both;
  END_HANDLE_TH_ERRORS
}

// bind(addresses of d3_page_plan, d3_paged_append, d3_paged_attention, d3_paged_attention_workspace, D3Error)
PyObject *bind(PyObject *, PyObject *args) {
  unsigned long long p, ap, at, ws;
  PyObject *cls;
  if (!PyArg_ParseTuple(args, "KKKKO", &p, &ap, &at, &ws, &cls)) return nullptr;
  plan_call = reinterpret_cast<decltype(plan_call)>(p);
  append_call = reinterpret_cast<decltype(append_call)>(ap);
  attention_call = reinterpret_cast<decltype(attention_call)>(at);
  workspace_call = reinterpret_cast<decltype(workspace_call)>(ws);
  Py_INCREF(cls);
  Py_XDECREF(error_class);
  error_class = cls;
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_VARARGS, "the library's functions and the error class"},
    {"plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(plan)), METH_FASTCALL, "d3_page_plan"},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(append)), METH_FASTCALL, "d3_paged_append"},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention)), METH_FASTCALL, "d3_paged_attention"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_paged_call", "calls of the paged key-value operators", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_call() { return PyModule_Create(&kModule); }
