// The operators' calls from Python in one step each: checks, output tensors, stream and the C entry point.  A decoding
// step makes hundreds of such calls of a few microseconds each; made through ctypes and Python checks a call took
// 12 us of host time.  Every function returns its result, or the admmq_status of the check or call that failed as an
// int; adapt.py then repeats the call on its own path, which words the error.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>

#include "../../include/admmq_cache.h"

namespace {

using at::Tensor;

struct Refused {                       // a check or call that failed
  int status;
};
void need(bool ok, int status = ADMMQ_ERR_INVALID_ARG) {
  if (!ok) throw Refused{status};
}
const Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o));
  return THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  need(v != -1 || !PyErr_Occurred());
  return v;
}
template <class T>
T* pointer(PyObject* o) {
  return reinterpret_cast<T*>(static_cast<uintptr_t>(integer(o)));
}
bool on(const Tensor& t, at::ScalarType type, int index) {
  return t.is_cuda() && t.get_device() == index && t.scalar_type() == type;
}
Tensor make(at::IntArrayRef size, at::ScalarType type, int index) {
  return at::detail::empty_cuda(size, type, c10::Device(c10::kCUDA, static_cast<c10::DeviceIndex>(index)), std::nullopt);
}
// A device made current for the call, if it is not.
struct Current {
  std::optional<c10::cuda::CUDAGuard> guard;
  void* stream;
  explicit Current(int index) {
    if (c10::cuda::current_device() != index) guard.emplace(static_cast<c10::DeviceIndex>(index));
    stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(index)).stream();
  }
};
// An input that requires grad, with grad mode on: a graph that would end here.
bool in_a_graph(const Tensor& t) { return t.requires_grad() && c10::GradMode::is_enabled(); }
// A [rows, width] bf16 tensor of adjacent values; returns its row stride (that of a single row does not matter).
long long rows_of(const Tensor& t, long long width, int index) {
  need(t.dim() == 2 && on(t, at::kBFloat16, index));
  need(t.size(1) == width && (t.size(0) == 0 || t.stride(1) == 1), ADMMQ_ERR_SHAPE);
  return t.size(0) > 1 ? t.stride(0) : width;
}
// A tuple of tensors; an undefined one is None.
PyObject* tuple_of(std::initializer_list<Tensor> tensors) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(tensors.size()));
  Py_ssize_t i = 0;
  for (const Tensor& t : tensors) {
    PyObject* o = r ? THPVariable_Wrap(t) : nullptr;       // (an undefined tensor wraps as None)
    if (!o) {
      Py_XDECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}
PyObject* status_of(const Refused& r) {
  PyErr_Clear();
  return PyLong_FromLong(r.status);
}

// linear(grad, layer, d_in, d_out, device, status, x) or
// linear(grad, layer, d_in, d_out, device, status, x, bank, rank, n_rows, row_adapter, down, up, scale) -> (y, h or None)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 7 || n == 14);
    const bool grad = a[0] == Py_True;
    const auto* layer = pointer<const admmq_packed_layer>(a[1]);
    const long long d_in = integer(a[2]), d_out = integer(a[3]), k = grad ? d_out : d_in, m = grad ? d_in : d_out;
    const int index = static_cast<int>(integer(a[4]));
    int* status = pointer<int>(a[5]);
    const Tensor& x = tensor(a[6]);
    const long long ld = rows_of(x, k, index), t = x.size(0);
    need(grad || !in_a_graph(x));
    const auto call = grad ? admmq_linear_grad_input : admmq_linear_forward;
    const Current on_device(index);
    const Tensor y = make({t, m}, at::kBFloat16, index);
    if (n == 7) {
      const int st = call(layer, nullptr, t, nullptr, x.const_data_ptr(), ld, y.mutable_data_ptr(), m, nullptr, status,
                          on_device.stream);
      need(st == ADMMQ_OK, st);
      return tuple_of({y, Tensor()});
    }
    need(integer(a[9]) == t, ADMMQ_ERR_SHAPE);
    const auto* bank = pointer<const admmq_adapters>(a[7]);
    need(tensor(a[11]).const_data_ptr() == bank->d_down && tensor(a[12]).const_data_ptr() == bank->d_up &&
         tensor(a[13]).const_data_ptr() == bank->d_scale);
    const Tensor h = make({t, integer(a[8])}, at::kFloat, index);
    const int st = call(layer, bank, t, pointer<const int>(a[10]), x.const_data_ptr(), ld,
                        y.mutable_data_ptr(), m, static_cast<float*>(h.mutable_data_ptr()), status, on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({y, h});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// adapter_grad(device, n_rows, order, offsets, x, codes, scale, h, dy, u, down, up) -> (grad_down, grad_up); x or
// codes and scale are None
PyObject* adapter_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 12);
    const int index = static_cast<int>(integer(a[0]));
    admmq_adapter_grad_args g = {};
    g.struct_size = sizeof(g);
    g.n_rows = integer(a[1]);
    g.d_order = pointer<const int>(a[2]);
    g.d_offsets = pointer<const int>(a[3]);
    const Tensor &h = tensor(a[7]), &dy = tensor(a[8]), &u = tensor(a[9]), &down = tensor(a[10]), &up = tensor(a[11]);
    g.n_adapters = static_cast<int>(down.size(0));
    g.rank = static_cast<int>(down.size(1));
    g.d_in = static_cast<int>(down.size(2));
    g.d_out = static_cast<int>(up.size(2));
    if (a[4] != Py_None) {
      const Tensor& x = tensor(a[4]);
      g.ldx = rows_of(x, g.d_in, index);
      need(x.size(0) == g.n_rows, ADMMQ_ERR_SHAPE);
      g.d_x = x.const_data_ptr();
    } else {
      const Tensor &codes = tensor(a[5]), &scale = tensor(a[6]);
      need(on(codes, at::kChar, index) && on(scale, at::kFloat, index));
      need(codes.dim() == 2 && codes.size(0) == g.n_rows && codes.size(1) == g.d_in, ADMMQ_ERR_SHAPE);
      g.d_x_codes = static_cast<const signed char*>(codes.const_data_ptr());
      g.d_x_scale = static_cast<const float*>(scale.const_data_ptr());
    }
    for (const Tensor* f : {&h, &u}) {
      need(on(*f, at::kFloat, index) && f->is_contiguous());
      need(f->dim() == 2 && f->size(0) == g.n_rows && f->size(1) == g.rank, ADMMQ_ERR_SHAPE);
    }
    g.d_h = static_cast<const float*>(h.const_data_ptr());
    g.d_u = static_cast<const float*>(u.const_data_ptr());
    g.lddy = rows_of(dy, g.d_out, index);
    need(dy.size(0) == g.n_rows, ADMMQ_ERR_SHAPE);
    g.d_dy = dy.const_data_ptr();
    const Current on_device(index);
    const Tensor gd = make(down.sizes(), at::kBFloat16, index), gu = make(up.sizes(), at::kBFloat16, index);
    g.d_grad_down = gd.mutable_data_ptr();
    g.d_grad_up = gu.mutable_data_ptr();
    const int st = admmq_adapter_grad(&g, on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({gd, gu});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// checkpoint_save(x) -> (codes, scale)
PyObject* checkpoint_save(PyObject*, PyObject* o) {
  HANDLE_TH_ERRORS
  try {
    const Tensor& x = tensor(o);
    const bool bf16 = x.scalar_type() == at::kBFloat16;
    need(x.dim() == 2 && x.is_cuda() && (bf16 || x.scalar_type() == at::kFloat));
    const long long t = x.size(0), n = x.size(1);
    need(n <= (1 << 20) && (t == 0 || x.stride(1) == 1), ADMMQ_ERR_SHAPE);
    const int index = static_cast<int>(x.get_device());
    const Current on_device(index);
    const Tensor codes = make({t, n}, at::kChar, index);
    const Tensor scale = make({t, (n + ADMMQ_CHECKPOINT_BLOCK - 1) / ADMMQ_CHECKPOINT_BLOCK}, at::kFloat, index);
    const int st = admmq_checkpoint_save(x.const_data_ptr(), bf16 ? ADMMQ_BF16 : ADMMQ_F32, t, static_cast<int>(n),
                                         t > 1 ? x.stride(0) : n, static_cast<signed char*>(codes.mutable_data_ptr()),
                                         static_cast<float*>(scale.mutable_data_ptr()), on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({codes, scale});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// checkpoint_restore(codes, scale, bf16) -> out; codes and scale as Checkpoint holds them
PyObject* checkpoint_restore(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 3);
    const Tensor &codes = tensor(a[0]), &scale = tensor(a[1]);
    const bool bf16 = a[2] == Py_True;
    const int index = static_cast<int>(codes.get_device());
    const long long t = codes.size(0), w = codes.size(1);
    const Current on_device(index);
    const Tensor out = make({t, w}, bf16 ? at::kBFloat16 : at::kFloat, index);
    const int st = admmq_checkpoint_restore(static_cast<const signed char*>(codes.const_data_ptr()),
                                            static_cast<const float*>(scale.const_data_ptr()), t, static_cast<int>(w),
                                            out.mutable_data_ptr(), bf16 ? ADMMQ_BF16 : ADMMQ_F32, w, on_device.stream);
    need(st == ADMMQ_OK, st);
    return THPVariable_Wrap(out);
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// Row and head strides of a [rows, heads, dim] tensor; those that a single row or head never uses are 0.
void heads_of(const Tensor& x, long long t, long long heads, long long d, at::ScalarType type, int index, long long* row,
              long long* head) {
  need(on(x, type, index));
  need(x.dim() == 3 && x.size(0) == t && x.size(1) == heads && x.size(2) == d, ADMMQ_ERR_SHAPE);
  need(x.stride(2) == 1 || x.numel() == 0, ADMMQ_ERR_SHAPE);
  *row = t > 1 ? x.stride(0) : 0;
  *head = heads > 1 ? x.stride(1) : 0;
}

// qk(status, q, k, wq, wk, cos, sin, positions, eps) -> (q', k'), with two more, dq and dk: -> four gradients
PyObject* qk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 9 || n == 11);
    const bool back = n == 11;
    const Tensor &q = tensor(a[1]), &k = tensor(a[2]), &wq = tensor(a[3]), &wk = tensor(a[4]), &cos = tensor(a[5]),
                 &sin = tensor(a[6]), &pos = tensor(a[7]);
    const at::ScalarType type = q.scalar_type();
    need(q.is_cuda() && (type == at::kBFloat16 || type == at::kFloat));
    need(back || !(in_a_graph(q) || in_a_graph(k)));
    need(q.dim() == 3 && k.dim() == 3, ADMMQ_ERR_SHAPE);
    const int index = static_cast<int>(q.get_device());
    const long long t = q.size(0), hq = q.size(1), hk = k.size(1), d = q.size(2);
    need(hq <= 65536 && hk <= 65536 && d <= 256, ADMMQ_ERR_SHAPE);
    admmq_qk_args g = {};
    g.struct_size = sizeof(g);
    g.dtype = type == at::kBFloat16 ? ADMMQ_BF16 : ADMMQ_F32;
    g.q_heads = static_cast<int>(hq);
    g.k_heads = static_cast<int>(hk);
    g.head_dim = static_cast<int>(d);
    g.n_rows = t;
    g.eps = PyFloat_AsDouble(a[8]);
    need(g.eps != -1.0 || !PyErr_Occurred());
    heads_of(q, t, hq, d, type, index, &g.q_row, &g.q_head);
    heads_of(k, t, hk, d, type, index, &g.k_row, &g.k_head);
    for (const Tensor* w : {&wq, &wk}) {
      need(on(*w, type, index) && w->is_contiguous());
      need(w->dim() == 1 && w->size(0) == d, ADMMQ_ERR_SHAPE);
    }
    for (const Tensor* c : {&cos, &sin}) need(on(*c, at::kFloat, index) && c->is_contiguous());
    need(cos.dim() == 2 && cos.sizes() == sin.sizes() && cos.size(1) <= 128, ADMMQ_ERR_SHAPE);
    need(on(pos, at::kInt, index) && pos.is_contiguous());
    need(pos.dim() == 1 && pos.size(0) == t, ADMMQ_ERR_SHAPE);
    g.rot_dim = static_cast<int>(2 * cos.size(1));
    g.n_positions = cos.size(0);
    g.d_q = q.const_data_ptr();
    g.d_k = k.const_data_ptr();
    g.d_wq = wq.const_data_ptr();
    g.d_wk = wk.const_data_ptr();
    g.d_cos = static_cast<const float*>(cos.const_data_ptr());
    g.d_sin = static_cast<const float*>(sin.const_data_ptr());
    g.d_pos = static_cast<const int*>(pos.const_data_ptr());
    g.d_status = pointer<int>(a[0]);
    const Current on_device(index);
    const Tensor oq = make({t, hq, d}, type, index), ok = make({t, hk, d}, type, index);
    g.d_out_q = oq.mutable_data_ptr();
    g.d_out_k = ok.mutable_data_ptr();
    g.out_q_row = hq * d;
    g.out_k_row = hk * d;
    g.out_q_head = g.out_k_head = d;
    if (!back) {
      const int st = admmq_qk_norm_rope(&g, on_device.stream);
      need(st == ADMMQ_OK, st);
      return tuple_of({oq, ok});
    }
    const Tensor &dq = tensor(a[9]), &dk = tensor(a[10]);
    heads_of(dq, t, hq, d, type, index, &g.dy_q_row, &g.dy_q_head);
    heads_of(dk, t, hk, d, type, index, &g.dy_k_row, &g.dy_k_head);
    g.d_dy_q = dq.const_data_ptr();
    g.d_dy_k = dk.const_data_ptr();
    const Tensor gq = make({d}, type, index), gk = make({d}, type, index);
    g.d_grad_wq = gq.mutable_data_ptr();
    g.d_grad_wk = gk.mutable_data_ptr();
    g.workspace_bytes = admmq_qk_workspace_bytes(g.head_dim);
    need(g.workspace_bytes > 0, ADMMQ_ERR_SHAPE);
    const Tensor work = make({static_cast<long long>(g.workspace_bytes)}, at::kByte, index);
    g.d_workspace = work.mutable_data_ptr();
    const int st = admmq_qk_norm_rope_backward(&g, on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({oq, ok, gq, gk});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// The cache and the plan of a call, if their tensors are where they were: a[1] cache, a[2] plan, a[3..4] codes and scale,
// a[5..6] tables and held.
struct CacheCall {
  const admmq_cache* cache;
  const admmq_cache_plan* plan;
  int* status;
  int index;
  explicit CacheCall(PyObject* const* a) {
    status = pointer<int>(a[0]);
    cache = pointer<const admmq_cache>(a[1]);
    plan = pointer<const admmq_cache_plan>(a[2]);
    const Tensor &codes = tensor(a[3]), &tables = tensor(a[5]);
    need(codes.const_data_ptr() == cache->d_codes && tensor(a[4]).const_data_ptr() == cache->d_scale);
    need(tables.const_data_ptr() == plan->d_tables && tensor(a[6]).const_data_ptr() == plan->d_held);
    index = static_cast<int>(codes.get_device());
    need(tables.is_cuda() && tables.get_device() == index);
  }
};

// cache_write(status, cache, plan, codes, scale, tables, held, k, v) -> None
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 9);
    const CacheCall c(a);
    const Tensor &k = tensor(a[7]), &v = tensor(a[8]);
    const at::ScalarType type = k.scalar_type();
    need(type == at::kBFloat16 || type == at::kFloat);
    need(!in_a_graph(k) && !in_a_graph(v));
    long long kr, kh, vr, vh;
    heads_of(k, c.plan->n_rows, c.cache->kv_heads, c.cache->head_dim, type, c.index, &kr, &kh);
    heads_of(v, c.plan->n_rows, c.cache->kv_heads, c.cache->head_dim, type, c.index, &vr, &vh);
    const Current on_device(c.index);
    const int st = admmq_cache_write(c.cache, c.plan, type == at::kFloat ? ADMMQ_F32 : ADMMQ_BF16, k.const_data_ptr(), kr, kh,
                                     v.const_data_ptr(), vr, vh, c.status, on_device.stream);
    need(st == ADMMQ_OK, st);
    Py_RETURN_NONE;
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// cache_read(status, cache, plan, codes, scale, tables, held, bf16) -> (k, v)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 8);
    const CacheCall c(a);
    const bool bf16 = a[7] == Py_True;
    const long long h = c.cache->kv_heads, d = c.cache->head_dim;
    const Current on_device(c.index);
    const Tensor k = make({c.plan->n_rows, h, d}, bf16 ? at::kBFloat16 : at::kFloat, c.index);
    const Tensor v = make({c.plan->n_rows, h, d}, bf16 ? at::kBFloat16 : at::kFloat, c.index);
    const int st = admmq_cache_read(c.cache, c.plan, bf16 ? ADMMQ_BF16 : ADMMQ_F32, k.mutable_data_ptr(), h * d, d,
                                    v.mutable_data_ptr(), h * d, d, c.status, on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({k, v});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

// cache_attend(status, cache, plan, codes, scale, tables, held, q, softmax scale, window) -> (out, lse)
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    need(n == 10);
    const CacheCall c(a);
    const Tensor& q = tensor(a[7]);
    const double scale = PyFloat_AsDouble(a[8]);
    need(scale != -1.0 || !PyErr_Occurred());
    const long long window = integer(a[9]), rows = c.plan->n_rows, heads = (long long)c.cache->kv_heads * c.plan->group,
                    d = c.cache->head_dim;
    need(window >= 0 && window <= 0x7fffffff);
    need(!in_a_graph(q));
    long long qr, qh;
    heads_of(q, rows, heads, d, at::kBFloat16, c.index, &qr, &qh);
    const Current on_device(c.index);
    const Tensor out = make({rows, heads, d}, at::kBFloat16, c.index), lse = make({rows, heads}, at::kFloat, c.index);
    const size_t bytes = admmq_cache_attend_workspace(c.cache, c.plan);
    const Tensor work = make({static_cast<long long>(bytes < 16 ? 16 : bytes)}, at::kByte, c.index);
    const int st = admmq_cache_attend(c.cache, c.plan, scale, static_cast<int>(window), q.const_data_ptr(), qr, qh,
                                      out.mutable_data_ptr(), heads * d, d, static_cast<float*>(lse.mutable_data_ptr()),
                                      work.mutable_data_ptr(), bytes, c.status, on_device.stream);
    need(st == ADMMQ_OK, st);
    return tuple_of({out, lse});
  } catch (const Refused& r) {
    return status_of(r);
  }
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"adapter_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(adapter_grad)), METH_FASTCALL, nullptr},
    {"checkpoint_save", checkpoint_save, METH_O, nullptr},
    {"checkpoint_restore", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(checkpoint_restore)), METH_FASTCALL,
     nullptr},
    {"qk", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk)), METH_FASTCALL, nullptr},
    {"cache_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_write)), METH_FASTCALL, nullptr},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, nullptr},
    {"cache_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attend)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_adapt", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__adapt() { return PyModule_Create(&module); }
