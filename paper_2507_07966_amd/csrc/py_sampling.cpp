// Python side of the sampling phase's calls: checks of the tensors, then the C ABI (include/paged_attn.h).
//
// A decode step's calls run for a few microseconds on the GPU, and the checks of ten tensors' types, shapes, devices and strides
// take longer than that in Python (rope_axes_forward 12.1 us a call, paged_attn_forward 16.3 us, both bound by them); here they
// take 0.1 (0.4 with the call in Python; a name looked up in the package for every call, instead of once, adds 3.9).  Every function returns None, or (status, text) of what it refuses; nothing has been enqueued then.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <string>

#include "paged.h"

namespace {

struct Refusal {
  int status;
  std::string text;
};

template <typename... A>
[[noreturn]] void refuse(int status, const A&... parts) {
  std::ostringstream s;
  (s << ... << parts);
  throw Refusal{status, s.str()};
}

std::string list(at::IntArrayRef v) {
  std::ostringstream s;
  s << '[';
  for (size_t i = 0; i < v.size(); ++i) s << (i ? ", " : "") << v[i];
  s << ']';
  return s.str();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PA_ERR_UNSUPPORTED, name, " has to be a tensor");
  return THPVariable_Unpack(o);
}

// What the tensors of a call have in common: `device` is the ordinal, -1 for tensors of a host-only plan.
struct Kind {
  at::ScalarType dtype;
  int device;
};

void check_kind(const at::Tensor& x, const char* name, at::ScalarType dtype, int device) {
  const bool there = device < 0 ? x.device().is_cpu() : x.device().is_cuda() && x.device().index() == device;
  if (x.scalar_type() != dtype || !there || x.layout() != at::kStrided)
    refuse(PA_ERR_UNSUPPORTED, name, " has to be ", c10::toString(dtype), device < 0 ? " on the CPU" : " on GPU ", device < 0 ? "" : std::to_string(device),
           ", not ", c10::toString(x.scalar_type()), " on ", x.device().str());
}

// A contiguous tensor of this shape.
void* array(PyObject* o, const char* name, std::initializer_list<int64_t> shape, at::ScalarType dtype, int device) {
  const at::Tensor& x = tensor(o, name);
  check_kind(x, name, dtype, device);
  if (x.sizes() != at::IntArrayRef(shape) || !x.is_contiguous())
    refuse(PA_ERR_SHAPE, name, " has to be a contiguous ", list(at::IntArrayRef(shape)), ", not ", list(x.sizes()), " of strides ", list(x.strides()));
  return x.data_ptr();
}

// [tokens, heads, dim] with each token's heads contiguous.
struct Rows {
  void* ptr;
  int64_t stride;
};
Rows rows(PyObject* o, const char* name, int64_t tokens, int64_t heads, int64_t dim, const Kind& k) {
  const at::Tensor& x = tensor(o, name);
  check_kind(x, name, k.dtype, k.device);
  const int64_t shape[3] = {tokens, heads, dim};
  if (x.sizes() != at::IntArrayRef(shape)) refuse(PA_ERR_SHAPE, name, " has to be ", list(at::IntArrayRef(shape)), ", not ", list(x.sizes()));
  if (tokens && heads && (x.stride(2) != 1 || (heads > 1 && x.stride(1) != dim)))
    refuse(PA_ERR_SHAPE, name, "'s heads have to be contiguous, its strides are ", list(x.strides()));
  return {x.data_ptr(), tokens > 1 ? x.stride(0) : heads * dim};
}

void* address(PyObject* o) {
  if (o == Py_None) return nullptr;
  void* p = PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) throw Refusal{-1, ""};
  return p;
}

// The plan, and what its tensors are.
struct Call {
  const paged_attn_plan_t* plan;
  Kind kind;
  explicit Call(PyObject* handle) : plan(static_cast<const paged_attn_plan_t*>(address(handle))) {
    if (!plan) refuse(PA_ERR_NULL, "no plan");
    kind = {plan->desc.dtype == PA_BF16 ? at::kBFloat16 : at::kFloat, plan->desc.device};
  }
};

// k_cache, v_cache, page_table, seq_lens, cu_new
struct Cache {
  void *k, *v;
  const int32_t *table, *lens, *cu;
  int32_t seqs;
  Cache(const Call& c, PyObject* const* o) {
    const paged_attn_desc_t& d = c.plan->desc;
    const at::Tensor& l = tensor(o[3], "seq_lens");
    if (l.dim() != 1 || l.size(0) > d.max_seqs) refuse(PA_ERR_SHAPE, "seq_lens has to be a list of at most ", d.max_seqs, ", not ", list(l.sizes()));
    const int64_t n = l.size(0);
    seqs = (int32_t)n;
    k = array(o[0], "k_cache", {d.num_pages, d.num_kv_heads, d.page_size, d.head_dim}, c.kind.dtype, c.kind.device);
    v = array(o[1], "v_cache", {d.num_pages, d.num_kv_heads, d.page_size, d.head_dim}, c.kind.dtype, c.kind.device);
    table = static_cast<const int32_t*>(array(o[2], "page_table", {n, d.max_pages_per_seq}, at::kInt, c.kind.device));
    lens = static_cast<const int32_t*>(array(o[3], "seq_lens", {n}, at::kInt, c.kind.device));
    cu = static_cast<const int32_t*>(array(o[4], "cu_new", {n + 1}, at::kInt, c.kind.device));
  }
};

int64_t first_size(const at::Tensor& x, const char* name) {
  if (x.dim() != 3) refuse(PA_ERR_SHAPE, name, " has to be [tokens, heads, channels], not ", list(x.sizes()));
  return x.size(0);
}

// (backward, rope, q, k, positions, inv_freq, q_out, k_out, stream); rope: the address of a rope_axes_desc_t
int rope_call(PyObject* const* o) {
  const rope_axes_desc_t* d = static_cast<const rope_axes_desc_t*>(address(o[1]));
  const at::Tensor& q = tensor(o[2], "q");
  const int64_t tokens = first_size(q, "q"), hq = q.size(1);
  if (q.scalar_type() != at::kFloat && q.scalar_type() != at::kBFloat16)
    refuse(PA_ERR_UNSUPPORTED, "q has to be Float or BFloat16, not ", c10::toString(q.scalar_type()));
  if (!q.device().is_cuda() || q.device() != c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice())
    refuse(PA_ERR_UNSUPPORTED, "tensors have to be on the current GPU, not on ", q.device().str());
  const Kind kind{q.scalar_type(), q.device().index()};
  const Rows rq = rows(o[2], "q", tokens, hq, d->head_dim, kind), rqo = rows(o[6], "q_out", tokens, hq, d->head_dim, kind);
  Rows rk{nullptr, 0}, rko{nullptr, 0};
  int64_t hk = 0;
  if ((o[3] == Py_None) != (o[7] == Py_None)) refuse(PA_ERR_SHAPE, "k and k_out go together");
  if (o[3] != Py_None) {
    const at::Tensor& k = tensor(o[3], "k");
    first_size(k, "k");
    hk = k.size(1);
    rk = rows(o[3], "k", tokens, hk, d->head_dim, kind);
    rko = rows(o[7], "k_out", tokens, hk, d->head_dim, kind);
  }
  if (hq > 65536 || hk > 65536) refuse(PA_ERR_SHAPE, "too many heads");
  const int32_t* pos = static_cast<const int32_t*>(array(o[4], "positions", {d->num_axes, tokens}, at::kInt, kind.device));
  const float* freq = static_cast<const float*>(array(o[5], "inv_freq", {d->rotary_dim / 2}, at::kFloat, kind.device));
  const auto call = o[0] == Py_True ? rope_axes_backward : rope_axes_forward;
  return call(d, kind.dtype == at::kBFloat16 ? PA_BF16 : PA_F32, rq.ptr, rq.stride, rk.ptr, rk.stride, tokens, (int32_t)hq, (int32_t)hk, pos, freq,
              rqo.ptr, rqo.stride, rko.ptr, rko.stride, address(o[8]));
}

// (plan, rope or None, q or None, k, v, positions, inv_freq, q_out, k_cache, v_cache, page_table, seq_lens, cu_new, stream)
int append_call(PyObject* const* o) {
  const Call c(o[0]);
  const paged_attn_desc_t& d = c.plan->desc;
  const Cache cache(c, o + 8);
  const int64_t tokens = first_size(tensor(o[3], "k"), "k");
  const Rows k = rows(o[3], "k", tokens, d.num_kv_heads, d.head_dim, c.kind), v = rows(o[4], "v", tokens, d.num_kv_heads, d.head_dim, c.kind);
  void* stream = address(o[13]);
  if (o[1] == Py_None)
    return paged_kv_append(c.plan, k.ptr, k.stride, v.ptr, v.stride, cache.k, cache.v, cache.table, cache.lens, cache.cu, cache.seqs, tokens, stream);
  const rope_axes_desc_t* r = static_cast<const rope_axes_desc_t*>(address(o[1]));
  if (r->head_dim != d.head_dim) refuse(PA_ERR_SHAPE, "the rotation is of heads of ", r->head_dim, " channels, the plan's have ", d.head_dim);
  if ((o[2] == Py_None) != (o[7] == Py_None)) refuse(PA_ERR_SHAPE, "q and q_out go together");
  Rows q{nullptr, 0}, qo{nullptr, 0};
  if (o[2] != Py_None) {
    q = rows(o[2], "q", tokens, d.num_q_heads, d.head_dim, c.kind);
    qo = rows(o[7], "q_out", tokens, d.num_q_heads, d.head_dim, c.kind);
  }
  const int32_t* pos = static_cast<const int32_t*>(array(o[5], "positions", {r->num_axes, tokens}, at::kInt, c.kind.device));
  const float* freq = static_cast<const float*>(array(o[6], "inv_freq", {r->rotary_dim / 2}, at::kFloat, c.kind.device));
  return paged_kv_append_rope(c.plan, r, q.ptr, q.stride, k.ptr, k.stride, v.ptr, v.stride, pos, freq, qo.ptr, qo.stride, cache.k, cache.v,
                              cache.table, cache.lens, cache.cu, cache.seqs, tokens, stream);
}

// (plan, q, k_cache, v_cache, page_table, seq_lens, cu_new, out, lse_out or None, workspace, shared_len or None, stream)
int attend_call(PyObject* const* o) {
  const Call c(o[0]);
  const paged_attn_desc_t& d = c.plan->desc;
  const Cache cache(c, o + 2);
  const int64_t tokens = first_size(tensor(o[1], "q"), "q");
  const Rows q = rows(o[1], "q", tokens, d.num_q_heads, d.head_dim, c.kind);
  void* out = array(o[7], "out", {tokens, d.num_q_heads, d.head_dim}, c.kind.dtype, c.kind.device);
  float* lse = o[8] == Py_None ? nullptr : static_cast<float*>(array(o[8], "lse_out", {d.num_q_heads, tokens}, at::kFloat, c.kind.device));
  const int32_t* shared = o[10] == Py_None ? nullptr : static_cast<const int32_t*>(array(o[10], "shared_len", {1}, at::kInt, c.kind.device));
  const at::Tensor& ws = tensor(o[9], "workspace");
  check_kind(ws, "workspace", ws.scalar_type(), c.kind.device);
  if (!ws.is_contiguous()) refuse(PA_ERR_SHAPE, "workspace has to be contiguous");
  return paged_attn_forward(c.plan, q.ptr, q.stride, cache.k, cache.v, cache.table, cache.lens, cache.cu, cache.seqs, tokens, shared, out, lse,
                            ws.data_ptr(), ws.nbytes(), address(o[11]));
}

template <int (*CALL)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", N, n);
    return nullptr;
  }
  try {
    const int st = CALL(args);
    if (st == PA_OK) Py_RETURN_NONE;
    return Py_BuildValue("is", st, "");
  } catch (const Refusal& r) {
    if (r.status < 0) return nullptr;  // a Python error is set
    return Py_BuildValue("is", r.status, r.text.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<rope_call, 9>)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<append_call, 14>)), METH_FASTCALL, nullptr},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<attend_call, 12>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sampling", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sampling() { return PyModule_Create(&module); }
