// Python entry points of the calls that a decode step makes once per layer (8-bit cache, sampling): argument checks, result
// memory and the current stream handled here, so that the host side of a call is a few microseconds.  The work itself is
// the C ABI's; binding.py holds the signatures and their documentation.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/as_strided_native.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "edgeshard.h"

namespace {

PyObject* g_error = nullptr;                  // binding.EsError
PyObject* g_out_of_memory = nullptr;          // torch.cuda.OutOfMemoryError

struct Refusal {
  int status;
  std::string message;
};

[[noreturn]] void refuse(std::string message) { throw Refusal{ES_ERR_INVALID_ARG, std::move(message)}; }

struct PythonError {};                        // an exception is already set

// ---- arguments ---------------------------------------------------------------------------------

const at::Tensor* maybe_tensor(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
  return &THPVariable_Unpack(o);
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  const at::Tensor* t = maybe_tensor(o, name);
  if (!t) refuse(std::string(name) + " must be a tensor");
  return *t;
}

int int_arg(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  if (v < INT32_MIN || v > INT32_MAX) throw Refusal{ES_ERR_RANGE, std::string(name) + " does not fit 32 bits"};
  return (int)v;
}

struct Named {
  const at::Tensor* t;
  const char* name;
};

// The stream to launch on.  The library launches on the current device: everything has to be there.
cudaStream_t launch_stream(std::initializer_list<Named> tensors) {
  const int current = (int)c10::cuda::current_device();
  for (const Named& n : tensors) {
    if (!n.t) continue;
    if (!n.t->is_cuda()) refuse(std::string(n.name) + " must be a CUDA tensor");
    if (n.t->get_device() != current)
      refuse(std::string(n.name) + " is on cuda:" + std::to_string(n.t->get_device()) + ", the current device is cuda:" + std::to_string(current));
  }
  return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)current).stream();
}

void need_cuda_first(const at::Tensor& t, const char* name) {      // before anything asks the CUDA runtime
  if (!t.is_cuda()) refuse(std::string(name) + " must be a CUDA tensor");
}

void need_ints(std::initializer_list<Named> tensors) {
  for (const Named& n : tensors)
    if (n.t && (n.t->scalar_type() != at::kInt || !n.t->is_contiguous())) refuse(std::string(n.name) + " must be a contiguous int32 tensor");
}

int value_dtype(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kHalf: return ES_DTYPE_F16;
    case at::kBFloat16: return ES_DTYPE_BF16;
    case at::kFloat: return ES_DTYPE_F32;
    default: return -1;
  }
}

at::ScalarType scalar_of(int dtype) { return dtype == ES_DTYPE_F16 ? at::kHalf : dtype == ES_DTYPE_BF16 ? at::kBFloat16 : at::kFloat; }

struct Pool {
  int n_pages, Hkv, P, hd, code;
};

int fit(int64_t v, const char* what) {
  if (v > INT32_MAX) throw Refusal{ES_ERR_RANGE, std::string(what) + " does not fit 32 bits"};
  return (int)v;
}

Pool check_pool(const at::Tensor& k, const at::Tensor& v, const at::Tensor& ks, const at::Tensor& vs) {
  if (k.dim() != 4 || v.sizes() != k.sizes()) refuse("k_pages and v_pages must be [n_pages, Hkv, P, hd] of one shape");
  int code = -1;
  if (k.scalar_type() == at::kChar) code = ES_DTYPE_I8;
  if (k.scalar_type() == at::kFloat8_e4m3fn) code = ES_DTYPE_F8E4M3;
  if (code < 0 || v.scalar_type() != k.scalar_type()) refuse("pages must be int8 or float8_e4m3fn, both the same");
  if (!k.is_contiguous() || !v.is_contiguous()) refuse("pages must be contiguous");
  for (const at::Tensor* s : {&ks, &vs})
    if (s->scalar_type() != at::kFloat || !s->is_contiguous() || s->dim() != 2 || s->size(0) != k.size(0) || s->size(1) != k.size(1))
      refuse("k_scale and v_scale must be contiguous fp32 [n_pages, Hkv]");
  return Pool{fit(k.size(0), "n_pages"), fit(k.size(1), "Hkv"), fit(k.size(2), "page_tokens"), fit(k.size(3), "hd"), code};
}

// Elements from row to row of [..., heads, hd] whose last two dimensions are dense and whose leading ones, if several,
// step evenly: a slice of a fused projection's output is such a tensor.
int64_t row_stride(const at::Tensor& t, const char* name) {
  const auto size = t.sizes(), stride = t.strides();
  const int n = (int)size.size();
  if (stride[n - 1] != 1 || (stride[n - 2] != size[n - 1] && size[n - 2] != 1)) refuse(std::string("the heads of a row of ") + name + " must be contiguous");
  int64_t step = 0, span = 0;
  for (int i = n - 3; i >= 0; --i) {
    if (size[i] == 1) continue;
    if (stride[i] <= 0) refuse(std::string("the rows of ") + name + " must lie one after the other (no expanded dimensions)");
    if (span && stride[i] != span) refuse(std::string("the rows of ") + name + " must be evenly spaced");
    if (!step) step = stride[i];
    span = stride[i] * size[i];
  }
  return step ? step : size[n - 1] * size[n - 2];
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dtype, const at::Tensor& like) {
  return at::empty(shape, at::TensorOptions().dtype(dtype).device(like.device()));
}

// The call itself, other Python threads running meanwhile.
template <class F>
void call(F f) {
  es_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  if (st != ES_OK) throw Refusal{(int)st, es_last_error()};
}

// ---- entry points ------------------------------------------------------------------------------

PyObject* kv_plan(PyObject* const* a) {
  const at::Tensor &old_len = tensor(a[0], "old_len"), &new_len = tensor(a[1], "new_len"), &table = tensor(a[2], "block_table");
  const int P = int_arg(a[3], "page_tokens"), max_rows = int_arg(a[4], "max_rows");
  const at::Tensor *free_pages = maybe_tensor(a[5], "free_pages"), *free_count = maybe_tensor(a[6], "free_count");
  if (!free_pages != !free_count) refuse("free_pages and free_count go together");
  need_cuda_first(old_len, "old_len");
  cudaStream_t stream = launch_stream({{&old_len, "old_len"}, {&new_len, "new_len"}, {&table, "block_table"}, {free_pages, "free_pages"}, {free_count, "free_count"}});
  need_ints({{&old_len, "old_len"}, {&new_len, "new_len"}, {&table, "block_table"}, {free_pages, "free_pages"}, {free_count, "free_count"}});
  if (table.dim() != 2 || old_len.dim() != 1 || old_len.size(0) != table.size(0) || new_len.dim() != 1 || new_len.size(0) != table.size(0))
    refuse("lengths must be [B], block_table [B, pages]");
  const int B = fit(table.size(0), "B"), pps = fit(table.size(1), "pages_per_seq");
  int n_pages;
  if (free_pages) {
    if (free_pages->dim() != 1 || free_count->numel() != 1) refuse("free_pages must be [n_pages], free_count one number");
    n_pages = fit(free_pages->size(0), "n_pages");
    if (a[7] != Py_None && int_arg(a[7], "n_pages") != n_pages) refuse("n_pages must be the size of free_pages");
  } else {
    n_pages = a[7] != Py_None ? int_arg(a[7], "n_pages") : INT32_MAX / (P > 0 ? P : 1);
  }
  const int max_runs = es_op_kv_plan_max_runs(B, max_rows, P);
  const int64_t sizes[6] = {(int64_t)B + 1, max_rows, max_rows, max_rows, max_runs, B};
  at::Tensor out[6];
  if (a[8] == Py_None) {
    if (max_rows <= 0 || B <= 0) refuse("bad sizes");
    int64_t all = 0, begin = 0;
    for (int64_t s : sizes) all += s;
    const at::Tensor flat = empty({all}, at::kInt, old_len);
    for (int i = 0; i < 6; ++i) { out[i] = at::native::as_strided_tensorimpl(flat, {sizes[i]}, {1}, begin); begin += sizes[i]; }
  } else {
    if (!PyTuple_Check(a[8]) || PyTuple_GET_SIZE(a[8]) != 6) refuse("out must be a KvPlan");
    for (int i = 0; i < 6; ++i) {
      out[i] = tensor(PyTuple_GET_ITEM(a[8], i), "out");
      launch_stream({{&out[i], "out"}});
      need_ints({{&out[i], "out"}});
      if (out[i].dim() != 1 || out[i].size(0) != sizes[i]) refuse("out[" + std::to_string(i) + "] must have " + std::to_string(sizes[i]) + " entries");
    }
  }
  int32_t* o[6];
  for (int i = 0; i < 6; ++i) o[i] = (int32_t*)out[i].data_ptr();
  call([&] {
    return es_op_kv_plan((const int32_t*)old_len.data_ptr(), (const int32_t*)new_len.data_ptr(), (int32_t*)table.data_ptr(),
                         free_pages ? (int32_t*)free_pages->data_ptr() : nullptr, free_count ? (int32_t*)free_count->data_ptr() : nullptr, B, pps, P,
                         n_pages, max_rows, o[0], o[1], o[2], o[3], o[4], o[5], stream);
  });
  if (a[8] != Py_None) { Py_INCREF(a[8]); return a[8]; }
  PyObject* result = PyTuple_New(6);
  if (!result) throw PythonError{};
  for (int i = 0; i < 6; ++i) PyTuple_SET_ITEM(result, i, THPVariable_Wrap(std::move(out[i])));
  return result;
}

PyObject* kv8_append(PyObject* const* a) {
  const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v"), &slots = tensor(a[2], "slot_map"), &kp = tensor(a[3], "k_pages"),
                   &vp = tensor(a[4], "v_pages"), &ks = tensor(a[5], "k_scale"), &vs = tensor(a[6], "v_scale");
  const at::Tensor* runs = maybe_tensor(a[7], "runs");
  need_cuda_first(k, "k");
  cudaStream_t stream = launch_stream({{&k, "k"}, {&v, "v"}, {&slots, "slot_map"}, {&kp, "k_pages"}, {&vp, "v_pages"}, {&ks, "k_scale"}, {&vs, "v_scale"}, {runs, "runs"}});
  const Pool p = check_pool(kp, vp, ks, vs);
  need_ints({{&slots, "slot_map"}, {runs, "runs"}});
  if (k.dim() != 3 || k.size(1) != p.Hkv || k.size(2) != p.hd || v.sizes() != k.sizes()) refuse("k and v must be [n, Hkv, hd]");
  const int dtype = value_dtype(k);
  if (dtype < 0 || dtype == ES_DTYPE_F32 || v.scalar_type() != k.scalar_type()) refuse("k and v must be fp16 or bf16, both the same");
  const int n = fit(k.size(0), "n");
  if (slots.numel() < n) refuse("slot_map must have an entry for every row");
  const int64_t stride = row_stride(k, "k");
  if (stride != row_stride(v, "v")) refuse("k and v must have the same row stride");
  const int n_runs = runs ? fit(runs->numel(), "runs") : 0;
  call([&] {
    return es_op_kv8_append(k.data_ptr(), v.data_ptr(), dtype, stride, n, (const int32_t*)slots.data_ptr(), runs ? (const int32_t*)runs->data_ptr() : nullptr,
                            n_runs, kp.data_ptr(), vp.data_ptr(), p.code, (float*)ks.data_ptr(), (float*)vs.data_ptr(), p.Hkv, p.hd, p.P, p.n_pages, stream);
  });
  Py_RETURN_NONE;
}

PyObject* kv8_gather(PyObject* const* a) {
  const at::Tensor &slots = tensor(a[0], "slot_map"), &kp = tensor(a[1], "k_pages"), &vp = tensor(a[2], "v_pages"), &ks = tensor(a[3], "k_scale"),
                   &vs = tensor(a[4], "v_scale");
  const int dtype = int_arg(a[5], "dtype");
  need_cuda_first(slots, "slot_map");
  cudaStream_t stream = launch_stream({{&slots, "slot_map"}, {&kp, "k_pages"}, {&vp, "v_pages"}, {&ks, "k_scale"}, {&vs, "v_scale"}});
  const Pool p = check_pool(kp, vp, ks, vs);
  need_ints({{&slots, "slot_map"}});
  if (dtype != ES_DTYPE_F16 && dtype != ES_DTYPE_BF16 && dtype != ES_DTYPE_F32) refuse("dtype must be fp16, bf16 or fp32");
  const int n = fit(slots.numel(), "n");
  at::Tensor out[2];
  if (a[6] == Py_None) {
    const at::Tensor both = empty({2, n, p.Hkv, p.hd}, scalar_of(dtype), kp);
    const int64_t head = p.hd, row = head * p.Hkv;
    for (int i = 0; i < 2; ++i) out[i] = at::native::as_strided_tensorimpl(both, {n, p.Hkv, p.hd}, {row, head, 1}, i * n * row);
  } else {
    if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 2) refuse("out must be two tensors");
    for (int i = 0; i < 2; ++i) {
      out[i] = tensor(PyTuple_GET_ITEM(a[6], i), "out");
      launch_stream({{&out[i], "out"}});
      const at::Tensor& t = out[i];
      if (t.scalar_type() != scalar_of(dtype) || !t.is_contiguous() || t.dim() != 3 || t.size(0) != n || t.size(1) != p.Hkv || t.size(2) != p.hd)
        refuse("out must be two contiguous [n, Hkv, hd] tensors of dtype");
    }
  }
  call([&] {
    return es_op_kv8_gather((const int32_t*)slots.data_ptr(), n, kp.data_ptr(), vp.data_ptr(), p.code, (const float*)ks.data_ptr(), (const float*)vs.data_ptr(),
                            p.Hkv, p.hd, p.P, p.n_pages, out[0].data_ptr(), out[1].data_ptr(), dtype, stream);
  });
  if (a[6] != Py_None) { Py_INCREF(a[6]); return a[6]; }
  PyObject* result = PyTuple_New(2);
  if (!result) throw PythonError{};
  for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(result, i, THPVariable_Wrap(std::move(out[i])));
  return result;
}

PyObject* decode_attention_kv8(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0], "q"), &kp = tensor(a[1], "k_pages"), &vp = tensor(a[2], "v_pages"), &ks = tensor(a[3], "k_scale"),
                   &vs = tensor(a[4], "v_scale"), &table = tensor(a[5], "block_table"), &ctx = tensor(a[6], "ctx_len");
  const int max_ctx = int_arg(a[7], "max_ctx");
  const at::Tensor *scratch = maybe_tensor(a[8], "scratch"), *given = maybe_tensor(a[9], "out");
  need_cuda_first(q, "q");
  cudaStream_t stream = launch_stream({{&q, "q"}, {&kp, "k_pages"}, {&vp, "v_pages"}, {&ks, "k_scale"}, {&vs, "v_scale"}, {&table, "block_table"}, {&ctx, "ctx_len"},
                                       {scratch, "scratch"}, {given, "out"}});
  const Pool p = check_pool(kp, vp, ks, vs);
  need_ints({{&table, "block_table"}, {&ctx, "ctx_len"}});
  const int dims = (int)q.dim(), dtype = value_dtype(q);
  if ((dims != 3 && dims != 4) || q.size(dims - 1) != p.hd || dtype < 0 || dtype == ES_DTYPE_F32) refuse("q must be fp16 or bf16 [B, T, Hq, hd] or [B, Hq, hd]");
  const int B = fit(q.size(0), "B"), T = dims == 4 ? fit(q.size(1), "T") : 1, Hq = fit(q.size(dims - 2), "Hq");
  if (table.dim() != 2 || table.size(0) != B || ctx.dim() != 1 || ctx.size(0) != B) refuse("block_table must be [B, pages], ctx_len [B]");
  const int64_t stride = row_stride(q, "q"), width = (int64_t)Hq * p.hd;
  at::Tensor own_scratch, out;
  size_t bytes = 0;
  void* work = nullptr;
  if (scratch) {
    if (!scratch->is_contiguous()) refuse("scratch must be contiguous");
    work = scratch->data_ptr();
    bytes = scratch->nbytes();
  } else {
    bytes = es_op_decode_attention_kv8_scratch_bytes(B, T, Hq, p.Hkv, p.hd, p.P, max_ctx);
    if (bytes) {
      own_scratch = empty({(int64_t)bytes}, at::kByte, q);
      work = own_scratch.data_ptr();
    }
  }
  if (given) {
    if (given->scalar_type() != q.scalar_type() || !given->is_contiguous() || given->dim() != dims - 1 || given->size(0) != B || (dims == 4 && given->size(1) != T) ||
        given->size(dims - 2) != width)
      refuse("out must be contiguous [B, T, Hq * hd] (or [B, Hq * hd]) of q's type");
    out = *given;
  } else {
    out = dims == 4 ? empty({B, T, width}, q.scalar_type(), q) : empty({B, width}, q.scalar_type(), q);
  }
  const int pps = fit(table.size(1), "pages_per_seq");
  call([&] {
    return es_op_decode_attention_kv8(q.data_ptr(), dtype, stride, kp.data_ptr(), vp.data_ptr(), p.code, (const float*)ks.data_ptr(), (const float*)vs.data_ptr(),
                                      (const int32_t*)table.data_ptr(), (const int32_t*)ctx.data_ptr(), out.data_ptr(), B, T, Hq, p.Hkv, p.hd, p.P, pps, p.n_pages,
                                      max_ctx, work, bytes, stream);
  });
  return THPVariable_Wrap(std::move(out));
}

PyObject* sample(PyObject* const* a) {
  const at::Tensor &logits = tensor(a[0], "logits"), &u = tensor(a[1], "u");
  const at::Tensor *temperature = maybe_tensor(a[2], "temperature"), *top_k = maybe_tensor(a[3], "top_k"), *top_p = maybe_tensor(a[4], "top_p"),
                   *min_p = maybe_tensor(a[5], "min_p");
  need_cuda_first(logits, "logits");
  cudaStream_t stream = launch_stream({{&logits, "logits"}, {&u, "u"}, {temperature, "temperature"}, {top_k, "top_k"}, {top_p, "top_p"}, {min_p, "min_p"}});
  const int dtype = value_dtype(logits);
  if (logits.dim() != 2 || dtype < 0 || (logits.stride(1) != 1 && logits.size(1) != 1)) refuse("logits must be fp32, fp16 or bf16 [B, V] with dense rows");
  const int B = fit(logits.size(0), "B"), V = fit(logits.size(1), "V");
  const Named settings[] = {{&u, "u"}, {temperature, "temperature"}, {top_p, "top_p"}, {min_p, "min_p"}};
  for (const Named& n : settings)
    if (n.t && (n.t->scalar_type() != at::kFloat || !n.t->is_contiguous() || n.t->dim() != 1 || n.t->size(0) != B)) refuse(std::string(n.name) + " must be contiguous fp32 [B]");
  if (top_k && (top_k->scalar_type() != at::kInt || !top_k->is_contiguous() || top_k->dim() != 1 || top_k->size(0) != B)) refuse("top_k must be contiguous int32 [B]");
  at::Tensor tokens, logprobs;
  if (a[6] == Py_None) {
    if (B <= 0) refuse("bad sizes");
    tokens = empty({B}, at::kInt, logits);
    logprobs = empty({B}, at::kFloat, logits);
  } else {
    if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 2) refuse("out must be two tensors");
    tokens = tensor(PyTuple_GET_ITEM(a[6], 0), "out[0]");
    logprobs = tensor(PyTuple_GET_ITEM(a[6], 1), "out[1]");
    launch_stream({{&tokens, "out[0]"}, {&logprobs, "out[1]"}});
    if (tokens.scalar_type() != at::kInt || logprobs.scalar_type() != at::kFloat || !tokens.is_contiguous() || !logprobs.is_contiguous() || tokens.dim() != 1 ||
        logprobs.dim() != 1 || tokens.size(0) != B || logprobs.size(0) != B)
      refuse("out must be contiguous int32 [B] and fp32 [B]");
  }
  const int64_t stride = B > 1 ? logits.stride(0) : V;
  auto f = [](const at::Tensor* t) { return t ? (const float*)t->data_ptr() : nullptr; };
  call([&] {
    return es_op_sample(logits.data_ptr(), dtype, stride, f(&u), f(temperature), top_k ? (const int32_t*)top_k->data_ptr() : nullptr, f(top_p), f(min_p),
                        (int32_t*)tokens.data_ptr(), (float*)logprobs.data_ptr(), B, V, stream);
  });
  if (a[6] != Py_None) { Py_INCREF(a[6]); return a[6]; }
  PyObject* result = PyTuple_New(2);
  if (!result) throw PythonError{};
  PyTuple_SET_ITEM(result, 0, THPVariable_Wrap(std::move(tokens)));
  PyTuple_SET_ITEM(result, 1, THPVariable_Wrap(std::move(logprobs)));
  return result;
}

// ---- module ------------------------------------------------------------------------------------

void raise_refusal(int status, const std::string& message) {
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", status, message.c_str()) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, message.c_str());
  }
}

// N positional arguments; no C++ exception leaves.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
    return nullptr;
  }
  try {
    // results are plain memory: views and allocations go past autograd
    at::AutoDispatchBelowADInplaceOrView no_autograd;
    return F(args);
  } catch (const Refusal& r) {
    raise_refusal(r.status, r.message);
  } catch (const PythonError&) {
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(g_out_of_memory ? g_out_of_memory : PyExc_MemoryError, e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

PyObject* set_errors(PyObject*, PyObject* args) {
  PyObject *error = nullptr, *memory = nullptr;
  if (!PyArg_ParseTuple(args, "OO", &error, &memory)) return nullptr;
  Py_INCREF(error);
  Py_INCREF(memory);
  Py_XSETREF(g_error, error);
  Py_XSETREF(g_out_of_memory, memory);
  Py_RETURN_NONE;
}

#define ENTRY(name, f, n) {name, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    ENTRY("kv_plan", kv_plan, 9), ENTRY("kv8_append", kv8_append, 8), ENTRY("kv8_gather", kv8_gather, 7),
    ENTRY("decode_attention_kv8", decode_attention_kv8, 10), ENTRY("sample", sample, 7),
    {"set_errors", set_errors, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native_binding(void) { return PyModule_Create(&g_module); }
