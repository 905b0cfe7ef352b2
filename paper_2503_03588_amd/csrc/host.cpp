// The calls of binding.py for the ordinary case, in one step from Python to the library: tensors that are plain, contiguous
// and on the GPU, the current stream.  Each function takes the arguments of the Python function of the same name, looks at
// them, allocates what the caller did not pass and calls the C entry point; it returns NotImplemented, having done nothing,
// whenever anything is out of the ordinary, and the Python function then goes its own way.  The library is called once: a
// status it reports is raised as the Python functions raise it.
//
// Reason: the smallest calls take 8 to 12 us on the GPU, and marshalling them in Python took 6 to 8 us each (tensor
// attributes, shapes, ctypes); now 3.5 to 5.  A list and a prefill of 1024 fp32 queries, two calls, were paced by it: 16.2 us
// -> 12.0; a call that is waited for: one decode step 21.7 -> 18.6 us, a chunk 46.3 -> 42.7, list and prefill 32.8 -> 25.6.
// The calls around the attention have more arguments to look at, us a pass, marshalled in Python -> here: pages and slots of 128
// sequences 11.5 -> 5.2, norm and rotation of 2 x 1000 rows 15.4 -> 5.5, its gradients (2 x 777) 30.3 -> 10.5 (the GPU's time), 128 rows stored and
// loaded 26.8 -> 8.7, a whole decode step of 64 sequences 52.5 -> 23.9 (the GPU's time).
#include <algorithm>
#include <array>
#include <initializer_list>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include "../../include/powattn.h"

#ifndef POWATTN_HOST_DEVICE            // (the tests build this file for ordinary memory, where they stand in for the library)
#define POWATTN_HOST_DEVICE at::kCUDA
#endif

namespace {

// the library's entry points (addresses handed over by binding.py, which loads the library)
struct {
  decltype(&powattn_num_blocks) num_blocks;
  decltype(&powattn_max_k) max_k;
  decltype(&powattn_mask_build) mask_build;
  decltype(&powattn_prefill) prefill;
  decltype(&powattn_prefill_chunk) prefill_chunk;
  decltype(&powattn_prefill_chunk_paged) prefill_chunk_paged;
  decltype(&powattn_prefill_batch_paged) prefill_batch_paged;
  decltype(&powattn_prefill_varlen) prefill_varlen;
  decltype(&powattn_decode) decode;
  decltype(&powattn_decode_paged) decode_paged;
  decltype(&powattn_backward_workspace_bytes) backward_workspace_bytes;
  decltype(&powattn_backward) backward;
  decltype(&powattn_page_tables) page_tables;
  decltype(&powattn_qk_norm_rope) qk_norm_rope;
  decltype(&powattn_qk_norm_rope_backward) qk_norm_rope_backward;
  decltype(&powattn_cache_store_q4) cache_store_q4;
  decltype(&powattn_cache_load_q4) cache_load_q4;
  decltype(&powattn_decode_paged_q4) decode_paged_q4;
} lib;
PyObject* get_device = nullptr;       // torch._C._cuda_getDevice
PyObject* get_stream = nullptr;       // torch._C._cuda_getCurrentRawStream
PyObject* tensor_type = nullptr;      // torch.Tensor
PyObject* check = nullptr;            // binding._check: raises for a status

struct other_way {};                  // thrown: not the ordinary case
struct raised {};                     // thrown: the Python exception is set

void need(bool ok) { if (!ok) throw other_way{}; }

// plain tensors only: no subclass, no wrapper of a transform, nothing that a mode would want to see
const at::Tensor& strided_tensor(PyObject* o) {
  need((PyObject*)Py_TYPE(o) == tensor_type);
  const at::Tensor& t = THPVariable_Unpack(o);
  need(t.defined() && t.device().type() == POWATTN_HOST_DEVICE && t.layout() == at::kStrided);
  static const c10::DispatchKeySet wrappers({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
                                             c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                             c10::DispatchKey::Conjugate, c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
  need(!t.key_set().has_any(wrappers));
  return t;
}
const at::Tensor& tensor(PyObject* o) {
  const at::Tensor& t = strided_tensor(o);
  need(t.is_contiguous());
  return t;
}
const at::Tensor& tensor_of(PyObject* o, at::ScalarType type, int64_t dims) {
  const at::Tensor& t = tensor(o);
  need(t.scalar_type() == type && t.dim() == dims);
  return t;
}
void* data(const at::Tensor& t) { return t.data_ptr(); }

int64_t whole(PyObject* o) {
  need(PyLong_CheckExact(o));
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); throw other_way{}; }
  return x;
}
float number(PyObject* o) {
  need(PyFloat_CheckExact(o));
  return (float)PyFloat_AS_DOUBLE(o);
}
powattn_pattern pattern(PyObject* values) {     // (block, window, sink, flags)
  need(PyTuple_CheckExact(values) && PyTuple_GET_SIZE(values) == 4);
  int64_t x[4];
  for (int i = 0; i < 4; ++i) {
    x[i] = whole(PyTuple_GET_ITEM(values, i));
    need(x[i] >= 0 && x[i] <= 0x7fffffff);
  }
  return {(int32_t)x[0], (int32_t)x[1], (int32_t)x[2], (uint32_t)x[3]};
}
// index: the GPU that the tensors are on, where that has to be the current one
void* current_stream(int index = -1) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  if (!dev) { PyErr_Clear(); throw other_way{}; }
  if (index >= 0 && PyLong_AsLong(dev) != index) { Py_DECREF(dev); PyErr_Clear(); throw other_way{}; }
  PyObject* s = PyObject_CallOneArg(get_stream, dev);
  Py_DECREF(dev);
  if (!s) { PyErr_Clear(); throw other_way{}; }
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return p;
}
// no mode that wants to see the allocations below or the tensors
void no_modes() {
  need(!at::impl::torch_function_mode_enabled());
  const auto tls = c10::impl::tls_local_dispatch_key_set();
  need(!tls.included_.has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::Functionalize,
                                                  c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchDynamicLayerFrontMode})));
}
int32_t dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return POWATTN_BF16;
  need(t.scalar_type() == at::kFloat);
  return POWATTN_F32;
}
// Other Python threads run while it lives, as in torch's own allocations (one that waits for the GPU may wait for a callback
// that needs the interpreter).  The interpreter is this thread's again whichever way the scope is left: the outputs are
// allocated and the library's arguments formed inside it, and both throw.
struct without_gil {
  PyThreadState* ts = PyEval_SaveThread();
  ~without_gil() { PyEval_RestoreThread(ts); }
};
// the allocations and the library's call, `name` being its entry point
template <class F>
void call(const char* name, F&& f, int index = -1) {
  void* stream = current_stream(index);
  int st;
  {
    without_gil others_run;
    st = f(stream);
  }
  if (st == POWATTN_OK) return;
  // (not other_way: the Python way would call again, and a HIP error is reported once: the second call would launch)
  PyObject* r = PyObject_CallFunction(check, "is", st, name);
  if (r) {
    Py_DECREF(r);
    PyErr_Format(PyExc_RuntimeError, "%s: status %d", name, st);
  }
  throw raised{};
}
int32_t small(int64_t x) { need(x >= 0 && x <= 0x7fffffff); return (int32_t)x; }

// o and lse: the caller's, or new ones (allocate(), with other threads running); returned as the pair that the Python
// functions return
struct outputs {
  PyObject* o_arg; PyObject* lse_arg;
  const at::Tensor& q;
  std::array<int64_t, 3> lse_shape;
  size_t lse_dims;
  bool new_lse, zeros;
  at::Tensor o, lse;
  outputs(PyObject* o_in, PyObject* lse_in, PyObject* want_lse, const at::Tensor& queries, std::initializer_list<int64_t> shape,
          bool zeroed = false)
      : o_arg(o_in), lse_arg(lse_in), q(queries), lse_dims(shape.size()), zeros(zeroed) {
    need(want_lse == Py_True || want_lse == Py_False);
    std::copy(shape.begin(), shape.end(), lse_shape.begin());
    if (o_arg != Py_None) o = tensor(o_arg);
    if (lse_arg != Py_None) lse = tensor(lse_arg);
    new_lse = lse_arg == Py_None && want_lse == Py_True;
  }
  void allocate() {
    if (o_arg == Py_None) o = zeros ? at::zeros_like(q) : at::empty_like(q);
    if (new_lse) {
      const auto opt = q.options().dtype(at::kFloat);
      const at::IntArrayRef shape(lse_shape.data(), lse_dims);
      lse = zeros ? at::zeros(shape, opt) : at::empty(shape, opt);
    }
  }
  float* lse_ptr() { return lse.defined() ? (float*)data(lse) : nullptr; }
  PyObject* pair() {
    PyObject* t = PyTuple_New(2);
    if (!t) return nullptr;
    if (o_arg != Py_None) { Py_INCREF(o_arg); PyTuple_SET_ITEM(t, 0, o_arg); } else PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(o));
    if (lse_arg != Py_None) { Py_INCREF(lse_arg); PyTuple_SET_ITEM(t, 1, lse_arg); }
    else if (lse.defined()) PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(lse));
    else { Py_INCREF(Py_None); PyTuple_SET_ITEM(t, 1, Py_None); }
    return t;
  }
};
struct lists {
  const int32_t* cnt = nullptr; const int32_t* idx = nullptr;
  int32_t max_k = 0;
  int64_t rows = 0;
  bool given;
  lists(PyObject* c, PyObject* i) : given(i != Py_None) {
    need((c == Py_None) == (i == Py_None));
    if (!given) return;
    const at::Tensor& tc = tensor_of(c, at::kInt, 1);
    const at::Tensor& ti = tensor_of(i, at::kInt, 2);
    cnt = (const int32_t*)data(tc); idx = (const int32_t*)data(ti);
    max_k = small(ti.size(1));
    rows = tc.size(0);
  }
};
struct pages {                         // [n_pages, hkv, block, d] twice, and the table [batch, stride]
  const void* k; const void* v; const int32_t* table;
  int64_t n; int32_t hkv, stride;
  pages(PyObject* ko, PyObject* vo, PyObject* to, const powattn_pattern& pat, int64_t batch, int64_t d, at::ScalarType type) {
    const at::Tensor& tk = tensor_of(ko, type, 4);
    const at::Tensor& tv = tensor_of(vo, type, 4);
    const at::Tensor& tt = tensor_of(to, at::kInt, 2);
    need(tk.sizes() == tv.sizes() && tk.size(2) == pat.block && tk.size(3) == d && tt.size(0) == batch);
    k = data(tk); v = data(tv); table = (const int32_t*)data(tt);
    n = tk.size(0); hkv = small(tk.size(1)); stride = small(tt.size(1));
  }
};

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t expected, F&& f) {
  if (n != expected) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
  try {
    no_modes();
    PyObject* r = f();
    if (r) return r;
    PyErr_Clear();
  } catch (const raised&) {
    return nullptr;
  } catch (const other_way&) {
  } catch (const std::exception&) {    // (an allocation that failed: the Python way raises it)
  }
  Py_INCREF(Py_NotImplemented);
  return Py_NotImplemented;
}

PyObject* f_mask_build(PyObject*, PyObject* const* a, Py_ssize_t n) {   // values, seq_len
  return guarded(n, 2, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const int64_t len = whole(a[1]);
    const int64_t nb = lib.num_blocks(&pat, len);
    const int32_t mk = lib.max_k(&pat, len);
    need(nb > 0 && mk > 0);
    const auto opt = at::TensorOptions().dtype(at::kInt).device(POWATTN_HOST_DEVICE);
    at::Tensor idx, cnt;
    call("powattn_mask_build", [&](void* stream) {
      idx = at::empty({nb, (int64_t)mk}, opt);
      cnt = at::empty({nb}, opt);
      return lib.mask_build(&pat, len, (int32_t*)data(cnt), (int32_t*)data(idx), mk, nullptr, stream);
    });
    PyObject* t = PyTuple_New(3);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(cnt));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(idx));
    Py_INCREF(Py_None);
    PyTuple_SET_ITEM(t, 2, Py_None);
    return t;
  });
}
// values, kv_cnt, kv_idx, q, k, v, o, lse, softmax_scale, want_lse
PyObject* f_prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4);
    const int64_t b = q.size(0), hq = q.size(1), len = q.size(2), d = q.size(3);
    const at::Tensor& k = tensor_of(a[4], q.scalar_type(), 4);
    const at::Tensor& v = tensor_of(a[5], q.scalar_type(), 4);
    need(k.sizes() == v.sizes() && k.size(0) == b && k.size(2) == len && k.size(3) == d);
    need(!l.given || l.rows * pat.block >= len);
    const int32_t code = dtype_code(q);
    const float scale = number(a[8]);
    outputs out(a[6], a[7], a[9], q, {b, hq, len});
    call("powattn_prefill", [&](void* stream) { out.allocate(); return lib.prefill(&pat, l.cnt, l.idx, l.max_k, data(q), data(k), data(v), data(out.o), out.lse_ptr(), small(b), small(hq),
                     small(k.size(1)), len, small(d), code, scale, stream); });
    return out.pair();
  });
}
// values, kv_cnt, kv_idx, q, k_cache, v_cache, q_start, o, lse, softmax_scale, want_lse
PyObject* f_prefill_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4);
    const int64_t b = q.size(0), hq = q.size(1), len = q.size(2), d = q.size(3), start = whole(a[6]);
    const at::Tensor& k = tensor_of(a[4], q.scalar_type(), 4);
    const at::Tensor& v = tensor_of(a[5], q.scalar_type(), 4);
    need(k.sizes() == v.sizes() && k.size(0) == b && k.size(3) == d);
    need(!l.given || l.rows * pat.block >= start + len);
    const int32_t code = dtype_code(q);
    const float scale = number(a[9]);
    outputs out(a[7], a[8], a[10], q, {b, hq, len});
    call("powattn_prefill_chunk", [&](void* stream) { out.allocate(); return lib.prefill_chunk(&pat, l.cnt, l.idx, l.max_k, data(q), data(k), data(v), data(out.o), out.lse_ptr(), small(b), small(hq),
                           small(k.size(1)), start, len, k.size(2), small(d), code, scale, stream); });
    return out.pair();
  });
}
// values, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, o, lse, softmax_scale, want_lse
PyObject* f_prefill_chunk_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4 && l.given);
    const int64_t b = q.size(0), hq = q.size(1), len = q.size(2), d = q.size(3), start = whole(a[7]);
    const pages pg(a[4], a[5], a[6], pat, b, d, q.scalar_type());
    need(l.rows * pat.block >= start + len);
    const int32_t code = dtype_code(q);
    const float scale = number(a[10]);
    outputs out(a[8], a[9], a[11], q, {b, hq, len});
    call("powattn_prefill_chunk_paged", [&](void* stream) { out.allocate(); return lib.prefill_chunk_paged(&pat, l.cnt, l.idx, l.max_k, data(q), pg.k, pg.v, pg.table, pg.stride, pg.n, data(out.o), out.lse_ptr(),
                                 small(b), small(hq), pg.hkv, start, len, small(d), code, scale, stream); });
    return out.pair();
  });
}
// values, kv_cnt, kv_idx, q, k_pages, v_pages, block_table, q_start, q_len, o, lse, softmax_scale, want_lse
PyObject* f_prefill_batch_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4 && l.given);
    const int64_t b = q.size(0), hq = q.size(1), rows = q.size(2), d = q.size(3);
    const pages pg(a[4], a[5], a[6], pat, b, d, q.scalar_type());
    const at::Tensor& start = tensor_of(a[7], at::kInt, 1);
    const at::Tensor& len = tensor_of(a[8], at::kInt, 1);
    need(start.size(0) == b && len.size(0) == b && start.device() == q.device() && len.device() == q.device() && l.rows >= pg.stride);
    const int32_t code = dtype_code(q);
    const float scale = number(a[11]);
    outputs out(a[9], a[10], a[12], q, {b, hq, rows});
    call("powattn_prefill_batch_paged", [&](void* stream) { out.allocate(); return lib.prefill_batch_paged(&pat, l.cnt, l.idx, l.max_k, data(q), pg.k, pg.v, pg.table, pg.stride, pg.n, (const int32_t*)data(start),
                                 (const int32_t*)data(len), rows, data(out.o), out.lse_ptr(), small(b), small(hq), pg.hkv, small(d),
                                 code, scale, stream); });
    return out.pair();
  });
}
// values, kv_cnt, kv_idx, q, k, v, seq_lens, o, lse, softmax_scale, want_lse
PyObject* f_prefill_varlen(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4);
    const int64_t b = q.size(0), hq = q.size(1), len = q.size(2), d = q.size(3);
    const at::Tensor& k = tensor_of(a[4], q.scalar_type(), 4);
    const at::Tensor& v = tensor_of(a[5], q.scalar_type(), 4);
    const at::Tensor& lens = tensor_of(a[6], at::kInt, 1);
    need(k.sizes() == v.sizes() && k.size(0) == b && k.size(2) == len && k.size(3) == d && lens.size(0) == b && lens.device() == q.device());
    need(!l.given || l.rows * pat.block >= len);
    const int32_t code = dtype_code(q);
    const float scale = number(a[9]);
    outputs out(a[7], a[8], a[10], q, {b, hq, len}, true);
    call("powattn_prefill_varlen", [&](void* stream) { out.allocate(); return lib.prefill_varlen(&pat, l.cnt, l.idx, l.max_k, data(q), data(k), data(v), data(out.o), out.lse_ptr(), small(b), small(hq),
                            small(k.size(1)), (const int32_t*)data(lens), len, small(d), code, scale, stream); });
    return out.pair();
  });
}
// values, q, k_cache, v_cache, kv_len, o, lse, softmax_scale, workspace, want_lse
PyObject* f_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const at::Tensor& q = tensor(a[1]);
    need(q.dim() == 3);
    const int64_t b = q.size(0), hq = q.size(1), d = q.size(2);
    const at::Tensor& k = tensor_of(a[2], q.scalar_type(), 4);
    const at::Tensor& v = tensor_of(a[3], q.scalar_type(), 4);
    const at::Tensor& lens = tensor_of(a[4], at::kInt, 1);
    need(k.sizes() == v.sizes() && k.size(0) == b && k.size(3) == d && lens.size(0) == b);
    const at::Tensor& ws = tensor(a[8]);
    const int32_t code = dtype_code(q);
    const float scale = number(a[7]);
    outputs out(a[5], a[6], a[9], q, {b, hq});
    call("powattn_decode", [&](void* stream) { out.allocate(); return lib.decode(&pat, data(q), data(k), data(v), (const int32_t*)data(lens), k.size(2), data(out.o), out.lse_ptr(), small(b), small(hq),
                    small(k.size(1)), small(d), code, scale, data(ws), ws.nbytes(), stream); });
    return out.pair();
  });
}
// values, q, k_pages, v_pages, block_table, kv_len, o, lse, softmax_scale, workspace, want_lse
PyObject* f_decode_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const at::Tensor& q = tensor(a[1]);
    need(q.dim() == 3);
    const int64_t b = q.size(0), hq = q.size(1), d = q.size(2);
    const pages pg(a[2], a[3], a[4], pat, b, d, q.scalar_type());
    const at::Tensor& lens = tensor_of(a[5], at::kInt, 1);
    need(lens.size(0) == b);
    const at::Tensor& ws = tensor(a[9]);
    const int32_t code = dtype_code(q);
    const float scale = number(a[8]);
    outputs out(a[6], a[7], a[10], q, {b, hq});
    call("powattn_decode_paged", [&](void* stream) { out.allocate(); return lib.decode_paged(&pat, data(q), pg.k, pg.v, pg.n, pg.table, pg.stride, (const int32_t*)data(lens), data(out.o), out.lse_ptr(),
                          small(b), small(hq), pg.hkv, small(d), code, scale, data(ws), ws.nbytes(), stream); });
    return out.pair();
  });
}

// values, kv_cnt, kv_idx, q, k, v, o, lse, d_o, dq, dk, dv, softmax_scale, workspace
PyObject* f_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    const lists l(a[1], a[2]);
    const at::Tensor& q = tensor(a[3]);
    need(q.dim() == 4 && l.given);
    const int64_t b = q.size(0), hq = q.size(1), len = q.size(2), d = q.size(3);
    const at::ScalarType type = q.scalar_type();
    const at::Tensor& k = tensor_of(a[4], type, 4);
    const at::Tensor& v = tensor_of(a[5], type, 4);
    const at::Tensor& o = tensor_of(a[6], type, 4);
    const at::Tensor& lse = tensor_of(a[7], at::kFloat, 3);
    const at::Tensor& dout = tensor_of(a[8], type, 4);
    need(k.sizes() == v.sizes() && k.size(0) == b && k.size(2) == len && k.size(3) == d && o.sizes() == q.sizes() && dout.sizes() == q.sizes()
         && lse.size(0) == b && lse.size(1) == hq && lse.size(2) == len);
    const int32_t code = dtype_code(q), hkv = small(k.size(1));
    const float scale = number(a[12]);
    const at::Tensor* like[3] = {&q, &k, &v};
    at::Tensor grad[3], ws;
    for (int i = 0; i < 3; ++i) if (a[9 + i] != Py_None) grad[i] = tensor(a[9 + i]);
    if (a[13] != Py_None) ws = tensor(a[13]);
    size_t bytes = 0;
    if (!ws.defined()) {
      bytes = lib.backward_workspace_bytes(&pat, small(b), small(hq), hkv, len, small(d));
      need(bytes > 0);
    }
    call("powattn_backward", [&](void* stream) {
      for (int i = 0; i < 3; ++i) if (!grad[i].defined()) grad[i] = at::empty_like(*like[i]);
      if (!ws.defined()) ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
      return lib.backward(&pat, l.cnt, l.idx, l.max_k, data(q), data(k), data(v), data(o), (const float*)data(lse), data(dout),
                          data(grad[0]), data(grad[1]), data(grad[2]), small(b), small(hq), hkv, len, small(d), code,
                          scale, data(ws), ws.nbytes(), stream);
    });
    PyObject* t = PyTuple_New(3);
    if (!t) return nullptr;
    for (int i = 0; i < 3; ++i) {
      if (a[9 + i] != Py_None) { Py_INCREF(a[9 + i]); PyTuple_SET_ITEM(t, i, a[9 + i]); }
      else PyTuple_SET_ITEM(t, i, THPVariable_Wrap(grad[i]));
    }
    return t;
  });
}

// ---- around the attention calls ----
// Every tensor of a call on one GPU, the current one.
struct one_gpu {
  int index = -2;
  const at::Tensor& operator()(const at::Tensor& t) {
    const int i = t.device().index();
    need(index == -2 || index == i);
    index = i;
    return t;
  }
};
// an output: the caller's, which has to be what a new one would be, or (allocate) a new one; `out` is a new reference to what
// is returned
struct output {
  PyObject* arg;
  at::Tensor t;
  c10::SmallVector<int64_t, 4> shape;
  at::ScalarType type;
  bool zeros;
  output(PyObject* o, one_gpu& on, std::initializer_list<int64_t> s, at::ScalarType ty, bool zeroed = false)
      : arg(o), shape(s), type(ty), zeros(zeroed) {
    if (arg == Py_None) return;
    t = on(tensor(arg));
    need(t.scalar_type() == type && t.sizes() == at::IntArrayRef(shape));
  }
  void allocate(const at::TensorOptions& like) {
    if (arg != Py_None) return;
    const auto opt = like.dtype(type);
    t = zeros ? at::zeros(shape, opt) : at::empty(shape, opt);
  }
  PyObject* out() {
    if (arg == Py_None) return THPVariable_Wrap(t);
    Py_INCREF(arg);
    return arg;
  }
};
PyObject* tuple_of(std::initializer_list<PyObject*> items) {      // takes the references
  PyObject* t = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (t && o) PyTuple_SET_ITEM(t, i++, o);
    else { Py_XDECREF(o); Py_CLEAR(t); }
  }
  return t;
}
// rows [batch, heads, rows, head_dim] in any layout with contiguous components
struct rows_of {
  const at::Tensor& t;
  int64_t strides[3];
  rows_of(PyObject* o, one_gpu& on) : t(on(strided_tensor(o))) {
    need(t.dim() == 4 && (t.size(3) <= 1 || t.stride(3) == 1));
    for (int i = 0; i < 3; ++i) strides[i] = t.stride(i);
  }
  bool apart() const {                   // no two rows share memory
    std::array<std::pair<int64_t, int64_t>, 3> d;
    int n = 0;
    for (int i = 0; i < 3; ++i) if (t.size(i) > 1) d[n++] = {t.stride(i), t.size(i)};
    std::sort(d.begin(), d.begin() + n);
    int64_t extent = t.size(3);
    for (int i = 0; i < n; ++i) {
      if (d[i].first < extent) return false;
      extent += d[i].first * (d[i].second - 1);
    }
    return true;
  }
};
const int32_t* int32_or_none(PyObject* o, one_gpu& on, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = on(tensor_of(o, at::kInt, 1));
  need(t.size(0) == n);
  return (const int32_t*)data(t);
}
bool truth(PyObject* o) { need(o == Py_True || o == Py_False); return o == Py_True; }

// values, q_start, q_len, free_pages, block_table, n_pages, q_rows, slots, kv_len, n_taken
PyObject* f_page_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    one_gpu on;
    const at::Tensor& start = on(tensor_of(a[1], at::kInt, 1));
    const at::Tensor& len = on(tensor_of(a[2], at::kInt, 1));
    const at::Tensor& free_pages = on(tensor_of(a[3], at::kInt, 1));
    const at::Tensor& table = on(tensor_of(a[4], at::kInt, 2));
    const int64_t b = start.size(0), n_pages = whole(a[5]), rows = whole(a[6]);
    need(len.size(0) == b && table.size(0) == b && rows > 0);
    output slots(a[7], on, {b, rows}, at::kInt), kv_len(a[8], on, {b}, at::kInt), taken(a[9], on, {1}, at::kInt);
    call("powattn_page_tables", [&](void* stream) {
      for (output* o : {&slots, &kv_len, &taken}) o->allocate(start.options());
      return lib.page_tables(&pat, (const int32_t*)data(start), (const int32_t*)data(len), small(b), rows, (const int32_t*)data(free_pages),
                             small(free_pages.size(0)), n_pages, (int32_t*)data(table), small(table.size(1)), (int32_t*)data(slots.t),
                             (int32_t*)data(kv_len.t), (int32_t*)data(taken.t), stream);
    }, on.index);
    return tuple_of({slots.out(), kv_len.out(), taken.out()});
  });
}

// q, k, q_weight, k_weight, inv_freq, q_start, q_len, eps, interleaved
struct rope_arguments {
  one_gpu on;
  rows_of q, k;
  int64_t b, hq, hkv, rows, d;
  int32_t code, rot = 0;
  const void* qw; const void* kw; const float* inv = nullptr;
  const int32_t* start; const int32_t* len;
  float eps; uint32_t flags;
  const at::Tensor& weight(PyObject* o) {
    const at::Tensor& w = on(tensor_of(o, q.t.scalar_type(), 1));
    need(w.size(0) == d);
    return w;
  }
  explicit rope_arguments(PyObject* const* a) : q(a[0], on), k(a[1], on) {
    b = q.t.size(0); hq = q.t.size(1); rows = q.t.size(2); d = q.t.size(3); hkv = k.t.size(1);
    need(k.t.scalar_type() == q.t.scalar_type() && k.t.size(0) == b && k.t.size(2) == rows && k.t.size(3) == d);
    code = dtype_code(q.t);
    qw = data(weight(a[2])); kw = data(weight(a[3]));
    if (a[4] != Py_None) {
      const at::Tensor& f = on(tensor_of(a[4], at::kFloat, 1));
      need(f.size(0) <= 1 << 20);
      inv = (const float*)data(f); rot = (int32_t)(2 * f.size(0));
    }
    start = int32_or_none(a[5], on, b); len = int32_or_none(a[6], on, b);
    eps = number(a[7]); flags = truth(a[8]) ? POWATTN_ROPE_INTERLEAVED : 0u;
  }
};
// ..., q_out, k_out
PyObject* f_qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    rope_arguments r(a);
    const at::ScalarType type = r.q.t.scalar_type();
    output qo(a[9], r.on, {r.b, r.hq, r.rows, r.d}, type, r.len), ko(a[10], r.on, {r.b, r.hkv, r.rows, r.d}, type, r.len);
    call("powattn_qk_norm_rope", [&](void* stream) {
      for (output* o : {&qo, &ko}) o->allocate(r.q.t.options());
      return lib.qk_norm_rope(data(r.q.t), r.q.strides, data(r.k.t), r.k.strides, r.qw, r.kw, r.inv, r.rot, r.flags, r.start, r.len, data(qo.t),
                              data(ko.t), small(r.b), small(r.hq), small(r.hkv), r.rows, small(r.d), r.code, r.eps, stream);
    }, r.on.index);
    return tuple_of({qo.out(), ko.out()});
  });
}
// ..., dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace
PyObject* f_qk_norm_rope_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&]() -> PyObject* {
    rope_arguments r(a);
    const at::ScalarType type = r.q.t.scalar_type();
    need(a[9] != Py_None && a[10] != Py_None && a[11] != Py_None && a[12] != Py_None);
    const output gq(a[9], r.on, {r.b, r.hq, r.rows, r.d}, type), gk(a[10], r.on, {r.b, r.hkv, r.rows, r.d}, type);
    const rows_of dq(a[11], r.on), dk(a[12], r.on);
    need(dq.t.sizes() == r.q.t.sizes() && dk.t.sizes() == r.k.t.sizes() && dq.t.scalar_type() == type && dk.t.scalar_type() == type
         && dq.apart() && dk.apart());
    output dqw(a[13], r.on, {r.d}, at::kFloat), dkw(a[14], r.on, {r.d}, at::kFloat);
    const at::Tensor& ws = r.on(tensor(a[15]));
    call("powattn_qk_norm_rope_backward", [&](void* stream) {
      for (output* o : {&dqw, &dkw}) o->allocate(r.q.t.options());
      return lib.qk_norm_rope_backward(data(r.q.t), r.q.strides, data(r.k.t), r.k.strides, r.qw, r.kw, r.inv, r.rot, r.flags, r.start, r.len,
                                       data(gq.t), data(gk.t), data(dq.t), dq.strides, data(dk.t), dk.strides, (float*)data(dqw.t),
                                       (float*)data(dkw.t), small(r.b), small(r.hq), small(r.hkv), r.rows, small(r.d), r.code, r.eps,
                                       data(ws), ws.nbytes(), stream);
    }, r.on.index);
    Py_INCREF(a[11]);
    Py_INCREF(a[12]);
    return tuple_of({a[11], a[12], dqw.out(), dkw.out()});
  });
}

struct cache_q4 {                        // (k, v, k_scale, v_scale)
  void* k; void* v; void* ks; void* vs;
  int64_t n, hkv, d;
  cache_q4(PyObject* o, one_gpu& on, const powattn_pattern& pat) {
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4);
    const at::Tensor* t[4];
    for (int i = 0; i < 4; ++i) t[i] = &on(tensor_of(PyTuple_GET_ITEM(o, i), at::kByte, 4));
    n = t[0]->size(0); hkv = t[0]->size(1); d = 2 * t[0]->size(3);
    need(t[0]->size(2) == pat.block && t[1]->sizes() == t[0]->sizes());
    for (int i = 2; i < 4; ++i)
      need(t[i]->size(0) == n && t[i]->size(1) == hkv && t[i]->size(2) == d / 32 && t[i]->size(3) == pat.block);
    k = data(*t[0]); v = data(*t[1]); ks = data(*t[2]); vs = data(*t[3]);
  }
};
// values, k, v, cache, slots
PyObject* f_cache_store_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    one_gpu on;
    const rows_of k(a[1], on), v(a[2], on);
    const cache_q4 c(a[3], on, pat);
    const at::Tensor& slots = on(tensor_of(a[4], at::kInt, 2));
    need(k.t.sizes() == v.t.sizes() && k.t.scalar_type() == v.t.scalar_type() && k.t.size(1) == c.hkv && k.t.size(3) == c.d
         && slots.size(0) == k.t.size(0) && slots.size(1) == k.t.size(2));
    const int32_t code = dtype_code(k.t);
    call("powattn_cache_store_q4", [&](void* stream) {
      return lib.cache_store_q4(&pat, data(k.t), k.strides, data(v.t), v.strides, (const int32_t*)data(slots), c.k, c.v, c.ks, c.vs, c.n,
                                small(k.t.size(0)), small(c.hkv), k.t.size(2), small(c.d), code, stream);
    }, on.index);
    Py_INCREF(Py_None);
    return Py_None;
  });
}
// values, cache, block_table, rows, start, length, k, v
PyObject* f_cache_load_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    one_gpu on;
    const cache_q4 c(a[1], on, pat);
    const at::Tensor& table = on(tensor_of(a[2], at::kInt, 2));
    const int64_t b = table.size(0), rows = whole(a[3]);
    need(rows > 0);
    const int32_t* start = int32_or_none(a[4], on, b);
    const int32_t* len = int32_or_none(a[5], on, b);
    output k(a[6], on, {b, c.hkv, rows, c.d}, at::kBFloat16, true), v(a[7], on, {b, c.hkv, rows, c.d}, at::kBFloat16, true);
    call("powattn_cache_load_q4", [&](void* stream) {
      for (output* o : {&k, &v}) o->allocate(table.options());
      return lib.cache_load_q4(&pat, c.k, c.v, c.ks, c.vs, c.n, (const int32_t*)data(table), small(table.size(1)), start, len, data(k.t),
                               data(v.t), small(b), small(c.hkv), rows, small(c.d), POWATTN_BF16, stream);
    }, on.index);
    return tuple_of({k.out(), v.out()});
  });
}
// values, q, cache, block_table, kv_len, o, lse, softmax_scale, workspace, want_lse
PyObject* f_decode_paged_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const powattn_pattern pat = pattern(a[0]);
    one_gpu on;
    const at::Tensor& q = on(tensor(a[1]));
    need(q.dim() == 3);
    const int64_t b = q.size(0), hq = q.size(1), d = q.size(2);
    const cache_q4 c(a[2], on, pat);
    const at::Tensor& table = on(tensor_of(a[3], at::kInt, 2));
    const at::Tensor& lens = on(tensor_of(a[4], at::kInt, 1));
    need(c.d == d && table.size(0) == b && lens.size(0) == b);
    const int32_t code = dtype_code(q);
    const float scale = number(a[7]);
    const bool want = truth(a[9]);
    output o(a[5], on, {b, hq, d}, q.scalar_type()), lse(a[6], on, {b, hq}, at::kFloat);
    const at::Tensor& ws = on(tensor(a[8]));
    const bool with_lse = want || a[6] != Py_None;
    call("powattn_decode_paged_q4", [&](void* stream) {
      o.allocate(q.options());
      if (with_lse) lse.allocate(q.options());
      return lib.decode_paged_q4(&pat, data(q), c.k, c.v, c.ks, c.vs, c.n, (const int32_t*)data(table), small(table.size(1)),
                                 (const int32_t*)data(lens), data(o.t), with_lse ? (float*)data(lse.t) : nullptr, small(b), small(hq),
                                 small(c.hkv), small(d), code, scale, data(ws), ws.nbytes(), stream);
    }, on.index);
    if (!with_lse) Py_INCREF(Py_None);
    return tuple_of({o.out(), with_lse ? lse.out() : Py_None});
  });
}

// addresses of the entry points in the order of `lib`, torch.Tensor, the device and the stream look-up, binding._check
PyObject* f_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr Py_ssize_t N_FN = sizeof(lib) / sizeof(void*);
  if (n != N_FN + 4) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
  void* fn[N_FN];
  for (Py_ssize_t i = 0; i < N_FN; ++i) {
    fn[i] = PyLong_AsVoidPtr(a[i]);
    if (!fn[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point"); return nullptr; }
  }
  memcpy(&lib, fn, sizeof lib);
  for (int i = 0; i < 4; ++i) Py_INCREF(a[N_FN + i]);
  tensor_type = a[N_FN]; get_device = a[N_FN + 1]; get_stream = a[N_FN + 2]; check = a[N_FN + 3];
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)())f_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind), FAST(mask_build), FAST(prefill), FAST(prefill_chunk), FAST(prefill_chunk_paged), FAST(prefill_batch_paged),
                         FAST(prefill_varlen), FAST(decode), FAST(decode_paged), FAST(backward), FAST(page_tables), FAST(qk_norm_rope),
                         FAST(qk_norm_rope_backward), FAST(cache_store_q4), FAST(cache_load_q4), FAST(decode_paged_q4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
