// Native half of the Python binding: unpacks torch tensors and calls the C ABI.
//
// A call of the library is worth 3-7 us of host time (one to two kernel launches).  Marshalling the arguments of such a
// call through ctypes cost as much again and more (attn_decode 11.1 us, of which 4.2 in the library; attn_extend_append
// 15.6 and 7.2), which bounded every small call: the kernel behind a decode of one sequence takes 4.2 us.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kvattn.h"

namespace {

// Thrown with a Python exception set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* what) {
  PyErr_SetString(type, what);
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_contiguous()) raise(PyExc_AssertionError, "tensors passed to the library must be contiguous");
  if (!t.is_cuda()) raise(PyExc_AssertionError, "expected a CUDA tensor");
  return t;
}

// Addresses are taken before the interpreter lock is let go: a tensor without storage of its own (a fake one) throws here.
// read: for what the library only reads; written: the tensor's own memory, brought about if it still shares another's.
template <typename T = void>
const T* read(const at::Tensor& t) { return static_cast<const T*>(t.const_data_ptr()); }
template <typename T = void>
T* written(const at::Tensor& t) { return static_cast<T*>(t.mutable_data_ptr()); }
template <typename T = void>
const T* read(PyObject* o) { return o == Py_None ? nullptr : read<T>(tensor(o)); }
template <typename T = void>
T* written(PyObject* o) { return o == Py_None ? nullptr : written<T>(tensor(o)); }
int size(const at::Tensor& t, int dim) {
  if (dim >= t.dim()) raise(PyExc_IndexError, "tensor has too few dimensions");
  return (int)t.size(dim);
}

void expect(bool ok, const char* what) {
  if (!ok) raise(PyExc_ValueError, what);
}
// The kernels go by the pool's head_dim: rows of another size would be read, and results written, past their ends.
void of_pool(const kv_pool_t* p, const at::Tensor& t, const char* what) {
  if (p != nullptr && t.dim() == 3) expect(t.size(2) == kv_pool_elem_offset(p, 0, 0, 8, 0) / 8, what);  // (slot 8 of a block lies eight rows behind its first)
}
void rows_of_pool(const kv_pool_t* p, const at::Tensor& q) { of_pool(p, q, "q must have the pool's head_dim"); }
void new_rows_of_pool(const kv_pool_t* p, const at::Tensor& k, const at::Tensor& v) {
  of_pool(p, k, "k_new must have the pool's head_dim");
  // (a place of a head that the pool has not got is -1)
  if (p != nullptr && k.dim() == 3) expect(kv_pool_elem_offset(p, 0, size(k, 1) - 1, 0, 0) >= 0 && kv_pool_elem_offset(p, 0, size(k, 1), 0, 0) < 0, "k_new must have the pool's heads");
  expect(v.nbytes() >= k.nbytes(), "v_new must have the shape of k_new");
}
// (both may be larger: buffers for the largest step there is)
void results_hold(const at::Tensor& q, const at::Tensor& out, const at::Tensor& lse) {
  expect(out.nbytes() >= q.nbytes(), "out must have the shape of q");
  expect(lse.numel() >= q.size(0) * q.size(1), "lse must have an entry for each row of q");
}

// What the calls around attention add to that: the device, types and sizes, which a strided row would otherwise hide.
thread_local int here = -1;  // the current device, once a call has asked
void on_current_device(const at::Tensor& t) {
  if (here < 0) here = c10::cuda::current_device();
  if (t.get_device() != here) raise(PyExc_ValueError, "tensor on another device than the current one");
}
const at::Tensor& typed(PyObject* o, at::ScalarType type) {
  const at::Tensor& t = tensor(o);
  on_current_device(t);
  if (t.scalar_type() != type) raise(PyExc_TypeError, type == at::kInt ? "expected an int32 tensor" : type == at::kFloat ? "expected a float32 tensor" : "expected a bfloat16 tensor");
  return t;
}
int count(int64_t n) {
  expect(n <= 0x7fffffff, "more entries than an int holds");
  return (int)n;
}
int* ints(PyObject* o, int64_t n, const char* what) {  // (None: nullptr)
  if (o == Py_None) return nullptr;
  const at::Tensor& t = typed(o, at::kInt);
  expect(t.numel() == n, what);
  return written<int>(t);
}
const int* read_ints(PyObject* o, int64_t n, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = typed(o, at::kInt);
  expect(t.numel() == n, what);
  return read<int>(t);
}
// bf16 [tokens][heads][head_dim], dense inside a token, any distance from token to token (a part of a fused projection's rows).
const at::Tensor& rows(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) raise(PyExc_AssertionError, "expected a CUDA tensor");
  on_current_device(t);
  if (t.scalar_type() != at::kBFloat16) raise(PyExc_TypeError, "expected a bfloat16 tensor");
  expect(t.dim() == 3 && (t.size(2) < 2 || t.stride(2) == 1) && (t.size(1) < 2 || t.stride(1) == t.size(2)), "rows must be [tokens][heads][head_dim], dense inside a token");
  return t;
}

int integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v != (int)v) raise(PyExc_OverflowError, "whole number beyond an int");  // (its lower half would pass for another number)
  return (int)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return (float)v;
}
kv_pool_t* pool(PyObject* o) {
  if (o == Py_None) return nullptr;
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw Raised{};
  return static_cast<kv_pool_t*>(p);
}
// None: torch's current stream; else a stream object or its handle (anything that int() takes).
void* stream(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* h = PyObject_HasAttrString(o, "cuda_stream") ? PyObject_GetAttrString(o, "cuda_stream") : PyNumber_Long(o);
  if (h == nullptr) throw Raised{};
  void* p = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (p == nullptr && PyErr_Occurred()) throw Raised{};
  return p;
}
struct Workspace {
  void* p = nullptr;
  size_t bytes = 0;
  explicit Workspace(PyObject* o) {
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o);
    p = written(t);
    bytes = t.nbytes();
  }
};
// A ctypes structure (or None).
struct Struct {
  Py_buffer view{};
  explicit Struct(PyObject* o) {
    if (o != Py_None && PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Raised{};
  }
  ~Struct() {
    if (view.obj != nullptr) PyBuffer_Release(&view);
  }
  template <typename T>
  const T* as() const {
    if (view.buf == nullptr) return nullptr;
    if (view.len != (Py_ssize_t)sizeof(T)) raise(PyExc_TypeError, "argument structure of the wrong size");
    return static_cast<const T*>(view.buf);
  }
};

// Runs body(args), which returns a function to be called without the interpreter lock, and returns its status.
template <typename Body>
PyObject* call(Py_ssize_t got, Py_ssize_t want, Body body) {
  if (got != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return PyLong_FromLong(body());
  } catch (const Raised&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
// Calls f without the interpreter lock, which is held again however f is left.
template <typename F>
long unlocked(F f) {
  struct Unlock {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlock() { PyEval_RestoreThread(state); }
  } unlock;
  return f();
}

PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 8, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &k = tensor(a[1]), &start = tensor(a[4]), &bt = tensor(a[6]);
    const void *kp = read(k), *vp = read(a[2]);
    if (a[2] != Py_None) new_rows_of_pool(p, k, tensor(a[2]));
    const int *cu = read<int>(a[3]), *startp = read<int>(start), *row = read<int>(a[5]), *btp = read<int>(bt);
    void* st = stream(a[7]);
    const int pages = size(bt, 1), segs = (int)start.numel(), total = size(k, 0);
    return unlocked([&] { return kv_append(p, kp, vp, cu, startp, row, btp, pages, segs, total, st); });
  });
}

PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 10, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &q = tensor(a[1]), &bt = tensor(a[2]);
    const void* qp = read(q);
    rows_of_pool(p, q);
    const int *btp = read<int>(bt), *ctx = read<int>(a[3]);
    const int max_ctx = integer(a[4]), hq = size(q, 1), pages = size(bt, 1), batch = size(q, 0);
    const float scale = real(a[5]);
    void *out = written(a[6]), *st = stream(a[9]);
    float* lse = written<float>(a[7]);
    if (a[6] != Py_None && a[7] != Py_None) results_hold(q, tensor(a[6]), tensor(a[7]));
    const Workspace ws(a[8]);
    return unlocked([&] { return attn_decode(p, qp, hq, btp, pages, ctx, batch, max_ctx, scale, out, lse, ws.p, ws.bytes, st); });
  });
}

// what attn_extend, attn_extend_planned and attn_extend_append share
template <typename F>
PyObject* extend_like(PyObject* const* a, Py_ssize_t n, int lead, F f) {  // lead: arguments before cu_q
  return call(n, lead + 11, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor& q = tensor(a[1]);
    PyObject* const* b = a + lead;
    const at::Tensor &bt = tensor(b[1]), &pl = tensor(b[2]);
    const void* qp = read(q);
    rows_of_pool(p, q);
    if (lead == 4 && a[2] != Py_None && a[3] != Py_None) {
      new_rows_of_pool(p, tensor(a[2]), tensor(a[3]));
      expect(size(tensor(a[2]), 0) >= size(q, 0), "k_new must have a row for each of q's tokens");
    }
    const int *cu = read<int>(b[0]), *btp = read<int>(bt), *plp = read<int>(pl), *el = read<int>(b[3]);
    const int batch = (int)pl.numel(), max_e = integer(b[4]), max_l = integer(b[5]), hq = size(q, 1), total = size(q, 0), pages = size(bt, 1);
    const float scale = real(b[6]);
    void *out = written(b[7]), *st = stream(b[10]);
    float* lse = written<float>(b[8]);
    if (b[7] != Py_None && b[8] != Py_None) results_hold(q, tensor(b[7]), tensor(b[8]));
    const Workspace ws(b[9]);
    const void *k = lead == 4 ? read(a[2]) : nullptr, *v = lead == 4 ? read(a[3]) : nullptr;
    return unlocked([&] {
      return f(p, qp, k, v, hq, cu, btp, pages, plp, el, batch, total, max_e, max_l, scale, out, lse, ws.p, ws.bytes, st);
    });
  });
}
PyObject* extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return extend_like(a, n, 2, [](kv_pool_t* p, const void* q, const void*, const void*, auto... rest) { return attn_extend(p, q, rest...); });
}
PyObject* extend_planned(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return extend_like(a, n, 2, [](kv_pool_t* p, const void* q, const void*, const void*, auto... rest) { return attn_extend_planned(p, q, rest...); });
}
PyObject* extend_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return extend_like(a, n, 4, [](auto... all) { return attn_extend_append(all...); });
}

PyObject* extend_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 11, [&] {
    kv_pool_t* p = pool(a[0]);
    const int hq = integer(a[1]), total = integer(a[6]), max_e = integer(a[7]), max_l = integer(a[8]);
    const at::Tensor &bt = tensor(a[3]), &pl = tensor(a[4]);
    const int *cu = read<int>(a[2]), *btp = read<int>(bt), *plp = read<int>(pl), *el = read<int>(a[5]);
    const int pages = size(bt, 1), batch = (int)pl.numel();
    const Workspace ws(a[9]);
    void* st = stream(a[10]);
    return unlocked([&] { return attn_extend_plan(p, hq, cu, btp, pages, plp, el, batch, total, max_e, max_l, ws.p, ws.bytes, st); });
  });
}

PyObject* extend_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 16, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &q = tensor(a[1]), &pt = tensor(a[4]), &pl = tensor(a[5]), &ct = tensor(a[6]), &cl = tensor(a[7]);
    const void* qp = read(q);
    rows_of_pool(p, q);
    const int *cu = read<int>(a[2]), *cc = read<int>(a[3]), *ptp = read<int>(pt), *plp = read<int>(pl), *ctp = read<int>(ct), *clp = read<int>(cl);
    const int max_c = integer(a[8]), max_rows = integer(a[9]), max_p = integer(a[10]), parents = (int)pl.numel(), children = (int)cl.numel();
    const int hq = size(q, 1), total = size(q, 0), pages_p = size(pt, 1), pages_c = size(ct, 1);
    const float scale = real(a[11]);
    void *out = written(a[12]), *st = stream(a[15]);
    float* lse = written<float>(a[13]);
    if (a[12] != Py_None && a[13] != Py_None) results_hold(q, tensor(a[12]), tensor(a[13]));
    const Workspace ws(a[14]);
    return unlocked([&] {
      return attn_extend_shared(p, qp, hq, cu, cc, ptp, pages_p, plp, ctp, pages_c, clp, parents, children, total, max_c, max_rows, max_p,
                                scale, out, lse, ws.p, ws.bytes, st);
    });
  });
}

PyObject* mixed(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 7, [&] {
    kv_pool_t* p = pool(a[0]);
    const int hq = integer(a[1]);
    const float scale = real(a[2]);
    const Struct ext(a[3]), dec(a[4]);
    const auto* e = ext.as<attn_extend_args_t>();
    const auto* d = dec.as<attn_decode_args_t>();
    const Workspace ws(a[5]);
    void* st = stream(a[6]);
    return unlocked([&] { return attn_mixed(p, hq, scale, e, d, ws.p, ws.bytes, st); });
  });
}

PyObject* step_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  here = -1;
  return call(n, 12, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &ctx = typed(a[1], at::kInt), &fresh = typed(a[3], at::kInt), &bt = typed(a[4], at::kInt), &slots = typed(a[7], at::kInt);
    const int64_t batch = ctx.numel(), total = slots.numel();
    expect(bt.dim() == 2 && bt.size(0) == batch, "block_tables must have a row for each sequence");
    const int* news = read_ints(a[2], batch, "new_lens must have an entry for each sequence");
    int* cu = ints(a[5], batch + 1, "cu_new must have an entry for each sequence and one more");
    int* pos = ints(a[6], total, "positions must have an entry for each slot");
    int* next = ints(a[8], batch, "next_lens must have an entry for each sequence");
    const int* cursor = read_ints(a[9], 1, "cursor must have one entry");
    int* next_cursor = ints(a[10], 1, "next_cursor must have one entry");
    const int *ctxp = read<int>(ctx), *freshp = read<int>(fresh);
    int *btp = written<int>(bt), *slotp = written<int>(slots);
    void* st = stream(a[11]);
    const int pages = count(fresh.numel()), width = count(bt.size(1)), n_seq = count(batch), n_rows = count(total);
    return unlocked([&] {
      return kv_step_tables(p, ctxp, news, n_seq, freshp, pages, btp, width, n_rows, cu, pos, slotp, next, cursor, next_cursor, st);
    });
  });
}

PyObject* append_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  here = -1;
  return call(n, 13, [&] {
    kv_pool_t* p = pool(a[0]);
    const bool has_q = a[1] != Py_None, has_kv = a[2] != Py_None;
    expect(has_kv == (a[3] != Py_None), "k_new and v_new go together");
    expect(has_q || has_kv, "neither q nor k_new is given");
    expect(has_q == (a[8] != Py_None), "q and q_out go together");
    const at::Tensor &lead = rows(has_q ? a[1] : a[2]), &pos = typed(a[5], at::kInt), &freq = typed(a[6], at::kFloat);
    const int64_t total = lead.size(0), dim = lead.size(2);
    const void *q = nullptr, *k = nullptr, *v = nullptr;
    void* out = nullptr;
    int64_t qs = 0, ks = 0, vs = 0, os = 0;
    int heads = 0;
    if (has_q) {
      const at::Tensor& o = rows(a[8]);
      expect(o.sizes() == lead.sizes(), "q_out must have the shape of q");
      q = read(lead), out = written(o), qs = lead.stride(0), os = o.stride(0), heads = count(lead.size(1));
    }
    if (has_kv) {
      const at::Tensor &kt = rows(a[2]), &vt = rows(a[3]);
      expect(kt.sizes() == vt.sizes() && kt.size(0) == total && kt.size(2) == dim, "k_new and v_new must have the same shape, and q's tokens and head_dim");
      expect(kt.size(1) == integer(a[10]) && dim == integer(a[11]), "k_new must have the pool's heads");
      k = read(kt), v = read(vt), ks = kt.stride(0), vs = vt.stride(0);
    }
    expect(dim == integer(a[11]), "rows must have the pool's head_dim");
    const int* slots = read_ints(a[4], total, "slots must have an entry for each token");
    expect(pos.dim() >= 1 && pos.dim() <= 2 && pos.size(-1) == total, "positions must be [tokens] or [axes][tokens]");
    const int axes = pos.dim() == 2 ? count(pos.size(0)) : 1, rot = count(2 * freq.numel()), n_rows = count(total);
    const int* axis = read_ints(a[7], freq.numel(), "freq_axis must have an entry for each frequency");
    const int* posp = read<int>(pos);
    const float* freqp = read<float>(freq);
    const int neighbours = integer(a[9]);
    void* st = stream(a[12]);
    return unlocked([&] {
      return kv_append_rotary(p, q, qs, k, ks, v, vs, heads, slots, posp, axes, freqp, axis, rot, neighbours, n_rows, out, os, st);
    });
  });
}

PyObject* page_bounds(PyObject*, PyObject* const* a, Py_ssize_t n) {
  here = -1;
  return call(n, 4, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &slots = typed(a[1], at::kInt), &bounds = typed(a[2], at::kBFloat16);
    expect(bounds.nbytes() >= kv_page_bounds_bytes(p), "bounds must have kv_page_bounds_bytes() bytes");
    const int* sp = read<int>(slots);
    void *bp = written(bounds), *st = stream(a[3]);
    const int total = count(slots.numel());
    return unlocked([&] { return kv_page_bounds(p, sp, total, bp, st); });
  });
}

PyObject* select_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  here = -1;
  return call(n, 12, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &q = typed(a[1], at::kBFloat16), &bounds = typed(a[2], at::kBFloat16), &bt = typed(a[3], at::kInt), &list = typed(a[8], at::kInt);
    expect(q.dim() == 3 && bt.dim() == 2 && list.dim() == 3, "q must be [batch][heads][head_dim], block_tables [batch][pages], pages [batch][kv heads][n]");
    rows_of_pool(p, q);
    const int64_t batch = q.size(0);
    expect(bounds.nbytes() >= kv_page_bounds_bytes(p), "bounds must have kv_page_bounds_bytes() bytes");
    expect(bt.size(0) == batch && list.size(0) == batch && list.size(1) == integer(a[11]), "block_tables and pages must have a row for each sequence, pages for each of the pool's heads");
    const int* ctx = read_ints(a[4], batch, "ctx_lens must have an entry for each sequence");
    int* counts = ints(a[9], batch * list.size(1), "counts must be [batch][kv heads]");
    const int max_ctx = integer(a[5]), first = integer(a[6]), last = integer(a[7]), hq = count(q.size(1)), width = count(bt.size(1)), want = count(list.size(2)), n_seq = count(batch);
    const void *qp = read(q), *bp = read(bounds);
    const int* btp = read<int>(bt);
    int* lp = written<int>(list);
    void* st = stream(a[10]);
    return unlocked([&] { return attn_select_pages(p, qp, hq, bp, btp, width, ctx, n_seq, max_ctx, want, first, last, lp, counts, st); });
  });
}

PyObject* decode_selected(PyObject*, PyObject* const* a, Py_ssize_t n) {
  here = -1;
  return call(n, 12, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &q = typed(a[1], at::kBFloat16), &bt = typed(a[2], at::kInt), &list = typed(a[5], at::kInt), &out = typed(a[8], at::kBFloat16), &lse = typed(a[9], at::kFloat);
    expect(q.dim() == 3 && bt.dim() == 2 && list.dim() == 3, "q must be [batch][heads][head_dim], block_tables [batch][pages], pages [batch][kv heads][n]");
    rows_of_pool(p, q);
    const int64_t batch = q.size(0);
    expect(bt.size(0) == batch && list.size(0) == batch && list.size(1) == integer(a[11]), "block_tables and pages must have a row for each sequence, pages for each of the pool's heads");
    expect(out.sizes() == q.sizes() && lse.numel() == batch * q.size(1), "out must have the shape of q, lse an entry for each of its rows");
    const int* ctx = read_ints(a[3], batch, "ctx_lens must have an entry for each sequence");
    const int* counts = read_ints(a[6], batch * list.size(1), "counts must be [batch][kv heads]");
    const int max_ctx = integer(a[4]), hq = count(q.size(1)), pages = count(bt.size(1)), width = count(list.size(2)), n_seq = count(batch);
    const float scale = real(a[7]);
    const void* qp = read(q);
    const int *btp = read<int>(bt), *lp = read<int>(list);
    void *op = written(out), *st = stream(a[10]);
    float* lsep = written<float>(lse);
    return unlocked([&] { return attn_decode_selected(p, qp, hq, btp, pages, ctx, n_seq, max_ctx, lp, counts, width, scale, op, lsep, st); });
  });
}

const at::Tensor& host_tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.is_cuda() || !t.is_contiguous()) raise(PyExc_ValueError, "attn_extend_host takes contiguous host tensors");
  return t;
}
PyObject* extend_host(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return call(n, 15, [&] {
    kv_pool_t* p = pool(a[0]);
    const at::Tensor &q = host_tensor(a[1]), &k = host_tensor(a[2]), &v = host_tensor(a[3]), &cu = host_tensor(a[4]), &bt = host_tensor(a[5]),
                     &pl = host_tensor(a[6]), &el = host_tensor(a[7]), &out = host_tensor(a[11]), &lse = host_tensor(a[12]);
    const void *qp = read(q), *kp = read(k), *vp = read(v);
    const int *cup = read<int>(cu), *btp = read<int>(bt), *plp = read<int>(pl), *elp = read<int>(el);
    const int max_e = integer(a[8]), max_l = integer(a[9]), hq = size(q, 1), total = size(q, 0), pages = size(bt, 1), batch = (int)pl.numel();
    rows_of_pool(p, q);
    new_rows_of_pool(p, k, v);
    expect(size(k, 0) >= total, "k_new must have a row for each of q's tokens");
    results_hold(q, out, lse);
    const float scale = real(a[10]);
    void* outp = written(out);
    float* lsep = written<float>(lse);
    const Workspace staging(a[13]);
    void* st = stream(a[14]);
    return unlocked([&] {
      return attn_extend_host(p, qp, kp, vp, hq, cup, btp, pages, plp, elp, batch, total, max_e, max_l, scale, outp, lsep, staging.p,
                              staging.bytes, st);
    });
  });
}

#define ENTRY(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY("kv_append", append),
                         ENTRY("attn_decode", decode),
                         ENTRY("attn_extend", extend),
                         ENTRY("attn_extend_append", extend_append),
                         ENTRY("attn_extend_plan", extend_plan),
                         ENTRY("attn_extend_planned", extend_planned),
                         ENTRY("attn_extend_shared", extend_shared),
                         ENTRY("attn_mixed", mixed),
                         ENTRY("kv_step_tables", step_tables),
                         ENTRY("kv_append_rotary", append_rotary),
                         ENTRY("kv_page_bounds", page_bounds),
                         ENTRY("attn_select_pages", select_pages),
                         ENTRY("attn_decode_selected", decode_selected),
                         ENTRY("attn_extend_host", extend_host),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvattn_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvattn_native(void) { return PyModule_Create(&module); }
