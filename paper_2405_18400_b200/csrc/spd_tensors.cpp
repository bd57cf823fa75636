// Marshalling of the beams' operators for torch: tensors in, the argument structs of spd.h out, outputs allocated by torch.
//
// A timestep's calls are a few microseconds on the device, and in Python the attributes of a dozen tensors, their checks and the
// struct cost more than that (append 11 us, attention 15): here 1 to 3.  The library itself is reached through the
// addresses that bind() is given, so that this module works with whichever build of it the process has loaded.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <stdexcept>
#include <vector>

#include "spd.h"

namespace {

int (*g_append)(const spd_append_args *);
int (*g_attention)(const spd_attention_args *);
int (*g_attention_bytes)(const spd_attention_args *, size_t *);
int (*g_select)(const spd_select_args *);
int (*g_select_bytes)(const spd_select_args *, size_t *);
int (*g_reorder)(const spd_reorder_args *);
PyObject *g_fail;    // called with (status, name): raises
PyObject *g_memory;  // the exception for device memory that torch could not allocate

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct Raised {};  // a Python error is set
[[noreturn]] void refuse(const char *what) { throw Refused(what); }

const char *const kDevices = "tensors on different devices (all belong on one CUDA device)";

const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) refuse(what);
  return THPVariable_Unpack(o);
}
bool given(PyObject *o) { return o != Py_None; }
long integer(PyObject *o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}
int32_t int32(PyObject *o) {
  const long v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) refuse("an argument does not fit 32 bits");
  return (int32_t)v;
}
float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return (float)v;
}
int32_t size32(int64_t v) {
  if (v > INT32_MAX) refuse("a dimension does not fit 32 bits");
  return (int32_t)v;
}
int type_of(const at::Tensor &t, const char *what) {
  const auto s = t.scalar_type();
  if (s != at::kFloat && s != at::kBFloat16) refuse(what);
  return s == at::kFloat ? SPD_F32 : SPD_BF16;
}
int cuda_of(const at::Tensor &t) {
  if (!t.is_cuda()) {
    PyErr_SetString(PyExc_RuntimeError, "the operators need CUDA tensors; there is no CPU path");
    throw Raised();
  }
  return t.get_device();
}
void on(int device, const at::Tensor &t) {
  if (!t.is_cuda() || t.get_device() != device) refuse(kDevices);
}
// int32, one dimension of n entries.
const int32_t *ints(PyObject *o, int64_t n, int device, const char *what) {
  if (!given(o)) return nullptr;
  const at::Tensor &t = tensor(o, what);
  if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || !t.is_contiguous()) refuse(what);
  on(device, t);
  return static_cast<const int32_t *>(t.const_data_ptr());
}
struct Table {
  const int32_t *at = nullptr;
  int64_t row = 0;
  int32_t rows = 0, cols = 0;
};
Table table(PyObject *o, int device, const char *what) {
  Table r;
  if (!given(o)) return r;
  const at::Tensor &t = tensor(o, what);
  if (t.scalar_type() != at::kInt || t.dim() != 2 || (t.stride(1) != 1 && t.size(1) > 1)) refuse(what);
  on(device, t);
  r.at = static_cast<const int32_t *>(t.const_data_ptr());
  r.row = t.stride(0);
  r.rows = size32(t.size(0)), r.cols = size32(t.size(1));
  return r;
}
// [rows][heads][dim] with a contiguous last dimension: strides of rows and heads.
void rows_of(const at::Tensor &t, int device, const char *what, int64_t *row, int64_t *head) {
  if (t.dim() != 3 || (t.stride(2) != 1 && t.size(2) > 1)) refuse(what);
  on(device, t);
  *row = t.stride(0), *head = t.stride(1);
}
// The same of a tensor that is written: no element may be there twice.
void written(const at::Tensor &t, int device, const char *what, int64_t *row, int64_t *head) {
  rows_of(t, device, what, row, head);
  if ((*row == 0 && t.size(0) > 1) || (*head == 0 && t.size(1) > 1)) refuse("a tensor that is written repeats its elements");
}
// A workspace: what the call may write is its bytes, which have to be there (a view that repeats elements counts more).
void room(const at::Tensor &t, int device) {
  if (!t.is_contiguous()) refuse("workspace: a contiguous tensor expected");
  on(device, t);
}
void *data(const at::Tensor &t) { return const_cast<void *>(t.const_data_ptr()); }

void check(int rc, const char *name) {
  if (rc == SPD_OK) return;
  PyObject *r = PyObject_CallFunction(g_fail, "is", rc, name);
  if (r) {
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, name);
  }
  throw Raised();
}

template <typename F>
PyObject *guarded(F body) {
  try {
    return body();
  } catch (const Raised &) {
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::OutOfMemoryError &e) {
    PyErr_SetString(g_memory, e.what_without_backtrace());
  } catch (const c10::Error &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}
#define SPD_ARGS(n)                                                            \
  if (nargs != n) {                                                            \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");             \
    return nullptr;                                                            \
  }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like) { return at::empty(shape, like.options().dtype(type)); }

// bind(append, attention, attention_bytes, select, select_bytes, reorder, fail, memory): the library's functions by address, the exceptions.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(8)
  void *at[6];
  for (int i = 0; i < 6; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (!at[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
      return nullptr;
    }
  }
  std::memcpy(&g_append, &at[0], sizeof at[0]);
  std::memcpy(&g_attention, &at[1], sizeof at[0]);
  std::memcpy(&g_attention_bytes, &at[2], sizeof at[0]);
  std::memcpy(&g_select, &at[3], sizeof at[0]);
  std::memcpy(&g_select_bytes, &at[4], sizeof at[0]);
  std::memcpy(&g_reorder, &at[5], sizeof at[0]);
  Py_INCREF(a[6]);
  Py_XSETREF(g_fail, a[6]);
  Py_INCREF(a[7]);
  Py_XSETREF(g_memory, a[7]);
  Py_RETURN_NONE;
}

// cache_append(k, v, k_cache, v_cache, pos, rope, q, q_out, index, seq, table, page, pairs, status)
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(14)
  return guarded([&]() -> PyObject * {
    const bool kv = given(a[0]), queries = given(a[6]);
    if ((!kv && !queries) || kv != given(a[1])) refuse("k with v, q, or all three expected, [tokens, heads, dim]");
    const at::Tensor &lead = tensor(kv ? a[0] : a[6], "k, q: tensors expected");
    if (lead.dim() != 3) refuse("k with v, q, or all three expected, [tokens, heads, dim]");
    const int device = cuda_of(lead);
    spd_append_args p = {};
    p.n = size32(lead.size(0)), p.head_dim = size32(lead.size(2));
    p.x_dtype = type_of(lead, "k, v, q: float32 or bfloat16 expected");
    at::Tensor out;
    if (queries) {
      const at::Tensor &q = tensor(a[6], "q: a tensor expected");
      rows_of(q, device, "q: [tokens, heads, dim] with a contiguous last dimension expected", &p.q_row, &p.q_head);
      out = given(a[7]) ? tensor(a[7], "q_out: a tensor expected") : empty(q.sizes(), q.scalar_type(), q);
      written(out, device, "q_out: [tokens, heads, dim] with a contiguous last dimension expected", &p.qo_row, &p.qo_head);
      if (q.size(0) != p.n || q.size(2) != p.head_dim || out.sizes() != q.sizes() || q.scalar_type() != lead.scalar_type() || out.scalar_type() != lead.scalar_type())
        refuse("q, q_out and k disagree in shape or type");
      p.n_heads = size32(q.size(1));
      p.q = data(q), p.q_out = data(out);
    }
    if (kv) {
      const at::Tensor &v = tensor(a[1], "v: a tensor expected"), &kc = tensor(a[2], "k_cache: a tensor expected"), &vc = tensor(a[3], "v_cache: a tensor expected");
      rows_of(lead, device, "k: [tokens, heads, dim] with a contiguous last dimension expected", &p.k_row, &p.k_head);
      rows_of(v, device, "v: [tokens, heads, dim] with a contiguous last dimension expected", &p.v_row, &p.v_head);
      written(kc, device, "k_cache: [slots, heads, dim] with a contiguous last dimension expected", &p.kc_slot, &p.kc_head);
      written(vc, device, "v_cache: [slots, heads, dim] with a contiguous last dimension expected", &p.vc_slot, &p.vc_head);
      p.kv_dtype = type_of(kc, "caches: float32 or bfloat16 expected");
      if (v.sizes() != lead.sizes() || v.scalar_type() != lead.scalar_type() || vc.sizes() != kc.sizes() || vc.scalar_type() != kc.scalar_type() ||
          kc.size(1) != lead.size(1) || kc.size(2) != lead.size(2))
        refuse("k, v and the caches disagree in shape or type");
      p.n_kv_heads = size32(lead.size(1));
      p.slots = kc.size(0);
      p.k = data(lead), p.v = data(v), p.k_cache = data(kc), p.v_cache = data(vc);
    }
    p.pos = ints(a[4], p.n, device, "pos: contiguous int32, one per token, expected");
    if (!p.pos && p.n) refuse("pos: contiguous int32, one per token, expected");
    p.index = ints(a[8], p.n, device, "index: contiguous int32, one per token, expected");
    p.seq = ints(a[9], p.n, device, "seq: contiguous int32, one per token, expected");
    const Table t = table(a[10], device, "table: int32 [sequences, pages] with contiguous rows expected");
    if (given(a[10]) && p.n && (!t.rows || !t.cols)) refuse("table: at least one page expected");   // (a null table would make places slots)
    p.table = t.at, p.table_row = t.row, p.table_rows = t.rows, p.table_cols = t.cols;
    p.page = int32(a[11]), p.pairs = int32(a[12]);
    if (given(a[5])) {
      const at::Tensor &r = tensor(a[5], "rope: a tensor expected");
      if (r.scalar_type() != at::kFloat || r.dim() != 3 || r.size(2) != 2 || !r.is_contiguous()) refuse("rope: contiguous float32 [positions, rot_dim / 2, 2] expected");
      on(device, r);
      p.rope = static_cast<const float *>(r.const_data_ptr()), p.rope_rows = size32(r.size(0)), p.rot_dim = size32(2 * r.size(1));
    }
    p.status = const_cast<int32_t *>(ints(a[13], 1, device, "status: contiguous int32 of one entry expected"));
    p.stream = c10::cuda::getCurrentCUDAStream(device).stream();
    const c10::cuda::CUDAGuard guard(device);
    check(g_append(&p), "spd_cache_append");
    if (!queries) Py_RETURN_NONE;
    if (given(a[7])) {
      Py_INCREF(a[7]);
      return a[7];
    }
    return THPVariable_Wrap(std::move(out));
  });
}

// shared_attention_bytes(n, b, g, heads, kv_heads, dim, x_dtype, kv_dtype): for calls with q_start, the larger need.
PyObject *shared_attention_bytes(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(8)
  return guarded([&]() -> PyObject * {
    spd_attention_args p = {};
    p.n = int32(a[0]), p.b = int32(a[1]), p.g = int32(a[2]), p.n_heads = int32(a[3]), p.n_kv_heads = int32(a[4]), p.head_dim = int32(a[5]);
    p.x_dtype = int32(a[6]), p.kv_dtype = int32(a[7]);
    static const int32_t some = 0;
    p.q_start = &some;
    size_t bytes = 0;
    check(g_attention_bytes(&p, &bytes), "spd_shared_attention_bytes");
    return PyLong_FromSize_t(bytes);
  });
}

// shared_attention(q, k_cache, v_cache, own_table, own_len, own_page, prefix_table, prefix_len, prefix_page, group_start, q_start,
//                  scale, out, return_lse, workspace, status)
PyObject *shared_attention(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(16)
  return guarded([&]() -> PyObject * {
    const at::Tensor &q = tensor(a[0], "q: a tensor expected"), &kc = tensor(a[1], "k_cache: a tensor expected"), &vc = tensor(a[2], "v_cache: a tensor expected");
    const int device = cuda_of(q);
    spd_attention_args p = {};
    rows_of(q, device, "q: [rows, heads, dim] with a contiguous last dimension expected", &p.q_row, &p.q_head);
    rows_of(kc, device, "k_cache: [slots, heads, dim] with a contiguous last dimension expected", &p.kc_slot, &p.kc_head);
    rows_of(vc, device, "v_cache: [slots, heads, dim] with a contiguous last dimension expected", &p.vc_slot, &p.vc_head);
    p.n = size32(q.size(0)), p.n_heads = size32(q.size(1)), p.head_dim = size32(q.size(2));
    p.slots = kc.size(0), p.n_kv_heads = size32(kc.size(1));
    p.x_dtype = type_of(q, "q: float32 or bfloat16 expected"), p.kv_dtype = type_of(kc, "caches: float32 or bfloat16 expected");
    if (vc.sizes() != kc.sizes() || vc.scalar_type() != kc.scalar_type() || kc.size(2) != q.size(2)) refuse("q and the caches disagree in shape or type");
    const Table own = table(a[3], device, "own_table: int32 [sequences, pages] with contiguous rows expected");
    if (!given(a[3])) refuse("own_table: int32 [sequences, pages] with contiguous rows expected");
    p.b = own.rows, p.own_table = own.at, p.own_row = own.row, p.own_cols = own.cols;
    p.own_len = ints(a[4], p.b, device, "own_len: contiguous int32, one per sequence, expected");
    if (!given(a[4])) refuse("own_len: contiguous int32, one per sequence, expected");
    p.own_page = int32(a[5]), p.prefix_page = int32(a[8]);
    if (given(a[6])) {
      const Table pre = table(a[6], device, "prefix_table: int32 [prefixes, pages] with contiguous rows expected");
      p.g = pre.rows, p.prefix_table = pre.at, p.prefix_row = pre.row, p.prefix_cols = pre.cols;
      p.prefix_len = ints(a[7], p.g, device, "prefix_len: contiguous int32, one per prefix, expected");
      if (!given(a[7])) refuse("prefix_len: contiguous int32, one per prefix, expected");
      p.group_start = ints(a[9], (int64_t)p.g + 1, device, "group_start: contiguous int32, one per prefix and one more, expected");
    }
    p.q_start = ints(a[10], (int64_t)p.b + 1, device, "q_start: contiguous int32, one per sequence and one more, expected");
    p.scale = given(a[11]) ? real(a[11]) : 1.f / std::sqrt((float)p.head_dim);
    at::Tensor out = given(a[12]) ? tensor(a[12], "out: a tensor expected") : empty(q.sizes(), q.scalar_type(), q), lse, space;
    written(out, device, "out: [rows, heads, dim] with a contiguous last dimension expected", &p.o_row, &p.o_head);
    if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type()) refuse("out and q disagree in shape or type");
    const bool with_lse = truth(a[13]);
    if (with_lse) {
      lse = empty({q.size(0), q.size(1)}, at::kFloat, q);
      p.lse = static_cast<float *>(data(lse));
    }
    p.q = data(q), p.k_cache = data(kc), p.v_cache = data(vc), p.out = data(out);
    p.status = const_cast<int32_t *>(ints(a[15], 1, device, "status: contiguous int32 of one entry expected"));
    p.stream = c10::cuda::getCurrentCUDAStream(device).stream();
    const c10::cuda::CUDAGuard guard(device);
    if (given(a[14])) {
      space = tensor(a[14], "workspace: a tensor expected");
      room(space, device);
    } else {
      size_t bytes = 0;
      check(g_attention_bytes(&p, &bytes), "spd_shared_attention_bytes");
      space = empty({(int64_t)bytes}, at::kByte, q);
    }
    p.workspace = data(space), p.workspace_bytes = (int64_t)space.nbytes();
    check(g_attention(&p), "spd_shared_attention");
    PyObject *o = a[12];
    if (given(o)) Py_INCREF(o);
    else if (!(o = THPVariable_Wrap(std::move(out)))) throw Raised();
    if (!with_lse) return o;
    PyObject *l = THPVariable_Wrap(std::move(lse));
    PyObject *pair = l ? PyTuple_New(2) : nullptr;
    if (!pair) {
      Py_DECREF(o);
      Py_XDECREF(l);
      throw Raised();
    }
    PyTuple_SET_ITEM(pair, 0, o);
    PyTuple_SET_ITEM(pair, 1, l);
    return pair;
  });
}

void select_shape(const at::Tensor &z, spd_select_args *p) {
  if (z.dim() != 3 || (z.stride(2) != 1 && z.size(2) > 1)) refuse("logits: [requests, beams, vocab] with a contiguous last dimension expected");
  p->x_dtype = type_of(z, "logits: float32 or bfloat16 expected");
  p->requests = size32(z.size(0)), p->beams = size32(z.size(1)), p->vocab = size32(z.size(2));
}
const at::Tensor &per_beam(PyObject *o, const at::Tensor &z, int device, at::ScalarType type, const char *what) {
  const at::Tensor &t = tensor(o, what);
  if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != z.size(0) || t.size(1) != z.size(1) || !t.is_contiguous()) refuse(what);
  on(device, t);
  return t;
}
// beam_select_bytes(logits)
PyObject *beam_select_bytes(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(1)
  return guarded([&]() -> PyObject * {
    spd_select_args p = {};
    select_shape(tensor(a[0], "logits: a tensor expected"), &p);
    size_t bytes = 0;
    check(g_select_bytes(&p, &bytes), "spd_beam_select_bytes");
    return PyLong_FromSize_t(bytes);
  });
}
// beam_select(logits, score, length, finished, eos_id, tau, length_alpha, workspace)
PyObject *beam_select(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(8)
  return guarded([&]() -> PyObject * {
    const at::Tensor &z = tensor(a[0], "logits: a tensor expected");
    const int device = cuda_of(z);
    spd_select_args p = {};
    select_shape(z, &p);
    const at::Tensor &score = per_beam(a[1], z, device, at::kFloat, "score: contiguous float32 [requests, beams] on the logits' device expected");
    if (given(a[2])) p.length = static_cast<const int32_t *>(data(per_beam(a[2], z, device, at::kInt, "length: contiguous int32 [requests, beams] on the logits' device expected")));
    if (given(a[3])) p.ended = static_cast<const uint8_t *>(data(per_beam(a[3], z, device, at::kBool, "finished: contiguous bool [requests, beams] on the logits' device expected")));
    p.eos_id = int32(a[4]), p.tau = real(a[5]), p.alpha = real(a[6]);
    const at::Tensor &space = tensor(a[7], "workspace: a tensor expected");
    room(space, device);
    const int64_t shape[2] = {z.size(0), z.size(1)};
    at::Tensor out[5] = {empty(shape, at::kInt, z), empty(shape, at::kInt, z), empty(shape, at::kFloat, z), empty(shape, at::kInt, z), empty(shape, at::kBool, z)};
    p.logits = data(z), p.score = static_cast<const float *>(data(score));
    p.new_token = static_cast<int32_t *>(data(out[0])), p.new_parent = static_cast<int32_t *>(data(out[1])), p.new_score = static_cast<float *>(data(out[2]));
    p.new_length = static_cast<int32_t *>(data(out[3])), p.new_ended = static_cast<uint8_t *>(data(out[4]));
    p.workspace = data(space), p.workspace_bytes = (int64_t)space.nbytes();
    p.request_stride = z.stride(0), p.beam_stride = z.stride(1);
    p.stream = c10::cuda::getCurrentCUDAStream(device).stream();
    const c10::cuda::CUDAGuard guard(device);
    check(g_select(&p), "spd_beam_select");
    PyObject *all = PyTuple_New(5);
    if (!all) throw Raised();
    for (int i = 0; i < 5; ++i) {
      PyObject *o = THPVariable_Wrap(std::move(out[i]));
      if (!o) {
        Py_DECREF(all);
        throw Raised();
      }
      PyTuple_SET_ITEM(all, i, o);
    }
    return all;
  });
}

// beam_reorder(states (a tuple or list), parent, dim, status)
PyObject *beam_reorder(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
  SPD_ARGS(4)
  return guarded([&]() -> PyObject * {
    const at::Tensor &parent = tensor(a[1], "parent: a tensor expected");
    const int device = cuda_of(parent);
    if (parent.dim() != 2 || parent.scalar_type() != at::kInt || !parent.is_contiguous()) refuse("parent: contiguous int32 [requests, beams] expected");
    const int64_t r = parent.size(0), w = parent.size(1), dim = integer(a[2]);
    if (dim < 0) refuse("dim: not negative");
    spd_reorder_args p = {};
    p.parent = static_cast<const int32_t *>(data(parent));
    p.requests = size32(r), p.beams = size32(w);
    p.status = const_cast<int32_t *>(ints(a[3], 1, device, "status: contiguous int32 of one entry expected"));
    p.stream = c10::cuda::getCurrentCUDAStream(device).stream();
    const c10::cuda::CUDAGuard guard(device);
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    PyObject **items = PySequence_Fast_ITEMS(a[0]);
    std::vector<const void *> starts;   // of the states that have rows to move
    const auto apart = [](int64_t stride, int64_t row) { return (stride < 0 ? -stride : stride) >= row; };
    for (int launch = 0; launch < 2; ++launch) {  // all states are looked over before the first is touched
      if (launch) {
        std::sort(starts.begin(), starts.end());
        if (std::adjacent_find(starts.begin(), starts.end()) != starts.end()) refuse("a state given twice");
      }
      for (Py_ssize_t first = 0; first < n; first += SPD_MAX_STATES) {
        p.n_states = (int32_t)(n - first < SPD_MAX_STATES ? n - first : SPD_MAX_STATES);
        for (int i = 0; i < p.n_states; ++i) {
          const at::Tensor &t = tensor(items[first + i], "states: tensors expected");
          on(device, t);
          const int64_t size = (int64_t)t.element_size();
          if (t.dim() < dim + 2 || t.size(dim) != r || t.size(dim + 1) != w) refuse("a state's dimensions `dim` and `dim` + 1 are not parent's requests and beams");
          int64_t row = 1, outer = 1, step = 0;
          for (int64_t k = t.dim() - 1; k > dim + 1; --k) {
            if (t.size(k) != 1 && t.stride(k) != row) refuse("what a beam of a state holds must be contiguous");
            row *= t.size(k);
          }
          for (int64_t k = dim - 1; k >= 0; --k) {
            if (t.size(k) == 1) continue;
            if (outer == 1) step = t.stride(k);
            else if (t.stride(k) != outer * step) refuse("a state's dimensions in front of the requests need one stride");
            outer *= t.size(k);
          }
          if (!launch && w > 1 && t.numel()) {
            if (!apart(t.stride(dim + 1), row) || (r > 1 && !apart(t.stride(dim), row)) || (outer > 1 && !apart(step, row))) refuse("a state's rows lie on one another");
            starts.push_back(t.const_data_ptr());
          }
          p.state[i] = data(t);
          p.outer[i] = outer, p.outer_stride[i] = step * size, p.request_stride[i] = t.stride(dim) * size, p.beam_stride[i] = t.stride(dim + 1) * size;
          p.row_bytes[i] = row * size;
        }
        if (launch) check(g_reorder(&p), "spd_beam_reorder");
      }
    }
    Py_RETURN_NONE;
  });
}

#define SPD_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {SPD_METHOD(bind), SPD_METHOD(cache_append), SPD_METHOD(shared_attention_bytes), SPD_METHOD(shared_attention),
                           SPD_METHOD(beam_select_bytes), SPD_METHOD(beam_select), SPD_METHOD(beam_reorder), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_spd_tensors", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__spd_tensors(void) { return PyModule_Create(&g_module); }
