// Marshalling of the operators that a decoding or training loop calls once a layer: checks of the tensors, allocation of the outputs, and the call of the
// C entry point.  It does what binding.py's other functions do in Python, where the checks and the packing of some twenty arguments take longer
// than most of these kernels run (one token's rotary: 9.8 us a call there, of which the launch is 3).
//
// Functions return their outputs, or the entry point's status as an int where it is not 0; binding.py raises it.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Functions.h>
#include <ATen/core/grad_mode.h>
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <initializer_list>
#include <map>
#include <string>
#include <utility>

#include "../../include/spec_b200.h"

namespace {

decltype(&spec_rotary) rotary_;
decltype(&spec_kv_append) append_;
decltype(&spec_kv_read) read_;
decltype(&spec_decode_attention) attend_;
decltype(&spec_decode_attention_workspace_bytes) workspace_bytes_;
decltype(&spec_embedding) embedding_;
decltype(&spec_embedding_backward_scratch_bytes) embedding_scratch_;
decltype(&spec_embedding_backward) embedding_backward_;
decltype(&spec_rms_norm) norm_;
decltype(&spec_rms_norm_backward_scratch_bytes) norm_scratch_;
decltype(&spec_rms_norm_backward) norm_backward_;
decltype(&spec_distill) distill_;

struct Refusal {
  PyObject *type;
  std::string what;
};
void need(bool ok, const char *what) {
  if (!ok) throw Refusal{PyExc_ValueError, what};
}

const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) throw Refusal{PyExc_TypeError, std::string(what) + " is a tensor"};
  return THPVariable_Unpack(o);
}
int dtype_of(at::ScalarType t) {
  if (t == at::kFloat) return SPEC_F32;
  if (t == at::kBFloat16) return SPEC_BF16;
  throw Refusal{PyExc_TypeError, std::string("unsupported dtype ") + c10::toString(t)};
}
bool truth(PyObject *o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw python_error();
  return t;
}
// The current device, asked for once a call (each of the binding's functions sets it to -1): a launch goes there, so every tensor has to be there.
thread_local int device_of_call = -1;
void *address(const at::Tensor &t) {
  if (device_of_call < 0) device_of_call = c10::cuda::current_device();
  need(t.is_cuda() && t.get_device() == device_of_call, "a tensor is on another device than the current one");
  return t.data_ptr();
}
// int32 of n elements, one behind the other, on the GPU
void *ints(PyObject *o, int64_t n, const char *what) {
  const at::Tensor &t = tensor(o, what);
  need(t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == n && t.is_cuda() && t.is_contiguous(), what);
  return address(t);
}
int32_t *status_of(PyObject *o) { return o == Py_None ? nullptr : (int32_t *)ints(o, 4, "status: int32 [4] on the GPU"); }

void *stream_of_call() { return c10::cuda::getCurrentCUDAStream(device_of_call).stream(); }      // after the first address()

struct Heads {
  void *p;
  int64_t ts, hs;
};
// [tokens][heads][head_dim] on the GPU with adjacent dimensions
Heads heads(const at::Tensor &t, const char *what) {
  need(t.dim() == 3 && t.is_cuda() && (t.stride(2) == 1 || t.size(2) == 1), what);
  for (int64_t n : t.sizes()) need(n <= INT32_MAX, "a tensor with more than 2^31 - 1 of something");
  return {address(t), t.stride(0), t.stride(1)};
}

bool rope_of(PyObject *freq, PyObject *layout, PyObject *mscale, spec_rope *r) {
  if (freq == Py_None) return false;
  const at::Tensor &f = tensor(freq, "inv_freq");
  need(f.scalar_type() == at::kDouble && f.dim() == 1 && f.is_contiguous() && f.is_cuda(), "inv_freq: float64 [pairs] on the GPU");
  const bool half = PyUnicode_Check(layout) && PyUnicode_CompareWithASCIIString(layout, "half") == 0;
  need(half || (PyUnicode_Check(layout) && PyUnicode_CompareWithASCIIString(layout, "interleaved") == 0), "layout is 'half' or 'interleaved'");
  const double m = PyFloat_AsDouble(mscale);
  if (m == -1.0 && PyErr_Occurred()) throw python_error();
  *r = spec_rope{(const double *)address(f), (int32_t)(2 * f.size(0)), half ? 0 : 1, (float)m};
  return true;
}

spec_kv_cache cache_of(PyObject *const *a) {             // k_pool, v_pool, page_table, k_scale, v_scale
  const at::Tensor &k = tensor(a[0], "k_pool"), &v = tensor(a[1], "v_pool"), &table = tensor(a[2], "page_table");
  spec_kv_cache c{};
  switch (k.scalar_type()) {
    case at::kFloat: c.format = SPEC_KV_F32; break;
    case at::kBFloat16: c.format = SPEC_KV_BF16; break;
    case at::kFloat8_e4m3fn: c.format = SPEC_KV_E4M3; break;
    case at::kChar: c.format = SPEC_KV_INT8; break;
    default: throw Refusal{PyExc_TypeError, std::string("unsupported cache dtype ") + c10::toString(k.scalar_type())};
  }
  need(k.dim() == 4 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type() && k.is_contiguous() && v.is_contiguous() && k.is_cuda() && v.is_cuda(),
       "pools: two contiguous [pages][kv heads][page size][head_dim] of one dtype on the GPU");
  need(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous() && table.is_cuda(), "page_table: contiguous int32 [sequences][pages] on the GPU");
  if (c.format >= SPEC_KV_E4M3) {
    for (int i = 3; i < 5; i++) {
      const char *what = "scales of an 8-bit cache: contiguous float32 [pages][kv heads][page size] on the GPU";
      need(a[i] != Py_None, what);
      const at::Tensor &s = tensor(a[i], what);
      need(s.scalar_type() == at::kFloat && s.sizes() == k.sizes().slice(0, 3) && s.is_contiguous() && s.is_cuda(), what);
      (i == 3 ? c.k_scale : c.v_scale) = (float *)address(s);
    }
  }
  for (int64_t n : {k.size(0), k.size(1), k.size(2), k.size(3), table.size(0), table.size(1)}) need(n <= INT32_MAX, "a cache with more than 2^31 - 1 of something");
  c.k = address(k);
  c.v = address(v);
  c.page_table = (const int32_t *)address(table);
  c.n_seq = (int32_t)table.size(0);
  c.pages_per_seq = (int32_t)table.size(1);
  c.num_pages = (int32_t)k.size(0);
  c.n_kv_heads = (int32_t)k.size(1);
  c.page_size = (int32_t)k.size(2);
  c.head_dim = (int32_t)k.size(3);
  return c;
}

template <typename F> PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f) {
  HANDLE_TH_ERRORS
  try {
    device_of_call = -1;
    if (have != want) throw Refusal{PyExc_TypeError, "wrong number of arguments"};
    return f();
  } catch (const Refusal &r) {
    PyErr_SetString(r.type, r.what.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
template <typename F> int call(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

// Whether autograd has to record a call on these: backwards, or forwards, where one carries a tangent (which no_grad does not turn off).
template <typename... T> bool records(const T &...t) {
  return (at::GradMode::is_enabled() && (... || (t.defined() && t.requires_grad()))) ||
         (c10::AutogradState::get_tls_state().get_fw_grad_mode() && (... || (t.defined() && t._fw_grad(0).defined())));
}

// x, positions, inv_freq, layout, mscale, out, transpose.  NotImplemented where autograd has to record it: binding.py wraps it then.
PyObject *rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject * {
    const at::Tensor &x = tensor(a[0], "x");
    const Heads from = heads(x, "rotary: x [tokens][heads][head_dim] on the GPU with adjacent dimensions");
    spec_rope r;
    const int dtype = dtype_of(x.scalar_type());
    const at::Tensor out = a[5] == Py_None ? at::empty(x.sizes(), x.options(), at::MemoryFormat::Contiguous) : tensor(a[5], "out");
    need(out.sizes() == x.sizes() && out.scalar_type() == x.scalar_type(), "rotary: out has x's shape and dtype");
    if (records(x, out)) Py_RETURN_NOTIMPLEMENTED;
    const Heads to = heads(out, "rotary: out [tokens][heads][head_dim] on the GPU with adjacent dimensions");
    need(rope_of(a[2], a[3], a[4], &r), "rotary: inv_freq");
    const int32_t *pos = (const int32_t *)ints(a[1], x.size(0), "rotary: positions int32 [tokens] on the GPU");
    void *const s = stream_of_call();
    const bool transpose = truth(a[6]);
    const int32_t T = (int32_t)x.size(0), H = (int32_t)x.size(1), hd = (int32_t)x.size(2);
    const int rc = call([&] { return rotary_(dtype, from.p, from.ts, from.hs, to.p, to.ts, to.hs, pos, T, H, hd, &r, transpose, s); });
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

// k, v, [k_pool, v_pool, page_table, k_scale, v_scale], row_seq, row_pos, row_kvpos, q, inv_freq, layout, mscale, status
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject * {
    const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
    const spec_kv_cache c = cache_of(a + 2);
    const Heads hk = heads(k, "kv_append: k [tokens][kv heads][head_dim] on the GPU with adjacent dimensions");
    const Heads hv = heads(v, "kv_append: v [tokens][kv heads][head_dim] on the GPU with adjacent dimensions");
    const int64_t T = k.size(0), hd = k.size(2);
    need(k.size(1) == c.n_kv_heads && hd == c.head_dim && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type(),
         "kv_append: k and v [tokens][kv heads][head_dim] of the cache's heads");
    const int dtype = dtype_of(k.scalar_type());
    at::Tensor q_out;
    Heads hq{nullptr, 0, 0};
    int64_t H = 0;
    if (a[10] != Py_None) {
      const at::Tensor &q = tensor(a[10], "q");
      hq = heads(q, "kv_append: q [tokens][heads][head_dim] on the GPU with adjacent dimensions");
      H = q.size(1);
      need(q.size(0) == T && q.size(2) == hd && q.scalar_type() == k.scalar_type(), "kv_append: q [tokens][heads][head_dim] of k's dtype");
      q_out = at::empty(q.sizes(), q.options(), at::MemoryFormat::Contiguous);
    }
    spec_rope r;
    const bool turn = rope_of(a[11], a[12], a[13], &r);
    const int32_t *seq = (const int32_t *)ints(a[7], T, "kv_append: row_seq int32 [tokens] on the GPU");
    const int32_t *pos = (const int32_t *)ints(a[8], T, "kv_append: row_pos int32 [tokens] on the GPU");
    const int32_t *kvpos = a[9] == Py_None ? nullptr : (const int32_t *)ints(a[9], T, "kv_append: row_kvpos int32 [tokens] on the GPU");
    int32_t *const status = status_of(a[14]);
    void *const s = stream_of_call();
    // a call without tokens has queries without an address
    const int rc = T == 0 ? SPEC_OK : call([&] {
      return append_(dtype, hq.p, hq.ts, hq.hs, q_out.defined() ? q_out.data_ptr() : nullptr, (int32_t)H, hk.p, hk.ts, hk.hs, hv.p, hv.ts, hv.hs, seq, pos, kvpos, (int32_t)T,
                     turn ? &r : nullptr, &c, status, s);
    });
    if (rc) return PyLong_FromLong(rc);
    if (!q_out.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(q_out);
  });
}

PyObject *pair(const at::Tensor &a, const at::Tensor &b) {
  PyObject *t = PyTuple_New(2);
  if (!t) return nullptr;
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  return t;
}

// [k_pool, v_pool, page_table, k_scale, v_scale], row_seq, row_kvpos, dtype's code, status
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject * {
    const spec_kv_cache c = cache_of(a);
    const at::Tensor &pool = THPVariable_Unpack(a[0]), &seq_t = tensor(a[5], "row_seq");
    const int64_t rows = seq_t.dim() == 1 ? seq_t.size(0) : -1;
    need(rows <= INT32_MAX, "a tensor with more than 2^31 - 1 of something");
    const int32_t *seq = (const int32_t *)ints(a[5], rows, "kv_read: row_seq int32 [rows] on the GPU");
    const int32_t *pos = (const int32_t *)ints(a[6], rows, "kv_read: row_kvpos int32 [rows] on the GPU");
    const long dtype = PyLong_AsLong(a[7]);
    if (dtype == -1 && PyErr_Occurred()) throw python_error();
    int32_t *const status = status_of(a[8]);
    const auto options = pool.options().dtype(dtype == SPEC_F32 ? at::kFloat : at::kBFloat16);
    const at::Tensor k = at::empty({rows, c.n_kv_heads, c.head_dim}, options), v = at::empty({rows, c.n_kv_heads, c.head_dim}, options);
    void *const s = stream_of_call();
    const int rc = call([&] { return read_(&c, seq, pos, (int32_t)rows, (int32_t)dtype, k.data_ptr(), v.data_ptr(), status, s); });
    return rc ? PyLong_FromLong(rc) : pair(k, v);
  });
}

// A workspace for each stream that a call without one of its own was made on, kept for the next.  A graph never gets it: its replays may run on
// any stream, beside the stream's own calls or another graph's.  (Never taken down: the process's end may have taken the driver down first.)
at::Tensor workspace_of(const at::Tensor &q, void *stream) {
  need(c10::cuda::currentStreamCaptureStatusMayInitCtx() == c10::cuda::CaptureStatus::None, "decode_attention: under graph capture a workspace of decode_workspace()");
  static auto *kept = new std::map<std::pair<int, void *>, at::Tensor>;
  at::Tensor &w = (*kept)[{(int)q.get_device(), stream}];
  if (!w.defined()) w = at::zeros({(int64_t)workspace_bytes_()}, q.options().dtype(at::kByte));
  return w;
}

// q, [k_pool, v_pool, page_table, k_scale, v_scale], lengths, scale, want_lse, out, workspace, status
PyObject *decode_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject * {
    const at::Tensor &q = tensor(a[0], "q");
    const spec_kv_cache c = cache_of(a + 1);
    const Heads hq = heads(q, "decode_attention: q [batch][heads][head_dim] on the GPU, heads adjacent");
    const int64_t B = q.size(0), H = q.size(1), hd = q.size(2);
    need(hd == c.head_dim && (hq.hs == hd || H == 1), "decode_attention: q [batch][heads][head_dim] on the GPU, heads adjacent");
    const int dtype = dtype_of(q.scalar_type());
    double scale = 0.0;
    if (a[7] != Py_None) {
      scale = PyFloat_AsDouble(a[7]);
      if (scale == -1.0 && PyErr_Occurred()) throw python_error();
      need((float)scale < 0 || (float)scale > 0, "decode_attention: scale is a number, and not 0 in 32 bits");      // 0: the entry point's default
    }
    const at::Tensor out = a[9] == Py_None ? at::empty(q.sizes(), q.options(), at::MemoryFormat::Contiguous) : tensor(a[9], "out");
    need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type() && out.is_contiguous() && out.is_cuda(), "decode_attention: out contiguous, of q's shape and dtype");
    void *const to = address(out);
    const bool want_lse = truth(a[8]);
    at::Tensor lse;
    if (want_lse) lse = at::empty({B, H}, q.options().dtype(at::kFloat));
    const int32_t *length = (const int32_t *)ints(a[6], B, "decode_attention: lengths int32 [batch] on the GPU");
    int32_t *const status = status_of(a[11]);
    void *const s = stream_of_call();
    const at::Tensor w = a[10] == Py_None ? workspace_of(q, s) : tensor(a[10], "workspace");
    need(w.is_cuda() && w.is_contiguous(), "decode_attention: workspace of decode_workspace()");
    void *const work = address(w);
    const int rc = call([&] {
      return attend_(dtype, hq.p, hq.ts, &c, length, (int32_t)B, (int32_t)H, (float)scale, to, want_lse ? (float *)lse.data_ptr() : nullptr, work, w.nbytes(),
                     status, s);
    });
    if (rc) return PyLong_FromLong(rc);
    return want_lse ? pair(out, lse) : THPVariable_Wrap(out);
  });
}

// ---------------------------------------------------------------- embedding, norms, distillation: rows of elements
double number(PyObject *o, const char *what) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refusal{PyExc_TypeError, what};
  }
  return v;
}
at::ScalarType type_or(PyObject *o, at::ScalarType otherwise, const char *what) {
  if (o == Py_None) return otherwise;
  if (!THPDtype_Check(o)) throw Refusal{PyExc_TypeError, what};
  return ((THPDtype *)o)->scalar_type;
}
int row_type(at::ScalarType t, bool eight = false) {
  if (eight && t == at::kFloat8_e4m3fn) return SPEC_KV_E4M3;
  if (eight && t == at::kChar) return SPEC_KV_INT8;
  return dtype_of(t);                                    // the codes of fp32 and bf16 are the same
}
// [rows][columns] on the GPU with adjacent columns
spec_rows rows_of(const at::Tensor &t, const char *what, bool eight = false) {
  need(t.dim() == 2 && t.is_cuda() && (t.stride(1) == 1 || t.size(1) == 1), what);
  for (int64_t n : t.sizes()) need(n <= INT32_MAX, "a tensor with more than 2^31 - 1 of something");
  return {address(t), t.stride(0), row_type(t.scalar_type(), eight)};
}
struct IdList {
  const void *p;
  int bits;
};
IdList ids_of(const at::Tensor &t, const char *what) {
  need((t.scalar_type() == at::kInt || t.scalar_type() == at::kLong) && t.is_cuda() && t.is_contiguous(), what);
  for (int64_t n : t.sizes()) need(n <= INT32_MAX, "a tensor with more than 2^31 - 1 of something");
  return {address(t), t.scalar_type() == at::kInt ? 32 : 64};
}
// float32 of this shape up to dimensions of 1, or flat, contiguous on the GPU
float *floats(PyObject *o, std::initializer_list<int64_t> shape, const char *what) {
  const at::Tensor &t = tensor(o, what);
  int64_t n = 1;
  for (int64_t k : shape) n *= k;
  bool fits = t.dim() >= 1 && t.numel() == n;
  if (fits && t.dim() > 1) {
    auto at = shape.begin();
    for (int64_t k : t.sizes()) {
      if (k == 1) continue;
      while (at != shape.end() && *at == 1) at++;
      fits = fits && at != shape.end() && *at++ == k;
    }
  }
  need(t.scalar_type() == at::kFloat && fits && t.is_cuda() && t.is_contiguous(), what);
  return (float *)address(t);
}
at::Tensor scratch_of(size_t bytes, const at::Tensor &like) { return at::empty({(int64_t)std::max<size_t>(bytes, 256)}, like.options().dtype(at::kByte)); }
// A caller's tensor is about to be written: autograd refuses to go back through what saved it before.
void written(const at::Tensor &t) { t.unsafeGetTensorImpl()->bump_version(); }

// ids, weight, scale, dtype, out, status.  NotImplemented where autograd has to record it: binding.py wraps it then (as those below).
PyObject *embedding(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject * {
    const char *const what = "embedding: weight [vocabulary][width] on the GPU with adjacent columns", *const ids_are = "embedding: ids int32 or int64 [tokens], contiguous on the GPU";
    const at::Tensor &ids = tensor(a[0], ids_are), &w = tensor(a[1], what);
    const spec_rows from = rows_of(w, what);
    const double scale = number(a[2], "embedding: scale is a number");
    need(ids.dim() == 1, ids_are);
    const IdList id = ids_of(ids, ids_are);
    const int64_t T = ids.size(0), k = w.size(1);
    const at::ScalarType type = type_or(a[3], a[4] == Py_None ? w.scalar_type() : tensor(a[4], "out").scalar_type(), "embedding: dtype is a torch.dtype");
    row_type(type);
    const at::Tensor out = a[4] == Py_None ? at::empty({T, k}, w.options().dtype(type)) : tensor(a[4], "out");
    need(out.dim() == 2 && out.size(0) == T && out.size(1) == k && out.scalar_type() == type, "embedding: out [tokens][width] of dtype");
    if (records(w, out)) Py_RETURN_NOTIMPLEMENTED;
    const spec_rows to = rows_of(out, "embedding: out [tokens][width] on the GPU with adjacent columns");
    int32_t *const status = status_of(a[5]);
    void *const s = stream_of_call();
    if (a[4] != Py_None) written(out);
    const int rc = call([&] { return embedding_(&from, (int32_t)w.size(0), (int32_t)k, id.bits, id.p, (int32_t)T, (float)scale, &to, status, s); });
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

// grad, ids, vocab, scale, dtype, out, accumulate, status
PyObject *embedding_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject * {
    const char *const what = "embedding_backward: grad [tokens][width] on the GPU with adjacent columns", *const ids_are = "embedding_backward: ids int32 or int64 [tokens], contiguous on the GPU";
    const at::Tensor &g = tensor(a[0], what), &ids = tensor(a[1], ids_are);
    const spec_rows from = rows_of(g, what);
    const int64_t T = g.size(0), k = g.size(1);
    need(ids.dim() == 1 && ids.size(0) == T, ids_are);
    const IdList id = ids_of(ids, ids_are);
    const long long V = PyLong_AsLongLong(a[2]);
    if (V == -1 && PyErr_Occurred()) throw python_error();
    need(V >= 1 && V <= INT32_MAX, "embedding_backward: vocab is a number of rows");
    const double scale = number(a[3], "embedding_backward: scale is a number");
    const bool accumulate = truth(a[6]);
    need(!accumulate || a[5] != Py_None, "embedding_backward: accumulate goes with out");
    const at::ScalarType type = type_or(a[4], a[5] == Py_None ? g.scalar_type() : tensor(a[5], "out").scalar_type(), "embedding_backward: dtype is a torch.dtype");
    row_type(type);
    const at::Tensor out = a[5] == Py_None ? at::empty({V, k}, g.options().dtype(type)) : tensor(a[5], "out");
    need(out.dim() == 2 && out.size(0) == V && out.size(1) == k && out.scalar_type() == type && !records(out), "embedding_backward: out [vocabulary][width] of dtype, without a gradient");
    const spec_rows to = rows_of(out, "embedding_backward: out [vocabulary][width] on the GPU with adjacent columns");
    int32_t *const status = status_of(a[7]);
    void *const s = stream_of_call();
    const size_t bytes = embedding_scratch_((int32_t)T, (int32_t)V, (int32_t)k);
    const at::Tensor scratch = scratch_of(bytes, g);
    if (a[5] != Py_None) written(out);
    const int rc = call([&] {
      return embedding_backward_(&from, id.bits, id.p, (int32_t)T, (int32_t)V, (int32_t)k, (float)scale, accumulate, &to, scratch.data_ptr(), scratch.nbytes(), status, s);
    });
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  });
}

PyObject *several(std::initializer_list<at::Tensor> t) {
  PyObject *r = PyTuple_New((Py_ssize_t)t.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor &x : t) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(x));
  return r;
}
const void *gain_of(const at::Tensor &w, int64_t k, const char *what) {
  need(w.dim() == 1 && w.size(0) == k && w.is_cuda() && w.is_contiguous(), what);
  return address(w);
}

// x, gain, eps, residual, dtype, group, sum_out
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject * {
    const char *const what = "rms_norm: x [rows][width] on the GPU with adjacent columns", *const gain_is = "rms_norm: gain [width] on the GPU";
    const at::Tensor &x = tensor(a[0], what), &w = tensor(a[1], gain_is);
    const spec_rows from = rows_of(x, what);
    const int64_t R = x.size(0), k = x.size(1);
    const int gain_type = dtype_of(w.scalar_type());
    const void *const gain = gain_of(w, k, gain_is);
    const double eps = number(a[2], "rms_norm: eps is a number");
    const at::ScalarType type = type_or(a[4], x.scalar_type(), "rms_norm: dtype is a torch.dtype");
    const bool eight = row_type(type, true) >= SPEC_KV_E4M3;
    const long group = PyLong_AsLong(a[5]);
    if (group == -1 && PyErr_Occurred()) throw python_error();
    need(group >= 0 && group % 16 == 0 && group <= INT32_MAX, "rms_norm: group is 0 or a multiple of 16");
    at::Tensor res, sum, scale;
    spec_rows add{}, total{};
    if (a[3] != Py_None) {
      const char *const res_is = "rms_norm: residual [rows][width] on the GPU with adjacent columns", *const sum_is = "rms_norm: sum_out [rows][width] of residual's dtype on the GPU with adjacent columns";
      res = tensor(a[3], res_is);
      need(res.sizes() == x.sizes(), res_is);
      add = rows_of(res, res_is);
      if (a[6] != Py_None) {
        sum = tensor(a[6], sum_is);
        need(sum.sizes() == x.sizes() && sum.scalar_type() == res.scalar_type(), sum_is);
      } else {
        sum = at::empty({R, k}, res.options());
      }
      total = rows_of(sum, sum_is);
    } else {
      need(a[6] == Py_None, "rms_norm: sum_out goes with residual");
    }
    if (records(x, w, res, sum)) Py_RETURN_NOTIMPLEMENTED;
    const at::Tensor y = at::empty({R, k}, x.options().dtype(type));
    const spec_rows to = rows_of(y, "y", true);
    if (a[6] != Py_None) written(sum);
    if (eight) scale = at::empty({R, k == 0 ? 0 : group ? (k + group - 1) / group : 1}, x.options().dtype(at::kFloat));
    void *const s = stream_of_call();
    const int rc = call([&] {
      return norm_(&from, res.defined() ? &add : nullptr, gain_type, gain, (float)eps, res.defined() ? &total : nullptr, &to, eight ? (float *)scale.data_ptr() : nullptr,
                   eight ? (int32_t)group : 0, (int32_t)R, (int32_t)k, s);
    });
    if (rc) return PyLong_FromLong(rc);
    if (eight) return res.defined() ? several({y, scale, sum}) : several({y, scale});
    return res.defined() ? several({y, sum}) : THPVariable_Wrap(y);
  });
}

// grad, s, gain, eps, grad_sum, dtype
PyObject *rms_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject * {
    const char *const grad_is = "rms_norm_backward: grad [rows][width] on the GPU with adjacent columns", *const x_is = "rms_norm_backward: x [rows][width] on the GPU with adjacent columns",
                      *const gain_is = "rms_norm_backward: gain [width] on the GPU", *const sum_is = "rms_norm_backward: grad_sum [rows][width] on the GPU with adjacent columns";
    const at::Tensor &g = tensor(a[0], grad_is), &x = tensor(a[1], x_is), &w = tensor(a[2], gain_is);
    const spec_rows of_y = rows_of(g, grad_is), of_x = rows_of(x, x_is);
    const int64_t R = x.size(0), k = x.size(1);
    need(g.sizes() == x.sizes(), grad_is);
    const int gain_type = dtype_of(w.scalar_type());
    const void *const gain = gain_of(w, k, gain_is);
    const double eps = number(a[3], "rms_norm_backward: eps is a number");
    spec_rows carried{};
    if (a[4] != Py_None) {
      const at::Tensor &c = tensor(a[4], sum_is);
      need(c.sizes() == x.sizes(), sum_is);
      carried = rows_of(c, sum_is);
    }
    const at::ScalarType type = type_or(a[5], x.scalar_type(), "rms_norm_backward: dtype is a torch.dtype");
    row_type(type);
    const at::Tensor dx = at::empty({R, k}, x.options().dtype(type)), dw = at::empty({k}, w.options());
    const spec_rows to = rows_of(dx, "dx");
    void *const s = stream_of_call();
    const at::Tensor scratch = scratch_of(norm_scratch_((int32_t)R, (int32_t)k), x);
    const int rc = call([&] {
      return norm_backward_(&of_y, &of_x, gain_type, gain, (float)eps, a[4] != Py_None ? &carried : nullptr, &to, dw.data_ptr(), scratch.data_ptr(), scratch.nbytes(), (int32_t)R,
                            (int32_t)k, s);
    });
    return rc ? PyLong_FromLong(rc) : several({dx, dw});
  });
}

// logits, ids, values, id_map, values_lse, temperature, kl, grad, stats, want: 0 the loss, 1 the loss and stats, 2 the gradient from stats, 3 loss and gradient; dtype, out, status
PyObject *distill(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject * {
    const char *const z_is = "distill_loss: logits [rows][vocabulary] on the GPU with adjacent columns", *const ids_are = "distill_loss: ids int32 or int64 [rows][K], contiguous on the GPU",
                      *const values_are = "distill_loss: values [rows][K], contiguous on the GPU, without a gradient";
    const at::Tensor &z = tensor(a[0], z_is), &ids = tensor(a[1], ids_are), &v = tensor(a[2], values_are);
    const spec_rows from = rows_of(z, z_is);
    const int64_t R = z.size(0), V = z.size(1);
    need(ids.dim() == 2 && ids.size(0) == R, ids_are);
    const IdList id = ids_of(ids, ids_are);
    need(v.sizes() == ids.sizes() && v.is_cuda() && v.is_contiguous() && !records(v), values_are);
    spec_teacher t{id.p, address(v), nullptr, nullptr, id.bits, dtype_of(v.scalar_type()), 0, (int32_t)ids.size(1)};
    if (a[3] != Py_None) {
      const at::Tensor &map = tensor(a[3], "distill_loss: id_map");
      need(map.numel() > 0, "distill_loss: id_map without an entry");      // and so without an address, which would stand for no map
      t.id_map_n = (int32_t)std::min<int64_t>(map.numel(), INT32_MAX);
      t.id_map = (const int32_t *)ints(a[3], t.id_map_n, "distill_loss: id_map int32 [teacher's vocabulary] on the GPU");
    }
    if (a[4] != Py_None) {
      need(!records(tensor(a[4], "distill_loss: values_lse")), "distill_loss: values_lse without a gradient");
      t.lse = floats(a[4], {R}, "distill_loss: values_lse float32 [rows] on the GPU");
    }
    const double temperature = number(a[5], "distill_loss: temperature is a number");
    const bool kl = truth(a[6]);
    const long want = PyLong_AsLong(a[9]);
    if (want < 2 && records(z)) Py_RETURN_NOTIMPLEMENTED;
    const float *const grad = a[7] == Py_None ? nullptr : floats(a[7], {R}, "distill_loss: grad float32 [rows] on the GPU");
    at::Tensor loss, stats, dz;
    float *known = nullptr;
    if (want != 2) loss = at::empty({R}, z.options().dtype(at::kFloat));
    if (want == 1) stats = at::empty({R, 2}, z.options().dtype(at::kFloat)), known = (float *)stats.data_ptr();
    if (want == 2) known = floats(a[8], {R, 2}, "distill_loss: stats float32 [rows][2] on the GPU");
    spec_rows to{};
    if (want >= 2) {
      const char *const out_is = "distill_loss: out [rows][vocabulary] of dtype on the GPU with adjacent columns, without a gradient";
      const at::ScalarType type = type_or(a[10], a[11] == Py_None ? z.scalar_type() : tensor(a[11], out_is).scalar_type(), "distill_loss: dtype is a torch.dtype");
      row_type(type);
      dz = a[11] == Py_None ? at::empty({R, V}, z.options().dtype(type)) : tensor(a[11], out_is);
      need(dz.sizes() == z.sizes() && dz.scalar_type() == type && (a[11] == Py_None || !records(dz)), out_is);
      to = rows_of(dz, out_is);
      if (a[11] != Py_None) written(dz);
    }
    int32_t *const status = status_of(a[12]);
    void *const s = stream_of_call();
    const int rc = call([&] {
      return distill_(&from, (int32_t)R, (int32_t)V, &t, (float)temperature, kl, grad, loss.defined() ? (float *)loss.data_ptr() : nullptr, known, dz.defined() ? &to : nullptr, status, s);
    });
    if (rc) return PyLong_FromLong(rc);
    if (want == 1) return several({loss, stats});
    if (want == 3) return several({loss, dz});
    return THPVariable_Wrap(want == 2 ? dz : loss);
  });
}

// addresses of the entry points, in the order of the declarations above
PyObject *use(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject * {
    void *p[12];
    for (int i = 0; i < 12; i++) {
      p[i] = PyLong_AsVoidPtr(a[i]);
      if (!p[i]) throw Refusal{PyExc_ValueError, "an entry point without an address"};
    }
    rotary_ = (decltype(rotary_))p[0];
    append_ = (decltype(append_))p[1];
    read_ = (decltype(read_))p[2];
    attend_ = (decltype(attend_))p[3];
    workspace_bytes_ = (decltype(workspace_bytes_))p[4];
    embedding_ = (decltype(embedding_))p[5];
    embedding_scratch_ = (decltype(embedding_scratch_))p[6];
    embedding_backward_ = (decltype(embedding_backward_))p[7];
    norm_ = (decltype(norm_))p[8];
    norm_scratch_ = (decltype(norm_scratch_))p[9];
    norm_backward_ = (decltype(norm_backward_))p[10];
    distill_ = (decltype(distill_))p[11];
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {{"rotary", (PyCFunction)(void *)rotary, METH_FASTCALL, nullptr},
                         {"kv_append", (PyCFunction)(void *)kv_append, METH_FASTCALL, nullptr},
                         {"kv_read", (PyCFunction)(void *)kv_read, METH_FASTCALL, nullptr},
                         {"decode_attention", (PyCFunction)(void *)decode_attention, METH_FASTCALL, nullptr},
                         {"embedding", (PyCFunction)(void *)embedding, METH_FASTCALL, nullptr},
                         {"embedding_backward", (PyCFunction)(void *)embedding_backward, METH_FASTCALL, nullptr},
                         {"rms_norm", (PyCFunction)(void *)rms_norm, METH_FASTCALL, nullptr},
                         {"rms_norm_backward", (PyCFunction)(void *)rms_norm_backward, METH_FASTCALL, nullptr},
                         {"distill", (PyCFunction)(void *)distill, METH_FASTCALL, nullptr},
                         {"use", (PyCFunction)(void *)use, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of the operators beside the step", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
