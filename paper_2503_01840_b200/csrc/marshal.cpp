// Marshalling of the operators that a decoding loop calls once a layer: checks of the tensors, allocation of the outputs, and the call of the
// C entry point.  It does what binding.py's other functions do in Python, where the checks and the packing of some twenty arguments take longer
// than most of these kernels run (one token's rotary: 9.8 us a call there, of which the launch is 3).
//
// Functions return their outputs, or the entry point's status as an int where it is not 0; binding.py raises it.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Functions.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAStream.h>

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

// x, positions, inv_freq, layout, mscale, out, transpose.  NotImplemented where autograd has to record it: binding.py wraps it then.
PyObject *rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject * {
    const at::Tensor &x = tensor(a[0], "x");
    const Heads from = heads(x, "rotary: x [tokens][heads][head_dim] on the GPU with adjacent dimensions");
    spec_rope r;
    const int dtype = dtype_of(x.scalar_type());
    const at::Tensor out = a[5] == Py_None ? at::empty(x.sizes(), x.options(), at::MemoryFormat::Contiguous) : tensor(a[5], "out");
    need(out.sizes() == x.sizes() && out.scalar_type() == x.scalar_type(), "rotary: out has x's shape and dtype");
    if (at::GradMode::is_enabled() && (x.requires_grad() || out.requires_grad())) Py_RETURN_NOTIMPLEMENTED;
    const Heads to = heads(out, "rotary: out [tokens][heads][head_dim] on the GPU with adjacent dimensions");
    need(rope_of(a[2], a[3], a[4], &r), "rotary: inv_freq");
    const int32_t *pos = (const int32_t *)ints(a[1], x.size(0), "rotary: positions int32 [tokens] on the GPU");
    void *const s = stream_of_call();
    const bool transpose = PyObject_IsTrue(a[6]) == 1;
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
    const bool want_lse = PyObject_IsTrue(a[8]) == 1;
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

// addresses of the entry points, in the order of the declarations above
PyObject *use(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject * {
    void *p[5];
    for (int i = 0; i < 5; i++) {
      p[i] = PyLong_AsVoidPtr(a[i]);
      if (!p[i]) throw Refusal{PyExc_ValueError, "an entry point without an address"};
    }
    rotary_ = (decltype(rotary_))p[0];
    append_ = (decltype(append_))p[1];
    read_ = (decltype(read_))p[2];
    attend_ = (decltype(attend_))p[3];
    workspace_bytes_ = (decltype(workspace_bytes_))p[4];
    Py_RETURN_NONE;
  });
}

PyMethodDef methods[] = {{"rotary", (PyCFunction)(void *)rotary, METH_FASTCALL, nullptr},
                         {"kv_append", (PyCFunction)(void *)kv_append, METH_FASTCALL, nullptr},
                         {"kv_read", (PyCFunction)(void *)kv_read, METH_FASTCALL, nullptr},
                         {"decode_attention", (PyCFunction)(void *)decode_attention, METH_FASTCALL, nullptr},
                         {"use", (PyCFunction)(void *)use, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of the operators of serving loops", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
