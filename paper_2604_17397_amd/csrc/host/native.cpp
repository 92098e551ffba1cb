// Argument marshalling of the calls a denoising loop makes most often (attention, rotary embedding, the routing
// decision, commit, rollback, snapshot) and of the paged cache's, in C++: the same checks and the same call into libsdvg as
// binding.py makes. Every function either finds all checks of its Python counterpart satisfied and
// makes the call, or returns None without having done anything; the Python counterpart then takes
// over, raises what it always raised, or handles the rarer form (fp32, tensor subclasses, ...).
//
// Why: on a small layer the GPU is done in 4 to 16 us, while checking and converting six tensors
// through ctypes took 15 us per attention call and 12 per rotary pass. A batch of 1, 2 or 3 items took 21, 32 and 43 us,
// commit, rollback and snapshot 7 to 10, which the GPU waits for behind a routing decision. The paged cache's calls took 15
// (plan) to 23 us (attention).
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/core/Stream.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>

#include <string.h>

#include <optional>

#include "sdvg.h"

namespace {

constexpr int kMaxItems = 8;  // of a batch; larger ones are Python's, which raises

using attn_fn = int (*)(const sdvg_attn_desc *, const void *, const void *, const void *, const void *, const void *,
                        int64_t, void *, void *);
using attn_commit_fn = int (*)(const sdvg_attn_desc *, const void *, void *, void *, const void *, const void *, int64_t,
                               void *, void *);
using rope_fn = int (*)(const void *, const float *, const float *, void *, int64_t, int32_t, int32_t, int64_t, int64_t,
                        int64_t, int64_t, void *);
using route_fn = int (*)(const float *, int32_t, float, int32_t, float *, void *);
using batch_fn = int (*)(const sdvg_attn_desc *, int32_t, const void *const *, const void *const *, const void *const *,
                         const void *const *, const void *const *, int64_t, void *const *, void *, int64_t, int32_t, void *);
using batch_static_fn = int (*)(const sdvg_attn_desc *, int32_t, const void *const *, const void *const *,
                                const void *const *, const void *const *, const void *const *, int64_t, void *const *,
                                int32_t, void *);
using commit_fn = int (*)(sdvg_kv_cache *, const void *, const void *, int32_t, void *);
using commit_rope_fn = int (*)(sdvg_kv_cache *, const void *, const void *, int32_t, const float *, const float *, void *);
using rollback_fn = int (*)(sdvg_kv_cache *, int64_t, void *);
using snapshot_fn = int (*)(void *, const void *, int64_t, void *);
using page_plan_fn = int (*)(const sdvg_page_plan_args *, void *);
using rope_positions_fn = int (*)(const sdvg_rope_desc *, const sdvg_rows *, const sdvg_rows *, int64_t, int32_t, int32_t, void *);
using paged_commit_fn = int (*)(const sdvg_paged_kv *, const sdvg_rows *, const sdvg_rows *, const int64_t *, int64_t, int32_t,
                                const sdvg_rope_desc *, const sdvg_rows *, void *);
using paged_attn_fn = int (*)(const sdvg_paged_attn_desc *, const sdvg_paged_kv *, const void *, const int32_t *, const int32_t *,
                              const int32_t *, void *, float *, void *, int64_t, void *);
using paged_prefix_attn_fn = int (*)(const sdvg_paged_attn_desc *, const sdvg_paged_kv *, const void *, const int32_t *, const int32_t *,
                                     const int32_t *, int32_t, const int32_t *, const int32_t *, void *, float *, void *, int64_t, void *);
using sample_tokens_fn = int (*)(const sdvg_sample_args *, void *, int64_t, void *);

// Entry points of the libsdvg that binding.py has loaded, and torch's current-stream functions.
struct Api {
  attn_fn attn = nullptr;
  attn_commit_fn attn_commit = nullptr;
  rope_fn rope = nullptr;
  route_fn route_min = nullptr, route_mean = nullptr;
  batch_fn batch = nullptr;
  batch_static_fn batch_static = nullptr;
  commit_fn commit = nullptr;
  commit_rope_fn commit_rope = nullptr;
  rollback_fn rollback = nullptr;
  snapshot_fn snapshot = nullptr;
  page_plan_fn page_plan = nullptr;
  rope_positions_fn rope_positions = nullptr;
  paged_commit_fn paged_commit = nullptr;
  paged_attn_fn paged_attn = nullptr;
  paged_prefix_attn_fn paged_prefix_attn = nullptr;
  sample_tokens_fn sample_tokens = nullptr;
  PyObject *get_device = nullptr, *get_raw_stream = nullptr, *float32 = nullptr, *cache_type = nullptr, *paged_type = nullptr;
} api;

// A plain strided GPU tensor, or null (subclasses, wrappers and CPU tensors are Python's).
const at::Tensor *gpu_tensor(PyObject *o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.unsafeGetTensorImpl()->is_python_dispatch())
    return nullptr;
  return &t;
}

bool integer(PyObject *o, int64_t &v) {
  if (!PyLong_CheckExact(o)) return false;
  v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// The stream to launch on: torch's current one for None, else the raw pointer binding.py passes.
bool stream_ptr(PyObject *o, void *&s) {
  if (o != Py_None) {
    int64_t v;
    if (!integer(o, v)) return false;
    s = reinterpret_cast<void *>(v);
    return true;
  }
  PyObject *dev = PyObject_CallNoArgs(api.get_device);
  PyObject *raw = dev ? PyObject_CallOneArg(api.get_raw_stream, dev) : nullptr;
  Py_XDECREF(dev);
  int64_t v;
  const bool ok = raw && integer(raw, v);
  Py_XDECREF(raw);
  if (!ok) {
    PyErr_Clear();
    return false;
  }
  s = reinterpret_cast<void *>(v);
  return true;
}

// Makes `stream` a device's current one for as long as this lives, unless the call names none (`given` is None): 0.1 us of the host's time,
// 8 in Python.
struct StreamGuard {
  std::optional<c10::Stream> before;
  StreamGuard(PyObject *given, const at::Device &device, void *stream) {
    if (given == Py_None) return;
    // (a stream that torch did not make has its pointer for an id, and one that it made is the same to the allocator by its pointer)
    before = c10::impl::getDeviceGuardImpl(device.type())
                 ->exchangeStream(c10::Stream(c10::Stream::UNSAFE, device, reinterpret_cast<c10::StreamId>(stream)));
  }
  ~StreamGuard() {
    if (before) c10::impl::getDeviceGuardImpl(before->device_type())->exchangeStream(*before);
  }
  StreamGuard(const StreamGuard &) = delete;
  StreamGuard &operator=(const StreamGuard &) = delete;
};

// The output tensor: the one given if it matches `like`, a new one for None; undefined if neither. A new one comes from the memory of
// the call's stream, as in binding.py.
at::Tensor output(PyObject *o, const at::Tensor &like, PyObject *given_stream, void *stream) {
  if (o == Py_None) {
    const StreamGuard guard(given_stream, like.device(), stream);
    at::Tensor out = at::empty(like.sizes(), at::TensorOptions().dtype(like.scalar_type()).device(like.device()));
    return out.unsafeGetTensorImpl()->is_python_dispatch() ? at::Tensor() : out;
  }
  const at::Tensor *out = gpu_tensor(o);
  if (!out || out->sizes() != like.sizes() || out->scalar_type() != like.scalar_type() || out->stride(2) != 1 ||
      out->device() != like.device())
    return at::Tensor();
  return *out;
}

// What a call returns to binding.py: the output for status 0, the status otherwise.
PyObject *result(int status, PyObject *given, const at::Tensor &out) {
  if (status != 0) return PyLong_FromLong(status);
  if (given == Py_None) return THPVariable_Wrap(out);
  Py_INCREF(given);
  return given;
}

#define PYTHON_TAKES_OVER \
  do {                    \
    Py_RETURN_NONE;       \
  } while (0)

// One (q, k_cache, v_cache, k_blk, v_blk) set that passes every check but the output's.
struct Item {
  const at::Tensor *q, *kc, *vc, *kb, *vb;  // kc, vc null without a cache
};
bool attn_item(PyObject *const *a, int64_t cache_len, Item &it) {
  const bool cached = a[1] != Py_None;
  it = Item{gpu_tensor(a[0]), cached ? gpu_tensor(a[1]) : nullptr, cached ? gpu_tensor(a[2]) : nullptr, gpu_tensor(a[3]),
            gpu_tensor(a[4])};
  if (!it.q || !it.kb || !it.vb || cache_len < 0) return false;
  if (cached ? (!it.kc || !it.vc) : (a[2] != Py_None || cache_len > 0)) return false;
  const at::Tensor &q = *it.q;
  if (q.scalar_type() != at::kBFloat16 || q.dim() != 3 || q.stride(2) != 1) return false;
  for (const at::Tensor *t : {it.kc, it.vc, it.kb, it.vb})
    if (t && (t->scalar_type() != at::kBFloat16 || t->dim() != 3 || t->stride(2) != 1 || t->size(1) != q.size(1) ||
              t->size(2) != q.size(2) || t->device() != q.device()))
      return false;
  if (it.kb->sizes() != it.vb->sizes() || it.kb->strides() != it.vb->strides()) return false;
  return !cached || (it.kc->sizes() == it.vc->sizes() && it.kc->strides() == it.vc->strides() && cache_len <= it.kc->size(0));
}
sdvg_attn_desc attn_desc(const Item &it, const at::Tensor &out, double scale) {
  return sdvg_attn_desc{static_cast<int32_t>(it.q->size(0)), static_cast<int32_t>(it.kb->size(0)),
                        static_cast<int32_t>(it.q->size(1)), static_cast<int32_t>(it.q->size(2)),
                        it.q->stride(0), it.q->stride(1), out.stride(0), out.stride(1),
                        it.kc ? it.kc->stride(0) : 128, it.kc ? it.kc->stride(1) : 128, it.kb->stride(0), it.kb->stride(1),
                        static_cast<float>(scale), SDVG_BF16};
}
bool scale_of(PyObject *o, double &scale) {
  scale = 0.0;
  if (o == Py_None) return true;
  if (!PyFloat_CheckExact(o)) return false;
  scale = PyFloat_AS_DOUBLE(o);
  return true;
}

// (q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale, stream, commit)
PyObject *block_attn_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 10) PYTHON_TAKES_OVER;
  const bool commit = a[9] == Py_True;
  Item it;
  int64_t cache_len;
  double scale;
  if (!integer(a[5], cache_len) || !attn_item(a, cache_len, it) || !scale_of(a[7], scale)) PYTHON_TAKES_OVER;
  if (commit && (!it.kc || cache_len + it.kb->size(0) > it.kc->size(0))) PYTHON_TAKES_OVER;
  void *stream;
  if (!stream_ptr(a[8], stream)) PYTHON_TAKES_OVER;
  const at::Tensor out = output(a[6], *it.q, a[8], stream);
  if (!out.defined()) PYTHON_TAKES_OVER;
  const sdvg_attn_desc d = attn_desc(it, out, scale);
  void *const qp = it.q->data_ptr(), *const kcp = it.kc ? it.kc->data_ptr() : nullptr,
             *const vcp = it.vc ? it.vc->data_ptr() : nullptr, *const kbp = it.kb->data_ptr(),
             *const vbp = it.vb->data_ptr(), *const op = out.data_ptr();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = commit ? api.attn_commit(&d, qp, kcp, vcp, kbp, vbp, cache_len, op, stream)
                  : api.attn(&d, qp, kcp, vcp, kbp, vbp, cache_len, op, stream);
  Py_END_ALLOW_THREADS
  return result(status, a[6], out);
}

// Item i of a list or tuple (borrowed), or null.
PyObject *entry(PyObject *seq, Py_ssize_t i) {
  if (PyList_CheckExact(seq)) return i < PyList_GET_SIZE(seq) ? PyList_GET_ITEM(seq, i) : nullptr;
  return PyTuple_CheckExact(seq) && i < PyTuple_GET_SIZE(seq) ? PyTuple_GET_ITEM(seq, i) : nullptr;
}
bool has_length(PyObject *seq, Py_ssize_t n) {
  return PyList_CheckExact(seq) ? PyList_GET_SIZE(seq) == n : PyTuple_CheckExact(seq) && PyTuple_GET_SIZE(seq) == n;
}

// (qs, k_caches, v_caches, k_blks, v_blks, cache_len, outs, workspace, split, scale, stream, static)
PyObject *batch_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != 12) PYTHON_TAKES_OVER;
  const Py_ssize_t n = PyList_CheckExact(a[0]) ? PyList_GET_SIZE(a[0]) : PyTuple_CheckExact(a[0]) ? PyTuple_GET_SIZE(a[0]) : 0;
  if (n < 1 || n > kMaxItems || !has_length(a[3], n) || !has_length(a[4], n)) PYTHON_TAKES_OVER;
  const bool no_caches = a[1] == Py_None, own_outs = a[6] == Py_None, is_static = a[11] == Py_True;
  if (!no_caches && (!has_length(a[1], n) || !has_length(a[2], n))) PYTHON_TAKES_OVER;
  int64_t cache_len, split;
  double scale;
  if (!integer(a[5], cache_len) || !integer(a[8], split) || !scale_of(a[9], scale)) PYTHON_TAKES_OVER;
  Item items[kMaxItems];
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *const set[5] = {entry(a[0], i), no_caches ? Py_None : entry(a[1], i), no_caches ? Py_None : entry(a[2], i),
                              entry(a[3], i), entry(a[4], i)};
    if (!attn_item(set, cache_len, items[i]) || items[i].q->device() != items[0].q->device()) PYTHON_TAKES_OVER;
  }
  const at::Tensor *ws = a[7] == Py_None ? nullptr : gpu_tensor(a[7]);
  if (a[7] != Py_None && (!ws || !ws->is_contiguous() || ws->device() != items[0].q->device())) PYTHON_TAKES_OVER;
  void *stream;
  if (!stream_ptr(a[10], stream)) PYTHON_TAKES_OVER;
  at::Tensor outs[kMaxItems];
  sdvg_attn_desc d{};
  const void *qp[kMaxItems], *kcp[kMaxItems], *vcp[kMaxItems], *kbp[kMaxItems], *vbp[kMaxItems];
  void *op[kMaxItems];
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *given = own_outs ? Py_None : entry(a[6], i);
    if (!given || (given == Py_None && !own_outs)) PYTHON_TAKES_OVER;
    outs[i] = output(given, *items[i].q, a[10], stream);
    if (!outs[i].defined()) PYTHON_TAKES_OVER;
    const sdvg_attn_desc di = attn_desc(items[i], outs[i], scale);
    if (i == 0)
      d = di;
    else if (memcmp(&di, &d, sizeof d) != 0)
      PYTHON_TAKES_OVER;
    qp[i] = items[i].q->data_ptr();
    kcp[i] = items[i].kc ? items[i].kc->data_ptr() : nullptr;
    vcp[i] = items[i].vc ? items[i].vc->data_ptr() : nullptr;
    kbp[i] = items[i].kb->data_ptr();
    vbp[i] = items[i].vb->data_ptr();
    op[i] = outs[i].data_ptr();
  }
  PyObject *ret = a[6];
  if (own_outs) {
    ret = PyList_New(n);
    if (!ret) return nullptr;
    for (Py_ssize_t i = 0; i < n; ++i) PyList_SET_ITEM(ret, i, THPVariable_Wrap(outs[i]));
  } else {
    Py_INCREF(ret);
  }
  void *const wp = ws ? ws->data_ptr() : nullptr;
  const int64_t w_bytes = ws ? static_cast<int64_t>(ws->nbytes()) : 0;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = is_static ? api.batch_static(&d, static_cast<int32_t>(n), qp, kcp, vcp, kbp, vbp, cache_len, op,
                                        static_cast<int32_t>(split), stream)
                     : api.batch(&d, static_cast<int32_t>(n), qp, kcp, vcp, kbp, vbp, cache_len, op, wp, w_bytes,
                                 static_cast<int32_t>(split), stream);
  Py_END_ALLOW_THREADS
  if (status == 0) return ret;
  Py_DECREF(ret);
  return PyLong_FromLong(status);
}

// The descriptor S inside a ctypes structure of binding.py (of class `type`), for as long as this lives.
template <typename S>
struct DescRef {
  Py_buffer view{};
  S *c = nullptr;
  DescRef(PyObject *o, PyObject *type) {
    if (reinterpret_cast<PyObject *>(Py_TYPE(o)) != type) return;
    if (PyObject_GetBuffer(o, &view, PyBUF_WRITABLE) != 0) {
      PyErr_Clear();
      return;
    }
    if (view.len == static_cast<Py_ssize_t>(sizeof(S))) c = static_cast<S *>(view.buf);
  }
  ~DescRef() {
    if (view.obj) PyBuffer_Release(&view);
  }
  DescRef(const DescRef &) = delete;
  DescRef &operator=(const DescRef &) = delete;
};

// A dense bf16 [layers][T][heads][dim] block of the cache's shape.
const at::Tensor *block_tensor(PyObject *o, const sdvg_kv_cache &c) {
  const at::Tensor *t = gpu_tensor(o);
  if (!t || t->scalar_type() != at::kBFloat16 || t->dim() != 4 || !t->is_contiguous() || t->size(0) != c.n_layers ||
      t->size(1) != c.block_tokens || t->size(2) != c.n_heads || t->size(3) != c.head_dim)
    return nullptr;
  return t;
}

// (cache.c, k_blk, v_blk, slot, stream), and cos, sin with the rotation of K
PyObject *commit_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 5 && n != 7) PYTHON_TAKES_OVER;
  const DescRef<sdvg_kv_cache> cache(a[0], api.cache_type);
  int64_t slot;
  if (!cache.c || !integer(a[3], slot) || slot != static_cast<int32_t>(slot)) PYTHON_TAKES_OVER;
  const at::Tensor *kb = block_tensor(a[1], *cache.c), *vb = block_tensor(a[2], *cache.c);
  if (!kb || !vb) PYTHON_TAKES_OVER;
  const float *tables[2] = {nullptr, nullptr};
  for (int i = 0; n == 7 && i < 2; ++i) {
    const at::Tensor *t = gpu_tensor(a[5 + i]);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != cache.c->block_tokens || t->size(1) != 64 ||
        !t->is_contiguous() || t->device() != kb->device())
      PYTHON_TAKES_OVER;
    tables[i] = static_cast<const float *>(t->data_ptr());
  }
  void *stream;
  if (!stream_ptr(a[4], stream)) PYTHON_TAKES_OVER;
  const void *const kp = kb->data_ptr(), *const vp = vb->data_ptr();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = n == 5 ? api.commit(cache.c, kp, vp, static_cast<int32_t>(slot), stream)
                  : api.commit_rope(cache.c, kp, vp, static_cast<int32_t>(slot), tables[0], tables[1], stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (cache.c, new_len, stream)
PyObject *rollback_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 3) PYTHON_TAKES_OVER;
  const DescRef<sdvg_kv_cache> cache(a[0], api.cache_type);
  int64_t new_len;
  void *stream;
  if (!cache.c || !integer(a[1], new_len) || !stream_ptr(a[2], stream)) PYTHON_TAKES_OVER;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.rollback(cache.c, new_len, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (dst, src, n_bytes, stream)
PyObject *snapshot_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 4) PYTHON_TAKES_OVER;
  const at::Tensor *dst = gpu_tensor(a[0]), *src = gpu_tensor(a[1]);
  if (!dst || !src || !dst->is_contiguous() || !src->is_contiguous()) PYTHON_TAKES_OVER;
  const int64_t dst_bytes = static_cast<int64_t>(dst->nbytes()), src_bytes = static_cast<int64_t>(src->nbytes());
  int64_t n_bytes = src_bytes;
  if (a[2] != Py_None && !integer(a[2], n_bytes)) PYTHON_TAKES_OVER;
  void *stream;
  if (n_bytes > dst_bytes || n_bytes > src_bytes || !stream_ptr(a[3], stream)) PYTHON_TAKES_OVER;
  void *const dp = dst->data_ptr(), *const sp = src->data_ptr();
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.snapshot(dp, sp, n_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (x, cos, sin, out, stream)
PyObject *rope_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 5) PYTHON_TAKES_OVER;
  const at::Tensor *x = gpu_tensor(a[0]), *cos = gpu_tensor(a[1]), *sin = gpu_tensor(a[2]);
  if (!x || !cos || !sin) PYTHON_TAKES_OVER;
  if (x->scalar_type() != at::kBFloat16 || x->dim() != 3 || x->size(2) != 128 || x->stride(2) != 1) PYTHON_TAKES_OVER;
  for (const at::Tensor *t : {cos, sin})
    if (t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != x->size(0) || t->size(1) != 64 ||
        !t->is_contiguous() || t->device() != x->device())
      PYTHON_TAKES_OVER;
  void *stream;
  if (!stream_ptr(a[4], stream)) PYTHON_TAKES_OVER;
  const at::Tensor out = output(a[3], *x, a[4], stream);
  if (!out.defined()) PYTHON_TAKES_OVER;
  void *const xp = x->data_ptr(), *const op = out.data_ptr();
  const float *const cp = static_cast<const float *>(cos->data_ptr()), *const sp = static_cast<const float *>(sin->data_ptr());
  const int64_t n_tokens = x->size(0), xs0 = x->stride(0), xs1 = x->stride(1), os0 = out.stride(0), os1 = out.stride(1);
  const int32_t heads = static_cast<int32_t>(x->size(1));
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.rope(xp, cp, sp, op, n_tokens, heads, 128, xs0, xs1, os0, os1, stream);
  Py_END_ALLOW_THREADS
  return result(status, a[3], out);
}

// (frame_scores, tau, block_idx, mean, stream) -> (decision, numpy float32), a negative status, or None
PyObject *route_impl(PyObject *const *a, Py_ssize_t n) {
  if (n != 5) PYTHON_TAKES_OVER;
  const at::Tensor *s = gpu_tensor(a[0]);
  int64_t block_idx;
  if (!s || s->scalar_type() != at::kFloat || s->dim() != 1 || !s->is_contiguous()) PYTHON_TAKES_OVER;
  if (!PyFloat_CheckExact(a[1]) || !integer(a[2], block_idx) || block_idx != static_cast<int32_t>(block_idx) ||
      s->size(0) > INT32_MAX)
    PYTHON_TAKES_OVER;
  void *stream;
  if (!stream_ptr(a[4], stream)) PYTHON_TAKES_OVER;
  const float *const sp = static_cast<const float *>(s->data_ptr());
  const int32_t frames = static_cast<int32_t>(s->size(0));
  const float tau = static_cast<float>(PyFloat_AS_DOUBLE(a[1]));
  const route_fn fn = a[3] == Py_True ? api.route_mean : api.route_min;
  float q_b = 0.f;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = fn(sp, frames, tau, static_cast<int32_t>(block_idx), &q_b, stream);
  Py_END_ALLOW_THREADS
  if (status < 0) return PyLong_FromLong(status);
  PyObject *value = PyFloat_FromDouble(static_cast<double>(q_b));
  PyObject *scalar = value ? PyObject_CallOneArg(api.float32, value) : nullptr;
  Py_XDECREF(value);
  return scalar ? Py_BuildValue("(iN)", status, scalar) : nullptr;
}

// ---- paged cache

// The current device, which all tensors of a call have to be on, and the stream to launch on.
bool launch_place(PyObject *stream, int64_t &device, void *&s) {
  PyObject *dev = PyObject_CallNoArgs(api.get_device);
  bool ok = dev && integer(dev, device);
  if (ok && stream == Py_None) {
    PyObject *raw = PyObject_CallOneArg(api.get_raw_stream, dev);
    int64_t v = 0;
    ok = raw && integer(raw, v);
    Py_XDECREF(raw);
    s = reinterpret_cast<void *>(v);
  } else if (ok) {
    ok = stream_ptr(stream, s);
  }
  Py_XDECREF(dev);
  if (!ok) PyErr_Clear();
  return ok;
}

// A dense tensor of n elements of one type, in one dimension.
const at::Tensor *array(PyObject *o, at::ScalarType type, int64_t n, int64_t device) {
  const at::Tensor *t = gpu_tensor(o);
  return t && t->scalar_type() == type && t->dim() == 1 && t->size(0) == n && t->is_contiguous() && t->get_device() == device ? t : nullptr;
}
bool optional_array(PyObject *o, int64_t n, int64_t device, const int32_t *&p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor *t = array(o, at::kInt, n, device);
  if (t) p = static_cast<const int32_t *>(t->data_ptr());
  return t;
}
const at::Tensor *table_tensor(PyObject *o, int64_t device) {
  const at::Tensor *t = gpu_tensor(o);
  return t && t->scalar_type() == at::kInt && t->dim() == 2 && (t->size(1) <= 1 || t->stride(1) == 1) && t->get_device() == device &&
                 t->size(0) <= INT32_MAX && t->size(1) <= INT32_MAX
             ? t
             : nullptr;
}
// Rows [tokens][heads][128]; their type as sdvg.h has it, or -1.
const at::Tensor *rows_tensor(PyObject *o, int64_t device) {
  const at::Tensor *t = gpu_tensor(o);
  return t && t->dim() == 3 && t->size(2) == 128 && t->stride(2) == 1 && t->get_device() == device && t->size(0) <= INT32_MAX &&
                 t->size(1) <= INT32_MAX
             ? t
             : nullptr;
}
int type_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return SDVG_BF16;
    case at::kFloat: return SDVG_F32;
    case at::kHalf: return SDVG_F16;
    default: return -1;
  }
}
sdvg_rows rows_of(const at::Tensor &in, const at::Tensor *out) {
  return sdvg_rows{in.data_ptr(), out ? out->data_ptr() : nullptr, static_cast<int32_t>(in.size(1)), in.stride(0), in.stride(1),
                   out ? out->stride(0) : 0, out ? out->stride(1) : 0};
}
bool rope_of(PyObject *positions, PyObject *freqs, PyObject *layout, PyObject *gain, int64_t n_tokens, int64_t device,
             sdvg_rope_desc &d) {
  const at::Tensor *p = array(positions, at::kInt, n_tokens, device), *f = gpu_tensor(freqs);
  int64_t how;
  if (!p || !f || f->scalar_type() != at::kDouble || f->dim() != 1 || !f->is_contiguous() || f->get_device() != device ||
      f->size(0) > 64 || !integer(layout, how) || !PyFloat_CheckExact(gain))
    return false;
  d = sdvg_rope_desc{static_cast<const int32_t *>(p->data_ptr()), static_cast<const double *>(f->data_ptr()),
                     static_cast<int32_t>(2 * f->size(0)), static_cast<int32_t>(how), static_cast<float>(PyFloat_AS_DOUBLE(gain))};
  return true;
}

// (cached, new_tokens, block_table, page_tokens, free_pages, held, next_free, q_start, kv_lens, positions, held_out,
// next_free_out, slots, stream) -> 0, a negative status, or None
PyObject *page_plan_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != 14) PYTHON_TAKES_OVER;
  int64_t device, page;
  void *stream;
  if (!launch_place(a[13], device, stream) || !integer(a[3], page) || page != static_cast<int32_t>(page)) PYTHON_TAKES_OVER;
  const at::Tensor *table = table_tensor(a[2], device), *slots = gpu_tensor(a[12]);
  if (!table || !slots || slots->dim() != 1) PYTHON_TAKES_OVER;
  const int64_t n = table->size(0), m = slots->size(0);
  if (n < 1 || m < 1) PYTHON_TAKES_OVER;  // (empty tensors have no address)
  const at::Tensor *const cached = array(a[0], at::kInt, n, device), *const fresh = array(a[1], at::kInt, n, device),
                   *const starts = array(a[7], at::kInt, n + 1, device), *const lens = array(a[8], at::kInt, n, device),
                   *const positions = array(a[9], at::kInt, m, device), *const held_out = array(a[10], at::kInt, n, device),
                   *const next_out = array(a[11], at::kInt, 1, device);
  if (!cached || !fresh || !starts || !lens || !positions || !held_out || !next_out || !array(a[12], at::kLong, m, device)) PYTHON_TAKES_OVER;
  const at::Tensor *const free = a[4] == Py_None ? nullptr : gpu_tensor(a[4]);
  if (a[4] != Py_None && (!free || free->dim() != 1 || free->size(0) > INT32_MAX || !array(a[4], at::kInt, free->size(0), device)))
    PYTHON_TAKES_OVER;
  const int32_t *held, *next;
  if (!optional_array(a[5], n, device, held) || !optional_array(a[6], 1, device, next) || (!held && (free || next))) PYTHON_TAKES_OVER;
  const auto ints = [](const at::Tensor *t) { return static_cast<int32_t *>(t->data_ptr()); };
  const sdvg_page_plan_args args{static_cast<int32_t>(n), static_cast<int32_t>(page), static_cast<int32_t>(table->size(1)),
                                 free ? static_cast<int32_t>(free->size(0)) : 0, n > 1 ? table->stride(0) : table->size(1), m,
                                 ints(cached), ints(fresh), free && free->size(0) > 0 ? ints(free) : nullptr, held, next, ints(table),
                                 ints(starts), ints(lens), ints(positions), ints(held_out), ints(next_out),
                                 static_cast<int64_t *>(slots->data_ptr())};
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.page_plan(&args, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// (x, positions, freqs, y, layout, gain, out, y_out, stream) -> out or (out, y_out), a negative status, or None
PyObject *rope_positions_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != 9) PYTHON_TAKES_OVER;
  int64_t device;
  void *stream;
  if (!launch_place(a[8], device, stream)) PYTHON_TAKES_OVER;
  const bool two = a[3] != Py_None;
  const at::Tensor *x = rows_tensor(a[0], device), *y = two ? rows_tensor(a[3], device) : nullptr;
  if (!x || type_of(*x) < 0 || x->size(0) < 1) PYTHON_TAKES_OVER;
  if (two ? (!y || y->scalar_type() != x->scalar_type() || y->size(0) != x->size(0)) : a[7] != Py_None) PYTHON_TAKES_OVER;
  sdvg_rope_desc rope;
  if (!rope_of(a[1], a[2], a[4], a[5], x->size(0), device, rope)) PYTHON_TAKES_OVER;
  const at::Tensor out = output(a[6], *x, a[8], stream), y_out = two ? output(a[7], *y, a[8], stream) : at::Tensor();
  if (!out.defined() || (two && !y_out.defined())) PYTHON_TAKES_OVER;
  const sdvg_rows rx = rows_of(*x, &out), ry = two ? rows_of(*y, &y_out) : sdvg_rows{};
  const int64_t n = x->size(0);
  const int32_t type = type_of(*x);
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.rope_positions(&rope, &rx, two ? &ry : nullptr, n, 128, type, stream);
  Py_END_ALLOW_THREADS
  PyObject *first = result(status, a[6], out);
  if (status != 0 || !two || !first) return first;
  PyObject *second = result(status, a[7], y_out);
  return Py_BuildValue("(NN)", first, second);
}

// (cache.c, cache.k, k, v, slots, positions, freqs, q, q_out, layout, gain, stream) -> q_out, 0 without q, a negative status, or None
PyObject *paged_commit_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != 12) PYTHON_TAKES_OVER;
  int64_t device;
  void *stream;
  if (!launch_place(a[11], device, stream)) PYTHON_TAKES_OVER;
  const DescRef<const sdvg_paged_kv> cache(a[0], api.paged_type);
  const at::Tensor *pool = gpu_tensor(a[1]), *k = rows_tensor(a[2], device), *v = rows_tensor(a[3], device);
  if (!cache.c || !pool || pool->get_device() != device || !k || !v || k->size(0) < 1 || k->sizes() != v->sizes() ||
      k->scalar_type() != v->scalar_type() || k->size(1) != cache.c->n_kv_heads)
    PYTHON_TAKES_OVER;
  const int type = type_of(*k);
  if ((type != SDVG_BF16 && type != SDVG_F16) || (cache.c->dtype != type && cache.c->dtype != SDVG_E4M3)) PYTHON_TAKES_OVER;
  const int64_t n = k->size(0);
  const at::Tensor *slots = array(a[4], at::kLong, n, device);
  if (!slots) PYTHON_TAKES_OVER;
  const bool turn = a[5] != Py_None, with_q = a[7] != Py_None;
  sdvg_rope_desc rope;
  if (turn != (a[6] != Py_None) || (with_q && !turn) || (!with_q && a[8] != Py_None)) PYTHON_TAKES_OVER;
  if (turn && !rope_of(a[5], a[6], a[9], a[10], n, device, rope)) PYTHON_TAKES_OVER;
  const at::Tensor *q = with_q ? rows_tensor(a[7], device) : nullptr;
  if (with_q && (!q || q->size(0) != n || q->scalar_type() != k->scalar_type())) PYTHON_TAKES_OVER;
  const at::Tensor q_out = with_q ? output(a[8], *q, a[11], stream) : at::Tensor();
  if (with_q && !q_out.defined()) PYTHON_TAKES_OVER;
  const sdvg_rows rk = rows_of(*k, nullptr), rv = rows_of(*v, nullptr), rq = with_q ? rows_of(*q, &q_out) : sdvg_rows{};
  const int64_t *const sp = static_cast<const int64_t *>(slots->data_ptr());
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.paged_commit(cache.c, &rk, &rv, sp, n, type, turn ? &rope : nullptr, with_q ? &rq : nullptr, stream);
  Py_END_ALLOW_THREADS
  return with_q ? result(status, a[8], q_out) : PyLong_FromLong(status);
}

// (q, cache.c, cache.k, block_table, q_start, kv_lens, out, lse, scale, window, workspace, stream)
// (kPrefix: of groups that share their first keys; two arguments more, prefix_lens and group_start)
template <bool kPrefix>
PyObject *paged_attn_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != (kPrefix ? 14 : 12)) PYTHON_TAKES_OVER;
  int64_t device, window;
  void *stream;
  double scale;
  if (!launch_place(a[11], device, stream) || !integer(a[9], window) || window != static_cast<int32_t>(window) || !scale_of(a[8], scale))
    PYTHON_TAKES_OVER;
  const DescRef<const sdvg_paged_kv> cache(a[1], api.paged_type);
  const at::Tensor *pool = gpu_tensor(a[2]), *q = rows_tensor(a[0], device), *table = table_tensor(a[3], device);
  if (!cache.c || !pool || pool->get_device() != device || !q || !table || q->size(0) < 1 || table->size(0) < 1) PYTHON_TAKES_OVER;
  const int type = type_of(*q);
  if ((type != SDVG_BF16 && type != SDVG_F16) || (cache.c->dtype != type && cache.c->dtype != SDVG_E4M3)) PYTHON_TAKES_OVER;
  const int64_t n = table->size(0);
  const at::Tensor *starts = array(a[4], at::kInt, n + 1, device), *lens = array(a[5], at::kInt, n, device);
  if (!starts || !lens) PYTHON_TAKES_OVER;
  const at::Tensor *lse = a[7] == Py_None ? nullptr : gpu_tensor(a[7]), *ws = a[10] == Py_None ? nullptr : gpu_tensor(a[10]);
  if (a[7] != Py_None && (!lse || lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != q->size(0) ||
                          lse->size(1) != q->size(1) || !lse->is_contiguous() || lse->get_device() != device))
    PYTHON_TAKES_OVER;
  if (a[10] != Py_None && (!ws || !ws->is_contiguous() || ws->get_device() != device)) PYTHON_TAKES_OVER;
  const int32_t *group_p = nullptr, *prefix_p = nullptr;
  int64_t n_groups = 0;
  if constexpr (kPrefix) {
    const at::Tensor *lens_t = gpu_tensor(a[12]);
    if (!lens_t || lens_t->dim() != 1) PYTHON_TAKES_OVER;
    n_groups = lens_t->size(0);
    const at::Tensor *prefix = array(a[12], at::kInt, n_groups, device), *starts_t = a[13] == Py_None ? nullptr : array(a[13], at::kInt, n_groups + 1, device);
    if (!prefix || n_groups > INT32_MAX - 1 || (!starts_t && (a[13] != Py_None || n_groups > 1))) PYTHON_TAKES_OVER;
    prefix_p = static_cast<const int32_t *>(prefix->data_ptr());
    if (starts_t) group_p = static_cast<const int32_t *>(starts_t->data_ptr());
  }
  const at::Tensor out = output(a[6], *q, a[11], stream);
  if (!out.defined()) PYTHON_TAKES_OVER;
  const sdvg_paged_attn_desc d{static_cast<int32_t>(n), static_cast<int32_t>(q->size(0)), static_cast<int32_t>(q->size(1)), 128,
                               static_cast<int32_t>(table->size(1)), static_cast<int32_t>(window), table->stride(0), q->stride(0),
                               q->stride(1), out.stride(0), out.stride(1), static_cast<float>(scale), type};
  const auto ints = [](const at::Tensor *t) { return static_cast<const int32_t *>(t->data_ptr()); };
  const void *const qp = q->data_ptr();
  const int32_t *const tp = ints(table), *const sp = ints(starts), *const lp = ints(lens);
  void *const op = out.data_ptr(), *const wp = ws ? ws->data_ptr() : nullptr;
  float *const ep = lse ? static_cast<float *>(lse->data_ptr()) : nullptr;
  const int64_t w_bytes = ws ? static_cast<int64_t>(ws->nbytes()) : 0;
  int status;
  Py_BEGIN_ALLOW_THREADS
  if constexpr (kPrefix)
    status = api.paged_prefix_attn(&d, cache.c, qp, tp, sp, lp, static_cast<int32_t>(n_groups), group_p, prefix_p, op, ep, wp, w_bytes, stream);
  else
    status = api.paged_attn(&d, cache.c, qp, tp, sp, lp, op, ep, wp, w_bytes, stream);
  Py_END_ALLOW_THREADS
  return result(status, a[6], out);
}

// A setting of sample_tokens: an array [n] or a number for all rows (None: `all` stays as it is).
bool setting(PyObject *o, int64_t n, int64_t device, const float *&p, float &all) {
  if (o == Py_None) return true;
  if (PyFloat_CheckExact(o)) {
    all = static_cast<float>(PyFloat_AS_DOUBLE(o));
    return true;
  }
  const at::Tensor *t = array(o, at::kFloat, n, device);
  if (t) p = static_cast<const float *>(t->data_ptr());
  return t;
}
bool setting(PyObject *o, int64_t n, int64_t device, const int32_t *&p, int32_t &all) {
  if (o == Py_None) return true;
  int64_t v;
  if (PyLong_CheckExact(o)) {
    if (!integer(o, v) || v != static_cast<int32_t>(v)) return false;
    all = static_cast<int32_t>(v);
    return true;
  }
  return optional_array(o, n, device, p);
}

// (logits, u, temperature, top_k, top_p, min_p, out, logprob, workspace, stream) -> out, a negative status, or None
PyObject *sample_tokens_impl(PyObject *const *a, Py_ssize_t n_args) {
  if (n_args != 10) PYTHON_TAKES_OVER;
  int64_t device;
  void *stream;
  if (!launch_place(a[9], device, stream)) PYTHON_TAKES_OVER;
  const at::Tensor *x = gpu_tensor(a[0]), *ws = gpu_tensor(a[8]);
  if (!x || x->dim() != 2 || x->get_device() != device || type_of(*x) < 0 || x->size(0) < 1 || x->size(0) > INT32_MAX || x->size(1) < 1 ||
      x->size(1) > INT32_MAX || (x->size(1) > 1 && x->stride(1) != 1) || !ws || !ws->is_contiguous() || ws->get_device() != device)
    PYTHON_TAKES_OVER;
  const int64_t n = x->size(0);
  sdvg_sample_args s{};
  s.all_temperature = s.all_top_p = 1.0f;
  const at::Tensor *u = array(a[1], at::kFloat, n, device);
  if (!u || !setting(a[2], n, device, s.temperature, s.all_temperature) || !setting(a[3], n, device, s.top_k, s.all_top_k) ||
      !setting(a[4], n, device, s.top_p, s.all_top_p) || !setting(a[5], n, device, s.min_p, s.all_min_p))
    PYTHON_TAKES_OVER;
  const at::Tensor *lp = a[7] == Py_None ? nullptr : array(a[7], at::kFloat, n, device);
  if (a[7] != Py_None && !lp) PYTHON_TAKES_OVER;
  at::Tensor out;
  if (a[6] == Py_None) {
    const StreamGuard guard(a[9], x->device(), stream);
    out = at::empty({n}, at::TensorOptions().dtype(at::kInt).device(x->device()));
    if (out.unsafeGetTensorImpl()->is_python_dispatch()) PYTHON_TAKES_OVER;
  } else {
    const at::Tensor *t = array(a[6], at::kInt, n, device);
    if (!t) PYTHON_TAKES_OVER;
    out = *t;
  }
  s.logits = x->data_ptr();
  s.u = static_cast<const float *>(u->data_ptr());
  s.tokens = static_cast<int32_t *>(out.data_ptr());
  s.logprob = lp ? static_cast<float *>(lp->data_ptr()) : nullptr;
  s.row_stride = x->stride(0);
  s.n_rows = static_cast<int32_t>(n);
  s.vocab = static_cast<int32_t>(x->size(1));
  s.dtype = type_of(*x);
  void *const wp = ws->data_ptr();
  const int64_t w_bytes = static_cast<int64_t>(ws->nbytes());
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = api.sample_tokens(&s, wp, w_bytes, stream);
  Py_END_ALLOW_THREADS
  return result(status, a[6], out);
}

// Anything torch throws (a tensor without storage, ...) happens before the launch: Python repeats
// the call and reports it its own way.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n) {
  try {
    return F(args, n);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (addresses of attn, attn_commit, rope, route_min, route_mean, batch, batch_static, commit, commit_rope, rollback,
// snapshot, page_plan, rope_positions, paged_commit, paged_attn, paged_prefix_attn, sample_tokens; torch._C._cuda_getDevice,
// torch._C._cuda_getCurrentRawStream, numpy.float32, the ctypes classes of the cache and of the paged cache)
PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n) {
  constexpr int kEntries = 17;
  int64_t p[kEntries];
  if (n != kEntries + 5) {
    PyErr_SetString(PyExc_TypeError, "init takes 22 arguments");
    return nullptr;
  }
  for (int i = 0; i < kEntries; ++i)
    if (!integer(a[i], p[i]) || !p[i]) {
      PyErr_SetString(PyExc_TypeError, "init: not an address");
      return nullptr;
    }
  for (int i = kEntries; i < n; ++i) Py_INCREF(a[i]);
  api = Api{reinterpret_cast<attn_fn>(p[0]),    reinterpret_cast<attn_commit_fn>(p[1]),  reinterpret_cast<rope_fn>(p[2]),
            reinterpret_cast<route_fn>(p[3]),   reinterpret_cast<route_fn>(p[4]),        reinterpret_cast<batch_fn>(p[5]),
            reinterpret_cast<batch_static_fn>(p[6]), reinterpret_cast<commit_fn>(p[7]),  reinterpret_cast<commit_rope_fn>(p[8]),
            reinterpret_cast<rollback_fn>(p[9]), reinterpret_cast<snapshot_fn>(p[10]),   reinterpret_cast<page_plan_fn>(p[11]),
            reinterpret_cast<rope_positions_fn>(p[12]), reinterpret_cast<paged_commit_fn>(p[13]),
            reinterpret_cast<paged_attn_fn>(p[14]), reinterpret_cast<paged_prefix_attn_fn>(p[15]),
            reinterpret_cast<sample_tokens_fn>(p[16]), a[17], a[18], a[19], a[20], a[21]};
  Py_RETURN_NONE;
}

#define METHOD(name, fn) \
  { name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr }
PyMethodDef methods[] = {METHOD("init", init), METHOD("block_attn", guarded<block_attn_impl>),
                         METHOD("rope", guarded<rope_impl>), METHOD("route", guarded<route_impl>),
                         METHOD("batch", guarded<batch_impl>), METHOD("commit", guarded<commit_impl>),
                         METHOD("rollback", guarded<rollback_impl>), METHOD("snapshot", guarded<snapshot_impl>),
                         METHOD("page_plan", guarded<page_plan_impl>), METHOD("rope_positions", guarded<rope_positions_impl>),
                         METHOD("paged_commit", guarded<paged_commit_impl>), METHOD("paged_attn", guarded<paged_attn_impl<false>>),
                         METHOD("paged_prefix_attn", guarded<paged_attn_impl<true>>), METHOD("sample_tokens", guarded<sample_tokens_impl>),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of libsdvg's most frequent calls.",
                          -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__native() { return PyModule_Create(&module_def); }
