"""ctypes binding of libsdvg.so. Argument marshalling only: same names as the C entry points.

PyTorch tensors supply device memory (`data_ptr()`) and the HIP stream; nothing is computed
here and there is no fallback: a missing library raises. The most frequent calls are marshalled by
the extension module _native.so (csrc/host/native.cpp), which makes the same checks in C++ and
leaves every call it does not recognise as valid to the Python code here, which also works alone.

A result that a call with stream= makes for itself belongs to that stream, its memory too: another stream waits for
that one before it reads the result, and names itself with record_stream if it still reads when the result is dropped.
"""
import contextlib
import ctypes
import importlib.util
import math
import os
import warnings

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# SDVG_LIBRARY names another build of the same library (e.g. one with host sanitizers); there is
# still no fallback: whatever path is named must exist.
LIB_PATH = os.environ.get("SDVG_LIBRARY") or os.path.join(HERE, "libsdvg.so")

NATIVE_PATH = os.path.join(HERE, "_native.so")

SDVG_BF16, SDVG_F32, SDVG_F16, SDVG_E4M3 = 0, 1, 2, 3
SDVG_SPLIT_NEVER, SDVG_SPLIT_AUTO, SDVG_SPLIT_ALWAYS = 0, 1, 2
SDVG_ROPE_INTERLEAVED, SDVG_ROPE_HALF = 0, 1
_LAYOUT = {"interleaved": 0, "half": 1}
_SPLIT = {"never": 0, "auto": 1, "always": 2}


class SdvgError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__("%s failed: %s" % (where, status_string(status)))


class sdvg_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("n_layers", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("capacity_tokens", ctypes.c_int64), ("cache_len", ctypes.c_int64),
                ("layer_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class sdvg_attn_desc(ctypes.Structure):
    _fields_ = [("n_q", ctypes.c_int32), ("n_blk", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("o_token_stride", ctypes.c_int64), ("o_head_stride", ctypes.c_int64),
                ("kv_token_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64),
                ("blk_token_stride", ctypes.c_int64), ("blk_head_stride", ctypes.c_int64),
                ("scale", ctypes.c_float), ("dtype", ctypes.c_int32)]


class sdvg_paged_kv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class sdvg_rope_desc(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("gain", ctypes.c_float)]


class sdvg_rows(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n_heads", ctypes.c_int32),
                ("in_token_stride", ctypes.c_int64), ("in_head_stride", ctypes.c_int64),
                ("out_token_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64)]


class sdvg_paged_attn_desc(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("table_width", ctypes.c_int32), ("window", ctypes.c_int32),
                ("table_stride", ctypes.c_int64), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("o_token_stride", ctypes.c_int64), ("o_head_stride", ctypes.c_int64), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int32)]


class sdvg_page_plan_args(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("table_width", ctypes.c_int32),
                ("n_free", ctypes.c_int32), ("table_stride", ctypes.c_int64), ("max_tokens", ctypes.c_int64),
                ("cached", ctypes.c_void_p), ("new_tokens", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
                ("held", ctypes.c_void_p), ("next_free", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("q_start", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("held_out", ctypes.c_void_p), ("next_free_out", ctypes.c_void_p), ("slots", ctypes.c_void_p)]


class sdvg_sample_args(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("u", ctypes.c_void_p), ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("all_temperature", ctypes.c_float),
                ("all_top_k", ctypes.c_int32), ("all_top_p", ctypes.c_float), ("all_min_p", ctypes.c_float),
                ("tokens", ctypes.c_void_p), ("logprob", ctypes.c_void_p), ("row_stride", ctypes.c_int64),
                ("n_rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32)]


_LIB = None


def lib():
    """The loaded libsdvg.so; raises if it was never built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libsdvg.so is missing: build it with `python -m paper_2604_17397_amd.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        L.sdvg_block_attn.restype = ctypes.c_int
        L.sdvg_block_attn.argtypes = [ctypes.POINTER(sdvg_attn_desc), vp, vp, vp, vp, vp, i64, vp, vp]
        L.sdvg_block_attn_commit.restype = ctypes.c_int
        L.sdvg_block_attn_commit.argtypes = [ctypes.POINTER(sdvg_attn_desc), vp, vp, vp, vp, vp, i64, vp, vp]
        L.sdvg_kv_commit_mark.restype = ctypes.c_int
        L.sdvg_kv_commit_mark.argtypes = [ctypes.POINTER(sdvg_kv_cache), i32]
        pp = ctypes.POINTER(ctypes.c_void_p)
        L.sdvg_block_attn_batch.restype = ctypes.c_int
        L.sdvg_block_attn_batch.argtypes = [ctypes.POINTER(sdvg_attn_desc), i32, pp, pp, pp, pp, pp, i64, pp,
                                            vp, i64, i32, vp]
        L.sdvg_block_attn_batch_static.restype = ctypes.c_int
        L.sdvg_block_attn_batch_static.argtypes = [ctypes.POINTER(sdvg_attn_desc), i32, pp, pp, pp, pp, pp, i64, pp,
                                                   i32, vp]
        L.sdvg_block_attn_static_workspace_limit.restype = ctypes.c_int64
        L.sdvg_block_attn_workspace_bytes.restype = ctypes.c_int64
        L.sdvg_block_attn_workspace_bytes.argtypes = [ctypes.POINTER(sdvg_attn_desc), i32, i64, i32]
        L.sdvg_kv_commit.restype = ctypes.c_int
        L.sdvg_kv_commit.argtypes = [ctypes.POINTER(sdvg_kv_cache), vp, vp, i32, vp]
        L.sdvg_rope.restype = ctypes.c_int
        L.sdvg_rope.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, i64, i64, i64, vp]
        L.sdvg_kv_commit_rope.restype = ctypes.c_int
        L.sdvg_kv_commit_rope.argtypes = [ctypes.POINTER(sdvg_kv_cache), vp, vp, i32, vp, vp, vp]
        L.sdvg_kv_rollback.restype = ctypes.c_int
        L.sdvg_kv_rollback.argtypes = [ctypes.POINTER(sdvg_kv_cache), i64, vp]
        L.sdvg_worst_frame_route.restype = ctypes.c_int
        L.sdvg_worst_frame_route.argtypes = [vp, i32, f32, i32, ctypes.POINTER(f32), vp]
        L.sdvg_worst_frame_route_batch.restype = ctypes.c_int
        L.sdvg_worst_frame_route_batch.argtypes = [vp, i32, i32, f32, vp, i32, vp, vp, vp]
        L.sdvg_buffer_snapshot.restype = ctypes.c_int
        L.sdvg_buffer_snapshot.argtypes = [vp, vp, i64, vp]
        L.sdvg_avg_frame_route.restype = ctypes.c_int
        L.sdvg_avg_frame_route.argtypes = [vp, i32, f32, i32, ctypes.POINTER(f32), vp]
        L.sdvg_avg_frame_route_batch.restype = ctypes.c_int
        L.sdvg_avg_frame_route_batch.argtypes = [vp, i32, i32, f32, vp, i32, vp, vp, vp]
        L.sdvg_page_plan.restype = ctypes.c_int
        L.sdvg_page_plan.argtypes = [ctypes.POINTER(sdvg_page_plan_args), vp]
        rd, rows = ctypes.POINTER(sdvg_rope_desc), ctypes.POINTER(sdvg_rows)
        L.sdvg_rope_positions.restype = ctypes.c_int
        L.sdvg_rope_positions.argtypes = [rd, rows, rows, i64, i32, i32, vp]
        L.sdvg_paged_commit.restype = ctypes.c_int
        L.sdvg_paged_commit.argtypes = [ctypes.POINTER(sdvg_paged_kv), rows, rows, vp, i64, i32, rd, rows, vp]
        pa, pc = ctypes.POINTER(sdvg_paged_attn_desc), ctypes.POINTER(sdvg_paged_kv)
        L.sdvg_paged_attn.restype = ctypes.c_int
        L.sdvg_paged_attn.argtypes = [pa, pc, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.sdvg_paged_attn_workspace_bytes.restype = ctypes.c_int64
        L.sdvg_paged_attn_workspace_bytes.argtypes = [pa, pc]
        L.sdvg_paged_prefix_attn.restype = ctypes.c_int
        L.sdvg_paged_prefix_attn.argtypes = [pa, pc, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, i64, vp]
        L.sdvg_paged_prefix_attn_workspace_bytes.restype = ctypes.c_int64
        L.sdvg_paged_prefix_attn_workspace_bytes.argtypes = [pa, pc, i32]
        L.sdvg_sample_tokens.restype = ctypes.c_int
        L.sdvg_sample_tokens.argtypes = [ctypes.POINTER(sdvg_sample_args), vp, i64, vp]
        L.sdvg_sample_tokens_workspace_bytes.restype = ctypes.c_int64
        L.sdvg_sample_tokens_workspace_bytes.argtypes = [i32, i32]
        L.sdvg_probe_mfma.restype = ctypes.c_int
        L.sdvg_probe_mfma.argtypes = [vp, i64, vp, i32, ctypes.POINTER(ctypes.c_double), vp]
        L.sdvg_probe_mfma_changing.restype = ctypes.c_int
        L.sdvg_probe_mfma_changing.argtypes = [vp, i64, vp, i32, ctypes.POINTER(ctypes.c_double), vp]
        L.sdvg_status_string.restype = ctypes.c_char_p
        L.sdvg_status_string.argtypes = [ctypes.c_int]
        L.sdvg_last_device_error.restype = ctypes.c_int
        L.sdvg_version.restype = ctypes.c_int
        L.sdvg_shutdown.restype = None
        _bind_native(L)
        _LIB = L
    return _LIB


class _PythonOnly:
    """Stands in for the marshalling module where it has not been built: Python handles every call."""
    block_attn = rope = route = batch = commit = rollback = snapshot = staticmethod(lambda *args: None)
    page_plan = rope_positions = paged_commit = paged_attn = paged_prefix_attn = sample_tokens = staticmethod(lambda *args: None)


_NATIVE = None


def _bind_native(L):
    """Loads the marshalling module and hands it the entry points of the loaded libsdvg.so. The Python
    code makes every call by itself, so a library built alone works too, and says that it is slower."""
    global _NATIVE
    if not os.path.exists(NATIVE_PATH):
        warnings.warn("_native.so is missing, small calls take longer: build it with "
                      "`python -m paper_2604_17397_amd.build`", RuntimeWarning, stacklevel=3)
        _NATIVE = _PythonOnly
        return
    import numpy as np
    spec = importlib.util.spec_from_file_location("_native", NATIVE_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    entry = [ctypes.cast(f, ctypes.c_void_p).value for f in
             (L.sdvg_block_attn, L.sdvg_block_attn_commit, L.sdvg_rope, L.sdvg_worst_frame_route, L.sdvg_avg_frame_route,
              L.sdvg_block_attn_batch, L.sdvg_block_attn_batch_static, L.sdvg_kv_commit, L.sdvg_kv_commit_rope,
              L.sdvg_kv_rollback, L.sdvg_buffer_snapshot, L.sdvg_page_plan, L.sdvg_rope_positions, L.sdvg_paged_commit,
              L.sdvg_paged_attn, L.sdvg_paged_prefix_attn, L.sdvg_sample_tokens)]
    module.init(*entry, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, np.float32, sdvg_kv_cache, sdvg_paged_kv)
    _NATIVE = module


def _native():
    lib()
    return _NATIVE


def status_string(status):
    return lib().sdvg_status_string(int(status)).decode()


def _stream_ptr(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _memory_of(stream, device):
    """Context in which new tensors come from the memory of `stream`, a torch stream or anything with a cuda_stream."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    return torch.cuda.stream(stream)


def _empty(shape, dtype, device, stream):
    """A new tensor for a call on `stream` (None: the current one) to write. It comes from that stream's memory: a block that
    the allocator has for the current stream may still be written by work that is queued there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _memory_of(stream, device):
        return torch.empty(shape, dtype=dtype, device=device)


def _empty_like(t, stream):
    return _empty(t.shape, t.dtype, t.device, stream)


def _check_dev(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("libsdvg takes device tensors")


class KVCache:
    """Caller-owned KV cache of one model: k, v are bf16 device tensors whose logical view is
    [layers, capacity_tokens, heads, 128] (any layer/token/head strides, unit dim stride)."""

    def __init__(self, k, v, block_tokens, cache_len=0):
        _check_dev(k, v)
        assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16
        assert k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.stride(3) == 1
        self.k, self.v = k, v
        self.c = sdvg_kv_cache(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[2], k.shape[3],
                               int(block_tokens), k.shape[1], int(cache_len),
                               k.stride(0), k.stride(1), k.stride(2))

    @property
    def cache_len(self):
        return int(self.c.cache_len)

    def layer(self, i):
        """(k, v) views [capacity, heads, 128] of layer i."""
        return self.k[i], self.v[i]


def _attn_desc(q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale):
    """Checks one (q, cache, block, out) set and returns its descriptor. Shapes are checked
    against each other here, because a wrong length or head count would make the kernel read
    outside the tensors."""
    _check_dev(q, k_cache, v_cache, k_blk, v_blk, out)
    if q.dtype == torch.bfloat16:
        dtype = SDVG_BF16
    elif q.dtype == torch.float32:
        dtype = SDVG_F32
    else:
        raise TypeError("q must be bfloat16 or float32")
    if q.dim() != 3 or q.stride(2) != 1:
        raise ValueError("q must be 3-d with unit dim stride")
    if (k_cache is None) != (v_cache is None):
        raise ValueError("k_cache and v_cache come together")
    for t in (k_cache, v_cache, k_blk, v_blk):
        if t is not None and (t.dtype != q.dtype or t.dim() != 3 or t.stride(2) != 1):
            raise ValueError("all tensors share q's dtype, are 3-d and have unit dim stride")
        if t is not None and (t.shape[1] != q.shape[1] or t.shape[2] != q.shape[2]):
            raise ValueError("all tensors share q's head count and head_dim")
        if t is not None and t.device != q.device:
            raise ValueError("all tensors live on q's device")
    if v_blk.shape != k_blk.shape:
        raise ValueError("k_blk and v_blk must have the same shape")
    if cache_len < 0 or (cache_len > 0 and k_cache is None):
        raise ValueError("cache_len is negative, or positive without a cache")
    if k_cache is not None and (v_cache.shape != k_cache.shape or cache_len > k_cache.shape[0]):
        raise ValueError("cache_len exceeds the cache tensors (or k_cache / v_cache differ in shape)")
    if (out.shape != q.shape or out.dtype != q.dtype or out.stride(2) != 1 or out.device != q.device):
        raise ValueError("out must match q in shape, dtype and device and have unit dim stride")
    if k_blk.stride() != v_blk.stride() or (k_cache is not None and k_cache.stride() != v_cache.stride()):
        raise ValueError("k and v must share strides")
    kv_ts, kv_hs = (k_cache.stride(0), k_cache.stride(1)) if k_cache is not None else (128, 128)
    return sdvg_attn_desc(q.shape[0], k_blk.shape[0], q.shape[1], q.shape[2],
                          q.stride(0), q.stride(1), out.stride(0), out.stride(1),
                          kv_ts, kv_hs, k_blk.stride(0), k_blk.stride(1),
                          0.0 if scale is None else float(scale), dtype)


def block_attn(q, k_cache, v_cache, k_blk, v_blk, cache_len, out=None, scale=None, stream=None):
    """sdvg_block_attn: q, k_blk, v_blk [tokens, heads, 128]; k_cache, v_cache one layer's
    [>= cache_len, heads, 128] (may be None when cache_len == 0). `scale=None` passes 0, which the
    library reads as 1/sqrt(head_dim). `out` defaults to a new tensor; pass out=q for in place. Returns out."""
    r = (_NATIVE or _native()).block_attn(q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale,
                                         None if stream is None else stream.cuda_stream, False)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_block_attn")
        return r
    cache_len = int(cache_len)
    if out is None:
        out = _empty_like(q, stream)
    d = _attn_desc(q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale)
    st = lib().sdvg_block_attn(ctypes.byref(d), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_blk),
                               _ptr(v_blk), cache_len, _ptr(out), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_block_attn")
    return out


def block_attn_commit(q, k_cache, v_cache, k_blk, v_blk, cache_len, out=None, scale=None, stream=None):
    """sdvg_block_attn_commit: block_attn for one layer that also copies k_blk / v_blk into tokens
    [cache_len, cache_len + n_blk) of k_cache / v_cache (which must be long enough). Returns out."""
    r = (_NATIVE or _native()).block_attn(q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale,
                                         None if stream is None else stream.cuda_stream, True)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_block_attn_commit")
        return r
    cache_len = int(cache_len)
    if out is None:
        out = _empty_like(q, stream)
    if k_cache is None or v_cache is None:
        raise ValueError("the fused commit needs the layer's cache tensors")
    d = _attn_desc(q, k_cache, v_cache, k_blk, v_blk, cache_len, out, scale)
    if cache_len + k_blk.shape[0] > k_cache.shape[0]:
        raise ValueError("the cache has no room for the block after cache_len")
    st = lib().sdvg_block_attn_commit(ctypes.byref(d), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_blk),
                                      _ptr(v_blk), cache_len, _ptr(out), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_block_attn_commit")
    return out


def kv_commit_mark(cache, slot):
    st = lib().sdvg_kv_commit_mark(ctypes.byref(cache.c), int(slot))
    if st != 0:
        raise SdvgError(st, "sdvg_kv_commit_mark")


def _desc_key(d):
    return tuple(getattr(d, f) for f, _ in d._fields_)


def block_attn_workspace_bytes(q, k_cache, v_cache, k_blk, v_blk, cache_len, n_items=1, split="auto", scale=None):
    """sdvg_block_attn_workspace_bytes for the shape of these tensors; split is "never", "auto" or
    "always". For block_attn_batch; of block_attn_batch_static it tells the need under "always" only."""
    cache_len = int(cache_len)
    d = _attn_desc(q, k_cache, v_cache, k_blk, v_blk, cache_len, q, scale)
    n = lib().sdvg_block_attn_workspace_bytes(ctypes.byref(d), int(n_items), cache_len, _SPLIT[split])
    if n < 0:
        raise SdvgError(n, "sdvg_block_attn_workspace_bytes")
    return int(n)


def block_attn_batch_static(qs, k_caches, v_caches, k_blks, v_blks, cache_len, outs, split="auto", scale=None,
                            stream=None):
    """sdvg_block_attn_batch_static: as block_attn_batch, with the library's fixed workspace. `outs`
    is required (this entry point is for callers that do not allocate)."""
    return block_attn_batch(qs, k_caches, v_caches, k_blks, v_blks, cache_len, outs=outs, split=split, scale=scale,
                            stream=stream, _static=True)


def block_attn_batch(qs, k_caches, v_caches, k_blks, v_blks, cache_len, outs=None, workspace=None,
                     split="auto", scale=None, stream=None, _static=False):
    """sdvg_block_attn_batch: lists of n tensors each (k_caches / v_caches may be None when
    cache_len == 0); every item must have the same shapes and strides. `workspace`: optional
    device tensor (any dtype) the library may use to split keys over workgroups, under the policy
    `split` ("never", "auto", "always"). Returns outs."""
    if type(split) is str and split in _SPLIT:
        r = (_NATIVE or _native()).batch(qs, k_caches, v_caches, k_blks, v_blks, cache_len, outs, workspace,
                                        _SPLIT[split], scale, None if stream is None else stream.cuda_stream, _static)
        if r is not None:
            if type(r) is int:
                raise SdvgError(r, "sdvg_block_attn_batch_static" if _static else "sdvg_block_attn_batch")
            return r
    cache_len = int(cache_len)
    n = len(qs)
    if k_caches is None:
        k_caches, v_caches = [None] * n, [None] * n
    if not (len(k_caches) == len(v_caches) == len(k_blks) == len(v_blks) == n):
        raise ValueError("every list needs one tensor per item")
    if outs is None:
        outs = [_empty_like(q, stream) for q in qs]
    descs = [_attn_desc(qs[i], k_caches[i], v_caches[i], k_blks[i], v_blks[i], cache_len, outs[i], scale)
             for i in range(n)]
    if any(_desc_key(d) != _desc_key(descs[0]) for d in descs[1:]):
        raise ValueError("all items of a batch must share shapes, strides and dtype")
    if any(t.device != qs[0].device for t in qs):
        raise ValueError("all items live on one device")

    def arr(ts):
        return (ctypes.c_void_p * n)(*[t.data_ptr() if t is not None else None for t in ts])
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        _check_dev(workspace)
        if not workspace.is_contiguous() or workspace.device != qs[0].device:
            raise ValueError("workspace must be a contiguous tensor on the items' device")
        ws_ptr, ws_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
    if _static:
        st = lib().sdvg_block_attn_batch_static(ctypes.byref(descs[0]), n, arr(qs), arr(k_caches), arr(v_caches),
                                                arr(k_blks), arr(v_blks), cache_len, arr(outs), _SPLIT[split],
                                                _stream_ptr(stream))
    else:
        st = lib().sdvg_block_attn_batch(ctypes.byref(descs[0]), n, arr(qs), arr(k_caches), arr(v_caches),
                                         arr(k_blks), arr(v_blks), cache_len, arr(outs), ws_ptr, ws_bytes,
                                         _SPLIT[split], _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_block_attn_batch_static" if _static else "sdvg_block_attn_batch")
    return outs


def kv_commit(cache, k_blk, v_blk, slot, stream=None):
    """sdvg_kv_commit: k_blk, v_blk dense bf16 [layers, T, heads, 128]."""
    r = (_NATIVE or _native()).commit(cache.c, k_blk, v_blk, slot, None if stream is None else stream.cuda_stream)
    if r is not None:
        if r != 0:
            raise SdvgError(r, "sdvg_kv_commit")
        return
    _check_dev(k_blk, v_blk)
    if not (k_blk.is_contiguous() and v_blk.is_contiguous()):
        raise ValueError("k_blk and v_blk must be dense")
    L, T, H, D = cache.c.n_layers, cache.c.block_tokens, cache.c.n_heads, cache.c.head_dim
    if tuple(k_blk.shape) != (L, T, H, D) or tuple(v_blk.shape) != (L, T, H, D):
        raise ValueError("block shape must be [layers, T, heads, dim] of the cache")
    if k_blk.dtype != torch.bfloat16 or v_blk.dtype != torch.bfloat16:
        raise TypeError("k_blk and v_blk must be bfloat16")
    st = lib().sdvg_kv_commit(ctypes.byref(cache.c), _ptr(k_blk), _ptr(v_blk), int(slot),
                              _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_kv_commit")


def _check_tables(cos, sin, n_tokens, device):
    _check_dev(cos, sin)
    for t in (cos, sin):
        if t.dtype != torch.float32 or tuple(t.shape) != (n_tokens, 64) or not t.is_contiguous() or t.device != device:
            raise ValueError("cos / sin must be dense float32 [tokens, 64] on the tensors' device")


def rope(x, cos, sin, out=None, stream=None):
    """sdvg_rope: rotary embedding of bf16 rows x [tokens, heads, 128] by the angle tables cos, sin
    float32 [tokens, 64]. out defaults to a new tensor; pass out=x for in place."""
    r = (_NATIVE or _native()).rope(x, cos, sin, out, None if stream is None else stream.cuda_stream)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_rope")
        return r
    _check_dev(x, out)
    if x.dtype != torch.bfloat16 or x.dim() != 3 or x.shape[2] != 128 or x.stride(2) != 1:
        raise ValueError("x must be bfloat16 [tokens, heads, 128] with unit dim stride")
    if out is None:
        out = _empty_like(x, stream)
    elif out.shape != x.shape or out.dtype != x.dtype or out.stride(2) != 1 or out.device != x.device:
        raise ValueError("out must match x")
    _check_tables(cos, sin, x.shape[0], x.device)
    st = lib().sdvg_rope(_ptr(x), _ptr(cos), _ptr(sin), _ptr(out), x.shape[0], x.shape[1], x.shape[2],
                         x.stride(0), x.stride(1), out.stride(0), out.stride(1), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_rope")
    return out


def kv_commit_rope(cache, k_blk, v_blk, slot, cos, sin, stream=None):
    """sdvg_kv_commit_rope: kv_commit with k_blk (dense bf16 [layers, T, heads, 128], BEFORE the
    rotary embedding) rotated on its way into the cache; cos, sin float32 [T, 64]."""
    r = (_NATIVE or _native()).commit(cache.c, k_blk, v_blk, slot, None if stream is None else stream.cuda_stream, cos, sin)
    if r is not None:
        if r != 0:
            raise SdvgError(r, "sdvg_kv_commit_rope")
        return
    _check_dev(k_blk, v_blk)
    if not (k_blk.is_contiguous() and v_blk.is_contiguous()):
        raise ValueError("k_blk and v_blk must be dense")
    L, T, H, D = cache.c.n_layers, cache.c.block_tokens, cache.c.n_heads, cache.c.head_dim
    if tuple(k_blk.shape) != (L, T, H, D) or tuple(v_blk.shape) != (L, T, H, D):
        raise ValueError("block shape must be [layers, T, heads, dim] of the cache")
    if k_blk.dtype != torch.bfloat16 or v_blk.dtype != torch.bfloat16:
        raise TypeError("k_blk and v_blk must be bfloat16")
    _check_tables(cos, sin, T, k_blk.device)
    st = lib().sdvg_kv_commit_rope(ctypes.byref(cache.c), _ptr(k_blk), _ptr(v_blk), int(slot), _ptr(cos), _ptr(sin),
                                   _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_kv_commit_rope")


def kv_rollback(cache, new_len, stream=None):
    r = (_NATIVE or _native()).rollback(cache.c, new_len, None if stream is None else stream.cuda_stream)
    if r is not None:
        if r != 0:
            raise SdvgError(r, "sdvg_kv_rollback")
        return
    st = lib().sdvg_kv_rollback(ctypes.byref(cache.c), int(new_len), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_kv_rollback")


def buffer_snapshot(dst, src, n_bytes=None, stream=None):
    """sdvg_buffer_snapshot: dst[:n_bytes] = src[:n_bytes] for two device tensors viewed as bytes
    (n_bytes defaults to the size of src)."""
    r = (_NATIVE or _native()).snapshot(dst, src, n_bytes, None if stream is None else stream.cuda_stream)
    if r is not None:
        if r != 0:
            raise SdvgError(r, "sdvg_buffer_snapshot")
        return
    _check_dev(dst, src)
    if not (dst.is_contiguous() and src.is_contiguous()):
        raise ValueError("buffer_snapshot needs contiguous tensors")
    if n_bytes is None:
        n_bytes = src.numel() * src.element_size()
    if n_bytes > dst.numel() * dst.element_size() or n_bytes > src.numel() * src.element_size():
        raise ValueError("n_bytes exceeds a buffer")
    st = lib().sdvg_buffer_snapshot(_ptr(dst), _ptr(src), int(n_bytes), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_buffer_snapshot")


def worst_frame_route(frame_scores, tau, block_idx, stream=None, mode="min"):
    """sdvg_worst_frame_route (mode "min") or sdvg_avg_frame_route (mode "mean"): returns
    (decision, q_b) with q_b a numpy float32 scalar."""
    if mode in ("min", "mean"):
        r = (_NATIVE or _native()).route(frame_scores, tau, block_idx, mode == "mean",
                                        None if stream is None else stream.cuda_stream)
        if r is not None:
            if type(r) is int:
                raise SdvgError(r, "sdvg_worst_frame_route")
            return r
    import numpy as np
    fn = {"min": lib().sdvg_worst_frame_route, "mean": lib().sdvg_avg_frame_route}[mode]
    _check_dev(frame_scores)
    if frame_scores.dtype != torch.float32 or frame_scores.dim() != 1 or not frame_scores.is_contiguous():
        raise ValueError("frame_scores must be a dense 1-d float32 tensor")
    qb = np.zeros(1, dtype=np.float32)
    st = fn(_ptr(frame_scores), frame_scores.numel(), float(tau), int(block_idx),
            qb.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), _stream_ptr(stream))
    if st < 0:
        raise SdvgError(st, "sdvg_worst_frame_route")
    return int(st), qb[0]


def worst_frame_route_batch(frame_scores, tau, block_idx=None, first_block_idx=0, stream=None, mode="min"):
    """sdvg_worst_frame_route_batch (mode "min") or sdvg_avg_frame_route_batch (mode "mean"):
    frame_scores [n_blocks, n_frames] fp32; returns device tensors (decisions int32 [n_blocks],
    q_b float32 [n_blocks]). Asynchronous."""
    fn = {"min": lib().sdvg_worst_frame_route_batch, "mean": lib().sdvg_avg_frame_route_batch}[mode]
    _check_dev(frame_scores, block_idx)
    if frame_scores.dtype != torch.float32 or frame_scores.dim() != 2 or not frame_scores.is_contiguous():
        raise ValueError("frame_scores must be a dense 2-d float32 tensor")
    n_blocks, n_frames = frame_scores.shape
    if block_idx is not None and (block_idx.dtype != torch.int32 or block_idx.numel() != n_blocks):
        raise ValueError("block_idx must be int32 [n_blocks]")
    dec = _empty(n_blocks, torch.int32, frame_scores.device, stream)
    qb = _empty(n_blocks, torch.float32, frame_scores.device, stream)
    st = fn(_ptr(frame_scores), n_blocks, n_frames, float(tau), _ptr(block_idx), int(first_block_idx),
            _ptr(dec), _ptr(qb), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_worst_frame_route_batch")
    return dec, qb


# ---- paged cache

def _check_here(*tensors):
    """Device tensors on the current device, which is the one that calls launch on."""
    _check_dev(*tensors)
    for t in tensors:
        if t is not None and t.device.index != torch.cuda.current_device():
            raise ValueError("all tensors live on the current device")


class PagePlan:
    """What page_plan computes, in device tensors of its own that every plan of as many requests may reuse (max_tokens is the most
    new tokens that have rows): q_start int32 [requests + 1], kv_lens and held int32 [requests], positions int32 and slots
    int64 [max_tokens], next_free int32 [1] (held and next_free are written only by plans that take pages). Cleared on the
    current stream."""

    def __init__(self, n_requests, max_tokens, device="cuda"):
        n_requests, max_tokens = int(n_requests), int(max_tokens)
        if n_requests < 0 or max_tokens < 0:
            raise ValueError("negative size")
        ints = torch.zeros(3 * n_requests + 2 + max_tokens, dtype=torch.int32, device=device)
        self.q_start, self.kv_lens, self.held, self.next_free, self.positions = ints.split(
            [n_requests + 1, n_requests, n_requests, 1, max_tokens])
        self.slots = torch.zeros(max_tokens, dtype=torch.int64, device=device)


def _int32(name, v):
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError("%s must fit 32 bits" % name)
    return v


def _int_array(name, t, n, dtype=torch.int32):
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be a dense %s tensor of %d elements" % (name, str(dtype)[6:], n))


def page_plan(cached, new_tokens, block_table, page_tokens, free_pages=None, held=None, next_free=None, max_tokens=None,
              out=None, stream=None):
    """sdvg_page_plan: cached, new_tokens int32 [requests]; block_table int32 [requests, pages] (written in place);
    held int32 [requests], free_pages int32 [n] and next_free int32 [1] say which pages may be taken (held=None: none is).
    `out`: a PagePlan for as many requests (its positions and slots hold the new tokens), or None for a new one
    of `max_tokens` tokens. Returns the PagePlan."""
    if out is None:
        if max_tokens is None:
            raise ValueError("page_plan needs max_tokens or out")
        if stream is None:
            out = PagePlan(cached.shape[0], max_tokens, cached.device)
        else:
            with _memory_of(stream, cached.device):   # (its zeros must not come behind the plan)
                out = PagePlan(cached.shape[0], max_tokens, cached.device)
    elif max_tokens is not None and max_tokens != out.slots.shape[0]:
        raise ValueError("out holds another number of tokens than max_tokens")
    r = (_NATIVE or _native()).page_plan(cached, new_tokens, block_table, page_tokens, free_pages, held, next_free, out.q_start,
                                        out.kv_lens, out.positions, out.held, out.next_free, out.slots,
                                        None if stream is None else stream.cuda_stream)
    if r is not None:
        if r != 0:
            raise SdvgError(r, "sdvg_page_plan")
        return out
    n = cached.shape[0]
    _check_here(cached, new_tokens, block_table, free_pages, held, next_free, out.q_start, out.slots)
    _int_array("cached", cached, n)
    _int_array("new_tokens", new_tokens, n)
    _int_array("out.kv_lens", out.kv_lens, n)
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.shape[0] != n or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be int32 [requests, pages] with unit stride along the pages")
    if held is None and (free_pages is not None or next_free is not None):
        raise ValueError("free_pages and next_free come with held")
    if held is not None:
        _int_array("held", held, n)
    if free_pages is not None:
        _int_array("free_pages", free_pages, free_pages.shape[0])
    if next_free is not None:
        _int_array("next_free", next_free, 1)

    def p(t):
        return None if t is None or t.numel() == 0 else t.data_ptr()
    a = sdvg_page_plan_args(n, _int32("page_tokens", page_tokens), block_table.shape[1], 0 if free_pages is None else free_pages.shape[0],
                            block_table.stride(0) if n > 1 else block_table.shape[1], out.slots.shape[0],
                            p(cached), p(new_tokens), p(free_pages),
                            # (without requests an empty `held` has no address, and still says that pages may be taken)
                            None if held is None else p(held) or p(out.q_start),
                            p(next_free), p(block_table), p(out.q_start), p(out.kv_lens), p(out.positions), p(out.held),
                            p(out.next_free), p(out.slots))
    st = lib().sdvg_page_plan(ctypes.byref(a), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_page_plan")
    return out


def rope_frequencies(rotary_dim, theta=10000.0, scaling="none", factor=1.0, original=None, beta_fast=32.0, beta_slow=1.0,
                     device="cuda"):
    """(freqs, gain) for rope_positions and paged_commit: radians per position of every pair, theta^(-2p / rotary_dim), as
    float64 [rotary_dim / 2], and the factor of cos and sin. For contexts `factor` times the original length:
    "linear" divides every frequency by factor; "ntk" takes theta * factor^(rotary_dim / (rotary_dim - 2)), which leaves
    the fastest pair alone and divides the slowest by factor; "yarn" (Peng et al., 2023) interpolates pairs that turn at
    most beta_slow times over `original` positions, leaves those that turn at least beta_fast times, mixes in between, and
    has gain 0.1 ln(factor) + 1."""
    rotary_dim, theta, factor = int(rotary_dim), float(theta), float(factor)
    if rotary_dim < 16 or rotary_dim > 128 or rotary_dim % 16:
        raise ValueError("rotary_dim must be a multiple of 16, at most 128")
    if not (0 < theta < math.inf and 1 <= factor < math.inf):
        raise ValueError("theta must be positive and factor at least 1")
    if scaling not in ("none", "linear", "ntk", "yarn"):
        raise ValueError("scaling must be none, linear, ntk or yarn")
    p = torch.arange(0, rotary_dim, 2, dtype=torch.float64)
    if scaling == "ntk":
        theta *= factor ** (rotary_dim / (rotary_dim - 2))
    w = theta ** (-p / rotary_dim)
    gain = 1.0
    if scaling == "linear":
        w = w / factor
    elif scaling == "yarn":
        if original is None or not original > 0 or not 0 <= beta_slow < beta_fast:
            raise ValueError("yarn needs the original length and 0 <= beta_slow < beta_fast")
        keep = ((original * w / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow)).clamp(0, 1)
        w = w * keep + w / factor * (1 - keep)
        gain = 0.1 * math.log(factor) + 1.0
    return w.to(device), gain


_ROW_TYPES = {torch.bfloat16: SDVG_BF16, torch.float32: SDVG_F32, torch.float16: SDVG_F16}


def _rope_desc(positions, freqs, layout, gain, n_tokens):
    _check_here(positions, freqs)
    _int_array("positions", positions, n_tokens)
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError("freqs must be a dense float64 tensor [rotary_dim / 2]")
    if layout not in _LAYOUT:
        raise ValueError("layout must be half or interleaved")
    return sdvg_rope_desc(positions.data_ptr(), freqs.data_ptr(), 2 * freqs.shape[0], _LAYOUT[layout], float(gain))


def _check_rows(name, t, like=None):
    if t.dim() != 3 or t.shape[2] != 128 or t.stride(2) != 1 or t.dtype not in _ROW_TYPES:
        raise ValueError("%s must be [tokens, heads, 128] of 16 or 32 bit floats with unit dim stride" % name)
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype):
        raise ValueError("%s must match its input" % name)


def _rows(t, out):
    return sdvg_rows(t.data_ptr(), None if out is None else out.data_ptr(), t.shape[1], t.stride(0), t.stride(1),
                     0 if out is None else out.stride(0), 0 if out is None else out.stride(1))


def rope_positions(x, positions, freqs, y=None, layout="half", gain=1.0, out=None, y_out=None, stream=None):
    """sdvg_rope_positions: rotary embedding of x [tokens, heads, 128], and of y (as many tokens and the same dtype, any
    number of heads) in the same launch, at int32 positions [tokens] with float64 freqs [rotary_dim / 2] (rope_frequencies).
    layout "half" pairs elements p and p + rotary_dim / 2, "interleaved" 2p and 2p + 1. out / y_out default to new tensors;
    pass the input for in place. Returns out, or (out, y_out) with y."""
    if type(layout) is str and layout in _LAYOUT:
        r = (_NATIVE or _native()).rope_positions(x, positions, freqs, y, _LAYOUT[layout], gain, out, y_out,
                                                 None if stream is None else stream.cuda_stream)
        if r is not None:
            if type(r) is int:
                raise SdvgError(r, "sdvg_rope_positions")
            return r
    _check_here(x, y, out, y_out)
    _check_rows("x", x)
    if y is None and y_out is not None:
        raise ValueError("y_out comes with y")
    if y is not None:
        _check_rows("y", y)
        if y.dtype != x.dtype or y.shape[0] != x.shape[0]:
            raise ValueError("y must have x's tokens and dtype")
    rope = _rope_desc(positions, freqs, layout, gain, x.shape[0])
    out = _empty_like(x, stream) if out is None else out
    _check_rows("out", out, x)
    if y is not None:
        y_out = _empty_like(y, stream) if y_out is None else y_out
        _check_rows("y_out", y_out, y)
    st = lib().sdvg_rope_positions(ctypes.byref(rope), ctypes.byref(_rows(x, out)),
                                   None if y is None else ctypes.byref(_rows(y, y_out)), x.shape[0], 128,
                                   _ROW_TYPES[x.dtype], _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_rope_positions")
    return out if y is None else (out, y_out)


class PagedKV:
    """Caller-owned paged KV cache of one layer: k, v device tensors [pages, page_tokens, kv_heads, 128] (any page / token /
    head strides, unit dim stride) of bfloat16, float16 or float8_e4m3fn; the latter with optional float32 scales
    [kv_heads] (a stored number x stands for x * scale)."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        _check_dev(k, v, k_scale, v_scale)
        types = {torch.bfloat16: SDVG_BF16, torch.float16: SDVG_F16, torch.float8_e4m3fn: SDVG_E4M3}
        if k.dtype not in types or v.dtype != k.dtype:
            raise TypeError("k and v must both be bfloat16, float16 or float8_e4m3fn")
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.stride(3) != 1 or v.device != k.device:
            raise ValueError("k and v must be [pages, page_tokens, kv_heads, 128] with the same strides and unit dim stride")
        for t in (k_scale, v_scale):
            if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (k.shape[2],) or not t.is_contiguous()
                                  or t.device != k.device):
                raise ValueError("k_scale and v_scale must be dense float32 [kv_heads] on the cache's device")
            if t is not None and k.dtype != torch.float8_e4m3fn:
                raise ValueError("scales come with a float8 cache")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.c = sdvg_paged_kv(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                               None if v_scale is None else v_scale.data_ptr(), k.shape[0], k.shape[1], k.shape[2], k.shape[3],
                               k.stride(0), k.stride(1), k.stride(2), types[k.dtype])


def paged_commit(cache, k, v, slots, positions=None, freqs=None, q=None, q_out=None, layout="half", gain=1.0, stream=None):
    """sdvg_paged_commit: rows k, v [tokens, kv_heads, 128] of bfloat16 or float16 into the int64 slots [tokens] of a PagedKV;
    a negative slot writes nothing. With positions and freqs (as for rope_positions) K is rotated on its way, and so is
    q [tokens, heads, 128] into q_out (default: a new tensor; pass q for in place). Returns q_out, or None without q."""
    if type(layout) is str and layout in _LAYOUT:
        r = (_NATIVE or _native()).paged_commit(cache.c, cache.k, k, v, slots, positions, freqs, q, q_out, _LAYOUT[layout], gain,
                                               None if stream is None else stream.cuda_stream)
        if r is not None:
            if type(r) is int:
                if r != 0:
                    raise SdvgError(r, "sdvg_paged_commit")
                return None
            return r
    _check_here(cache.k, k, v, slots, q, q_out)
    for name, t in (("k", k), ("v", v)):
        _check_rows(name, t)
        if t.shape[1] != cache.c.n_kv_heads or t.shape[0] != k.shape[0] or t.dtype != k.dtype:
            raise ValueError("k and v must have the cache's heads, the same tokens and dtype")
    if k.dtype == torch.float32 or (cache.k.dtype != torch.float8_e4m3fn and cache.k.dtype != k.dtype):
        raise ValueError("k and v must be bfloat16 or float16, of the cache's own dtype unless that is float8")
    _int_array("slots", slots, k.shape[0], torch.int64)
    if (positions is None) != (freqs is None) or (q is not None and positions is None) or (q is None and q_out is not None):
        raise ValueError("positions and freqs come together, q with both, q_out with q")
    rope = None if positions is None else _rope_desc(positions, freqs, layout, gain, k.shape[0])
    if q is not None:
        _check_rows("q", q)
        if q.dtype != k.dtype or q.shape[0] != k.shape[0]:
            raise ValueError("q must have k's tokens and dtype")
        q_out = _empty_like(q, stream) if q_out is None else q_out
        _check_rows("q_out", q_out, q)
    st = lib().sdvg_paged_commit(ctypes.byref(cache.c), ctypes.byref(_rows(k, None)), ctypes.byref(_rows(v, None)),
                                 _ptr(slots), k.shape[0], _ROW_TYPES[k.dtype], None if rope is None else ctypes.byref(rope),
                                 None if q is None else ctypes.byref(_rows(q, q_out)), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_paged_commit")
    return q_out


def _paged_attn_desc(q, cache, block_table, out, scale, window):
    _check_rows("q", q)
    if q.dtype == torch.float32 or (cache.k.dtype != torch.float8_e4m3fn and cache.k.dtype != q.dtype):
        raise ValueError("q must be bfloat16 or float16, of the cache's dtype unless that is float8")
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise ValueError("block_table must be int32 [requests, pages] with unit stride along the pages")
    _check_rows("out", out, q)
    n = block_table.shape[0]
    return sdvg_paged_attn_desc(n, q.shape[0], q.shape[1], q.shape[2], block_table.shape[1], _int32("window", window),
                                block_table.stride(0), q.stride(0), q.stride(1), out.stride(0), out.stride(1),
                                0.0 if scale is None else float(scale), _ROW_TYPES[q.dtype])


def paged_attn_workspace_bytes(q, cache, block_table):
    """sdvg_paged_attn_workspace_bytes for the shapes of these tensors."""
    _check_here(q, cache.k, block_table)
    d = _paged_attn_desc(q, cache, block_table, q, None, 0)
    n = lib().sdvg_paged_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(cache.c))
    if n < 0:
        raise SdvgError(n, "sdvg_paged_attn_workspace_bytes")
    return int(n)


def _attn_args(q, cache, block_table, q_start, kv_lens, out, lse, scale, window, workspace, stream):
    """Checks what paged_attn and paged_prefix_attn have in common; the descriptor and the output."""
    _check_here(q, cache.k, block_table, q_start, kv_lens, out, lse, workspace)
    if out is None:
        out = _empty_like(q, stream)
    d = _paged_attn_desc(q, cache, block_table, out, scale, window)
    _int_array("q_start", q_start, d.n_requests + 1)
    _int_array("kv_lens", kv_lens, d.n_requests)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous()):
        raise ValueError("lse must be dense float32 [tokens, heads]")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return d, out


def paged_attn(q, cache, block_table, q_start, kv_lens, out=None, lse=None, scale=None, window=0, workspace=None, stream=None):
    """sdvg_paged_attn: attention of the new tokens q [tokens, heads, 128] of several requests over their pages in a PagedKV.
    block_table int32 [requests, pages], q_start int32 [requests + 1] and kv_lens int32 [requests] as page_plan leaves
    them. `window` > 0: every token sees the last `window` keys only. `lse`: optional float32 [tokens, heads] for the log of the sums.
    `workspace`: optional device tensor of paged_attn_workspace_bytes, with which the keys of long requests are split
    over the chip. `scale=None` is 1/sqrt(128). out defaults to a new tensor; pass out=q for in place. Returns out."""
    r = (_NATIVE or _native()).paged_attn(q, cache.c, cache.k, block_table, q_start, kv_lens, out, lse, scale, window, workspace,
                                         None if stream is None else stream.cuda_stream)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_paged_attn")
        return r
    d, out = _attn_args(q, cache, block_table, q_start, kv_lens, out, lse, scale, window, workspace, stream)
    st = lib().sdvg_paged_attn(ctypes.byref(d), ctypes.byref(cache.c), _ptr(q), _ptr(block_table), _ptr(q_start), _ptr(kv_lens),
                               _ptr(out), _ptr(lse), _ptr(workspace),
                               0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_paged_attn")
    return out


def _n_groups(prefix_lens, group_start):
    n = prefix_lens.shape[0] if prefix_lens.dim() == 1 else -1
    _int_array("prefix_lens", prefix_lens, n)
    if group_start is not None:
        _int_array("group_start", group_start, n + 1)
    elif n > 1:
        raise ValueError("several prefixes need group_start")
    return n


def paged_prefix_attn_workspace_bytes(q, cache, block_table, n_groups=1):
    """sdvg_paged_prefix_attn_workspace_bytes for the shapes of these tensors and a number of groups."""
    _check_here(q, cache.k, block_table)
    d, n_groups = _paged_attn_desc(q, cache, block_table, q, None, 0), _int32("n_groups", n_groups)
    n = lib().sdvg_paged_prefix_attn_workspace_bytes(ctypes.byref(d), ctypes.byref(cache.c), n_groups)
    if n < 0:
        raise SdvgError(n, "sdvg_paged_prefix_attn_workspace_bytes")
    return int(n)


def paged_prefix_attn(q, cache, block_table, q_start, kv_lens, prefix_lens, group_start=None, out=None, lse=None, scale=None,
                      window=0, workspace=None, stream=None):
    """sdvg_paged_prefix_attn: paged_attn where the requests of a group share their first keys, which are then read once for the
    group. prefix_lens int32 [groups]: shared keys, which the rows of block_table of a group's requests name alike; group_start int32
    [groups + 1]: first request of every group and the end of the last one (None: one group of all requests). kv_lens and
    positions count the shared keys, and no new token lies among them. `workspace`: device tensor of
    paged_prefix_attn_workspace_bytes; without it, or with one that is too small, the call is paged_attn: the same result, nothing shared. Pays from
    some 150000 to 200000 keys on that are not read again, (requests - 1) x shared keys x key heads. Everything else as in paged_attn. Returns out."""
    r = (_NATIVE or _native()).paged_prefix_attn(q, cache.c, cache.k, block_table, q_start, kv_lens, out, lse, scale, window, workspace,
                                                None if stream is None else stream.cuda_stream, prefix_lens, group_start)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_paged_prefix_attn")
        return r
    _check_here(q, prefix_lens, group_start)
    n_groups = _n_groups(prefix_lens, group_start)
    d, out = _attn_args(q, cache, block_table, q_start, kv_lens, out, lse, scale, window, workspace, stream)
    st = lib().sdvg_paged_prefix_attn(ctypes.byref(d), ctypes.byref(cache.c), _ptr(q), _ptr(block_table), _ptr(q_start), _ptr(kv_lens),
                                      n_groups, _ptr(group_start), _ptr(prefix_lens), _ptr(out), _ptr(lse), _ptr(workspace),
                                      0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_paged_prefix_attn")
    return out


def sample_tokens_workspace_bytes(n_rows, vocab):
    """sdvg_sample_tokens_workspace_bytes: for logits [n_rows, vocab] of any type."""
    n_rows, vocab = _int32("n_rows", n_rows), _int32("vocab", vocab)
    n = lib().sdvg_sample_tokens_workspace_bytes(n_rows, vocab)
    if n < 0:
        raise SdvgError(n, "sdvg_sample_tokens_workspace_bytes")
    return int(n)


def _setting(name, x, dtype, n, off):
    """A setting of sample_tokens: one per row, as an array, or one number for all (None: off)."""
    if isinstance(x, torch.Tensor):
        if x.dtype != dtype or x.shape != (n,) or not x.is_contiguous():
            raise ValueError("%s must be a number or dense %s [rows]" % (name, str(dtype)[6:]))
        return x, off
    return None, off if x is None else _int32(name, x) if dtype == torch.int32 else float(x)


def sample_tokens(logits, u, temperature=1.0, top_k=None, top_p=None, min_p=None, out=None, logprob=None, workspace=None, stream=None):
    """sdvg_sample_tokens: a token for every row of logits [rows, vocab] (float32, bfloat16 or float16), from the random numbers u
    float32 [rows] in [0, 1). temperature, top_p, min_p (float32) and top_k (int32): an array [rows] each, or a number for all rows, or
    None (off); temperature 0 takes the largest logit. `logprob`: optional float32 [rows] for the log of the drawn token's probability among
    the kept ones. `workspace`: device tensor of sample_tokens_workspace_bytes; None makes one for the call. out defaults to a new
    int32 tensor [rows]. Returns out."""
    r = (_NATIVE or _native()).sample_tokens(logits, u, temperature, top_k, top_p, min_p, out, logprob, workspace,
                                            None if stream is None else stream.cuda_stream)
    if r is not None:
        if type(r) is int:
            raise SdvgError(r, "sdvg_sample_tokens")
        return r
    arrays = [x for x in (temperature, top_k, top_p, min_p) if isinstance(x, torch.Tensor)]
    _check_here(logits, u, out, logprob, workspace, *arrays)
    if logits.dtype not in _ROW_TYPES or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be float32, bfloat16 or float16 [rows, vocab] with unit stride along the vocabulary")
    n, vocab = logits.shape
    if u.dtype != torch.float32 or u.shape != (n,) or not u.is_contiguous():
        raise ValueError("u must be dense float32 [rows]")
    (t, all_t), (k, all_k) = _setting("temperature", temperature, torch.float32, n, 1.0), _setting("top_k", top_k, torch.int32, n, 0)
    (p, all_p), (m, all_m) = _setting("top_p", top_p, torch.float32, n, 1.0), _setting("min_p", min_p, torch.float32, n, 0.0)
    if out is not None and (out.dtype != torch.int32 or out.shape != (n,) or not out.is_contiguous()):
        raise ValueError("out must be dense int32 [rows]")
    if logprob is not None and (logprob.dtype != torch.float32 or logprob.shape != (n,) or not logprob.is_contiguous()):
        raise ValueError("logprob must be dense float32 [rows]")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if workspace is None:
        workspace = _empty((sample_tokens_workspace_bytes(n, vocab),), torch.uint8, logits.device, stream)
    if out is None:
        out = _empty((n,), torch.int32, logits.device, stream)
    a = sdvg_sample_args(logits.data_ptr(), u.data_ptr(), t.data_ptr() if t is not None else None, k.data_ptr() if k is not None else None,
                         p.data_ptr() if p is not None else None, m.data_ptr() if m is not None else None, all_t, all_k, all_p, all_m,
                         out.data_ptr(), logprob.data_ptr() if logprob is not None else None, logits.stride(0), n, vocab, _ROW_TYPES[logits.dtype])
    st = lib().sdvg_sample_tokens(ctypes.byref(a), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, "sdvg_sample_tokens")
    return out


def probe_mfma(iters=20000, stream=None, changing=False):
    """sdvg_probe_mfma (or, with changing=True, sdvg_probe_mfma_changing): enqueues the MFMA-only
    measurement kernel. Returns (flops, cycles) with cycles a device uint64 tensor (as int64)
    holding wave 0's shader clocks once it has run."""
    dev = torch.device("cuda", torch.cuda.current_device())
    out = _empty(256 * 256, torch.float32, dev, stream)
    with contextlib.nullcontext() if stream is None else _memory_of(stream, dev):
        cycles = torch.zeros(1, dtype=torch.int64, device=dev)
    flops = ctypes.c_double(0.0)
    name = "sdvg_probe_mfma_changing" if changing else "sdvg_probe_mfma"
    st = getattr(lib(), name)(_ptr(out), out.numel(), _ptr(cycles), int(iters), ctypes.byref(flops),
                              _stream_ptr(stream))
    if st != 0:
        raise SdvgError(st, name)
    return flops.value, cycles
