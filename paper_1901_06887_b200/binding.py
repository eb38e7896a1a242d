"""Thin ctypes binding of libmt.so: the same entry points as include/mt.h, argument marshalling only.

Every step of the inference path runs inside the CUDA library.  There is no fallback: if libmt.so has
not been built (``python -m paper_1901_06887_b200.build``) importing a function from here raises.
torch is used for device memory and streams only.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmt.so")

MT_OK = 0
STATUS_NAMES = {0: "MT_OK", 1: "MT_ERR_INVALID_ARG", 2: "MT_ERR_BAD_MODEL_ID", 3: "MT_ERR_SHAPE",
                4: "MT_ERR_UNSUPPORTED", 5: "MT_ERR_OOM", 6: "MT_ERR_CUDA", 7: "MT_ERR_ARCH",
                8: "MT_ERR_TIMEOUT", 9: "MT_ERR_NOT_INIT", 10: "MT_ERR_NOT_RESIDENT"}

EXPORTS = ["mt_init", "mt_shutdown", "mt_register_model", "mt_infer", "mt_infer_host", "mt_infer_host_async", "mt_release",
           "mt_get_async_status", "mt_status_string", "mt_debug_last_bucketing", "mt_set_kernel_timing",
           "mt_get_kernel_times", "mt_bucket_noalloc", "mt_debug_wait_timeout", "mt_debug_launch_count", "mt_debug_set_option", "mt_debug_empty_launches", "mt_debug_item_cost",
           "mt_debug_schedule_balance", "mt_set_cache_bytes", "mt_prefetch", "mt_get_cache_stats", "mt_cache_sim_create",
           "mt_cache_sim_access", "mt_cache_sim_release", "mt_cache_sim_read", "mt_cache_sim_batch", "mt_cache_sim_wait", "mt_cache_sim_stats", "mt_cache_sim_destroy", "mt_output_elems", "mt_input_elems",
           "mt_prompt_attention", "mt_kv_append", "mt_kv_read", "mt_kv_attention", "mt_quant_packed_bytes", "mt_quant_pack",
           "mt_quant_linear", "mt_token_logprobs", "mt_cross_attention", "mt_rotate", "mt_kv_reserve", "mt_kv_fork", "mt_kv_release",
           "mt_kv_compact", "mt_kv_copy", "mt_token_sample"]


class MtError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__("%s failed: %s (%d)" % (where, STATUS_NAMES.get(int(code), "?"), int(code)))


class CacheStats(ctypes.Structure):
    _fields_ = [(k, ctypes.c_uint64) for k in ("capacity_bytes", "resident_bytes", "tenant_hits", "tenant_misses",
                                               "request_hits", "request_misses", "evictions", "bytes_loaded")]

    def as_dict(self):
        return {k: int(getattr(self, k)) for k, _ in self._fields_}


class LayerDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("in_ch", ctypes.c_int32), ("out_ch", ctypes.c_int32),
                ("h", ctypes.c_int32), ("w", ctypes.c_int32), ("relu", ctypes.c_int32), ("residual", ctypes.c_int32),
                ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


# mt_prompt_desc as bytes: n_tokens, n_seqs, q_heads, kv_heads, head_dim, scale, then token and head strides of q, k, v
_prompt_desc = struct.Struct("=5if6q").pack
# mt_cross_desc: n_tokens, n_states, n_seqs, q_heads, kv_heads, head_dim, scale, four bytes of padding, strides of q, k, v
_cross_desc = struct.Struct("=6if4x6q").pack
# mt_rotate_desc: n, heads, head_dim, rotary_dim, axes, four sections, neighbours, inverse, dtype, token and head strides of x and out
_rotate_desc = struct.Struct("=12i4q").pack


class KvCacheDesc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("n_pages", "page_tokens", "kv_heads", "head_dim")] + \
               [(k, ctypes.c_void_p) for k in ("k_codes", "k_params", "v_codes", "v_params")]


class KvPagesDesc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("n_pages", "page_tokens", "n_rows", "table_width")] + \
               [(k, ctypes.c_void_p) for k in ("refs", "tables", "lengths")]


class QuantBankDesc(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("tenants", "in_features", "out_features", "group")] + \
               [(k, ctypes.c_void_p) for k in ("packed", "bias")]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libmt.so (once).  Raises if it is missing: there is no other implementation to fall back to."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("CUDA library %s not built; run `python -m paper_1901_06887_b200.build`" % LIB_PATH)
        l = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        l.mt_init.argtypes = [i32, i32, i32]
        l.mt_shutdown.argtypes = []
        l.mt_register_model.argtypes = [ctypes.POINTER(LayerDesc), i32, ctypes.POINTER(i32)]
        l.mt_infer.argtypes = [vp, vp, i32, vp, vp]
        l.mt_infer_host.argtypes = [vp, vp, i32, vp, vp]
        l.mt_infer_host_async.argtypes = [vp, vp, i32, vp, vp]
        l.mt_release.argtypes = [i32]
        l.mt_get_async_status.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        l.mt_status_string.argtypes = [i32]
        l.mt_status_string.restype = ctypes.c_char_p
        l.mt_debug_last_bucketing.argtypes = [vp] * 4 + [ctypes.POINTER(i32)]
        l.mt_set_kernel_timing.argtypes = [i32]
        l.mt_get_kernel_times.argtypes = [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                                          ctypes.POINTER(i32), i32, ctypes.POINTER(i32)]
        l.mt_bucket_noalloc.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
        l.mt_debug_wait_timeout.argtypes = [i32, vp]
        l.mt_debug_launch_count.argtypes = [ctypes.POINTER(ctypes.c_int64)]
        l.mt_debug_set_option.argtypes = [ctypes.c_char_p, i32]
        l.mt_debug_empty_launches.argtypes = [i32, vp]
        l.mt_output_elems.argtypes = [ctypes.POINTER(i32)]
        l.mt_input_elems.argtypes = [ctypes.POINTER(i32)]
        l.mt_set_cache_bytes.argtypes = [ctypes.c_size_t]
        l.mt_prefetch.argtypes = [vp, i32, vp]
        l.mt_get_cache_stats.argtypes = [ctypes.POINTER(CacheStats), i32]
        l.mt_cache_sim_create.argtypes = [ctypes.c_size_t, ctypes.POINTER(vp)]
        l.mt_cache_sim_access.argtypes = [vp, i32, ctypes.c_size_t, ctypes.c_uint64, ctypes.POINTER(i32),
                                          ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(i32), i32, ctypes.POINTER(i32)]
        l.mt_cache_sim_release.argtypes = [vp, i32]
        l.mt_cache_sim_read.argtypes = [vp, i32]
        l.mt_cache_sim_batch.argtypes = [vp, i32]
        l.mt_cache_sim_wait.argtypes = [vp, ctypes.POINTER(ctypes.c_uint64)]
        l.mt_cache_sim_stats.argtypes = [vp, ctypes.POINTER(CacheStats)]
        l.mt_cache_sim_destroy.argtypes = [vp]
        l.mt_debug_item_cost.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_double)]
        l.mt_debug_schedule_balance.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32), ctypes.POINTER(i32)]
        i64, f32 = ctypes.c_int64, ctypes.c_float
        l.mt_prompt_attention.argtypes = [vp] * 7
        l.mt_kv_append.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp, i32, vp]
        l.mt_kv_read.argtypes = [vp, vp, i32, vp, vp, vp]
        l.mt_kv_attention.argtypes = [vp, vp, i64, i64, vp, i32, vp, i32, i32, f32, vp, vp]
        l.mt_quant_packed_bytes.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        l.mt_quant_pack.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp]
        l.mt_quant_linear.argtypes = [vp, vp, i64, vp, i32, vp, i64, i32, vp]
        l.mt_token_logprobs.argtypes = [vp, i32, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp]
        l.mt_cross_attention.argtypes = [vp] * 8
        l.mt_rotate.argtypes = [vp] * 6
        l.mt_kv_reserve.argtypes = [vp, vp, vp, i32, vp, i64, vp]
        l.mt_kv_fork.argtypes = [vp, vp, vp, i32, vp, vp]
        l.mt_kv_release.argtypes = [vp, vp, i32, vp]
        l.mt_kv_compact.argtypes = [vp, vp, i32, vp]
        l.mt_kv_copy.argtypes = [vp, i32, vp, i32, vp]
        l.mt_token_sample.argtypes = [vp, i32, i64, i32, i32] + [vp] * 8
        for name in EXPORTS:
            if name != "mt_status_string":
                getattr(l, name).restype = ctypes.c_int
        _lib = l
    return _lib


def _check(code: int, where: str) -> None:
    if code != MT_OK:
        raise MtError(code, where)


def _ptr(x) -> Optional[int]:
    """Address of a torch tensor (device or host), a numpy array, or None."""
    if x is None:
        return None
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return x.data_ptr()


_raw_stream = None


def _stream_handle(stream) -> Optional[int]:
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            raw, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            torch.cuda.current_stream()          # (initialises CUDA)
            if raw is not None and dev is not None:
                _raw_stream = lambda: raw(dev())     # torch.cuda.current_stream().cuda_stream without the stream object: 0.2 instead of 3 us
            else:
                _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
        return _raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_device = None          # the context's device


def mt_init(device: int = 0, max_models: int = 1024, max_batch: int = 0) -> None:
    global _device
    _check(lib().mt_init(device, max_models, max_batch), "mt_init")
    if _device is None:      # (a context that is there keeps its device)
        _device = int(device)


def mt_shutdown() -> None:
    global _device
    _check(lib().mt_shutdown(), "mt_shutdown")
    _device = None


def mt_register_model(layers: Sequence) -> int:
    """layers: objects with kind, in_ch, out_ch, h, w, relu, weight, bias and optionally residual (weight: uint16 numpy array of bf16
    bit patterns or a torch bf16 tensor, host or device; bias: float32 or None).  Returns the model id."""
    arr = (LayerDesc * len(layers))()
    keep = []
    for i, l in enumerate(layers):
        w, b = l.weight, l.bias
        if isinstance(w, np.ndarray):
            w = np.ascontiguousarray(w, dtype=np.uint16)
        if isinstance(b, np.ndarray):
            b = np.ascontiguousarray(b, dtype=np.float32)
        keep += [w, b]
        arr[i] = LayerDesc(int(l.kind), int(l.in_ch), int(l.out_ch), int(l.h), int(l.w), int(l.relu), int(getattr(l, "residual", 0)),
                           _ptr(w), _ptr(b))
    mid = ctypes.c_int32(-1)
    _check(lib().mt_register_model(arr, len(layers), ctypes.byref(mid)), "mt_register_model")
    return int(mid.value)


def mt_release(model_id: int) -> None:
    _check(lib().mt_release(int(model_id)), "mt_release")


def mt_infer(inputs, model_ids, n: int, outputs, stream=None) -> None:
    """inputs: device bf16 [n, in_elems]; model_ids: device int32 [n]; outputs: device fp32 [n, out_elems]."""
    _check(lib().mt_infer(_ptr(inputs), _ptr(model_ids), int(n), _ptr(outputs), _stream_handle(stream)), "mt_infer")


def mt_infer_host(inputs, model_ids, n: int, outputs, stream=None) -> None:
    """Same with host buffers (pinned torch tensors or numpy arrays); returns after the outputs have landed."""
    _check(lib().mt_infer_host(_ptr(inputs), _ptr(model_ids), int(n), _ptr(outputs), _stream_handle(stream)),
           "mt_infer_host")


def mt_infer_host_async(inputs, model_ids, n: int, outputs, stream=None) -> None:
    """mt_infer_host without the final synchronisation: pinned host buffers, everything enqueued on `stream`.
    Alternate between two streams to overlap one batch's copies with the next batch's kernels; synchronise the
    stream before reading `outputs`."""
    _check(lib().mt_infer_host_async(_ptr(inputs), _ptr(model_ids), int(n), _ptr(outputs), _stream_handle(stream)),
           "mt_infer_host_async")


def mt_get_async_status(stream=None) -> Tuple[int, int]:
    st, bad = ctypes.c_int32(0), ctypes.c_int32(-1)
    _check(lib().mt_get_async_status(_stream_handle(stream), ctypes.byref(st), ctypes.byref(bad)), "mt_get_async_status")
    return int(st.value), int(bad.value)


def mt_status_string(code: int) -> str:
    return lib().mt_status_string(int(code)).decode()


def mt_debug_last_bucketing(n: int):
    """Copies of (counts[T], offsets[T+2], perm[n], inv[n]) of the last mt_infer (batch size n) as numpy int32."""
    T = ctypes.c_int32(0)
    _check(lib().mt_debug_last_bucketing(None, None, None, None, ctypes.byref(T)), "mt_debug_last_bucketing")
    arrs = [np.zeros(T.value, np.int32), np.zeros(T.value + 2, np.int32), np.zeros(n, np.int32), np.zeros(n, np.int32)]
    _check(lib().mt_debug_last_bucketing(*[a.ctypes.data for a in arrs], None), "mt_debug_last_bucketing")
    return tuple(arrs)


def mt_debug_wait_timeout(limit_ms: int = 20, stream=None) -> None:
    """Enqueue the bounded-wait self-test (a wait nothing satisfies); mt_get_async_status then reports MT_ERR_TIMEOUT."""
    _check(lib().mt_debug_wait_timeout(int(limit_ms), _stream_handle(stream)), "mt_debug_wait_timeout")


def mt_debug_launch_count() -> int:
    """Kernels enqueued by mt_infer / mt_infer_host since the library was loaded."""
    c = ctypes.c_int64(0)
    _check(lib().mt_debug_launch_count(ctypes.byref(c)), "mt_debug_launch_count")
    return int(c.value)


def mt_output_elems() -> int:
    """Row stride (elements) of mt_infer's output buffer: the widest registered model's output width."""
    v = ctypes.c_int32(0)
    _check(lib().mt_output_elems(ctypes.byref(v)), "mt_output_elems")
    return int(v.value)


def mt_input_elems() -> int:
    """Row stride (elements) of mt_infer's input buffer: the widest registered model's input width."""
    v = ctypes.c_int32(0)
    _check(lib().mt_input_elems(ctypes.byref(v)), "mt_input_elems")
    return int(v.value)


def mt_set_cache_bytes(device_bytes: int) -> None:
    """Switch to a weight cache of this many device bytes (0: every model resident).  Only while no model is registered."""
    _check(lib().mt_set_cache_bytes(int(device_bytes)), "mt_set_cache_bytes")


def mt_prefetch(model_ids, stream=None) -> None:
    """Make these tenants (host ints) resident for work enqueued on `stream` afterwards."""
    ids = np.ascontiguousarray(model_ids, dtype=np.int32)
    _check(lib().mt_prefetch(ids.ctypes.data, int(ids.size), _stream_handle(stream)), "mt_prefetch")


def mt_get_cache_stats(reset: bool = False) -> dict:
    st = CacheStats()
    _check(lib().mt_get_cache_stats(ctypes.byref(st), int(bool(reset))), "mt_get_cache_stats")
    return st.as_dict()


def mt_cache_sim_create(capacity_bytes: int):
    """A stand-alone instance of the cache's policy (host code of the library; needs no GPU).  Returns its handle."""
    h = ctypes.c_void_p()
    _check(lib().mt_cache_sim_create(int(capacity_bytes), ctypes.byref(h)), "mt_cache_sim_create")
    return h


def mt_cache_sim_access(sim, model_id: int, nbytes: int, tick: int):
    """Returns (result, offset, evicted ids): result 0 hit, 1 placed, -1 no room."""
    res, off, n = ctypes.c_int32(0), ctypes.c_int64(0), ctypes.c_int32(0)
    ev = (ctypes.c_int32 * 4096)()
    _check(lib().mt_cache_sim_access(sim, int(model_id), int(nbytes), int(tick), ctypes.byref(res), ctypes.byref(off),
                                     ev, 4096, ctypes.byref(n)), "mt_cache_sim_access")
    return int(res.value), int(off.value), [int(ev[i]) for i in range(min(n.value, 4096))]


def mt_cache_sim_release(sim, model_id: int) -> None:
    _check(lib().mt_cache_sim_release(sim, int(model_id)), "mt_cache_sim_release")


def mt_cache_sim_read(sim, model_id: int) -> None:
    """The batch being prepared reads a resident block."""
    _check(lib().mt_cache_sim_read(sim, int(model_id)), "mt_cache_sim_read")


def mt_cache_sim_batch(sim, finished: bool = False) -> None:
    """The batch being prepared has been enqueued; or all of them are known to have finished."""
    _check(lib().mt_cache_sim_batch(sim, int(bool(finished))), "mt_cache_sim_batch")


def mt_cache_sim_wait(sim) -> int:
    """The batch that what is now written into the arena has to wait for (0: none); asking is waiting."""
    b = ctypes.c_uint64(0)
    _check(lib().mt_cache_sim_wait(sim, ctypes.byref(b)), "mt_cache_sim_wait")
    return int(b.value)


def mt_cache_sim_stats(sim) -> dict:
    st = CacheStats()
    _check(lib().mt_cache_sim_stats(sim, ctypes.byref(st)), "mt_cache_sim_stats")
    return st.as_dict()


def mt_cache_sim_destroy(sim) -> None:
    _check(lib().mt_cache_sim_destroy(sim), "mt_cache_sim_destroy")


def mt_debug_item_cost(k_blocks: int, n_cols: int, rows: int) -> float:
    """Modelled SM cycles of one dense work item (host code only; needs no GPU)."""
    c = ctypes.c_double(0.0)
    _check(lib().mt_debug_item_cost(int(k_blocks), int(n_cols), int(rows), ctypes.byref(c)), "mt_debug_item_cost")
    return float(c.value)


def mt_debug_schedule_balance(layer: int) -> Tuple[float, int, int]:
    """(heaviest CTA's modelled cost / mean, work items, CTAs) of a dense layer of the last mt_infer."""
    r, n, g = ctypes.c_double(0.0), ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().mt_debug_schedule_balance(int(layer), ctypes.byref(r), ctypes.byref(n), ctypes.byref(g)),
           "mt_debug_schedule_balance")
    return float(r.value), int(n.value), int(g.value)


def mt_debug_empty_launches(count: int, stream=None) -> None:
    """Enqueue `count` empty kernels chained like the kernels of the path (to time the launch floor)."""
    _check(lib().mt_debug_empty_launches(int(count), _stream_handle(stream)), "mt_debug_empty_launches")


def mt_debug_set_option(name: str, value: int) -> None:
    """Switch an executor choice ("fused", "pair", "conv_pair", "pool_head") on or off for the calls that follow."""
    _check(lib().mt_debug_set_option(name.encode(), int(value)), "mt_debug_set_option")


def mt_set_kernel_timing(enable) -> None:
    """0/False off, 1/True every kernel, 2 only the grouped layer executors, 3 the same on every fourth call."""
    _check(lib().mt_set_kernel_timing(int(enable)), "mt_set_kernel_timing")


def mt_get_kernel_times() -> List[Tuple[str, float, int]]:
    cap = 16
    names = (ctypes.c_char_p * cap)()
    ms = (ctypes.c_double * cap)()
    cnt = (ctypes.c_int32 * cap)()
    n = ctypes.c_int32(0)
    _check(lib().mt_get_kernel_times(names, ms, cnt, cap, ctypes.byref(n)), "mt_get_kernel_times")
    return [(names[i].decode(), float(ms[i]), int(cnt[i])) for i in range(n.value)]


def mt_bucket_noalloc(model_ids, n: int, n_models: int, counts_out, offsets_out, perm_out, inv_out, stream=None) -> None:
    """Stable bucketing of a batch by model id for callers that must not allocate device memory (allocator
    hooks, frozen-memory serving loops): all six buffers are the caller's device tensors, the scratch is a
    fixed array inside the library.  Limits: n <= 65536, n_models <= 1024 (else MtError MT_ERR_UNSUPPORTED).
    Calls that overlap on the GPU share that scratch and race."""
    _check(lib().mt_bucket_noalloc(_ptr(model_ids), int(n), int(n_models), _ptr(counts_out), _ptr(offsets_out),
                                   _ptr(perm_out), _ptr(inv_out), _stream_handle(stream)), "mt_bucket_noalloc")


# ------------------------------------------------------------------------------------------------
# Operators of language-model tenants.  These take torch tensors on the context's device and read sizes and strides from
# them; a tensor of another type, shape or place is refused here (MT_ERR_INVALID_ARG), sizes are checked by the library.  A
# call's time on the host is the floor of a token step, so the checks are few, flat expressions: 3 to 5 us a call.
# ------------------------------------------------------------------------------------------------
class _Types:
    bf16 = f32 = i32 = i64 = u8 = None


def _types():
    if _Types.bf16 is None:
        import torch
        _Types.f32, _Types.i32, _Types.i64, _Types.u8, _Types.bf16 = torch.float32, torch.int32, torch.int64, torch.uint8, torch.bfloat16
    return _Types


def _refuse(where: str, needs_context: bool = True) -> None:
    raise MtError(9 if needs_context and _device is None else 1, where) from None      # without a context no tensor is in the right place


_MOST = 0x7fffffff       # of sizes: C's int32, which ctypes would cut larger numbers to


def _place(t) -> int:
    """Where the tensors of a cache, a bank or a book of pages have to be: on the context's device.  (They may be put together before there is one, or
    outlive one; each call asks again.)"""
    return t.get_device() if _device is None else _device


def mt_prompt_attention(q, k, v, offsets, out, scale: Optional[float] = None, stream=None) -> None:
    """Causal attention over packed prompts: q bf16 [n, q_heads, dim], k and v [n, kv_heads, dim] (any token and head strides),
    offsets int32 [sequences + 1], out bf16 [n, q_heads, dim] contiguous.  scale: 1 / sqrt(dim) if None."""
    T = _types()
    bf16 = T.bf16
    try:
        n, hq, d = shape = q.shape
        nk, hk, dk = kshape = k.shape
        q0, q1, q2 = q.stride()
        k0, k1, k2 = k.stride()
        v0, v1, v2 = v.stride()
    except ValueError:
        _refuse("mt_prompt_attention")
    if not (q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and out.dtype is bf16 and offsets.dtype is T.i32 and
            q.get_device() == k.get_device() == v.get_device() == out.get_device() == offsets.get_device() == _device and
            nk == n and dk == d and v.shape == kshape and
            out.shape == shape and out.is_contiguous() and offsets.dim() == 1 and offsets.is_contiguous() and offsets.numel() > 0 and
            (n == 0 or q2 == k2 == v2 == 1)):
        _refuse("mt_prompt_attention")
    try:
        desc = _prompt_desc(n, offsets.numel() - 1, hq, hk, d, d ** -0.5 if scale is None else scale, q0, q1, k0, k1, v0, v1)
    except (struct.error, OverflowError, ZeroDivisionError):       # a number that the description does not hold; a head of no elements
        _refuse("mt_prompt_attention")
    code = (_lib or lib()).mt_prompt_attention(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets.data_ptr(), out.data_ptr(),
                                               _stream_handle(stream))
    if code:
        raise MtError(code, "mt_prompt_attention")


class KvCache:
    """The caller's tensors as one 4-bit cache: codes uint8 [pages, kv_heads, page_tokens, dim / 2], params bf16
    [pages, kv_heads, page_tokens, 2] (scale, bias), contiguous.  Keeps them alive; allocates nothing."""

    def __init__(self, k_codes, k_params, v_codes, v_params):
        T, at = _types(), _place(k_codes)
        try:
            pages, heads, page, half = k_codes.shape
        except ValueError:
            _refuse("KvCache", False)
        for c, p in ((k_codes, k_params), (v_codes, v_params)):
            if not (c.dtype is T.u8 and p.dtype is T.bf16 and c.is_cuda and pages <= _MOST and heads <= _MOST and c.get_device() == p.get_device() == at and c.is_contiguous() and p.is_contiguous() and
                    tuple(c.shape) == (pages, heads, page, half) and tuple(p.shape) == (pages, heads, page, 2)):
                _refuse("KvCache", False)
        self.tensors, self.device = (k_codes, k_params, v_codes, v_params), at
        self.heads, self.dim = heads, 2 * half
        self.desc = KvCacheDesc(pages, page, heads, 2 * half, *[x.data_ptr() for x in self.tensors])
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda"):
        """A new cache of zeros."""
        import torch
        t = []
        for _ in range(2):
            t.append(torch.zeros((n_pages, kv_heads, page_tokens, head_dim // 2), dtype=torch.uint8, device=device))
            t.append(torch.zeros((n_pages, kv_heads, page_tokens, 2), dtype=torch.bfloat16, device=device))
        return cls(*t)


def mt_kv_append(cache: KvCache, k, v, slots, stream=None) -> None:
    """Round k and v, bf16 [n, kv_heads, dim] (any token and head strides), to 4 bits and write token i to slot slots[i] (int64 [n])."""
    T = _types()
    try:
        n, h, d = shape = k.shape
        k0, k1, k2 = k.stride()
        v0, v1, v2 = v.stride()
    except ValueError:
        _refuse("mt_kv_append")
    if not (k.dtype is T.bf16 and v.dtype is T.bf16 and slots.dtype is T.i64 and
            k.get_device() == v.get_device() == slots.get_device() == cache.device == _device and
            v.shape == shape and h == cache.heads and d == cache.dim and slots.dim() == 1 and slots.numel() == n and slots.is_contiguous() and
            (n == 0 or k2 == v2 == 1) and n <= _MOST):
        _refuse("mt_kv_append")
    code = (_lib or lib()).mt_kv_append(cache.ref, k.data_ptr(), k0, k1, v.data_ptr(), v0, v1, slots.data_ptr(), n, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_append")


def mt_kv_read(cache: KvCache, slots, k_out, v_out, stream=None) -> None:
    """The cached values of slots (int64 [n]) as bf16 [n, kv_heads, dim]."""
    T = _types()
    try:
        n, h, d = shape = k_out.shape
    except ValueError:
        _refuse("mt_kv_read")
    if not (k_out.dtype is T.bf16 and v_out.dtype is T.bf16 and slots.dtype is T.i64 and slots.dim() == 1 and slots.numel() == n and
            k_out.get_device() == v_out.get_device() == slots.get_device() == cache.device == _device and v_out.shape == shape and h == cache.heads and d == cache.dim and
            k_out.is_contiguous() and v_out.is_contiguous() and slots.is_contiguous() and n <= _MOST):
        _refuse("mt_kv_read")
    code = (_lib or lib()).mt_kv_read(cache.ref, slots.data_ptr(), n, k_out.data_ptr(), v_out.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_read")


def mt_kv_attention(cache: KvCache, q, tables, lengths, out, scale: Optional[float] = None, stream=None) -> None:
    """One new token per sequence over its cached tokens: q bf16 [sequences, q_heads, dim] (any strides), tables int32
    [sequences, width], lengths int32 [sequences], out bf16 like q, contiguous.  scale: 1 / sqrt(dim) if None."""
    T = _types()
    try:
        n, hq, d = shape = q.shape
        q0, q1, q2 = q.stride()
        rows, width = tables.shape
    except ValueError:
        _refuse("mt_kv_attention")
    if not (q.dtype is T.bf16 and out.dtype is T.bf16 and tables.dtype is T.i32 and lengths.dtype is T.i32 and
            q.get_device() == out.get_device() == tables.get_device() == lengths.get_device() == cache.device == _device and d == cache.dim and out.shape == shape and rows == n and lengths.dim() == 1 and
            lengths.numel() == n and out.is_contiguous() and tables.is_contiguous() and lengths.is_contiguous() and (n == 0 or q2 == 1) and
            n <= _MOST and hq <= _MOST and width <= _MOST):
        _refuse("mt_kv_attention")
    code = (_lib or lib()).mt_kv_attention(cache.ref, q.data_ptr(), q0, q1, tables.data_ptr(), width, lengths.data_ptr(), n, hq,
                                           d ** -0.5 if scale is None else scale, out.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_attention")


def mt_quant_packed_bytes(in_features: int, out_features: int, group: int) -> int:
    """Bytes of one tenant's packed weights (host code only; needs no GPU)."""
    b = ctypes.c_size_t(0)
    if not -_MOST <= min(in_features, out_features, group) <= max(in_features, out_features, group) <= _MOST:
        _refuse("mt_quant_packed_bytes", False)
    _check(lib().mt_quant_packed_bytes(int(in_features), int(out_features), int(group), ctypes.byref(b)), "mt_quant_packed_bytes")
    return int(b.value)


def mt_quant_pack(codes, scales, packed, stream=None) -> None:
    """codes uint8 [tenants, out, in / 2], scales bf16 [tenants, out, in / group] -> packed uint8 [tenants, mt_quant_packed_bytes]."""
    T, at = _types(), _place(codes)
    if not (codes.dtype is T.u8 and scales.dtype is T.bf16 and packed.dtype is T.u8 and codes.is_cuda and
            codes.get_device() == scales.get_device() == packed.get_device() == at and
            codes.dim() == 3 and scales.dim() == 3 and codes.shape[:2] == scales.shape[:2] and codes.is_contiguous() and
            scales.is_contiguous() and packed.is_contiguous() and scales.shape[2] > 0 and 2 * codes.shape[2] % scales.shape[2] == 0):
        _refuse("mt_quant_pack", False)
    t, n, half = codes.shape
    group = 2 * half // scales.shape[2]
    if t > _MOST or packed.numel() < t * mt_quant_packed_bytes(2 * half, n, group):
        _refuse("mt_quant_pack", False)
    _check(lib().mt_quant_pack(codes.data_ptr(), scales.data_ptr(), t, 2 * half, n, group, packed.data_ptr(), _stream_handle(stream)), "mt_quant_pack")


class QuantBank:
    """The packed 4-bit weights of several tenants' layer, with an optional fp32 bias [tenants, out].  Packed on `stream`."""

    def __init__(self, codes, scales, bias=None, stream=None):
        import torch
        try:
            t, n, half = codes.shape
        except ValueError:
            _refuse("QuantBank", False)
        k = 2 * half
        if codes.get_device() != _place(codes) or scales.dim() != 3 or scales.shape[2] <= 0 or k % scales.shape[2]:
            _refuse("QuantBank", False)
        group = k // scales.shape[2]
        if bias is not None and not (bias.dtype is torch.float32 and bias.is_cuda and bias.get_device() == codes.get_device() and bias.is_contiguous() and tuple(bias.shape) == (t, n)):
            _refuse("QuantBank", False)
        # (memory of the stream that writes it: the current stream's may still be in use there)
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=codes.device)
        with torch.cuda.stream(stream):
            self.packed = torch.empty((t, mt_quant_packed_bytes(k, n, group)), dtype=torch.uint8, device=codes.device)
        mt_quant_pack(codes, scales, self.packed, stream)
        self.bias, self.in_features, self.out_features, self.device = bias, k, n, codes.get_device()
        self.desc = QuantBankDesc(t, k, n, group, self.packed.data_ptr(), _ptr(bias))
        self.ref = ctypes.byref(self.desc)


def mt_quant_linear(x, ids, bank: QuantBank, y, stream=None) -> None:
    """y[i] = weight[ids[i]] x[i] + bias[ids[i]]: x bf16 [n, in] (any row stride), ids int32 [n], y bf16 or fp32 [n, out]."""
    T = _types()
    try:
        n, k = x.shape
        rows, out = y.shape
        x0, x1 = x.stride()
        y0, y1 = y.stride()
    except ValueError:
        _refuse("mt_quant_linear")
    wide = y.dtype is T.f32
    if not (x.dtype is T.bf16 and ids.dtype is T.i32 and (wide or y.dtype is T.bf16) and
            x.get_device() == ids.get_device() == y.get_device() == bank.device == _device and
            k == bank.in_features and rows == n and out == bank.out_features and ids.dim() == 1 and ids.numel() == n and
            ids.is_contiguous() and (n == 0 or (x1 == 1 and (y1 == 1 or out == 1))) and n <= _MOST):
        _refuse("mt_quant_linear")
    code = (_lib or lib()).mt_quant_linear(bank.ref, x.data_ptr(), x0, ids.data_ptr(), n, y.data_ptr(), y0, 1 if wide else 0, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_quant_linear")


def mt_token_logprobs(logits, tokens, logprobs, entropies=None, top_ids=None, top_logprobs=None, stream=None) -> None:
    """logits bf16 or fp32 [n, vocab] (any row stride), tokens int32 [n] -> logprobs fp32 [n], entropies fp32 [n] (or None),
    top_ids int32 [n, top] and top_logprobs fp32 [n, top] (or None)."""
    T = _types()
    f32, top = T.f32, 0
    try:
        n, vocab = logits.shape
        s0, s1 = logits.stride()
    except ValueError:
        _refuse("mt_token_logprobs")
    wide = logits.dtype is f32
    ok = (wide or logits.dtype is T.bf16) and tokens.dtype is T.i32 and logprobs.dtype is f32 and \
        logits.get_device() == tokens.get_device() == logprobs.get_device() == _device and tokens.dim() == 1 and tokens.numel() == n and logprobs.dim() == 1 and logprobs.numel() == n and \
        tokens.is_contiguous() and logprobs.is_contiguous() and (n == 0 or vocab <= 1 or s1 == 1) and \
        n <= _MOST and vocab <= _MOST
    if entropies is not None:
        ok = ok and entropies.dtype is f32 and entropies.get_device() == _device and entropies.dim() == 1 and entropies.numel() == n and entropies.is_contiguous()
    if ok and (top_ids is not None or top_logprobs is not None):
        ok = top_ids is not None and top_logprobs is not None and top_ids.dtype is T.i32 and top_logprobs.dtype is f32 and \
            top_ids.get_device() == top_logprobs.get_device() == _device and top_ids.dim() == 2 and top_ids.shape[0] == n and \
            top_ids.shape == top_logprobs.shape and top_ids.is_contiguous() and top_logprobs.is_contiguous()
        top = min(top_ids.shape[1], _MOST) if ok else 0
    if not ok:
        _refuse("mt_token_logprobs")
    code = (_lib or lib()).mt_token_logprobs(logits.data_ptr(), 1 if wide else 0, s0, n, vocab, tokens.data_ptr(), top, logprobs.data_ptr(),
                                             None if entropies is None else entropies.data_ptr(), None if top_ids is None else top_ids.data_ptr(),
                                             None if top_logprobs is None else top_logprobs.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_token_logprobs")


def mt_cross_attention(q, k, v, offsets, ranges, out, scale: Optional[float] = None, stream=None) -> None:
    """Attention to an encoder's states: q bf16 [n, q_heads, dim], k and v [states, kv_heads, dim] (any token and head strides), offsets int32
    [sequences + 1] of the queries, ranges int32 [sequences, 2] (first state, end), out bf16 like q, contiguous.  scale: 1 / sqrt(dim) if None."""
    T = _types()
    bf16, i32 = T.bf16, T.i32
    try:
        n, hq, d = shape = q.shape
        m, hk, dk = kshape = k.shape
        q0, q1, q2 = q.stride()
        k0, k1, k2 = k.stride()
        v0, v1, v2 = v.stride()
        seqs, two = ranges.shape
    except ValueError:
        _refuse("mt_cross_attention")
    if not (q.dtype is bf16 and k.dtype is bf16 and v.dtype is bf16 and out.dtype is bf16 and offsets.dtype is i32 and ranges.dtype is i32 and
            q.get_device() == k.get_device() == v.get_device() == out.get_device() == offsets.get_device() == ranges.get_device() == _device and
            dk == d and v.shape == kshape and out.shape == shape and out.is_contiguous() and offsets.dim() == 1 and offsets.is_contiguous() and
            offsets.numel() == seqs + 1 and two == 2 and ranges.is_contiguous() and (n == 0 or q2 == 1) and (m == 0 or k2 == v2 == 1)):
        _refuse("mt_cross_attention")
    if m == 0:
        k0 = v0 = hk * d               # (strides of what holds nothing)
        k1 = v1 = d
    try:
        desc = _cross_desc(n, m, seqs, hq, hk, d, d ** -0.5 if scale is None else scale, q0, q1, k0, k1, v0, v1)
    except (struct.error, OverflowError, ZeroDivisionError):
        _refuse("mt_cross_attention")
    code = (_lib or lib()).mt_cross_attention(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), offsets.data_ptr(), ranges.data_ptr(),
                                              out.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_cross_attention")


def mt_rotate(x, positions, frequencies, out, sections: Optional[Sequence[int]] = None, neighbours: bool = False, inverse: bool = False,
              stream=None) -> None:
    """Rotary positions: x bf16 or fp32 [n, heads, dim] (any token and head strides), positions int32 [n] or [n, axes], frequencies fp32
    [rotary / 2], out like x (or x itself).  sections: pairs of each axis, adding up to rotary / 2 (None: one axis has them all)."""
    T = _types()
    wide = x.dtype is T.f32
    try:
        n, h, d = shape = x.shape
        x0, x1, x2 = x.stride()
        o0, o1, o2 = out.stride()
    except ValueError:
        _refuse("mt_rotate")
    half = frequencies.numel()
    axes = positions.shape[1] if positions.dim() == 2 else 1
    cut = (half,) if sections is None else tuple(sections)
    if not ((wide or x.dtype is T.bf16) and out.dtype is x.dtype and positions.dtype is T.i32 and frequencies.dtype is T.f32 and
            x.get_device() == out.get_device() == positions.get_device() == frequencies.get_device() == _device and out.shape == shape and
            0 < positions.dim() <= 2 and positions.shape[0] == n and positions.is_contiguous() and frequencies.dim() == 1 and
            frequencies.is_contiguous() and len(cut) == axes <= 4 and (n == 0 or d <= 1 or x2 == o2 == 1)):
        _refuse("mt_rotate")
    try:
        desc = _rotate_desc(n, h, d, 2 * half, axes, *cut, *(0,) * (4 - axes), bool(neighbours), bool(inverse), 1 if wide else 0, x0, x1, o0, o1)
    except struct.error:
        _refuse("mt_rotate")
    code = (_lib or lib()).mt_rotate(desc, x.data_ptr(), positions.data_ptr(), frequencies.data_ptr(), out.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_rotate")


class KvPages:
    """The caller's tensors as the book of a cache's pages: refs int32 [pages], tables int32 [rows, width], lengths int32 [rows], contiguous.  Keeps them
    alive; allocates nothing."""

    def __init__(self, refs, tables, lengths, page_tokens: int):
        T, at = _types(), _place(refs)
        if not (refs.dtype is T.i32 and tables.dtype is T.i32 and lengths.dtype is T.i32 and refs.is_cuda and
                refs.get_device() == tables.get_device() == lengths.get_device() == at and refs.dim() == 1 and tables.dim() == 2 and
                lengths.dim() == 1 and lengths.numel() == tables.shape[0] and refs.is_contiguous() and tables.is_contiguous() and
                lengths.is_contiguous() and max(refs.numel(), *tables.shape) <= _MOST and 0 <= page_tokens <= _MOST):
            _refuse("KvPages", False)
        self.refs, self.tables, self.lengths, self.page_tokens, self.device = refs, tables, lengths, page_tokens, at
        self.desc = KvPagesDesc(refs.numel(), page_tokens, *tables.shape, refs.data_ptr(), tables.data_ptr(), lengths.data_ptr())
        self.ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, n_pages: int, page_tokens: int, rows: int, table_width: int, device="cuda"):
        """A new book: every page free, every row without tokens."""
        import torch
        zeros = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
        return cls(zeros(n_pages), zeros(rows, table_width), zeros(rows), page_tokens)


def _is_ints(t, n: int) -> bool:
    return t.dtype is _Types.i32 and t.get_device() == _device and t.shape == (n,) and t.is_contiguous() and n <= _MOST


def _is_copies(t, n: int) -> bool:
    return t.dtype is _Types.i32 and t.get_device() == _device and t.shape == (n, 3) and t.is_contiguous() and n <= _MOST


def mt_kv_reserve(pages: KvPages, rows, counts, slots, stream=None) -> None:
    """Room for counts[i] more tokens in row rows[i] (int32); slots int64 (at least sum(counts)): where they go, for mt_kv_append."""
    T, n, m = _types(), rows.numel(), slots.numel()
    if not (pages.device == _device and _is_ints(rows, n) and _is_ints(counts, n) and slots.dtype is T.i64 and slots.get_device() == _device and slots.shape == (m,) and slots.is_contiguous()):
        _refuse("mt_kv_reserve")
    code = (_lib or lib()).mt_kv_reserve(pages.ref, rows.data_ptr(), counts.data_ptr(), n, slots.data_ptr(), m, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_reserve")


def mt_kv_fork(pages: KvPages, parents, children, copies, stream=None) -> None:
    """Row children[i] becomes what row parents[i] was (int32); copies int32 [n, 3]: what mt_kv_copy has to copy."""
    _types()
    n = parents.numel()
    if not (pages.device == _device and _is_ints(parents, n) and _is_ints(children, n) and _is_copies(copies, n)):
        _refuse("mt_kv_fork")
    code = (_lib or lib()).mt_kv_fork(pages.ref, parents.data_ptr(), children.data_ptr(), n, copies.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_fork")


def mt_kv_release(pages: KvPages, rows, stream=None) -> None:
    """Gives the pages of rows (int32) back; their lengths become 0."""
    _types()
    n = rows.numel()
    if not (pages.device == _device and _is_ints(rows, n)):
        _refuse("mt_kv_release")
    code = (_lib or lib()).mt_kv_release(pages.ref, rows.data_ptr(), n, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_release")


def mt_kv_compact(pages: KvPages, copies, stream=None) -> None:
    """Moves used pages to the front, at most copies.shape[0] of them; copies int32 [n, 3]: what mt_kv_copy has to copy."""
    _types()
    n = copies.numel() // 3
    if not (pages.device == _device and _is_copies(copies, n)):
        _refuse("mt_kv_compact")
    code = (_lib or lib()).mt_kv_compact(pages.ref, copies.data_ptr(), n, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_compact")


class KvCopier:
    """The caches of a model (one a layer, with the same pages) that mt_kv_copy copies in.  Keeps them alive."""

    def __init__(self, caches: Sequence[KvCache]):
        self.caches = list(caches)
        self.array = (ctypes.POINTER(KvCacheDesc) * len(self.caches))(*[ctypes.pointer(c.desc) for c in self.caches])
        self.n = len(self.caches)
        self.devices = {c.device for c in self.caches}


def mt_kv_copy(copier: KvCopier, copies, stream=None) -> None:
    """Copies pages in every cache: copies int32 [n, 3], page from, page to, tokens; -1, -1 is left out."""
    _types()
    n = copies.numel() // 3
    if not (_is_copies(copies, n) and copier.devices <= {_device}):
        _refuse("mt_kv_copy")
    code = (_lib or lib()).mt_kv_copy(copier.array, copier.n, copies.data_ptr(), n, _stream_handle(stream))
    if code:
        raise MtError(code, "mt_kv_copy")


def mt_token_sample(logits, uniform, ids, logprobs=None, temperature=None, top_k=None, top_p=None, min_p=None, stream=None) -> None:
    """logits bf16 or fp32 [n, vocab] (any row stride), uniform fp32 [n] in [0, 1) -> ids int32 [n], logprobs fp32 [n] (or None).  temperature, top_p and
    min_p fp32 [n], top_k int32 [n], or None."""
    T = _types()
    f32 = T.f32
    try:
        n, vocab = logits.shape
        s0, s1 = logits.stride()
    except ValueError:
        _refuse("mt_token_sample")
    wide = logits.dtype is f32
    ok = (wide or logits.dtype is T.bf16) and logits.get_device() == _device and (n == 0 or vocab <= 1 or s1 == 1) and n <= _MOST and vocab <= _MOST and \
        _is_ints(ids, n) and (top_k is None or _is_ints(top_k, n))
    for x in (uniform, logprobs, temperature, top_p, min_p):
        if x is not None:
            ok = ok and x.dtype is f32 and x.get_device() == _device and x.dim() == 1 and x.numel() == n and x.is_contiguous()
    if not ok:
        _refuse("mt_token_sample")
    code = (_lib or lib()).mt_token_sample(logits.data_ptr(), 1 if wide else 0, s0, n, vocab, None if temperature is None else temperature.data_ptr(),
                                           None if top_k is None else top_k.data_ptr(), None if top_p is None else top_p.data_ptr(),
                                           None if min_p is None else min_p.data_ptr(), uniform.data_ptr(), ids.data_ptr(),
                                           None if logprobs is None else logprobs.data_ptr(), _stream_handle(stream))
    if code:
        raise MtError(code, "mt_token_sample")
