"""ctypes binding of libsimsd.so: argument marshalling only.

Every computation runs in the HIP kernels behind the C ABI declared in
include/simsd.h.  torch is used for device memory (tensors, workspace) and for
the current HIP stream handle.  If the shared library is missing this module
raises at load time; there is no fallback path.
"""

from __future__ import annotations

import ctypes
import functools
import operator
import os
import threading
from typing import NamedTuple, Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsimsd.so")

SIMSD_F32, SIMSD_BF16 = 0, 1
STATUS = {0: "SIMSD_OK", 1: "SIMSD_ERR_NULL_POINTER", 2: "SIMSD_ERR_BAD_SHAPE",
          3: "SIMSD_ERR_UNSUPPORTED", 4: "SIMSD_ERR_ALIGNMENT", 5: "SIMSD_ERR_WORKSPACE",
          6: "SIMSD_ERR_INVALID_STEP_MAP", 7: "SIMSD_ERR_HIP"}


class AttnDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("max_ref", ctypes.c_int32),
                ("max_prefix_len", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_pages_per_seq", ctypes.c_int32), ("kv_chunk", ctypes.c_int32),
                ("cache_stride_seq", ctypes.c_int64), ("cache_stride_token", ctypes.c_int64),
                ("cache_stride_head", ctypes.c_int64), ("scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("rope_theta", ctypes.c_float)]


class AcceptDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_ref", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("chunks_per_row", ctypes.c_int32), ("logits_dtype", ctypes.c_int)]


class LmheadDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("max_ref", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("dtype", ctypes.c_int)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("num_tokens", "num_q_heads", "num_kv_heads", "head_dim", "rotary_dim", "interleaved",
                 "batch", "max_kv_len", "page_size", "max_pages_per_seq", "num_pages")] + \
               [("attn_factor", ctypes.c_float)] + \
               [(n, ctypes.c_int64) for n in
                ("q_stride_token", "q_stride_head", "k_stride_token", "k_stride_head",
                 "v_stride_token", "v_stride_head", "q_out_stride_token", "q_out_stride_head",
                 "k_out_stride_token", "k_out_stride_head", "cache_stride_seq",
                 "cache_stride_token", "cache_stride_head")] + [("dtype", ctypes.c_int)]


class ChunkDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("num_tokens", "batch", "num_q_heads", "num_kv_heads", "head_dim", "max_q_len",
                 "max_kv_len", "mask_block", "page_size", "max_pages_per_seq", "kv_chunk")] + \
               [(n, ctypes.c_int64) for n in
                ("cache_stride_seq", "cache_stride_token", "cache_stride_head")] + \
               [("scale", ctypes.c_float), ("dtype", ctypes.c_int)]


class SampleDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("top_k", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("min_p", ctypes.c_float), ("dtype", ctypes.c_int)]


class Fp4Pointers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scales", "v_scales")] + \
               [(n, ctypes.c_int64) for n in
                ("scale_stride_seq", "scale_stride_token", "scale_stride_head")]


class Fp4ValuesDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num", "tokens", "num_kv_heads", "head_dim")] + \
               [(n, ctypes.c_int64) for n in
                ("cache_stride_seq", "cache_stride_token", "cache_stride_head")]


class SimsdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


_lib = None
_P = ctypes.c_void_p
_I32P = ctypes.POINTER(ctypes.c_int32)


def lib() -> ctypes.CDLL:
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        L.simsd_verify_attention_workspace_size.argtypes = [ctypes.POINTER(AttnDesc)]
        L.simsd_verify_attention_workspace_size.restype = ctypes.c_size_t
        L.simsd_verify_accept_workspace_size.argtypes = [ctypes.POINTER(AcceptDesc)]
        L.simsd_verify_accept_workspace_size.restype = ctypes.c_size_t
        L.simsd_verify_attention.argtypes = [ctypes.POINTER(AttnDesc)] + [_P] * 5 + [_P] * 4 + \
            [_P, _P, _P, ctypes.c_size_t, _P]
        L.simsd_verify_attention.restype = ctypes.c_int
        L.simsd_verify_accept.argtypes = [ctypes.POINTER(AcceptDesc)] + [_P] * 8 + \
            [_P, ctypes.c_size_t, _P]
        L.simsd_verify_accept.restype = ctypes.c_int
        L.simsd_verify_accept_noalloc.argtypes = [ctypes.POINTER(AcceptDesc)] + [_P] * 9
        L.simsd_verify_accept_noalloc.restype = ctypes.c_int
        L.simsd_verify_accept_sampled_workspace_size.argtypes = [ctypes.POINTER(AcceptDesc)]
        L.simsd_verify_accept_sampled_workspace_size.restype = ctypes.c_size_t
        L.simsd_verify_accept_sampled.argtypes = [ctypes.POINTER(AcceptDesc), ctypes.c_float] + \
            [_P] * 10 + [_P, ctypes.c_size_t, _P]
        L.simsd_verify_accept_sampled.restype = ctypes.c_int
        L.simsd_verify_accept_lmhead_workspace_size.argtypes = [ctypes.POINTER(LmheadDesc)]
        L.simsd_verify_accept_lmhead_workspace_size.restype = ctypes.c_size_t
        L.simsd_verify_accept_lmhead.argtypes = [ctypes.POINTER(LmheadDesc)] + [_P] * 9 + \
            [_P, ctypes.c_size_t, _P]
        L.simsd_verify_accept_lmhead.restype = ctypes.c_int
        L.simsd_rotary.argtypes = [ctypes.POINTER(RotaryDesc)] + [_P] * 7
        L.simsd_rotary.restype = ctypes.c_int
        L.simsd_rotary_append.argtypes = [ctypes.POINTER(RotaryDesc)] + [_P] * 12
        L.simsd_rotary_append.restype = ctypes.c_int
        L.simsd_rope_frequencies.argtypes = [ctypes.c_int32, ctypes.c_double, ctypes.c_int,
                                             ctypes.c_double, ctypes.c_int32, ctypes.c_double,
                                             ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                             ctypes.POINTER(ctypes.c_float)]
        L.simsd_rope_frequencies.restype = ctypes.c_int
        L.simsd_chunk_attention_workspace_size.argtypes = [ctypes.POINTER(ChunkDesc)]
        L.simsd_chunk_attention_workspace_size.restype = ctypes.c_size_t
        L.simsd_chunk_attention.argtypes = [ctypes.POINTER(ChunkDesc)] + [_P] * 9 + \
            [ctypes.c_size_t, _P]
        L.simsd_chunk_attention.restype = ctypes.c_int
        L.simsd_sample.argtypes = [ctypes.POINTER(SampleDesc)] + [_P] * 10
        L.simsd_sample.restype = ctypes.c_int
        for kind, desc in (("chunk", ChunkDesc), ("verify", AttnDesc)):
            for form in ("window", "fp4"):
                size = getattr(L, f"simsd_{kind}_attention_{form}_workspace_size")
                size.argtypes = [ctypes.POINTER(desc), ctypes.c_int32, ctypes.c_int32]
                size.restype = ctypes.c_size_t
        head = [ctypes.POINTER(ChunkDesc), ctypes.c_int32, ctypes.c_int32, _P]
        tail = [_P] * 6 + [ctypes.c_size_t, _P]
        L.simsd_chunk_attention_window.argtypes = head + [_P, _P] + tail
        L.simsd_chunk_attention_window.restype = ctypes.c_int
        L.simsd_chunk_attention_fp4.argtypes = head + [ctypes.POINTER(Fp4Pointers)] + tail
        L.simsd_chunk_attention_fp4.restype = ctypes.c_int
        head = [ctypes.POINTER(AttnDesc), ctypes.c_int32, ctypes.c_int32, _P, _P, _P]
        tail = [_P] * 7 + [ctypes.c_size_t, _P]
        L.simsd_verify_attention_window.argtypes = head + [_P, _P] + tail
        L.simsd_verify_attention_window.restype = ctypes.c_int
        L.simsd_verify_attention_fp4.argtypes = head + [ctypes.POINTER(Fp4Pointers)] + tail
        L.simsd_verify_attention_fp4.restype = ctypes.c_int
        L.simsd_rotary_append_fp4.argtypes = [ctypes.POINTER(RotaryDesc)] + [_P] * 6 + \
            [ctypes.POINTER(Fp4Pointers)] + [_P] * 4
        L.simsd_rotary_append_fp4.restype = ctypes.c_int
        L.simsd_fp4_values.argtypes = [ctypes.POINTER(Fp4ValuesDesc), ctypes.POINTER(Fp4Pointers),
                                       _P, _P, _P]
        L.simsd_fp4_values.restype = ctypes.c_int
        L.simsd_validate_step_map.argtypes = [_I32P, _I32P, ctypes.c_int32, ctypes.c_int32,
                                              ctypes.c_int32]
        L.simsd_validate_step_map.restype = ctypes.c_int
        L.simsd_status_string.argtypes = [ctypes.c_int]
        L.simsd_status_string.restype = ctypes.c_char_p
        L.simsd_last_error.argtypes = []
        L.simsd_last_error.restype = ctypes.c_char_p
        L.simsd_version.argtypes = []
        L.simsd_version.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise SimsdError(status, lib().simsd_last_error().decode())


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return SIMSD_BF16
    if dt == torch.float32:
        return SIMSD_F32
    raise ValueError(f"unsupported dtype {dt}")


def _stream_of(stream, device: torch.device):
    """The torch stream a call runs on: the given one, else the current stream
    of the tensors' device."""
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream


# ----------------------------------------------------------------------------
# Argument checks.  The C library checks sizes, alignment and the workspace,
# but it only sees pointers: shapes, dtypes, strides and devices of the
# tensors are checked here, before any call, and raise ValueError.
#
# Each call first asks the short tests (_is, _attention_hkv), which only say
# whether everything holds: formatting the messages of tests that pass, and
# walking shapes one by one, took most of a small call's host time.  What they
# do not accept goes through the checks below, which say what is wrong.
# ----------------------------------------------------------------------------
def _need(cond: bool, msg: str):
    if not cond:
        raise ValueError(msg)


def _is(t, shape, dtype, device) -> bool:
    return (t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous())


def _tensor(name: str, t, shape, dtype=None, device=None):
    """t is a contiguous tensor of the given shape (None entries: any size),
    dtype and device."""
    if isinstance(t, torch.Tensor) and _is(t, shape, dtype, device):
        return
    _need(isinstance(t, torch.Tensor), f"{name} must be a torch.Tensor")
    _need(t.dim() == len(shape), f"{name} must have {len(shape)} dimensions, got shape {tuple(t.shape)}")
    for i, n in enumerate(shape):
        _need(n is None or t.shape[i] == n,
              f"{name} has shape {tuple(t.shape)}, expected {tuple('*' if x is None else x for x in shape)}")
    if dtype is not None:
        _need(t.dtype == dtype, f"{name} must be {dtype}, got {t.dtype}")
    if device is not None:
        _need(t.device == device, f"{name} is on {t.device}, expected {device}")
    _need(t.is_contiguous(), f"{name} must be contiguous")


def _int32(name, t, shape, device):
    _tensor(name, t, shape, torch.int32, device)


def _out(name, t, shape, dtype, device):
    if t is not None:
        _tensor(name, t, shape, dtype, device)


def _check_cache(k_cache, v_cache, dtype, device, hkv, d, page_size, max_prefix_len,
                 batch, block_table):
    """k/v caches: same dtype as q, same shape and strides as each other, head
    dim innermost with stride 1 (other strides are passed to the library)."""
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _need(isinstance(t, torch.Tensor) and t.dim() == 4,
              f"{name} must be a 4-D tensor [seq or page, token, Hkv, d]")
        _need(t.dtype == dtype, f"{name} must be {dtype} (the dtype of q), got {t.dtype}")
        _need(t.device == device, f"{name} is on {t.device}, expected {device}")
        _need(t.shape[2] == hkv and t.shape[3] == d,
              f"{name} has shape {tuple(t.shape)}: need [*, *, {hkv}, {d}]")
        _need(t.stride(3) == 1, f"{name} must have a unit stride over the head dimension")
    _need(tuple(k_cache.shape) == tuple(v_cache.shape), "k_cache and v_cache shapes differ")
    _need(k_cache.stride() == v_cache.stride(), "k_cache and v_cache strides differ")
    if page_size > 0:
        _need(k_cache.shape[1] == page_size,
              f"paged cache: dimension 1 is {k_cache.shape[1]}, page_size is {page_size}")
        _need(block_table is not None, "paged cache needs a block_table")
        _int32("block_table", block_table, (batch, None), device)
        _need(block_table.shape[1] * page_size >= max_prefix_len,
              "block_table has too few pages per sequence for max_prefix_len")
    else:
        _need(k_cache.shape[0] == batch,
              f"contiguous cache: dimension 0 is {k_cache.shape[0]}, batch is {batch}")
        _need(k_cache.shape[1] >= max_prefix_len,
              f"contiguous cache holds {k_cache.shape[1]} tokens, max_prefix_len is {max_prefix_len}")


class _Workspaces:
    """Scratch buffers for the workspace argument, one per (device, stream,
    kind), grown on demand.  The library needs no initialised contents.

    Keyed by stream so that calls on different streams never share a buffer
    (they could overlap on the device).  A buffer that is replaced by a larger
    one is kept alive (in ``_retired``) rather than freed: a HIP graph captured
    earlier may still launch kernels on it, and freed memory would be handed
    to other tensors by the caching allocator.  ``clear()`` drops everything
    and is only safe once no captured graph that used these buffers will be
    replayed again."""

    def __init__(self):
        self._bufs = {}
        self._retired = []

    def get(self, device: torch.device, stream_handle: int, kind: str,
            nbytes: int) -> Optional[torch.Tensor]:
        if nbytes == 0:
            return None
        key = (device, int(stream_handle), kind)
        buf = self._bufs.get(key)
        if buf is None or buf.numel() < nbytes:
            if buf is not None:
                self._retired.append(buf)
            buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
            self._bufs[key] = buf
        return buf

    def held(self, device: torch.device, stream_handle: int, kind: str) -> Optional[torch.Tensor]:
        """The buffer held for this stream, whatever its size, or None."""
        return self._bufs.get((device, stream_handle, kind))

    def clear(self):
        self._bufs.clear()
        self._retired.clear()


WORKSPACES = _Workspaces()


def attention_desc(q: torch.Tensor, k_cache: torch.Tensor, *, num_kv_heads: int,
                   block_size: int, max_ref: int, max_prefix_len: int, page_size: int = 0,
                   max_pages_per_seq: int = 0, kv_chunk: int = 0,
                   scale: float = 0.0, rope_theta: float = 0.0) -> AttnDesc:
    """Descriptor for q [batch, B+L, Hq, d] and a cache laid out as
    [batch, cap, Hkv, d] (contiguous) or [pages, page_size, Hkv, d] (paged)."""
    b, n_new, hq, d = q.shape
    st = k_cache.stride()
    return AttnDesc(batch=b, num_q_heads=hq, num_kv_heads=num_kv_heads, head_dim=d,
                    block_size=block_size, max_ref=max_ref, max_prefix_len=max_prefix_len,
                    page_size=page_size, max_pages_per_seq=max_pages_per_seq,
                    kv_chunk=kv_chunk, cache_stride_seq=st[0], cache_stride_token=st[1],
                    cache_stride_head=st[2], scale=scale, dtype=_dtype_code(q.dtype),
                    rope_theta=rope_theta)


def attention_workspace_size(desc: AttnDesc) -> int:
    return int(lib().simsd_verify_attention_workspace_size(ctypes.byref(desc)))


def accept_workspace_size(desc: AcceptDesc) -> int:
    return int(lib().simsd_verify_accept_workspace_size(ctypes.byref(desc)))


def _nbytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def check_attention_tensors(q, k_new, v_new, k_cache, v_cache, block_table, prefix_lens,
                            step_map, num_ref, out, lse, *, block_size: int, max_ref: int,
                            max_prefix_len: int, page_size: int):
    """Shapes, dtypes, devices and layouts of the attention arguments."""
    _need(isinstance(q, torch.Tensor) and q.dim() == 4, "q must be a 4-D tensor [batch, B+L, Hq, d]")
    _need(q.dtype in (torch.bfloat16, torch.float32), f"q must be bfloat16 or float32, got {q.dtype}")
    b, n_new, hq, d = q.shape
    dev = q.device
    _need(n_new == block_size + max_ref, f"q has {n_new} slots, block_size + max_ref is {block_size + max_ref}")
    _tensor("q", q, (b, n_new, hq, d), q.dtype, dev)
    _need(isinstance(k_new, torch.Tensor) and k_new.dim() == 4, "k_new must be a 4-D tensor")
    hkv = k_new.shape[2]
    _tensor("k_new", k_new, (b, n_new, hkv, d), q.dtype, dev)
    _tensor("v_new", v_new, (b, n_new, hkv, d), q.dtype, dev)
    if max_prefix_len > 0:
        _check_cache(k_cache, v_cache, q.dtype, dev, hkv, d, page_size, max_prefix_len, b,
                     block_table)
    _int32("prefix_lens", prefix_lens, (b,), dev)
    _int32("step_map", step_map, (b, block_size), dev)
    _int32("num_ref", num_ref, (b,), dev)
    _out("out", out, (b, n_new, hq, d), q.dtype, dev)
    _out("lse", lse, (b, hq, n_new), torch.float32, dev)
    return hkv


def _attention_hkv(q, k_new, v_new, k_cache, v_cache, block_table, prefix_lens, step_map,
                   num_ref, out, lse, block_size, max_ref, max_prefix_len, page_size):
    """KV heads if every argument passes check_attention_tensors, else None."""
    try:
        b, n_new, hq, d = q.shape
        hkv = k_new.shape[2]
        dt, dev, new = q.dtype, q.device, (b, n_new, hkv, d)
        if not ((dt is torch.bfloat16 or dt is torch.float32) and n_new == block_size + max_ref
                and q.is_contiguous() and _is(k_new, new, dt, dev) and _is(v_new, new, dt, dev)
                and _is(prefix_lens, (b,), torch.int32, dev)
                and _is(step_map, (b, block_size), torch.int32, dev)
                and _is(num_ref, (b,), torch.int32, dev)
                and (out is None or _is(out, q.shape, dt, dev))
                and (lse is None or _is(lse, (b, hq, n_new), torch.float32, dev))):
            return None
        if max_prefix_len > 0:
            shape, stride = k_cache.shape, k_cache.stride()
            if not (k_cache.dtype is dt and v_cache.dtype is dt and k_cache.device == dev
                    and v_cache.device == dev and v_cache.shape == shape
                    and v_cache.stride() == stride and len(shape) == 4 and stride[3] == 1
                    and shape[2] == hkv and shape[3] == d):
                return None
            if page_size > 0:
                pages = block_table.shape
                if not (shape[1] == page_size and len(pages) == 2
                        and _is(block_table, (b, pages[1]), torch.int32, dev)
                        and pages[1] * page_size >= max_prefix_len):
                    return None
            elif not (shape[0] == b and shape[1] >= max_prefix_len):
                return None
        return hkv
    except (AttributeError, TypeError, ValueError, IndexError):
        return None


# The cached descriptors are keyed by plain numbers: a tensor or array given for
# one is read on every call (its content may have changed, and it hashes by
# identity or not at all), and a float is no key for an integer field.
@functools.lru_cache(maxsize=1024)
def _attn_desc(device: torch.device, *fields):
    """AttnDesc of these field values (read only: calls share it) and the
    workspace bytes of its call on `device`."""
    desc = AttnDesc(*fields)
    if device.type != "cuda":
        return desc, attention_workspace_size(desc)
    with torch.cuda.device(device):
        return desc, attention_workspace_size(desc)


@functools.lru_cache(maxsize=1024)
def _accept_desc(*fields) -> AcceptDesc:
    return AcceptDesc(*fields)


@functools.lru_cache(maxsize=1024)
def _lmhead_desc(*fields) -> LmheadDesc:
    return LmheadDesc(*fields)


_NEEDS_WORKSPACE = 5             # SIMSD_ERR_WORKSPACE


def _run(fn, head, args, workspace, device, handle, kind, size_of, desc, nbytes=0):
    """fn(*head, *args, workspace, bytes, stream).  Without a caller's workspace
    the buffer held for this stream is offered, grown to `nbytes` first (the
    attention takes a slower decomposition in a smaller one); the library refuses
    one that is too small before it enqueues anything, and only then is the size
    asked for and the buffer grown."""
    if workspace is not None:
        _tensor("workspace", workspace, (None,), None, device)
        _check(fn(*head, *args, workspace.data_ptr(), _nbytes(workspace), handle))
        return
    buf = WORKSPACES.held(device, handle, kind)
    if nbytes and (buf is None or buf.numel() < nbytes):
        buf = WORKSPACES.get(device, handle, kind, nbytes)
    status = fn(*head, *args, *((None, 0) if buf is None else (buf.data_ptr(), buf.numel())), handle)
    if status == _NEEDS_WORKSPACE:
        buf = WORKSPACES.get(device, handle, kind, size_of(desc))
        status = fn(*head, *args, *((None, 0) if buf is None else (buf.data_ptr(), buf.numel())), handle)
    _check(status)


def verify_attention(q, k_new, v_new, k_cache, v_cache, block_table, prefix_lens, step_map,
                     num_ref, *, block_size: int, max_ref: int, max_prefix_len: int,
                     page_size: int = 0, kv_chunk: int = 0, scale: float = 0.0,
                     rope_theta: float = 0.0,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     want_lse: bool = True, workspace: Optional[torch.Tensor] = None,
                     stream=None, desc: Optional[AttnDesc] = None, window: int = 0, sinks: int = 0):
    """simsd_verify_attention on torch tensors, or with a window
    simsd_verify_attention_window (without `desc`).  Returns (out, lse).

    Raises ValueError on tensors whose shape, dtype, device or layout does not
    match (before anything is launched), SimsdError if the library rejects
    the call."""
    hkv = _attention_hkv(q, k_new, v_new, k_cache, v_cache, block_table, prefix_lens, step_map,
                         num_ref, out, lse, block_size, max_ref, max_prefix_len, page_size)
    if hkv is None:
        hkv = check_attention_tensors(q, k_new, v_new, k_cache, v_cache, block_table, prefix_lens,
                                      step_map, num_ref, out, lse, block_size=block_size,
                                      max_ref=max_ref, max_prefix_len=max_prefix_len,
                                      page_size=page_size)
    if window or sinks:
        if desc is not None:
            _raise("a window and a descriptor of the caller's do not go together")
        st = k_cache.stride()[:3] if max_prefix_len > 0 else (0, 0, 0)
        pages = block_table.shape[1] if max_prefix_len > 0 and page_size > 0 else 0
        return _verify_span("window", q, k_new, v_new, (_addr(k_cache), _addr(v_cache)), st, pages,
                            block_table, prefix_lens, step_map, num_ref, hkv, block_size, max_ref,
                            max_prefix_len, page_size, kv_chunk, scale, rope_theta, window, sinks,
                            out, lse, want_lse, workspace, stream)
    b, n_new, hq, d = q.shape
    dev = q.device
    if desc is None:
        st = (k_cache if max_prefix_len > 0 else k_new).stride()
        pages = block_table.shape[1] if block_table is not None and page_size > 0 else 0
        if not (type(block_size) is type(max_ref) is type(max_prefix_len) is type(page_size)
                is type(kv_chunk) is int and type(scale) is type(rope_theta) is float):
            block_size, max_ref, max_prefix_len, page_size, kv_chunk = map(
                operator.index, (block_size, max_ref, max_prefix_len, page_size, kv_chunk))
            scale, rope_theta = ctypes.c_float(scale).value, ctypes.c_float(rope_theta).value
        desc, nbytes = _attn_desc(dev, b, hq, hkv, d, block_size, max_ref, max_prefix_len,
                                  page_size, pages, kv_chunk, st[0], st[1], st[2], scale,
                                  _dtype_code(q.dtype), rope_theta)
    else:
        nbytes = 0 if workspace is not None else attention_workspace_size(desc)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None and want_lse:
        lse = torch.empty((b, hq, n_new), dtype=torch.float32, device=dev)
    _run(lib().simsd_verify_attention, (ctypes.byref(desc),),
         (q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), _addr(k_cache), _addr(v_cache),
          _addr(block_table), prefix_lens.data_ptr(), step_map.data_ptr(), num_ref.data_ptr(),
          out.data_ptr(), _addr(lse)),
         workspace, dev, _stream_of(stream, dev).cuda_stream, "attn", attention_workspace_size, desc,
         nbytes)
    return out, lse


def accept_desc(logits: torch.Tensor, max_ref: int, chunks_per_row: int = 0) -> AcceptDesc:
    b, B, V = logits.shape
    return AcceptDesc(batch=b, block_size=B, max_ref=max_ref, vocab=V,
                      chunks_per_row=chunks_per_row, logits_dtype=_dtype_code(logits.dtype))


def _check_accept_inputs(logits, draft_ids, step_map, num_ref):
    _need(isinstance(logits, torch.Tensor) and logits.dim() == 3, "logits must be a 3-D tensor [batch, B, V]")
    _need(logits.dtype in (torch.bfloat16, torch.float32),
          f"logits must be bfloat16 or float32, got {logits.dtype}")
    b, B, V = logits.shape
    dev = logits.device
    _tensor("logits", logits, (b, B, V), logits.dtype, dev)
    _need(isinstance(draft_ids, torch.Tensor) and draft_ids.dim() == 2,
          "draft_ids must be a 2-D tensor [batch, L]")
    _int32("draft_ids", draft_ids, (b, None), dev)
    _int32("step_map", step_map, (b, B), dev)
    _int32("num_ref", num_ref, (b,), dev)
    return b, B, V, draft_ids.shape[1], dev


def _accept_inputs(logits, draft_ids, step_map, num_ref):
    """_check_accept_inputs, by the short tests where they hold."""
    try:
        b, B, V = logits.shape
        dt, dev, L = logits.dtype, logits.device, draft_ids.shape[1]
        if ((dt is torch.bfloat16 or dt is torch.float32) and logits.is_contiguous()
                and _is(draft_ids, (b, L), torch.int32, dev)
                and _is(step_map, (b, B), torch.int32, dev) and _is(num_ref, (b,), torch.int32, dev)):
            return b, B, V, L, dev
    except (AttributeError, TypeError, ValueError, IndexError):
        pass
    return _check_accept_inputs(logits, draft_ids, step_map, num_ref)


def _given(name, t, shape, dtype, device):
    """An output: the caller's tensor (checked), or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _tensor(name, t, shape, dtype, device)
    return t


def verify_accept(logits, draft_ids, step_map, num_ref, *, chunks_per_row: int = 0,
                  target_ids=None, confidence=None, draft_prob=None, accept_len=None,
                  workspace=None, stream=None, desc: Optional[AcceptDesc] = None):
    """simsd_verify_accept on torch tensors.
    Returns (target_ids, confidence, draft_prob, accept_len)."""
    b, B, V, L, dev = _accept_inputs(logits, draft_ids, step_map, num_ref)
    target_ids = _given("target_ids", target_ids, (b, B), torch.int32, dev)
    confidence = _given("confidence", confidence, (b, B), torch.float32, dev)
    draft_prob = _given("draft_prob", draft_prob, (b, L), torch.float32, dev)
    accept_len = _given("accept_len", accept_len, (b,), torch.int32, dev)
    if desc is None:
        desc = _accept_desc(b, B, L, V, operator.index(chunks_per_row), _dtype_code(logits.dtype))
    _run(lib().simsd_verify_accept, (ctypes.byref(desc),),
         (logits.data_ptr(), draft_ids.data_ptr(), step_map.data_ptr(), num_ref.data_ptr(),
          target_ids.data_ptr(), confidence.data_ptr(), draft_prob.data_ptr(),
          accept_len.data_ptr()),
         workspace, dev, _stream_of(stream, dev).cuda_stream, "accept", accept_workspace_size, desc)
    return target_ids, confidence, draft_prob, accept_len


NOALLOC_SCRATCH_BYTES = 4 << 20      # SIMSD_NOALLOC_SCRATCH_BYTES


def verify_accept_noalloc(logits, draft_ids, step_map, num_ref, *, target_ids=None,
                          confidence=None, draft_prob=None, accept_len=None, stream=None):
    """simsd_verify_accept_noalloc on torch tensors: the greedy accept with the
    library's fixed per-device scratch instead of a workspace (for callers that
    cannot allocate; pass preallocated outputs to allocate nothing at all).
    Calls overlapping on one GPU race on that scratch.
    Returns (target_ids, confidence, draft_prob, accept_len)."""
    b, B, V, L, dev = _accept_inputs(logits, draft_ids, step_map, num_ref)
    target_ids = _given("target_ids", target_ids, (b, B), torch.int32, dev)
    confidence = _given("confidence", confidence, (b, B), torch.float32, dev)
    draft_prob = _given("draft_prob", draft_prob, (b, L), torch.float32, dev)
    accept_len = _given("accept_len", accept_len, (b,), torch.int32, dev)
    desc = _accept_desc(b, B, L, V, 0, _dtype_code(logits.dtype))
    _check(lib().simsd_verify_accept_noalloc(
        ctypes.byref(desc), logits.data_ptr(), draft_ids.data_ptr(), step_map.data_ptr(),
        num_ref.data_ptr(), target_ids.data_ptr(), confidence.data_ptr(), draft_prob.data_ptr(),
        accept_len.data_ptr(), _stream_of(stream, dev).cuda_stream))
    return target_ids, confidence, draft_prob, accept_len


def accept_sampled_workspace_size(desc: AcceptDesc) -> int:
    return int(lib().simsd_verify_accept_sampled_workspace_size(ctypes.byref(desc)))


def verify_accept_sampled(logits, draft_logits, draft_ids, step_map, num_ref, uniforms, *,
                          temperature: float = 1.0, chunks_per_row: int = 0, p_target=None,
                          p_draft=None, accept_len=None, correction=None, workspace=None,
                          stream=None, desc: Optional[AcceptDesc] = None):
    """simsd_verify_accept_sampled on torch tensors.
    Returns (p_target, p_draft, accept_len, correction)."""
    b, B, V, L, dev = _accept_inputs(logits, draft_ids, step_map, num_ref)
    _tensor("draft_logits", draft_logits, (b, L, V), logits.dtype, dev)
    _tensor("uniforms", uniforms, (b, L + 1), torch.float32, dev)
    p_target = _given("p_target", p_target, (b, L), torch.float32, dev)
    p_draft = _given("p_draft", p_draft, (b, L), torch.float32, dev)
    accept_len = _given("accept_len", accept_len, (b,), torch.int32, dev)
    correction = _given("correction", correction, (b,), torch.int32, dev)
    if desc is None:
        desc = _accept_desc(b, B, L, V, operator.index(chunks_per_row), _dtype_code(logits.dtype))
    _run(lib().simsd_verify_accept_sampled, (ctypes.byref(desc), ctypes.c_float(temperature)),
         (logits.data_ptr(), draft_logits.data_ptr(), draft_ids.data_ptr(), step_map.data_ptr(),
          num_ref.data_ptr(), uniforms.data_ptr(), p_target.data_ptr(), p_draft.data_ptr(),
          accept_len.data_ptr(), correction.data_ptr()),
         workspace, dev, _stream_of(stream, dev).cuda_stream, "accept_sampled",
         accept_sampled_workspace_size, desc)
    return p_target, p_draft, accept_len, correction


def lmhead_desc(hidden: torch.Tensor, weight: torch.Tensor, max_ref: int) -> LmheadDesc:
    b, B, H = hidden.shape
    return LmheadDesc(batch=b, block_size=B, max_ref=max_ref, vocab=weight.shape[0], hidden=H,
                      dtype=_dtype_code(hidden.dtype))


def lmhead_workspace_size(desc: LmheadDesc) -> int:
    return int(lib().simsd_verify_accept_lmhead_workspace_size(ctypes.byref(desc)))


def _check_lmhead_inputs(hidden, weight, draft_ids, step_map, num_ref):
    _need(isinstance(hidden, torch.Tensor) and hidden.dim() == 3,
          "hidden must be a 3-D tensor [batch, B, H]")
    b, B, H = hidden.shape
    dev = hidden.device
    _tensor("hidden", hidden, (b, B, H), torch.bfloat16, dev)
    _need(isinstance(weight, torch.Tensor) and weight.dim() == 2, "weight must be a 2-D tensor [V, H]")
    _tensor("weight", weight, (None, H), torch.bfloat16, dev)
    V = weight.shape[0]
    _need(isinstance(draft_ids, torch.Tensor) and draft_ids.dim() == 2,
          "draft_ids must be a 2-D tensor [batch, L]")
    _int32("draft_ids", draft_ids, (b, None), dev)
    _int32("step_map", step_map, (b, B), dev)
    _int32("num_ref", num_ref, (b,), dev)
    return b, B, H, V, draft_ids.shape[1], dev


def _lmhead_inputs(hidden, weight, draft_ids, step_map, num_ref):
    """_check_lmhead_inputs, by the short tests where they hold."""
    try:
        b, B, H = hidden.shape
        V, L, dev = weight.shape[0], draft_ids.shape[1], hidden.device
        if (_is(hidden, (b, B, H), torch.bfloat16, dev) and _is(weight, (V, H), torch.bfloat16, dev)
                and _is(draft_ids, (b, L), torch.int32, dev)
                and _is(step_map, (b, B), torch.int32, dev) and _is(num_ref, (b,), torch.int32, dev)):
            return b, B, H, V, L, dev
    except (AttributeError, TypeError, ValueError, IndexError):
        pass
    return _check_lmhead_inputs(hidden, weight, draft_ids, step_map, num_ref)


def verify_accept_lmhead(hidden, weight, draft_ids, step_map, num_ref, *, target_ids=None,
                         confidence=None, draft_prob=None, accept_len=None, workspace=None,
                         stream=None, desc: Optional[LmheadDesc] = None):
    """simsd_verify_accept_lmhead on torch tensors (hidden [b, B, H], weight [V, H]).
    Returns (target_ids, confidence, draft_prob, accept_len)."""
    b, B, H, V, L, dev = _lmhead_inputs(hidden, weight, draft_ids, step_map, num_ref)
    target_ids = _given("target_ids", target_ids, (b, B), torch.int32, dev)
    confidence = _given("confidence", confidence, (b, B), torch.float32, dev)
    draft_prob = _given("draft_prob", draft_prob, (b, L), torch.float32, dev)
    accept_len = _given("accept_len", accept_len, (b,), torch.int32, dev)
    if desc is None:
        desc = _lmhead_desc(b, B, L, V, H, _dtype_code(hidden.dtype))
    _run(lib().simsd_verify_accept_lmhead, (ctypes.byref(desc),),
         (hidden.data_ptr(), weight.data_ptr(), draft_ids.data_ptr(), step_map.data_ptr(),
          num_ref.data_ptr(), target_ids.data_ptr(), confidence.data_ptr(), draft_prob.data_ptr(),
          accept_len.data_ptr()),
         workspace, dev, _stream_of(stream, dev).cuda_stream, "lmhead", lmhead_workspace_size, desc)
    return target_ids, confidence, draft_prob, accept_len


def validate_step_map(step_map, num_ref, max_ref: int):
    """Host-side step-map check (simsd_validate_step_map); raises SimsdError."""
    import numpy as np
    sm = np.ascontiguousarray(step_map, dtype=np.int32)
    nr = np.ascontiguousarray(num_ref, dtype=np.int32)
    _check(lib().simsd_validate_step_map(sm.ctypes.data_as(_I32P), nr.ctypes.data_as(_I32P),
                                         sm.shape[0], sm.shape[1], max_ref))


# ----------------------------------------------------------------------------
# Operators beside the verification step: rotary positions and the write into
# the cache, sampling.  Their tests format no message for arguments that pass.
# New outputs are allocated on the call's stream.
# ----------------------------------------------------------------------------
def _raise(msg: str):
    raise ValueError(msg)


# The current stream's handle without the Stream object around it, where torch has
# the call (2 us of a small call's 15).
_current_handle = getattr(torch._C, "_cuda_getCurrentRawStream",
                          lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Launch:
    """Where a call runs: `handle` is the stream's, and inside the context the
    tensors' device and (when the caller gave one) the stream are current, for
    the launch and for new outputs."""

    def __init__(self, device: torch.device, stream):
        if device.type != "cuda":
            _raise(f"tensors must be on a GPU, got {device}")
        self._contexts = []
        if stream is not None:
            if stream.device != device:
                _raise(f"stream is on {stream.device}, tensors are on {device}")
            self.handle = stream.cuda_stream
            if stream != torch.cuda.current_stream(device):
                self._contexts.append(torch.cuda.stream(stream))
        else:
            self.handle = _current_handle(device.index)
        if torch.cuda.current_device() != device.index:
            self._contexts.append(torch.cuda.device(device))

    def __enter__(self):
        for c in self._contexts:
            c.__enter__()
        return self

    def __exit__(self, *exc):
        for c in reversed(self._contexts):
            c.__exit__(*exc)


def _heads(name: str, t, shape, dtype, device):
    """t is [tokens, heads, d] of this shape, dtype and device with a unit
    stride over d; returns its (token, head) strides (0 where there is one)."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        _raise(f"{name} must be a 3-D tensor [tokens, heads, d]")
    if t.shape != shape:
        _raise(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        _raise(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        _raise(f"{name} is on {t.device}, expected {device}")
    st = t.stride()
    if st[2] != 1:
        _raise(f"{name} must have a unit stride over the head dimension")
    return (st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0)


def _vector(name: str, t, n: int, dtype, device):
    if not (isinstance(t, torch.Tensor) and _is(t, (n,), dtype, device)):
        _tensor(name, t, (n,), dtype, device)


def _in_32_bits(name: str, x: int) -> int:
    if not -2 ** 31 <= x < 2 ** 31:
        _raise(f"{name} = {x} does not fit 32 bits")
    return x


def _filled(kind, fields):
    """A descriptor of these values.  ctypes drops the upper bits of an integer that
    its field does not hold: such a value would be taken for another one."""
    if not (min(fields) >= -2 ** 31 and max(fields) < 2 ** 31):   # (a wide stride, a NaN or a number too large)
        for (name, field), x in zip(kind._fields_, fields):
            if field is ctypes.c_int32:
                _in_32_bits(name, x)
    return kind(*fields)


@functools.lru_cache(maxsize=1024)
def _rotary_desc(*fields) -> RotaryDesc:
    return _filled(RotaryDesc, fields)


def _rotary_parts(q, k, freq):
    """Tokens, (Hq, Hkv), d, dtype and device of a rotary call's inputs, and
    the rotary dims its frequencies turn."""
    x = q if q is not None else k
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        _raise("q (or k) must be a 3-D tensor [tokens, heads, d]")
    if x.dtype is not torch.bfloat16 and x.dtype is not torch.float32:
        _raise(f"q and k must be bfloat16 or float32, got {x.dtype}")
    if not isinstance(freq, torch.Tensor) or freq.dim() != 1:
        _raise("freq must be a 1-D tensor [rotary_dim / 2]")
    _vector("freq", freq, freq.shape[0], torch.float64, x.device)
    return x.shape[0], x.shape[2], x.dtype, x.device, 2 * freq.shape[0]


def rope_frequencies(rotary_dim: int, theta: float, *, scaling: str = "none", factor: float = 1.0,
                     original_context: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                     device="cuda"):
    """simsd_rope_frequencies: (freq, attn_factor) for rotary and rotary_append,
    freq a float64 tensor [rotary_dim / 2] on `device`.  scaling is "none",
    "linear", "ntk" or "yarn"."""
    kinds = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
    if scaling not in kinds:
        _raise(f"scaling must be one of {sorted(kinds)}, got {scaling!r}")
    n = _in_32_bits("rotary_dim", operator.index(rotary_dim))
    context = _in_32_bits("original_context", operator.index(original_context))
    freq = torch.empty(max(n, 2) // 2, dtype=torch.float64)
    attn_factor = ctypes.c_float()
    _check(lib().simsd_rope_frequencies(
        n, theta, kinds[scaling], factor, context, beta_fast, beta_slow,
        ctypes.cast(freq.data_ptr(), ctypes.POINTER(ctypes.c_double)), ctypes.byref(attn_factor)))
    return freq.to(device), attn_factor.value


def rotary(q, k, positions, freq, *, interleaved: bool = False, attn_factor: float = 1.0,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """simsd_rotary on torch tensors: q [tokens, Hq, d] and k [tokens, Hkv, d]
    (either may be None) turned by positions [tokens] (int32), freq as from
    rope_frequencies.  Inputs and outputs may be strided over tokens and heads;
    q_out=q or k_out=k turns in place.  Returns (q_out, k_out)."""
    T, d, dt, dev, rot = _rotary_parts(q, k, freq)
    strides = []
    heads = []
    outs = []
    for name, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            if out is not None:
                _raise(f"{name}_out without {name}")
            strides += [0, 0, 0, 0]
            heads.append(0)
            outs.append(None)
            continue
        if not isinstance(x, torch.Tensor) or x.dim() != 3:
            _raise(f"{name} must be a 3-D tensor [tokens, heads, d]")
        shape = (T, x.shape[1], d)
        strides += _heads(name, x, shape, dt, dev)
        heads.append(shape[1])
        strides += _heads(name + "_out", out, shape, dt, dev) if out is not None else \
            (shape[1] * d if T > 1 else 0, d if shape[1] > 1 else 0)
        outs.append(out)
    _vector("positions", positions, T, torch.int32, dev)
    with _Launch(dev, stream) as at:
        for i, x in enumerate((q, k)):
            if x is not None and outs[i] is None:
                outs[i] = torch.empty_like(x, memory_format=torch.contiguous_format)
        qs, ks = strides[:4], strides[4:]
        desc = _rotary_desc(T, heads[0], heads[1], d, rot, int(bool(interleaved)), 0, 0, 0, 0, 0,
                            float(attn_factor), qs[0], qs[1], ks[0], ks[1], 0, 0, qs[2], qs[3],
                            ks[2], ks[3], 0, 0, 0, _dtype_code(dt))
        _check(lib().simsd_rotary(ctypes.byref(desc), _addr(q), _addr(k), positions.data_ptr(),
                                  freq.data_ptr(), _addr(outs[0]), _addr(outs[1]), at.handle))
    return outs[0], outs[1]


def _ragged(q_starts, kv_lens, device) -> int:
    """Sequences of a ragged batch: q_starts [batch + 1], kv_lens [batch]."""
    if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1 or kv_lens.shape[0] < 1:
        _raise("kv_lens must be a 1-D tensor [batch]")
    b = kv_lens.shape[0]
    _vector("kv_lens", kv_lens, b, torch.int32, device)
    _vector("q_starts", q_starts, b + 1, torch.int32, device)
    return b


def _cache_strides(k_cache, v_cache, dtype, device, hkv, d, page_size, max_kv_len, batch,
                   block_table):
    """Strides and pages per sequence of a call's cache, which passes _check_cache."""
    if max_kv_len <= 0:
        return (0, 0, 0), 0
    try:
        shape, st = k_cache.shape, k_cache.stride()
        ok = (k_cache.dtype is dtype and v_cache.dtype is dtype and k_cache.device == device
              and v_cache.device == device and v_cache.shape == shape and v_cache.stride() == st
              and len(shape) == 4 and st[3] == 1 and shape[2] == hkv and shape[3] == d)
        if ok and page_size > 0:
            pages = block_table.shape[1]
            if (shape[1] == page_size and _is(block_table, (batch, pages), torch.int32, device)
                    and pages * page_size >= max_kv_len):
                return st[:3], pages
        elif ok and shape[0] == batch and shape[1] >= max_kv_len:
            return st[:3], 0
    except (AttributeError, TypeError, ValueError, IndexError):
        pass
    _check_cache(k_cache, v_cache, dtype, device, hkv, d, page_size, max_kv_len, batch, block_table)
    return k_cache.stride()[:3], block_table.shape[1] if page_size > 0 else 0


def rotary_append(q, k, v, k_cache, v_cache, block_table, q_starts, kv_lens, freq, *,
                  max_kv_len: int, page_size: int = 0, positions=None, interleaved: bool = False,
                  attn_factor: float = 1.0, q_out: Optional[torch.Tensor] = None, stream=None):
    """simsd_rotary_append on torch tensors: turns q [tokens, Hq, d] (may be
    None) into q_out and writes the turned k and v [tokens, Hkv, d] to the cache
    rows of the last q_starts[b+1] - q_starts[b] of each sequence's kv_lens[b]
    tokens.  Returns q_out (None without q); rows outside q_starts' range are
    left as they were."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        _raise("k must be a 3-D tensor [tokens, Hkv, d]")
    T, d, dt, dev, rot = _rotary_parts(k, None, freq)
    hkv, hq = k.shape[1], 0
    qs, qo = (0, 0), (0, 0)
    if q is not None:
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            _raise("q must be a 3-D tensor [tokens, Hq, d]")
        hq = q.shape[1]
        qs = _heads("q", q, (T, hq, d), dt, dev)
        qo = (hq * d if T > 1 else 0, d if hq > 1 else 0) if q_out is None else \
            _heads("q_out", q_out, (T, hq, d), dt, dev)
    elif q_out is not None:
        _raise("q_out without q")
    ks, vs = _heads("k", k, (T, hkv, d), dt, dev), _heads("v", v, (T, hkv, d), dt, dev)
    b = _ragged(q_starts, kv_lens, dev)
    page_size, max_kv_len = operator.index(page_size), operator.index(max_kv_len)
    cs, pages = _cache_strides(k_cache, v_cache, dt, dev, hkv, d, page_size, max_kv_len, b, block_table)
    if max_kv_len > 0 and any(n > 1 and st == 0 for n, st in zip(k_cache.shape, k_cache.stride())):
        _raise("the cache must not be an expanded tensor: its rows are written")
    if positions is not None:
        _vector("positions", positions, T, torch.int32, dev)
    with _Launch(dev, stream) as at:
        if q is not None and q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        desc = _rotary_desc(T, hq, hkv, d, rot, int(bool(interleaved)), b, max_kv_len, page_size, pages,
                            k_cache.shape[0] if pages else 0, float(attn_factor), qs[0], qs[1],
                            ks[0], ks[1], vs[0], vs[1], qo[0], qo[1], 0, 0, cs[0], cs[1], cs[2],
                            _dtype_code(dt))
        _check(lib().simsd_rotary_append(
            ctypes.byref(desc), _addr(q), k.data_ptr(), v.data_ptr(), _addr(positions),
            freq.data_ptr(), _addr(q_out), _addr(k_cache), _addr(v_cache),
            _addr(block_table if pages else None), q_starts.data_ptr(), kv_lens.data_ptr(), at.handle))
    return q_out


# Host threads that call on one stream share its buffer: the two kernels of a call are
# enqueued with no other call's between them.  (A ctypes call releases the interpreter's
# own lock.)
_chunk_order = threading.Lock()


def chunk_workspace_size(desc: ChunkDesc) -> int:
    return int(lib().simsd_chunk_attention_workspace_size(ctypes.byref(desc)))


@functools.lru_cache(maxsize=1024)
def _chunk_desc(device: torch.device, *fields):
    """ChunkDesc of these field values (read only: calls share it) and the
    workspace bytes of its call on `device`, which is current."""
    desc = _filled(ChunkDesc, fields)
    if desc.scale == 0.0 and fields[-2] != 0.0:
        _raise(f"scale = {fields[-2]} is 0 in fp32, which stands for 1/sqrt(head_dim)")
    return desc, chunk_workspace_size(desc)


def chunk_attention(q, k_cache, v_cache, block_table, q_starts, kv_lens, *, max_q_len: int,
                    max_kv_len: int, page_size: int = 0, mask_block: int = 1, kv_chunk: int = 0,
                    scale: float = 0.0, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                    workspace: Optional[torch.Tensor] = None, stream=None, window: int = 0,
                    sinks: int = 0):
    """simsd_chunk_attention on torch tensors: q [tokens, Hq, d], contiguous, the
    new tokens of a ragged batch, over a cache that holds their keys and values.
    Returns (out [tokens, Hq, d], lse [Hq, tokens] or None); rows outside
    q_starts' range are left as they were.  With a window it is
    simsd_chunk_attention_window: a token sees its mask's block, the window - 1
    keys before that and the first `sinks` keys.

    Without a caller's workspace a call takes the buffer held for its stream; one
    that is captured into a graph takes memory of that graph's own."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        _raise("q must be a 3-D tensor [tokens, Hq, d]")
    (T, hq, d), dt, dev = q.shape, q.dtype, q.device
    if dt is not torch.bfloat16 and dt is not torch.float32:
        _raise(f"q must be bfloat16 or float32, got {dt}")
    if not q.is_contiguous():
        _raise("q must be contiguous")
    b = _ragged(q_starts, kv_lens, dev)
    max_q_len, max_kv_len, page_size, mask_block, kv_chunk = map(
        operator.index, (max_q_len, max_kv_len, page_size, mask_block, kv_chunk))
    if max_kv_len > 0:
        if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
            _raise("k_cache must be a 4-D tensor [seq or page, token, Hkv, d]")
        hkv = k_cache.shape[2]
    else:
        hkv = hq
    cs, pages = _cache_strides(k_cache, v_cache, dt, dev, hkv, d, page_size, max_kv_len, b, block_table)
    if window or sinks:
        return _chunk_span("window", q, (_addr(k_cache), _addr(v_cache)), cs, pages, block_table, q_starts,
                           kv_lens, b, hkv, max_q_len, max_kv_len, page_size, mask_block, kv_chunk, scale,
                           window, sinks, out, lse, want_lse, workspace, stream)
    if out is not None:
        _tensor("out", out, (T, hq, d), dt, dev)
    if lse is not None:
        _tensor("lse", lse, (hq, T), torch.float32, dev)
    with _Launch(dev, stream) as at:
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            lse = torch.empty((hq, T), dtype=torch.float32, device=dev)
        desc, nbytes = _chunk_desc(dev, T, b, hq, hkv, d, max_q_len, max_kv_len, mask_block, page_size,
                                   pages, kv_chunk, cs[0], cs[1], cs[2], float(scale), _dtype_code(dt))
        if workspace is not None:
            _tensor("workspace", workspace, (None,), None, dev)
        elif nbytes:
            if torch.cuda.is_current_stream_capturing():
                workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            else:
                workspace = WORKSPACES.get(dev, at.handle, "chunk", nbytes)
        with _chunk_order:
            _check(lib().simsd_chunk_attention(
                ctypes.byref(desc), q.data_ptr(), _addr(k_cache), _addr(v_cache),
                _addr(block_table if pages else None), q_starts.data_ptr(), kv_lens.data_ptr(),
                out.data_ptr(), _addr(lse), _addr(workspace), _nbytes(workspace), at.handle))
    return out, lse


# ----------------------------------------------------------------------------
# A sliding window with sinks, and a cache held in 4 bits
# ----------------------------------------------------------------------------
class Fp4Cache(NamedTuple):
    """Keys and values in 4 bits: codes [seq or page, token, Hkv, d / 2] and scales
    [seq or page, token, Hkv, d / 32], uint8 (the form is simsd_fp4_cache's)."""

    k: torch.Tensor
    v: torch.Tensor
    k_scales: torch.Tensor
    v_scales: torch.Tensor


def fp4_cache(num: int, tokens: int, num_kv_heads: int, head_dim: int, *, device="cuda") -> Fp4Cache:
    """A cache of zeros for `num` sequences (or pages) of `tokens` tokens.  A head's
    tokens lie next to each other, so that a head is read without its neighbours."""
    if head_dim not in (64, 128):
        _raise(f"head_dim must be 64 or 128, got {head_dim}")

    def part(width):
        return torch.zeros((num, num_kv_heads, tokens, width), dtype=torch.uint8, device=device).transpose(1, 2)

    return Fp4Cache(part(head_dim // 2), part(head_dim // 2), part(head_dim // 32), part(head_dim // 32))


def _fp4_short(cache, device):
    """Shape and strides of a cache's codes and strides of its scales if everything that
    _fp4_parts checks holds, else None."""
    try:
        k, v, ks, vs = cache
        shape, st, ss = k.shape, k.stride(), ks.stride()
        n, tokens, hkv, half = shape
        small = (n, tokens, hkv, half // 16)
        if (k.dtype is v.dtype is ks.dtype is vs.dtype is torch.uint8 and v.shape == shape
                and v.stride() == st and vs.stride() == ss and ks.shape == small and vs.shape == small
                and st[3] == ss[3] == 1 and half % 16 == 0 and k.device == device and v.device == device
                and ks.device == device and vs.device == device):
            return shape, st, ss
    except (AttributeError, TypeError, ValueError, IndexError):
        pass
    return None


def _fp4_parts(cache, device, width: int = 0):
    """Shape and strides of a cache's codes and strides of its scales, which pass the
    checks here."""
    found = _fp4_short(cache, device)
    if found is not None and isinstance(cache, tuple) and width in (0, 2 * found[0][3]):
        return found
    if not isinstance(cache, tuple) or len(cache) != 4:
        _raise("cache must be an Fp4Cache (codes and scales of keys and values)")
    for name, t in zip(Fp4Cache._fields, cache):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            _raise(f"cache.{name} must be a 4-D tensor [seq or page, token, Hkv, *]")
        if t.dtype is not torch.uint8:
            _raise(f"cache.{name} must be uint8, got {t.dtype}")
        if t.device != device:
            _raise(f"cache.{name} is on {t.device}, expected {device}")
        if t.stride(3) != 1:
            _raise(f"cache.{name} must have a unit stride over the head dimension")
    k, v, ks, vs = cache
    if k.shape != v.shape or k.stride() != v.stride():
        _raise("shapes or strides of the keys' and values' codes differ")
    if ks.shape != vs.shape or ks.stride() != vs.stride():
        _raise("shapes or strides of the keys' and values' scales differ")
    n, tokens, hkv, half = k.shape
    if half % 16 or (width and half != width // 2):
        _raise(f"the codes hold heads of {2 * half} dims" + (f", expected {width}" if width else ": need a multiple of 32"))
    if ks.shape != (n, tokens, hkv, half // 16):
        _raise(f"the scales have shape {tuple(ks.shape)}, expected {(n, tokens, hkv, half // 16)}")
    return k.shape, k.stride(), ks.stride()


def _fp4_pointers(cache: Fp4Cache, ss):
    k, v, ks, vs = cache
    return Fp4Pointers(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), ss[0], ss[1], ss[2])


def _fp4_call(cache, device, d, page_size, max_len, batch, block_table):
    """KV heads, pointers, strides and pages per sequence of a call's 4-bit cache, and
    whether its rows lie apart."""
    if max_len <= 0:
        return None, Fp4Pointers(), (0, 0, 0), 0, True
    (n, tokens, hkv, _), st, ss = _fp4_parts(cache, device, d)
    pages = 0
    if page_size > 0:
        if tokens != page_size:
            _raise(f"paged cache: dimension 1 is {tokens}, page_size is {page_size}")
        if block_table is None:
            _raise("paged cache needs a block_table")
        _int32("block_table", block_table, (batch, None), device)
        pages = block_table.shape[1]
        if pages * page_size < max_len:
            _raise("block_table has too few pages per sequence")
    else:
        if n != batch:
            _raise(f"contiguous cache: dimension 0 is {n}, batch is {batch}")
        if tokens < max_len:
            _raise(f"contiguous cache holds {tokens} tokens, need {max_len}")
    apart = not ((n > 1 and not (st[0] and ss[0])) or (tokens > 1 and not (st[1] and ss[1]))
                 or (hkv > 1 and not (st[2] and ss[2])))
    return hkv, _fp4_pointers(cache, ss), st[:3], pages, apart


@functools.lru_cache(maxsize=1024)
def _span_desc(kind, form, device: torch.device, window: int, sinks: int, *fields):
    """Descriptor of these field values (read only: calls share it) and the workspace
    bytes of its call on `device`, which is current."""
    desc = _filled(kind, fields)
    scale = fields[14 if kind is ChunkDesc else 13]
    if desc.scale == 0.0 and scale != 0.0:
        _raise(f"scale = {scale} is 0 in fp32, which stands for 1/sqrt(head_dim)")
    what = "chunk" if kind is ChunkDesc else "verify"
    size = getattr(lib(), f"simsd_{what}_attention_{form}_workspace_size")
    return desc, int(size(ctypes.byref(desc), window, sinks))


def _span_workspace(workspace, nbytes, device, handle):
    """The caller's buffer, the one held for the stream, or (captured into a graph)
    memory of that graph's own."""
    if workspace is not None:
        _tensor("workspace", workspace, (None,), None, device)
        return workspace
    if not nbytes:
        return None
    if torch.cuda.is_current_stream_capturing():
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    return WORKSPACES.get(device, handle, "span", nbytes)


def _window(window, sinks):
    return (_in_32_bits("window", operator.index(window)), _in_32_bits("sinks", operator.index(sinks)))


def _chunk_span(form, q, cache, cs, pages, block_table, q_starts, kv_lens, b, hkv, max_q_len, max_kv_len,
                page_size, mask_block, kv_chunk, scale, window, sinks, out, lse, want_lse, workspace, stream):
    """Chunk attention by the entry of this form ("window" or "fp4"); the arguments of
    chunk_attention are checked, `cache` is what that entry takes for it."""
    (T, hq, d), dt, dev = q.shape, q.dtype, q.device
    window, sinks = _window(window, sinks)
    if out is not None:
        _tensor("out", out, (T, hq, d), dt, dev)
    if lse is not None:
        _tensor("lse", lse, (hq, T), torch.float32, dev)
    with _Launch(dev, stream) as at:
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            lse = torch.empty((hq, T), dtype=torch.float32, device=dev)
        desc, nbytes = _span_desc(ChunkDesc, form, dev, window, sinks, T, b, hq, hkv, d, max_q_len,
                                  max_kv_len, mask_block, page_size, pages, kv_chunk, cs[0], cs[1], cs[2],
                                  float(scale), _dtype_code(dt))
        workspace = _span_workspace(workspace, nbytes, dev, at.handle)
        with _chunk_order:
            _check(getattr(lib(), f"simsd_chunk_attention_{form}")(
                ctypes.byref(desc), window, sinks, q.data_ptr(), *cache, _addr(block_table if pages else None),
                q_starts.data_ptr(), kv_lens.data_ptr(), out.data_ptr(), _addr(lse), _addr(workspace),
                _nbytes(workspace), at.handle))
    return out, lse


def chunk_attention_fp4(q, cache: Optional[Fp4Cache], block_table, q_starts, kv_lens, *, max_q_len: int,
                        max_kv_len: int, page_size: int = 0, mask_block: int = 1, kv_chunk: int = 0,
                        scale: float = 0.0, window: int = 0, sinks: int = 0,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        want_lse: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """simsd_chunk_attention_fp4 on torch tensors: chunk_attention of bf16 queries over
    a 4-bit cache.  Returns (out, lse)."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        _raise("q must be a 3-D tensor [tokens, Hq, d]")
    if q.dtype is not torch.bfloat16:
        _raise(f"q must be bfloat16, got {q.dtype}")
    if not q.is_contiguous():
        _raise("q must be contiguous")
    b = _ragged(q_starts, kv_lens, q.device)
    max_q_len, max_kv_len, page_size, mask_block, kv_chunk = map(
        operator.index, (max_q_len, max_kv_len, page_size, mask_block, kv_chunk))
    hkv, pointers, cs, pages, _ = _fp4_call(cache, q.device, q.shape[2], page_size, max_kv_len, b, block_table)
    return _chunk_span("fp4", q, (ctypes.byref(pointers),), cs, pages, block_table, q_starts, kv_lens, b,
                       q.shape[1] if hkv is None else hkv, max_q_len, max_kv_len, page_size, mask_block,
                       kv_chunk, scale, window, sinks, out, lse, want_lse, workspace, stream)


def _verify_span(form, q, k_new, v_new, cache, cs, pages, block_table, prefix_lens, step_map, num_ref, hkv,
                 block_size, max_ref, max_prefix_len, page_size, kv_chunk, scale, rope_theta, window, sinks,
                 out, lse, want_lse, workspace, stream):
    """Verification attention by the entry of this form ("window" or "fp4"); the tensors
    are checked, `cache` is what that entry takes for it."""
    (b, n_new, hq, d), dt, dev = q.shape, q.dtype, q.device
    window, sinks = _window(window, sinks)
    block_size, max_ref, max_prefix_len, page_size, kv_chunk = map(
        operator.index, (block_size, max_ref, max_prefix_len, page_size, kv_chunk))
    with _Launch(dev, stream) as at:
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            lse = torch.empty((b, hq, n_new), dtype=torch.float32, device=dev)
        desc, nbytes = _span_desc(AttnDesc, form, dev, window, sinks, b, hq, hkv, d, block_size, max_ref,
                                  max_prefix_len, page_size if max_prefix_len > 0 else 0, pages, kv_chunk,
                                  cs[0], cs[1], cs[2], float(scale), _dtype_code(dt), float(rope_theta))
        workspace = _span_workspace(workspace, nbytes, dev, at.handle)
        with _chunk_order:
            _check(getattr(lib(), f"simsd_verify_attention_{form}")(
                ctypes.byref(desc), window, sinks, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), *cache,
                _addr(block_table if pages else None), prefix_lens.data_ptr(), step_map.data_ptr(),
                num_ref.data_ptr(), out.data_ptr(), _addr(lse), _addr(workspace), _nbytes(workspace),
                at.handle))
    return out, lse


def verify_attention_fp4(q, k_new, v_new, cache: Optional[Fp4Cache], block_table, prefix_lens, step_map,
                         num_ref, *, block_size: int, max_ref: int, max_prefix_len: int, page_size: int = 0,
                         kv_chunk: int = 0, scale: float = 0.0, window: int = 0, sinks: int = 0,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         want_lse: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """simsd_verify_attention_fp4 on torch tensors: verify_attention over a 4-bit
    prefix.  Returns (out, lse)."""
    hkv = _attention_hkv(q, k_new, v_new, None, None, block_table, prefix_lens, step_map, num_ref, out, lse,
                         block_size, max_ref, 0, page_size)
    if hkv is None:
        hkv = check_attention_tensors(q, k_new, v_new, None, None, block_table, prefix_lens, step_map, num_ref,
                                      out, lse, block_size=block_size, max_ref=max_ref, max_prefix_len=0,
                                      page_size=page_size)
    b, _, _, d = q.shape
    held, pointers, cs, pages, _ = _fp4_call(cache, q.device, d, operator.index(page_size),
                                          operator.index(max_prefix_len), b, block_table)
    if held is not None and held != hkv:
        _raise(f"the cache has {held} KV heads, k_new has {hkv}")
    return _verify_span("fp4", q, k_new, v_new, (ctypes.byref(pointers),), cs, pages, block_table, prefix_lens,
                        step_map, num_ref, hkv, block_size, max_ref, max_prefix_len, page_size, kv_chunk, scale,
                        0.0, window, sinks, out, lse, want_lse, workspace, stream)


def rotary_append_fp4(q, k, v, cache: Fp4Cache, block_table, q_starts, kv_lens, freq, *, max_kv_len: int,
                      page_size: int = 0, positions=None, interleaved: bool = False, attn_factor: float = 1.0,
                      q_out: Optional[torch.Tensor] = None, stream=None):
    """simsd_rotary_append_fp4 on torch tensors: rotary_append of bf16 heads to a 4-bit
    cache.  Returns q_out (None without q)."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        _raise("k must be a 3-D tensor [tokens, Hkv, d]")
    T, d, dt, dev, rot = _rotary_parts(k, None, freq)
    if dt is not torch.bfloat16:
        _raise(f"q, k and v must be bfloat16, got {dt}")
    hkv, hq = k.shape[1], 0
    qs, qo = (0, 0), (0, 0)
    if q is not None:
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            _raise("q must be a 3-D tensor [tokens, Hq, d]")
        hq = q.shape[1]
        qs = _heads("q", q, (T, hq, d), dt, dev)
        qo = (hq * d if T > 1 else 0, d if hq > 1 else 0) if q_out is None else \
            _heads("q_out", q_out, (T, hq, d), dt, dev)
    elif q_out is not None:
        _raise("q_out without q")
    ks, vs = _heads("k", k, (T, hkv, d), dt, dev), _heads("v", v, (T, hkv, d), dt, dev)
    b = _ragged(q_starts, kv_lens, dev)
    page_size, max_kv_len = operator.index(page_size), operator.index(max_kv_len)
    held, pointers, cs, pages, apart = _fp4_call(cache, dev, d, page_size, max_kv_len, b, block_table)
    if held is not None:
        if held != hkv:
            _raise(f"the cache has {held} KV heads, k has {hkv}")
        if not apart:
            _raise("the cache must not be an expanded tensor: its rows are written")
    if positions is not None:
        _vector("positions", positions, T, torch.int32, dev)
    with _Launch(dev, stream) as at:
        if q is not None and q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        desc = _rotary_desc(T, hq, hkv, d, rot, int(bool(interleaved)), b, max_kv_len, page_size, pages,
                            cache[0].shape[0] if pages else 0, float(attn_factor), qs[0], qs[1],
                            ks[0], ks[1], vs[0], vs[1], qo[0], qo[1], 0, 0, cs[0], cs[1], cs[2],
                            _dtype_code(dt))
        _check(lib().simsd_rotary_append_fp4(
            ctypes.byref(desc), _addr(q), k.data_ptr(), v.data_ptr(), _addr(positions), freq.data_ptr(),
            _addr(q_out), ctypes.byref(pointers), _addr(block_table if pages else None),
            q_starts.data_ptr(), kv_lens.data_ptr(), at.handle))
    return q_out


@functools.lru_cache(maxsize=1024)
def _fp4_values_desc(*fields) -> Fp4ValuesDesc:
    return _filled(Fp4ValuesDesc, fields)


def fp4_values(cache: Fp4Cache, *, k_out: Optional[torch.Tensor] = None,
               v_out: Optional[torch.Tensor] = None, stream=None):
    """simsd_fp4_values: the values of a cache's keys and of its values, (k, v), bf16
    [seq or page, token, Hkv, d], contiguous."""
    if not isinstance(cache, tuple) or len(cache) != 4 or not isinstance(cache[0], torch.Tensor):
        _raise("cache must be an Fp4Cache (codes and scales of keys and values)")
    dev = cache[0].device
    (n, tokens, hkv, half), st, ss = _fp4_parts(cache, dev)
    shape = (n, tokens, hkv, 2 * half)
    for name, out in (("k_out", k_out), ("v_out", v_out)):
        if out is not None:
            _tensor(name, out, shape, torch.bfloat16, dev)
    with _Launch(dev, stream) as at:
        if k_out is None:
            k_out = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        if v_out is None:
            v_out = torch.empty(shape, dtype=torch.bfloat16, device=dev)
        desc = _fp4_values_desc(n, tokens, hkv, 2 * half, st[0], st[1], st[2])
        _check(lib().simsd_fp4_values(ctypes.byref(desc), ctypes.byref(_fp4_pointers(cache, ss)),
                                      k_out.data_ptr(), v_out.data_ptr(), at.handle))
    return k_out, v_out


@functools.lru_cache(maxsize=1024)
def _sample_desc(*fields) -> SampleDesc:
    return _filled(SampleDesc, fields)


def sample(logits, uniforms, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, token=None,
           prob=None, kept=None, stream=None):
    """simsd_sample on torch tensors: one token for each row of logits [rows, V],
    drawn by uniforms [rows] (float32).  temperature, top_p and min_p are numbers
    or float32 tensors [rows], top_k a number or an int32 tensor [rows].
    Returns (token, prob, kept)."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        _raise("logits must be a 2-D tensor [rows, V]")
    dt, dev, (n, V) = logits.dtype, logits.device, logits.shape
    if dt is not torch.bfloat16 and dt is not torch.float32:
        _raise(f"logits must be bfloat16 or float32, got {dt}")
    if not logits.is_contiguous():
        _raise("logits must be contiguous")
    _vector("uniforms", uniforms, n, torch.float32, dev)
    rows = [None] * 4
    numbers = [temperature, top_k, top_p, min_p]
    for i, (name, kind, off) in enumerate((("temperature", torch.float32, 1.0), ("top_k", torch.int32, 0),
                                           ("top_p", torch.float32, 1.0), ("min_p", torch.float32, 0.0))):
        x = numbers[i]
        if isinstance(x, torch.Tensor):
            _vector(name, x, n, kind, dev)
            rows[i], numbers[i] = x, off
        else:
            numbers[i] = operator.index(x) if kind is torch.int32 else float(x)
    with _Launch(dev, stream) as at:
        token = torch.empty_like(uniforms, dtype=torch.int32) if token is None else _given("token", token, (n,), torch.int32, dev)
        prob = torch.empty_like(uniforms) if prob is None else _given("prob", prob, (n,), torch.float32, dev)
        kept = torch.empty_like(token) if kept is None else _given("kept", kept, (n,), torch.int32, dev)
        desc = _sample_desc(n, V, *numbers, _dtype_code(dt))
        _check(lib().simsd_sample(ctypes.byref(desc), logits.data_ptr(), uniforms.data_ptr(),
                                  *map(_addr, rows), token.data_ptr(), prob.data_ptr(),
                                  kept.data_ptr(), at.handle))
    return token, prob, kept
