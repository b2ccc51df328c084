"""Attention and KV-cache operators on torch tensors (the operators of gm.h).

Argument marshalling only, as in :mod:`model`: shapes and dtypes are checked
here, pointers and the stream go to libgm, which checks the rest and enqueues
its kernels.  Nothing synchronises; every call can be captured into a graph.

Tensors are ``[batch, tokens, heads, head_dim]`` of float32, bfloat16 or
float16 on one HIP device.  The channels of a head are contiguous; the base
address and the other strides are multiples of 16 bytes (views of a fused
q | k | v projection will do).  Work runs on ``stream`` (default: the current
stream of the tensors' device), and what a call allocates belongs to it;
tensors made on another stream have to be ready there.  ``out`` may not overlap
an input.  Forward only: results carry no gradient.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct
from typing import Optional, Tuple

import torch

from . import gm

_DTYPES = {torch.float32: gm.GM_DTYPE_F32, torch.bfloat16: gm.GM_DTYPE_BF16,
           torch.float16: gm.GM_DTYPE_F16}


# The arguments as the C structs lay them out, packed in one go: filling nested
# ctypes structures field by field takes longer than a small kernel runs.
_CACHED = struct.Struct("@P4i" + 2 * "P3q" + "P" + "2fP" + "PQ")
_PROMPT = struct.Struct("@7i" + 4 * "P3q" + "2i" + "2fP" + "4P")
_TENSOR = struct.Struct("@P3q")
assert _CACHED.size == ctypes.sizeof(gm.gm_cached_attention)
assert _PROMPT.size == ctypes.sizeof(gm.gm_prompt_attention)
assert _TENSOR.size == ctypes.sizeof(gm.gm_tensor)


def _rows(t: torch.Tensor, name: str, shape, dtype, device) -> Tuple[int, int, int, int]:
    """The fields of a gm_tensor."""
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    batch, token, head, channel = t.stride()
    if channel != 1 and t.numel():
        raise ValueError(f"the channels of {name} must be contiguous")
    return t.data_ptr(), batch, token, head


def _ints(t: Optional[torch.Tensor], name: str, shape: Tuple[int, ...], device,
          dtype=torch.int32) -> int:
    """Address of a small array, 0 for none."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    return t.data_ptr()


def _first(t: torch.Tensor, name: str):
    """(dtype, its gm code, device) of a call, by its first tensor."""
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a HIP device, not {t.device}")
    if t.dim() != 4:
        raise ValueError(f"{name} must be [batch, tokens, heads, head_dim]")
    return t.dtype, code, t.device


# The current stream's handle by device index: torch.cuda.current_stream without the
# Stream object around it, which takes as long to make as half a launch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


@contextlib.contextmanager
def _there(device, stream, *tensors):
    """The device made current and, if one is given, the stream: what a call
    allocates then belongs to it, and the allocator is told that the tensors are
    in use there."""
    if stream is None:
        with torch.cuda.device(device):
            yield
        return
    if stream.device != device:
        raise ValueError(f"the stream must be on {device}, not {stream.device}")
    with torch.cuda.stream(stream):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        yield


def _elsewhere(device, stream) -> bool:
    return stream is not None or device.index != torch.cuda.current_device()


def _tensor(*fields) -> gm.gm_tensor:
    return gm.gm_tensor.from_buffer_copy(_TENSOR.pack(*fields))


def _empty(like: torch.Tensor, shape) -> torch.Tensor:
    """A new contiguous tensor of that shape."""
    if like.shape == shape and like.is_contiguous():
        return torch.empty_like(like)      # (a third faster)
    return torch.empty(shape, dtype=like.dtype, device=like.device)


class KvCache:
    """Keys and values of one layer in 8 or 4 bits, [batch, positions, heads,
    head_dim] (gm_kv_cache: groups of 32 channels share a bfloat16 scale).

    ``max_seq`` positions per sequence; ``masked`` keeps a byte per position
    that says whether it may be attended (``write(mask=...)``).  Positions never
    written read as zeros.
    """

    def __init__(self, batch: int, heads: int, max_seq: int, head_dim: int, bits: int = 8,
                 device="cuda", masked: bool = False):
        if bits not in (8, 4):
            raise ValueError("bits must be 8 or 4")
        if head_dim not in (32, 64, 128):
            raise ValueError("head_dim must be 32, 64 or 128")
        if batch < 1 or heads < 1 or not 1 <= max_seq < (1 << 24) - 64:
            raise ValueError("batch, heads and max_seq must be positive, max_seq below 2^24 - 64")
        self.batch, self.heads, self.max_seq = batch, heads, max_seq
        self.head_dim, self.bits = head_dim, bits
        cap = (max_seq + 63) // 64 * 64
        # codes are stored plus 2^(bits - 1); with scale 0 their value is 0
        shape = (batch, heads, cap, head_dim * bits // 8)
        self.k = torch.zeros(shape, dtype=torch.uint8, device=device)
        self.v = torch.zeros(shape, dtype=torch.uint8, device=device)
        shape = (batch, heads, head_dim // 32, cap)
        self.k_scale = torch.zeros(shape, dtype=torch.bfloat16, device=device)
        self.v_scale = torch.zeros(shape, dtype=torch.bfloat16, device=device)
        self.valid = torch.zeros((batch, cap), dtype=torch.uint8, device=device) if masked else None
        self.device = self.k.device
        self.c = gm.gm_kv_cache(bits, batch, heads, cap, head_dim, self.k.data_ptr(),
                                self.v.data_ptr(), self.k_scale.data_ptr(),
                                self.v_scale.data_ptr(),
                                self.valid.data_ptr() if masked else None)
        self._ref = ctypes.byref(self.c)
        self._workspace = {}      # bytes that attention needs, by dtype and shape of the queries

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self._tensors())

    def _tensors(self):
        return [t for t in (self.k, self.v, self.k_scale, self.v_scale, self.valid)
                if t is not None]

    def write(self, k: torch.Tensor, v: torch.Tensor, start: Optional[torch.Tensor] = None,
              count: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
              stream=None) -> None:
        """Quantise k and v [B, n, heads, head_dim] into positions start[b] + i
        (``start`` int32 [B]; None: 0) of the first B sequences, for i <
        count[b] (``count`` int32 [B]; None: all n).  Positions outside the
        cache are not stored.  ``mask`` int32 [B, n]: 0 hides a position from
        attention (a ``masked`` cache; without it every stored position may be
        attended)."""
        dtype, code, device = _first(k, "k")
        if device != self.device:
            raise ValueError(f"the cache is on {self.device}, the rows on {device}")
        if _elsewhere(device, stream):
            with _there(device, stream, k, v, start, count, mask, *self._tensors()):
                return self.write(k, v, start, count, mask)
        B, n = k.shape[0], k.shape[1]
        if B > self.batch:
            raise ValueError(f"the rows' batch {B} exceeds the cache's {self.batch}")
        shape = (B, n, self.heads, self.head_dim)
        rc = gm.lib().gm_kv_write(
            self._ref, code, B, n, _tensor(*_rows(k, "k", shape, dtype, device)),
            _tensor(*_rows(v, "v", shape, dtype, device)), _ints(start, "start", (B,), device),
            _ints(count, "count", (B,), device), _ints(mask, "mask", (B, n), device),
            _raw_stream(device.index))
        if rc:
            raise gm.GmError(rc, "gm_kv_write")

    def read(self, n: int, start: Optional[torch.Tensor] = None,
             count: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
             out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, batch: Optional[int] = None,
             stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """k and v [B, n, heads, head_dim] of positions start[b] + i as the
        cache holds them, rounded once to ``dtype``; rows at or past count[b]
        and positions outside the cache are zeros.  ``out``: (k, v) to write
        into; ``batch``: the first B sequences (default: all)."""
        if out is not None:
            dtype = out[0].dtype
        code = _DTYPES.get(dtype)
        if code is None:
            raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
        B = self.batch if batch is None else batch
        if not 0 <= B <= self.batch or n < 0:
            raise ValueError("batch must be at most the cache's, and n not negative")
        shape, device = (B, n, self.heads, self.head_dim), self.device
        if device.type != "cuda":
            raise ValueError(f"the cache must be on a HIP device, not {device}")
        if _elsewhere(device, stream):
            with _there(device, stream, start, count, *(out or ()), *self._tensors()):
                return self.read(n, start, count, dtype, out, batch)
        k, v = out if out is not None else (torch.empty(shape, dtype=dtype, device=device),
                                            torch.empty(shape, dtype=dtype, device=device))
        rc = gm.lib().gm_kv_read(
            self._ref, code, B, n, _ints(start, "start", (B,), device),
            _ints(count, "count", (B,), device), _tensor(*_rows(k, "k", shape, dtype, device)),
            _tensor(*_rows(v, "v", shape, dtype, device)), _raw_stream(device.index))
        if rc:
            raise gm.GmError(rc, "gm_kv_read")
        return k, v


def cached_attention(q: torch.Tensor, cache: KvCache, lengths: torch.Tensor, *,
                     softcap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                     scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Attention of the newest tokens q [B, Sq, n_heads, head_dim] over the
    cache, which already holds their keys and values (gm_attention_cached).

    ``lengths`` int32 [B]: positions in use, read on the device; query i of
    sequence b is at position lengths[b] - Sq + i and sees the positions up to
    its own.  ``n_heads`` is a multiple of the cache's heads.  Scores are
    ``scale`` (default 1/sqrt(head_dim)) times q.k, capped as softcap *
    tanh(score / softcap) when softcap > 0, less slopes[h] * distance
    (``slopes`` float32 [n_heads])."""
    dtype, code, device = _first(q, "q")
    shape = q.shape
    B, Sq, H, hd = shape
    if device != cache.device or B > cache.batch or hd != cache.head_dim:
        raise ValueError(f"q must be on the cache's device {cache.device}, with at most its "
                         f"{cache.batch} sequences and its head_dim {cache.head_dim}")
    if lengths is None:
        raise ValueError("lengths is missing")
    if _elsewhere(device, stream):
        with _there(device, stream, q, out, lengths, slopes, *cache._tensors()):
            return cached_attention(q, cache, lengths, softcap=softcap, slopes=slopes, scale=scale,
                                    out=out)
    need = cache._workspace.get((code, B, Sq, H))
    if need is None:
        need = gm.gm_attention_cached_workspace(cache.c, code, B, Sq, H)
        cache._workspace[code, B, Sq, H] = need
    if out is None:
        out = _empty(q, shape)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    a = gm.gm_cached_attention.from_buffer_copy(_CACHED.pack(
        ctypes.addressof(cache.c), code, B, Sq, H, *_rows(q, "q", shape, dtype, device),
        *_rows(out, "out", shape, dtype, device), _ints(lengths, "lengths", (B,), device),
        1.0 / math.sqrt(hd) if scale is None else scale, softcap,
        _ints(slopes, "slopes", (H,), device, torch.float32),
        work.data_ptr() if need else 0, need))
    rc = gm.lib().gm_attention_cached(ctypes.byref(a), _raw_stream(device.index))
    if rc:
        raise gm.GmError(rc, "gm_attention_cached")
    return out


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = False,
              softcap: float = 0.0, slopes: Optional[torch.Tensor] = None,
              key_mask: Optional[torch.Tensor] = None, q_doc: Optional[torch.Tensor] = None,
              k_doc: Optional[torch.Tensor] = None, prefix: Optional[torch.Tensor] = None,
              q_offset: Optional[int] = None, scale: Optional[float] = None,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of q [B, Sq, n_heads, head_dim] over k and v [B, Sk, kv_heads,
    head_dim] (gm_attention).

    Query i is at position i + ``q_offset`` (default Sk - Sq: the queries are
    the last tokens).  It sees key j when ``key_mask`` [B, Sk] is not 0 there,
    ``q_doc`` [B, Sq] equals ``k_doc`` [B, Sk], and, if ``causal``, j is not
    past the query or lies before ``prefix`` [B] (all int32, each optional); a
    query that sees nothing gives zeros.  Scores as in
    :func:`cached_attention`."""
    dtype, code, device = _first(q, "q")
    if k.dim() != 4:
        raise ValueError("k must be [batch, tokens, heads, head_dim]")
    if _elsewhere(device, stream):
        with _there(device, stream, q, k, v, out, slopes, key_mask, q_doc, k_doc, prefix):
            return attention(q, k, v, causal=causal, softcap=softcap, slopes=slopes,
                             key_mask=key_mask, q_doc=q_doc, k_doc=k_doc, prefix=prefix,
                             q_offset=q_offset, scale=scale, out=out)
    shape = q.shape
    B, Sq, H, hd = shape
    _, Sk, Hkv, _ = k.shape
    keys = (B, Sk, Hkv, hd)
    if out is None:
        out = _empty(q, shape)
    a = gm.gm_prompt_attention.from_buffer_copy(_PROMPT.pack(
        code, B, Sq, Sk, H, Hkv, hd, *_rows(q, "q", shape, dtype, device),
        *_rows(k, "k", keys, dtype, device), *_rows(v, "v", keys, dtype, device),
        *_rows(out, "out", shape, dtype, device), bool(causal),
        Sk - Sq if q_offset is None else q_offset, 1.0 / math.sqrt(hd) if scale is None else scale,
        softcap, _ints(slopes, "slopes", (H,), device, torch.float32),
        _ints(key_mask, "key_mask", (B, Sk), device), _ints(q_doc, "q_doc", (B, Sq), device),
        _ints(k_doc, "k_doc", (B, Sk), device), _ints(prefix, "prefix", (B,), device)))
    rc = gm.lib().gm_attention(ctypes.byref(a), _raw_stream(device.index))
    if rc:
        raise gm.GmError(rc, "gm_attention")
    return out
