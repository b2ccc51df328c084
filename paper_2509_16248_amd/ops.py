"""Attention and KV-cache operators on torch tensors (the operators of gm.h).

Argument marshalling only, as in :mod:`model`: shapes and dtypes are checked
here, pointers and the stream go to libgm, which checks the rest and enqueues
its kernels.  Nothing synchronises; every call can be captured into a graph.

Tensors are ``[batch, tokens, heads, head_dim]`` of float32, bfloat16 or
float16 on one HIP device.  The channels of a head are contiguous; the base
address and the other strides are multiples of 16 bytes (views of a fused
q | k | v projection will do).  Work runs on ``stream`` (default: the current
stream of the tensors' device), and what a call allocates belongs to it;
tensors made on another stream have to be ready there.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import gm

_DTYPES = {torch.float32: gm.GM_DTYPE_F32, torch.bfloat16: gm.GM_DTYPE_BF16,
           torch.float16: gm.GM_DTYPE_F16}


def _rows(t: torch.Tensor, name: str, shape: Tuple[int, ...], dtype, device) -> gm.gm_tensor:
    if t.dim() != 4 or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    if t.numel() and t.stride(3) != 1:
        raise ValueError(f"the channels of {name} must be contiguous")
    return gm.gm_tensor(t.data_ptr() or None, t.stride(0), t.stride(1), t.stride(2))


def _ints(t: Optional[torch.Tensor], name: str, shape: Tuple[int, ...], device,
          dtype=torch.int32) -> Optional[int]:
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, not {t.device}")
    return t.data_ptr() or None


def _first(t: torch.Tensor, name: str):
    """(dtype, device) of a call, by its first tensor."""
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a HIP device, not {t.device}")
    return t.dtype, t.device


def _scores(scale: Optional[float], softcap: float, slopes: Optional[torch.Tensor], heads: int,
            head_dim: int, device) -> gm.gm_scores:
    return gm.gm_scores(1.0 / math.sqrt(head_dim) if scale is None else scale, softcap,
                        _ints(slopes, "slopes", (heads,), device, torch.float32))


class _On:
    """The device and the stream of a call, and the tensors it uses."""

    def __init__(self, device, stream):
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream must be on {device}, not {stream.device}")
        self.given = stream is not None
        self.stream = stream if self.given else torch.cuda.current_stream(device)
        self.context = torch.cuda.stream(self.stream)   # also makes its device current

    def __enter__(self):
        self.context.__enter__()
        return self

    def __exit__(self, *exc):
        return self.context.__exit__(*exc)

    def uses(self, *tensors):
        """On a stream given by the caller the allocator has to know that the
        tensors are in use there."""
        if self.given:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.stream)


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
        dtype, device = _first(k, "k")
        B, n = self._shape(k, device)
        shape = (B, n, self.heads, self.head_dim)
        kt, vt = (_rows(t, name, shape, dtype, device) for t, name in ((k, "k"), (v, "v")))
        with _On(device, stream) as on:
            on.uses(k, v, start, count, mask, *self._tensors())
            gm.gm_kv_write(self.c, _DTYPES[dtype], B, n, kt, vt,
                           _ints(start, "start", (B,), device), _ints(count, "count", (B,), device),
                           _ints(mask, "mask", (B, n), device), on.stream.cuda_stream)

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
        if dtype not in _DTYPES:
            raise ValueError(f"dtype must be float32, bfloat16 or float16, not {dtype}")
        B = self.batch if batch is None else batch
        if not 0 <= B <= self.batch or n < 0:
            raise ValueError("batch must be at most the cache's, and n not negative")
        shape = (B, n, self.heads, self.head_dim)
        with _On(self.device, stream) as on:
            if out is None:
                out = tuple(torch.empty(shape, dtype=dtype, device=self.device) for _ in "kv")
            kt, vt = (_rows(t, name, shape, dtype, self.device)
                      for t, name in zip(out, ("k", "v")))
            on.uses(start, count, *out, *self._tensors())
            gm.gm_kv_read(self.c, _DTYPES[dtype], B, n, _ints(start, "start", (B,), self.device),
                          _ints(count, "count", (B,), self.device), kt, vt, on.stream.cuda_stream)
        return tuple(out)

    def _shape(self, t: torch.Tensor, device) -> Tuple[int, int]:
        if device != self.device:
            raise ValueError(f"the cache is on {self.device}, the rows on {device}")
        if t.dim() != 4 or t.shape[0] > self.batch:
            raise ValueError("rows must be [B, n, heads, head_dim] with B at most the cache's batch")
        return t.shape[0], t.shape[1]


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
    dtype, device = _first(q, "q")
    if q.dim() != 4 or q.shape[0] > cache.batch or device != cache.device:
        raise ValueError("q must be [B, Sq, n_heads, head_dim] on the cache's device, with B at "
                         "most the cache's batch")
    B, Sq, H, hd = q.shape
    if hd != cache.head_dim:
        raise ValueError(f"q must have the cache's head_dim {cache.head_dim}, not {hd}")
    if lengths is None:
        raise ValueError("lengths is missing")
    with _On(device, stream) as on:
        if out is None:
            out = torch.empty((B, Sq, H, hd), dtype=dtype, device=device)
        need = gm.gm_attention_cached_workspace(cache.c, _DTYPES[dtype], B, Sq, H)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        a = gm.gm_cached_attention(
            ctypes.pointer(cache.c), _DTYPES[dtype], B, Sq, H,
            _rows(q, "q", q.shape, dtype, device), _rows(out, "out", q.shape, dtype, device),
            _ints(lengths, "lengths", (B,), device),
            _scores(scale, softcap, slopes, H, hd, device),
            work.data_ptr() if need else None, need)
        on.uses(q, out, lengths, slopes, *cache._tensors())
        gm.gm_attention_cached(a, on.stream.cuda_stream)
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
    dtype, device = _first(q, "q")
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [batch, tokens, heads, head_dim]")
    B, Sq, H, hd = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    shape = (B, Sk, Hkv, hd)
    with _On(device, stream) as on:
        if out is None:
            out = torch.empty((B, Sq, H, hd), dtype=dtype, device=device)
        a = gm.gm_prompt_attention(
            _DTYPES[dtype], B, Sq, Sk, H, Hkv, hd, _rows(q, "q", q.shape, dtype, device),
            _rows(k, "k", shape, dtype, device), _rows(v, "v", shape, dtype, device),
            _rows(out, "out", q.shape, dtype, device), int(causal),
            Sk - Sq if q_offset is None else q_offset,
            _scores(scale, softcap, slopes, H, hd, device),
            _ints(key_mask, "key_mask", (B, Sk), device), _ints(q_doc, "q_doc", (B, Sq), device),
            _ints(k_doc, "k_doc", (B, Sk), device), _ints(prefix, "prefix", (B,), device))
        on.uses(q, k, v, out, slopes, key_mask, q_doc, k_doc, prefix)
        gm.gm_attention(a, on.stream.cuda_stream)
    return out
