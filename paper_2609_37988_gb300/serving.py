"""Rotary positions, a paged cache and attention over whole prompts
(include/kvk.h, serving section): argument marshalling only.

Tokens are packed: a batch's new tokens lie one behind another in the first
dimension, sequence ``b``'s from ``cu[b]`` to ``cu[b + 1] - 1`` (int32, on the
device).  Queries, keys and values are ``[tokens, heads, head_dim]``, channels
contiguous, any other strides (views of a fused projection, say).

    rot = Rotary(head_dim=128, base=1e6, sections=(16, 24, 24))   # time, height, width
    pages = PagedCache(n_layers=48, n_q_heads=40, n_kv_heads=8, head_dim=128, n_pages=4096, page_size=16)
    q = pages.append(layer, k, v, cu, lengths, table, rotary=rot, positions=pos, q=q)
    o = pages.attend(layer, q, cu, lengths, table, scale, max_new=1)
    o = prompt_attention(q, k, v, cu, scale)          # before anything is cached

Calls run on the current stream, or on ``stream``: the caller then orders it with
the streams its tensors belong to, and keeps them until it has run.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import _lib
from ._lib import DTYPE_BF16, DTYPE_F16, DTYPE_F32, KVKError, PagedBatch, PagedDesc, Rows, check, load
from .cache import _ptr, _stream

__all__ = ["Rotary", "PagedCache", "prompt_attention", "prompt_error", "prompt_give_up", "KVKError"]

_CODES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}

# A serving step's small calls take 3-8 us on the GPU, so the binding's own time
# counts: structures are packed as bytes (0.05 us against 0.2 for a ctypes one),
# each tensor's strides and shape are read once, and outputs come from
# empty_like (1.0 us against 3.1 for torch.empty with shape, dtype and device).
_pack_rows = struct.Struct("Pqq").pack              # kvk_rows
_pack_batch = struct.Struct("PPPiiii").pack         # kvk_paged_batch
assert struct.calcsize("Pqq") == ctypes.sizeof(Rows) and struct.calcsize("PPPiiii") == ctypes.sizeof(PagedBatch)
_current_device = torch._C._cuda_getDevice


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _rows(t: torch.Tensor, name: str, dtype, index: int, shape) -> bytes:
    """``t`` as a kvk_rows: ``shape`` (tokens, heads, head_dim) of ``dtype`` on
    GPU ``index``, channels contiguous."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise (TypeError if t.dtype is not dtype else ValueError)(
            f"{name} must be {dtype} {tuple(shape)} on cuda:{index}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    ts, hs, cs = t.stride()
    if cs != 1 and shape[2] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return _pack_rows(t.data_ptr(), ts, hs)


def _ints(t: torch.Tensor, name: str, shape, index: int) -> int:
    if t.shape != shape or t.dtype is not torch.int32 or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {tuple(shape)} on cuda:{index}")
    return t.data_ptr()


def _shape(t: torch.Tensor, name: str):
    shape = t.shape
    if len(shape) != 3 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor [tokens, heads, head_dim]")
    return shape


def _int32(x: int) -> int:
    """``x``, or the nearest number that an int32 holds (ctypes would drop bits)."""
    return x if -2 ** 31 <= x < 2 ** 31 else 2 ** 31 - 1 if x > 0 else -2 ** 31


def _call(index: int, stream, fn, *args):
    """The library's call on GPU ``index``, which it wants to be the current one."""
    if stream is not None and stream.device.index != index:
        raise ValueError(f"stream of {stream.device}, tensors on cuda:{index}")
    if _current_device() == index:
        st = fn(*args, _stream(stream))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _stream(stream))
    if st:
        check(st)


def _new_like(t: torch.Tensor, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):  # the memory is that stream's
        return torch.empty_like(t, memory_format=torch.contiguous_format)


def _out_like(out: torch.Tensor, t: torch.Tensor, stream) -> torch.Tensor:
    if out is None:
        return _new_like(t, stream)
    if out.shape != t.shape or out.dtype is not t.dtype or out.device != t.device or not out.is_contiguous():
        raise ValueError("out must be contiguous, of q's shape, dtype and device")
    return out


class Rotary:
    """Rotation frequencies ``base ** (-2 i / rotary_dim)`` (or ``inv_freq``) on
    one axis, or on several: ``sections`` gives how many consecutive frequencies
    turn with each axis, ``axes`` names each frequency's axis instead.
    ``adjacent`` pairs channels (2i, 2i+1) instead of (i, i + rotary_dim / 2);
    ``factor`` scales cos and sin."""

    def __init__(self, *, head_dim: int, rotary_dim: int = None, base: float = 10000.0, sections=None, axes=None,
                 inv_freq=None, adjacent: bool = False, factor: float = 1.0):
        self.handle = None
        self.lib = load()
        self.head_dim = head_dim
        self.rotary_dim = head_dim if rotary_dim is None else rotary_dim
        n = self.rotary_dim // 2
        if inv_freq is None:
            inv_freq = [float(base) ** (-2.0 * i / self.rotary_dim) for i in range(n)]
        inv_freq = [float(f) for f in inv_freq]
        if axes is None:
            axes = [a for a, m in enumerate(sections or [n]) for _ in range(m)]
        elif sections is not None:
            raise ValueError("give sections or axes, not both")
        axes = [int(a) for a in axes]
        if len(inv_freq) != n or len(axes) != n:
            raise ValueError(f"{n} frequencies: got {len(inv_freq)} and axes of {len(axes)}")
        self.n_axes = len(sections) if sections else max(axes, default=0) + 1
        h = ctypes.c_void_p()
        check(self.lib.kvk_rotary_create(head_dim, self.rotary_dim, self.n_axes, (ctypes.c_double * n)(*inv_freq),
                                         (ctypes.c_int32 * n)(*axes), int(adjacent), float(factor), ctypes.byref(h)))
        self.handle = h
        self._apply = self.lib.kvk_rotary_apply

    def __del__(self):
        if getattr(self, "handle", None):
            self.lib.kvk_rotary_destroy(self.handle)
            self.handle = None

    def _positions(self, positions, n, index):
        if positions.dim() == 1:
            positions = positions.unsqueeze(0)
        return _ints(positions, "positions", (self.n_axes, n), index)

    def apply(self, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, out=None, stream=None):
        """Rotates ``q`` and ``k`` (either may be ``None``) to ``positions``
        (int32 ``[axes, tokens]``, or ``[tokens]`` for one axis).  ``out``: the
        pair to write, which may be ``(q, k)``; returns the pair."""
        x = q if q is not None else k
        if x is None:
            raise ValueError("q or k must be given")
        n, d, index, dtype = _shape(x, "q or k")[0], self.head_dim, x.get_device(), x.dtype
        code = _code(x)
        rq = oq = rk = ok = q_out = k_out = None
        hq = hk = 0
        if q is not None:
            hq = q.shape[1]
            shape = (n, hq, d)
            rq = _rows(q, "q", dtype, index, shape)
            if out is None:
                q_out = _new_like(q, stream)
                oq = _pack_rows(q_out.data_ptr(), hq * d, d)
            else:
                q_out = out[0]
                oq = _rows(q_out, "q_out", dtype, index, shape)
        if k is not None:
            hk = _shape(k, "k")[1]
            shape = (n, hk, d)
            rk = _rows(k, "k", dtype, index, shape)
            if out is None:
                k_out = _new_like(k, stream)
                ok = _pack_rows(k_out.data_ptr(), hk * d, d)
            else:
                k_out = out[1]
                ok = _rows(k_out, "k_out", dtype, index, shape)
        _call(index, stream, self._apply, self.handle, rq, oq, hq, rk, ok, hk, code, n, self._positions(positions, n, index))
        return q_out, k_out


class PagedCache:
    """Keys and values of ``n_layers`` layers in pages.  ``k_pages`` and
    ``v_pages``: one pool ``[n_pages, n_kv_heads, page_size, head_dim]`` per
    layer (bf16 or fp16); without them the pools are allocated.

    Calls take the batch as device int32 tensors: ``cu [B + 1]`` offsets of the
    new tokens, ``lengths [B]`` positions held with the new tokens, ``table
    [B, max_pages]`` each sequence's pages.  Calls on one object share its
    workspace: order them on the GPU (one stream, say; threads may call at the
    same time)."""

    def __init__(self, *, n_q_heads: int, n_layers: int = None, n_kv_heads: int = None, head_dim: int = None,
                 n_pages: int = None, page_size: int = 16, dtype=torch.bfloat16, device=None, k_pages=None, v_pages=None):
        self.handle = None
        self.lib = load()
        if (k_pages is None) != (v_pages is None):
            raise ValueError("k_pages and v_pages go together")
        if k_pages is not None:
            k_pages, v_pages = list(k_pages), list(v_pages)
            if not k_pages or len(k_pages) != len(v_pages):
                raise ValueError("one pool of keys and one of values per layer")
            x = k_pages[0]
            for t in k_pages + v_pages:
                if not (t.is_cuda and t.is_contiguous()) or t.dim() != 4 or t.shape != x.shape or t.dtype != x.dtype or \
                        t.device != x.device:
                    raise ValueError("pools must be contiguous CUDA tensors [n_pages, n_kv_heads, page_size, head_dim], all alike")
            n_layers, dtype, dev = len(k_pages), x.dtype, x.device
            n_pages, n_kv_heads, page_size, head_dim = x.shape
        else:
            if None in (n_layers, n_kv_heads, head_dim, n_pages):
                raise ValueError("n_layers, n_kv_heads, head_dim and n_pages, or the pools, must be given")
            dev = torch.device(device) if device is not None else torch.device("cuda")
            if dev.index is None:
                dev = torch.device("cuda", torch.cuda.current_device())
        if dtype not in _CODES:
            raise TypeError(f"unsupported dtype {dtype}")
        self.device, self.dtype = dev, dtype
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.desc = PagedDesc(n_layers, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, _CODES[dtype])
        pool, ws = ctypes.c_size_t(), ctypes.c_size_t()
        check(self.lib.kvk_paged_plan(ctypes.byref(self.desc), ctypes.byref(pool), ctypes.byref(ws)))
        if k_pages is None:
            shape = (n_pages, n_kv_heads, page_size, head_dim)
            k_pages = [torch.empty(shape, dtype=dtype, device=dev) for _ in range(n_layers)]
            v_pages = [torch.empty(shape, dtype=dtype, device=dev) for _ in range(n_layers)]
        self.k_pages, self.v_pages = k_pages, v_pages
        self.workspace = torch.empty(ws.value, dtype=torch.uint8, device=dev)
        h = ctypes.c_void_p()
        ptrs = [(ctypes.c_void_p * n_layers)(*[t.data_ptr() for t in p]) for p in (k_pages, v_pages)]
        with torch.cuda.device(dev):
            check(self.lib.kvk_paged_create(ctypes.byref(self.desc), ptrs[0], ptrs[1], _ptr(self.workspace), ws.value,
                                            ctypes.byref(h)))
            self.handle = h
            check(self.lib.kvk_paged_reset(h, _stream()))
            torch.cuda.current_stream().synchronize()  # calls on any stream may follow
        self._index = dev.index
        self._append, self._attend = self.lib.kvk_paged_append, self.lib.kvk_paged_attention

    def close(self):
        if getattr(self, "handle", None):
            self.lib.kvk_paged_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _batch(self, n, cu, lengths, table) -> bytes:
        if lengths.dim() != 1 or table.dim() != 2:
            raise ValueError("lengths must be [B], table [B, max_pages]")
        B, width, index = lengths.shape[0], table.shape[1], self._index
        return _pack_batch(_ints(cu, "cu", (B + 1,), index), _ints(lengths, "lengths", (B,), index),
                           _ints(table, "table", (B, width), index), B, width, n, 0)

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, lengths: torch.Tensor,
               table: torch.Tensor, *, rotary: Rotary = None, positions: torch.Tensor = None, q: torch.Tensor = None,
               q_out: torch.Tensor = None, stream=None):
        """Writes the new tokens' ``k`` and ``v`` into the layer's pages, keys
        rotated on the way where ``rotary`` is given (to ``positions``, or to the
        tokens' own positions); rotates ``q`` beside them and returns it
        (``q_out`` may be ``q``).  Rows of ``q`` in no sequence stay unwritten."""
        n, index, dtype = k.shape[0], self._index, self.dtype
        shape = (n, self.n_kv_heads, self.head_dim)
        rk, rv = _rows(k, "k", dtype, index, shape), _rows(v, "v", dtype, index, shape)
        rq = ro = None
        if q is not None:
            shape = (n, self.n_q_heads, self.head_dim)
            rq = _rows(q, "q", dtype, index, shape)
            if q_out is None:
                q_out = _new_like(q, stream)
                ro = _pack_rows(q_out.data_ptr(), shape[1] * shape[2], shape[2])
            else:
                ro = _rows(q_out, "q_out", dtype, index, shape)
        if positions is not None and rotary is None:
            raise ValueError("positions without a rotary")
        pos = 0 if positions is None else rotary._positions(positions, n, index)
        _call(index, stream, self._append, self.handle, _int32(layer), self._batch(n, cu, lengths, table), rk, rv,
              rotary.handle if rotary is not None else None, pos, rq, ro)
        return q_out if q is not None else None

    def attend(self, layer: int, q: torch.Tensor, cu: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
               scale: float, *, max_new: int = None, window: int = 0, out: torch.Tensor = None,
               stream=None) -> torch.Tensor:
        """Causal attention of the new tokens' queries over the layer's pages
        (appended first); ``window``: a query sees that many positions at most
        (0: all).  ``max_new``: no sequence has more new tokens (default: all of
        them); a tight one lets decode steps run the form for few tokens, and a
        ``table`` no wider than the contexts the quickest cut of the work.
        ``out`` may be ``q``.
        Returns ``[tokens, n_q_heads, head_dim]``; rows in no sequence stay
        unwritten."""
        n = q.shape[0]
        rq = _rows(q, "q", self.dtype, self._index, (n, self.n_q_heads, self.head_dim))
        out = _out_like(out, q, stream)
        _call(self._index, stream, self._attend, self.handle, _int32(layer), self._batch(n, cu, lengths, table), rq, scale,
              n if max_new is None else _int32(max_new), _int32(window), out.data_ptr())
        return out

    def set_give_up(self, give_up: bool):
        """Whether attentions give up before their first tile, as if a bounded wait
        had run out (setting the timeout error): for tests of that path."""
        check(self.lib.kvk_paged_set_give_up(self.handle, int(give_up)))

    def device_error(self, stream=None) -> int:
        """Synchronise, read and clear the device error word (0 = none)."""
        code = ctypes.c_int32()
        with torch.cuda.device(self.device):
            st = self.lib.kvk_paged_get_device_error(self.handle, _stream(stream), ctypes.byref(code))
        if st not in (0, 7):
            check(st)
        return code.value


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, scale: float, *,
                     window: int = 0, out: torch.Tensor = None, error: torch.Tensor = None, stream=None) -> torch.Tensor:
    """Causal attention of whole packed prompts to themselves: ``q [tokens, H_q,
    head_dim]``, ``k`` and ``v`` ``[tokens, H_kv, head_dim]`` (bf16 or fp16,
    post-RoPE), sequence ``b``'s tokens ``cu_seqlens[b]`` .. ``cu_seqlens[b + 1]
    - 1``; ``window``: a query sees that many positions at most (0: all).
    ``out`` may be ``q``.  ``error``: an int32 tensor of one element that gets device error bits
    (without one, ``prompt_error`` tells).
    Returns ``[tokens, H_q, head_dim]``; rows in no sequence stay unwritten."""
    n, hq, d = _shape(q, "q")
    index, dtype = q.get_device(), q.dtype
    kv = (n, _shape(k, "k")[1], d)
    rq = _rows(q, "q", dtype, index, q.shape)
    rk, rv = _rows(k, "k", dtype, index, kv), _rows(v, "v", dtype, index, kv)
    out = _out_like(out, q, stream)
    B = cu_seqlens.numel() - 1
    if B < 0:
        raise ValueError("cu_seqlens must be [sequences + 1]")
    _call(index, stream, load().kvk_prompt_attention, rq, rk, rv, n, hq, kv[1], d, _code(q),
          _ints(cu_seqlens, "cu_seqlens", (B + 1,), index), B, scale, _int32(window), out.data_ptr(),
          0 if error is None else _ints(error, "error", (1,), index))
    return out


def prompt_error(device=None, stream=None) -> int:
    """Synchronise, read and clear the device error word of the prompts on
    ``device`` (default: the current one) that were given no word (0 = none)."""
    code = ctypes.c_int32()
    with torch.cuda.device(device):
        st = load().kvk_prompt_get_device_error(_stream(stream), ctypes.byref(code))
    if st not in (0, 7):
        check(st)
    return code.value


def prompt_give_up(give_up: bool):
    """As ``PagedCache.set_give_up``, for all prompts."""
    check(load().kvk_prompt_set_give_up(int(give_up)))
