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
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import DTYPE_BF16, DTYPE_F16, DTYPE_F32, KVKError, PagedBatch, PagedDesc, Rows, check, load
from .cache import _ptr, _stream

__all__ = ["Rotary", "PagedCache", "prompt_attention", "KVKError"]

_CODES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _rows(t: torch.Tensor, name: str, like: torch.Tensor = None, shape=None) -> Rows:
    if t.dim() != 3 or not t.is_cuda or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be a CUDA tensor [tokens, heads, head_dim] with contiguous channels")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} is {t.dtype}, expected {like.dtype}")
        if t.device != like.device:
            raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    return Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _ints(t: torch.Tensor, name: str, shape, device):
    if t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != tuple(shape) or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor {tuple(shape)} on {device}")
    return t.data_ptr()


class _On:
    """Makes the tensors' device current where it is not (the library's calls
    launch on the current device)."""

    def __init__(self, device, stream):
        self.prev = torch._C._cuda_getDevice()
        self.want = device.index
        if stream is not None and stream.device != device:
            raise ValueError(f"stream of {stream.device}, tensors on {device}")

    def __enter__(self):
        if self.want != self.prev:
            torch.cuda.set_device(self.want)

    def __exit__(self, *exc):
        if self.want != self.prev:
            torch.cuda.set_device(self.prev)


def _new(shape, dtype, device, stream):
    out = torch.empty(shape, dtype=dtype, device=device)
    if stream is not None:
        out.record_stream(stream)
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

    def __del__(self):
        if getattr(self, "handle", None):
            self.lib.kvk_rotary_destroy(self.handle)
            self.handle = None

    def _positions(self, positions, n, device):
        if positions.dim() == 1:
            positions = positions.unsqueeze(0)
        return _ints(positions, "positions", (self.n_axes, n), device)

    def apply(self, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, out=None, stream=None):
        """Rotates ``q`` and ``k`` (either may be ``None``) to ``positions``
        (int32 ``[axes, tokens]``, or ``[tokens]`` for one axis).  ``out``: the
        pair to write, which may be ``(q, k)``; returns the pair."""
        x = q if q is not None else k
        if x is None:
            raise ValueError("q or k must be given")
        if x.dim() != 3:
            raise ValueError("q and k must be [tokens, heads, head_dim]")
        n, dev = x.shape[0], x.device
        args, res = [], []
        for i, (t, name) in enumerate(((q, "q"), (k, "k"))):
            if t is None:
                args += [None, None, 0]
                res.append(None)
                continue
            rows = _rows(t, name, x, (n, t.shape[1] if t.dim() == 3 else 0, self.head_dim))
            o = out[i] if out is not None else _new(t.shape, t.dtype, dev, stream)
            args += [rows, _rows(o, name + "_out", x, t.shape), t.shape[1]]
            res.append(o)
        pos = self._positions(positions, n, dev)
        with _On(dev, stream):
            check(self.lib.kvk_rotary_apply(self.handle, args[0], args[1], args[2], args[3], args[4], args[5], _code(x), n,
                                            pos, _stream(stream)))
        return tuple(res)


class PagedCache:
    """Keys and values of ``n_layers`` layers in pages.  ``k_pages`` and
    ``v_pages``: one pool ``[n_pages, n_kv_heads, page_size, head_dim]`` per
    layer (bf16 or fp16); without them the pools are allocated.

    Calls take the batch as device int32 tensors: ``cu [B + 1]`` offsets of the
    new tokens, ``lengths [B]`` positions held with the new tokens, ``table
    [B, max_pages]`` each sequence's pages.  Calls on one object share its
    workspace: order them."""

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
        with _On(dev, None):
            check(self.lib.kvk_paged_create(ctypes.byref(self.desc), ptrs[0], ptrs[1], _ptr(self.workspace), ws.value,
                                            ctypes.byref(h)))
            self.handle = h
            check(self.lib.kvk_paged_reset(h, _stream()))

    def close(self):
        if getattr(self, "handle", None):
            self.lib.kvk_paged_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _batch(self, n, cu, lengths, table) -> PagedBatch:
        if lengths.dim() != 1 or table.dim() != 2:
            raise ValueError("lengths must be [B], table [B, max_pages]")
        B, dev = lengths.shape[0], self.device
        return PagedBatch(_ints(cu, "cu", (B + 1,), dev), _ints(lengths, "lengths", (B,), dev),
                          _ints(table, "table", (B, table.shape[1]), dev), B, table.shape[1], n)

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, lengths: torch.Tensor,
               table: torch.Tensor, *, rotary: Rotary = None, positions: torch.Tensor = None, q: torch.Tensor = None,
               q_out: torch.Tensor = None, stream=None):
        """Writes the new tokens' ``k`` and ``v`` into the layer's pages, keys
        rotated on the way where ``rotary`` is given (to ``positions``, or to the
        tokens' own positions); rotates ``q`` beside them and returns it
        (``q_out`` may be ``q``).  Rows of ``q`` in no sequence stay unwritten."""
        if k.dim() != 3:
            raise ValueError("k must be [tokens, n_kv_heads, head_dim]")
        n = k.shape[0]
        like = self.k_pages[0]
        shape = (n, self.n_kv_heads, self.head_dim)
        rk, rv = _rows(k, "k", like, shape), _rows(v, "v", like, shape)
        rq = ro = None
        if q is not None:
            shape = (n, self.n_q_heads, self.head_dim)
            rq = _rows(q, "q", like, shape)
            if q_out is None:
                q_out = _new(shape, q.dtype, q.device, stream)
            ro = _rows(q_out, "q_out", like, shape)
        if positions is not None and rotary is None:
            raise ValueError("positions without a rotary")
        pos = 0 if positions is None else rotary._positions(positions, n, self.device)
        b = self._batch(n, cu, lengths, table)
        with _On(self.device, stream):
            check(self.lib.kvk_paged_append(self.handle, layer, b, rk, rv, rotary.handle if rotary is not None else None,
                                            pos, rq, ro, _stream(stream)))
        return q_out if q is not None else None

    def attend(self, layer: int, q: torch.Tensor, cu: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor,
               scale: float, *, max_new: int = None, window: int = 0, out: torch.Tensor = None,
               stream=None) -> torch.Tensor:
        """Causal attention of the new tokens' queries over the layer's pages
        (appended first); ``window``: a query sees that many positions at most
        (0: all).  ``max_new``: no sequence has more new tokens (default: all of
        them); a tight one lets decode steps run the form for few tokens.
        Returns ``[tokens, n_q_heads, head_dim]``; rows in no sequence stay
        unwritten."""
        if q.dim() != 3:
            raise ValueError("q must be [tokens, n_q_heads, head_dim]")
        n = q.shape[0]
        rq = _rows(q, "q", self.k_pages[0], (n, self.n_q_heads, self.head_dim))
        out = self._out(out, q, stream)
        b = self._batch(n, cu, lengths, table)
        with _On(self.device, stream):
            check(self.lib.kvk_paged_attention(self.handle, layer, b, rq, float(scale), n if max_new is None else max_new,
                                               window, _ptr(out), _stream(stream)))
        return out

    @staticmethod
    def _out(out, q, stream):
        if out is None:
            return _new(q.shape, q.dtype, q.device, stream)
        if out.shape != q.shape or out.dtype != q.dtype or out.device != q.device or not out.is_contiguous():
            raise ValueError("out must be contiguous, of q's shape, dtype and device")
        return out

    def device_error(self, stream=None) -> int:
        """Synchronise, read and clear the device error word (0 = none)."""
        code = ctypes.c_int32()
        with _On(self.device, stream):
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
    ``error``: an int32 tensor of one element that gets device error bits.
    Returns ``[tokens, H_q, head_dim]``; rows in no sequence stay unwritten."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [tokens, heads, head_dim]")
    n, hq, d = q.shape
    kv = (n, k.shape[1], d)
    rq, rk, rv = _rows(q, "q"), _rows(k, "k", q, kv), _rows(v, "v", q, kv)
    out = PagedCache._out(out, q, stream)
    if cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 1:
        raise ValueError("cu_seqlens must be [sequences + 1]")
    B = cu_seqlens.shape[0] - 1
    cu = _ints(cu_seqlens, "cu_seqlens", (B + 1,), q.device)
    err = 0 if error is None else _ints(error, "error", (1,), q.device)
    with _On(q.device, stream):
        check(load().kvk_prompt_attention(rq, rk, rv, n, hq, kv[1], d, _code(q), cu, B, float(scale), window, _ptr(out), err,
                                          _stream(stream)))
    return out
