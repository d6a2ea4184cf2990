"""Python binding of libtr's attention-layer operators: rotary positions with
several axes (``Rotary``) and the paged key/value cache (``PagedCache``).

As in api.py the kernels run in libtr on the current stream and nothing here
computes on the host: the binding checks what the C side cannot (types,
shapes, the device), supplies outputs and workspaces, and raises when libtr.so
is missing or a tensor is not on the CUDA device.  No call synchronises.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

import torch

from ._lib import TR_BF16, TR_F16, TR_F32, TR_ROTARY_LAYOUT, TrCache, TrHeads, TrRotary, check, load

_CODES = {torch.bfloat16: TR_BF16, torch.float16: TR_F16, torch.float32: TR_F32}
_byref = ctypes.byref


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _heads(t, name, tokens, heads, d, dtype, device):
    """A [tokens, heads, d] tensor (its channels contiguous) as a tr_heads."""
    if t.dim() != 3 or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor [tokens, heads, {d}] on {device}")
    shape, stride = t.shape, t.stride()
    if shape[0] != tokens or (heads is not None and shape[1] != heads) or shape[2] != d:
        raise ValueError(f"{name} must be [{tokens}, {'heads' if heads is None else heads}, {d}], not {tuple(shape)}")
    if stride[2] != 1 and d > 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return TrHeads(t.data_ptr(), stride[0], stride[1], shape[1])


def _vector(t, name, d, device):
    """An fp32 [d] device vector's address (None passes)."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (d,) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor [{d}] on {device}")
    return t.data_ptr()


def _ints(t, name, shape, device):
    if t.dtype != torch.int32 or tuple(t.shape) != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on {device}")
    return t.data_ptr()


def _out(t, like, name):
    if t is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    if t.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}")
    return t


@dataclass
class RotaryGrads:
    q: torch.Tensor                 # gradient of the queries, their dtype
    k: torch.Tensor | None          # of the keys
    q_weight: torch.Tensor | None   # fp32 [head_dim], of the query norm's weight
    k_weight: torch.Tensor | None


class Rotary:
    """Rotary positions of heads of ``head_dim`` channels, several axes, with
    an optional RMS norm of each head in the same pass (tr_rotary_apply).

    Frequency i of the ``rot_dim`` / 2 (default: all channels) turns its pair
    of channels by position * f_i, f_i = ``base`` ** (-2 i / rot_dim) unless
    ``inv_freq`` lists them; ``sections`` says how many consecutive
    frequencies belong to each axis (default: one axis), and ``layout`` which
    channels pair up: "half" (i with i + rot_dim / 2) or "pairs" (2 i with
    2 i + 1).  Positions are int32 and may be of any size and sign."""

    def __init__(self, head_dim, device, base=10000.0, rot_dim=None, sections=None, layout="half", inv_freq=None):
        lib = self.lib = load()
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("Rotary needs a CUDA device (libtr has no CPU path)")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        if layout not in TR_ROTARY_LAYOUT:
            raise ValueError(f"layout must be one of {sorted(TR_ROTARY_LAYOUT)}")
        self.head_dim, self.rot_dim = int(head_dim), int(head_dim if rot_dim is None else rot_dim)
        half = self.rot_dim // 2
        freq = [float(base) ** (-i / half) for i in range(half)] if inv_freq is None else [float(f) for f in inv_freq]
        sections = [half] if sections is None else [int(n) for n in sections]
        if len(freq) != half or sum(sections) != half or any(n < 0 for n in sections):
            raise ValueError(f"inv_freq and sections must cover the {half} frequencies of rot_dim {self.rot_dim}")
        self.axes, self.layout = len(sections), layout
        turns = (ctypes.c_uint64 * max(half, 1))()
        check("tr_rotary_turns", lib.tr_rotary_turns((ctypes.c_double * max(half, 1))(*freq), half, turns))
        signed = [t - (1 << 64) if t >> 63 else t for t in turns]
        self.turns = torch.tensor(signed, dtype=torch.int64, device=self.device)
        self.axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)] or [0], dtype=torch.int32,
                                 device=self.device)
        self._s = TrRotary(self.turns.data_ptr(), self.axis.data_ptr(), self.head_dim, self.rot_dim, self.axes,
                           TR_ROTARY_LAYOUT[layout])
        self._ref = _byref(self._s)

    def _pos(self, pos, tokens):
        if pos.dim() == 1 and self.axes == 1:
            return _ints(pos, "pos", (tokens,), self.device)
        return _ints(pos, "pos", (self.axes, tokens), self.device)

    def apply(self, q, k, pos, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
        """rotate(norm(q)), rotate(norm(k)) for q [T, q heads, head_dim] and k
        [T, k heads, head_dim] (or None), any strides with contiguous
        channels; ``pos`` int32 [axes, T].  A head is normed where its fp32
        [head_dim] weight is given.  ``q_out`` / ``k_out`` may be q / k
        themselves.  Returns (q_out, k_out)."""
        code = _CODES.get(q.dtype)
        if code is None:
            raise TypeError("q must be bf16, fp16 or fp32")
        t, d, dev = q.shape[0], self.head_dim, self.device
        hq = _heads(q, "q", t, None, d, q.dtype, dev)
        p = self._pos(pos, t)
        qo = _out(q_out, q, "q_out")
        hqo = _heads(qo, "q_out", t, hq.heads, d, q.dtype, dev)
        hk = hko = ko = None
        if k is not None:
            hk = _heads(k, "k", t, None, d, q.dtype, dev)
            ko = _out(k_out, k, "k_out")
            hko = _heads(ko, "k_out", t, hk.heads, d, q.dtype, dev)
        if t == 0:
            return qo, ko
        check("tr_rotary_apply", self.lib.tr_rotary_apply(
            self._ref, code, t, p, hq, _vector(q_weight, "q_weight", d, dev), hqo, hk,
            _vector(k_weight, "k_weight", d, dev), hko, eps, _stream(dev)))
        return qo, ko

    def backward(self, dq, dk, pos, q=None, k=None, q_weight=None, k_weight=None, eps=1e-6) -> RotaryGrads:
        """Gradients of ``apply`` from those of its outputs (tr_rotary_backward);
        the forward inputs q and k are needed where their weight was given."""
        code = _CODES.get(dq.dtype)
        if code is None:
            raise TypeError("dq must be bf16, fp16 or fp32")
        t, d, dev = dq.shape[0], self.head_dim, self.device
        hdq = _heads(dq, "dq", t, None, d, dq.dtype, dev)
        p = self._pos(pos, t)
        gq = torch.empty(dq.shape, dtype=dq.dtype, device=dev)
        hgq = _heads(gq, "dq", t, hdq.heads, d, dq.dtype, dev)
        hq = hk = hdk = hgk = gk = wq = wk = None
        if q_weight is not None:
            if q is None:
                raise ValueError("q (the forward input) is needed for the gradient through its norm")
            hq = _heads(q, "q", t, hdq.heads, d, dq.dtype, dev)
            wq = torch.empty(d, dtype=torch.float32, device=dev)
        if dk is not None:
            hdk = _heads(dk, "dk", t, None, d, dq.dtype, dev)
            gk = torch.empty(dk.shape, dtype=dq.dtype, device=dev)
            hgk = _heads(gk, "dk", t, hdk.heads, d, dq.dtype, dev)
        if k_weight is not None:
            if dk is None or k is None:
                raise ValueError("dk and k (the forward input) are needed for the gradient through the keys' norm")
            hk = _heads(k, "k", t, hdk.heads, d, dq.dtype, dev)
            wk = torch.empty(d, dtype=torch.float32, device=dev)
        if t == 0:
            return RotaryGrads(gq, gk, None if wq is None else wq.zero_(), None if wk is None else wk.zero_())
        ws = ws_ptr = None
        nbytes = 0
        if wq is not None or wk is not None:
            nbytes = self.lib.tr_rotary_backward_workspace_bytes(self._ref, t)
            ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            ws_ptr = ws.data_ptr()
        check("tr_rotary_backward", self.lib.tr_rotary_backward(
            self._ref, code, t, p, hdq, hq, _vector(q_weight, "q_weight", d, dev), hgq,
            None if wq is None else wq.data_ptr(), hdk, hk, _vector(k_weight, "k_weight", d, dev), hgk,
            None if wk is None else wk.data_ptr(), eps, ws_ptr, nbytes, _stream(dev)))
        return RotaryGrads(gq, gk, wq, wk)


class PagedCache:
    """A paged key/value cache of one layer: ``k`` and ``v`` [pages, heads,
    page, head_dim] (bf16 or fp16), key j of a sequence in the page its row of
    the table names at j // page, slot j % page.

    A step describes its new tokens with three int32 device tensors, read by
    the kernels only (so they may change between replays of a captured
    graph): ``table`` [batch, max_pages] page ids, ``lens`` [batch] the keys
    of each sequence with the new ones, ``cu_new`` [batch + 1] prefix sums of
    the new tokens, which are each sequence's last.  ``error`` (int32[1])
    collects TR_CACHE_ERR_PAGE / TR_CACHE_ERR_WAIT."""

    def __init__(self, k, v):
        self.lib = load()
        if k.device.type != "cuda" or v.device != k.device:
            raise ValueError("the cache must live on one CUDA device (libtr has no CPU path)")
        if k.dtype not in (torch.bfloat16, torch.float16) or v.dtype != k.dtype:
            raise TypeError("the cache must be bf16 or fp16")
        if k.dim() != 4 or v.shape != k.shape or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("k and v must be contiguous [pages, heads, page, head_dim]")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self.pages, self.heads, self.page, self.head_dim = k.shape
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)

    @classmethod
    def empty(cls, pages, heads, page, head_dim, dtype=torch.bfloat16, device="cuda"):
        """An uninitialised cache."""
        mk = lambda: torch.empty(pages, heads, page, head_dim, dtype=dtype, device=device)
        return cls(mk(), mk())

    def _struct(self, table, lens, cu_new, tokens):
        dev, batch = self.device, lens.shape[0]
        if table.dim() != 2:
            raise ValueError("table must be [batch, max_pages]")
        return TrCache(self.k.data_ptr(), self.v.data_ptr(), _CODES[self.dtype], self.pages, self.heads, self.page,
                       self.head_dim, _ints(table, "table", (batch, table.shape[1]), dev), batch, table.shape[1],
                       _ints(lens, "lens", (batch,), dev), _ints(cu_new, "cu_new", (batch + 1,), dev), tokens)

    def append(self, k, v, table, lens, cu_new, rotary=None, pos=None, k_weight=None, q=None, q_weight=None,
               q_out=None, eps=1e-6):
        """Writes the new tokens' keys rotate(norm(k)) and values v, both [T,
        heads, head_dim], into their pages (tr_cache_append); ``rotary`` (a
        Rotary, with ``pos``) and ``k_weight`` are optional.  ``q`` [T, q
        heads, head_dim], when given, is normed and rotated in the same
        launch; returns it (``q_out``, which may be q), else None."""
        t, d, dev, dt = k.shape[0], self.head_dim, self.device, self.dtype
        c = self._struct(table, lens, cu_new, t)
        hk, hv = _heads(k, "k", t, self.heads, d, dt, dev), _heads(v, "v", t, self.heads, d, dt, dev)
        r = p = hq = hqo = None
        if rotary is not None:
            if rotary.device != dev or pos is None:
                raise ValueError("rotary must live on the cache's device and needs pos")
            r, p = rotary._ref, rotary._pos(pos, t)
        if q is not None:
            hq = _heads(q, "q", t, None, d, dt, dev)
            q_out = _out(q_out, q, "q_out")
            hqo = _heads(q_out, "q_out", t, hq.heads, d, dt, dev)
        if t == 0:
            return q_out if q is not None else None
        check("tr_cache_append", self.lib.tr_cache_append(
            c, hk, hv, r, p, _vector(k_weight, "k_weight", d, dev), hq, _vector(q_weight, "q_weight", d, dev), hqo,
            eps, self.error.data_ptr(), _stream(dev)))
        return q_out if q is not None else None

    def attend(self, q, table, lens, cu_new, scale=None, causal=True, window=0, max_new=None, max_len=None, out=None,
               return_lse=False):
        """Attention of the new tokens' queries q [T, q heads, head_dim] over
        the cache (tr_cache_attend), their own keys appended first.  With
        ``causal`` a token sees the keys up to its own, with ``window`` > 0 only
        the last ``window`` of those.  ``max_new`` and ``max_len``, what the
        host knows of a sequence's new tokens and length at most, only choose
        the launch (defaults: all T, and what the table can hold).  Returns
        out, or (out, lse fp32 [T, q heads])."""
        t, d, dev = q.shape[0], self.head_dim, self.device
        c = self._struct(table, lens, cu_new, t)
        hq = _heads(q, "q", t, None, d, self.dtype, dev)
        out = _out(out, q, "out")
        ho = _heads(out, "out", t, hq.heads, d, self.dtype, dev)
        lse = torch.empty(t, hq.heads, dtype=torch.float32, device=dev) if return_lse else None
        if t == 0:
            return (out, lse) if return_lse else out
        max_new = t if max_new is None else int(max_new)
        max_len = table.shape[1] * self.page if max_len is None else int(max_len)
        nbytes = self.lib.tr_cache_attend_workspace_bytes(c, hq.heads, window, max_new, max_len)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
        check("tr_cache_attend", self.lib.tr_cache_attend(
            c, hq, ho, None if lse is None else lse.data_ptr(), 1.0 / math.sqrt(d) if scale is None else scale,
            1 if causal else 0, window, max_new, max_len, None if ws is None else ws.data_ptr(), nbytes,
            self.error.data_ptr(), _stream(dev)))
        return (out, lse) if return_lse else out
