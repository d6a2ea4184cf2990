"""Python binding of libtr's attention-layer operators: rotary positions with
several axes (``Rotary``) and the paged key/value cache, in 16 bits
(``PagedCache``) and in 8 (``PagedCache8``).

As in api.py the kernels run in libtr on the current stream and nothing here
computes on the host: the binding checks what the C side cannot (types,
shapes, the device), supplies outputs and workspaces, makes the tensors' device
current around the call, and raises when libtr.so is missing or a tensor is not
on the CUDA device.  No call synchronises.
"""
from __future__ import annotations

import ctypes
import math
import struct
from dataclasses import dataclass

import torch

from . import _lib
from ._device import at, resolved
from ._lib import TR_BF16, TR_F16, TR_F32, TR_ROTARY_LAYOUT, check, load

_MOST = 2 ** 31 - 1
_CODES = {torch.bfloat16: TR_BF16, torch.float16: TR_F16, torch.float32: TR_F32}

# The C structs are packed with struct.Struct and passed as bytes through
# function objects of their own (void pointers throughout): a call on one
# token takes the GPU two or three microseconds, so what the binding spends
# per argument counts.
_pack_heads = struct.Struct("@Pqqi0q").pack           # tr_heads
_pack_rotary = struct.Struct("@PPiiii").pack          # tr_rotary
_pack_cache = struct.Struct("@PPiiiiiPiiPPi0q").pack  # tr_cache
_pack_scales = struct.Struct("@PP").pack              # what follows it in tr_cache8
assert len(_pack_heads(0, 0, 0, 0)) == ctypes.sizeof(_lib.TrHeads)
assert len(_pack_rotary(0, 0, 0, 0, 0, 0)) == ctypes.sizeof(_lib.TrRotary)
assert len(_pack_cache(*([0] * 13))) == ctypes.sizeof(_lib.TrCache)
assert len(_pack_cache(*([0] * 13)) + _pack_scales(0, 0)) == ctypes.sizeof(_lib.TrCache8)


def _raw(lib, name):
    """A function of the library with raw argument types."""
    known, fn = getattr(lib, name), lib[name]  # indexing gives a function object of our own
    fn.argtypes = [a if a in (ctypes.c_int32, ctypes.c_float, ctypes.c_size_t) else ctypes.c_void_p
                   for a in known.argtypes]
    fn.restype = known.restype
    return fn


class _Calls:
    """The library's attention entry points with raw argument types."""

    def __init__(self, lib):
        for name in ("tr_rotary_apply", "tr_rotary_backward", "tr_rotary_backward_workspace_bytes", "tr_cache_append",
                     "tr_cache_attend", "tr_cache_attend_workspace_bytes"):
            setattr(self, name[3:], _raw(lib, name))
        self.cache8 = _Calls8(lib)


class _Calls8:
    """The same of the cache held in 8 bits, by the same names."""

    def __init__(self, lib):
        for name in ("cache_append", "cache_attend", "cache_attend_workspace_bytes"):
            setattr(self, name, _raw(lib, name.replace("cache", "tr_cache8")))


_calls = None


def _library():
    global _calls
    lib = load()
    if _calls is None or _calls.lib is not lib:
        _calls = _Calls(lib)
        _calls.lib = lib
    return _calls


def _device(device):
    if torch.device(device).type != "cuda":
        raise ValueError("a CUDA device is needed (libtr has no CPU path)")
    return resolved(device)


try:  # the raw handle without a Stream object around it
    from torch._C import _cuda_getCurrentRawStream as _stream
except ImportError:
    def _stream(index):
        return torch.cuda.current_stream(index).cuda_stream


def _heads(t, name, tokens, heads, d, dtype, index):
    """A [tokens, heads, d] tensor (its channels contiguous) on CUDA device
    `index` as a tr_heads; heads None: any number."""
    shape = t.shape
    if (len(shape) != 3 or shape[0] != tokens or shape[2] != d or t.dtype is not dtype or t.get_device() != index
            or (heads is not None and shape[1] != heads)):
        raise ValueError(f"{name} must be {dtype} [{tokens}, {'heads' if heads is None else heads}, {d}] on CUDA device "
                         f"{index}, not {t.dtype} {list(shape)} on {t.device}")
    s0, s1, s2 = t.stride()
    if s2 != 1 and d > 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return _pack_heads(t.data_ptr(), s0, s1, shape[1])


def _vector(t, name, d, index):
    """An fp32 [d] device vector's address (None passes)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (d,) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor [{d}] on CUDA device {index}")
    return t.data_ptr()


def _ints(t, name, shape, index):
    if t.dtype is not torch.int32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on CUDA device {index}")
    return t.data_ptr()


def _output(out, like, name, index):
    """`out`, or a new contiguous tensor like `like`, with its tr_heads."""
    t, h, d = like.shape
    if out is None:
        out = torch.empty((t, h, d), dtype=like.dtype, device=like.device)
        return out, _pack_heads(out.data_ptr(), h * d, d, h)
    return out, _heads(out, name, t, h, d, like.dtype, index)


@dataclass
class RotaryGrads:
    q: torch.Tensor                 # gradient of the queries, their dtype
    k: torch.Tensor | None          # of the keys
    q_weight: torch.Tensor | None   # fp32 [head_dim], of the query norm's weight
    k_weight: torch.Tensor | None


def _readable(t):
    """A gradient as the kernels can read it: autograd hands on whatever strides it has."""
    es = t.element_size()
    s0, s1, s2 = t.stride()
    if s2 == 1 and s0 * es % 16 == 0 and s1 * es % 16 == 0 and t.data_ptr() % 16 == 0:
        return t
    # (contiguous() would keep the odd strides of a single row, or of none)
    return torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)


class _Turned(torch.autograd.Function):
    """Rotary.apply as a node of the graph."""

    @staticmethod
    def forward(ctx, rotary, eps, pos, q, k, q_weight, k_weight):
        ctx.rotary, ctx.eps = rotary, eps
        ctx.save_for_backward(pos, None if q_weight is None else q, None if k_weight is None else k, q_weight, k_weight)
        return rotary._apply(q, k, pos, q_weight, k_weight, eps)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        pos, q, k, q_weight, k_weight = ctx.saved_tensors
        g = ctx.rotary.backward(_readable(dq), None if dk is None else _readable(dk), pos, q=q, k=k, q_weight=q_weight,
                                k_weight=k_weight, eps=ctx.eps)
        return None, None, None, g.q, g.k, g.q_weight, g.k_weight


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
        lib = load()
        self.calls = _library()
        self.device = _device(device)
        self.index = self.device.index
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
        self._struct = _pack_rotary(self.turns.data_ptr(), self.axis.data_ptr(), self.head_dim, self.rot_dim, self.axes,
                                    TR_ROTARY_LAYOUT[layout])

    def _pos(self, pos, tokens):
        if self.axes == 1 and pos.dim() == 1:
            return _ints(pos, "pos", (tokens,), self.index)
        return _ints(pos, "pos", (self.axes, tokens), self.index)

    def apply(self, q, k, pos, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
        """rotate(norm(q)), rotate(norm(k)) for q [T, q heads, head_dim] and k
        [T, k heads, head_dim] (or None), any strides with contiguous
        channels; ``pos`` int32 [axes, T].  A head is normed where its fp32
        [head_dim] weight is given.  ``q_out`` / ``k_out`` may be q / k
        themselves.  Returns (q_out, k_out), part of the graph where autograd
        records an input that requires a gradient (then without q_out and
        k_out)."""
        if (q.requires_grad or (k is not None and k.requires_grad) or (q_weight is not None and q_weight.requires_grad)
                or (k_weight is not None and k_weight.requires_grad)) and torch.is_grad_enabled():
            if q_out is not None or k_out is not None:
                raise ValueError("no gradient goes through q_out and k_out: leave them out or use torch.no_grad()")
            return _Turned.apply(self, eps, pos, q, k, q_weight, k_weight)
        return self._apply(q, k, pos, q_weight, k_weight, eps, q_out, k_out)

    def _apply(self, q, k, pos, q_weight, k_weight, eps, q_out=None, k_out=None):
        dt, i, d = q.dtype, self.index, self.head_dim
        code = _CODES.get(dt)
        if code is None:
            raise TypeError("q must be bf16, fp16 or fp32")
        t = q.shape[0]
        hq = _heads(q, "q", t, None, d, dt, i)
        p = self._pos(pos, t)
        q_out, hqo = _output(q_out, q, "q_out", i)
        hk = hko = None
        if k is not None:
            hk = _heads(k, "k", t, None, d, dt, i)
            k_out, hko = _output(k_out, k, "k_out", i)
        wq, wk = _vector(q_weight, "q_weight", d, i), _vector(k_weight, "k_weight", d, i)
        if t:
            rc = at(i, self.calls.rotary_apply)(self._struct, code, t, p, hq, wq, hqo, hk, wk, hko, eps, _stream(i))
            if rc:
                check("tr_rotary_apply", rc)
        return q_out, k_out

    def backward(self, dq, dk, pos, q=None, k=None, q_weight=None, k_weight=None, eps=1e-6) -> RotaryGrads:
        """Gradients of ``apply`` from those of its outputs (tr_rotary_backward);
        the forward inputs q and k are needed where their weight was given."""
        dt, i, d = dq.dtype, self.index, self.head_dim
        code = _CODES.get(dt)
        if code is None:
            raise TypeError("dq must be bf16, fp16 or fp32")
        t = dq.shape[0]
        hdq = _heads(dq, "dq", t, None, d, dt, i)
        p = self._pos(pos, t)
        gq, hgq = _output(None, dq, "dq", i)
        hq = hk = hdk = hgk = gk = wq = wk = ws = None
        if q_weight is not None:
            if q is None:
                raise ValueError("q (the forward input) is needed for the gradient through its norm")
            hq = _heads(q, "q", t, dq.shape[1], d, dt, i)
            wq = torch.empty(d, dtype=torch.float32, device=self.device)
        if dk is not None:
            hdk = _heads(dk, "dk", t, None, d, dt, i)
            gk, hgk = _output(None, dk, "dk", i)
        if k_weight is not None:
            if dk is None or k is None:
                raise ValueError("dk and k (the forward input) are needed for the gradient through the keys' norm")
            hk = _heads(k, "k", t, dk.shape[1], d, dt, i)
            wk = torch.empty(d, dtype=torch.float32, device=self.device)
        pq, pk = _vector(q_weight, "q_weight", d, i), _vector(k_weight, "k_weight", d, i)
        if t == 0:  # empty sums
            return RotaryGrads(gq, gk, None if wq is None else wq.zero_(), None if wk is None else wk.zero_())
        nbytes = 0
        if wq is not None or wk is not None:
            nbytes = at(i, self.calls.rotary_backward_workspace_bytes)(self._struct, t)
            ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        ptr = lambda x: None if x is None else x.data_ptr()
        rc = at(i, self.calls.rotary_backward)(self._struct, code, t, p, hdq, hq, pq, hgq, ptr(wq), hdk, hk, pk, hgk,
                                               ptr(wk), eps, ptr(ws), nbytes, _stream(i))
        if rc:
            check("tr_rotary_backward", rc)
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
    collects TR_CACHE_ERR_PAGE / TR_CACHE_ERR_WAIT.  No gradient goes through
    a cache: what ``append`` and ``attend`` return is no part of a graph."""

    _name = "tr_cache_"  # of the entry points

    def __init__(self, k, v):
        self.calls = _library()
        if k.device.type != "cuda" or v.device != k.device:
            raise ValueError("the cache must live on one CUDA device (libtr has no CPU path)")
        if k.dtype not in (torch.bfloat16, torch.float16) or v.dtype != k.dtype:
            raise TypeError("the cache must be bf16 or fp16")
        if k.dim() != 4 or v.shape != k.shape or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("k and v must be contiguous [pages, heads, page, head_dim]")
        self.k, self.v, self.device, self.dtype, self.index = k, v, k.device, k.dtype, k.get_device()
        self.pages, self.heads, self.page, self.head_dim = k.shape
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._fixed = (k.data_ptr(), v.data_ptr(), _CODES[k.dtype], *k.shape)
        self._sizes = {}  # workspace bytes by the sizes they follow from

    @classmethod
    def empty(cls, pages, heads, page, head_dim, dtype=torch.bfloat16, device="cuda"):
        """An uninitialised cache."""
        mk = lambda: torch.empty(pages, heads, page, head_dim, dtype=dtype, device=device)
        return cls(mk(), mk())

    def _rows_type(self, rows, name):
        """The type of a step's rows."""
        return self.dtype

    def _struct(self, table, lens, cu_new, tokens, dtype):
        return self._pack(self._fixed, table, lens, cu_new, tokens)

    def _pack(self, fixed, table, lens, cu_new, tokens):
        i, batch, shape = self.index, lens.shape[0], table.shape
        if len(shape) != 2 or shape[0] != batch:
            raise ValueError("table must be [batch, max_pages], lens [batch]")
        return _pack_cache(*fixed, _ints(table, "table", shape, i), batch, shape[1],
                           _ints(lens, "lens", (batch,), i), _ints(cu_new, "cu_new", (batch + 1,), i), tokens)

    def append(self, k, v, table, lens, cu_new, rotary=None, pos=None, k_weight=None, q=None, q_weight=None,
               q_out=None, eps=1e-6):
        """Writes the new tokens' keys rotate(norm(k)) and values v, both [T,
        heads, head_dim], into their pages (tr_cache_append); ``rotary`` (a
        Rotary, with ``pos``) and ``k_weight`` are optional.  ``q`` [T, q
        heads, head_dim], when given, is normed and rotated in the same
        launch; returns it (``q_out``, which may be q), else None."""
        t, d, i, dt = k.shape[0], self.head_dim, self.index, self._rows_type(k, "k")
        c = self._struct(table, lens, cu_new, t, dt)
        hk, hv = _heads(k, "k", t, self.heads, d, dt, i), _heads(v, "v", t, self.heads, d, dt, i)
        r = p = hq = hqo = None
        if rotary is not None:
            if rotary.index != i or pos is None:
                raise ValueError("rotary must live on the cache's device and needs pos")
            r, p = rotary._struct, rotary._pos(pos, t)
        if q is not None:
            hq = _heads(q, "q", t, None, d, dt, i)
            q_out, hqo = _output(q_out, q, "q_out", i)
        wq, wk = _vector(q_weight, "q_weight", d, i), _vector(k_weight, "k_weight", d, i)
        if t:
            rc = at(i, self.calls.cache_append)(c, hk, hv, r, p, wk, hq, wq, hqo, eps, self.error.data_ptr(),
                                                _stream(i))
            if rc:
                check(self._name + "append", rc)
        return None if q is None else q_out

    def attend(self, q, table, lens, cu_new, scale=None, causal=True, window=0, max_new=None, max_len=None, out=None,
               return_lse=False):
        """Attention of the new tokens' queries q [T, q heads, head_dim] over
        the cache (tr_cache_attend), their own keys appended first.  With
        ``causal`` a token sees the keys up to its own, with ``window`` > 0 only
        the last ``window`` of those.  ``max_new`` and ``max_len``, what the
        host knows of a sequence's new tokens and length at most, only choose
        the launch (defaults: all T, and what the table can hold).  Rows from
        cu_new[batch] on are zeros.  ``out`` does not overlap q.  Returns
        out, or (out, lse fp32 [T, q heads])."""
        t, d, i, dt = q.shape[0], self.head_dim, self.index, self._rows_type(q, "q")
        c = self._struct(table, lens, cu_new, t, dt)
        hq = _heads(q, "q", t, None, d, dt, i)
        out, ho = _output(out, q, "out", i)
        heads = q.shape[1]
        lse = torch.empty((t, heads), dtype=torch.float32, device=self.device) if return_lse else None
        if t:
            if max_new is None:
                max_new = t
            if max_len is None:
                max_len = table.shape[1] * self.page
            if window > _MOST or max_new > _MOST or max_len > _MOST:  # (ctypes would take them modulo 2^32)
                window, max_new, max_len = min(window, _MOST), min(max_new, _MOST), min(max_len, _MOST)
            key = (t, lens.shape[0], table.shape[1], heads, window, max_new, max_len)
            nbytes = self._sizes.get(key)
            if nbytes is None:
                if len(self._sizes) >= 4096:
                    self._sizes.clear()
                nbytes = at(i, self.calls.cache_attend_workspace_bytes)(c, heads, window, max_new, max_len)
                self._sizes[key] = nbytes
            ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes else None
            rc = at(i, self.calls.cache_attend)(
                c, hq, ho, None if lse is None else lse.data_ptr(),
                1.0 / math.sqrt(d) if scale is None else scale, 1 if causal else 0, window, max_new, max_len,
                None if ws is None else ws.data_ptr(), nbytes, self.error.data_ptr(), _stream(i))
            if rc:
                check(self._name + "attend", rc)
        return (out, lse) if return_lse else out


class PagedCache8(PagedCache):
    """A paged key/value cache of one layer in 8 bits: ``k`` and ``v``
    (float8_e4m3fn [pages, heads, page, head_dim]) hold codes, and every 16
    keys of a head share a power-of-two scale, ``k_scale`` and ``v_scale``
    (float8_e8m0fnu [pages, heads, page // 16]): a key's channel stands for
    code * scale.  A page is a power of two from 16 to 256.

    ``append`` and ``attend`` are PagedCache's, with rows (queries, new keys
    and values, outputs) in bf16 or fp16, whichever a call brings.  A block's
    scale is the least that holds what was appended to it, and grows with it:
    its older keys are then coded anew, by a power of two.  What is not finite
    is held as NaN."""

    _name = "tr_cache8_"

    def __init__(self, k, v, k_scale, v_scale):
        self.calls = _library().cache8
        if k.device.type != "cuda" or any(t.device != k.device for t in (v, k_scale, v_scale)):
            raise ValueError("the cache must live on one CUDA device (libtr has no CPU path)")
        if k.dtype != torch.float8_e4m3fn or v.dtype != k.dtype:
            raise TypeError("k and v must be float8_e4m3fn")
        if k_scale.dtype != torch.float8_e8m0fnu or v_scale.dtype != k_scale.dtype:
            raise TypeError("k_scale and v_scale must be float8_e8m0fnu")
        if k.dim() != 4 or v.shape != k.shape or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("k and v must be contiguous [pages, heads, page, head_dim]")
        scales = (k.shape[0], k.shape[1], k.shape[2] // 16)
        for t in (k_scale, v_scale):
            if t.shape != scales or not t.is_contiguous():
                raise ValueError(f"k_scale and v_scale must be contiguous {list(scales)}")
        self.k, self.v, self.device, self.dtype, self.index = k, v, k.device, k.dtype, k.get_device()
        self.k_scale, self.v_scale = k_scale, v_scale
        self.pages, self.heads, self.page, self.head_dim = k.shape
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._fixed = {t: (k.data_ptr(), v.data_ptr(), _CODES[t], *k.shape) for t in (torch.bfloat16, torch.float16)}
        self._scales = _pack_scales(k_scale.data_ptr(), v_scale.data_ptr())
        self._sizes = {}

    @classmethod
    def empty(cls, pages, heads, page, head_dim, device="cuda"):
        """An uninitialised cache."""
        mk = lambda d, t: torch.empty(pages, heads, *d, dtype=torch.uint8, device=device).view(t)
        codes, scales = (page, head_dim), (page // 16,)
        return cls(mk(codes, torch.float8_e4m3fn), mk(codes, torch.float8_e4m3fn), mk(scales, torch.float8_e8m0fnu),
                   mk(scales, torch.float8_e8m0fnu))

    def _rows_type(self, rows, name):
        if rows.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"{name} must be bf16 or fp16")
        return rows.dtype

    def _struct(self, table, lens, cu_new, tokens, dtype):
        return self._pack(self._fixed[dtype], table, lens, cu_new, tokens) + self._scales
