"""Python binding of libtr's block tables (``PageTable``): which pages of a paged
cache the keys of each sequence lie in, kept on the GPU.

As in attention.py the kernels run in libtr on the current stream and no call
synchronises.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple

import torch

from . import _lib, attention
from ._device import at
from ._lib import check, load

_pack_pages = struct.Struct("@PPPPPiiii").pack  # tr_pages
assert len(_pack_pages(*([0] * 9))) == ctypes.sizeof(_lib.TrPages)

_calls = None


class _Calls:
    def __init__(self, lib):
        self.lib = lib
        self.extend, self.truncate = (attention._raw(lib, n) for n in ("tr_pages_extend", "tr_pages_truncate"))


def _library():
    global _calls
    lib = load()
    if _calls is None or _calls.lib is not lib:
        _calls = _Calls(lib)
    return _calls


class Step(NamedTuple):
    cu_new: torch.Tensor  # int32 [batch + 1], prefix sums of the new tokens
    slots: torch.Tensor   # int32 [rows], place of the row's key in the cache (page id * page + place in the page), or -1
    pos: torch.Tensor     # int32 [rows], its position in its sequence, or -1
    seq: torch.Tensor     # int32 [rows], its sequence, or -1


class PageTable:
    """The block tables of ``batch`` sequences in a paged cache of ``pages``
    pages of ``page`` keys, at most ``max_pages`` of them a sequence: ``table``
    int32 [batch, max_pages] and ``lens`` int32 [batch] as PagedCache and
    PagedCache8 read them, and a stack of free pages, ``free`` int32 [pages]
    with ``free_count`` int32 [1] of them in use, the last the next to be
    taken.  New: no sequence has a token, and page 0 is the next.

    ``extend`` and ``truncate`` change them on the GPU from device tensors, so
    a captured step follows its requests.  Calls on one table come one after
    another (one stream, or events between streams).  A call that cannot be
    carried out changes nothing, and ``error`` (int32[1]) collects
    TR_PAGES_ERR_FULL, _LONG, _ROWS or _STATE."""

    def __init__(self, batch, max_pages, pages, page, device="cuda"):
        self.calls = _library()
        self.device = attention._device(device)
        self.index = self.device.index
        self.batch, self.max_pages, self.pages, self.page = int(batch), int(max_pages), int(pages), int(page)
        if min(self.batch, self.max_pages, self.pages) < 0:
            raise ValueError("batch, max_pages and pages cannot be negative")
        if not 16 <= self.page <= 256 or self.page & (self.page - 1):
            raise ValueError("page must be a power of two from 16 to 256")
        if self.pages * self.page > attention._MOST or self.max_pages * self.page > attention._MOST - 65536:
            raise ValueError("slots and positions are 32-bit numbers: fewer pages")
        mk = lambda *s: torch.zeros(s, dtype=torch.int32, device=self.device)
        self._table, self._lens = mk(self.batch, self.max_pages).fill_(-1), mk(self.batch)
        self._free = torch.arange(self.pages - 1, -1, -1, dtype=torch.int32, device=self.device)
        self._free_count = mk(1).fill_(self.pages)
        self._errors, self._ticket = mk(1), mk(1)
        self._error = self._errors.data_ptr()
        self._struct = _pack_pages(*(x.data_ptr() for x in (self._table, self._lens, self._free, self._free_count, self._ticket)),
                                   self.batch, self.max_pages, self.pages, self.page)

    # (written in place, never replaced: the calls go by their addresses)
    table = property(lambda self: self._table)
    lens = property(lambda self: self._lens)
    free = property(lambda self: self._free)
    free_count = property(lambda self: self._free_count)
    error = property(lambda self: self._errors)

    def extend(self, new, rows) -> Step:
        """``new`` int32 [batch] more tokens for each sequence (negative:
        none), ``rows`` of them at most in all: their pages are taken from the
        free ones and ``lens`` grows (tr_pages_extend).  Returns what the rows
        need, rows behind the last token with -1.  If a step cannot be taken,
        cu_new is zeros and every row has -1."""
        i, b = self.index, self.batch
        rows = int(rows)
        if not 0 <= rows <= attention._MOST:
            raise ValueError("rows must be a 32-bit number that is not negative")
        p = attention._ints(new, "new", (b,), i)
        mk, dt, dev = torch.empty, torch.int32, self.device
        # (each by itself: views of one buffer take the host longer)
        s = Step(mk(b + 1, dtype=dt, device=dev), mk(rows, dtype=dt, device=dev), mk(rows, dtype=dt, device=dev),
                 mk(rows, dtype=dt, device=dev))
        rc = at(i, self.calls.extend)(self._struct, p, rows, s[0].data_ptr(), s[1].data_ptr(), s[2].data_ptr(),
                                      s[3].data_ptr(), self._error, attention._stream(i))
        if rc:
            check("tr_pages_extend", rc)
        return s

    def truncate(self, keep):
        """Every sequence keeps its first ``keep`` int32 [batch] tokens at
        most (0 or less: none), and the pages behind them are free again
        (tr_pages_truncate).  Directly after an extend, to the lengths before
        it, table, lens and free pages are as they were; the cache keeps what
        was appended meanwhile (a PagedCache8 the larger scale of a block that
        older keys share with tokens taken back)."""
        i = self.index
        p = attention._ints(keep, "keep", (self.batch,), i)
        rc = at(i, self.calls.truncate)(self._struct, p, self._error, attention._stream(i))
        if rc:
            check("tr_pages_truncate", rc)
