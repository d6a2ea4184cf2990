"""What the 8-bit cache's binding says of a refused call (no GPU needed: a
cache of host tensors and a stand-in for the library)."""
import pytest
import torch

import paper_2607_13500_gb300 as altr
from paper_2607_13500_gb300 import _build, _lib, attention

HOST = -1  # the index that host tensors report


@pytest.fixture(scope="module", autouse=True)
def _built():
    _build.build()


@pytest.mark.parametrize("kind", [altr.PagedCache, altr.PagedCache8])
def test_a_refusal_names_the_entry_point(kind, monkeypatch):
    monkeypatch.setattr(attention, "_stream", lambda i: 0)
    monkeypatch.setattr(attention, "at", lambda i, fn: fn)

    class Library:
        cache_append = cache_attend = staticmethod(lambda *a: 7)
        cache_attend_workspace_bytes = staticmethod(lambda *a: 0)

    eight = kind is altr.PagedCache8
    c = kind.__new__(kind)
    c.calls, c.device, c.index, c.dtype = Library(), torch.device("cpu"), HOST, torch.bfloat16
    c.pages, c.heads, c.page, c.head_dim = 4, 2, 16, 64
    fixed = (1, 2, attention._CODES[torch.bfloat16], 4, 2, 16, 64)
    c._fixed = {torch.bfloat16: fixed} if eight else fixed
    c.error, c._scales, c._sizes = torch.zeros(1, dtype=torch.int32), attention._pack_scales(3, 4), {}
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32)
    rows = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    name = "tr_cache8_" if eight else "tr_cache_"
    with pytest.raises(_lib.TrError, match=name + "append failed"):
        c.append(rows, rows, i32(0, 1)[None], i32(3), i32(0, 3))
    with pytest.raises(_lib.TrError, match=name + "attend failed"):
        c.attend(rows, i32(0, 1)[None], i32(3), i32(0, 3))
