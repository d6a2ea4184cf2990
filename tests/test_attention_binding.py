"""What the attention binding hands to the library (no GPU needed: a cache of
host tensors and a stand-in for the library)."""
import ctypes
import sys

import pytest
import torch

import paper_2607_13500_gb300 as altr
from paper_2607_13500_gb300 import _device, attention

HOST = -1  # the index that host tensors report


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(_device, "_current", lambda: HOST)
    monkeypatch.setattr(attention, "_stream", lambda i: 0)
    c = altr.PagedCache.__new__(altr.PagedCache)
    c.seen = {}

    class Library:
        def cache_attend_workspace_bytes(self, struct, heads, window, max_new, max_len):
            c.seen["sizes"] = tuple(ctypes.c_int32(v).value for v in (heads, window, max_new, max_len))
            return 0

        def cache_attend(self, struct, q, o, lse, scale, causal, window, max_new, max_len, *rest):
            c.seen["call"] = tuple(ctypes.c_int32(v).value for v in (causal, window, max_new, max_len))
            return 0

    c.k = c.v = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    c.calls, c.device, c.index, c.dtype = Library(), torch.device("cpu"), HOST, torch.bfloat16
    c.pages, c.heads, c.page, c.head_dim = c.k.shape
    c.error, c._fixed, c._sizes = torch.zeros(1, dtype=torch.int32), (1, 2, 1, 4, 2, 16, 64), {}
    return c


def _attend(c, **kw):
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32)
    return c.attend(torch.zeros(3, 4, 64, dtype=torch.bfloat16), i32(0, 1)[None], i32(3), i32(0, 3), **kw)


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 5, sys.maxsize, 10 ** 30])
def test_limits_past_32_bits_are_the_most_there_is(cache, big):
    # ctypes takes an int modulo 2^32: a window of 2^32 + 5 keys must not become one of 5
    _attend(cache, window=big, max_new=big, max_len=big)
    most = 2 ** 31 - 1
    assert cache.seen["call"] == (1, most, most, most)
    assert cache.seen["sizes"] == (4, most, most, most)


def test_what_is_left_out_is_what_the_tensors_say(cache):
    _attend(cache, causal=False)
    assert cache.seen["call"] == (0, 0, 3, 32)
    assert cache.seen["sizes"] == (4, 0, 3, 32)
