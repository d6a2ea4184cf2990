"""What the 8-bit cache and the block tables refuse, on the host (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2607_13500_gb300 as altr
from paper_2607_13500_gb300 import _build, _lib, attention, pages

ARG, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 3, 4, 5, 7
v = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return _lib.load()


def _heads(**kw):
    return _lib.TrHeads(**(dict(p=0x10000, token_stride=32 * 128, head_stride=128, heads=32) | kw))


def _cache(k_scale=0x6000, v_scale=0x7000, **kw):
    base = dict(k=0x100000, v=0x200000, dtype=1, pages=64, heads=4, page=16, head_dim=128, table=0x3000, batch=2,
                max_pages=8, lens=0x4000, cu_new=0x5000, total_new=0)
    return _lib.TrCache8(_lib.TrCache(**(base | kw)), k_scale, v_scale)


def _pages(**kw):
    return _lib.TrPages(**(dict(table=0x1000, lens=0x2000, free=0x3000, free_count=0x4000, ticket=0x5000, batch=2,
                                max_pages=8, pages=64, page=16) | kw))


def test_cache_refusals(lib):
    def append(c=None, k=None, vv=None, r=None, pos=None, kw=None, q=None, qo=None):
        return lib.tr_cache8_append(c or _cache(), k or _heads(heads=4), vv or _heads(heads=4), r, pos, kw, q, None, qo,
                                    1e-6, None, None)

    def attend(c=None, q=None, o=None, lse=None, scale=0.1, window=0, max_new=8, max_len=128, ws=None, nbytes=0):
        return lib.tr_cache8_attend(c or _cache(), q or _heads(heads=28), o or _heads(heads=28), lse, scale, 1, window,
                                    max_new, max_len, ws, nbytes, None, None)

    for call in (append, attend):
        assert call() == 0
        assert call(c=_cache(k_scale=None)) == ARG
        assert call(c=_cache(v_scale=None)) == ARG
        assert call(c=_cache(k=None)) == ARG
        assert call(c=_cache(dtype=0)) == DTYPE            # rows of fp32
        assert call(c=_cache(page=24)) == UNSUPPORTED
        assert call(c=_cache(page=8)) == UNSUPPORTED
        assert call(c=_cache(head_dim=72)) == ALIGN
        assert call(c=_cache(head_dim=256)) == UNSUPPORTED
        assert call(c=_cache(v=0x200008)) == ALIGN
        assert call(c=_cache(total_new=-1)) == ARG
        assert call(c=_cache(max_pages=1 << 28)) == UNSUPPORTED
    assert append(k=_heads(heads=8)) == ARG
    assert append(vv=_heads(heads=4, token_stride=4)) == ALIGN
    rot = _lib.TrRotary(turns=0x1000, axis=0x2000, head_dim=128, rot_dim=128, axes=3, layout=0)
    assert append(r=rot) == ARG                            # without pos
    assert append(r=rot, pos=v(0x6000)) == 0
    assert append(kw=v(0x6004)) == ALIGN
    assert append(q=_heads()) == ARG                       # without q_out
    assert append(c=_cache(batch=1 << 30)) == UNSUPPORTED
    assert attend(q=_heads(heads=30), o=_heads(heads=30)) == ARG
    assert attend(q=_heads(heads=4)) == ARG
    assert attend(o=_heads(heads=28, p=0x10004)) == ALIGN
    assert attend(lse=v(0x7002)) == ALIGN
    assert attend(scale=float("inf")) == ARG
    assert attend(window=-1) == ARG and attend(max_new=-1) == ARG and attend(max_len=-1) == ARG
    assert attend(c=_cache(total_new=1 << 28)) == UNSUPPORTED
    assert attend(c=_cache(heads=1 << 17), q=_heads(heads=1 << 17), o=_heads(heads=1 << 17)) == UNSUPPORTED
    assert lib.tr_cache8_attend_workspace_bytes(_cache(page=5), 28, 0, 1, 100) == 0
    assert lib.tr_cache8_attend_workspace_bytes(_cache(), 27, 0, 1, 100) == 0


def test_table_refusals(lib):
    def extend(p=None, new=v(0x8000), rows=4, cu=v(0x9000), slots=v(0xa000), pos=v(0xb000), seq=v(0xc000)):
        return lib.tr_pages_extend(p or _pages(), new, rows, cu, slots, pos, seq, None, None)

    def truncate(p=None, keep=v(0x8000)):
        return lib.tr_pages_truncate(p or _pages(), keep, None, None)

    for call in (extend, truncate):
        for name in ("table", "lens", "free", "free_count", "ticket"):
            assert call(_pages(**{name: None})) == ARG
            assert call(_pages(**{name: 0x1002})) == ALIGN
        for name in ("batch", "max_pages", "pages"):
            assert call(_pages(**{name: -1})) == ARG
        for page in (0, 8, 24, 512):
            assert call(_pages(page=page)) == UNSUPPORTED
        assert call(_pages(pages=1 << 28)) == UNSUPPORTED
        assert call(_pages(max_pages=1 << 27)) == UNSUPPORTED
        assert call(_pages(batch=2 ** 31 - 1)) == UNSUPPORTED
    assert extend(new=None) == ARG and truncate(keep=None) == ARG
    assert extend(rows=-1) == ARG and extend(cu=None) == ARG and extend(slots=None) == ARG and extend(seq=None) == ARG
    assert extend(pos=v(0xb001)) == ALIGN and truncate(keep=v(0x8001)) == ALIGN
    assert extend(rows=2 ** 31 - 1) == UNSUPPORTED
    assert truncate(_pages(batch=0), keep=None) == 0       # nothing to do


def test_binding_refuses_before_the_library(lib):
    e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    z = lambda *s, t=e4: torch.zeros(s, dtype=torch.uint8).view(t)
    with pytest.raises(ValueError, match="CUDA"):
        altr.PagedCache8(z(2, 1, 16, 64), z(2, 1, 16, 64), z(2, 1, 1, t=e8), z(2, 1, 1, t=e8))
    with pytest.raises(ValueError, match="CUDA"):
        altr.PageTable(2, 3, 4, 16, "cpu")
    for bad, what in (((2, 3, 4, 24), "power of two"), ((2, 3, 4, 512), "power of two"), ((-1, 3, 4, 16), "negative"),
                      ((2, 3, 1 << 28, 16), "32-bit"), ((2, 1 << 27, 4, 16), "32-bit")):
        with pytest.raises(ValueError, match=what):
            altr.PageTable(*bad, "cuda:0")
    # the packed structs are the C structs
    c = _lib.TrCache8.from_buffer_copy(attention._pack_cache(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13)
                                       + attention._pack_scales(14, 15))
    assert [getattr(c.c, n) for n, _ in c.c._fields_] == list(range(1, 14)) and (c.k_scale, c.v_scale) == (14, 15)
    p = _lib.TrPages.from_buffer_copy(pages._pack_pages(*range(1, 10)))
    assert [getattr(p, n) for n, _ in p._fields_] == list(range(1, 10))


HOST = -1  # the index that host tensors report


@pytest.fixture
def cache(monkeypatch):
    """A cache of host tensors on a stand-in for the library."""
    monkeypatch.setattr(attention, "_stream", lambda i: 0)
    switched = []
    monkeypatch.setattr(attention, "at", lambda i, fn: switched.append(i) or fn)
    c = altr.PagedCache8.__new__(altr.PagedCache8)
    c.seen, c.switched = {}, switched

    class Library:
        def __getattr__(self, name):
            def call(*args):
                c.seen[name] = args
                return 0
            return call

    c.k = c.v = torch.zeros(4, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    c.calls, c.device, c.index, c.dtype = Library(), torch.device("cpu"), HOST, c.k.dtype
    c.pages, c.heads, c.page, c.head_dim = c.k.shape
    c._fixed = {t: (1, 2, attention._CODES[t], 4, 2, 16, 64) for t in (torch.bfloat16, torch.float16)}
    c.error, c._scales, c._sizes = torch.zeros(1, dtype=torch.int32), attention._pack_scales(3, 4), {}
    return c


def test_what_the_binding_hands_on(cache):
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32)
    table, lens, cu = i32(0, 1)[None], i32(3), i32(0, 3)
    for t in (torch.bfloat16, torch.float16):
        rows = torch.zeros(3, 8, 64, dtype=t)
        cache.append(rows[:, :2], rows[:, 2:4], table, lens, cu)
        o = cache.attend(rows[:, 4:], table, lens, cu, window=2 ** 40)
        assert o.dtype == t
        for name in ("cache_append", "cache_attend"):
            c = _lib.TrCache8.from_buffer_copy(cache.seen[name][0])
            assert (c.c.dtype, c.c.pages, c.c.total_new, c.k_scale, c.v_scale) == (attention._CODES[t], 4, 3, 3, 4)
        assert cache.seen["cache_attend"][6:9] == (2 ** 31 - 1, 3, 32)
    assert set(cache.switched) == {HOST}
    bf, fp = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.float16)
    with pytest.raises(TypeError, match="bf16 or fp16"):
        cache.append(bf.float(), bf, table, lens, cu)
    with pytest.raises(TypeError, match="bf16 or fp16"):
        cache.attend(bf.to(torch.float8_e4m3fn), table, lens, cu)
    with pytest.raises(ValueError, match="v must"):        # types that differ
        cache.append(bf, fp, table, lens, cu)
    with pytest.raises(ValueError, match="q must"):
        cache.append(bf, bf, table, lens, cu, q=fp)
    with pytest.raises(ValueError, match="q must"):        # another head size
        cache.attend(torch.zeros(3, 2, 32, dtype=torch.bfloat16), table, lens, cu)
    with pytest.raises(ValueError, match="table must"):
        cache.attend(bf, table[0], lens, cu)


def test_tables_run_on_their_device(monkeypatch):
    monkeypatch.setattr(attention, "_stream", lambda i: 0)
    switched, ran = [], []
    monkeypatch.setattr(pages, "at", lambda i, fn: switched.append(i) or fn)
    t = altr.PageTable.__new__(altr.PageTable)

    class Library:
        extend = staticmethod(lambda *a: ran.append(a) or 0)
        truncate = staticmethod(lambda *a: ran.append(a) or 0)

    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    t.calls, t.device, t.index, t.batch, t.max_pages, t.pages, t.page = Library, torch.device("cpu"), HOST, 2, 3, 5, 16
    t._error, t._struct = 11, pages._pack_pages(*range(1, 10))
    s = t.extend(i32(2), 7)
    assert s.cu_new.shape == (3,) and s.slots.shape == s.pos.shape == s.seq.shape == (7,)
    t.truncate(i32(2))
    assert switched == [HOST, HOST] and ran[0][2] == 7 and len(ran) == 2
    for bad in (i32(3), i32(2).long(), i32(2, 1), i32(4)[::2]):
        with pytest.raises(ValueError, match="new must"):
            t.extend(bad, 7)
        with pytest.raises(ValueError, match="keep must"):
            t.truncate(bad)
    for rows in (-1, 2 ** 31, 2 ** 32 + 3):  # ctypes would take them modulo 2^32
        with pytest.raises(ValueError, match="rows"):
            t.extend(i32(2), rows)
    with pytest.raises(AttributeError):  # the calls go by the tensors' addresses
        t.lens = i32(2)
