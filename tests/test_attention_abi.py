"""What the attention-layer operators refuse, checked on the host before
anything is launched (no GPU needed), and the rotary frequencies' fixed-point
table against exact rationals."""
import ctypes
from fractions import Fraction

import pytest
import torch

from paper_2607_13500_gb300 import _build, _lib

ARG, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 3, 4, 5, 7
v = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return _lib.load()


def _rotary(**kw):
    base = dict(turns=0x1000, axis=0x2000, head_dim=128, rot_dim=128, axes=3, layout=0)
    base.update(kw)
    return _lib.TrRotary(**base)


def _heads(**kw):
    base = dict(p=0x10000, token_stride=32 * 128, head_stride=128, heads=32)
    base.update(kw)
    return _lib.TrHeads(**base)


def _cache(**kw):
    base = dict(k=0x100000, v=0x200000, dtype=1, pages=64, heads=4, page=16, head_dim=128, table=0x3000, batch=2,
                max_pages=8, lens=0x4000, cu_new=0x5000, total_new=0)
    base.update(kw)
    return _lib.TrCache(**base)


def test_turns_are_the_frequencies_as_fractions_of_a_turn(lib):
    pi2 = Fraction(6.283185307179586) + Fraction(2.4492935982947064e-16)  # 2 pi to 107 bits
    freq = [1.0, 0.5, 1e-6, 3.0, 7.0, -0.25, 0.0, 123.456]
    out = (ctypes.c_uint64 * len(freq))()
    assert lib.tr_rotary_turns((ctypes.c_double * len(freq))(*freq), len(freq), out) == 0
    for f, got in zip(freq, out):
        turn = Fraction(f) / pi2
        want = (turn - turn.__floor__()) * 2 ** 64
        # one rounding of the quotient (2^-53 of it) and of its fraction
        off = abs(Fraction(got) - want)
        assert min(off, 2 ** 64 - off) <= 2 ** 64 * (abs(turn) + 1) * Fraction(1, 2 ** 52)
    one = (ctypes.c_uint64 * 1)()
    for bad in (float("nan"), float("inf")):
        assert lib.tr_rotary_turns((ctypes.c_double * 1)(bad), 1, one) == ARG
    assert lib.tr_rotary_turns(None, 1, one) == ARG
    assert lib.tr_rotary_turns(None, 0, None) == 0


def test_rotary_refusals(lib):
    def call(r=None, dtype=1, tokens=0, pos=v(0x6000), q=None, qw=None, qo=None, k=None, kw=None, ko=None):
        r, q, qo = r or _rotary(), q or _heads(), qo or _heads(p=0x20000)
        return lib.tr_rotary_apply(r, dtype, tokens, pos, q, qw, qo, k, kw, ko, 1e-6, None)

    assert call() == 0  # no tokens: nothing to do
    assert call(tokens=-1) == ARG
    assert call(dtype=7) == DTYPE
    assert call(pos=None) == ARG
    assert call(pos=v(0x6002)) == ALIGN
    assert call(r=_rotary(head_dim=264)) == UNSUPPORTED
    assert call(r=_rotary(head_dim=124, rot_dim=64)) == ALIGN
    assert call(r=_rotary(rot_dim=60)) == ALIGN
    assert call(r=_rotary(rot_dim=136)) == ARG
    assert call(r=_rotary(rot_dim=-8)) == ARG
    assert call(r=_rotary(axes=0)) == ARG
    assert call(r=_rotary(layout=2)) == ARG
    assert call(r=_rotary(turns=None)) == ARG
    assert call(r=_rotary(rot_dim=0, turns=None, axis=None, axes=0), pos=None) == 0
    assert call(q=_heads(p=None)) == ARG
    assert call(q=_heads(heads=0), qo=_heads(heads=0)) == ARG
    assert call(q=_heads(heads=31)) == ARG           # out has other heads
    assert call(q=_heads(p=0x10008)) == ALIGN
    assert call(q=_heads(head_stride=132)) == ALIGN
    assert call(q=_heads(token_stride=-4096)) == ARG
    assert call(qw=v(0x7004)) == ALIGN
    assert call(k=_heads()) == ARG                    # k without k_out
    assert call(ko=_heads()) == ARG
    assert call(k=_heads(heads=4), ko=_heads(heads=4)) == 0

    def back(tokens=0, qw=None, q=None, dqw=None, ws=None, nbytes=0, kw=None, dkw=None, dk=None, dko=None):
        return lib.tr_rotary_backward(_rotary(), 1, tokens, v(0x6000), _heads(), q, qw, _heads(p=0x20000), dqw, dk,
                                      None, kw, dko, dkw, 1e-6, ws, nbytes, None)

    assert back() == 0
    assert back(qw=v(0x7000)) == ARG                  # a weight without its gradient and input
    assert back(qw=v(0x7000), dqw=v(0x8000)) == ARG
    assert back(dqw=v(0x8000)) == ARG                 # a gradient without its weight
    assert back(kw=v(0x7000), dkw=v(0x8000)) == ARG   # a key weight without keys
    full = dict(qw=v(0x7000), q=_heads(), dqw=v(0x8000), tokens=5)
    assert back(**full) == WORKSPACE
    assert back(**full, ws=v(0x9010), nbytes=1 << 30) == WORKSPACE
    assert lib.tr_rotary_backward_workspace_bytes(_rotary(layout=5), 10) == 0


def test_append_refusals(lib):
    def call(c=None, k=None, vv=None, r=None, pos=None, kw=None, q=None, qo=None):
        return lib.tr_cache_append(c or _cache(), k or _heads(heads=4), vv or _heads(heads=4), r, pos, kw, q, None, qo,
                                   1e-6, None, None)

    assert call() == 0
    assert call(c=_cache(k=None)) == ARG
    assert call(c=_cache(dtype=0)) == DTYPE           # an fp32 cache
    assert call(c=_cache(page=24)) == UNSUPPORTED
    assert call(c=_cache(page=8)) == UNSUPPORTED
    assert call(c=_cache(page=512)) == UNSUPPORTED
    assert call(c=_cache(head_dim=72)) == ALIGN
    assert call(c=_cache(head_dim=256)) == UNSUPPORTED
    assert call(c=_cache(heads=0)) == ARG
    assert call(c=_cache(lens=None)) == ARG
    assert call(c=_cache(table=None)) == ARG
    assert call(c=_cache(total_new=-1)) == ARG
    assert call(c=_cache(k=0x100008)) == ALIGN
    assert call(c=_cache(pages=1 << 30, heads=64)) == UNSUPPORTED
    assert call(c=_cache(max_pages=1 << 28)) == UNSUPPORTED
    assert call(k=_heads(heads=8)) == ARG             # other heads than the cache
    assert call(vv=_heads(heads=4, p=None)) == ARG
    assert call(k=_heads(heads=4, token_stride=4)) == ALIGN
    assert call(r=_rotary()) == ARG                   # rotary without pos
    assert call(r=_rotary(head_dim=64, rot_dim=64), pos=v(0x6000)) == ARG
    assert call(r=_rotary(), pos=v(0x6000)) == 0
    assert call(q=_heads()) == ARG                    # q without q_out
    assert call(q=_heads(), qo=_heads()) == 0


def test_attend_refusals(lib):
    def call(c=None, q=None, o=None, lse=None, scale=0.1, window=0, max_new=8, max_len=128, ws=None, nbytes=0):
        return lib.tr_cache_attend(c or _cache(), q or _heads(heads=28), o or _heads(heads=28), lse, scale, 1, window,
                                   max_new, max_len, ws, nbytes, None, None)

    assert call() == 0
    assert call(c=_cache(dtype=0)) == DTYPE
    assert call(q=_heads(heads=30), o=_heads(heads=30)) == ARG   # not a multiple of the key heads
    assert call(q=_heads(heads=4)) == ARG                        # q and o differ
    assert call(q=_heads(heads=28, p=None)) == ARG
    assert call(o=_heads(heads=28, p=0x10004)) == ALIGN
    assert call(lse=v(0x7002)) == ALIGN
    assert call(scale=float("nan")) == ARG
    assert call(window=-1) == ARG
    assert call(max_new=-1) == ARG
    assert call(max_len=-1) == ARG
    assert lib.tr_cache_attend_workspace_bytes(_cache(page=5), 28, 0, 1, 100) == 0


def test_binding_refuses_before_the_library(lib):
    import paper_2607_13500_gb300 as altr
    with pytest.raises(ValueError, match="CUDA"):
        altr.Rotary(64, "cpu")
    with pytest.raises(ValueError, match="CUDA"):
        altr.PagedCache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))
    from paper_2607_13500_gb300 import attention
    cpu = -1  # the device index of host tensors
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    h = _lib.TrHeads.from_buffer_copy(attention._heads(x[:, 1:3], "q", 3, 2, 64, torch.bfloat16, cpu))
    assert (h.token_stride, h.head_stride, h.heads) == (256, 64, 2) and h.p == x.data_ptr() + 128
    with pytest.raises(ValueError, match="q must"):  # on another device
        attention._heads(x, "q", 3, None, 64, torch.bfloat16, 0)
    for bad in (x[0], x.float(), x[:2], x[..., :32], x.transpose(1, 2)):
        with pytest.raises(ValueError, match="q must"):
            attention._heads(bad, "q", 3, None, 64, torch.bfloat16, cpu)
    with pytest.raises(ValueError, match="channels"):
        attention._heads(torch.zeros(3, 64, 4, dtype=torch.bfloat16).transpose(1, 2), "q", 3, 4, 64, torch.bfloat16,
                         cpu)
    for bad in (torch.zeros(4, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="lens must"):
            attention._ints(bad, "lens", (4,), cpu)
    with pytest.raises(ValueError, match="weight must"):
        attention._vector(torch.zeros(64, dtype=torch.bfloat16), "weight", 64, cpu)
    # the packed structs are the C structs
    c = _lib.TrCache.from_buffer_copy(attention._pack_cache(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13))
    assert [getattr(c, n) for n, _ in c._fields_] == list(range(1, 14))
    r = _lib.TrRotary.from_buffer_copy(attention._pack_rotary(1, 2, 3, 4, 5, 6))
    assert [getattr(r, n) for n, _ in r._fields_] == list(range(1, 7))
