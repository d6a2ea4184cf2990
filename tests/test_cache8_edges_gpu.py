"""The attention over the 8-bit cache where its numbers lie far apart, where its
keys are taken in parts, and past the sizes that its kernels count in 31 bits.

Tolerances are those of test_cache8_gpu.py, except that what a key adds is
measured by what the row sees: a probability enters its product with the
value as a half, relative to the greatest probability times scale among the
keys that the row sees (a block's largest code is 448 at most, and at least
224 where its rows set the scale; for random codes the largest of 16 keys is
taken to be within 2 of it), so small ones are off by 2^-25 of twice the
greatest p_j max |v_j|, n of them at most.
"""
import math

import pytest
import torch

from test_cache8_gpu import BF, DEV, FP, U, _alt, _bytes, _cache, _cum, _held, _i32, _randn, _reference, _spoil, _table, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _parts(c):
    """Whether the last calls' plans took the keys in parts (chunks: only then is there a workspace)."""
    return max(c._sizes.values()) > 0


def _seen_reference(c, q, table, n, scale=None, window=0):
    """o, lse and their tolerances for one sequence, its new tokens the last (causal)."""
    t, hq, d = q.shape
    group, scale = hq // c.heads, 1 / math.sqrt(d) if scale is None else scale
    o, lse = torch.zeros(t, hq, d, dtype=torch.float64, device=DEV), torch.zeros(t, hq, dtype=torch.float64, device=DEV)
    tol_o, tol_l = torch.zeros_like(o), torch.zeros_like(lse)
    k, v = (_held(x, s, table, 0, n) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    own = n - t + torch.arange(t, device=DEV)[:, None]
    j = torch.arange(n, device=DEV)
    seen = j <= own
    if window:
        seen &= j > own - window
    for h in range(hq):
        kh, vh, qh = k[:, h // group], v[:, h // group], q[:, h].double()
        s = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
        z = torch.logsumexp(s, -1)
        p = (s - z[:, None].nan_to_num(0, 0, 0)).exp()
        mag = vh.abs().amax(-1)
        e = d * 2.0 ** -23 * abs(scale) * ((qh.abs() @ kh.abs().T) * seen).amax(-1)
        e = e + abs(scale) * qh.abs().sum(-1) * 2.0 ** -38 * kh.abs().amax()
        o[:, h], lse[:, h] = p @ vh, z
        tol_o[:, h] = U[q.dtype] * (p @ vh).abs() + (2.0 ** -11 + 2 * e + 2.0 ** -17)[:, None] * (p @ vh.abs())
        tol_o[:, h] += (n * 2.0 ** -25 * 2 * (p * mag).amax(-1))[:, None] + 2.0 ** -133  # (and the types' subnormal numbers)
        tol_l[:, h] = e + 2.0 ** -17 * (1 + z.nan_to_num(0, 0, 0).abs())
    return o, lse, tol_o, tol_l


def _blocks(table, n, first=0):
    """The pages of a sequence of n keys (16 a page: a block each), from the first."""
    return table[0, first:(n + 15) // 16].long()


@pytest.mark.parametrize("power", [60, 88, 110, 119])
@pytest.mark.parametrize("new,group", [(40, 4), (40, 1), (300, 4), (9, 1)])
def test_rows_without_a_key_are_zeros_whatever_the_scales(new, group, power):
    """More new tokens than keys: the first see nothing, beside rows that see large values."""
    n, hk, d = new // 2 + 3, 2, 64
    table, pages = _table([n], 16, 201)
    c = _cache(pages, hk, 16, d, 202)
    _bytes(c.v_scale)[:] = 127 + power
    q = _randn(new, group * hk, d, dtype=BF, seed=203)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    none = torch.arange(new, device=DEV) < new - n
    assert (o[none] == 0).all() and (lse[none] == -math.inf).all()
    _within(o[~none], ro[~none], to[~none], "o")
    _within(lse[~none], rl[~none], tl[~none], "lse")


@pytest.mark.parametrize("length", [200, 7000, 40000])
@pytest.mark.parametrize("new,group", [(1, 4), (8, 4), (40, 1), (40, 4), (300, 4)])
def test_the_largest_values(new, group, length):
    """Values up to 448 * 2^119, near the end of fp32: their means are below it, whoever joins them."""
    n, hk, d = length + new, 2, 64
    table, pages = _table([n], 16, 205)
    c = _cache(pages, hk, 16, d, 206)
    _bytes(c.v_scale)[:] = 127 + 119
    _bytes(c.v)[:] = 0x7e
    _bytes(c.v)[:, 1] ^= 0x80
    q = _randn(new, group * hk, d, dtype=BF, seed=207, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("length,width", [(200, 1), (7000, 1), (7000, 180), (40000, 1), (40000, 700)])
@pytest.mark.parametrize("new,group", [(1, 4), (2, 4), (8, 4), (40, 1), (40, 4), (300, 4)])
@pytest.mark.parametrize("place", ["first", "middle", "last"])
def test_values_that_outweigh_their_small_probability(new, group, length, width, place):
    """Blocks whose scores are 104 below the others' (probabilities of 2^-150) and whose values are 2^179 times theirs:
    the result is their own, whether other keys are taken with them or apart."""
    n, hk, d = length + new, 2, 64
    table, pages = _table([n], 16, 271)
    c = _cache(pages, hk, 16, d, 272)
    at = _blocks(table, n)
    i = {"first": 0, "middle": length // 32, "last": (n - new) // 16 - width}[place]
    heavy = at[i:i + width]
    _bytes(c.k)[:], _bytes(c.k_scale)[:] = 0, 127
    _bytes(c.k)[heavy, :, :, 0] = 0xed  # -104
    _bytes(c.v_scale)[at], _bytes(c.v_scale)[heavy] = 127 - 60, 127 + 119
    q = _randn(new, group * hk, d, dtype=BF, seed=273)
    q[:, :, 0] = 1
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), scale=1.0, return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n, scale=1.0)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


FAR = [(73, -60), (17, -116), (119, -100), (101, 0)]  # exponents of the values' scales, in turn


@pytest.mark.parametrize("length", [200, 7000])
@pytest.mark.parametrize("new,group", [(1, 4), (8, 4), (40, 1), (40, 4), (300, 4)])
@pytest.mark.parametrize("scales", FAR, ids=str)
def test_values_whose_scales_lie_far_apart(scales, new, group, length):
    """Every second block's values are smaller by far than the others': their keys count in the sum all the same."""
    n, hk, d = length + new, 2, 64
    table, pages = _table([n], 16, 211)
    c = _cache(pages, hk, 16, d, 212)
    at = _blocks(table, n)
    _bytes(c.v_scale)[at[0::2]], _bytes(c.v_scale)[at[1::2]] = 127 + scales[0], 127 + scales[1]
    q = _randn(new, group * hk, d, dtype=BF, seed=213, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    assert length < 1000 or new <= 8 or _parts(c)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new,group", [(8, 4), (40, 1), (40, 4), (300, 4)])
@pytest.mark.parametrize("hidden", [90, 119])
def test_small_values_beside_hidden_large_ones(hidden, new, group):
    """Rows that see values of 2^-20 alone, where the last rows see ones of 2^90 and more too."""
    n, hk, d = 636 + new, 2, 128
    table, pages = _table([n], 16, 221)
    c = _cache(pages, hk, 16, d, 222)
    at = _blocks(table, n)
    _bytes(c.v_scale)[at], _bytes(c.v_scale)[at[-1]] = 127 - 20, 127 + hidden
    q = _randn(new, group * hk, d, dtype=BF, seed=223, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


def test_the_sum_over_small_values_does_not_overflow():
    """40 000 keys whose values are 2^100 smaller than those of the last block, their scores 2^8 above the first tile's."""
    n, new, heads, d = 40016, 40, 152, 64
    table = torch.arange(n // 16, dtype=torch.int32, device=DEV)[None]
    c = _alt().PagedCache8.empty(n // 16, heads, 16, d, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(231)
    _bytes(c.v).copy_(torch.randint(0, 0x7f, c.v.shape, generator=g, device=DEV, dtype=torch.uint8))
    _bytes(c.k)[:], _bytes(c.k_scale)[:] = 0, 127
    _bytes(c.k)[8:, :, :, 0] = 0x4b  # 5.5: 2^7.93, below the 2^8 that the softmax's maximum may lag by
    _bytes(c.v_scale)[:], _bytes(c.v_scale)[-1] = 127 - 27, 127 + 73
    q = torch.zeros(new, heads, d, dtype=BF, device=DEV)
    q[:, :, 0] = 1
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), scale=1.0, return_lse=True)
    assert not _parts(c)
    ro, rl, to, tl = _seen_reference(c, q, table, n, scale=1.0)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new,group", [(1, 4), (8, 4), (40, 1), (40, 4), (300, 4)])
def test_the_largest_and_the_smallest_scales_side_by_side(new, group):
    """Bytes 254 and 11 (2^127 and 2^-116): every scale is taken as it stands."""
    n, hk, d = 200 + new, 2, 64
    table, pages = _table([n], 16, 241)
    c = _cache(pages, hk, 16, d, 242)
    at = _blocks(table, n)
    _bytes(c.v)[at[0::2]] &= 0xb7  # codes below 1, so that the values are numbers of 32 bits
    _bytes(c.v_scale)[at[0::2]], _bytes(c.v_scale)[at[1::2]] = 254, 11
    q = _randn(new, group * hk, d, dtype=BF, seed=243, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("hidden", [127, 127 - 40, 127 + 80])
@pytest.mark.parametrize("new,group", [(8, 4), (40, 1), (40, 4), (300, 4)])
def test_rows_that_see_the_smallest_scales_alone(new, group, hidden):
    """Values held with bytes 0 to 10, beside others that the last rows see too."""
    n, hk, d = 636 + new, 2, 64
    table, pages = _table([n], 16, 251)
    c = _cache(pages, hk, 16, d, 252)
    at = _blocks(table, n)
    g = torch.Generator().manual_seed(253)
    _bytes(c.v_scale)[at] = torch.randint(0, 11, (len(at), hk, 1), generator=g, dtype=torch.uint8).to(DEV)
    _bytes(c.v_scale)[at[-1]] = hidden
    q = _randn(new, group * hk, d, dtype=BF, seed=254, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _seen_reference(c, q, table, n)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new,group", [(8, 4), (40, 4), (300, 4)])
def test_blocks_of_zeros_beside_others(new, group):
    """Blocks of zeros as the append leaves them (byte 10): seen alone, and beside large values."""
    n, hk, d = 7000 + new, 2, 64
    table, pages = _table([n], 16, 261)
    c = _cache(pages, hk, 16, d, 262)
    at = _blocks(table, n)
    _bytes(c.v)[at[3:-2]], _bytes(c.v_scale)[at[3:-2]] = 0, 10
    _bytes(c.v_scale)[at[-1]] = 127 + 60
    q = _randn(new, group * hk, d, dtype=BF, seed=263, gain=0.1)
    for window in (0, 300):
        o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), window=window, return_lse=True)
        ro, rl, to, tl = _seen_reference(c, q, table, n, window=window)
        _within(o, ro, to, "o")
        _within(lse, rl, tl, "lse")

