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


@pytest.mark.parametrize("new,group", [(8, 4), (40, 1), (40, 4), (300, 4)])
@pytest.mark.parametrize("garbage", [0, 10, 255])
def test_scales_of_pages_given_away(new, group, garbage):
    """Pages before every window hold any scales and codes: nothing of them enters."""
    n, hk, d, window = 2000 + new, 2, 64, 700
    table, pages = _table([n], 16, 361)
    c = _cache(pages, hk, 16, d, 362)
    at = _blocks(table, n)
    gone = at[:(n - new - window + 1) // 16]
    for x in (c.k_scale, c.v_scale):
        _bytes(x)[gone] = garbage
    for x in (c.k, c.v):
        _bytes(x)[gone] = 0x7f
    q = _randn(new, group * hk, d, dtype=BF, seed=363, gain=0.5)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), window=window, return_lse=True)
    for x in (c.k, c.v):
        _bytes(x)[gone] = 0
    ro, rl, to, tl = _seen_reference(c, q, table, n, window=window)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new,group", [(1, 4), (8, 4), (40, 1), (40, 4), (300, 4)])
@pytest.mark.parametrize("length", [200, 7000])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_up_to_2_to_the_22(new, group, length, sign):
    """One key of 16 has the greatest score, 2^22, and is the result; the next is 2^18 below it.  (Scores and their
    difference are exact, so that nothing but the value's probability, 1, and the result is rounded.)"""
    n, hk, d = length + new, 2, 64
    table, pages = _table([n], 16, 351)
    c = _cache(pages, hk, 16, d, 352, spread=30)
    at = _blocks(table, n)
    _bytes(c.k)[:], _bytes(c.k_scale)[:] = 0, 127 + 2
    _bytes(c.k)[at, :, :, 0] = 0x77  # 240
    best = length // 2
    _bytes(c.k)[at[best // 16], :, best % 16, 0] = 0x78  # 256
    if sign < 0:
        _bytes(c.k)[at, :, :, 0] ^= 0x80
    q = torch.zeros(new, group * hk, d, dtype=BF, device=DEV)
    q[:, :, 0] = 2.0 ** 12
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), scale=float(sign), return_lse=True)
    v = _held(c.v, c.v_scale, table, 0, n)[best].repeat_interleave(group, 0)[None].expand(new, -1, -1)
    _within(o, v, (U[BF] + 2.0 ** -11 + 2.0 ** -17) * v.abs() + 2.0 ** -133, "o")
    _within(lse, torch.full_like(lse, 2.0 ** 22, dtype=torch.float64), torch.full_like(lse, 2.0 ** 22 * 2.0 ** -17, dtype=torch.float64), "lse")


# ---------------------------------------------------------------- the keys in parts
@pytest.mark.parametrize("new", [40, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_parts_of_the_keys_with_codes_that_are_no_numbers(new, d):
    n, page, hq, hk = 6200 + new, 16, 8, 2
    table, pages = _table([n], page, 281)
    c = _cache(pages, hk, page, d, 282)
    clean = [_bytes(x).clone() for x in (c.k, c.v)]
    q = _randn(new, hq, d, dtype=BF, seed=283)
    own = n - new + torch.arange(new, device=DEV)
    for window in (0, 6000):
        for x, y in zip((c.k, c.v), clean):
            _bytes(x).copy_(y)
        want = torch.zeros(new, hq, d, dtype=torch.bool, device=DEV)
        for j in (n - 1, n - new // 2, n - new - 200, n - 6000 - new // 3, 17):
            _bytes(c.v)[table[0, j // page].long(), 1, j % page, (7 * j) % d] = 0xff
            sees = own >= j
            if window:
                sees &= j > own - window
            want[:, hq // 2:, (7 * j) % d] |= sees[:, None]
        o = c.attend(q, table, _i32([n]), _i32([0, new]), window=window)
        assert _parts(c) and torch.equal(o.isnan(), want)
        _bytes(c.v).copy_(clean[1])
        ro, _, to, _ = _reference(c, q, table, [n], [0, new], window=window)
        _within(o[~want], ro[~want], to[~want], "rows that do not see it")
        j = n - new // 2  # a key that is not a number
        _bytes(c.k)[table[0, j // page].long(), 0, j % page, 3] = 0x7f
        o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), window=window, return_lse=True)
        want = torch.zeros(new, hq, dtype=torch.bool, device=DEV)
        want[:, :hq // 2] = (own >= j)[:, None]
        assert torch.equal(lse.isnan(), want) and torch.equal(o.isnan().all(-1), want) and torch.equal(o.isnan().any(-1), want)


@pytest.mark.parametrize("new", [40, 300])
@pytest.mark.parametrize("power", [30, 90])
def test_parts_of_the_keys_whose_scales_differ_by_far(new, power):
    """One part holds values 2^power times the others', behind every window and before it; one none but zeros."""
    n, page, hq, hk, d, window = 9000 + new, 16, 8, 2, 128, 8000
    table, pages = _table([n], page, 291)
    c = _cache(pages, hk, page, d, 292)
    at = _blocks(table, n)
    _bytes(c.v_scale)[at[:40]] += power                       # before the windows
    _bytes(c.v_scale)[at[300:380]] -= power                   # a part's
    _bytes(c.v)[at[400:480]], _bytes(c.v_scale)[at[400:480]] = 0, 10
    _bytes(c.v_scale)[at[-1]] += power                        # seen by the last rows alone
    q = _randn(new, hq, d, dtype=BF, seed=293, gain=0.1)
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), window=window, return_lse=True)
    assert _parts(c)
    ro, rl, to, tl = _seen_reference(c, q, table, n, window=window)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [40, 300])
def test_parts_of_the_keys_with_pages_outside_the_cache(new):
    n, page, hq, hk, d = 6200 + new, 16, 4, 2, 64
    table, pages = _table([n], page, 301)
    c = _cache(pages, hk, page, d, 302)
    q = _randn(new, hq, d, dtype=BF, seed=303)
    table[0, 150:290] = -1  # whole tiles, and a part of a part
    table[0, 300] = pages
    o, lse = c.attend(q, table, _i32([n]), _i32([0, new]), return_lse=True)
    assert _parts(c) and int(c.error) == 1
    ro, rl, to, tl = _reference(c, q, table, [n], [0, new])
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [1, 5, 70])
def test_a_request_alone_as_among_others(new):
    """Within what either may be off, and bit for bit when nothing but the stream differs."""
    lens, page, hq, hk, d = [new + 6200, new + 333, new], 32, 8, 2, 128
    table, pages = _table(lens, page, 311)
    c = _cache(pages, hk, page, d, 312)
    cu = _cum([new] * 3)
    q = _randn(3 * new, hq, d, dtype=BF, seed=313)
    both, lse = c.attend(q, table, _i32(lens), _i32(cu), max_new=new, max_len=max(lens), return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, cu)
    _within(both, ro, to, "among others")
    for b, n in enumerate(lens):
        mine = slice(cu[b], cu[b + 1])
        o, l = c.attend(q[mine], table[b:b + 1], _i32([n]), _i32([0, new]), return_lse=True)
        _within(o, ro[mine], to[mine], "alone")
        _within(o, both[mine].double(), 2 * to[mine], "alone as among others")
        _within(l, rl[mine], tl[mine], "lse alone")
    if new > 32:
        c._sizes.clear()
        c.attend(q[:new], table[:1], _i32(lens[:1]), _i32([0, new]))
        assert _parts(c)  # the first has a workspace
    streams = [torch.cuda.Stream() for _ in range(2)]
    ts, ls, cs = table, _i32(lens), _i32(cu)
    first, one = c.attend(q[:new], ts[:1], ls[:1], _i32([0, new])), _i32([0, new])
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append((c.attend(q, ts, ls, cs, max_new=new, max_len=max(lens)), c.attend(q[:new], ts[:1], ls[:1], one)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, both) and torch.equal(b, first) for a, b in outs)


# ---------------------------------------------------------------- many sequences, large caches
def _single_tokens(c, table, lens, q, **kw):
    """One new token of each sequence, all keys short enough for one padded computation."""
    n, d, group = int(lens.max()), q.shape[2], q.shape[1] // c.heads
    o, lse = c.attend(q, table, lens, torch.arange(len(lens) + 1, dtype=torch.int32, device=DEV), max_new=1, return_lse=True, **kw)
    assert int(c.error) == 0
    pages = (n + c.page - 1) // c.page
    at = table[:, :pages].long()
    k, v = ((x.view(torch.uint8)[at].view(torch.float8_e4m3fn).double() *
             torch.exp2(_bytes(s)[at].double() - 127).repeat_interleave(16, 3)[..., None]).transpose(1, 2).flatten(2, 3)[:, :, :n]
            for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    x = q.double().view(len(lens), c.heads, group, d)
    seen = (torch.arange(n, device=DEV) < lens[:, None])[:, None, None]
    s = (x @ k.transpose(2, 3) / math.sqrt(d)).masked_fill(~seen, -math.inf)
    z = torch.logsumexp(s, -1)
    p = torch.where(seen, torch.exp(s - torch.where(z.isinf(), 0.0, z)[..., None]), 0.0)
    e = torch.where(seen, x.abs() @ k.abs().transpose(2, 3), 0.0).amax(-1) / math.sqrt(d) * d * 2.0 ** -23
    e = e + x.abs().sum(-1) * 2.0 ** -38 * k.abs().amax((2, 3))[..., None] / math.sqrt(d)
    ref, pv, top = p @ v, p @ v.abs(), v.abs().amax((2, 3))[..., None, None]
    _within(o.view(ref.shape), ref, U[q.dtype] * ref.abs() + (2.0 ** -11 + 2 * e + 2.0 ** -17)[..., None] * pv
            + (n * 2.0 ** -25 + 2.0 ** -38) * top, "o")
    lse = lse.view(z.shape)
    assert torch.equal(lse.isinf(), z.isinf())
    some = ~z.isinf()
    _within(lse[some], z[some], (e + 2.0 ** -17 * (1 + z.abs()))[some], "lse")


def test_more_sequences_than_the_kernel_of_few_rows_counts():
    g = torch.Generator(device=DEV).manual_seed(321)
    batch, page, d = 8300, 16, 64
    c = _cache(500, 1, page, d, 322)
    table = torch.randint(0, 500, (batch, 13), device=DEV, generator=g, dtype=torch.int32)
    lens = torch.randint(0, 13 * page + 1, (batch,), device=DEV, generator=g, dtype=torch.int32)
    q = _randn(batch, 2, d, dtype=BF, seed=323, gain=1.5)
    _single_tokens(c, table, lens, q)
    _single_tokens(c, table[:8192], lens[:8192], q[:8192])


def test_tables_whose_tiles_pass_31_bits():
    heads, page, d, most = 80, 256, 64, 2 ** 23 - 257
    c = _cache(5, heads, page, d, 331)
    table = torch.full((2, most), -1, dtype=torch.int32, device=DEV)
    table[0, :2], table[1, :3] = _i32([4, 0]), _i32([1, 3, 2])
    lens = _i32([300, 517])
    q = _randn(2, heads, d, dtype=BF, seed=332, gain=1.5)
    _single_tokens(c, table, lens, q)
    _single_tokens(c, table, lens, q, max_len=517)


@pytest.mark.parametrize("new", [1, 40])
def test_a_cache_past_32_bits(new):
    """4.5 GB of codes each of keys and of values: pages at both ends, appended to and read."""
    heads, page, d, pages = 8, 256, 128, 17200
    assert pages * heads * page * d > 2 ** 32
    c = _alt().PagedCache8.empty(pages, heads, page, d, device=DEV)
    table = _i32([[pages - 1, 0, pages // 2], [pages - 2, 1, pages // 2 + 1]])
    for x in (c.k, c.v, c.k_scale, c.v_scale):
        _bytes(x)[table.flatten().long()] = 127 if x.dim() == 3 else 0x38
    lens, cu, t = [600 + new, 300 + new], [0, new, 2 * new], 2 * new
    near = {p: [_bytes(x)[p].clone() for x in (c.k, c.v)] for p in (2, 3, pages // 2 - 1, pages - 3)}
    past, batch = [600, 300], 2
    rows = _randn(sum(past), 2 * heads, d, dtype=BF, seed=341)
    assert c.append(rows[:, :heads], rows[:, heads:], table, _i32(past), _i32(_cum(past))) is None
    x = _randn(t, 4 * heads, d, dtype=BF, seed=342)
    c.append(x[:, :heads], x[:, heads:2 * heads], table, _i32(lens), _i32(cu))
    for b in range(batch):  # (every row is where the table says: off by half a code's step at most)
        want = torch.cat([rows[_cum(past)[b]:_cum(past)[b + 1]], x[cu[b]:cu[b + 1], :2 * heads]]).double()
        for y, s, w in ((c.k, c.k_scale, want[:, :heads]), (c.v, c.v_scale, want[:, heads:])):
            j = torch.arange(lens[b], device=DEV)
            home = table[b].long()[j // page]
            sc = torch.exp2(_bytes(s)[home, :, j % page // 16].double() - 127)[..., None]
            got = _bytes(y)[home, :, j % page].view(torch.float8_e4m3fn).double() * sc
            # (twice for the keys that a larger scale coded anew)
            _within(got, w, 2.0 ** -4 * w.abs() + 2 * 2.0 ** -10 * sc, "where the table says")
    assert all(torch.equal(_bytes(y)[p], z) for p, was in near.items() for y, z in zip((c.k, c.v), was))
    o, lse = c.attend(x[:, 2 * heads:], table, _i32(lens), _i32(cu), max_new=new, return_lse=True)
    small = _alt().PagedCache8.empty(6, heads, page, d, device=DEV)
    for y, z in ((small.k, c.k), (small.v, c.v), (small.k_scale, c.k_scale), (small.v_scale, c.v_scale)):
        _bytes(y).copy_(_bytes(z)[table.flatten().long()])
    again, lse2 = small.attend(x[:, 2 * heads:], _i32([[0, 1, 2], [3, 4, 5]]), _i32(lens), _i32(cu), max_new=new, return_lse=True)
    assert torch.equal(o, again) and torch.equal(lse, lse2) and int(c.error) == 0

