"""The paged cache held in 8 bits (tr_cache8_append, tr_cache8_attend) against
plain implementations in 64 bits.

Tolerances, with u the rows' unit roundoff (2^-8 bf16, 2^-11 fp16), derived
from the arithmetic:
* append, values: nothing but the codes rounds (powers of two are exact), so
  codes and scales are equal to the reference's bit for bit; keys neither
  normed nor rotated likewise.
* append, normed or rotated keys: fp32 arithmetic as in tr_rotary_apply, within
  w = 2^-19 (|a| + |b|) of the pair; then half a step of the code: 2^-4 of the
  value, or 2^-10 of the scale below the normal codes.  The scale is that of
  a largest magnitude within 2^-18 of the exact one.
* attention: u |o| for the output; probabilities in half precision for their
  product with V: 2^-11 sum p |v|, small ones 2^-25 of the largest, at most
  n 2^-25 max |v|; values and keys may enter the products in half precision
  relative to the largest scale of a range of keys, exact but for what falls
  under 2^-24 / 2^15 of its largest code, at most 2^-38 of the largest
  magnitude there: 2^-38 max |v| for a weighted mean, scale sum |q| 2^-38 max
  |k| for a score.  A score's error with that, e = (d 2^-23) scale sum |q k| +
  scale sum |q| 2^-38 max |k| (fp32 accumulation of d exact products), enters p
  twice: 2 e sum p |v|; exponentials, sums and the final division 2^-17
  sum p |v|.  lse: e + 2^-17 (1 + |lse|).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DEV = "cuda"
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _alt():
    import paper_2607_13500_gb300 as altr
    return altr


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cum(v):
    out = [0]
    for n in v:
        out.append(out[-1] + n)
    return out


def _randn(*shape, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(*shape, generator=g)).to(dtype).to(DEV)


def _within(got, ref, tol, what):
    got = got.double()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / tol).nan_to_num(1e30).max()))


def _bytes(t):
    return t.view(torch.uint8)


def _cache(pages, heads, page, d, seed, spread=2):
    """A cache of random codes and scales."""
    g = torch.Generator().manual_seed(seed)
    c = _alt().PagedCache8.empty(pages, heads, page, d, device=DEV)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8)
        x[(x & 0x7f) == 0x7f] = 0x30  # no NaN
        _bytes(codes).copy_(x)
        _bytes(scale).copy_(127 - 6 + torch.randint(-spread, spread + 1, scale.shape, generator=g))
    return c


def _table(lens, page, seed, spare=3):
    """Page ids for every sequence, in a random order; the others are -7 (never to be read)."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for n in lens]
    order = torch.randperm(sum(need) + spare, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(need + [1])), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table.to(DEV), sum(need) + spare


def _spoil(c, table, lens):
    """NaN wherever no sequence has a key: pages of no sequence, slots behind the last key."""
    used = torch.zeros(c.pages, c.page, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        j = torch.arange(n, device=DEV)
        used[table[b].long()[j // c.page], j % c.page] = True
    for codes in (c.k, c.v):
        _bytes(codes).transpose(1, 2)[~used] = 0x7f
    free = ~used.view(c.pages, -1, 16).any(-1)
    for scale in (c.k_scale, c.v_scale):
        _bytes(scale).transpose(1, 2)[free] = 255


def _held(codes, scale, table, b, n):
    """The first n keys' values of sequence b, float64 [n, heads, d] (bad pages: zeros)."""
    pages, heads, page, d = codes.shape
    j = torch.arange(n, device=DEV)
    home = table[b].long()[j // page]
    ok = (home >= 0) & (home < pages)
    home = home.clamp(0, pages - 1)
    x = codes.double()[home, :, j % page] * torch.exp2(_bytes(scale).double() - 127)[home, :, j % page // 16][..., None]
    return torch.where(ok[:, None, None], x, torch.zeros_like(x))


def _reference(c, q, table, lens, cu, scale=None, causal=True, window=0):
    """o, lse and their tolerances [T, heads, ...] in float64."""
    t, hq, d = q.shape
    group, scale = hq // c.heads, 1 / math.sqrt(d) if scale is None else scale
    o, lse = torch.zeros(t, hq, d, dtype=torch.float64, device=DEV), torch.full((t, hq), -math.inf, dtype=torch.float64, device=DEV)
    tol_o, tol_l = torch.zeros_like(o), torch.zeros_like(lse)
    for b, n in enumerate(lens):
        t0, t1 = cu[b], cu[b + 1]
        if t0 == t1 or n == 0:
            continue
        k, v = (_held(x, s, table, b, n) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        own = n - (t1 - t0) + torch.arange(t1 - t0, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)
        seen = torch.ones(t1 - t0, n, dtype=torch.bool, device=DEV)
        if causal:
            seen &= j <= own
        if window:
            seen &= j > own - window
        for h in range(hq):
            kh, vh, qh = k[:, h // group], v[:, h // group], q[t0:t1, h].double()
            s = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
            z = torch.logsumexp(s, -1)
            p = torch.where(seen, (s - z[:, None]).exp(), torch.zeros_like(s))
            p[z == -math.inf] = 0
            o[t0:t1, h], lse[t0:t1, h] = p @ vh, z
            mag, top = p @ vh.abs(), vh.abs().amax()
            e = d * 2.0 ** -23 * abs(scale) * ((qh.abs() @ kh.abs().T) * seen).amax(-1)
            e = e + abs(scale) * qh.abs().sum(-1) * 2.0 ** -38 * kh.abs().amax()
            u = U[q.dtype]
            tol_o[t0:t1, h] = u * (p @ vh).abs() + ((2.0 ** -11 + 2 * e + 2.0 ** -17)[:, None] * mag
                                                    + (n * 2.0 ** -25 * top + 2.0 ** -38 * top))
            if q.dtype == FP:
                tol_o[t0:t1, h] += 2.0 ** -25  # the output's subnormal numbers
            tol_l[t0:t1, h] = e + 2.0 ** -17 * (1 + z.nan_to_num(0, 0, 0).abs())
    return o, lse, tol_o, tol_l


ATTEND = [  # new, lens, q heads, key heads, d, page, dtype, causal, window
    ([1], [1], 1, 1, 16, 16, BF, True, 0),
    ([1, 1, 1], [611, 17, 2], 32, 32, 128, 16, BF, True, 0),
    ([1] * 6, [300, 1, 128, 129, 4000, 16], 28, 4, 128, 64, BF, True, 0),
    ([1, 0, 1], [5000, 77, 0], 8, 1, 64, 32, FP, True, 0),
    ([1, 1], [20011, 333], 5, 1, 128, 256, BF, True, 0),
    ([3, 1, 2], [33, 1000, 2], 28, 4, 128, 16, FP, True, 0),
    ([5, 5, 5], [1003, 70, 5], 28, 4, 128, 32, BF, True, 0),
    ([2, 7, 1], [900, 8, 444], 4, 2, 96, 16, BF, True, 100),
    ([4, 4], [129, 260], 4, 4, 80, 128, FP, False, 0),
    ([1, 9, 40], [50, 9, 41], 6, 2, 48, 64, BF, True, 7),
    ([130, 1, 57], [130, 500, 1100], 8, 2, 64, 16, BF, True, 0),
    ([227, 227], [227, 227], 4, 4, 128, 16, BF, True, 0),
    ([784, 100], [1000, 6272], 14, 2, 128, 128, FP, True, 0),
    ([300, 17, 129], [300, 3000, 9000], 4, 4, 64, 32, FP, True, 513),
    ([65, 300], [1200, 301], 7, 1, 112, 64, BF, False, 200),
    ([600], [12345], 8, 1, 128, 64, BF, True, 0),
    ([40, 200], [30, 100], 2, 1, 128, 16, BF, True, 0),   # more new tokens than keys: the first see nothing
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "-".join(str(v) for v in c[2:6]) + f"-{max(c[0])}of{max(c[1])}")
def test_attend(case):
    new, lens, hq, hk, d, page, dtype, causal, window = case
    table, pages = _table(lens, page, 1)
    c = _cache(pages, hk, page, d, 2)
    _spoil(c, table, lens)
    cu = _cum(new)
    rows = 2  # of no sequence, behind the last
    q = _randn(cu[-1] + rows, hq + 1, d, dtype=dtype, seed=3, gain=1.5)[:, 1:]  # strided
    o, lse = c.attend(q, table, _i32(lens), _i32(cu), causal=causal, window=window, max_new=max(new), max_len=max(lens),
                      return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, cu, causal=causal, window=window)
    _within(o, ro, to, "o")
    none = rl == -math.inf
    assert torch.equal(lse == -math.inf, none) and (o[none] == 0).all()
    _within(lse[~none], rl[~none], tl[~none], "lse")
    assert int(c.error) == 0


@pytest.mark.parametrize("new", [1, 3, 40, 300])
@pytest.mark.parametrize("spread", [8, 20])
def test_scales_of_any_size_side_by_side(new, spread):
    lens, page, hq, hk, d = [new + 700, new + 35], 16, 8, 2, 128
    table, pages = _table(lens, page, 11)
    c = _cache(pages, hk, page, d, 12, spread)
    _spoil(c, table, lens)
    q, cu = _randn(2 * new, hq, d, dtype=BF, seed=13, gain=2.0 ** -spread), [0, new, 2 * new]
    o, lse = c.attend(q, table, _i32(lens), _i32(cu), max_new=new, max_len=max(lens), return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, cu)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [2, 5, 40, 300])
@pytest.mark.parametrize("power", [30, 90])
def test_values_that_a_row_does_not_see_take_none_of_its_bits(new, power):
    """Key blocks before every row's window and the last one, which the last rows alone see, 2^power times the others;
    and a block of zeros.  The tolerance is that of the keys that a row sees."""
    lens, page, hq, hk, d, window = [640 + new], 16, 8, 2, 128, 600
    table, pages = _table(lens, page, 61)
    c = _cache(pages, hk, page, d, 62)
    n, group = lens[0], hq // hk
    at = table[0].long()
    last = (n - 1) // 16
    _bytes(c.v_scale)[at[0]] += power
    _bytes(c.v_scale)[at[last]] += power
    _bytes(c.v)[at[20]], _bytes(c.v_scale)[at[20]] = 0, 10
    q = _randn(new, hq, d, dtype=BF, seed=63)
    o, lse = c.attend(q, table, _i32(lens), _i32([0, new]), window=window, return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, [0, new], window=window)
    few = n - new + torch.arange(new, device=DEV) < 16 * last  # rows without a large key
    own = (n - new + torch.arange(new, device=DEV))[few, None]
    j = torch.arange(n, device=DEV)
    seen = (j <= own) & (j > own - window)
    k, v = (_held(x, s, table, 0, n) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    for h in range(hq):
        kh, vh, qh = k[:, h // group], v[:, h // group], q[few, h].double()
        s = (qh @ kh.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
        p, mag = torch.softmax(s, -1), vh.abs().amax(-1)
        e = d * 2.0 ** -23 / math.sqrt(d) * ((qh.abs() @ kh.abs().T) * seen).amax(-1)
        e = e + qh.abs().sum(-1) * 2.0 ** -38 * kh.abs().amax() / math.sqrt(d)
        most = (p * mag).amax(-1)  # what the greatest key adds (its block's largest code is 448: within 2 of it)
        to[few, h] = U[BF] * (p @ vh).abs() + ((2.0 ** -11 + 2 * e + 2.0 ** -17)[:, None] * (p @ vh.abs())
                                               + (n * 2.0 ** -25 * 2 * most)[:, None])
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [1, 2, 200])
@pytest.mark.parametrize("power", [-110, -60, 60, 100])
def test_values_far_from_one(new, power):
    """All values 2^power times the usual, and queries that bring the scores back."""
    lens, page, hq, hk, d = [new + 200], 32, 4, 2, 64
    table, pages = _table(lens, page, 21)
    c = _cache(pages, hk, page, d, 22)
    for s in (c.k_scale, c.v_scale):
        _bytes(s).add_(power) if power > 0 else _bytes(s).sub_(-power)
    q = (_randn(new, hq, d, dtype=torch.float32, seed=23) * 2.0 ** -power).to(BF)
    o, lse = c.attend(q, table, _i32(lens), _i32([0, new]), return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, [0, new])
    _within(o, ro, to + 2.0 ** -126, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [1, 4, 150])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales_of_the_scores(new, scale):
    lens, page, hq, hk, d = [new + 99, new], 16, 6, 2, 64
    table, pages = _table(lens, page, 31)
    c = _cache(pages, hk, page, d, 32)
    q, cu = _randn(2 * new, hq, d, dtype=FP, seed=33), [0, new, 2 * new]
    o, lse = c.attend(q, table, _i32(lens), _i32(cu), scale=scale, return_lse=True)
    ro, rl, to, tl = _reference(c, q, table, lens, cu, scale=scale)
    _within(o, ro, to, "o")
    _within(lse, rl, tl, "lse")


@pytest.mark.parametrize("new", [1, 3, 30, 400])
@pytest.mark.parametrize("d", [64, 128])
def test_not_a_number_reaches_the_rows_that_see_it_and_no_others(new, d):
    lens, page, hq, hk, window = [900, new + 3], 16, 8, 2, 60
    table, pages = _table(lens, page, 41)
    c = _cache(pages, hk, page, d, 42)
    clean = _bytes(c.v).clone()
    cu = [0, new, 2 * new]
    spots = [(0, 899), (0, 880), (0, 900 - new - 10), (0, 500), (1, 1), (1, new + 2)]  # (sequence, key)
    for b, j in spots:
        if 0 <= j < lens[b]:
            _bytes(c.v)[table[b, j // page].long(), 1, j % page, (7 * j) % d] = 0xff
    q = _randn(2 * new, hq, d, dtype=BF, seed=43)
    o = c.attend(q, table, _i32(lens), _i32(cu), window=window, max_new=new, max_len=900)
    want = torch.zeros(2 * new, hq, d, dtype=torch.bool, device=DEV)
    for b, j in spots:
        if 0 <= j < lens[b]:
            own = lens[b] - new + torch.arange(new, device=DEV)
            sees = (own >= j) & (j > own - window)
            want[cu[b]:cu[b + 1], hq // 2:, (7 * j) % d] |= sees[:, None]
    assert torch.equal(o.isnan(), want)
    _bytes(c.v).copy_(clean)
    ro, _, to, _ = _reference(c, q, table, lens, cu, window=window)
    keep = ~want
    _within(o[keep], ro[keep], to[keep], "rows that do not see it")
    # a key that is not a number: every channel of the rows that see it
    _bytes(c.k)[table[0, 895 // page].long(), 0, 895 % page, 3] = 0x7f
    o, lse = c.attend(q, table, _i32(lens), _i32(cu), window=window, max_new=new, max_len=900, return_lse=True)
    own = 900 - new + torch.arange(new, device=DEV)
    want = torch.zeros(2 * new, hq, dtype=torch.bool, device=DEV)
    want[:new, :hq // 2] = ((own >= 895) & (895 > own - window))[:, None]
    assert torch.equal(lse.isnan(), want) and torch.equal(o.isnan().all(-1), want) and torch.equal(o.isnan().any(-1), want)


@pytest.mark.parametrize("new", [1, 4, 200])
def test_pages_outside_the_cache_read_as_zeros_and_are_told(new):
    lens, page, hq, hk, d = [new + 300, new + 40], 16, 4, 2, 64
    table, pages = _table(lens, page, 51)
    c = _cache(pages, hk, page, d, 52)
    q, cu = _randn(2 * new, hq, d, dtype=BF, seed=53), [0, new, 2 * new]
    table[0, 3], table[1, 1] = pages, -1
    o = c.attend(q, table, _i32(lens), _i32(cu), max_new=new)
    assert int(c.error) == 1
    ro, _, to, _ = _reference(c, q, table, lens, cu)
    _within(o, ro, to, "o")
    c.error.zero_()  # pages that no window reaches may be given away
    c.attend(q[:new], table[:1], _i32(lens[:1]), _i32(cu[:2]), max_new=new, window=lens[0] - new - 64)
    assert int(c.error) == 0


def test_no_sequences_no_tokens_no_keys():
    c = _cache(4, 2, 16, 64, 61)
    q = _randn(3, 4, 64, dtype=BF, seed=62)
    none = torch.empty(0, 5, dtype=torch.int32, device=DEV)
    o, lse = c.attend(q, none, _i32([]), _i32([0]), return_lse=True)
    assert (o == 0).all() and (lse == -math.inf).all()
    assert c.attend(q[:0], none, _i32([]), _i32([0])).shape == (0, 4, 64)
    o = c.attend(q, torch.empty(1, 0, dtype=torch.int32, device=DEV), _i32([3]), _i32([0, 3]))
    assert (o == 0).all()
    # the workspace and the launch bounds may be off: only time changes
    table = _i32([[0, 1, 2]])
    a = c.attend(q, table, _i32([40]), _i32([0, 3]), max_new=1, max_len=1)
    ro, _, to, _ = _reference(c, q, table, [40], [0, 3])
    _within(a, ro, to, "bounds that are off")


# ---------------------------------------------------------------- append
def _e4m3(x):
    """The nearest codes' values of float64 (ties to even, 448 at most)."""
    e = torch.frexp(x)[1] - 1
    step = torch.exp2(e.clamp(min=-6).double() - 3)
    return torch.where(x.isnan(), x, (torch.round(x / step) * step).clamp(-448, 448))


def _needed(top):
    """The least exponent with top <= 448 2^e, of a float."""
    if top == 0:
        return -117
    m, e = math.frexp(top)
    return min(max(e - 9 + (m > 0.875), -117), 119)


def _append_ref(codes, scale, rows, table, lens, new):
    """codes and exponents after the append of float64 rows [T, heads, d], block by block, plainly."""
    held, power = codes.double(), _bytes(scale).int().cpu() - 127
    page, heads = codes.shape[2], codes.shape[1]
    cu, tab = _cum(new), table.cpu()
    for b, n in enumerate(new):
        at, end = lens[b] - n, lens[b]
        first = at
        while at < end:
            stop = min(end, (at // 16 + 1) * 16)
            home, slot, old = int(tab[b, at // page]), at % page, at % 16
            x = rows[cu[b] + at - first:cu[b] + stop - first]
            tops = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax((0, 2)).tolist()
            for h in range(heads):
                before, e = int(power[home, h, slot // 16]), _needed(tops[h])
                if old:
                    e = max(e, before)
                    held[home, h, slot - old:slot] = _e4m3(held[home, h, slot - old:slot] * 2.0 ** (before - e))
                power[home, h, slot // 16] = e
                y = torch.where(x[:, h].isfinite(), x[:, h] * 2.0 ** -e, math.nan)
                held[home, h, slot:slot + stop - at] = _e4m3(y)
            at = stop
    return held, power.to(DEV)


APPEND = [  # new, lens, key heads, d, page, dtype
    ([1], [1], 1, 16, 16, BF),
    ([1] * 5, [16, 17, 18, 31, 32], 4, 128, 16, BF),
    ([3, 0, 20], [19, 40, 33], 2, 64, 32, FP),
    ([16, 17, 18, 33], [31, 32, 47, 33], 3, 80, 64, BF),
    ([250, 1], [300, 1000], 5, 96, 128, FP),
    ([100, 47], [100, 300], 8, 128, 256, BF),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(v) for v in c[2:5]))
def test_append_is_exact_without_arithmetic(case):
    new, lens, hk, d, page, dtype = case
    table, pages = _table(lens, page, 71)
    c = _cache(pages, hk, page, d, 72, spread=3)
    rows = _randn(sum(new) + 2, 2 * hk, d, dtype=dtype, seed=73, gain=0.7)  # two rows of no sequence
    k, v = rows[:, :hk], rows[:, hk:]
    want = [_append_ref(x, s, y.double(), table, lens, new) for x, s, y in ((c.k, c.k_scale, k), (c.v, c.v_scale, v))]
    assert c.append(k, v, table, _i32(lens), _i32(_cum(new))) is None
    for (held, power), x, s in zip(want, (c.k, c.v), (c.k_scale, c.v_scale)):
        assert torch.equal(_bytes(s).int() - 127, power)
        assert torch.equal(x.double(), held)
    assert int(c.error) == 0
    # the same call again changes nothing
    before = [_bytes(x).clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    c.append(k, v, table, _i32(lens), _i32(_cum(new)))
    assert all(torch.equal(_bytes(x), y) for x, y in zip((c.k, c.v, c.k_scale, c.v_scale), before))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_append_of_every_magnitude(dtype):
    """Zeros, subnormal, largest, infinite and not-a-number rows; blocks that grow by far."""
    hk, d, page = 2, 32, 16
    top = torch.finfo(dtype).max
    sizes = [0.0, torch.finfo(dtype).smallest_normal / 4, 1e-3, 448.0, 449.0, 464.0, 1.0, 3e4, top, math.inf, math.nan, 2.0]
    lens, new = [len(sizes)], [len(sizes)]
    table = _i32([[0, 1]])
    c = _cache(2, hk, page, d, 81)
    x = _randn(len(sizes), hk, d, dtype=torch.float32, seed=82).clamp(-1, 1)
    x[:, :, 0] = 1
    x = torch.stack([x[i] * s for i, s in enumerate(sizes)]).to(dtype)
    for i in range(len(sizes)):  # one at a time: the block's scale grows
        want = [_append_ref(y, s, z.double(), table, [i + 1], [1]) for y, s, z in
                ((c.k, c.k_scale, x[i:i + 1]), (c.v, c.v_scale, -x[i:i + 1]))]
        c.append(x[i:i + 1], -x[i:i + 1], table, _i32([i + 1]), _i32([0, 1]))
        for (held, power), y, s in zip(want, (c.k, c.v), (c.k_scale, c.v_scale)):
            assert torch.equal(_bytes(s).int() - 127, power), i
            assert torch.equal(y.double().nan_to_num(-5), held.nan_to_num(-5)), i
    # all at once: the largest finite one sets the scale
    c.append(x, x, table, _i32(lens), _i32([0, len(sizes)]))
    held, power = _append_ref(c.k, c.k_scale, x.double(), table, lens, new)
    assert torch.equal(c.k.double().nan_to_num(-5), held.nan_to_num(-5)) and torch.equal(_bytes(c.k_scale).int() - 127, power)


ROTATED = [  # new, lens, q heads, key heads, d, rot, page, sections, layout, dtype, norm
    ([1, 1, 1], [700, 16, 17], 28, 4, 128, 128, 16, (16, 24, 24), "half", BF, False),
    ([300, 5], [300, 105], 28, 4, 128, 128, 64, (16, 24, 24), "half", BF, True),
    ([61, 40], [68, 1000], 4, 4, 64, 64, 32, (32,), "pairs", FP, False),
    ([33, 2], [40, 18], 6, 3, 80, 40, 16, (10, 10), "half", FP, True),
    ([20, 20], [25, 20], 5, 1, 96, 48, 128, (24,), "pairs", BF, True),
    ([7], [9], 0, 2, 16, 8, 16, (4,), "half", BF, True),
]


@pytest.mark.parametrize("case", ROTATED, ids=lambda c: "-".join(str(v) for v in c[2:7]) + c[8])
def test_append_norms_and_rotates(case):
    new, lens, hq, hk, d, rot, page, sections, layout, dtype, norm = case
    altr = _alt()
    t, eps = sum(new), 1e-5
    table, pages = _table(lens, page, 91)
    c = _cache(pages, hk, page, d, 92)
    rows = _randn(t, hq + 2 * hk, d, dtype=dtype, seed=93, gain=2.0)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    g = torch.Generator().manual_seed(94)
    pos = torch.randint(-3, 100000, (len(sections), t), generator=g).to(torch.int32).to(DEV)
    wq, wk = (1 + 0.3 * _randn(d, dtype=torch.float32, seed=s) if norm else None for s in (95, 96))
    rotary = altr.Rotary(d, DEV, base=1e6, rot_dim=rot, sections=sections, layout=layout)
    old = [x.double().clone() for x in (c.k, c.v)]
    old_scale = [_bytes(s).int().clone() for s in (c.k_scale, c.v_scale)]
    want_v = _append_ref(c.v, c.v_scale, v.double(), table, lens, new)
    got = c.append(k, v, table, _i32(lens), _i32(_cum(new)), rotary=rotary, pos=pos, k_weight=wk, q=q if hq else None,
                   q_weight=wq if hq else None, eps=eps)
    if hq:  # the queries as Rotary.apply gives them, bit for bit
        assert torch.equal(got, rotary.apply(q, None, pos, q_weight=wq, eps=eps)[0])
    assert torch.equal(c.v.double(), want_v[0]) and torch.equal(_bytes(c.v_scale).int() - 127, want_v[1])
    # keys in 64 bits
    x = k.double()
    if norm:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * wk.double()
    half = rot // 2
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device=DEV)
    theta = pos[axis].double().T * torch.tensor([1e6 ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
    i = torch.arange(half, device=DEV)
    a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
    cos, sin = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    y, mag = x.clone(), x.abs().clone()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    touched = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
    cu = _cum(new)
    for s, n in enumerate(new):
        key = lens[s] - n + torch.arange(n, device=DEV)
        home = table[s].long()[key // page]
        touched[home, key % page] = True
        sc = torch.exp2(_bytes(c.k_scale).double() - 127)[home, :, key % page // 16]  # [n, heads]
        held = c.k.double()[home, :, key % page] * sc[..., None]
        ref = y[cu[s]:cu[s + 1]]
        _within(held, ref, 2.0 ** -4 * ref.abs() + 2.0 ** -10 * sc[..., None] + 2 * 2.0 ** -19 * mag[cu[s]:cu[s + 1]] + 2.0 ** -20,
                "keys")
        for blk in sorted(set((key // 16).tolist())):
            mine = key // 16 == blk
            top = ref[mine].abs().amax((0, 2))
            p, sub = int(table[s, blk * 16 // page]), blk * 16 % page // 16
            for h in range(hk):
                lo, hi = (_needed(float(top[h]) * f) for f in (1 - 2.0 ** -18, 1 + 2.0 ** -18))
                before = int(old_scale[0][p, h, sub]) - 127
                if blk * 16 < lens[s] - n:
                    lo, hi = max(lo, before), max(hi, before)
                e = int(_bytes(c.k_scale)[p, h, sub]) - 127
                assert lo <= e <= hi
                if blk * 16 < lens[s] - n:  # older keys of the block
                    r0 = (lens[s] - n) % 16
                    sl = slice(sub * 16, sub * 16 + r0)
                    assert torch.equal(c.k.double()[p, h, sl], _e4m3(old[0][p, h, sl] * 2.0 ** (before - e)))
                    touched[p, sl] = True
    for now, was in ((c.k, old[0]), (c.v, old[1])):  # nothing else is written
        assert torch.equal(now.double().transpose(1, 2)[~touched], was.transpose(1, 2)[~touched])


@pytest.mark.parametrize("hk,d,layout,dtype,norm", [(3, 128, "half", BF, True), (5, 64, "pairs", FP, False), (1, 48, "half", BF, True)])
def test_append_of_many_sequences_as_of_few(hk, d, layout, dtype, norm):
    """Bit for bit what calls of 100 sequences each leave (which take other CTAs for it)."""
    altr, hq, page, batch = _alt(), 3, 32, 701
    g = torch.Generator().manual_seed(97)
    new = torch.randint(0, 41, (batch,), generator=g).tolist()
    lens = [n + int(p) for n, p in zip(new, torch.randint(0, 51, (batch,), generator=g))]
    cu, t = _cum(new), sum(new)
    table, pages = _table(lens, page, 98)
    table[400, 0] = pages  # outside the cache
    one, few = _cache(pages, hk, page, d, 99), _cache(pages, hk, page, d, 99)
    rows = _randn(t + 5, hq + 2 * hk, d, dtype=dtype, seed=100)  # five rows of no sequence
    q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
    pos = torch.randint(0, 5000, (2, t + 5), generator=g).to(torch.int32).to(DEV)
    wq, wk = (1 + 0.3 * _randn(d, dtype=torch.float32, seed=x) if norm else None for x in (101, 102))
    rotary = altr.Rotary(d, DEV, sections=(d // 4, d // 4), layout=layout)
    got = one.append(k, v, table, _i32(lens), _i32(cu), rotary=rotary, pos=pos, k_weight=wk, q=q, q_weight=wq)
    for b0 in range(0, batch, 100):
        b1 = min(b0 + 100, batch)
        r = slice(cu[b0], cu[b1])
        part = few.append(k[r], v[r], table[b0:b1], _i32(lens[b0:b1]), _i32([x - cu[b0] for x in cu[b0:b1 + 1]]), rotary=rotary,
                          pos=pos[:, r].contiguous(), k_weight=wk, q=q[r], q_weight=wq)
        assert torch.equal(got[r], part)
    for a, b in zip((one.k, one.v, one.k_scale, one.v_scale), (few.k, few.v, few.k_scale, few.v_scale)):
        assert torch.equal(_bytes(a), _bytes(b))
    assert int(one.error) == int(few.error) != 0


def test_append_outside_the_cache_writes_nothing_and_is_told():
    c = _cache(3, 2, 16, 64, 101)
    before = [_bytes(x).clone() for x in (c.k, c.v, c.k_scale, c.v_scale)]
    rows = _randn(4, 2, 64, dtype=BF, seed=102)
    for table, lens in (([[-1, 3]], [20]), ([[0, 1]], [40]), ([[0, 1]], [2])):
        c.error.zero_()
        keep = _i32(table)
        # the 4 new tokens: pages outside, keys past the table, two tokens without a key
        c.append(rows, rows, keep, _i32(lens), _i32([0, 4]))
        assert int(c.error) == 1
        if lens != [2]:
            assert all(torch.equal(_bytes(x), y) for x, y in zip((c.k, c.v, c.k_scale, c.v_scale), before))
    held, power = _append_ref(before[0].view(torch.float8_e4m3fn), before[2], rows[2:].double(), _i32([[0, 1]]), [2], [2])
    assert torch.equal(c.k.double(), held) and torch.equal(_bytes(c.k_scale).int() - 127, power)
    c.error.zero_()
    none = torch.empty(0, 5, dtype=torch.int32, device=DEV)
    c.append(rows, rows, none, _i32([]), _i32([0]))
    c.append(rows[:0], rows[:0], none, _i32([]), _i32([0]))
    assert int(c.error) == 0


# ---------------------------------------------------------------- together
def test_prompt_then_single_tokens_in_a_captured_step():
    """Tables, append and attention as a serving loop uses them: a prompt in two
    chunks, then drafts of which some are refused, on a stream of its own, as a
    captured graph; against the same keys and values in 64 bits."""
    altr = _alt()
    batch, hq, hk, d, page, rows = 3, 8, 2, 64, 16, 12
    pages = altr.PageTable(batch, 20, 40, page, DEV)
    c = _cache(40, hk, page, d, 111)
    rotary = altr.Rotary(d, DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for chunk in ([37, 5, 16], [20, 0, 3]):
            t = sum(chunk) + 1
            x = _randn(t, hq + 2 * hk, d, dtype=BF, seed=112 + t)
            s = pages.extend(_i32(chunk), t)
            q = c.append(x[:, hq:hq + hk], x[:, hq + hk:], pages.table, pages.lens, s.cu_new, rotary=rotary, pos=s.pos,
                         q=x[:, :hq])
            o = c.attend(q, pages.table, pages.lens, s.cu_new)
            side.synchronize()
            lens, cu = pages.lens.tolist(), s.cu_new.tolist()
            ro, _, to, _ = _reference(c, q, pages.table, lens, cu)
            _within(o, ro, to, "chunk")
            # a slot is where the row's key lies
            slot, ok = s.slots.long(), s.slots >= 0
            assert ok.tolist() == [True] * (t - 1) + [False]
            held = c.v.transpose(1, 2).reshape(-1, hk, d).double()[slot[:-1]]
            sc = torch.exp2(_bytes(c.v_scale).double() - 127).repeat_interleave(16, 2).transpose(1, 2).reshape(-1, hk)[slot[:-1]]
            v = x[:-1, hq + hk:].double()
            _within(held * sc[..., None], v, 2.0 ** -4 * v.abs() + 2.0 ** -10 * sc[..., None], "slots")
        new, keep = _i32([1, 1, 1]), pages.lens.clone()
        x = _randn(rows, hq + 2 * hk, d, dtype=BF, seed=119)

        def step():
            pages.truncate(keep)
            s = pages.extend(new, rows)
            q = c.append(x[:, hq:hq + hk], x[:, hq + hk:], pages.table, pages.lens, s.cu_new, rotary=rotary,
                         pos=s.pos, q=x[:, :hq])
            return s, q, c.attend(q, pages.table, pages.lens, s.cu_new, max_new=4, max_len=320)

        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s, q, o = step()
        for drafts, kept in (([4, 1, 2], [0, 0, 0]), ([1, 4, 4], [2, 1, 2]), ([0, 3, 1], [0, 4, 0]), ([4, 4, 4], [0, 0, 1])):
            was = pages.lens.tolist()
            base = keep.tolist()
            new.copy_(_i32(drafts))
            keep.copy_(_i32([a + k for a, k in zip(base, kept)]))
            x.copy_(_randn(rows, hq + 2 * hk, d, dtype=BF, seed=sum(drafts)))
            graph.replay()
            side.synchronize()
            lens = [min(w, a + k) + n for w, a, k, n in zip(was, base, kept, drafts)]
            keep.copy_(_i32([n - m for n, m in zip(lens, drafts)]))
            assert pages.lens.tolist() == lens and s.cu_new.tolist() == _cum(drafts)
            ro, _, to, _ = _reference(c, q, pages.table, lens, _cum(drafts))
            _within(o, ro, to, "step")
    assert int(c.error) == 0 and int(pages.error) == 0
    torch.cuda.current_stream().wait_stream(side)


def test_results_do_not_depend_on_the_other_rows():
    """A request alone and among others, and two calls on two streams at once."""
    lens, page, hq, hk, d = [700, 333, 64], 32, 8, 2, 128
    table, pages = _table(lens, page, 121)
    c = _cache(pages, hk, page, d, 122)
    q = _randn(3, hq, d, dtype=BF, seed=123)
    both = c.attend(q, table, _i32(lens), _i32([0, 1, 2, 3]), max_new=1)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for s in (a, b):
            with torch.cuda.stream(s):
                outs.append(c.attend(q, table, _i32(lens), _i32([0, 1, 2, 3]), max_new=1))
    torch.cuda.synchronize()
    assert all(torch.equal(o, both) for o in outs)
    ro, _, to, _ = _reference(c, q, table, lens, [0, 1, 2, 3])
    _within(both, ro, to, "o")
