"""Rows and keys at the edges of tr_cache_attend: values that are not finite,
rows that no sequence owns, pages that no row sees.  The plain implementation,
the steps and the tolerances are those of test_attention_gpu."""
import math

import pytest
import torch

from test_attention_gpu import DEV, U, _alt, _attend_ref, _randn, _step, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt, causal=True, window=0, scale=None, channels=None):
    """Rows [token, head] of `spoilt` are NaN in out and lse, the others as the plain form has them (in `channels`)."""
    d, dtype = q.shape[2], q.dtype
    assert torch.isnan(got[spoilt]).all() and torch.isnan(lse[spoilt]).all()
    for b, (n, length) in enumerate(seqs):
        if n == 0:
            continue
        sl = slice(int(cu[b]), int(cu[b + 1]))
        keep = ~spoilt[sl]
        o, z, pv, e = _attend_ref(q[sl].nan_to_num(0, 0, 0), keys[b], vals[b], n, causal, window,
                                  1 / math.sqrt(d) if scale is None else scale)
        tol = U[dtype] * o.abs() + (U[dtype] + 2 * e + 2.0 ** -17)[..., None] * pv + 2.0 ** -24
        if dtype == torch.float16:
            tol = tol + length * 2.0 ** -25 * vals[b].double().nan_to_num(0, 0, 0).abs().max()
        if channels is not None:
            o = torch.where(channels[sl], o, 0.0)
        _within(got[sl][keep], o[keep], tol[keep], ("o", b))
        _within(lse[sl][keep], z[keep], (e + 2.0 ** -17 * (1 + z.abs()))[keep], ("lse", b))


# Single tokens: items cut into shares (a tile or two each), and whole ones (one tile).
FEW = [
    ([(1, 609), (1, 40)], 32, 32, 128, 16),
    ([(1, 513)], 32, 32, 128, 64),
    ([(1, 33), (1, 17), (1, 100)], 4, 2, 64, 16),
    ([(2, 1025), (1, 300)], 7, 1, 64, 32),
]


@pytest.mark.parametrize("case", FEW, ids=lambda c: f"{c[0][0][1]}-{c[1]}-{c[2]}-{c[3]}")
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_few_rows_nan_query(case, value):
    # one head's query of one token: its row and no other
    seqs, hq, hk, d, page = case
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, torch.bfloat16, 5)
    q = _randn(int(cu[-1]), hq, d, dtype=torch.bfloat16, seed=6, gain=1.5)
    q[0, 1, 5] = value
    spoilt = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    spoilt[0, 1] = True
    got, lse = cache.attend(q, table, lens, cu, max_new=2, return_lse=True)
    _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt)


@pytest.mark.parametrize("case", FEW, ids=lambda c: f"{c[0][0][1]}-{c[1]}-{c[2]}-{c[3]}")
def test_few_rows_nan_key(case):
    # a visible key of NaN, alone in the last 16 keys of its tile: every row that sees it
    seqs, hq, hk, d, page = case
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, torch.bfloat16, 5)
    q = _randn(int(cu[-1]), hq, d, dtype=torch.bfloat16, seed=6, gain=1.5)
    n, length = seqs[0]
    j = length - 1
    assert j % 16 == 0
    cache.k[table[0, j // page], 0, j % page, 3] = float("nan")
    spoilt = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    spoilt[n - 1, :hq // hk] = True  # the last token of the first sequence, the first key head's rows
    got, lse = cache.attend(q, table, lens, cu, max_new=2, return_lse=True)
    _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt)


def _check_bad_keys(seqs, hq, hk, d, page, dtype, bad, window=0, scale=None, repeats=1, **kw):
    """Keys `bad` (counted back from each sequence's end, 1 = the last) are NaN, their values infinite: rows that see
    one are NaN, the others as if it did not exist, and the same bits on every call."""
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, dtype, 5)
    q = _randn(int(cu[-1]), hq, d, dtype=dtype, seed=6, gain=1.5)
    spoilt = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    for b, (n, length) in enumerate(seqs):
        own = length - n + torch.arange(n, device=DEV)
        for j in (length - back for back in bad if back <= length):
            cache.k[table[b, j // page], :, j % page] = float("nan")
            cache.v[table[b, j // page], :, j % page] = float("inf") if j % 2 else float("-inf")
            keys[b][j] = vals[b][j] = 0
            spoilt[int(cu[b]):int(cu[b + 1])] |= ((own >= j) & ((own < j + window) if window else own >= 0))[:, None]
    assert not spoilt.all()
    got, lse = cache.attend(q, table, lens, cu, window=window, scale=scale, return_lse=True, **kw)
    _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt, window=window, scale=scale)
    for _ in range(repeats - 1):
        again, lse2 = cache.attend(q, table, lens, cu, window=window, scale=scale, return_lse=True, **kw)
        for x, y in ((again, got), (lse2, lse)):
            assert torch.equal(x.nan_to_num(9), y.nan_to_num(9))
    assert int(cache.error) == 0


CHUNKS = [  # sequences, q heads, k heads, d, page, dtype, window, scale, max_len
    ([(40, 1000), (90, 1111)], 4, 2, 64, 32, torch.bfloat16, 0, None, 1111),     # the keys in parts, joined
    ([(300, 2000)], 7, 1, 128, 64, torch.float16, 0, -0.2, 2000),
    ([(200, 1500)], 4, 2, 80, 16, torch.bfloat16, 100, None, 1500),
    ([(150, 150), (33, 500)], 4, 2, 64, 32, torch.bfloat16, 0, None, 500),       # in one part
    ([(300, 700)] * 16, 7, 1, 128, 64, torch.bfloat16, 0, 0.1, 700),
    ([(100, 700)] * 40, 8, 4, 64, 64, torch.float16, 90, None, 700),
]


@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}of{c[0][0][1]}-{c[3]}-w{c[6]}")
def test_chunk_rows_without_hidden_bad_keys(case):
    # rows taken again: their partial results and statistics are the second ones, on every call
    seqs, hq, hk, d, page, dtype, window, scale, max_len = case
    _check_bad_keys(seqs, hq, hk, d, page, dtype, (2, 9, 30), window=window, scale=scale, repeats=10,
                    max_new=max(n for n, _ in seqs), max_len=max_len)


FEW_BAD = [  # sequences, q heads, k heads, d, page, dtype, window, scale
    ([(3, 40), (2, 100), (1, 33)], 4, 2, 64, 16, torch.bfloat16, 0, None),           # whole items
    ([(4, 3000)], 4, 1, 128, 64, torch.bfloat16, 0, -0.15),                          # one item in many shares
    ([(2, 700), (2, 1300), (0, 9), (2, 64)], 28, 4, 128, 16, torch.float16, 0, None),
    ([(4, 400), (3, 130)] * 120, 4, 1, 64, 32, torch.bfloat16, 0, None),             # several items in a share
    ([(1, 333), (1, 1000), (1, 5000)], 8, 2, 80, 16, torch.bfloat16, 7, None),       # below the window
    ([(1, 250), (2, 900)] * 90, 8, 2, 64, 64, torch.float16, 20, -0.3),
]


@pytest.mark.parametrize("case", FEW_BAD, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}of{c[0][0][1]}-{c[3]}-w{c[6]}")
def test_few_rows_without_hidden_bad_keys(case):
    seqs, hq, hk, d, page, dtype, window, scale = case
    most = max(n for n, _ in seqs)
    bad = (window + 4, window + 9) if window else (1, 2)[:most - 1]  # a draft's first token sees none of them
    _check_bad_keys(seqs, hq, hk, d, page, dtype, bad, window=window, scale=scale, repeats=5, max_new=most)


def test_few_rows_taken_again_over_a_long_history():
    # 160 requests over the same pages, drafts of four tokens, an infinity in the last value: three tokens of each
    # are taken again over 800 000 keys while the rest of the step goes on.  The rows' sums are chains of at most
    # `length` additions in 32 bits.
    batch, length, page, d, hq = 160, 800000, 256, 64, 4
    g = torch.Generator(device=DEV).manual_seed(1)
    pages = length // page + 1
    k, v = (torch.randn(pages, 1, page, d, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    v[(length - 1) // page, 0, (length - 1) % page] = float("inf")
    cache = _alt().PagedCache(k, v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(batch, 1)
    lens = torch.full((batch,), length, dtype=torch.int32, device=DEV)
    cu = 4 * torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    q = _randn(4, hq, d, dtype=torch.bfloat16, seed=6)
    got, lse = cache.attend(q.repeat(batch, 1, 1), table, lens, cu, max_new=4, return_lse=True)
    assert int(cache.error) == 0
    got, lse = got.view(batch, 4, hq, d), lse.view(batch, 4, hq)
    keys, vals = k.reshape(-1, 1, d)[:length], v.reshape(-1, 1, d)[:length]
    o, z, pv, e = _attend_ref(q, keys, vals, 4, True, 0, 1 / math.sqrt(d))
    sums = 2.0 ** -17 + length * 2.0 ** -24
    tol = U[torch.bfloat16] * o.abs() + (U[torch.bfloat16] + 2 * e + sums)[..., None] * pv + 2.0 ** -24
    for b in range(batch):
        _within(got[b, :3], o[:3], tol[:3], ("o", b))
        _within(lse[b], z, e + sums * (1 + z.abs()), ("lse", b))
        assert not torch.isfinite(got[b, 3]).any()  # the token that sees the infinity


UNOWNED = [  # sequences (new, length), rows of the call, q heads, k heads, d, page, max_new, max_len
    ([(1, 50), (1, 300), (1, 17)], 5, 4, 2, 64, 16, 1, 300),      # few rows
    ([(1, 3000)], 2, 7, 1, 128, 64, 1, 3000),
    ([(40, 300), (1, 100)], 45, 14, 2, 128, 16, 40, 400),         # chunks, the keys in one part
    ([(3, 300)], 700, 7, 1, 64, 32, 700, 400),
    ([(127, 200)], 128, 4, 4, 80, 16, 128, 400),
    ([(128, 200)], 129, 4, 4, 80, 16, 128, 400),
    ([(300, 700)] * 16, 5000, 7, 1, 128, 64, 300, 700),
    ([(200, 4000)], 257, 4, 2, 64, 32, 200, 4000),                # in parts
    ([(0, 100), (0, 0)], 150, 4, 2, 64, 32, 100, 100),            # no new token at all
    ([], 3, 4, 2, 64, 16, 1, 100),                                # no sequence
    ([], 300, 4, 2, 64, 16, 300, 100),
]


@pytest.mark.parametrize("case", UNOWNED, ids=lambda c: f"{len(c[0])}seqs-{c[1]}rows-{c[2]}-{c[3]}-{c[4]}")
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_of_no_sequence_come_out_as_zeros(case, dtype):
    # more rows than cu_new hands out: the same zeros whichever kernel takes the call
    seqs, rows, hq, hk, d, page, max_new, max_len = case
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, dtype, 5)
    q = _randn(rows, hq, d, dtype=dtype, seed=6, gain=1.5)
    wide = torch.full((rows, hq + 1, d), 7.0, dtype=dtype, device=DEV)
    got, lse = cache.attend(q, table, lens, cu, max_new=max_new, max_len=max_len, return_lse=True, out=wide[:, :hq])
    owned = int(cu[-1])
    assert (got[owned:] == 0).all() and (lse[owned:] == -math.inf).all()
    assert (wide[:, hq] == 7).all()
    spoilt = torch.zeros(rows, hq, dtype=torch.bool, device=DEV)
    _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt)
    assert int(cache.error) == 0


def test_graph_with_fewer_rows_than_captured():
    # a graph captured for 300 rows serves 300, 40 and none
    cache, table, lens, cu, keys, vals = _step([(300, 900)], 2, 32, 64, torch.bfloat16, 5)
    q = _randn(300, 8, 64, dtype=torch.bfloat16, seed=6, gain=1.5)
    out = torch.empty_like(q)
    cache.attend(q, table, lens, cu, max_new=300, max_len=600, out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(q, table, lens, cu, max_new=300, max_len=600, out=out)
    for n in (300, 40, 0):
        cu[1] = n
        g.replay()
        assert (out[n:] == 0).all()
        if n:
            o, _, pv, e = _attend_ref(q[:n], keys[0], vals[0], n, True, 0, 1 / 8)
            _within(out[:n], o, U[torch.bfloat16] * o.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv
                    + 2.0 ** -24, n)


@pytest.mark.parametrize("seqs", [[(20, 100), (3, 40)], []])
def test_append_rows_of_no_sequence(seqs):
    # their keys and values go nowhere, their queries are turned all the same
    altr = _alt()
    cache, table, lens, cu, _, _ = _step(seqs, 2, 16, 64, torch.bfloat16, 5, stale=3.0)
    rows = _randn(40, 8, 64, dtype=torch.bfloat16, seed=6)
    q, k, v = rows[:, :4], rows[:, 4:6], rows[:, 6:]
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    r = altr.Rotary(64, DEV)
    want_k, want_v = cache.k.clone(), cache.v.clone()
    rq, rk = r.apply(q, k, pos)
    for b, (n, length) in enumerate(seqs):
        for i in range(n):
            j = length - n + i
            want_k[table[b, j // 16], :, j % 16] = rk[int(cu[b]) + i]
            want_v[table[b, j // 16], :, j % 16] = v[int(cu[b]) + i]
    out = torch.full_like(q, 7.0)
    got = cache.append(k, v, table, lens, cu, rotary=r, pos=pos, q=q, q_out=out)
    assert torch.equal(got, rq)
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
    assert int(cache.error) == 0


GIVEN_AWAY = [  # sequences, q heads, k heads, page, window
    ([(1, 300), (1, 1000), (1, 40)], 4, 2, 16, 50),       # few rows
    ([(3, 2000)], 4, 1, 32, 129),
    ([(1, 70)], 8, 8, 16, 1),
    ([(40, 300), (90, 1500)], 4, 2, 16, 50),              # chunks
    ([(300, 2000)], 7, 1, 64, 500),
    ([(33, 200)] * 30, 4, 4, 128, 20),
]


@pytest.mark.parametrize("case", GIVEN_AWAY, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}of{c[0][0][1]}-p{c[3]}-w{c[4]}")
@pytest.mark.parametrize("gone", [-1, 2 ** 31 - 1])
def test_pages_before_the_window_may_be_given_away(case, gone):
    # table entries that no row's window reaches are no error; the first one that a window reaches is
    seqs, hq, hk, page, window = case
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, 64, torch.bfloat16, 5)
    q = _randn(int(cu[-1]), hq, 64, dtype=torch.bfloat16, seed=6, gain=1.5)
    most = dict(max_new=max(n for n, _ in seqs), max_len=max(n for _, n in seqs))
    first = [max(0, length - n - window + 1) // page for n, length in seqs]  # the page of the first key in a window
    for b, p in enumerate(first):
        table[b, :p] = gone
    got, lse = cache.attend(q, table, lens, cu, window=window, return_lse=True, **most)
    assert int(cache.error) == 0
    spoilt = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    _check_rows(got, lse, q, keys, vals, seqs, cu, spoilt, window=window)
    for b, p in enumerate(first):
        cache.error.zero_()
        kept = int(table[b, p])
        table[b, p] = gone
        cache.attend(q, table, lens, cu, window=window, **most)
        assert int(cache.error) == 1, b
        table[b, p] = kept


VALUES = [  # sequences, q heads, k heads, d, page, dtype, window, max_len
    ([(1, 33), (1, 128), (1, 700)], 4, 2, 64, 16, torch.bfloat16, 0, 700),               # few rows, all see it
    ([(4, 3000)], 4, 1, 128, 64, torch.bfloat16, 0, 3000),
    ([(4, 400), (3, 130), (1, 20)] * 80, 4, 1, 64, 32, torch.float16, 0, 400),
    ([(1, 250), (2, 900)] * 90, 8, 2, 80, 64, torch.float16, 40, 900),
    ([(150, 150), (33, 500)], 4, 2, 64, 32, torch.bfloat16, 0, 500),                     # chunks, two CTAs an SM
    ([(227, 227)] * 20, 8, 8, 128, 16, torch.float16, 0, 227),
    ([(100, 700)] * 40, 8, 4, 64, 64, torch.float16, 90, 700),
    ([(40, 1000), (90, 1111)], 4, 2, 64, 32, torch.bfloat16, 0, 1111),                   # the keys in parts
    ([(300, 2000)], 7, 1, 128, 64, torch.float16, 33, 2000),
    ([(300, 700)] * 16, 7, 1, 128, 64, torch.bfloat16, 0, 700),                          # in one part, 256 rows a CTA
    ([(130, 2000)] * 20, 8, 8, 112, 128, torch.bfloat16, 0, 2000),
    ([(40, 2000)], 4, 1, 128, 64, torch.bfloat16, 0, 100),                               # a bound that is off
]


@pytest.mark.parametrize("case", VALUES, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}of{c[0][0][1]}-{c[3]}-w{c[6]}")
def test_values_that_are_not_finite(case):
    # single channels of a value: infinite or NaN for the rows that see them, in that channel and no other
    seqs, hq, hk, d, page, dtype, window, max_len = case
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, dtype, 5)
    q = _randn(int(cu[-1]), hq, d, dtype=dtype, seed=6, gain=1.5)
    inf, nan = float("inf"), float("nan")
    add = torch.zeros(q.shape, dtype=torch.float64, device=DEV)  # what they make of each channel
    for b, (n, length) in enumerate(seqs):
        own = length - n + torch.arange(n, device=DEV)
        rows = slice(int(cu[b]), int(cu[b + 1]))
        for back, ch, bad in ((1, 3, inf), (2, 3, -inf), (3, d - 1, nan), (7, 8, -inf), (16, 9, inf), (60, 10, inf),
                              (window + n // 2, 11, -inf)):
            if back > length or back < 1:
                continue
            j, head = length - back, back % hk
            cache.v[table[b, j // page], head, j % page, ch] = bad
            vals[b][j, head, ch] = 0
            see = (own >= j) & ((own < j + window) if window else own >= 0)
            group = slice(head * (hq // hk), (head + 1) * (hq // hk))
            add[rows, group, ch] += torch.where(see, bad, 0.0)[:, None]
    got, lse = cache.attend(q, table, lens, cu, window=window, max_new=max(n for n, _ in seqs), max_len=max_len,
                            return_lse=True)
    assert int(cache.error) == 0
    fine = add == 0
    assert torch.equal(got.double()[~fine].nan_to_num(7), add[~fine].nan_to_num(7))
    _check_rows(torch.where(fine, got, got.new_zeros(())), lse, q, keys, vals, seqs, cu,
                torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV), window=window, channels=fine)


@pytest.mark.parametrize("case", [([(4, 50000)] * 160, 4, 1), ([(2048, 8192)], 28, 4)], ids=["drafts", "chunk"])
def test_values_that_are_not_finite_cost_little(case):
    # an infinity that some rows do not see, against the same step without it: a few times as long at most, however
    # long the sequence
    seqs, hq, hk = case
    n, length = seqs[0]
    page, d = 64, 64
    pages = (length + page - 1) // page
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn(pages, hk, page, d, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    cache = _alt().PagedCache(k, v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(len(seqs), 1)  # the same pages for all
    lens = torch.full((len(seqs),), length, dtype=torch.int32, device=DEV)
    cu = n * torch.arange(len(seqs) + 1, dtype=torch.int32, device=DEV)
    q = _randn(n * len(seqs), hq, d, dtype=torch.bfloat16, seed=6)

    def took():
        times = []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            cache.attend(q, table, lens, cu, max_new=n, max_len=length)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    good = took()
    v[pages - 1, :, (length - 1) % page, 5] = float("inf")
    bad = took()
    assert bad <= 4 * good, (good, bad)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 32 + 5])
def test_window_wider_than_any_sequence(window):
    for seqs, new in (([(1, 900), (1, 30)], 1), ([(200, 900), (33, 40)], 200)):
        cache, table, lens, cu, _, _ = _step(seqs, 2, 32, 64, torch.bfloat16, 5)
        q = _randn(int(cu[-1]), 4, 64, dtype=torch.bfloat16, seed=6, gain=1.5)
        assert torch.equal(cache.attend(q, table, lens, cu, max_new=new, window=window),
                           cache.attend(q, table, lens, cu, max_new=new))


def _check_single_tokens(cache, table, lens, q, **kw):
    """One new token of each sequence, all keys short enough for one padded computation."""
    got, lse = cache.attend(q, table, lens, torch.arange(len(lens) + 1, dtype=torch.int32, device=DEV), max_new=1,
                            return_lse=True, **kw)
    assert int(cache.error) == 0
    d, group, n = q.shape[2], q.shape[1] // cache.heads, int(lens.max())
    pages = (n + cache.page - 1) // cache.page
    k, v = (t[table[:, :pages].long()].transpose(1, 2).flatten(2, 3)[:, :, :n].double() for t in (cache.k, cache.v))
    x = q.double().view(len(lens), cache.heads, group, d)
    seen = (torch.arange(n, device=DEV) < lens[:, None])[:, None, None]
    s = (x @ k.transpose(2, 3) / math.sqrt(d)).masked_fill(~seen, -math.inf)
    z = torch.logsumexp(s, -1)
    p = torch.where(seen, torch.exp(s - torch.where(z.isinf(), 0.0, z)[..., None]), 0.0)
    e = torch.where(seen, x.abs() @ k.abs().transpose(2, 3), 0.0).amax(-1) / math.sqrt(d) * d * 2.0 ** -23
    o, pv = p @ v, p @ v.abs()
    u = U[q.dtype]
    _within(got.view(o.shape), o, u * o.abs() + (u + 2 * e + 2.0 ** -17)[..., None] * pv + 2.0 ** -24, "o")
    lse = lse.view(z.shape)
    assert torch.equal(lse.isinf(), z.isinf())
    some = ~z.isinf()
    _within(lse[some], z[some], (e + 2.0 ** -17 * (1 + z.abs()))[some], "lse")


def test_more_sequences_than_shares_are_counted_for():
    # past 8192 sequences single tokens go to the kernel of chunks
    g = torch.Generator(device=DEV).manual_seed(7)
    batch, page, d = 8300, 16, 64
    k, v = (torch.randn(500, 1, page, d, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.randint(0, 500, (batch, 13), device=DEV, generator=g, dtype=torch.int32)
    lens = torch.randint(0, 13 * page + 1, (batch,), device=DEV, generator=g, dtype=torch.int32)
    q = _randn(batch, 2, d, dtype=torch.bfloat16, seed=6, gain=1.5)
    cache = _alt().PagedCache(k, v)
    _check_single_tokens(cache, table, lens, q)
    _check_single_tokens(cache, table[:8192], lens[:8192], q[:8192])  # the most that are


def test_tables_whose_tiles_pass_31_bits():
    # 2 sequences x 80 key heads x 16.8 million tiles that the table could hold: the kernel of chunks again
    g = torch.Generator(device=DEV).manual_seed(7)
    heads, page, d, most = 80, 256, 64, 2 ** 23 - 257
    k, v = (torch.randn(5, heads, page, d, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.full((2, most), -1, dtype=torch.int32, device=DEV)
    table[0, :2], table[1, :3] = torch.tensor([4, 0], device=DEV), torch.tensor([1, 3, 2], device=DEV)
    lens = torch.tensor([300, 517], dtype=torch.int32, device=DEV)
    q = _randn(2, heads, d, dtype=torch.bfloat16, seed=6, gain=1.5)
    cache = _alt().PagedCache(k, v)
    _check_single_tokens(cache, table, lens, q)
    _check_single_tokens(cache, table, lens, q, max_len=517)
