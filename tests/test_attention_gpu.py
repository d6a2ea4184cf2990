"""The attention-layer operators (tr_rotary_apply, tr_rotary_backward,
tr_cache_append, tr_cache_attend) against plain implementations in 64 bits.

Tolerances, with u the output type's unit roundoff (half the spacing at 1:
2^-8 bf16, 2^-11 fp16, 2^-24 fp32), derived from the arithmetic:
* rotation: u |y| for the one rounding; the angle's fixed-point fraction is
  rounded to 24 bits (pi 2^-25) and its sine and cosine are good to 2 ulp
  (2^-23), each product, sum and the norm's factor to a few 2^-24: together
  below 2^-19 (|a| + |b|) of the (normed) pair.
* weight gradients: fp32 sums of n terms in some order, n 2^-24 sum |terms|,
  plus the terms' own error, 2^-19 sum |terms|.
* attention: u |o| for the output; the probabilities may be rounded to the
  input type before their product with V (u sum p |v|; fp16 also 2^-25 of the
  largest probability for subnormal ones, at most n 2^-25 max |v|); a score's
  error e = (d 2^-23) scale sum |q k| (fp32 accumulation of d exact products)
  enters p twice (numerator and sum): 2 e sum p |v|; exponentials, sums and
  the final division 2^-17 sum p |v|.  lse: e + 2^-17 (1 + |lse|).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _alt():
    import paper_2607_13500_gb300 as altr
    return altr


def _randn(*shape, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(*shape, generator=g)).to(dtype).to(DEV)


def _within(got, ref, tol, what):
    got = got.double()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / tol).nan_to_num(1e30).max()))


# ---------------------------------------------------------------- rotary positions
def _pairs(rot, layout):
    half = rot // 2
    i = torch.arange(half, device=DEV)
    return (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)


def _turned(x, theta, layout, rot):
    """x [T, H, d] float64 turned by theta [T, rot / 2]."""
    a, b = _pairs(rot, layout)
    c, s = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def _spread(x, layout, rot):
    """|a| + |b| of each channel's pair (|x| past rot)."""
    a, b = _pairs(rot, layout)
    y = x.abs().clone()
    both = y[..., a] + y[..., b]
    y[..., a], y[..., b] = both, both
    return y


def _theta(pos, sections, rot, base):
    half = rot // 2
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device=DEV)
    freq = torch.tensor([base ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
    return pos.reshape(len(sections), -1)[axis].double().T * freq


def _normed(x, w, eps):
    if w is None:
        return x
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()


ROTARY = [  # tokens, q heads, k heads, d, rot, sections, layout, dtype, q norm, k norm
    (1, 28, 4, 128, 128, (16, 24, 24), "half", torch.bfloat16, False, False),
    (1, 1, 1, 8, 8, (4,), "half", torch.float32, True, False),
    (7, 5, 1, 64, 64, (32,), "pairs", torch.float16, True, True),
    (33, 3, 3, 80, 40, (8, 6, 6), "half", torch.bfloat16, False, True),
    (33, 3, 3, 80, 40, (10, 10), "pairs", torch.float32, True, True),
    (130, 2, 1, 256, 128, (64,), "half", torch.float32, True, True),
    (1000, 32, 8, 96, 48, (8, 8, 8), "pairs", torch.bfloat16, True, True),
    (2501, 28, 4, 128, 128, (16, 24, 24), "half", torch.bfloat16, True, True),
    (5000, 9, 0, 72, 24, (12,), "half", torch.float16, True, False),
    (300, 4, 2, 16, 0, (), "half", torch.bfloat16, True, False),
]


def _rotary_case(tokens, hq, hk, d, rot, sections, layout, dtype, seed):
    rows = _randn(tokens, hq + hk + 1, d, dtype=dtype, seed=seed)  # slices of a wider projection: strided
    q, k = rows[:, :hq], rows[:, hq:hq + hk] if hk else None
    g = torch.Generator().manual_seed(seed + 1)
    pos = torch.randint(-3, 100000, (max(len(sections), 1), tokens), generator=g).to(torch.int32)
    if tokens > 3 and sections:
        pos[0, :4] = torch.tensor([0, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1])
    return q, k, pos.to(DEV)


@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(str(v) for v in c[:5]))
def test_rotary_forward(case):
    tokens, hq, hk, d, rot, sections, layout, dtype, qn, kn = case
    q, k, pos = _rotary_case(tokens, hq, hk, d, rot, sections, layout, dtype, 11)
    r = _alt().Rotary(d, DEV, base=1e6, rot_dim=rot, sections=sections, layout=layout)
    if not sections:
        pos = pos[:0]
    wq = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=5) if qn else None
    wk = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=6) if kn else None
    before = q.clone()
    gq, gk = r.apply(q, k, pos, q_weight=wq, k_weight=wk, eps=1e-5)
    assert torch.equal(q, before)
    for x, w, got, what in ((q, wq, gq, "q"), (k, wk, gk, "k")):
        if x is None:
            assert got is None
            continue
        n = _normed(x.double(), w, 1e-5)
        if rot:
            ref, mag = _turned(n, _theta(pos, sections, rot, 1e6), layout, rot), _spread(n, layout, rot)
        else:
            ref, mag = n, n.abs()
        _within(got, ref, U[dtype] * ref.abs() + 2.0 ** -19 * mag + 2.0 ** -24, what)
        if w is None:
            assert torch.equal(got[..., rot:], x[..., rot:]), what
    # in place, through the strided slices themselves
    r.apply(q, k, pos, q_weight=wq, k_weight=wk, eps=1e-5, q_out=q, k_out=k)
    assert torch.equal(q, gq) and (k is None or torch.equal(k, gk))


def test_rotary_zero_positions_and_zero_rows():
    r = _alt().Rotary(64, DEV)
    x = _randn(5, 2, 64, dtype=torch.bfloat16, seed=3)
    x[2] = 0
    pos = torch.zeros(5, dtype=torch.int32, device=DEV)
    y, _ = r.apply(x, None, pos)
    assert torch.equal(x, y)  # turned by nothing: the same bits
    y, _ = r.apply(x, None, pos, q_weight=torch.ones(64, device=DEV))
    assert (y[2] == 0).all() and torch.isfinite(y).all()
    e, _ = r.apply(x[:0], None, pos[:0])
    assert e.shape == (0, 2, 64)


def test_rotary_non_finite_rows_stay_alone():
    r = _alt().Rotary(64, DEV)
    x = _randn(6, 3, 64, dtype=torch.float32, seed=4)
    ref, _ = r.apply(x, None, torch.arange(6, dtype=torch.int32, device=DEV), q_weight=torch.ones(64, device=DEV))
    x[2, 1, 5], x[4, 0, 7] = float("nan"), float("inf")
    got, _ = r.apply(x, None, torch.arange(6, dtype=torch.int32, device=DEV), q_weight=torch.ones(64, device=DEV))
    keep = torch.ones(6, 3, dtype=torch.bool, device=DEV)
    keep[2, 1] = keep[4, 0] = False
    assert torch.equal(got[keep], ref[keep])
    assert torch.isnan(got[2, 1]).all()


@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(str(v) for v in c[:5]))
def test_rotary_backward(case):
    tokens, hq, hk, d, rot, sections, layout, dtype, qn, kn = case
    q, k, pos = _rotary_case(tokens, hq, hk, d, rot, sections, layout, dtype, 21)
    dq, dk, _ = _rotary_case(tokens, hq, hk, d, rot, sections, layout, dtype, 23)
    r = _alt().Rotary(d, DEV, base=1e4, rot_dim=rot, sections=sections, layout=layout)
    if not sections:
        pos = pos[:0]
    wq = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=5) if qn else None
    wk = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=6) if kn else None
    got = r.backward(dq, dk, pos, q=q if qn else None, k=k if kn else None, q_weight=wq, k_weight=wk, eps=1e-5)
    again = r.backward(dq, dk, pos, q=q if qn else None, k=k if kn else None, q_weight=wq, k_weight=wk, eps=1e-5)
    for x, dy, w, dx, dw, dw2, what in ((q, dq, wq, got.q, got.q_weight, again.q_weight, "q"),
                                        (k, dk, wk, got.k, got.k_weight, again.k_weight, "k")):
        if dy is None:
            assert dx is None and dw is None
            continue
        g = dy.double()
        mag = g.abs()
        if rot:
            g, mag = _turned(g, -_theta(pos, sections, rot, 1e4), layout, rot), _spread(g, layout, rot)
        if w is None:
            assert dw is None
            _within(dx, g, U[dtype] * g.abs() + 2.0 ** -19 * mag + 2.0 ** -24, what)
            continue
        x64, w64 = x.double(), w.double()
        rms = torch.sqrt(x64.square().mean(-1, keepdim=True) + 1e-5)
        u = x64 / rms
        ref = (w64 * g - u * (u * w64 * g).mean(-1, keepdim=True)) / rms
        mag = w64.abs() * mag
        mag = (mag + u.abs() * (u.abs() * mag).mean(-1, keepdim=True)) / rms
        _within(dx, ref, U[dtype] * ref.abs() + 2.0 ** -19 * mag + 2.0 ** -24, what)
        terms = (g.abs() + _spread(dy.double(), layout, rot) * 2.0 ** -4 if rot else g.abs()) * u.abs()
        n = dy.shape[0] * dy.shape[1]
        _within(dw, (g * u).sum((0, 1)), (n * 2.0 ** -24 + 2.0 ** -15) * terms.sum((0, 1)), what + " weight")
        assert torch.equal(dw, dw2)  # a fixed order of summation


def test_rotary_backward_against_differences():
    # The directional derivative of L = sum(c * y) from central differences of
    # the fp32 forward; h = 2^-7 leaves an O(h^2) error and 2^-24 |L| / h noise.
    altr = _alt()
    r = altr.Rotary(64, DEV, base=100.0, sections=(12, 10, 10))
    x = _randn(9, 4, 64, dtype=torch.float32, seed=31)
    w = 1 + 0.3 * _randn(64, dtype=torch.float32, seed=32)
    c, v, vw = (_randn(*s, dtype=torch.float32, seed=n) for s, n in (((9, 4, 64), 33), ((9, 4, 64), 34), ((64,), 35)))
    pos = torch.randint(0, 50, (3, 9), generator=torch.Generator().manual_seed(36)).to(torch.int32).to(DEV)
    loss = lambda x, w: float((r.apply(x, None, pos, q_weight=w)[0].double() * c.double()).sum())
    g = r.backward(c, None, pos, q=x, q_weight=w)
    h = 2.0 ** -7
    num = (loss(x + h * v, w) - loss(x - h * v, w)) / (2 * h)
    ana = float((g.q.double() * v.double()).sum())
    scale = float((g.q.double() * v.double()).norm()) + 1.0
    assert abs(num - ana) < 2e-2 * scale, (num, ana)
    num = (loss(x, w + h * vw) - loss(x, w - h * vw)) / (2 * h)
    ana = float((g.q_weight.double() * vw.double()).sum())
    assert abs(num - ana) < 2e-2 * (float((g.q_weight.double() * vw.double()).norm()) + 1.0), (num, ana)


# ---------------------------------------------------------------- the paged cache
def _step(seqs, heads, page, d, dtype, seed, stale=float("nan"), spare=2, wide=0):
    """Cache, table, lens, cu_new and the dense keys / values of sequences
    given as (new, length); every slot no sequence owns holds `stale`, every
    table entry no sequence needs an id outside the cache."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for _, n in seqs]
    pages = sum(need) + spare
    k = torch.full((pages, heads, page, d), stale, dtype=dtype)
    v = k.clone()
    ids = torch.randperm(pages, generator=g).tolist()
    table = torch.full((len(seqs), max(need + [0]) + wide), -7, dtype=torch.int32)
    table[:, ::2] = 2 ** 31 - 1
    keys, vals = [], []
    for b, (_, n) in enumerate(seqs):
        kk = (1.5 * torch.randn(n, heads, d, generator=g)).to(dtype)
        vv = torch.randn(n, heads, d, generator=g).to(dtype)
        for i in range(need[b]):
            pid = ids.pop()
            table[b, i] = pid
            m = min(page, n - i * page)
            k[pid, :, :m] = kk[i * page:i * page + m].transpose(0, 1)
            v[pid, :, :m] = vv[i * page:i * page + m].transpose(0, 1)
        keys.append(kk.to(DEV))
        vals.append(vv.to(DEV))
    cu = [0]
    for n, _ in seqs:
        cu.append(cu[-1] + n)
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)
    cache = _alt().PagedCache(k.to(DEV), v.to(DEV))
    return cache, table.to(DEV), i32([n for _, n in seqs]), i32(cu), keys, vals


def _attend_ref(q, key, val, new, causal, window, scale):
    """One sequence, float64: o [n, Hq, d], lse [n, Hq], and sum p |v|, max |score| error terms."""
    n, hq, d = q.shape
    length, hk = key.shape[0], key.shape[1]
    group = hq // hk
    kk, vv = key.double().repeat_interleave(group, 1), val.double().repeat_interleave(group, 1)
    s = scale * torch.einsum("nhd,jhd->hnj", q.double(), kk)
    e = abs(scale) * torch.einsum("nhd,jhd->hnj", q.double().abs(), kk.abs()) * d * 2.0 ** -23
    i = (length - new + torch.arange(n, device=DEV))[:, None]
    j = torch.arange(length, device=DEV)
    seen = torch.ones(n, length, dtype=torch.bool, device=DEV)
    if causal:
        seen &= j <= i
    if window:
        seen &= j > i - window
    s = torch.where(seen, s, torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
    lse = torch.logsumexp(s, -1) if length else torch.full((hq, n), -math.inf, dtype=torch.float64, device=DEV)
    p = torch.where(seen, torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[..., None]), 0.0)
    e = torch.where(seen, e, 0.0).amax(-1) if length else torch.zeros_like(lse)
    # a key that a row does not see takes no part, whatever it holds
    vm = torch.where(torch.isfinite(vv), vv, 0.0)
    o = torch.einsum("hnj,jhd->nhd", p, vm)
    pv = torch.einsum("hnj,jhd->nhd", p, vm.abs())
    return o, lse.T, pv, e.T


def _check_attend(seqs, hq, hk, d, page, dtype, causal=True, window=0, seed=1, scale=None, max_new=None, max_len=None,
                  change=None, strided=False, wide=0):
    cache, table, lens, cu, keys, vals = _step(seqs, hk, page, d, dtype, seed, wide=wide)
    t = int(cu[-1])
    if strided:
        q = _randn(t, hq + 2 * hk, d, dtype=dtype, seed=seed + 1, gain=1.5)[:, :hq]
    else:
        q = _randn(t, hq, d, dtype=dtype, seed=seed + 1, gain=1.5)
    if change:
        change(cache, table, keys, vals, q)
    out = torch.full((t, hq, d), 7.0, dtype=dtype, device=DEV)
    got, lse = cache.attend(q, table, lens, cu, scale=scale, causal=causal, window=window, max_new=max_new,
                            max_len=max_len, return_lse=True, out=out)
    assert int(cache.error) == 0
    sc = 1 / math.sqrt(d) if scale is None else scale
    for b, (n, length) in enumerate(seqs):
        if n == 0:
            continue
        sl = slice(int(cu[b]), int(cu[b + 1]))
        o, z, pv, e = _attend_ref(q[sl], keys[b], vals[b], n, causal, window, sc)
        u = U[dtype]
        rel = (u + 2 * e + 2.0 ** -17)[..., None]
        tol = u * o.abs() + rel * pv + 2.0 ** -24
        if dtype == torch.float16 and length:
            tol = tol + length * 2.0 ** -25 * vals[b].double().nan_to_num(0, 0, 0).abs().max()
        _within(got[sl], o, tol, ("o", b))
        empty = z.isinf()
        assert torch.equal(lse[sl].isinf(), empty), b
        if not empty.all():
            _within(lse[sl][~empty], z[~empty], e[~empty] + 2.0 ** -17 * (1 + z[~empty].abs()), ("lse", b))
    return got


ATTEND = [  # sequences (new, length), q heads, k heads, d, page, dtype
    ([(1, 1)], 1, 1, 64, 16, torch.bfloat16),
    ([(1, 611)], 32, 32, 128, 16, torch.bfloat16),
    ([(1, 129), (1, 1), (1, 128), (1, 127), (1, 3000)], 28, 4, 128, 64, torch.bfloat16),
    ([(1, 40), (0, 17), (1, 0), (0, 0), (1, 5000)], 8, 1, 64, 32, torch.float16),
    ([(5, 5), (3, 900), (1, 77)], 7, 1, 128, 256, torch.float16),
    ([(227, 227), (64, 64), (1, 500)], 4, 4, 128, 16, torch.bfloat16),
    ([(300, 1000), (37, 38), (129, 129)], 28, 4, 128, 128, torch.bfloat16),
    ([(300, 1000), (37, 38), (129, 129)], 5, 1, 64, 64, torch.float16),
    ([(513, 2049)], 8, 2, 128, 32, torch.float16),
    ([(130, 1111)], 6, 2, 80, 16, torch.bfloat16),
    ([(3, 400), (200, 200)], 4, 4, 16, 16, torch.bfloat16),
    ([(70, 640)], 2, 2, 112, 64, torch.float16),
    ([(1, 70000)], 2, 1, 64, 64, torch.bfloat16),
    ([(n, n + 13 * i) for i, n in enumerate([1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 128])], 3, 3, 48, 16,
     torch.bfloat16),
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}of{c[0][0][1]}-{c[1]}-{c[2]}-{c[3]}-p{c[4]}")
@pytest.mark.parametrize("mode", ["causal", "full", "window", "window_full"])
def test_attend(case, mode):
    seqs, hq, hk, d, page, dtype = case
    if mode == "full" and any(n > length for n, length in seqs):
        seqs = [(min(n, length), length) for n, length in seqs]
    _check_attend(seqs, hq, hk, d, page, dtype, causal=mode in ("causal", "window"),
                  window=0 if mode in ("causal", "full") else 50, strided=mode == "window")


def test_attend_many_sequences():
    # more sequences than a warp has lanes, idle and empty ones among them, few and many rows
    lens = [(37 * i * i) % 900 for i in range(75)]
    seqs = [(0 if i % 7 == 3 else 1, n) for i, n in enumerate(lens)]
    _check_attend(seqs, 8, 2, 64, 16, torch.bfloat16, max_new=1)
    _check_attend([(0, 50)] * 40 + [(1, 300)] + [(0, 0)] * 30 + [(1, 20)], 7, 1, 128, 16, torch.float16, max_new=1)
    _check_attend([(n % 5, n) for n in lens], 12, 2, 64, 32, torch.bfloat16)


@pytest.mark.parametrize("case", [(8, 1, 128, 16), (8, 1, 128, 64), (2, 2, 128, 256), (8, 1, 64, 32), (2, 2, 80, 16)],
                         ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-p{c[3]}")
def test_attend_long_runs_repeat(case):
    # dozens of tiles per CTA: every ring position is filled many times over; the
    # same bits every time, alone and back to back
    hq, hk, d, page = case
    for seqs, new in (([(600, 9000), (64, 6001)], 600), ([(1, 20000), (1, 9999), (1, 3)], 1)):
        first = _check_attend(seqs, hq, hk, d, page, torch.bfloat16, max_new=new, max_len=20000, seed=3)
        cache, table, lens, cu, _, _ = _step(seqs, hk, page, d, torch.bfloat16, 3)
        q = _randn(int(cu[-1]), hq, d, dtype=torch.bfloat16, seed=4, gain=1.5)
        outs = [cache.attend(q, table, lens, cu, max_new=new, max_len=20000) for _ in range(12)]
        assert all(torch.equal(o, first) for o in outs)
        assert int(cache.error) == 0


@pytest.mark.parametrize("case", [(32, 32, 128, 16), (28, 4, 128, 64), (16, 16, 64, 32)],
                         ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-p{c[3]}")
@pytest.mark.parametrize("new", [227, 700])
def test_attend_many_blocks_repeat(case, new):
    # hundreds of short blocks per call, many calls: work of one block that the
    # next step takes up too early shows in a block in some thousands only
    hq, hk, d, page = case
    seqs = [(new, new)] * 16
    first = _check_attend(seqs, hq, hk, d, page, torch.bfloat16, max_new=new, max_len=new, seed=3)
    cache, table, lens, cu, _, _ = _step(seqs, hk, page, d, torch.bfloat16, 3)
    q = _randn(int(cu[-1]), hq, d, dtype=torch.bfloat16, seed=4, gain=1.5)
    for _ in range(60):
        assert torch.equal(cache.attend(q, table, lens, cu, max_new=new, max_len=new), first)
    assert int(cache.error) == 0


@pytest.mark.parametrize("bounds", [(None, None), (20, 700), (1000, 100000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attend_bounds_and_splits(bounds, dtype):
    # the host bounds size the launch and choose how the keys are split; none changes the result
    _check_attend([(20, 700), (1, 30), (7, 333)], 14, 2, 128, 16, dtype, max_new=bounds[0], max_len=bounds[1], wide=3)


@pytest.mark.parametrize("window", [1, 2, 127, 128, 129, 500])
def test_attend_window_edges(window):
    _check_attend([(1, 1000), (260, 777)], 4, 2, 64, 32, torch.bfloat16, window=window)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attend_scales(scale):
    _check_attend([(1, 300), (40, 500)], 4, 2, 64, 32, torch.bfloat16, scale=scale)


def test_attend_more_new_than_keys():
    # tokens whose own key would be negative see nothing: zeros and -inf
    cache, table, lens, cu, keys, vals = _step([(3, 5)], 1, 16, 64, torch.bfloat16, 9)
    cu = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    q = _randn(8, 2, 64, dtype=torch.bfloat16, seed=2)
    o, lse = cache.attend(q, table, lens, cu, return_lse=True)
    assert (o[:3] == 0).all() and (lse[:3] == -math.inf).all()
    ref, z, pv, e = _attend_ref(q[3:], keys[0], vals[0], 5, True, 0, 1 / 8)
    _within(o[3:], ref, U[torch.bfloat16] * ref.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv, "o")


@pytest.mark.parametrize("seqs", [[(1, 200)], [(150, 150), (1, 64)], [(40, 1000)]])
def test_attend_hidden_keys_take_no_part(seqs):
    # NaN and infinities in keys and values that a row may not see leave it untouched
    def plant(cache, table, keys, vals, q):
        page = cache.page
        for b, (n, length) in enumerate(seqs):
            if n < 3:
                continue
            for back, bad in ((1, float("nan")), (2, float("inf"))):
                j = length - back
                cache.k[table[b, j // page], :, j % page] = bad
                cache.v[table[b, j // page], :, j % page] = -bad
                vals[b][j] = -bad
                keys[b][j] = 0

    cache, table, lens, cu, keys, vals = _step(seqs, 2, 32, 64, torch.bfloat16, 5)
    q = _randn(int(cu[-1]), 4, 64, dtype=torch.bfloat16, seed=6, gain=1.5)
    plant(cache, table, keys, vals, q)
    got = cache.attend(q, table, lens, cu)
    for b, (n, length) in enumerate(seqs):
        rows = n if n < 3 else n - 2
        o, _, pv, e = _attend_ref(q[int(cu[b]):int(cu[b]) + n], keys[b], vals[b], n, True, 0, 1 / 8)
        tol = U[torch.bfloat16] * o.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv + 2.0 ** -24
        _within(got[int(cu[b]):int(cu[b]) + rows], o[:rows], tol[:rows], b)
        if n >= 3:
            assert torch.isnan(got[int(cu[b + 1]) - 1]).all()  # the row that sees the NaN


def test_attend_window_hides_bad_keys():
    # bad keys below the window of later rows
    cache, table, lens, cu, keys, vals = _step([(100, 400)], 1, 16, 64, torch.float16, 5)
    cache.k[table[0, 310 // 16], :, 310 % 16] = float("nan")
    cache.v[table[0, 310 // 16], :, 310 % 16] = float("inf")
    keys[0][310], vals[0][310] = 0, 0
    q = _randn(100, 2, 64, dtype=torch.float16, seed=6, gain=1.5)
    got = cache.attend(q, table, lens, cu, window=30)
    o, _, pv, e = _attend_ref(q, keys[0], vals[0], 100, True, 30, 1 / 8)
    keep = torch.ones(100, dtype=torch.bool, device=DEV)
    keep[10:40] = False  # rows 310 .. 339 see key 310
    tol = U[torch.float16] * o.abs() + (U[torch.float16] + 2 * e + 2.0 ** -17)[..., None] * pv + 400 * 2.0 ** -25 * 6
    _within(got[keep], o[keep], tol[keep], "o")
    assert torch.isnan(got[10:40]).all()


def test_attend_large_scores():
    # scores far apart: the running maximum moves by thousands, no overflow
    def grow(cache, table, keys, vals, q):
        q *= 30
        cache.k.mul_(8)
        for k in keys:
            k *= 8

    for dtype in (torch.bfloat16, torch.float16):
        _check_attend([(1, 700), (90, 500)], 4, 2, 64, 32, dtype, change=grow)


def test_attend_rising_scores():
    # every key scores higher than the one before: the maximum moves in every tile
    def rise(cache, table, keys, vals, q):
        q[:] = 1
        for b, k in enumerate(keys):
            n = k.shape[0]
            k[:] = (torch.arange(n, device=DEV) / 8).to(k.dtype)[:, None, None] / 8
            for i in range((n + 31) // 32):
                m = min(32, n - 32 * i)
                cache.k[table[b, i], :, :m] = k[32 * i:32 * i + m].transpose(0, 1)

    _check_attend([(1, 900), (150, 600)], 4, 2, 64, 32, torch.float16, change=rise)


def test_attend_bad_pages_read_as_zeros():
    cache, table, lens, cu, keys, vals = _step([(2, 100)], 1, 16, 64, torch.bfloat16, 7)
    q = _randn(2, 2, 64, dtype=torch.bfloat16, seed=8)
    for bad in (-1, cache.pages, 2 ** 31 - 1, -2 ** 31):
        table[0, 2] = bad
        cache.error.zero_()
        o = cache.attend(q, table, lens, cu)
        assert int(cache.error) == 1
        k, v = keys[0].clone(), vals[0].clone()
        k[32:48], v[32:48] = 0, 0
        ref, _, pv, e = _attend_ref(q, k, v, 2, True, 0, 1 / 8)
        _within(o, ref, U[torch.bfloat16] * ref.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv, bad)


def test_attend_repeats_bit_for_bit_and_in_graphs():
    cache, table, lens, cu, keys, vals = _step([(1, 3000), (1, 17), (1, 700)], 4, 64, 128, torch.bfloat16, 3)
    q = _randn(3, 28, 128, dtype=torch.bfloat16, seed=4)
    first = cache.attend(q, table, lens, cu, max_new=1)
    for _ in range(20):
        assert torch.equal(cache.attend(q, table, lens, cu, max_new=1), first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = cache.attend(q, table, lens, cu, max_new=1)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(again, first)
    g = torch.cuda.CUDAGraph()
    out = torch.empty_like(q)
    with torch.cuda.graph(g):
        cache.attend(q, table, lens, cu, max_new=1, out=out)
    lens -= 1  # the same graph serves other lengths
    g.replay()
    assert torch.equal(out, cache.attend(q, table, lens, cu, max_new=1))
    assert not torch.equal(out, first)


def test_attend_rows_past_32_bits():
    # page rows whose byte offsets pass 32 bits: 40000 pages x 2 heads x 32 x 128 channels, 2 bytes each
    d, page, heads, pages = 128, 32, 2, 40000
    k = torch.zeros(pages, heads, page, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    cache = _alt().PagedCache(k, v)
    keys, vals = (_randn(70, heads, d, dtype=torch.bfloat16, seed=n) for n in (1, 2))
    table = torch.tensor([[39999, 0, 20000]], dtype=torch.int32, device=DEV)
    lens, cu = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([70], [0, 70]))
    cache.append(keys, vals, table, lens, cu)
    assert torch.equal(k[39999].transpose(0, 1), keys[:32]) and torch.equal(v[20000, :, :6].transpose(0, 1), vals[64:])
    q = _randn(70, 4, d, dtype=torch.bfloat16, seed=3)
    o = cache.attend(q, table, lens, cu)
    ref, _, pv, e = _attend_ref(q, keys, vals, 70, True, 0, 1 / math.sqrt(d))
    _within(o, ref, U[torch.bfloat16] * ref.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv + 2.0 ** -24, "o")


# ---------------------------------------------------------------- append
APPEND = [  # sequences (new, length), q heads, k heads, d, rot, page, dtype, norm, layout, with rotary
    ([(1, 1)], 4, 1, 64, 64, 16, torch.bfloat16, False, "half", True),
    ([(1, 17), (1, 16), (1, 5000)], 28, 4, 128, 128, 16, torch.bfloat16, False, "half", True),
    ([(100, 100), (0, 5), (33, 70)], 8, 2, 128, 64, 32, torch.float16, True, "pairs", True),
    ([(700, 900), (31, 31)], 0, 3, 80, 40, 64, torch.bfloat16, True, "half", True),
    ([(40, 45)], 2, 2, 48, 48, 256, torch.float16, True, "half", False),
    ([(3000, 3000), (2000, 2100)], 4, 4, 96, 96, 128, torch.bfloat16, True, "half", True),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{len(c[0])}x{c[0][0][0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]}")
def test_append(case):
    seqs, hq, hk, d, rot, page, dtype, norm, layout, rotate = case
    altr = _alt()
    cache, table, lens, cu, _, _ = _step(seqs, hk, page, d, dtype, 5, stale=3.0)
    t = int(cu[-1])
    rows = _randn(t, hq + 2 * hk, d, dtype=dtype, seed=6)
    q, k, v = rows[:, :hq] if hq else None, rows[:, hq:hq + hk], rows[:, hq + hk:]
    r = altr.Rotary(d, DEV, rot_dim=rot, sections=(rot // 2 - 2 * (rot // 8), rot // 8, rot // 8), layout=layout)
    pos = torch.randint(0, 40000, (3, t), generator=torch.Generator().manual_seed(8)).to(torch.int32).to(DEV)
    wq = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=5) if norm and hq else None
    wk = 1 + 0.3 * _randn(d, dtype=torch.float32, seed=6) if norm else None
    want_k, want_v = cache.k.clone(), cache.v.clone()
    if rotate:  # the same rows through the rotation alone: the same bits
        some = q if hq else k
        rq, rk = r.apply(some, k, pos, q_weight=wq if hq else wk, k_weight=wk)
    else:
        r0 = altr.Rotary(d, DEV, rot_dim=0, sections=())
        rq, rk = r0.apply(q, k, pos[:0], q_weight=wq, k_weight=wk)
    for b, (n, length) in enumerate(seqs):
        for i in range(n):
            j = length - n + i
            want_k[table[b, j // page], :, j % page] = rk[int(cu[b]) + i]
            want_v[table[b, j // page], :, j % page] = v[int(cu[b]) + i]
    got = cache.append(k, v, table, lens, cu, rotary=r if rotate else None, pos=pos if rotate else None, k_weight=wk,
                       q=q, q_weight=wq)
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
    assert got is None if not hq else torch.equal(got, rq)
    assert int(cache.error) == 0


def test_append_bad_pages_write_nothing():
    cache, table, lens, cu, _, _ = _step([(40, 40), (8, 20)], 2, 16, 64, torch.bfloat16, 5, stale=3.0)
    before = cache.k.clone(), cache.v.clone()
    rows = _randn(48, 4, 64, dtype=torch.bfloat16, seed=6)
    table[:] = torch.tensor([-1, 2 ** 31 - 1, cache.pages], dtype=torch.int32, device=DEV)[:table.shape[1]]
    cache.append(rows[:, :2], rows[:, 2:], table, lens, cu)
    assert int(cache.error) == 1
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
    # lengths past the table, below the new tokens and negative
    cache.error.zero_()
    table[:] = 0
    for bad in ([1000, 1000], [3, 2], [-5, -2 ** 31]):
        cache.append(rows[:, :2], rows[:, 2:], table, torch.tensor(bad, dtype=torch.int32, device=DEV), cu)
        cache.attend(rows, table, torch.tensor(bad, dtype=torch.int32, device=DEV), cu)
    assert int(cache.error) == 1


def test_prefill_in_chunks_then_tokens_matches_one_prompt():
    # a prompt in one chunk, and the same prompt as 3 chunks and single tokens: the
    # outputs agree within the tolerance of two attentions over the same cache
    altr = _alt()
    hq, hk, d, page, n = 8, 2, 128, 16, 300
    r = altr.Rotary(d, DEV, sections=(32, 16, 16))
    rows = _randn(n, hq + 2 * hk, d, dtype=torch.bfloat16, seed=1)
    pos = torch.randint(0, 3000, (3, n), generator=torch.Generator().manual_seed(2)).to(torch.int32).to(DEV)
    table = torch.randperm(19, generator=torch.Generator().manual_seed(3))[None].to(torch.int32).to(DEV)
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32, device=DEV)

    def go(cuts):
        cache = altr.PagedCache.empty(19, hk, page, d, device=DEV)
        out = []
        for a, b in zip(cuts, cuts[1:]):
            x = rows[a:b]
            q = cache.append(x[:, hq:hq + hk], x[:, hq + hk:], table, i32(b), i32(0, b - a), rotary=r,
                             pos=pos[:, a:b].contiguous(), q=x[:, :hq])
            out.append(cache.attend(q, table, i32(b), i32(0, b - a)))
        return torch.cat(out), cache

    one, c1 = go([0, n])
    many, c2 = go([0, 120, 257, 290] + list(range(291, n + 1)))
    k = torch.cat([c1.k[p] for p in table[0].tolist()], 1)[:, :n].transpose(0, 1)
    v = torch.cat([c1.v[p] for p in table[0].tolist()], 1)[:, :n].transpose(0, 1)
    k2 = torch.cat([c2.k[p] for p in table[0].tolist()], 1)[:, :n].transpose(0, 1)
    assert torch.equal(k, k2)
    q, _ = r.apply(rows[:, :hq], None, pos)
    ref, _, pv, e = _attend_ref(q, k, v, n, True, 0, 1 / math.sqrt(d))
    tol = U[torch.bfloat16] * ref.abs() + (U[torch.bfloat16] + 2 * e + 2.0 ** -17)[..., None] * pv + 2.0 ** -24
    _within(one, ref, tol, "one")
    _within(many, ref, tol, "many")
