"""Rotary.apply as a node of the autograd graph: gradients against a plain
implementation differentiated in 64 bits.

Tolerance, u the type's unit roundoff, as for tr_rotary_backward's own tests:
u |g| for the rounding of a gradient to its type and 2^-16 of the largest
|gradient| of the case for the fp32 arithmetic (2^-19 of a row's terms, of
which the norm's gradient adds at most a few); weights 2^-13 of sum |terms|."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2607_13500_gb300 import _build
    _build.build()


def _rotary(d, sections=(16, 8, 8)):
    import paper_2607_13500_gb300 as altr
    return altr.Rotary(d, "cuda", base=1e4, sections=sections)


def _plain(x, w, theta):
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
    half = theta.shape[1]
    a, b, c, s = x[..., :half], x[..., half:], torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _inputs(dtype, tokens=37, hq=4, hk=2, d=64):
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(tokens, hq + hk, d, device="cuda", generator=g).to(dtype)
    pos = torch.randint(0, 5000, (3, tokens), device="cuda", generator=g, dtype=torch.int32)
    wq, wk = (1 + 0.3 * torch.randn(d, device="cuda", generator=g) for _ in range(2))
    cq, ck = (torch.randn(tokens, h, d, device="cuda", generator=g).to(dtype) for h in (hq, hk))
    axis = torch.tensor([0] * 16 + [1] * 8 + [2] * 8, device="cuda")
    freq = 1e4 ** (-torch.arange(32, dtype=torch.float64, device="cuda") / 32)
    return rows, pos, wq, wk, cq, ck, pos[axis].double().T * freq


@pytest.mark.parametrize("dtype", list(U))
@pytest.mark.parametrize("norm", ["", "q", "qk"])
def test_gradients_of_a_fused_projection(dtype, norm):
    rows, pos, wq, wk, cq, ck, theta = _inputs(dtype)
    rows.requires_grad_()
    wq, wk = wq.requires_grad_() if "q" in norm else None, wk.requires_grad_() if "k" in norm else None
    q, k = _rotary(64).apply(rows[:, :4], rows[:, 4:], pos, q_weight=wq, k_weight=wk)
    ((q * cq).float().sum() + (k * ck).float().sum()).backward()

    ref = rows.detach().double().requires_grad_()
    rq, rk = (None if w is None else w.detach().double().requires_grad_() for w in (wq, wk))
    loss = (_plain(ref[:, :4], rq, theta) * cq.double()).sum() + (_plain(ref[:, 4:], rk, theta) * ck.double()).sum()
    loss.backward()
    off = (rows.grad.double() - ref.grad).abs()
    assert (off <= U[dtype] * ref.grad.abs() + 2.0 ** -16 * ref.grad.abs().max()).all(), float(off.max())
    for w, r, c in ((wq, rq, cq), (wk, rk, ck)):
        if w is not None:
            terms = c.double().abs().sum((0, 1)).max() * 4  # |normed x| stays below 4 of its root mean square here
            assert ((w.grad.double() - r.grad).abs() <= 2.0 ** -13 * terms).all()


def test_what_backward_returns_is_what_the_graph_gets():
    rows, pos, wq, wk, cq, ck, _ = _inputs(torch.bfloat16)
    r = _rotary(64)
    x, y = rows[:, :4].clone().requires_grad_(), rows[:, 4:].clone().requires_grad_()
    wq.requires_grad_()
    q, k = r.apply(x, y, pos, q_weight=wq, k_weight=wk)
    torch.autograd.backward([q, k], [cq, ck])
    g = r.backward(cq, ck, pos, q=x.detach(), k=y.detach(), q_weight=wq.detach(), k_weight=wk)
    assert torch.equal(x.grad, g.q) and torch.equal(y.grad, g.k) and torch.equal(wq.grad, g.q_weight)
    assert torch.equal(q, r.apply(x.detach(), y.detach(), pos, q_weight=wq.detach(), k_weight=wk)[0])


@pytest.mark.parametrize("only", ["q", "k"])
def test_one_output_used_and_gradients_of_any_strides(only):
    # the other output's gradient is zero; sum() hands on a gradient with no strides at all, a transpose odd ones
    rows, pos, wq, wk, cq, ck, theta = _inputs(torch.float32)
    x, y = rows[:, :4].clone().requires_grad_(), rows[:, 4:].clone().requires_grad_()
    q, k = _rotary(64).apply(x, y, pos)
    if only == "q":
        q.sum().backward()
    else:
        (k.transpose(1, 2) * ck.transpose(1, 2).contiguous()).sum().backward()
    dy = torch.ones_like(q).double() if only == "q" else ck.double()
    used, other = (x, y) if only == "q" else (y, x)
    ref = _plain(dy, None, -theta)
    assert (used.grad.double() - ref).abs().max() <= 2.0 ** -16 * ref.abs().max()
    assert (other.grad == 0).all()


def test_without_keys_and_without_tokens():
    rows, pos, wq, _, cq, _, _ = _inputs(torch.bfloat16)
    x = rows[:, :4].clone().requires_grad_()
    q, k = _rotary(64).apply(x, None, pos, q_weight=wq)
    assert k is None
    q.backward(cq)
    assert x.grad.shape == x.shape and torch.isfinite(x.grad).all()
    e = rows[:0, :4].clone().requires_grad_()
    w = wq.clone().requires_grad_()
    _rotary(64).apply(e, None, pos[:, :0].contiguous(), q_weight=w)[0].sum().backward()
    assert e.grad.shape == (0, 4, 64) and (w.grad == 0).all()


def test_where_nothing_is_recorded():
    rows, pos, wq, wk, _, _, _ = _inputs(torch.bfloat16)
    r = _rotary(64)
    x = rows[:, :4].clone().requires_grad_()
    with torch.no_grad():
        q, _ = r.apply(x, None, pos, q_out=torch.empty_like(x))
    assert not q.requires_grad
    q, _ = r.apply(rows[:, :4], None, pos, q_weight=wq)
    assert not q.requires_grad
    with pytest.raises(ValueError, match="q_out"):
        r.apply(x, None, pos, q_out=torch.empty_like(x))
    with pytest.raises(ValueError, match="q_out"):
        r.apply(x, None, pos, q_out=x)
