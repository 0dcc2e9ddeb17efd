"""CPU pins of oracle/attn_oracle.py: its gradients against differentiation of a separately typed forward pass and against differences,
what masks do, and that its bounds hold for the roundings they speak of."""
import math

import pytest

torch = pytest.importorskip("torch")
from oracle import attn_oracle as ao  # noqa: E402


def make(seed, heads, kv, n, d):
    g = torch.Generator().manual_seed(seed)
    r = lambda h: torch.randn(h, n, d, generator=g, dtype=torch.float64)  # noqa: E731
    return r(heads), r(kv), r(kv), r(heads)


def plain(q, k, v, scale, causal):
    """The definition, row by row."""
    out = []
    for h in range(q.shape[0]):
        c = h // (q.shape[0] // k.shape[0])
        rows = []
        for i in range(q.shape[1]):
            j = i + 1 if causal else q.shape[1]
            e = torch.exp(scale * (k[c, :j] * q[h, i]).sum(1))
            rows.append((e[:, None] * v[c, :j]).sum(0) / e.sum())
        out.append(torch.stack(rows))
    return torch.stack(out)


@pytest.mark.parametrize("heads,kv,n,d,causal", [(2, 2, 1, 8, True), (4, 2, 7, 8, True), (3, 1, 9, 16, False), (2, 2, 12, 8, True)])
def test_gradients_are_those_of_the_definition(heads, kv, n, d, causal):
    q, k, v, do = make(n, heads, kv, n, d)
    scale = 0.37
    o, lse, p, _ = ao.forward(q, k, v, scale, causal)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    ref = plain(*leaves, scale, causal)
    assert torch.allclose(o, ref.detach(), rtol=1e-12, atol=1e-12) and torch.allclose(p.sum(2), torch.ones(heads, n, dtype=torch.float64))
    (got, _), want = ao.backward(q, k, v, do, scale, causal), torch.autograd.grad(ref, leaves, do)
    assert all(torch.allclose(a, b, rtol=1e-10, atol=1e-12) for a, b in zip(got, want))
    # and against differences of the loss sum(o do) along a direction, fourth order
    g = torch.Generator().manual_seed(1)
    for at, grad in enumerate(got):
        way = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        loss = lambda e: float((plain(*[t + e * way if at == x else t for x, t in enumerate((q, k, v))], scale, causal) * do).sum())  # noqa: E731
        h = 1e-3
        slope = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
        assert abs(slope - float((grad * way).sum())) <= 1e-9 * (1 + abs(slope))


def test_masked_places_have_no_part():
    q, k, v, _ = make(3, 2, 2, 6, 8)
    ref = ao.forward(q, k, v, 0.5, True)[0]
    k[0, 4, 1], v[1, 3, 2], v[0, 5, 0] = math.nan, math.inf, math.nan
    o = ao.forward(q, k, v, 0.5, True)[0]
    assert torch.equal(o[0, :4], ref[0, :4]) and o[0, 4:].isnan().all()
    assert torch.equal(o[1, :3], ref[1, :3]) and (o[1, 3:, 2] == math.inf).all()


@pytest.mark.parametrize("causal", [False, True])
def test_bounds_cover_the_roundings(causal):
    """p, ds and the results rounded to bf16 as the kernels round them, in 64 bits else: inside the bounds, and not far inside."""
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    q, k, v, do = (bf(t) for t in make(8, 4, 2, 40, 32))
    scale = 0.3
    o, lse, p, eps = ao.forward(q, k, v, scale, causal)
    kg, vg = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
    got = bf(bf(p) @ vg)
    r = ((got - o).abs() / ao.forward_bound(p, v, o, eps)).amax()
    assert 0.1 < r <= 1
    (dq, dk, dv), bounds = ao.backward(q, k, v, do, scale, causal)
    ds = bf(p * (do @ vg.transpose(1, 2) - (do * got).sum(2, keepdim=True)))
    fold = lambda t: t.reshape(2, 2, *t.shape[1:]).sum(1)  # noqa: E731
    mine = bf(scale * (ds @ kg)), bf(scale * fold(ds.transpose(1, 2) @ q)), bf(fold(bf(p).transpose(1, 2) @ do))
    for a, b, e in zip(mine, (dq, dk, dv), bounds):
        assert 0.02 < ((a - b).abs() / e).amax() <= 1


def test_decode_is_the_last_row_of_a_causal_prompt():
    q, k, v, _ = make(5, 6, 3, 11, 8)
    o = ao.forward(q, k, v, 0.4, True)[0]
    got, bound = ao.decode(q[:, -1], k, v, 0.4)
    assert torch.allclose(got, o[:, -1], rtol=1e-12, atol=1e-12) and (bound > 0).all()
    assert (ao.decode(q[:, -1], k[:, :0], v[:, :0], 0.4)[0] == 0).all()


@pytest.mark.parametrize("heads,kv,n,d,causal", [(2, 2, 40, 32, True), (4, 2, 60, 64, False), (4, 1, 33, 128, True)])
def test_bounds_with_an_exact_delta_tell_it_from_that_of_the_rounded_o(heads, kv, n, d, causal):
    """Values and keys that have much in common: what o loses when it is rounded is as large as what tells the values apart.  The kernels' arithmetic with its
    roundings, in 64 bits else, stays inside the bounds; the same with the rounded o's delta does not."""
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    q, k, v, do = make(n, heads, kv, n, d)
    q, k, v, do = bf(q), bf(k + 4), bf(v + 32), bf(do)
    scale, g = d ** -0.5 / 4, heads // kv
    o, _, p, _ = ao.forward(q, k, v, scale, causal)
    kg, vg = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    given = bf(bf(p) @ vg)
    (dq, b_q), (dk, b_k) = ao.exact_delta_bounds(q, k, v, do, given, scale, causal)
    want = ao.backward(q, k, v, do, scale, causal)[0]
    assert torch.allclose(dq, want[0], rtol=1e-9, atol=1e-11) and torch.allclose(dk, want[1], rtol=1e-9, atol=1e-11)
    delta, dp = (do * given).sum(2, keepdim=True), do @ vg.transpose(1, 2)
    z = p * (dp - delta)
    worst = {}
    for exact in (True, False):
        r = z.sum(2, keepdim=True) * exact
        mine_q = bf(scale * (bf(z) @ kg - r * (bf(p) @ kg)))
        mine_k = bf(scale * (bf(p * (dp - delta - r)).transpose(1, 2) @ q).reshape(-1, g, n, d).sum(1))
        worst[exact] = float(((mine_q - dq).abs() / b_q).amax()), float(((mine_k - dk).abs() / b_k).amax())
    assert 0.05 < worst[True][0] <= 1 and 0.02 < worst[True][1] <= 1, worst
    assert worst[False][0] > 4 and worst[False][1] > 2, worst
