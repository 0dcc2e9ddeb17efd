"""GPU parity of the norms around a block and their gradients against oracle/block_oracle.py.

Bars.  A row's statistics are sums of d terms in 32 bits, each thread's 16 or fewer in order and the rest in a tree: their relative
error stays below 32 x 2^-24.  Outputs are a handful of 32-bit operations on values that carry it, plus half a step of their type:
|error| <= 64 x 2^-24 (the largest magnitude that enters) + half a step of the result.  Gradients of parameters are fp32 sums over
at most 64 rows a block, joined in 64 bits: 128 x 2^-24 of the sum of the absolute terms."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def make(rng, rows, d, dtype, gate, res, post, pre, bias):
    v = dict(x=dev(2 * rng.standard_normal((rows, d)), DT[dtype]), o=None if post is None else dev(rng.standard_normal((rows, d)) + 0.3, DT[dtype]))
    p = {}
    if post:
        p["w_post"] = dev(1 + 0.2 * rng.standard_normal(d))
        if bias:
            p["b_post"] = dev(0.2 * rng.standard_normal(d))
    if gate:
        p["gate"] = dev(0.5 + 0.2 * rng.standard_normal(1 if gate == 1 else d))
    if res:
        p["res"] = dev(0.9 + 0.1 * rng.standard_normal(1))
    if pre:
        p["w_pre"] = dev(1 + 0.2 * rng.standard_normal(d))
        if bias:
            p["b_pre"] = dev(0.2 * rng.standard_normal(d))
    return v, p


def near(got, ref, scale, dtype, what):
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    err = 64 * U * scale + step * (np.abs(ref) + 64 * U * scale) + 1e-30
    worst = np.max(np.abs(host(got) - ref) / err) if ref.size else 0.0
    assert np.isfinite(host(got)).all() and worst <= 1.0, (what, worst)


FORMS = [dict(layer=False, gate=1, res=True, post=True, pre=True, bias=False), dict(layer=True, gate=2, res=True, post=True, pre=True, bias=True),
         dict(layer=True, gate=1, res=False, post=False, pre=True, bias=True), dict(layer=False, gate=2, res=True, post=True, pre=False, bias=True),
         dict(layer=False, gate=0, res=True, post=None, pre=True, bias=False), dict(layer=True, gate=0, res=False, post=False, pre=False, bias=False)]
SIZES = [(1, 1), (3, 2), (1, 64), (5, 63), (9, 96), (4, 768), (33, 1000), (2, 1024), (3, 1025), (70, 1032), (6, 4096), (3, 4099), (5, 5120),
         (2, 16384), (3, 16383), (1100, 40), (2100, 768)]


def ids(c):
    return "-".join(f"{k}{v}" for k, v in c.items())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", FORMS, ids=ids)
def test_forward_and_gradients(c, dtype):
    for rows, d in SIZES:
        rng = np.random.default_rng(rows * 31 + d)
        kw = {k: c[k] for k in ("gate", "res", "post", "pre", "bias")}
        v, p = make(rng, rows, d, dtype, **kw)
        # a row of zeros, a row far from zero, and one of tiny values
        if rows > 3:
            v["x"][0] = 0
            if v["o"] is not None:
                v["o"][0] = 0
                v["o"][1] *= 1e-4
        hx, ho = host(v["x"]), None if v["o"] is None else host(v["o"])
        hp = {k: host(t) for k, t in p.items()}
        bn = rt.BlockNorm(d, layer=c["layer"], eps=1e-5, **p)
        y, n = torch.full_like(v["x"], 9), torch.full_like(v["x"], 9) if c["pre"] else None
        bn.forward(v["x"], v["o"], y, n)
        ry, rn = bo.block_norm(hx, ho, layer=c["layer"], eps=1e-5, **hp)
        # what enters: rows of N are at most sqrt(d) large; an element's own error is relative to the parts it is summed from
        g, a = np.abs(hp.get("gate", 1.0)), abs(hp["res"][0]) if "res" in hp else 1.0
        part = a * np.abs(hx)
        if ho is not None:
            part = part + g * (np.abs(bo._norm(ho, c["layer"], 1e-5)[0]) + (np.abs(ho).max(1, keepdims=True) * bo._norm(ho, c["layer"], 1e-5)[1] if c["layer"] else 0) + 1) * np.abs(hp.get("w_post", 1.0)) if c["post"] else part + g * np.abs(ho)
            part = part + g * np.abs(hp.get("b_post", 0.0))
        near(y, ry, part, dtype, ("y", rows, d))
        if c["pre"]:
            h, r = bo._norm(ry, c["layer"], 1e-5)
            scale = (part.max(1, keepdims=True) * r + np.abs(h) + 1) * np.abs(hp["w_pre"]) + np.abs(hp.get("b_pre", 0.0))
            near(n, rn, scale, dtype, ("n", rows, d))

        dy = dev(rng.standard_normal((rows, d)), DT[dtype])
        dn = dev(rng.standard_normal((rows, d)), DT[dtype]) if c["pre"] else None
        dx, do = torch.full_like(v["x"], 9), None if v["o"] is None else torch.full_like(v["x"], 9)
        dp = {k: torch.full_like(t, 9) for k, t in p.items()}
        bn.backward(v["x"], v["o"], dy, dn, dx, do, dp)
        ref = bo.block_norm_grad(hx, ho, host(dy), None if dn is None else host(dn), layer=c["layer"], eps=1e-5, **hp)
        # the gradient of a norm is a difference of row-sized parts, each divided by the row's deviation
        gs = np.abs(host(dy))
        if c["pre"]:
            h, r = bo._norm(ry, c["layer"], 1e-5)
            dnw = np.abs(host(dn) * hp["w_pre"])
            amp = 1 + part.max(1, keepdims=True) * r   # how much of y's own error its norm shows
            gs = gs + r * amp * (dnw + dnw.mean(1, keepdims=True) + (np.abs(h) + 1) * (dnw * (np.abs(h) + 1)).mean(1, keepdims=True))
        near(dx, ref["x"], a * gs, dtype, ("dx", rows, d))
        os_ = None
        if ho is not None:
            os_ = gs * g
            if c["post"]:
                h, r = bo._norm(ho, c["layer"], 1e-5)
                amp = 1 + (np.abs(ho).max(1, keepdims=True) * r if c["layer"] else 0)
                w = os_ * np.abs(hp["w_post"])
                os_ = r * amp * (w + w.mean(1, keepdims=True) + (np.abs(h) + 1) * (w * (np.abs(h) + 1)).mean(1, keepdims=True))
            near(do, ref["o"], os_, dtype, ("do", rows, d))
        ph = np.zeros_like(hx) if ho is None else (np.abs(bo._norm(ho, c["layer"], 1e-5)[0]) + 1) if c["post"] else np.abs(ho)
        amp_o = 1 + (np.abs(ho).max(1, keepdims=True) * bo._norm(ho, c["layer"], 1e-5)[1] if c["post"] and c["layer"] else 0)
        terms = {"res": (gs * np.abs(hx)).sum()}
        if "gate" in p:
            t = gs * amp_o * (ph * np.abs(hp.get("w_post", 1.0)) + np.abs(hp.get("b_post", 0.0)))
            terms["gate"] = t.sum(0) if c["gate"] == 2 and d > 1 else t.sum()
        if c["post"]:
            terms["w_post"], terms["b_post"] = (gs * g * ph * amp_o).sum(0), (gs * g).sum(0)
        if c["pre"]:
            h, r = bo._norm(ry, c["layer"], 1e-5)
            terms["w_pre"] = (np.abs(host(dn)) * (np.abs(h) + 1) * (1 + part.max(1, keepdims=True) * r)).sum(0)
            terms["b_pre"] = np.abs(host(dn)).sum(0)
        for k, t in dp.items():
            worst = np.max(np.abs(host(t) - ref[k]) / (128 * U * terms[k] + 1e-30))
            assert worst <= 1.0, (k, rows, d, worst)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_partial_calls_and_places(dtype):
    """Outputs that are not wanted, dy that is not there, states one element off 16 bytes, in-place outputs: the same bits."""
    rng = np.random.default_rng(3)
    rows, d = 37, 96
    v, p = make(rng, rows, d, dtype, 2, True, True, True, True)
    bn = rt.BlockNorm(d, layer=True, **p)
    y, n = torch.empty_like(v["x"]), torch.empty_like(v["x"])
    bn.forward(v["x"], v["o"], y, n)
    only = torch.empty_like(n)
    bn.forward(v["x"], v["o"], None, only)
    assert torch.equal(only, n)
    x2, o2 = v["x"].clone(), v["o"].clone()
    bn.forward(x2, o2, x2, o2)
    assert torch.equal(x2, y) and torch.equal(o2, n)

    def off(t):
        s = torch.empty(rows * d + 1, dtype=t.dtype, device="cuda")[1:].view(rows, d)
        s.copy_(t)
        return s

    y3, n3 = off(y), off(n)
    bn.forward(off(v["x"]), off(v["o"]), y3, n3)           # another dealing of columns over threads: the sums' order differs
    assert (host(y3) - host(y)).__abs__().max() <= (2.0 ** -6 if dtype == "bf16" else 2.0 ** -19) * 4
    dy, dn = dev(rng.standard_normal((rows, d)), DT[dtype]), dev(rng.standard_normal((rows, d)), DT[dtype])
    full = dict(dx=torch.empty_like(y), do=torch.empty_like(y), dparams={k: torch.empty_like(t) for k, t in p.items()})
    bn.backward(v["x"], v["o"], dy, dn, **full)
    part = {k: torch.empty_like(p[k]) for k in ("gate", "b_pre")}
    bn.backward(v["x"], v["o"], dy, dn, dparams=part)
    assert all(torch.equal(part[k], full["dparams"][k]) for k in part)
    dy2, dn2 = dy.clone(), dn.clone()
    bn.backward(v["x"], v["o"], dy2, dn2, dx=dy2, do=dn2)
    assert torch.equal(dy2, full["dx"]) and torch.equal(dn2, full["do"])
    zero, none = torch.empty_like(y), torch.empty_like(y)
    bn.backward(v["x"], v["o"], torch.zeros_like(dy), dn, dx=zero)
    bn.backward(v["x"], v["o"], None, dn, dx=none)
    assert torch.equal(zero, none)
    empty = {k: torch.full_like(t, 9) for k, t in p.items()}
    e = v["x"][:0]
    bn.forward(e, e, e, e)
    bn.backward(e, e, e, e, e, e, empty)
    assert all((t == 0).all() for t in empty.values())


def test_a_row_without_a_value_spoils_no_other():
    rng = np.random.default_rng(4)
    rows, d = 11, 200
    v, p = make(rng, rows, d, "f32", 1, True, True, True, False)
    bn = rt.BlockNorm(d, **p)
    y, n, y2, n2 = (torch.empty_like(v["x"]) for _ in range(4))
    bn.forward(v["x"], v["o"], y, n)
    v["x"][4, 7], v["o"][6, 199] = float("nan"), float("inf")
    bn.forward(v["x"], v["o"], y2, n2)
    keep = [r for r in range(rows) if r not in (4, 6)]
    assert torch.equal(y2[keep], y[keep]) and torch.equal(n2[keep], n[keep])
    assert torch.isnan(n2[4]).all() and torch.isnan(n2[6]).any()


def test_same_bits_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(5)
    rows, d = 700, 768
    v, p = make(rng, rows, d, "bf16", 1, True, True, True, False)
    bn = rt.BlockNorm(d, **p)
    dy, dn = dev(rng.standard_normal((rows, d)), torch.bfloat16), dev(rng.standard_normal((rows, d)), torch.bfloat16)
    outs = lambda: [torch.empty_like(v["x"]) for _ in range(4)] + [torch.empty_like(t) for t in p.values()]  # noqa: E731

    def go(o):
        bn.forward(v["x"], v["o"], o[0], o[1])
        bn.backward(v["x"], v["o"], dy, dn, o[2], o[3], dict(zip(p, o[4:])))

    ref, other, graph = outs(), outs(), outs()
    go(ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go(other)
        go(graph)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go(graph)
    for k in range(3):
        v["o"].mul_(-0.5)
        go(ref)
        torch.cuda.synchronize()
        for t in graph:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, graph)), k


def test_what_python_refuses():
    one = torch.ones(8, device="cuda")
    x = torch.ones(3, 8, device="cuda")
    bn = rt.BlockNorm(8, w_post=one, w_pre=one)
    for bad in (lambda: rt.BlockNorm(8, w_post=one[:7]), lambda: rt.BlockNorm(8, gate=one[:2]), lambda: rt.BlockNorm(8, w_pre=one.bfloat16()),
                lambda: rt.BlockNorm(8, w_pre=one.cpu()), lambda: bn.forward(x, x.bfloat16(), x, x), lambda: bn.forward(x[:, :7], x[:, :7], x[:, :7], x[:, :7]),
                lambda: bn.forward(x, x[:2], x, x), lambda: bn.forward(x.t().contiguous().t(), x, x, x), lambda: bn.backward(x, x, x, x, x, x, {"gate": one})):
        with pytest.raises(ValueError):
            bad()


def test_sums_over_many_rows_lose_no_more_than_over_few():
    """2^23 rows: columns of equal terms, whose roundings all lean one way where they are added one after another."""
    rows, d = 1 << 23, 8
    rng = np.random.default_rng(6)
    x = dev(np.float32(1 + rng.random((1, d)))).expand(rows, d).contiguous()
    dn = dev(np.float32(1 + rng.random((1, d)))).expand(rows, d).contiguous()
    p = {"w_pre": torch.ones(d, device="cuda"), "b_pre": torch.zeros(d, device="cuda"), "res": torch.ones(1, device="cuda")}
    dp = {k: torch.empty_like(t) for k, t in p.items()}
    rt.BlockNorm(d, layer=True, **p).backward(x, None, None, dn, dparams=dp)
    hx, hn = host(x[:1]), host(dn[:1])
    ref = bo.block_norm_grad(hx, None, None, hn, layer=True, eps=1e-5, **{k: host(t) for k, t in p.items()})
    h, r = bo._norm(hx, True, 1e-5)
    amp = 1 + np.abs(hx).max() * r
    for k, scale in (("b_pre", np.abs(hn)[0]), ("w_pre", (np.abs(hn) * (np.abs(h) + 1) * amp)[0])):
        assert np.max(np.abs(host(dp[k]) - rows * ref[k]) / (128 * U * rows * scale)) <= 1.0, k


# (rows, d) whose blocks go on to a second and third row, the last round ragged: every count of threads a row, values held and
# loaded again, whole pieces and single values (a width or an address off 16 bytes)
ROUNDS = [(17003, 40), (17001, 130), (9003, 1000), (4103, 1500), (2081, 2056), (2051, 4096), (2053, 5120), (2050, 8200), (2049, 16383)]
ROUNDS_GRAD = [(9003, 40), (9001, 96), (4501, 392), (2077, 776), (1083, 1032), (531, 4096), (533, 4099), (517, 5120), (515, 16384), (515, 16383)]


def parts_of(rng, rows, d, dtype, form):
    kw = {k: form[k] for k in ("gate", "res", "post", "pre", "bias")}
    return make(rng, rows, d, dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", FORMS[:2], ids=ids)
@pytest.mark.parametrize("rows,d", ROUNDS)
def test_a_row_is_the_same_in_any_round_forward(rows, d, c, dtype):
    """A block's later rows give the bits that they give alone, at a place where a block has one row (a row's dealing over threads
    depends on d alone), and rows of the first, a middle and the last round agree with the oracle."""
    rng = np.random.default_rng(rows + d)
    v, p = parts_of(rng, rows, d, dtype, c)
    bn = rt.BlockNorm(d, layer=c["layer"], **p)
    y, n = torch.empty_like(v["x"]), torch.empty_like(v["x"])
    bn.forward(v["x"], v["o"], y, n)
    few = 500
    for at in range(0, rows, few):
        x, o = v["x"][at:at + few].clone(), v["o"][at:at + few].clone()
        y1, n1 = torch.empty_like(x), torch.empty_like(x)
        bn.forward(x, o, y1, n1)
        assert torch.equal(y1, y[at:at + few]) and torch.equal(n1, n[at:at + few]), at
    pick = [0, rows // 2, rows - 1]
    ry, rn = bo.block_norm(host(v["x"][pick]), host(v["o"][pick]), layer=c["layer"], eps=1e-5, **{k: host(t) for k, t in p.items()})
    big = 4 * np.abs(ry).max() + 4
    near(y[pick], ry, big, dtype, "y")
    near(n[pick], rn, big * np.abs(rn).max(), dtype, "n")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c", FORMS[:2], ids=ids)
@pytest.mark.parametrize("rows,d", ROUNDS_GRAD)
def test_a_row_is_the_same_in_any_round_backward(rows, d, c, dtype):
    """States' gradients: the bits that a block's single rows give.  Parameters': 128 x 2^-24 of the sum of the absolute terms off the sum
    of the single rounds' own, of which each is as near to its own."""
    rng = np.random.default_rng(rows * 3 + d)
    v, p = parts_of(rng, rows, d, dtype, c)
    bn = rt.BlockNorm(d, layer=c["layer"], **p)
    dy, dn = dev(rng.standard_normal((rows, d)), DT[dtype]), dev(rng.standard_normal((rows, d)), DT[dtype])
    dx, do = torch.empty_like(dy), torch.empty_like(dy)
    dp = {k: torch.empty_like(t) for k, t in p.items()}
    bn.backward(v["x"], v["o"], dy, dn, dx, do, dp)
    few, sums = 250, {k: np.zeros(t.numel()) for k, t in p.items()}
    for at in range(0, rows, few):
        s = slice(at, at + few)
        x, o, gy, gn = (t[s].clone() for t in (v["x"], v["o"], dy, dn))
        dx1, do1 = torch.empty_like(x), torch.empty_like(x)
        dp1 = {k: torch.empty_like(t) for k, t in p.items()}
        bn.backward(x, o, gy, gn, dx1, do1, dp1)
        assert torch.equal(dx1, dx[s]) and torch.equal(do1, do[s]), at
        for k in sums:
            sums[k] += host(dp1[k])
    # the terms' absolute values, from the oracle on all rows
    hp = {k: host(t) for k, t in p.items()}
    hx, ho, hy, hn = host(v["x"]), host(v["o"]), host(dy), host(dn)
    L = c["layer"]
    oh = bo._norm(ho, L, 1e-5)[0]
    post = oh * hp["w_post"] + hp.get("b_post", 0.0)
    yh, ry = bo._norm(hp["res"][0] * hx + hp["gate"] * post, L, 1e-5)
    g = np.abs(hy + bo._norm_back(hn * hp["w_pre"], yh, ry, L))
    gate = np.abs(hp["gate"])
    terms = {"w_post": (gate * g * np.abs(oh)).sum(0), "b_post": (gate * g).sum(0), "res": (g * np.abs(hx)).sum(), "w_pre": (np.abs(hn) * np.abs(yh)).sum(0),
             "b_pre": np.abs(hn).sum(0), "gate": (g * np.abs(post)).sum(0) if c["gate"] == 2 else (g * np.abs(post)).sum()}
    ref = bo.block_norm_grad(hx, ho, hy, hn, layer=L, eps=1e-5, **hp)
    for k, t in dp.items():
        assert np.max(np.abs(host(t) - sums[k]) / (2 * 128 * U * terms[k] + 1e-30)) <= 1.0, k
        # an element's own error: statistics of d terms (64 x 2^-24) of row-sized parts, in g through two norms
        own = 64 * U * 16 * (1 + np.abs(oh).max() + np.abs(yh).max())
        assert np.max(np.abs(host(t) - ref[k]) / ((128 * U + own) * (terms[k] + terms[k].max()))) <= 1.0, k


def test_parameters_given_other_storage():
    """What a parameter is at the call counts, wherever its storage is by then; what no longer fits is refused."""
    rng = np.random.default_rng(11)
    rows, d = 9, 96
    v, p = make(rng, rows, d, "f32", 2, True, True, True, True)
    bn = rt.BlockNorm(d, layer=True, **p)
    dy, dn = torch.ones_like(v["x"]), torch.ones_like(v["x"])

    def go(b):
        y, n, dx, do = (torch.empty_like(v["x"]) for _ in range(4))
        dp = {k: torch.empty_like(t) for k, t in p.items()}
        b.forward(v["x"], v["o"], y, n)
        b.backward(v["x"], v["o"], dy, dn, dx, do, dp)
        return [y, n, dx, do, *dp.values()]

    keep = []                                             # the old storages stay, so that a stale address would be read, not faulted on
    for k in list(p):
        before = go(bn)
        keep.append(p[k].detach())
        other = dev(rng.standard_normal(p[k].numel()))
        if k.startswith("w"):
            p[k].data = other
        elif k.startswith("b"):
            p[k].set_(other)
        else:
            p[k] = bn.params[k] = other
        after = go(bn)
        assert all(torch.equal(a, b) for a, b in zip(after, go(rt.BlockNorm(d, layer=True, **p)))), k
        assert any(not torch.equal(a, b) for a, b in zip(after, before)), k
    for k, bad in (("w_post", torch.ones(d - 1, device="cuda")), ("gate", torch.ones(d)), ("w_pre", None), ("b_pre", torch.ones(d, device="cuda").double())):
        was, bn.params[k] = bn.params[k], bad
        for call in (lambda: bn.forward(v["x"], v["o"], dy, dn), lambda: bn.backward(v["x"], v["o"], dy, dn)):
            with pytest.raises(ValueError):
                call()
        bn.params[k] = was
    go(bn)


def test_the_bindings_functions_are_the_layers_calls():
    """paper_2408_10746_amd.binding on addresses gives the bits that runtime gives on tensors."""
    from paper_2408_10746_amd import binding as pb
    rng = np.random.default_rng(16)
    rows, d, st = 70, 96, torch.cuda.current_stream().cuda_stream
    v, p = make(rng, rows, d, "bf16", 2, True, True, True, True)
    bn = rt.BlockNorm(d, layer=True, eps=1e-5, **p)
    at = lambda *ts: [t.data_ptr() for t in ts]  # noqa: E731
    names = ("w_post", "b_post", "gate", "res", "w_pre", "b_pre")
    b = pb.pac_block_norm(d, pb.PAC_BF16, 1, d, 1e-5, *at(*(p[k] for k in names)))
    dy, dn = dev(rng.standard_normal((rows, d)), torch.bfloat16), dev(rng.standard_normal((rows, d)), torch.bfloat16)
    y, n, dx, do, y2, n2, dx2, do2 = (torch.empty_like(dy) for _ in range(8))
    g, g2 = ({k: torch.empty_like(p[k]) for k in names} for _ in range(2))
    pb.pac_block_norm_forward(b, rows, *at(v["x"], v["o"], y, n), st)
    ws = torch.empty(pb.pac_block_norm_workspace_bytes(b, rows), dtype=torch.uint8, device="cuda")
    pb.pac_block_norm_backward(b, rows, *at(v["x"], v["o"], dy, dn, dx, do, *g.values()), ws.data_ptr(), ws.numel(), st)
    bn.forward(v["x"], v["o"], y2, n2)
    bn.backward(v["x"], v["o"], dy, dn, dx2, do2, g2)
    assert all(torch.equal(s, t) for s, t in zip([y, n, dx, do, *g.values()], [y2, n2, dx2, do2, *g2.values()]))
    with pytest.raises(pb.PacError):
        pb.pac_block_norm_forward(b, -1, *at(v["x"], v["o"], y, n), st)
