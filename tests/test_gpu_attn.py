"""GPU parity of attention over packed sequences and its gradients against oracle/attn_oracle.py (64 bits).

Bars are the oracle's: every value of every result against the error that the stated roundings may make there (p and ds to bf16, o to
bf16 before delta is made from it, results to bf16, scores and sums in 32 bits), from the absolute terms of its own sum."""
import math

import pytest
import torch

from oracle import attn_oracle as ao
from paper_2408_10746_amd import binding as pb
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def make(seed, rows, heads, kv, d, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h, s=1.0: (s * torch.randn(rows, h * d, generator=g, device="cuda")).to(BF)  # noqa: E731
    return r(heads, spread), r(kv), r(kv), r(heads)


def by_head(t, heads):
    return t.double().reshape(t.shape[0], heads, -1).transpose(0, 1)


def rows_of(t):
    return t.transpose(0, 1).reshape(t.shape[1], -1)


def run(a, q, k, v, do, offsets, grads=True):
    o, lse = torch.empty_like(q), torch.empty(a.heads, q.shape[0], device="cuda")
    a.forward(q, k, v, offsets, o, lse)
    if not grads:
        return o, lse
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    a.backward(q, k, v, offsets, o, lse, do, dq, dk, dv)
    return o, lse, dq, dk, dv


def inside(got, ref, bound, what):
    off = (got.double() - ref).abs()
    worst = float((off / bound).amax()) if off.numel() else 0.0
    assert torch.isfinite(got).all() and worst <= 1.0, (what, worst)


def check(a, lens, got, q, k, v, do, scale, causal, first=0):
    at = first
    for n in lens:
        s = slice(at, at + n)
        at += n
        if n == 0:
            continue
        qh, kh, vh = by_head(q[s], a.heads), by_head(k[s], a.kv_heads), by_head(v[s], a.kv_heads)
        o, lse, p, eps = ao.forward(qh, kh, vh, scale, causal)
        inside(got[0][s], rows_of(o), rows_of(ao.forward_bound(p, vh, o, eps)), ("o", n))
        assert float((got[1][:, s].double() - lse).abs().amax()) <= 2 * eps + 4 * ao.F32 * float(lse.abs().amax()), ("lse", n)
        if len(got) > 2:
            ref, bound = ao.backward(qh, kh, vh, by_head(do[s], a.heads), scale, causal)
            for name, g, r, b in zip(("dq", "dk", "dv"), got[2:], ref, bound):
                inside(g[s], rows_of(r), rows_of(b), (name, n))


CASES = [(1, 1, 64, [1]), (2, 2, 128, [1, 2, 3]), (4, 4, 128, [31, 32, 33]), (4, 2, 64, [0, 17, 0, 64, 65, 0]), (8, 2, 128, [127, 128, 129]),
         (6, 1, 32, [200, 1, 95]), (3, 3, 96, [63, 161]), (5, 5, 80, [40, 257]), (7, 1, 8, [130]), (16, 16, 40, [5, 66]), (2, 1, 104, [513]),
         (12, 12, 64, [128, 3, 77, 50]), (8, 8, 128, [700]), (9, 3, 24, [33, 300])]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,d,lens", CASES, ids=str)
def test_forward_and_gradients(heads, kv, d, lens, causal):
    rows = sum(lens)
    q, k, v, do = make(rows, rows, heads, kv, d, 1.5)
    a = rt.Attention(heads, d, kv_heads=kv, causal=causal)
    check(a, lens, run(a, q, k, v, do, rt.packed_offsets(lens)), q, k, v, do, d ** -0.5, causal)


@pytest.mark.parametrize("heads,kv,d,n,causal", [(8, 2, 128, 2500, True), (4, 4, 64, 3001, False), (2, 1, 96, 4100, True)])
def test_long_sequences(heads, kv, d, n, causal):
    q, k, v, do = make(n, n, heads, kv, d, 1.5)
    a = rt.Attention(heads, d, kv_heads=kv, causal=causal)
    check(a, [n], run(a, q, k, v, do, rt.packed_offsets([n])), q, k, v, do, d ** -0.5, causal)


@pytest.mark.parametrize("heads,kv", [(64, 1), (40, 2), (33, 3)])
def test_many_heads_share_keys(heads, kv):
    """Few tiles of keys, many queries each: gradients of shared heads."""
    lens = [150, 40]
    q, k, v, do = make(heads, sum(lens), heads, kv, 64)
    for causal in (False, True):
        a = rt.Attention(heads, 64, kv_heads=kv, causal=causal)
        check(a, lens, run(a, q, k, v, do, rt.packed_offsets(lens)), q, k, v, do, 0.125, causal)


@pytest.mark.parametrize("batch", [63, 64, 65, 700, 4097, 5000])
def test_many_short_sequences(batch):
    """The search for a tile's sequence: fewer and more than 64 and 64^2 of them, empty ones among them."""
    lens = [(7 * b) % 4 for b in range(batch)]
    q, k, v, do = make(batch, sum(lens), 2, 1, 32)
    a = rt.Attention(2, 32, kv_heads=1, causal=True)
    got = run(a, q, k, v, do, rt.packed_offsets(lens))
    whole = torch.tensor([float(r) for n in lens for r in [n] * n])  # length of each row's sequence
    # all sequences of one length at once: a batch of them, heads and sequences together
    at = torch.tensor([0] + lens).cumsum(0)[:-1]
    for n in (1, 2, 3):
        starts = at[torch.tensor(lens) == n]
        pick = (starts[:, None] + torch.arange(n)[None]).reshape(-1).cuda()
        assert int((whole == n).sum()) == pick.numel()
        fold = lambda t, h: t[pick].double().reshape(-1, n, h, 32).permute(0, 2, 1, 3).reshape(-1, n, 32)  # noqa: E731
        qh, kh, vh, doh = fold(q, 2), fold(k, 1), fold(v, 1), fold(do, 2)
        o, _, p, eps = ao.forward(qh, kh, vh, 32 ** -0.5, True)
        inside(fold(got[0], 2), o, ao.forward_bound(p, vh, o, eps), ("o", n))
        for g, r, b, h in zip(got[2:], *ao.backward(qh, kh, vh, doh, 32 ** -0.5, True), (2, 1, 1)):
            inside(fold(g, h), r, b, n)


def test_one_key_has_no_gradient_in_queries_and_keys():
    lens = [1, 1, 1]
    q, k, v, do = make(0, 3, 4, 4, 128)
    for causal in (False, True):
        a = rt.Attention(4, 128, causal=causal)
        o, lse, dq, dk, dv = run(a, q, k, v, do, rt.packed_offsets(lens))
        assert torch.equal(o, v) and torch.equal(dv, do) and not dq.any() and not dk.any()


def test_columns_of_one_matrix_and_rows_of_no_sequence():
    """q, k, v and their gradients as columns of wider matrices; rows before, between and behind the sequences stay as they were."""
    heads, kv, d, lens, lead, tail = 4, 2, 72, [40, 0, 101], 5, 9
    rows, wide = lead + sum(lens) + tail, (heads + 2 * kv) * d + 8
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dx = torch.randn(rows, wide, generator=g, device="cuda").to(BF), torch.full((rows, wide), 7.0, device="cuda", dtype=BF)
    cut = lambda m: (m[:, :heads * d], m[:, heads * d:(heads + kv) * d], m[:, (heads + kv) * d:(heads + 2 * kv) * d])  # noqa: E731
    (q, k, v), (dq, dk, dv) = cut(x), cut(dx)
    do = torch.randn(rows, heads * d, generator=g, device="cuda").to(BF)
    for t in (q, k, v, do):  # nothing outside the sequences is read
        t[:lead], t[-tail:] = math.nan, math.inf
    o, lse = torch.full_like(do, 7.0), torch.full((heads, rows), 7.0, device="cuda")
    off = rt.packed_offsets(lens) + lead
    for causal in (False, True):
        a = rt.Attention(heads, d, kv_heads=kv, causal=causal, scale=0.2)
        a.forward(q, k, v, off, o, lse)
        a.backward(q, k, v, off, o, lse, do, dq, dk, dv)
        check(a, lens, (o, lse, dq, dk, dv), q, k, v, do, 0.2, causal, first=lead)
        for t in (o, dx, lse.t()):
            assert (t[:lead] == 7).all() and (t[-tail:] == 7).all()
        assert (dx[:, -8:] == 7).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d,n,at", [(128, 150, 70), (64, 40, 39), (96, 200, 130), (32, 33, 0), (64, 129, 128)])
def test_values_that_are_none_stay_where_the_mask_lets_them(d, n, at, bad):
    """A key, value, query or gradient that is infinite or no number reaches only the rows that see it.  The others keep their bits, but for
    the 32 rows beside it: their sums may be taken in another order, so that both runs' results lie within the oracle's bound of one exact
    value and within twice that bound of each other."""
    heads = 2
    clean = make(d + n, n, heads, heads, d)
    a = rt.Attention(heads, d, causal=True)
    off = rt.packed_offsets([n])
    ref = run(a, *clean, off)
    q, k, v, do = (by_head(t, heads) for t in clean)
    o, lse, p, eps = ao.forward(q, k, v, d ** -0.5, True)
    bounds = [rows_of(b) for b in (ao.forward_bound(p, v, o, eps), *ao.backward(q, k, v, do, d ** -0.5, True)[1])]
    bounds.insert(1, torch.zeros(n, heads, device="cuda"))
    beside = torch.arange(n, device="cuda") // 32 == at // 32
    row = torch.arange(n, device="cuda")

    def alike(r, g, bound, rows, what):
        far, near = rows & ~beside, rows & beside
        assert torch.equal(r[far], g[far]), what
        assert bool(((r[near].double() - g[near].double()).abs() <= 2 * bound[near]).all()), what

    for which, name in enumerate(("q", "k", "v", "do")):
        t = [x.clone() for x in clean]
        t[which][at, 3] = bad  # head 0
        got = run(a, *t, off)
        for r, g, b, out in zip(ref, got, bounds, ("o", "lse", "dq", "dk", "dv")):
            r, g = (x.t() if out == "lse" else x for x in (r, g))
            other = slice(1, 2) if out == "lse" else slice(d, 2 * d)
            assert torch.equal(r[:, other], g[:, other]), (name, out, "the other head")
            if name == "q":  # row `at` alone, and the keys it sees
                alike(r, g, b, row != at if out in ("o", "lse", "dq") else row > at, (name, out))
            elif name == "do":
                alike(r, g, b, row >= 0 if out in ("o", "lse") else row != at if out == "dq" else row > at, (name, out))
            elif out in ("o", "lse", "dq"):  # k and v: rows before
                alike(r, g, b, row < at, (name, out))
        if name == "v":
            seen = got[0][at:, 3]
            assert seen.isnan().all() if math.isnan(bad) else (seen == bad).all()
        if name == "do":
            assert not got[4][:at + 1, 3].isfinite().any()


def test_neighbours_that_are_none():
    """Sequences beside one full of NaN, in one tile's reach."""
    lens = [20, 13, 50]
    clean = make(9, sum(lens), 2, 2, 64)
    for causal in (False, True):
        a, off = rt.Attention(2, 64, causal=causal), rt.packed_offsets(lens)
        ref = run(a, *clean, off)
        t = [x.clone() for x in clean]
        for x in t:
            x[20:33] = math.nan
        got = run(a, *t, off)
        for r, g, out in zip(ref, got, ("o", "lse", "dq", "dk", "dv")):
            r, g = (x.t() if out == "lse" else x for x in (r, g))
            assert torch.equal(r[:20], g[:20]) and torch.equal(r[33:], g[33:]) and g[20:33].isnan().all(), out


def test_scores_far_apart():
    """Scores of hundreds: probabilities that underflow, maxima that rise and fall along the keys, and any scale."""
    n, d = 300, 64
    q, k, v, do = make(1, n, 2, 2, d)
    for seed, scale in ((0, 8.0), (1, 1e-4), (2, 1.0)):
        up = torch.linspace(0.1, 3, n, device="cuda")[torch.randperm(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")]
        kk = (k.float() * up[:, None]).to(BF)
        for causal in (False, True):
            a = rt.Attention(2, d, causal=causal, scale=scale)
            check(a, [n], run(a, q, kk, v, do, rt.packed_offsets([n])), q, kk, v, do, scale, causal)


def test_offsets_that_point_outside_do_no_harm():
    """What lies outside 0..rows is cut off; memory around the results is left alone."""
    rows, heads, d = 50, 2, 64
    q, k, v, do = make(4, rows, heads, heads, d)
    pad = torch.full((rows + 400, heads * d), 5.0, device="cuda", dtype=BF)
    o = pad[200:200 + rows]
    a = rt.Attention(heads, d)
    for off, lens in (([0, 30, 1 << 30], [30, 20]), ([-7, 50, 50], [50, 0]), ([0, 50, 2147483647], [50, 0])):
        lse = torch.empty(heads, rows, device="cuda")
        a.forward(q, k, v, torch.tensor(off, dtype=torch.int32, device="cuda"), o, lse)
        check(a, lens, (o, lse), q, k, v, do, d ** -0.5, False)
        assert (pad[:200] == 5).all() and (pad[200 + rows:] == 5).all()
    for off in ([50, 20, 0], [40, 10, 45], [-5, -3, -9]):
        a.forward(q, k, v, torch.tensor(off, dtype=torch.int32, device="cuda"), o)
        assert (pad[:200] == 5).all() and (pad[200 + rows:] == 5).all()


def test_same_bits_streams_and_graphs():
    """The same call gives the same bits: again, on a stream of its own, captured and replayed with the program's own work between, two
    graphs side by side."""
    lens = [150, 1, 90, 300]
    rows, heads, kv, d = sum(lens), 8, 2, 128
    q, k, v, do = make(6, rows, heads, kv, d)
    a, off = rt.Attention(heads, d, kv_heads=kv, causal=True), rt.packed_offsets(lens)
    first = run(a, q, k, v, do, off)
    assert all(torch.equal(x, y) for x, y in zip(first, run(a, q, k, v, do, off)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(a, q, k, v, do, off)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(a, q, k, v, do, off)
        graphs.append((g, out))
    for turn in range(3):
        q.mul_(-0.5)
        want = run(a, q, k, v, do, off)
        for g, out in graphs:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(x, y) for x, y in zip(want, out)), turn


def test_the_bindings_functions_are_the_layers_calls():
    lens, heads, d = [70, 5], 4, 64
    q, k, v, do = make(3, 75, heads, heads, d)
    off, st = rt.packed_offsets(lens), torch.cuda.current_stream().cuda_stream
    ref = run(rt.Attention(heads, d, causal=True), q, k, v, do, off)
    s, a = heads * d, pb.pac_attn(heads, heads, d, 1, d ** -0.5)
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(heads, 75, device="cuda"), torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    m = lambda *ts: [x for t in ts for x in (t.data_ptr(), s)]  # noqa: E731
    pb.pac_attn_forward(a, off.data_ptr(), 2, 75, *m(q, k, v, o), lse.data_ptr(), st)
    need = pb.pac_attn_workspace_bytes(a, 2, 75)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    pb.pac_attn_backward(a, off.data_ptr(), 2, 75, *m(q, k, v, o), lse.data_ptr(), *m(do, dq, dk, dv), ws.data_ptr(), need, st)
    assert all(torch.equal(x, y) for x, y in zip(ref, (o, lse, dq, dk, dv)))


def test_runtime_refuses():
    q, k, v, do = make(0, 10, 4, 2, 64)
    a, off, o, lse = rt.Attention(4, 64, kv_heads=2), rt.packed_offsets([4, 6]), torch.empty_like(q), torch.empty(4, 10, device="cuda")
    go = lambda q=q, k=k, v=v, off=off, o=o, lse=lse: a.forward(q, k, v, off, o, lse)  # noqa: E731
    go(), go(lse=None), go(q[:0], k[:0], v[:0], rt.packed_offsets([]), o[:0], lse[:, :0].contiguous())
    odd = torch.empty(10, 4 * 64 + 4, device="cuda", dtype=BF)[:, :256]
    for kw in (dict(q=q.float()), dict(k=k[:9]), dict(v=v.cpu()), dict(off=off.long()), dict(off=off.cpu()), dict(o=o.t()), dict(lse=lse.double()),
               dict(lse=lse.t()), dict(off=off[:0]), dict(q=q[None])):
        with pytest.raises(ValueError):
            go(**kw)
    for kw in (dict(q=odd), dict(o=q), dict(o=q.view(-1)[8:].as_strided((9, 256), (256, 1)) if False else odd)):
        with pytest.raises(pb.PacError):
            go(**kw)
    with pytest.raises(ValueError):
        a.backward(q, k, v, off, o, None, do, q, k, v)
    with pytest.raises(pb.PacError) as e:  # a result in an operand's place
        a.backward(q, k, v, off, o, lse, do, q, torch.empty_like(k), torch.empty_like(v))
    assert e.value.status == pb.PAC_ERR_RANGE


@pytest.mark.parametrize("heads,kv,d,lens,causal", [(64, 1, 64, [500], True), (64, 1, 64, [500], False), (12, 1, 128, [1111, 300], True), (3, 3, 40, [2100], True),
                                                    (16, 2, 96, [0, 1025, 0], False), (32, 2, 128, [640, 1, 33], True)])
def test_queries_dealt_to_several_workgroups(heads, kv, d, lens, causal):
    """Few tiles of keys with many queries each: partial sums through memory (the workspace is more than the two values a row), rows of no
    sequence left alone."""
    lead, tail = 3, 6
    rows = lead + sum(lens) + tail
    q, k, v, do = make(heads + d, rows, heads, kv, d)
    a = rt.Attention(heads, d, kv_heads=kv, causal=causal)
    assert pb.pac_attn_workspace_bytes(a._a, len(lens), rows) > 2 * ((rows * heads * 4 + 255) // 256 * 256)
    off = rt.packed_offsets(lens) + lead
    o, lse = torch.empty_like(q), torch.empty(heads, rows, device="cuda")
    a.forward(q, k, v, off, o, lse)
    dq, dk, dv = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    a.backward(q, k, v, off, o, lse, do, dq, dk, dv)
    check(a, lens, (o, lse, dq, dk, dv), q, k, v, do, d ** -0.5, causal, first=lead)
    for t in (dq, dk, dv):
        assert (t[:lead] == 7).all() and (t[-tail:] == 7).all()
    again = torch.empty_like(dk)
    a.backward(q, k, v, off, o, lse, do, dq, again, dv)
    assert torch.equal(dk[lead:-tail], again[lead:-tail])


@pytest.mark.parametrize("heads,kv,d,lens,causal", [(2, 1, 128, [1000], True), (2, 2, 128, [777, 0, 130], False), (3, 1, 64, [129, 300, 257], True), (1, 1, 32, [2049], False),
                                                    (4, 2, 96, [160, 500], True), (2, 2, 40, [33, 640], False), (1, 1, 104, [1, 511], True)])
def test_few_rows(heads, kv, d, lens, causal):
    """Calls that leave most of the card idle deal the keys to the wavefronts of a workgroup (32 rows each); rows beside the sequences stay as
    they are, values that are none where the mask lets them."""
    lead, tail = 2, 5
    rows = lead + sum(lens) + tail
    assert (rows // 128 + len(lens)) * heads <= (192 if causal else 72) and rows >= 128 * len(lens)
    q, k, v, do = make(heads + d, rows, heads, kv, d, 1.5)
    for t in (q, k, v, do):
        t[:lead], t[-tail:] = math.nan, math.inf
    a, off = rt.Attention(heads, d, kv_heads=kv, causal=causal), rt.packed_offsets(lens) + lead
    o, lse = torch.full_like(q, 7.0), torch.full((heads, rows), 7.0, device="cuda")
    dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, k, v))
    a.forward(q, k, v, off, o, lse)
    a.backward(q, k, v, off, o, lse, do, dq, dk, dv)
    check(a, lens, (o, lse, dq, dk, dv), q, k, v, do, d ** -0.5, causal, first=lead)
    for t in (o, lse.t(), dq, dk, dv):
        assert (t[:lead] == 7).all() and (t[-tail:] == 7).all()


@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_none_in_many_rows(which, bad):
    """The same as for few rows, where 128 rows make a workgroup: 128 heads, a value in the last one's first tile and in its last."""
    heads, d, n = 128, 64, 200
    clean = dict(zip(("q", "k", "v", "do"), make(5, n, heads, heads, d)))
    a, off = rt.Attention(heads, d, causal=True), rt.packed_offsets([n])
    assert (n // 128 + 1) * heads > 192
    ref = run(a, *clean.values(), off)
    for at in (33, 190):
        t = {name: x.clone() for name, x in clean.items()}
        t[which][at, (heads - 1) * d + 5] = bad
        got = run(a, *t.values(), off)
        for r, g, out in zip(ref, got, ("o", "lse", "dq", "dk", "dv")):
            r, g = (x.t() if out == "lse" else x for x in (r, g))
            other = slice(0, heads - 1) if out == "lse" else slice(0, (heads - 1) * d)
            assert torch.equal(r[:, other], g[:, other]), (which, out)
            mine = torch.arange(n, device="cuda") // 32 < at // 32
            if out in ("o", "lse", "dq"):  # rows before see none of it
                assert torch.equal(r[mine], g[mine]), (which, out)
        if which == "v":
            seen = got[0][at:, (heads - 1) * d + 5]
            assert seen.isnan().all() if math.isnan(bad) else (seen == bad).all()


@pytest.mark.parametrize("d,lens,causal", [(128, [200], True), (128, [150, 50], True), (64, [131, 1, 70], False), (64, [200], False)])
def test_rows_as_far_apart_as_strides_go(d, lens, causal):
    """2^24 values from row to row: a tile's rows lie up to 2^32 bytes from its first, and the last ones past 2^32 values of the first."""
    heads, kv, rows, far = 2, 1, sum(lens), 1 << 24
    buffer = torch.empty(rows, far, device="cuda", dtype=BF)
    at, views = 0, []
    for h in (heads, kv, kv, heads, heads, heads, kv, kv):  # q, k, v, do, o, dq, dk, dv
        views.append(buffer[:, at:at + h * d])
        at += far // 8 // 8 * 8 - 8
    q, k, v, do, o, dq, dk, dv = views
    for to, x in zip((q, k, v, do), make(d, rows, heads, kv, d)):
        to.copy_(x)
    a, off, lse = rt.Attention(heads, d, kv_heads=kv, causal=causal), rt.packed_offsets(lens), torch.empty(heads, rows, device="cuda")
    a.forward(q, k, v, off, o, lse)
    a.backward(q, k, v, off, o, lse, do, dq, dk, dv)
    c = torch.Tensor.contiguous
    check(a, lens, (c(o), lse, c(dq), c(dk), c(dv)), c(q), c(k), c(v), c(do), d ** -0.5, causal)


@pytest.mark.parametrize("heads,kv,d,lens,causal", [(32, 8, 128, [300, 600, 450, 33], True), (16, 4, 64, [100, 200, 131, 64, 1, 177], True), (4, 4, 128, [900, 700], False),
                                                    (3, 3, 96, [200, 10, 0, 97], True), (32, 8, 128, [512], True)])
def test_queries_of_short_sequences_dealt_to_several_workgroups(heads, kv, d, lens, causal):
    """Few tiles of keys, few queries for each: parts of a handful of subtiles, some of them none in the shorter sequences."""
    rows = sum(lens)
    q, k, v, do = make(heads + d, rows, heads, kv, d)
    a, off = rt.Attention(heads, d, kv_heads=kv, causal=causal), rt.packed_offsets(lens)
    got = run(a, q, k, v, do, off)
    check(a, lens, got, q, k, v, do, d ** -0.5, causal)
    assert all(torch.equal(x, y) for x, y in zip(got, run(a, q, k, v, do, off)))
