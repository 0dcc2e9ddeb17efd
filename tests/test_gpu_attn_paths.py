"""GPU parity of packed attention on each of its kernels' paths against oracle/attn_oracle.py (64 bits), with that oracle's bounds: tiles without a
missing row at the end of their matrices, long sequences and values that are none on 128 and on 32 rows a workgroup, and what a call allocates."""
import math

import pytest
import torch

from attn_kernels import few
from oracle import attn_oracle as ao
from paper_2408_10746_amd import binding as pb
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def make(seed, rows, heads, kv, d, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h, s=1.0: (s * torch.randn(rows, h * d, generator=g, device="cuda")).to(BF)  # noqa: E731
    return r(heads, spread), r(kv), r(kv), r(heads)


def run(a, q, k, v, do, offsets):
    o, lse = torch.empty_like(q), torch.empty(a.heads, q.shape[0], device="cuda")
    a.forward(q, k, v, offsets, o, lse)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    a.backward(q, k, v, offsets, o, lse, do, dq, dk, dv)
    return o, lse, dq, dk, dv


def check(a, lens, got, q, k, v, do, scale, causal):
    """Sequence by sequence and key head by key head: 64-bit scores of all heads at once would not fit for long ones."""
    at, d, g = 0, a.d, a.heads // a.kv_heads
    for n in lens:
        rows = slice(at, at + n)
        at += n
        for h in range(a.kv_heads if n else 0):
            mine, kvs = slice(h * g * d, (h + 1) * g * d), slice(h * d, (h + 1) * d)
            by = lambda t, c: t[rows, c].double().reshape(n, -1, d).transpose(0, 1)  # noqa: E731
            qh, kh, vh = by(q, mine), by(k, kvs), by(v, kvs)
            o, lse, p, eps = ao.forward(qh, kh, vh, scale, causal)
            ref, bound = ao.backward(qh, kh, vh, by(do, mine), scale, causal)
            off = (got[1][h * g:(h + 1) * g, rows].double() - lse).abs()
            assert float(off.amax()) <= 2 * eps + 4 * ao.F32 * float(lse.abs().amax()), ("lse", n, h)
            for name, t, c, r, b in zip(("o", "dq", "dk", "dv"), (got[0], *got[2:]), (mine, mine, kvs, kvs), (o, *ref), (ao.forward_bound(p, vh, o, eps), *bound)):
                off = (by(t, c) - r).abs()
                assert torch.isfinite(off).all() and bool((off <= b).all()), (name, n, h, float((off / b).amax()))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,lens", [(2, 1, [32]), (3, 3, [64]), (2, 2, [96, 128]), (4, 2, [256]), (24, 24, [128, 128]), (96, 48, [64, 64]), (48, 12, [1, 31, 256])], ids=str)
def test_whole_tiles_of_96_values_at_the_end(heads, kv, lens, causal):
    """The last row of the last head ends the matrix, and a whole tile ends there."""
    q, k, v, do = make(sum(lens), sum(lens), heads, kv, 96, 1.5)
    a = rt.Attention(heads, 96, kv_heads=kv, causal=causal)
    check(a, lens, run(a, q, k, v, do, rt.packed_offsets(lens)), q, k, v, do, 96 ** -0.5, causal)


@pytest.mark.parametrize("heads,kv,d,rows,batch", [(32, 32, 128, 2000, 4), (12, 12, 64, 2000, 32), (32, 8, 128, 512, 1), (64, 1, 64, 500, 1)])
def test_gradients_take_no_more_scratch_than_their_call(heads, kv, d, rows, batch):
    """What the call itself asks for, and not room for every smaller one."""
    q, k, v, do = make(rows, rows, heads, kv, d)
    a, off = rt.Attention(heads, d, kv_heads=kv, causal=True), rt.packed_offsets([rows // batch] * (batch - 1) + [rows - rows // batch * (batch - 1)])
    o, lse = torch.empty_like(q), torch.empty(heads, rows, device="cuda")
    a.forward(q, k, v, off, o, lse)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    a.backward(q, k, v, off, o, lse, do, dq, dk, dv)
    assert torch.cuda.max_memory_allocated() - before <= pb.pac_attn_backward_bytes(a._a, batch, rows) + 512  # (the allocator's granularity)


@pytest.mark.parametrize("heads,kv,d,n,causal", [(16, 4, 128, 2500, True), (16, 16, 64, 3001, False), (24, 8, 96, 2600, True), (20, 20, 32, 2111, True), (8, 2, 104, 2333, False)])
def test_long_sequences_of_128_rows_a_workgroup(heads, kv, d, n, causal):
    assert not few(heads, d, 1, n, causal)
    q, k, v, do = make(n, n, heads, kv, d, 1.5)
    a = rt.Attention(heads, d, kv_heads=kv, causal=causal)
    check(a, [n], run(a, q, k, v, do, rt.packed_offsets([n])), q, k, v, do, d ** -0.5, causal)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
@pytest.mark.parametrize("heads,d,n", [(192, 32, 200), (192, 64, 200), (96, 96, 150), (96, 72, 161), (96, 128, 200), (2, 32, 200), (3, 64, 300), (2, 96, 200), (2, 128, 150)])
def test_values_that_are_none_beside_the_mask(heads, d, n, which, bad):
    """A value that is infinite or no number, in the last head alone, at places all over the tiles of 32 and 128 rows: who does not see it stays within
    the oracle's bound of the exact values without it, rows of the same tile among them, and the other heads keep their bits."""
    assert few(heads, d, 1, n, True) == (heads < 10)
    clean = dict(zip(("q", "k", "v", "do"), make(d + n, n, heads, heads, d)))
    a, off = rt.Attention(heads, d, causal=True), rt.packed_offsets([n])
    ref = run(a, *clean.values(), off)
    last, row, col = slice((heads - 1) * d, heads * d), torch.arange(n, device="cuda"), 5
    x = {name: t[:, last].double()[None] for name, t in clean.items()}
    o, lse, p, eps = ao.forward(x["q"], x["k"], x["v"], d ** -0.5, True)
    grads, bounds = ao.backward(*x.values(), d ** -0.5, True)
    exact = (o[0], lse[0][:, None], *(t[0] for t in grads))
    bounds = (ao.forward_bound(p, x["v"], o, eps)[0], torch.full((n, 1), 2 * eps + 4 * ao.F32 * float(lse.abs().amax()), device="cuda"), *(t[0] for t in bounds))
    for at in (0, 33, 127, n - 1):
        t = {name: y.clone() for name, y in clean.items()}
        t[which][at, last.start + col] = bad
        got = run(a, *t.values(), off)
        for g, r, e, b, out in zip(got, ref, exact, bounds, ("o", "lse", "dq", "dk", "dv")):
            mine, others = (g[-1:].t(), (g[:-1], r[:-1])) if out == "lse" else (g[:, last], (g[:, :last.start], r[:, :last.start]))
            assert torch.equal(*others), (at, out, "other heads")
            if which == "do" and out in ("o", "lse") or which == "v" and out == "lse":
                same = torch.ones_like(row, dtype=torch.bool)
            elif out in ("dk", "dv"):  # keys see the rows from their own on
                same = row > at if which in ("q", "do") else torch.zeros_like(row, dtype=torch.bool)
            else:
                same = row != at if which in ("q", "do") else row < at
            away = (mine.double() - e).abs()
            assert bool((away <= b)[same].all()), (at, out)
            if which == "v" and out == "o":  # one column of it
                rest = torch.arange(d, device="cuda") != col
                assert bool((away <= b)[:, rest].all()), (at, "the other columns")
                assert (mine[at:, col].isnan() if math.isnan(bad) else mine[at:, col] == bad).all()
            if which == "do" and out == "dv":
                rest = torch.arange(d, device="cuda") != col
                assert bool((away <= b)[:, rest].all()) and not mine[:at + 1, col].isfinite().any(), at
            if (which, out) in (("q", "o"), ("q", "lse"), ("q", "dq"), ("do", "dq")):
                assert not mine[at].isfinite().all(), (at, out)


def test_results_a_row_beside_an_operand_are_refused():
    """q in rows 0..9 of one buffer, o in rows 1..10."""
    q, k, v, _ = make(0, 11, 4, 2, 64)
    a, off, lse = rt.Attention(4, 64, kv_heads=2), rt.packed_offsets([4, 6]), torch.empty(4, 10, device="cuda")
    keep = q.clone()
    for o, x in ((q[1:], q[:10]), (q[:10], q[1:])):
        with pytest.raises(pb.PacError) as e:
            a.forward(x, k[:10], v[:10], off, o, lse)
        assert e.value.status == pb.PAC_ERR_RANGE
    assert torch.equal(q, keep)


@pytest.mark.parametrize("heads,kv,d,n,causal", [(2, 2, 32, 200, True), (2, 1, 64, 300, False), (2, 2, 96, 257, True), (4, 2, 128, 200, True), (192, 96, 64, 150, True),
                                                 (96, 96, 128, 140, True), (96, 48, 96, 130, False), (96, 96, 32, 200, False), (64, 1, 64, 300, True)])
def test_delta_is_exact_where_o_is_rounded(heads, kv, d, n, causal):
    """Values and keys that have much in common, so that the rounded o's delta would miss dq and dk by several times the bounds (the oracle's own test
    shows by how much)."""
    g = heads // kv
    q, k, v, do = make(n + d, n, heads, kv, d)
    k, v = (k.float() + 4).to(BF), (v.float() + 32).to(BF)
    scale = d ** -0.5 / 4
    a = rt.Attention(heads, d, kv_heads=kv, causal=causal, scale=scale)
    got = run(a, q, k, v, do, rt.packed_offsets([n]))
    for h in range(0, kv, max(1, kv // 5)):
        mine, kvs = slice(h * g * d, (h + 1) * g * d), slice(h * d, (h + 1) * d)
        by = lambda t, c: t[:, c].double().reshape(n, -1, d).transpose(0, 1)  # noqa: E731
        for name, t, c, (r, b) in zip(("dq", "dk"), (got[2], got[3]), (mine, kvs),
                                      ao.exact_delta_bounds(by(q, mine), by(k, kvs), by(v, kvs), by(do, mine), by(got[0], mine), scale, causal)):
            off = (by(t, c) - r).abs()
            assert bool((off <= b).all()), (name, h, float((off / b).amax()))
