"""CPU-only checks of the entry points of attention and the 4-bit key and value cache: sizes, and arguments that are refused on the host
before anything is launched (no GPU needed; no address is ever read)."""
import ctypes as C
import math

import pytest

from paper_2408_10746_amd import binding as pb

A = 1 << 20  # an aligned address that no refused call touches
FAR = [A * (2 * k + 1) for k in range(16)]


def attn(heads=4, kv_heads=2, d=64, causal=0, scale=0.125):
    return pb.pac_attn(heads, kv_heads, d, causal, scale)


def forward(a=None, off=FAR[0], batch=2, rows=10, q=FAR[1], sq=256, k=FAR[2], sk=128, v=FAR[3], sv=128, o=FAR[4], so=256, lse=FAR[5]):
    return pb.lib().pac_attn_forward(C.byref(a or attn()), off, batch, rows, q, sq, k, sk, v, sv, o, so, lse, None)


def backward(a=None, off=FAR[0], batch=2, rows=10, q=FAR[1], sq=256, k=FAR[2], sk=128, v=FAR[3], sv=128, o=FAR[4], so=256, lse=FAR[5], do=FAR[6],
             sdo=256, dq=FAR[7], sdq=256, dk=FAR[8], sdk=128, dv=FAR[9], sdv=128, ws=FAR[10], n=1 << 30):
    return pb.lib().pac_attn_backward(C.byref(a or attn()), off, batch, rows, q, sq, k, sk, v, sv, o, so, lse, do, sdo, dq, sdq, dk, sdk, dv, sdv,
                                      ws, n, None)


@pytest.mark.parametrize("kw", [dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(heads=4098, kv_heads=1), dict(d=0), dict(d=12), dict(d=136),
                                dict(d=-8), dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan)])
def test_attention_structures_that_are_refused(kw):
    assert forward(attn(**kw)) == backward(attn(**kw)) == pb.PAC_ERR_SHAPE
    assert pb.pac_attn_workspace_bytes(attn(**kw), 2, 10) == -1


def test_attention_calls_refuse():
    for f in (forward, backward):
        assert f(batch=0) == f(rows=0) == f(rows=0, q=None, k=None, v=None, o=None) == pb.PAC_OK
        for name in ("off", "q", "k", "v", "o"):
            assert f(**{name: None}) == pb.PAC_ERR_NULL, name
            assert f(**{name: A + 2}) == pb.PAC_ERR_ALIGN, name
        for name in ("sq", "sk", "sv", "so"):
            assert f(**{name: 120}) == pb.PAC_ERR_RANGE and f(**{name: 260}) == pb.PAC_ERR_ALIGN and f(**{name: (1 << 24) + 8}) == pb.PAC_ERR_UNSUPPORTED
        assert f(batch=-1) == pb.PAC_ERR_SHAPE and f(rows=-1) == f(rows=1 << 31) == pb.PAC_ERR_RANGE
        assert f(lse=A + 2) == pb.PAC_ERR_ALIGN
        assert f(batch=1 << 22) == f(rows=1 << 29, a=attn(64, 64)) == pb.PAC_ERR_UNSUPPORTED
    L = pb.lib()
    assert L.pac_attn_forward(None, *[FAR[0], 1, 1], *[FAR[1], 256] * 4, None, None) == pb.PAC_ERR_NULL
    for name in ("lse", "do", "dq", "dk", "dv", "ws"):
        assert backward(**{name: None}) == pb.PAC_ERR_NULL, name
        assert backward(**{name: A + 2}) == pb.PAC_ERR_ALIGN, name
    for name in ("sdo", "sdq", "sdk", "sdv"):
        assert backward(**{name: 120}) == pb.PAC_ERR_RANGE, name
    need = pb.pac_attn_workspace_bytes(attn(), 2, 10)
    assert need > 0 and backward(n=need - 1) == pb.PAC_ERR_WORKSPACE


def test_attention_results_that_share_memory_are_refused():
    for other in (FAR[1], FAR[2], FAR[3], FAR[5], FAR[1] + 10 * 512 - 16):
        assert forward(o=other) == pb.PAC_ERR_RANGE
    assert forward(lse=FAR[1]) == forward(lse=FAR[0]) == pb.PAC_ERR_RANGE
    for name in ("dq", "dk", "dv", "ws"):
        for other in FAR[:10]:
            own = dict(dq=FAR[7], dk=FAR[8], dv=FAR[9], ws=FAR[10])[name]
            if other != own:
                assert backward(**{name: other}) == pb.PAC_ERR_RANGE, (name, other)


def test_a_workspace_for_many_rows_serves_fewer():
    for a in (attn(), attn(64, 1, 128), attn(1, 1, 8), attn(32, 8, 96, 1)):
        for many in (range(0, 300), range(0, 200000, 977)):
            need = [pb.pac_attn_workspace_bytes(a, 3, r) for r in many]
            assert need[0] >= 0 and need == sorted(need)
        need = [pb.pac_attn_workspace_bytes(a, b, 1000) for b in range(0, 3000, 7)]
        assert need == sorted(need)


def kv4(at=A * 4, pages=10, page=16, kv_heads=2, d=64):
    return pb.pac_kv4(at, pages, page, kv_heads, d)


@pytest.mark.parametrize("kw", [dict(pages=-1), dict(pages=1 << 31), dict(page=0), dict(page=4), dict(page=24), dict(page=1 << 17), dict(kv_heads=0),
                                dict(kv_heads=4097), dict(d=0), dict(d=4), dict(d=136), dict(d=-8)])
def test_caches_that_are_refused(kw):
    c = kv4(**kw)
    L = pb.lib()
    assert pb.pac_kv4_bytes(c) == -1 and pb.pac_kv4_attend_workspace_bytes(c, 2, 1, 1) == -1
    for f in (L.pac_kv4_write, L.pac_kv4_read):
        assert f(C.byref(c), 1, A, 2 * A, 1 << 20, 3 * A, 1 << 20, pb.PAC_F32, None) == pb.PAC_ERR_SHAPE
    assert L.pac_kv4_attend(C.byref(c), 4096, 1.0, 1, A, 1, 1, A, A, 1 << 20, A, 1 << 20, A, 1 << 40, None) == pb.PAC_ERR_SHAPE


def test_cache_sizes():
    for d, blocks in ((8, 1), (32, 1), (40, 2), (64, 2), (72, 3), (96, 3), (104, 4), (128, 4)):
        assert pb.pac_kv4_bytes(kv4(None, 10, 16, 3, d)) == 10 * 16 * 3 * 2 * blocks * 17
    assert pb.pac_kv4_bytes(kv4(None, 0)) == 0
    assert pb.pac_kv4_bytes(kv4(None, (1 << 31) - 1, 65536, 1, 128)) == ((1 << 31) - 1) * 65536 * 136


def test_cache_conversions_refuse():
    L = pb.lib()

    def go(f, c=None, rows=4, slots=A, k=2 * A, sk=128, v=3 * A, sv=128, dt=pb.PAC_F32):
        return f(C.byref(c or kv4()), rows, slots, k, sk, v, sv, dt, None)

    for f in (L.pac_kv4_write, L.pac_kv4_read):
        assert go(f, rows=0) == go(f, rows=0, slots=None, k=None, v=None) == pb.PAC_OK
        assert f(None, 1, A, A, 128, A, 128, pb.PAC_F32, None) == pb.PAC_ERR_NULL
        assert go(f, slots=None) == go(f, k=None) == go(f, v=None) == go(f, kv4(at=None)) == pb.PAC_ERR_NULL
        assert go(f, dt=2) == pb.PAC_ERR_SHAPE
        assert go(f, rows=-1) == go(f, sk=127) == go(f, sv=100) == pb.PAC_ERR_RANGE
        assert go(f, kv4(at=4 * A + 8)) == go(f, slots=A + 4) == go(f, k=2 * A + 2) == go(f, v=3 * A + 1, dt=pb.PAC_BF16) == pb.PAC_ERR_ALIGN
        assert go(f, rows=1 << 30) == go(f, rows=1 << 62) == pb.PAC_ERR_UNSUPPORTED
        size = pb.pac_kv4_bytes(kv4())
        assert go(f, k=4 * A) == go(f, v=4 * A + size - 4) == go(f, slots=4 * A + 16) == go(f, k=4 * A - 16) == pb.PAC_ERR_RANGE
        assert go(f, kv4(at=None, pages=0)) == pb.PAC_OK
    assert go(L.pac_kv4_read, v=2 * A) == go(L.pac_kv4_read, slots=2 * A + 16) == go(L.pac_kv4_read, slots=3 * A) == pb.PAC_ERR_RANGE


def test_attending_refuses():
    L = pb.lib()
    big = 1 << 40

    def go(c=None, heads=4, scale=0.125, batch=3, table=A, tl=5, ts=5, lens=2 * A, q=3 * A, sq=256, o=big, so=256, ws=2 * big, n=1 << 30):
        return L.pac_kv4_attend(C.byref(c or kv4()), heads, scale, batch, table, tl, ts, lens, q, sq, o, so, ws, n, None)

    assert go(batch=0) == go(batch=0, table=None, lens=None, q=None, o=None) == pb.PAC_OK
    assert go(lens=None) == go(q=None) == go(o=None) == go(table=None) == go(kv4(at=None)) == pb.PAC_ERR_NULL
    assert go(heads=0) == go(heads=3) == go(heads=8192) == go(batch=-1) == go(tl=-1) == pb.PAC_ERR_SHAPE
    assert go(scale=0.0) == go(scale=-1.0) == go(scale=math.nan) == go(scale=math.inf) == pb.PAC_ERR_RANGE
    assert go(sq=255) == go(so=8) == go(ts=4) == pb.PAC_ERR_RANGE
    assert go(table=A + 2) == go(lens=2 * A + 1) == go(q=3 * A + 8) == go(o=big + 2) == go(sq=260) == go(so=260) == pb.PAC_ERR_ALIGN
    assert go(kv4(page=65536), tl=1 << 15, ts=1 << 15) == go(batch=1 << 22) == pb.PAC_ERR_UNSUPPORTED
    long = kv4(page=65536, pages=4)
    need = pb.pac_kv4_attend_workspace_bytes(long, 4, 1, 4)
    assert need > 0
    assert go(long, batch=1, tl=4, n=100) == pb.PAC_ERR_WORKSPACE and go(long, batch=1, tl=4, ws=None) == pb.PAC_ERR_NULL
    assert go(long, batch=1, tl=4, ws=2 * big + 8) == pb.PAC_ERR_ALIGN and go(long, batch=1, tl=4, ws=A) == pb.PAC_ERR_RANGE
    assert go(o=3 * A) == go(o=A) == go(o=2 * A) == go(o=4 * A) == go(o=4 * A + pb.pac_kv4_bytes(kv4()) - 16) == pb.PAC_ERR_RANGE


@pytest.mark.parametrize("heads,kv_heads,d,page", [(4, 2, 64, 16), (32, 8, 128, 64), (32, 1, 96, 8), (40, 40, 32, 1024)])
def test_a_workspace_for_a_large_batch_serves_smaller_ones(heads, kv_heads, d, page):
    c = kv4(kv_heads=kv_heads, d=d, page=page)
    need = lambda b, t: pb.pac_kv4_attend_workspace_bytes(c, heads, b, t)  # noqa: E731
    for t in (0, 1, 7, 100, 5000):
        by = [need(b, t) for b in range(0, 400)]
        assert by[0] >= 0 and by == sorted(by)
    for b in (1, 3, 64):
        by = [need(b, t) for t in range(0, 3000, 13)]
        assert by == sorted(by)


def test_caches_whose_bytes_are_no_number_are_refused():
    for pages, page, kv_heads, d in (((1 << 31) - 1, 65536, 4096, 128), (1 << 30, 32768, 4096, 72), ((1 << 31) - 1, 65536, 964, 128)):
        c = kv4(None, pages, page, kv_heads, d)
        assert pb.pac_kv4_bytes(c) == pb.pac_kv4_attend_workspace_bytes(c, kv_heads, 1, 1) == -1
    c = kv4(None, 1 << 30, 65536, 481, 128)  # as large as it gets
    assert pb.pac_kv4_bytes(c) == (1 << 30) * 65536 * 481 * 136 < 1 << 62


def test_tables_near_the_last_token_number_are_refused():
    """Token numbers have 32 bits and run a little past a sequence's end: the last few thousand are not for tables."""
    L = pb.lib()
    for page, refused, taken in ((8, (1 << 28) - 1, (1 << 28) - 513), (4096, (1 << 19) - 1, (1 << 19) - 2), (65536, (1 << 15) - 0, (1 << 15) - 1)):
        c = kv4(page=page, kv_heads=1)
        assert pb.pac_kv4_attend_workspace_bytes(c, 2, 1, refused) == -1 and pb.pac_kv4_attend_workspace_bytes(c, 2, 1, taken) > 0
        assert L.pac_kv4_attend(C.byref(c), 2, 1.0, 1, A, refused, refused, 1 << 50, 1 << 51, 128, 1 << 52, 128, 1 << 53, 1 << 40, None) == pb.PAC_ERR_UNSUPPORTED


def test_the_bound_of_the_workspace_is_enough_for_the_call():
    """A call that has as much as the bound says is refused for something else (dq in q's place)."""
    for heads, kv_heads, d in ((1, 1, 8), (8, 8, 64), (32, 8, 128), (64, 1, 64), (12, 12, 96), (500, 500, 8), (4096, 1, 128)):
        for causal in (0, 1):
            a = attn(heads, kv_heads, d, causal)
            far = [(1 << 45) * (k + 1) for k in range(11)]
            for batch in (1, 2, 5, 64, 300):
                for rows in (1, 31, 127, 128, 200, 1000, 1023, 5000, 16383, 16384, 70000, 200000):
                    if (rows // 128 + batch) * heads >= 1 << 23:
                        continue
                    sq, sk = heads * d, kv_heads * d
                    n = pb.pac_attn_workspace_bytes(a, batch, rows)
                    got = backward(a, far[0], batch, rows, far[1], sq, far[2], sk, far[3], sk, far[4], sq, far[5], far[6], sq, far[1], sq, far[7], sk, far[8], sk, far[9], n)
                    assert got == pb.PAC_ERR_RANGE, (heads, kv_heads, d, causal, batch, rows)


def test_attention_scales_whose_product_with_log2_e_is_none_are_refused():
    """Scores are taken times scale log2(e), in 32 bits: where that is infinite, a score of 0 would become none."""
    for scale, want in ((2.36e38, False), (3.4e38, False), (2.35e38, True), (1e-45, True)):
        a = attn(scale=scale)
        assert (pb.pac_attn_workspace_bytes(a, 2, 10) >= 0) == want, scale
        if not want:
            assert forward(a) == backward(a) == pb.PAC_ERR_SHAPE, scale


def test_attending_with_a_scale_whose_product_with_log2_e_is_none_is_refused():
    L, c, far = pb.lib(), kv4(), [1 << (40 + k) for k in range(5)]
    for scale, want in ((2.36e38, pb.PAC_ERR_RANGE), (3.4e38, pb.PAC_ERR_RANGE), (2.35e38, pb.PAC_OK), (1e-45, pb.PAC_OK)):
        assert L.pac_kv4_attend(C.byref(c), 4, scale, 0, far[0], 5, 5, far[1], far[2], 256, far[3], 256, far[4], 1 << 30, None) == want, scale


def test_the_bytes_of_a_call_are_what_the_call_asks_for():
    """No more than the bound for all smaller calls, and just what is refused when it is less (dq in q's place: with enough, that is what is refused)."""
    far = [(1 << 45) * (k + 1) for k in range(11)]
    for heads, kv_heads, d in ((1, 1, 8), (12, 12, 64), (32, 8, 128), (64, 1, 64), (500, 500, 8)):
        for causal in (0, 1):
            a = attn(heads, kv_heads, d, causal)
            for batch in (1, 2, 8, 64):
                for rows in (1, 127, 128, 512, 1000, 5000, 16384, 70000):
                    need, sq, sk = pb.pac_attn_backward_bytes(a, batch, rows), heads * d, kv_heads * d
                    assert 0 < need <= pb.pac_attn_workspace_bytes(a, batch, rows)
                    go = lambda n: backward(a, far[0], batch, rows, far[1], sq, far[2], sk, far[3], sk, far[4], sq, far[5], far[6], sq, far[1], sq, far[7], sk, far[8], sk, far[9], n)  # noqa: E731
                    assert go(need - 1) == pb.PAC_ERR_WORKSPACE and go(need) == pb.PAC_ERR_RANGE, (heads, kv_heads, d, causal, batch, rows)
    # two fp32 numbers a row and head where the queries are not dealt out, whatever smaller calls may take
    assert pb.pac_attn_backward_bytes(attn(32, 32, 128, 1), 8, 5120) == 2 * 5120 * 32 * 4
    assert pb.pac_attn_backward_bytes(attn(heads=3), 2, 10) == pb.pac_attn_backward_bytes(attn(), 2, -1) == pb.pac_attn_backward_bytes(attn(), -1, 10) == -1
    assert pb.pac_attn_backward_bytes(attn(), 0, 10) == 2 * 256 and pb.pac_attn_backward_bytes(attn(), 2, 0) == 0


def test_the_bytes_of_an_attend_are_what_it_asks_for():
    """No more than the bound for all smaller calls, and just what is refused when it is less; nothing where a sequence and head has one workgroup."""
    L, far = pb.lib(), [1 << (40 + k) for k in range(6)]
    for heads, kv_heads, d in ((1, 1, 8), (32, 8, 128), (32, 32, 64), (48, 3, 96), (64, 1, 128)):
        for page, tables in ((16, (0, 1, 50, 700, 5000)), (1024, (1, 3, 64))):
            c = kv4(1 << 50, 1 << 20, page, kv_heads, d)
            for batch in (1, 2, 7, 64, 500, 4096):
                for tl in tables:
                    need = pb.pac_kv4_attend_bytes(c, heads, batch, tl)
                    assert 0 <= need <= pb.pac_kv4_attend_workspace_bytes(c, heads, batch, tl)
                    # (o in q's place: with enough, that is what is refused)
                    go = lambda n: L.pac_kv4_attend(C.byref(c), heads, 0.1, batch, far[0], tl, tl, far[1], far[2], heads * d, far[2], heads * d, far[3], n, None)  # noqa: E731
                    assert go(need) == pb.PAC_ERR_RANGE and (need == 0 or go(need - 1) == pb.PAC_ERR_WORKSPACE), (heads, kv_heads, d, page, batch, tl)
    assert pb.pac_kv4_attend_bytes(kv4(kv_heads=8, d=128), 64, 4096, 100) == 0 < pb.pac_kv4_attend_bytes(kv4(kv_heads=8, d=128), 64, 4, 1000)
    assert pb.pac_kv4_attend_bytes(kv4(), 3, 1, 1) == pb.pac_kv4_attend_bytes(kv4(), 2, -1, 1) == pb.pac_kv4_attend_bytes(kv4(d=4), 2, 1, 1) == -1
