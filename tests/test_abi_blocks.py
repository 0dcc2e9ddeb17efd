"""CPU-only checks of the entry points for the backbone's blocks: sizes of the stored form, and arguments that are refused on the
host before anything is launched (no GPU needed; no address is ever read)."""
import ctypes as C

import pytest

from oracle import block_oracle as bo
from paper_2408_10746_amd import binding as pb

A = 1 << 20  # an aligned address that no refused call touches


def test_pitches_of_the_stored_form():
    for cols in (1, 31, 32, 255, 256, 257, 4096, 4097, 1 << 28):
        assert (pb.pac_mx4_code_pitch(cols), pb.pac_mx4_scale_pitch(cols)) == bo.pitches(cols)
    assert pb.pac_mx4_code_pitch(0) == -1 and pb.pac_mx4_scale_pitch(-3) == -1


def test_conversions_refuse():
    L = pb.lib()

    def q(x=A, dt=pb.PAC_F32, rows=4, cols=40, stride=40, codes=A, scales=A):
        one = L.pac_mx4_quantize(x, dt, rows, cols, stride, codes, scales, None)
        two = L.pac_mx4_dequantize(codes, scales, rows, cols, x, dt, stride, None)
        assert one == two
        return one

    assert q(rows=0) == q(rows=0, x=None, codes=None, scales=None) == pb.PAC_OK
    assert q(x=None) == q(codes=None) == q(scales=None) == pb.PAC_ERR_NULL
    assert q(cols=0) == q(dt=2) == pb.PAC_ERR_SHAPE
    assert q(rows=-1) == q(stride=39) == pb.PAC_ERR_RANGE
    assert q(x=A + 2) == q(codes=A + 8) == q(scales=A + 4) == q(x=A + 1, dt=pb.PAC_BF16) == pb.PAC_ERR_ALIGN
    assert q(rows=1 << 30, cols=1000, stride=1000) == q(cols=(1 << 28) + 1, stride=1 << 29) == pb.PAC_ERR_UNSUPPORTED


def test_products_refuse():
    L = pb.lib()

    def lin(x=A, M=4, K=40, sx=40, codes=A, scales=A, N=7, bias=None, act=0, y=A, dt=pb.PAC_F32, sy=7):
        return L.pac_mx4_linear(x, M, K, sx, codes, scales, N, bias, act, y, dt, sy, None)

    def lin4(x=A, xs=A, M=4, K=40, codes=A, scales=A, N=7, bias=None, act=0, y=A, dt=pb.PAC_F32, sy=7):
        return L.pac_mx4_linear_x4(x, xs, M, K, codes, scales, N, bias, act, y, dt, sy, None)

    def dx(dy=A, M=4, N=7, sdy=8, codes=A, scales=A, K=40, out=A, dt=pb.PAC_F32, sdx=40):
        return L.pac_mx4_linear_dx(dy, M, N, sdy, codes, scales, K, out, dt, sdx, None)

    assert lin(M=0, x=None, y=None) == lin4(M=0, x=None, xs=None, y=None) == dx(M=0, dy=None, out=None) == pb.PAC_OK
    for k in ("x", "codes", "scales", "y"):
        assert lin(**{k: None}) == lin4(**{k: None}) == pb.PAC_ERR_NULL
    assert lin4(xs=None) == dx(dy=None) == dx(out=None) == dx(codes=None) == dx(scales=None) == pb.PAC_ERR_NULL
    for f in (lin, lin4, dx):
        assert f(M=-1) == f(K=0) == f(N=0) == f(dt=5) == pb.PAC_ERR_SHAPE
        assert f(codes=A + 8) == f(scales=A + 4) == pb.PAC_ERR_ALIGN
        assert f(M=(1 << 28) + 1) == f(K=(1 << 28) + 1) == f(N=(1 << 28) + 1) == pb.PAC_ERR_UNSUPPORTED
    assert lin(act=2) == lin4(act=-1) == pb.PAC_ERR_SHAPE
    assert lin(sx=32) == lin(sy=6) == lin4(sy=6) == dx(sdy=6) == dx(sdx=39) == pb.PAC_ERR_RANGE
    assert lin(sx=44) == lin(x=A + 8) == lin(y=A + 2) == lin(bias=A + 2) == lin4(x=A + 8) == lin4(xs=A + 4) == pb.PAC_ERR_ALIGN
    assert dx(sdy=12) == dx(dy=A + 8) == dx(out=A + 1, dt=pb.PAC_BF16) == pb.PAC_ERR_ALIGN
    assert pb.pac_mx4_linear_qx_workspace_bytes(4, 40) == 4 * 136 and pb.pac_mx4_linear_qx_workspace_bytes(-1, 40) == -1
    assert pb.pac_mx4_linear_qx_workspace_bytes(4, 0) == -1

    def linq(x=A, xdt=pb.PAC_BF16, M=4, K=40, sx=40, codes=A, scales=A, N=7, bias=None, act=0, y=A, dt=pb.PAC_F32, sy=7, ws=A, n=4 * 136):
        return L.pac_mx4_linear_qx(x, xdt, M, K, sx, codes, scales, N, bias, act, y, dt, sy, ws, n, None)

    assert linq(M=0, x=None, y=None, ws=None, n=0) == pb.PAC_OK
    assert linq(x=None) == linq(codes=None) == linq(scales=None) == linq(y=None) == linq(ws=None) == pb.PAC_ERR_NULL
    assert linq(M=-1) == linq(K=0) == linq(N=0) == linq(dt=5) == linq(xdt=5) == linq(act=2) == pb.PAC_ERR_SHAPE
    assert linq(sx=39) == linq(sy=6) == pb.PAC_ERR_RANGE and linq(n=4 * 136 - 1) == pb.PAC_ERR_WORKSPACE
    assert linq(x=A + 1) == linq(x=A + 2, xdt=pb.PAC_F32) == linq(codes=A + 8) == linq(scales=A + 4) == linq(bias=A + 2) == linq(ws=A + 8) == pb.PAC_ERR_ALIGN
    assert linq(M=(1 << 28) + 1) == linq(K=(1 << 28) + 1, sx=1 << 29) == pb.PAC_ERR_UNSUPPORTED
    big = 1 << 28
    assert lin(M=big, N=big, sy=big) == lin4(M=big, N=big, sy=big) == dx(M=big, K=big, sdx=big) == pb.PAC_ERR_UNSUPPORTED


def norm(d=8, dtype=pb.PAC_F32, layer=0, gate_len=0, eps=1e-5, w_post=None, b_post=None, gate=None, res=None, w_pre=None, b_pre=None):
    return pb.pac_block_norm(d, dtype, layer, gate_len, eps, w_post, b_post, gate, res, w_pre, b_pre)


@pytest.mark.parametrize("kw,want", [
    (dict(d=0), pb.PAC_ERR_SHAPE), (dict(d=16385), pb.PAC_ERR_SHAPE), (dict(dtype=2), pb.PAC_ERR_SHAPE), (dict(layer=2), pb.PAC_ERR_SHAPE),
    (dict(eps=0.0), pb.PAC_ERR_SHAPE), (dict(eps=float("nan")), pb.PAC_ERR_SHAPE), (dict(eps=float("inf")), pb.PAC_ERR_SHAPE),
    (dict(gate=A), pb.PAC_ERR_SHAPE), (dict(gate=A, gate_len=7), pb.PAC_ERR_SHAPE), (dict(gate_len=1), pb.PAC_ERR_SHAPE),
    (dict(b_post=A), pb.PAC_ERR_NULL), (dict(b_pre=A), pb.PAC_ERR_NULL),
    (dict(w_post=A + 2), pb.PAC_ERR_ALIGN), (dict(gate=A + 1, gate_len=1), pb.PAC_ERR_ALIGN), (dict(res=A + 2), pb.PAC_ERR_ALIGN)])
def test_norm_structures_that_are_refused(kw, want):
    L, b = pb.lib(), norm(**kw)
    assert L.pac_block_norm_forward(C.byref(b), 2, A, A, A, None, None) == want
    assert L.pac_block_norm_backward(C.byref(b), 2, A, A, A, None, A, A, *[None] * 7, 0, None) == want
    assert pb.pac_block_norm_workspace_bytes(b, 2) == -1


def test_norm_calls_refuse():
    L = pb.lib()
    b = norm(w_post=A, w_pre=A, res=A, gate=A, gate_len=8)
    f = lambda b=b, rows=2, x=A, o=A, y=A, n=A: L.pac_block_norm_forward(C.byref(b), rows, x, o, y, n, None)  # noqa: E731
    assert f(rows=0, x=None, o=None, y=None, n=None) == pb.PAC_OK and L.pac_block_norm_forward(None, 0, A, A, A, A, None) == pb.PAC_ERR_NULL
    assert f(x=None) == f(o=None) == f(n=None) == f(b=norm(), n=A) == f(b=norm(), n=None, y=None) == pb.PAC_ERR_NULL
    assert f(rows=-1) == pb.PAC_ERR_RANGE
    assert f(x=A + 2) == f(o=A + 2) == f(y=A + 2) == f(n=A + 2) == pb.PAC_ERR_ALIGN
    need = pb.pac_block_norm_workspace_bytes(b, 2)
    assert need > 0 and need % 256 == 0 and pb.pac_block_norm_workspace_bytes(b, 1 << 40) > need

    def g(b=b, rows=2, x=A, o=A, dy=A, dn=A, dx=A, do=A, wp=A, bp=None, ga=A, re=A, wn=A, bn=None, ws=A, n=need):
        return L.pac_block_norm_backward(C.byref(b), rows, x, o, dy, dn, dx, do, wp, bp, ga, re, wn, bn, ws, n, None)

    assert g(x=None) == g(o=None) == g(dn=None) == g(bp=A) == g(bn=A) == g(ws=None) == pb.PAC_ERR_NULL
    assert g(b=norm(), dn=None, dy=None) == g(b=norm(), dn=A) == g(b=norm(), dn=None, wp=None, ga=None, wn=None) == pb.PAC_ERR_NULL
    assert g(rows=-1) == pb.PAC_ERR_RANGE and g(n=need - 1) == pb.PAC_ERR_WORKSPACE
    assert g(ws=A + 8) == g(dy=A + 2) == g(do=A + 2) == g(wp=A + 2) == g(re=A + 1) == pb.PAC_ERR_ALIGN


def test_tiles_of_the_products():
    """Host logic: every form of the three products is taken somewhere, and the line between them follows the sizes."""
    t = pb.pac_mx4_tiles
    assert t(0, 1, 4096, 4096) == t(1, 1, 4096, 4096) == (16, 16) and t(2, 1, 4096, 4096) == (16, 128)
    assert t(0, 4096, 4096, 4096) == t(1, 4096, 4096, 4096) == t(2, 4096, 4096, 4096) == (256, 256)
    assert t(0, 64, 4096, 4096) == (64, 64) and t(0, 1024, 2048, 4096) == (64, 128) and t(0, 5913, 541, 655) == (128, 128)
    assert t(1, 64, 4096, 2048) == (32, 16) and t(1, 1024, 2048, 4096) == (128, 128)
    big = 1 << 28
    assert t(0, big, big, big) == t(2, big, big, big) == (256, 256)
    out = (C.c_int32 * 2)()
    L = pb.lib()
    assert L.pac_mx4_tiles(0, 1, 1, 1, None) == pb.PAC_ERR_NULL
    assert L.pac_mx4_tiles(3, 1, 1, 1, out) == L.pac_mx4_tiles(-1, 1, 1, 1, out) == L.pac_mx4_tiles(0, 0, 1, 1, out) == pb.PAC_ERR_SHAPE
    assert L.pac_mx4_tiles(0, 1, big + 1, 1, out) == pb.PAC_ERR_UNSUPPORTED


@pytest.mark.parametrize("d", [40, 96, 768, 1032, 4096, 5120, 16384])
def test_a_workspace_for_many_rows_serves_fewer(d):
    """A caller sizes one workspace for its largest batch: the bytes never fall as rows grow (forms of every width)."""
    b = norm(d=d, w_post=A)
    for rows in (range(1, 2001), range(2001, 40000, 97), [1 << k for k in range(16, 40)]):
        need = [pb.pac_block_norm_workspace_bytes(b, r) for r in rows]
        assert need[0] > 0 and need == sorted(need)
    assert pb.pac_block_norm_workspace_bytes(b, 0) <= pb.pac_block_norm_workspace_bytes(b, 1)


@pytest.mark.parametrize("d", [40, 768, 4096, 16384])
def test_blocks_add_at_most_64_rows_one_after_another(d):
    """The workspace holds a block's sums, 16 bytes a column and 16 more; a block of narrow rows takes eight side by side."""
    b, side = norm(d=d, w_post=A), {40: 8, 768: 2}.get(d, 1)
    for rows in (1 << 16, 1 << 20, (1 << 26) + 1):
        assert pb.pac_block_norm_workspace_bytes(b, rows) >= rows / (64 * side) * (16 + 16 * d)


def test_tiles_fit_a_launch():
    """A launch takes fewer than 2^32 threads, 2^23 blocks of 512: a form with more tiles gives way to one with fewer."""
    t = pb.pac_mx4_tiles
    assert t(0, 1, 1024, (1 << 27) - 16) == (16, 16)
    for product in (0, 1, 2):
        for M, K, N in ((1, 1024, 1 << 27), (1, 1024, 1 << 28), (16, 2048, 1 << 28), (1, 1 << 28, 1 << 11), (1 << 28, 32, 16), (1 << 28, 16, 32), (1 << 28, 1, 1)):
            rows, cols = t(product, M, K, N)
            assert -(-M // rows) * -(-(K if product == 2 else N) // cols) < 1 << 23, (product, M, K, N)
