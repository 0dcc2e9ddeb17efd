"""GPU parity of microscaled 4-bit floating point (quantisation, its inverse, the products) against oracle/block_oracle.py.

Bars, derived from the arithmetic: codes, scale bytes and dequantised values equal; a product's elements within
2 K 2^-24 of the sum of the absolute products (each product is exact in fp32, and each of at most K additions loses at most one
unit in the last place of a partial sum that this sum bounds), the bias' and GELU's own part, and half a step of the output's type
(2^-8 bf16, 2^-24 fp32)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2408_10746_amd import binding as pb
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.cuda() if dtype is None else t.to(dtype).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


# ---- conversions -----------------------------------------------------------------------------------------------------------
def test_every_code_with_every_scale():
    scales = np.tile(np.arange(256, dtype=np.uint8).reshape(-1, 1), (1, 8))
    codes = np.tile(np.array([(2 * b) | ((2 * b + 1) << 4) for b in range(8)], np.uint8), (256, 16))
    ref = bo.values(codes, scales, 256)
    for name, dt in DT.items():
        out = torch.zeros(256, 256, dtype=dt, device="cuda")
        rt.mx4_dequantize(dev(codes), dev(scales), out)
        with np.errstate(over="ignore"):
            want = torch.from_numpy(ref).to(dt)         # 6 x 2^127 and its like pass the type's largest value
        got = out.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), name
        keep = ~torch.isnan(want)
        bad = (got[keep] != want[keep]).nonzero()
        assert bad.numel() == 0, (name, got[keep][bad[:4, 0]], want[keep][bad[:4, 0]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,stride", [(1, 1, 1), (3, 31, 31), (2, 32, 32), (5, 33, 40), (7, 255, 255), (4, 256, 256),
                                              (3, 257, 264), (70, 776, 776), (33, 1003, 1003), (9, 2048, 2056)])
def test_quantize_and_back(rows, cols, stride, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, stride)) * np.exp(rng.uniform(-20, 20, size=(rows, 1))) * np.exp(rng.uniform(-3, 3, size=(rows, stride)))
    x[:, :cols:5] = bo.GRID[rng.integers(0, 8, size=x[:, :cols:5].shape)]
    x[0, : min(cols, 32)] = 0.0
    xd = dev(x.astype(np.float32), DT[dtype])[:, :cols]
    ref_codes, ref_scales = bo.quantize(host(xd))
    codes, scales = rt.mx4_empty(rows, cols)
    codes.fill_(0xAA), scales.fill_(0xAA)               # the padding has to be written too
    rt.mx4_quantize(xd, codes, scales)
    assert np.array_equal(scales.cpu().numpy(), ref_scales)
    assert np.array_equal(codes.cpu().numpy(), ref_codes)
    out = torch.full((rows, stride), 7.0, dtype=DT[dtype], device="cuda")
    rt.mx4_dequantize(codes, scales, out[:, :cols])
    assert np.array_equal(host(out[:, :cols]), bo.values(ref_codes, ref_scales, cols))
    assert (out[:, cols:] == 7.0).all()                  # what lies past the columns is left alone


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_at_the_borders(dtype):
    """Ties, values next to them, saturation, infinities, NaN, denormals and the largest values, over the whole range of scales."""
    tie = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.9375])
    around = np.concatenate([tie, tie * (1 + 2.0 ** -7), tie * (1 - 2.0 ** -7)])
    row = np.zeros(32)
    row[:27], row[27], row[28] = around, 4.0, -0.0
    exps = np.arange(-149, 125)
    x = np.ldexp(row[None, :], exps[:, None]) * np.where(np.arange(32) % 3 == 0, -1.0, 1.0)
    x = np.concatenate([x, np.full((1, 32), np.finfo(np.float32).max), np.full((1, 32), -np.inf), np.where(np.arange(32) == 9, np.nan, 1.0)[None, :],
                        np.where(np.arange(32) == 31, np.inf, 0.0)[None, :], np.full((1, 32), 2.0 ** -149), np.full((1, 32), 2.0 ** -133)])
    xd = dev(x.astype(np.float32), DT[dtype])
    ref_codes, ref_scales = bo.quantize(host(xd))
    codes, scales = rt.mx4_empty(*x.shape)
    rt.mx4_quantize(xd, codes, scales)
    assert np.array_equal(scales.cpu().numpy(), ref_scales)
    # where zeros have a sign the value is what counts
    got, want = bo.values(codes.cpu().numpy(), scales.cpu().numpy(), 32), bo.values(ref_codes, ref_scales, 32)
    bad = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))))
    assert bad.size == 0, [(tuple(b), host(xd)[tuple(b)], got[tuple(b)], want[tuple(b)]) for b in bad[:8]]


# ---- products --------------------------------------------------------------------------------------------------------------
def layer(rng, N, K):
    w = rng.standard_normal((N, K)) / np.sqrt(K) * np.exp(rng.standard_normal((N, 1)))
    w.ravel()[rng.integers(0, N * K, size=max(1, N * K // 500))] *= 20.0
    codes, scales = bo.quantize(w) if N * K < 20000 else (None, None)
    if codes is None:
        cd, sd = rt.mx4_empty(N, K)
        rt.mx4_quantize(dev(w.astype(np.float32)), cd, sd)
        codes, scales = cd.cpu().numpy(), sd.cpu().numpy()
    return dev(codes), dev(scales), bo.values(codes, scales, K)


def rows_of(rng, M, K, junk=float("nan")):
    """bf16 rows that start on 16 bytes; what lies past them must not count."""
    stride = (K + 7) // 8 * 8 + 8
    t = torch.full((M, stride), junk, dtype=torch.bfloat16, device="cuda")
    t[:, :K] = dev(rng.standard_normal((M, K)) * np.exp(rng.uniform(-1, 1, size=(M, 1))), torch.bfloat16)
    return t[:, :K]


def bar(ref, absum, K, dtype, bias=None, gelu=False):
    err = 2 * K * 2.0 ** -24 * absum
    if bias is not None:
        err = err + 2.0 ** -23 * (absum + np.abs(bias))
    if gelu:
        # |GELU'| < 1.13; erf within 1.5e-7 and a few units of the last place of u itself
        err = 1.13 * err + 4e-7 * (absum + (0 if bias is None else np.abs(bias)))
    return err + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (np.abs(ref) + err) + 1e-38


def check(got, ref, err):
    assert got.shape == ref.shape and np.isfinite(got).all()
    worst = np.max(np.abs(got - ref) / err)
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 1), (1, 64, 16), (1, 4096, 128), (2, 33, 17), (16, 100, 31), (17, 256, 48), (31, 777, 130), (33, 512, 257), (64, 1000, 64),
          (65, 775, 100), (130, 1024, 300), (257, 320, 515), (300, 2048, 129), (520, 96, 1030)]


@pytest.mark.parametrize("x4", [False, True], ids=["x16", "x4"])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_linear(M, K, N, x4):
    rng = np.random.default_rng(M * 7 + K * 3 + N + x4)
    codes, scales, w = layer(rng, N, K)
    x = rows_of(rng, M, K)
    xv = host(x)
    if x4:
        xv = bo.values(*bo.quantize(xv), K)
    bias = rng.standard_normal(N)
    for dtype, use_bias, gelu in (("f32", False, False), ("bf16", True, True), ("f32", True, True), ("bf16", False, False)):
        b32 = bias.astype(np.float32).astype(np.float64) if use_bias else None
        ref, absum = bo.linear(xv, w, b32, int(gelu))
        store = torch.full((M, N + 3), 5.0, dtype=DT[dtype], device="cuda")
        y = store[:, :N]
        lin = rt.Mx4Linear(codes, scales, K, bias=dev(bias, torch.float32) if use_bias else None)
        lin.forward(x, y, gelu=gelu, x4=x4)
        check(host(y), ref, bar(ref, absum, K, dtype, b32, gelu))
        assert (store[:, N:] == 5.0).all()


@pytest.mark.parametrize("M,K,N", [(1, 8, 3), (1, 4096, 300), (5, 232, 77), (16, 1000, 64), (17, 2048, 33), (30, 777, 700), (2079, 32, 18), (300, 2048, 1030)])
def test_quantising_in_the_call_is_quantising_before_it(M, K, N):
    """The same bits from rows of any alignment and type, over the whole range of scales, with blocks that stand for nothing."""
    rng = np.random.default_rng(M + K + N)
    codes, scales, _ = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K)
    x = rows_of(rng, M, K)
    x *= torch.from_numpy(np.exp2(rng.integers(-140, 120, size=(M, 1)).astype(np.float64))).cuda()
    x[0, :5] = torch.tensor([0.25, -1.25, 2.5, 6.9, 0.0], device="cuda").bfloat16() * float(x[0].abs().max()) if K > 8 else 1.0
    if M > 3 and K > 70:
        x[2, 64], x[3, 3], x[1, :32] = float("inf"), float("nan"), 0
    xc, xs = rt.mx4_empty(M, K)
    rt.mx4_quantize(x, xc, xs)
    ref = torch.empty(M, N, device="cuda")
    pb.pac_mx4_linear_x4(xc.data_ptr(), xs.data_ptr(), M, K, codes.data_ptr(), scales.data_ptr(), N, None, 0, ref.data_ptr(), pb.PAC_F32, N,
                         torch.cuda.current_stream().cuda_stream)
    off = torch.empty(M * (K + 1) + 1, dtype=torch.bfloat16, device="cuda")[1:].as_strided((M, K), (K + 1, 1))
    off.copy_(x)
    for t in (x, off, x.float(), x.clone()):
        y = torch.empty(M, N, device="cuda")
        lin.forward(t, y, x4=True)
        same = (y == ref) | (torch.isnan(y) & torch.isnan(ref))
        assert same.all()


@pytest.mark.parametrize("M,K,N", SHAPES + [(1, 300, 4096), (40, 1030, 900)])
def test_input_grad(M, K, N):
    rng = np.random.default_rng(M * 5 + K + N * 11)
    codes, scales, w = layer(rng, N, K)
    dy = rows_of(rng, M, N)
    ref, absum = bo.linear(host(dy), w.T)
    for dtype in ("f32", "bf16"):
        store = torch.full((M, K + 5), 5.0, dtype=DT[dtype], device="cuda")
        lin = rt.Mx4Linear(codes, scales, K)
        lin.input_grad(dy, store[:, :K])
        check(host(store[:, :K]), ref, bar(ref, absum, N, dtype))
        assert (store[:, K:] == 5.0).all()


# Every form of the three products on tiles, steps and rows that end raggedly, and on sizes that divide; contractions that go round
# the rings of LDS stages more than once, and ones shorter than a ring
FORMS = [(0, (64, 64), 5582, 1036, 33), (0, (64, 64), 700, 100, 3001), (0, (64, 128), 194, 523, 7276), (0, (64, 128), 1024, 2048, 4096),
         (0, (128, 128), 5913, 541, 655), (0, (128, 128), 2050, 130, 4111), (0, (256, 256), 4237, 937, 3687), (0, (256, 256), 4096, 1024, 4096),
         (1, (32, 16), 2834, 30, 17), (1, (64, 64), 33, 1173, 5327), (1, (64, 64), 300, 2049, 1030), (1, (128, 128), 711, 1153, 7671),
         (1, (256, 256), 4231, 730, 3830), (1, (256, 256), 4096, 1024, 4096),
         (2, (32, 128), 5963, 30, 1123), (2, (64, 256), 5011, 286, 517), (2, (64, 256), 1024, 2049, 1000), (2, (128, 256), 5704, 562, 540),
         (2, (256, 256), 5447, 1482, 500), (2, (256, 256), 4096, 4096, 256)]


@pytest.mark.parametrize("product,tile,M,K,N", FORMS)
def test_products_on_each_form(product, tile, M, K, N):
    assert pb.pac_mx4_tiles(product, M, K, N) == tile
    rng = np.random.default_rng(M + K + N)
    codes, scales, w = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K)
    x = rows_of(rng, M, N if product == 2 else K)
    xv = host(x)
    if product == 1:
        xv = bo.values(*bo.quantize(xv), K)
    ref, absum = bo.linear(xv, w.T if product == 2 else w)
    for dtype in ("f32", "bf16"):
        wide = ref.shape[1]
        store = torch.full((M, wide + 3), 5.0, dtype=DT[dtype], device="cuda")  # rows that no whole store fits, too
        for y in (store[:, :wide], torch.empty(M, wide, dtype=DT[dtype], device="cuda")):
            if product == 2:
                lin.input_grad(x, y)
            else:
                lin.forward(x, y, x4=product == 1)
            check(host(y), ref, bar(ref, absum, N if product == 2 else K, dtype))
        assert (store[:, wide:] == 5.0).all()


def test_input_grad_is_the_forward_products_gradient():
    """<dy, x W^T> = <dx, x> for the library's own two products, with W only ever in the stored form."""
    rng = np.random.default_rng(5)
    M, K, N = 37, 300, 190
    codes, scales, w = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K)
    x, dy = rows_of(rng, M, K), rows_of(rng, M, N)
    y, dx = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda")
    lin.forward(x, y)
    lin.input_grad(dy, dx)
    a, b = (host(y) * host(dy)).sum(), (host(dx) * host(x)).sum()
    scale = (np.abs(host(dy)) @ np.abs(w) * np.abs(host(x))).sum()
    assert abs(a - b) <= 2 * (K + N) * 2.0 ** -24 * scale


def test_blocks_without_a_value_stay_where_they_are():
    """A block of W that stands for NaN makes its own outputs NaN and no others; an infinity in x the row's."""
    rng = np.random.default_rng(6)
    M, K, N = 40, 300, 70
    codes, scales, w = layer(rng, N, K)
    scales[9, 2] = 255
    x, dy = rows_of(rng, M, K), rows_of(rng, M, N)
    y, dx = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda")
    lin = rt.Mx4Linear(codes, scales, K)
    for x4 in (False, True):
        lin.forward(x, y, x4=x4)
        nan = torch.isnan(y)
        assert nan[:, 9].all() and int(nan.sum()) == M
    lin.input_grad(dy, dx)
    nan = torch.isnan(dx)
    assert nan[:, 64:96].all() and int(nan.sum()) == M * 32
    scales[9, 2] = 127
    x[3, 7] = float("inf")
    lin.forward(x, y)
    assert not torch.isfinite(y[3]).any() or (host(torch.isfinite(y[3])) <= (w[:, 7] == 0)).all()
    assert torch.isfinite(y[:3]).all() and torch.isfinite(y[4:]).all()
    lin.forward(x, y, x4=True)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[:3]).all() and torch.isfinite(y[4:]).all()


def test_no_rows_is_no_work():
    codes, scales = rt.mx4_empty(5, 40)
    rt.mx4_quantize(torch.ones(5, 40, device="cuda"), codes, scales)
    lin = rt.Mx4Linear(codes, scales, 40)
    x, y = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 5, device="cuda")
    lin.forward(x, y)
    lin.forward(x, y, x4=True)
    lin.input_grad(torch.empty(0, 8, dtype=torch.bfloat16, device="cuda")[:, :5], torch.empty(0, 40, device="cuda"))
    rt.mx4_quantize(torch.empty(0, 40, device="cuda"), *rt.mx4_empty(0, 40))


def test_the_same_call_gives_the_same_bits_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(8)
    M, K, N = 200, 1024, 500
    codes, scales, _ = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K)
    x, dy = rows_of(rng, M, K, 0.0), rows_of(rng, M, N, 0.0)
    outs = lambda: (torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"))  # noqa: E731

    def go(o):
        lin.forward(x, o[0])
        lin.forward(x, o[1], x4=True)
        lin.input_grad(dy, o[2])

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
        x.mul_(-1.0)
        for t in graph:
            t.zero_()
        go(ref)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, graph)), k


def test_layer_from_weights_and_what_python_refuses():
    w = torch.randn(24, 40, device="cuda")
    lin = rt.Mx4Linear.from_weights(w)
    x, y = torch.randn(3, 40, device="cuda").bfloat16(), torch.empty(3, 24, device="cuda")
    lin.forward(x, y)
    back = torch.empty(24, 40, device="cuda")
    rt.mx4_dequantize(lin.codes, lin.scales, back)
    ref, absum = bo.linear(host(x), host(back))
    check(host(y), ref, bar(ref, absum, 40, "f32"))
    for bad in (lambda: lin.forward(x.float(), y), lambda: lin.forward(x[:, :39], y), lambda: lin.forward(x, y[:, :23]),
                lambda: lin.forward(x, y.t().contiguous().t()), lambda: lin.forward(x.cpu(), y), lambda: lin.forward(x, y.half()),
                lambda: lin.input_grad(y, x), lambda: rt.Mx4Linear(lin.codes, lin.scales, 400),
                lambda: rt.Mx4Linear(lin.codes, lin.scales, 40, bias=torch.zeros(23, device="cuda")),
                # the last row's 16-byte piece would end past the allocation's last element
                lambda: rt.Mx4Linear(*rt.mx4_empty(24, 37), 37).forward(torch.empty(64, 40, dtype=torch.bfloat16, device="cuda").view(-1)[-40 * 2 + 3:][:77].as_strided((2, 37), (40, 1)), y[:2])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(pb.PacError) as e:                # rows that do not start on 16 bytes
        rt.Mx4Linear(*rt.mx4_empty(24, 37), 37).forward(torch.zeros(4, 37, dtype=torch.bfloat16, device="cuda")[:3], y)
    assert e.value.status == pb.PAC_ERR_ALIGN


def stored_rows(x, K):
    """The values that x's quantised rows stand for (the quantiser itself is compared with the oracle above)."""
    xc, xs = rt.mx4_empty(x.shape[0], K)
    rt.mx4_quantize(x, xc, xs)
    return bo.values(xc.cpu().numpy(), xs.cpu().numpy(), K)


@pytest.mark.parametrize("product,tile,M,K,N", [f for f in FORMS if f[0] != 2])
def test_bias_and_gelu_on_each_form(product, tile, M, K, N):
    """The epilogue of every tile form: bias at ragged edges and in whole stores, GELU, both types, rows that take whole stores and not."""
    assert pb.pac_mx4_tiles(product, M, K, N) == tile
    rng = np.random.default_rng(M * 3 + K + N)
    codes, scales, w = layer(rng, N, K)
    x = rows_of(rng, M, K)
    bias = rng.standard_normal(N).astype(np.float32)
    lin, plain = rt.Mx4Linear(codes, scales, K, bias=dev(bias)), rt.Mx4Linear(codes, scales, K)
    pre, absum = bo.linear(stored_rows(x, K) if product == 1 else host(x), w)
    bias = bias.astype(np.float64)
    act = lambda u: (0.5 * torch.from_numpy(u) * torch.special.erfc(torch.from_numpy(-u / np.sqrt(2)))).numpy()  # noqa: E731
    with_bias = pre + bias
    both = act(with_bias)
    for layer_, ref, b, gelu, dtype in ((lin, with_bias, bias, False, "f32"), (lin, both, bias, True, "bf16"), (lin, both, bias, True, "f32"),
                                        (lin, with_bias, bias, False, "bf16"), (plain, act(pre), None, True, "bf16")):
        err = bar(ref, absum, K, dtype, b, gelu)
        store = torch.full((M, N + 3), 5.0, dtype=DT[dtype], device="cuda")
        for y in (store[:, :N], torch.empty(M, N, dtype=DT[dtype], device="cuda")):
            layer_.forward(x, y, gelu=gelu, x4=product == 1)
            check(host(y), ref, err)
        assert (store[:, N:] == 5.0).all()


@pytest.mark.parametrize("product,tile,M,K,N", FORMS)
def test_blocks_without_a_value_on_each_form(product, tile, M, K, N):
    """As above on every tile form: a block of W that stands for NaN, an infinity in one row of x or dy."""
    assert pb.pac_mx4_tiles(product, M, K, N) == tile
    rng = np.random.default_rng(M + 2 * K + N)
    codes, scales, _ = layer(rng, N, K)
    row, block, bad = N - 1 - N // 3, (K - 1) // 64, M - 1 - M // 5
    lin = rt.Mx4Linear(codes, scales, K)
    x = rows_of(rng, M, N if product == 2 else K)
    y = torch.empty(M, K if product == 2 else N, device="cuda")
    go = (lambda: lin.input_grad(x, y)) if product == 2 else (lambda: lin.forward(x, y, x4=product == 1))  # noqa: E731
    was, scales[row, block] = int(scales[row, block]), 255
    go()
    nan = torch.isnan(y)
    if product == 2:
        wide = min(32, K - 32 * block)
        assert nan[:, 32 * block:32 * block + wide].all() and int(nan.sum()) == M * wide
    else:
        assert nan[:, row].all() and int(nan.sum()) == M
    scales[row, block] = was
    x[bad, x.shape[1] // 2] = float("inf")
    go()
    fine = torch.isfinite(y)
    assert not fine[bad].all() and int(fine.sum()) == (M - 1) * y.shape[1] + int(fine[bad].sum())
    if product == 1:
        assert torch.isnan(y[bad]).all()


@pytest.mark.parametrize("M,K,N", [(2000, 3001, 1000), (1024, 4096, 4096), (4096, 1024, 4096), (5447, 1482, 500)])
def test_tile_kernels_in_a_graph_and_on_another_stream(M, K, N):
    assert all(pb.pac_mx4_tiles(p, M, K, N)[0] >= 64 for p in (0, 1)) and pb.pac_mx4_tiles(2, M, K, N)[0] >= 64
    rng = np.random.default_rng(9)
    codes, scales, _ = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K, bias=dev(rng.standard_normal(N), torch.float32))
    x, dy = rows_of(rng, M, K, 0.0), rows_of(rng, M, N, 0.0)
    outs = lambda: (torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda"))  # noqa: E731

    def go(o):
        lin.forward(x, o[0], gelu=True)
        lin.forward(x, o[1], gelu=True, x4=True)
        lin.input_grad(dy, o[2])

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
        x.mul_(-0.5), dy.mul_(-0.5)
        for t in graph:
            t.zero_()
        go(ref)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, graph)), k


def test_conversions_of_more_groups_than_one_launch_takes():
    """2^27 and some rows of one group each: values on the grid come back as they are, the last ones too, and the stored form is that of
    the first rows again and again."""
    rows, cols, period = (1 << 27) + 4097, 32, 4096
    rng = np.random.default_rng(10)
    some = np.ldexp(bo.GRID[rng.integers(1, 8, size=(period, cols))] * rng.choice([-1.0, 1.0], size=(period, cols)), rng.integers(-100, 100, size=(period, 1)))
    some[:, 7] = 6.0 * np.exp2(np.floor(np.log2(np.abs(some).max(1))) - 2)
    x = dev(some, torch.bfloat16).repeat(-(-rows // period), 1)[:rows]
    codes, scales = rt.mx4_empty(rows, cols)
    rt.mx4_quantize(x, codes, scales)
    ref_codes, ref_scales = (dev(a) for a in bo.quantize(some))
    whole = rows // period * period
    for got, ref in ((codes, ref_codes), (scales, ref_scales)):
        assert (got[:whole].view(-1, *ref.shape) == ref).all() and torch.equal(got[whole:], ref[:rows - whole])
    out = torch.zeros_like(x)
    rt.mx4_dequantize(codes, scales, out)
    assert torch.equal(out, x)


@pytest.mark.parametrize("M", [1, 300])
def test_gelu_over_its_range(M):
    """u = bias (x is zero), on the row form and on tiles.  Bars: 2e-7 |u| and, for negative u down to -11, 1.4e-3 of the value (the stated
    ones, with 2^-22 |u| for the exponential's and the last rounding); below that less than 1e-26; infinities go to infinity and zero."""
    u = np.concatenate([np.linspace(-12, 12, 24001), -np.geomspace(1e-6, 60, 3000), np.geomspace(1e-30, 1e30, 500), [-1e30, -np.inf, np.inf, 0.0]]).astype(np.float32)
    K, N = 40, u.size
    codes, scales = rt.mx4_empty(N, K)
    rt.mx4_quantize(torch.ones(N, K, device="cuda"), codes, scales)
    lin = rt.Mx4Linear(codes, scales, K, bias=dev(u))
    assert (pb.pac_mx4_tiles(0, M, K, N)[0] == 16) == (pb.pac_mx4_tiles(1, M, K, N)[0] == 16) == (M == 1)
    x, y = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(M, N, device="cuda")
    h = torch.from_numpy(u).double()
    ref = torch.where(torch.isinf(h), h.clamp(min=0), 0.5 * h * torch.special.erfc(-h / np.sqrt(2))).numpy()
    off = lambda got: np.abs(np.where(got == ref, 0.0, got) - np.where(got == ref, 0.0, ref))  # noqa: E731
    size = np.abs(u.astype(np.float64))
    for x4 in (False, True):
        lin.forward(x, y, gelu=True, x4=x4)
        assert (y == y[0]).all()
        got = host(y[0])
        assert np.array_equal(got[np.isinf(u)], ref[np.isinf(u)])
        ok = np.isfinite(u)
        err = off(got)
        assert (err[ok] <= (2e-7 + 2.0 ** -22) * size[ok]).all(), u[ok][np.argmax(err[ok] / (size[ok] + 1e-300))]
        neg = ok & (u < -1) & (u >= -11)
        assert (err[neg] <= (1.4e-3 + 2.0 ** -16) * np.abs(ref[neg])).all(), u[neg][np.argmax(err[neg] / np.abs(ref[neg]))]
        assert (np.abs(got[ok & (u < -11)]) < 1e-26).all()
    low = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    lin.forward(x, low, gelu=True)
    got = host(low[0])
    neg = (u < 0) & (u >= -11)
    assert (off(got)[neg] <= (2.0 ** -8 + 1.4e-3) * np.abs(ref[neg]) + 2e-7 * size[neg]).all()


def test_weights_given_other_storage():
    """What the layer's tensors are at the call counts, wherever their storage is by then; what no longer fits is refused."""
    rng = np.random.default_rng(12)
    M, K, N = 5, 300, 70
    new = lambda: layer(rng, N, K)[:2] + (dev(rng.standard_normal(N), torch.float32),)  # noqa: E731
    codes, scales, bias = new()
    lin = rt.Mx4Linear(codes, scales, K, bias=bias)
    x, dy = rows_of(rng, M, K), rows_of(rng, M, N)

    def go(l):
        y, z, dx = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda")
        l.forward(x, y)
        l.forward(x, z, x4=True)
        l.input_grad(dy, dx)
        return y, z, dx

    keep = []                                             # the old storages stay, so that a stale address would be read, not faulted on
    for how in range(3):
        before = go(lin)
        keep += [t.detach() for t in (lin.codes, lin.scales, lin.bias)]
        other = new()
        if how == 0:
            lin.codes.data, lin.scales.data, lin.bias.data = other
        elif how == 1:
            for t, o in zip((lin.codes, lin.scales, lin.bias), other):
                t.set_(o)
        else:
            lin.codes, lin.scales, lin.bias = other
        after = go(lin)
        assert all(torch.equal(a, b) for a, b in zip(after, go(rt.Mx4Linear(*other[:2], K, bias=other[2])))), how
        assert not any(torch.equal(a, b) for a, b in zip(after, before)), how
    for name, bad in (("codes", lin.codes[:-1].clone()), ("scales", lin.scales.cpu()), ("bias", lin.bias.double())):
        was = getattr(lin, name)
        setattr(lin, name, bad)
        for call in (lambda: lin.forward(x, torch.empty(M, N, device="cuda")), lambda: lin.input_grad(dy, torch.empty(M, K, device="cuda"))):
            with pytest.raises(ValueError):
                call()
        setattr(lin, name, was)
    go(lin)


def test_rows_past_32_bits_are_refused_not_cut_off():
    """(the buffers are never touched)"""
    lin = rt.Mx4Linear.from_weights(torch.ones(1, 1, device="cuda"))
    rows = (1 << 32) + 4
    x, y = torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda")[:, :1], torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: lin.forward(x, y), lambda: lin.forward(x, y, x4=True), lambda: lin.input_grad(x, y)):
        with pytest.raises(ValueError):
            bad()


def test_results_beside_and_over_the_inputs():
    """x and y side by side in one buffer give what they give apart; y over x is refused, and nothing is written."""
    rng = np.random.default_rng(13)
    M, K, N = 70, 300, 64
    codes, scales, _ = layer(rng, N, K)
    lin = rt.Mx4Linear(codes, scales, K)
    apart = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    both = torch.zeros(M, 400, dtype=torch.bfloat16, device="cuda")
    both[:, :K] = dev(rng.standard_normal((M, K)), torch.bfloat16)
    x, y = both[:, :K], both[:, K:K + N]
    for x4 in (False, True):
        lin.forward(x.clone() if x4 else torch.nn.functional.pad(x, (0, 4))[:, :K], apart, x4=x4)
        lin.forward(x, y, x4=x4)
        assert torch.equal(y, apart)
    was = both.clone()
    for call in (lambda: lin.forward(x, both[:, K - 1:K - 1 + N]), lambda: lin.forward(x, x[:, :N], x4=True), lambda: lin.input_grad(both[:, :N], both[:, 50:50 + K]),
                 lambda: rt.mx4_quantize(x, both.view(-1).view(torch.uint8)[:M * 256].view(M, 256), scales[:1].expand(M, -1).contiguous())):
        with pytest.raises(pb.PacError) as e:
            call()
        assert e.value.status == pb.PAC_ERR_RANGE
    assert torch.equal(both, was)


@pytest.mark.parametrize("M,K,N", [(1, 300, 77), (40, 1030, 900), (700, 1000, 3001)])
def test_layers_that_share_a_stored_input(M, K, N):
    """x quantised once for two layers: the bits that each gives quantising it in the call."""
    rng = np.random.default_rng(14)
    x = rows_of(rng, M, K)
    xc, xs = rt.mx4_empty(M, K)
    rt.mx4_quantize(x, xc, xs)
    for n in (N, N + 5):
        codes, scales, _ = layer(rng, n, K)
        lin = rt.Mx4Linear(codes, scales, K, bias=dev(rng.standard_normal(n), torch.float32))
        for dtype, gelu in (("bf16", True), ("f32", False)):
            got, ref = torch.empty(M, n, dtype=DT[dtype], device="cuda"), torch.empty(M, n, dtype=DT[dtype], device="cuda")
            lin.forward_stored(xc, xs, got, gelu=gelu)
            lin.forward(x, ref, gelu=gelu, x4=True)
            assert torch.equal(got, ref)
    for bad in (lambda: lin.forward_stored(xc[:, :-128].contiguous(), xs, got), lambda: lin.forward_stored(xc, xs.cpu(), got), lambda: lin.forward_stored(xc, xs, got[:, 1:]),
                lambda: lin.forward_stored(xc.float(), xs, got), lambda: lin.forward_stored(xc, xs[:0], got)):
        with pytest.raises(ValueError):
            bad()
    lin.forward_stored(xc[:0], xs[:0], got[:0])


@pytest.mark.parametrize("M", [3, 300])
def test_the_bindings_functions_are_the_layers_calls(M):
    """paper_2408_10746_amd.binding on addresses gives the bits that runtime gives on tensors."""
    rng = np.random.default_rng(15)
    K, N, st = 320, 72, torch.cuda.current_stream().cuda_stream
    w, x, dy = dev(rng.standard_normal((N, K)), torch.float32), rows_of(rng, M, K), rows_of(rng, M, N)
    codes, scales = rt.mx4_empty(N, K)
    pb.pac_mx4_quantize(w.data_ptr(), pb.PAC_F32, N, K, K, codes.data_ptr(), scales.data_ptr(), st)
    lin = rt.Mx4Linear.from_weights(w, bias=dev(rng.standard_normal(N), torch.float32))
    assert torch.equal(codes, lin.codes) and torch.equal(scales, lin.scales)
    back, ref = torch.empty_like(w), torch.empty_like(w)
    pb.pac_mx4_dequantize(codes.data_ptr(), scales.data_ptr(), N, K, back.data_ptr(), pb.PAC_F32, K, st)
    rt.mx4_dequantize(codes, scales, ref)
    assert torch.equal(back, ref)
    y, z, d = (torch.empty(M, n, device="cuda") for n in (N, N, K))
    tail = (codes.data_ptr(), scales.data_ptr(), N, lin.bias.data_ptr(), pb.PAC_MX4_ACT_GELU)
    pb.pac_mx4_linear(x.data_ptr(), M, K, x.stride(0), *tail, y.data_ptr(), pb.PAC_F32, N, st)
    lin.forward(x, z, gelu=True)
    assert torch.equal(y, z)
    ws = torch.empty(pb.pac_mx4_linear_qx_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    pb.pac_mx4_linear_qx(x.data_ptr(), pb.PAC_BF16, M, K, x.stride(0), *tail, y.data_ptr(), pb.PAC_F32, N, ws.data_ptr(), ws.numel(), st)
    lin.forward(x, z, gelu=True, x4=True)
    assert torch.equal(y, z)
    pb.pac_mx4_linear_dx(dy.data_ptr(), M, N, dy.stride(0), codes.data_ptr(), scales.data_ptr(), K, d.data_ptr(), pb.PAC_F32, K, st)
    e = torch.empty_like(d)
    lin.input_grad(dy, e)
    assert torch.equal(d, e)
    with pytest.raises(pb.PacError):
        pb.pac_mx4_linear(x.data_ptr(), M, K, K - 8, *tail, y.data_ptr(), pb.PAC_F32, N, st)


@pytest.mark.parametrize("M,K,N", [(2, 200, 40), (40, 520, 900), (700, 320, 600), (4237, 937, 3687), (4096, 1024, 256)])
@pytest.mark.parametrize("ew,ex", [(-126, 110), (-121, 100), (110, -131), (100, -124), (-60, -40), (60, 50)])
def test_products_at_the_ends_of_the_range(M, K, N, ew, ex):
    """Stored values and activations below 2^-126, whose products are ordinary numbers, count in full."""
    rng = np.random.default_rng(17)
    w = rng.standard_normal((N, K)) * np.exp2(rng.integers(-2, 3, size=(N, 1)))
    w = np.ldexp(w, ew).astype(np.float32)
    codes, scales = rt.mx4_empty(N, K)
    rt.mx4_quantize(dev(w), codes, scales)
    wv = bo.values(codes.cpu().numpy(), scales.cpu().numpy(), K)
    lin = rt.Mx4Linear(codes, scales, K)
    few = np.r_[0:min(M, 40), M - 1]                     # the oracle takes some of the rows
    for product in (0, 1, 2):
        x = rows_of(rng, M, N if product == 2 else K)
        x *= torch.from_numpy(np.array(2.0 ** ex)).cuda()
        y = torch.empty(M, K if product == 2 else N, device="cuda")
        if product == 2:
            lin.input_grad(x, y)
        else:
            lin.forward(x, y, x4=product == 1)
        xv = (stored_rows(x, K) if product == 1 else host(x))[few]
        ref, absum = bo.linear(xv, wv.T if product == 2 else wv)
        assert product == 1 or np.abs(ref).max() > 0     # (x below half the format's least step is stored as zero)
        check(host(y)[few], ref, bar(ref, absum, x.shape[1], "f32"))


@pytest.mark.parametrize("M,K,N", [(3, 300, 70), (700, 100, 3001), (4096, 1024, 4096)])
def test_gelu_keeps_what_has_no_value(M, K, N):
    """NaN comes through the activation on every path, beside neighbours that it leaves alone."""
    rng = np.random.default_rng(18)
    codes, scales, _ = layer(rng, N, K)
    scales[N // 2, 0] = 255
    bias = torch.zeros(N, device="cuda")
    bias[1] = float("nan")
    lin = rt.Mx4Linear(codes, scales, K, bias=bias)
    x = rows_of(rng, M, K)
    for dtype in DT.values():
        y = torch.empty(M, N, dtype=dtype, device="cuda")
        for x4 in (False, True):
            lin.forward(x, y, gelu=True, x4=x4)
            nan = torch.isnan(y)
            assert nan[:, [1, N // 2]].all() and int(nan.sum()) == 2 * M
