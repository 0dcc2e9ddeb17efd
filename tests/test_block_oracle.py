"""Pins of oracle/block_oracle.py: closed forms and brute force for the 4-bit format, finite differences for the gradients of the
norms around a block."""
import numpy as np
import pytest

from oracle import block_oracle as bo


def test_values_on_the_grid_come_back_as_they_are():
    rng = np.random.default_rng(1)
    e = rng.integers(-100, 100, size=(5, 8))
    x = bo.GRID[rng.integers(0, 8, size=(5, 8, 32))] * rng.choice([-1.0, 1.0], size=(5, 8, 32))
    x[:, :, 3] = 6.0                                     # so that the block's scale is the grid's own
    x = np.ldexp(x, e[:, :, None]).reshape(5, 256)
    codes, scales = bo.quantize(x)
    assert np.array_equal(scales, e + 127) and np.array_equal(bo.values(codes, scales, 256), x)


def test_every_value_goes_to_the_nearest_and_ties_to_the_even_code():
    # 4 fixes the scale at 1
    ties = {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0, 7.0: 6.0, 7.99: 6.0}
    x = np.zeros((1, 32))
    x[0, 0] = 4.0
    for k, (v, want) in enumerate(ties.items()):
        x[0, 1 + k], x[0, 12 + k] = v, -v
    codes, scales = bo.quantize(x)
    got = bo.values(codes, scales, 32)[0]
    assert scales[0, 0] == 127
    for k, want in enumerate(ties.values()):
        assert got[1 + k] == want and got[12 + k] == -want
    rng = np.random.default_rng(2)
    x = rng.standard_normal((40, 32))
    got = bo.values(*bo.quantize(x), 32)
    s = np.exp2(np.floor(np.log2(np.abs(x).max(1))) - 2)[:, None]
    assert (np.abs(got - x) <= np.where(np.abs(x) < 2 * s, 0.25, np.where(np.abs(x) < 4 * s, 0.5, 2.0)) * s).all()


def test_zero_special_and_padded_blocks():
    x = np.zeros((2, 100))
    x[0, 40], x[0, 70], x[1, 5], x[1, 99] = np.inf, 2.0 ** -149, np.nan, -1.0
    codes, scales = bo.quantize(x)
    assert codes.shape == (2, 128) and scales.shape == (2, 8)
    assert scales.tolist() == [[0, 255, 0, 0, 0, 0, 0, 0], [255, 0, 0, 125, 0, 0, 0, 0]]
    v = bo.values(codes, scales, 100)
    assert np.isnan(v[0, 32:64]).all() and not v[0, :32].any() and np.isnan(v[1, :32]).all() and v[1, 99] == -1.0


CASES = [dict(layer=False, gate=1, res=True, post=True, pre=True, bias=False), dict(layer=True, gate=2, res=True, post=True, pre=True, bias=True),
         dict(layer=True, gate=1, res=False, post=False, pre=True, bias=True), dict(layer=False, gate=2, res=True, post=True, pre=False, bias=True),
         dict(layer=False, gate=0, res=True, post=None, pre=True, bias=False), dict(layer=True, gate=0, res=False, post=False, pre=False, bias=False)]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_gradients_of_the_norms_against_differences(c):
    rng = np.random.default_rng(3)
    rows, d = 3, 7
    v = dict(x=rng.standard_normal((rows, d)), o=None if c["post"] is None else rng.standard_normal((rows, d)))
    if c["post"]:
        v["w_post"] = rng.standard_normal(d)
        if c["bias"]:
            v["b_post"] = rng.standard_normal(d)
    if c["gate"]:
        v["gate"] = rng.standard_normal(1 if c["gate"] == 1 else d)
    if c["res"]:
        v["res"] = rng.standard_normal(1)
    if c["pre"]:
        v["w_pre"] = rng.standard_normal(d)
        if c["bias"]:
            v["b_pre"] = rng.standard_normal(d)
    dy, dn = rng.standard_normal((rows, d)), rng.standard_normal((rows, d)) if c["pre"] else None
    f = lambda u: sum((g * t).sum() for g, t in zip((dy, dn), bo.block_norm(layer=c["layer"], eps=1e-3, **u)) if g is not None)  # noqa: E731
    got = bo.block_norm_grad(v["x"], v["o"], dy, dn, layer=c["layer"], eps=1e-3, **{k: t for k, t in v.items() if k not in "xo"})
    assert sorted(got) == sorted(k for k, t in v.items() if t is not None)
    for name, t in v.items():
        if t is None:
            continue
        diff = np.empty(t.size)
        for j in range(t.size):
            h, at = 1e-5, t.flat[j]
            t.flat[j] = at + h
            up = f(v)
            t.flat[j] = at - h
            diff[j] = (up - f(v)) / (2 * h)
            t.flat[j] = at
        np.testing.assert_allclose(got[name].ravel(), diff, rtol=1e-6, atol=1e-7)  # differences: h^2 and 2^-52 / h, both about 1e-10
