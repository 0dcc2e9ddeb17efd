"""Plain numpy forms in 64 bits of the backbone's blocks: microscaled 4-bit floating point, products with it, and the norms around
a block with their gradients.  TEST INFRASTRUCTURE ONLY (imported by tests/ alone)."""
from __future__ import annotations

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def pitches(cols: int):
    groups = (cols + 255) // 256
    return 128 * groups, 8 * groups


def quantize(x):
    """x [rows][cols] (any float type) -> (codes uint8 [rows][code pitch], scales uint8 [rows][scale pitch])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    cp, sp = pitches(cols)
    codes, scales = np.zeros((rows, cp * 2), np.uint8), np.zeros((rows, sp), np.uint8)
    for r in range(rows):
        for b in range((cols + 31) // 32):
            v = x[r, 32 * b:32 * b + 32]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            if top == 0:
                continue
            e = min(max(math.frexp(top)[1] - 1 - 2, -127), 125)
            scales[r, b] = e + 127
            a = np.abs(np.ldexp(v, -e))
            far = np.abs(a[:, None] - GRID[None, :])
            near = far == far.min(1, keepdims=True)
            # of two as near the one with the even code
            pick = np.where(near[:, ::2].any(1), 2 * near[:, ::2].argmax(1), 2 * near[:, 1::2].argmax(1) + 1)
            codes[r, 32 * b:32 * b + v.size] = pick + 8 * (np.signbit(v))
    return codes[:, ::2] | (codes[:, 1::2] << 4), scales


def values(codes, scales, cols: int):
    """The matrix [rows][cols] that a stored form stands for."""
    c = np.empty((codes.shape[0], codes.shape[1] * 2), np.uint8)
    c[:, ::2], c[:, 1::2] = codes & 15, codes >> 4
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(codes.shape[0], -1, 32) * s[:, :, None]).reshape(codes.shape[0], -1)[:, :cols]


def gelu(u):
    return 0.5 * u * np.array([math.erfc(-t) for t in (u / math.sqrt(2)).ravel()]).reshape(u.shape)


def linear(x, w, bias=None, act=0):
    """(y, the sum of the absolute products): what rounding errors of a summation are measured against."""
    y = x @ w.T
    if bias is not None:
        y = y + bias
    return (gelu(y) if act else y), np.abs(x) @ np.abs(w).T


def _norm(z, layer, eps):
    m = z.mean(1, keepdims=True) if layer else 0.0
    r = 1.0 / np.sqrt(((z - m) ** 2).mean(1, keepdims=True) + eps)
    return (z - m) * r, r


def _norm_back(g, h, r, layer):
    g = g - h * (g * h).mean(1, keepdims=True) - (g.mean(1, keepdims=True) if layer else 0.0)
    return r * g


def block_norm(x, o, layer=False, eps=1e-5, w_post=None, b_post=None, gate=None, res=None, w_pre=None, b_pre=None):
    """(y, n) of the fused norms; o None: no block; n None without w_pre."""
    a = 1.0 if res is None else res[0]
    y = a * x
    if o is not None:
        p = o
        if w_post is not None:
            p = _norm(o, layer, eps)[0] * w_post + (0.0 if b_post is None else b_post)
        y = y + (1.0 if gate is None else gate) * p
    n = None
    if w_pre is not None:
        n = _norm(y, layer, eps)[0] * w_pre + (0.0 if b_pre is None else b_pre)
    return y, n


def block_norm_grad(x, o, dy, dn, layer=False, eps=1e-5, w_post=None, b_post=None, gate=None, res=None, w_pre=None, b_pre=None):
    """{name: gradient} of sum(dy y) + sum(dn n)."""
    a, g1 = (1.0 if res is None else res[0]), (1.0 if gate is None else gate)
    out = {}
    p, h = o, None
    if w_post is not None:
        h, r = _norm(o, layer, eps)
        p = h * w_post + (0.0 if b_post is None else b_post)
    y = a * x + (0.0 if o is None else g1 * p)
    g = np.zeros_like(x) if dy is None else dy
    if w_pre is not None:
        yh, ry = _norm(y, layer, eps)
        g = g + _norm_back(dn * w_pre, yh, ry, layer)
        out["w_pre"] = (dn * yh).sum(0)
        if b_pre is not None:
            out["b_pre"] = dn.sum(0)
    out["x"] = a * g
    if res is not None:
        out["res"] = np.array([(g * x).sum()])
    if o is not None:
        if gate is not None:
            out["gate"] = (g * p).sum(0) if len(gate) == x.shape[1] and len(gate) > 1 else np.array([(g * p).sum()])
        gp = g * g1
        out["o"] = gp
        if w_post is not None:
            out["w_post"] = (gp * h).sum(0)
            if b_post is not None:
                out["b_post"] = gp.sum(0)
            out["o"] = _norm_back(gp * w_post, h, r, layer)
    return out
