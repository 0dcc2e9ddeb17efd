"""Plain 64-bit forms of attention over packed sequences, its gradients, and attention over a 4-bit cache, with bounds of the errors that
the kernels' roundings may make.  TEST INFRASTRUCTURE ONLY (imported by tests/ alone).

Tensors are float64 torch tensors, [heads][n][d] for queries and [kv_heads][n][d] for keys and values of ONE sequence."""
from __future__ import annotations

import torch

BF16 = 2.0 ** -8   # half a step of bf16, relative to the value
F32 = 2.0 ** -24


def mask(n: int, causal: bool, device):
    m = torch.ones(n, n, dtype=torch.bool, device=device)
    return m.tril() if causal else m


def masked_product(p, v, m):
    """sum over j of p_ij v_jd for the j that m lets in, others having no part whatever they hold."""
    bad = ~torch.isfinite(v)
    out = p @ torch.where(bad, 0.0, v)
    for h, j, d in bad.nonzero().tolist():  # few, and only in tests of them
        out[h, :, d] = torch.where(m[:, j], out[h, :, d] + p[h, :, j] * v[h, j, d], out[h, :, d])
    return out


def forward(q, k, v, scale: float, causal: bool):
    """o, lse, p, and `eps`, the relative error of p in 32 bits: scores are sums of d products, exact as such; sums over keys follow."""
    g, n, d = q.shape[0] // k.shape[0], q.shape[1], q.shape[2]
    kg, vg = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    m = mask(n, causal, q.device)
    s = (q @ kg.transpose(1, 2) * scale).masked_fill(~m, -torch.inf)
    lse = torch.logsumexp(s, 2)
    p = torch.exp(s - lse[..., None]).masked_fill(~m, 0.0)
    size = (q.abs() @ kg.abs().transpose(1, 2) * scale).masked_fill(~m, 0.0)
    eps = 2 * F32 * ((d + 8) * float(size.nan_to_num(0, 0, 0).amax()) + n + 64)
    return masked_product(p, vg, m), lse, p, eps


def forward_bound(p, v, o, eps: float):
    """|error| of o: p in bf16 and its own error, against the absolute terms; one rounding of o; what underflows."""
    g = p.shape[0] // v.shape[0]
    return 1.01 * ((BF16 + eps) * (p @ v.abs().repeat_interleave(g, 0)) * (1 + BF16) + BF16 * o.abs()) + 1e-30


def backward(q, k, v, do, scale: float, causal: bool):
    """dq, dk, dv by the formulas, and bounds of their errors: o rounded before delta is made, p and ds in bf16."""
    g = q.shape[0] // k.shape[0]
    o, _, p, eps = forward(q, k, v, scale, causal)
    m = mask(q.shape[1], causal, q.device)
    kg, vg = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    dp = do @ vg.transpose(1, 2)
    delta = (do * o).sum(2, keepdim=True)
    ds = p * (dp - delta)
    fold = lambda t: t.reshape(-1, g, *t.shape[1:]).sum(1)  # noqa: E731
    dq, dk, dv = scale * (ds @ kg), scale * fold(ds.transpose(1, 2) @ q), fold(p.transpose(1, 2) @ do)
    # errors
    d = q.shape[2]
    e_delta = (do.abs() * forward_bound(p, v, o, eps)).sum(2, keepdim=True) + 2 * (d + 8) * F32 * (do.abs() * o.abs()).sum(2, keepdim=True)
    e_dp = 2 * (d + 8) * F32 * (do.abs() @ vg.abs().transpose(1, 2))
    e_ds = ((BF16 + 3 * eps) * ds.abs() + p * (1 + eps) * (e_dp + e_delta)) * (1 + BF16)
    e_ds = e_ds.masked_fill(~m, 0.0)
    e_p = (BF16 + 3 * eps) * p
    sums = 1 + 2 * F32 * (q.shape[1] * g + 64)
    b = (scale * (e_ds @ kg.abs()), scale * fold(e_ds.transpose(1, 2) @ q.abs()), fold(e_p.transpose(1, 2) @ do.abs()))
    t = (scale * (ds.abs() @ kg.abs()), scale * fold(ds.abs().transpose(1, 2) @ q.abs()), fold(p.transpose(1, 2) @ do.abs()))
    bounds = tuple(1.01 * (x * (1 + BF16) + (sums - 1) * y + BF16 * z.abs()) + 1e-30 for x, y, z in zip(b, t, (dq, dk, dv)))
    return (dq, dk, dv), bounds


def exact_delta_bounds(q, k, v, do, given, scale: float, causal: bool):
    """Bounds of the errors of dq and dk where delta is exact, although o is at hand as `given`, in bf16 (in 64 bits here).  With D_i = do_i . (given_i - o_i),
    the kernels' z_ij = p_ij (do_i . v_j - delta_i - D_i) and r_i = sum_j z_ij = -D_i,

        dq_i = scale (sum_j z_ij k_j - r_i sum_j p_ij k_j)     and delta_i = do_i . given_i + r_i for dk

    are free of D but for the roundings that it passes through: z and p to bf16, p's relative error e in 32 bits (so that the p of a row sum to 1 within e),
    that of do . v, and sums in 32 bits."""
    g, n, d = q.shape[0] // k.shape[0], q.shape[1], q.shape[2]
    o, _, p, eps = forward(q, k, v, scale, causal)
    kg, vg = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    m, e = mask(n, causal, q.device), 3 * eps
    dp = do @ vg.transpose(1, 2)
    ds = p * (dp - (do * o).sum(2, keepdim=True))
    far = (do * (given - o)).sum(2, keepdim=True).abs()
    e_dp = (2 * (d + 8) * F32 * (do.abs() @ vg.abs().transpose(1, 2))).masked_fill(~m, 0.0)
    e_far = 2 * (d + 8) * F32 * (do.abs() * given.abs()).sum(2, keepdim=True)  # of do . given
    z = ds.abs() + p * far + p * (e_dp + e_far)
    # r + D: p's sum, the errors of do . v, the sum itself; do . given's own error leaves as D does
    e_r = e * (far + e_far + ds.abs().sum(2, keepdim=True)) + (p * e_dp).sum(2, keepdim=True) + 2 * F32 * (n + 64) * z.sum(2, keepdim=True)
    y = p @ kg.abs()
    e_z = ((BF16 + e) * z + p * e_dp) * (1 + BF16)
    sums = 2 * F32 * (n * g + 64)
    ref_q, ref_k = scale * (ds @ kg), scale * (ds.transpose(1, 2) @ q).reshape(-1, g, n, d).sum(1)
    b_q = scale * ((e_z + sums * z) @ kg.abs() + (e_r + (far + e_far) * (BF16 + e + sums)) * y * (1 + BF16)) + BF16 * ref_q.abs()
    e_ds = ((BF16 + e) * ds.abs() + p * (1 + e) * (e_dp + e_r + 4 * F32 * (do.abs() * given.abs()).sum(2, keepdim=True))) * (1 + BF16)
    b_k = scale * ((e_ds + sums * ds.abs()).transpose(1, 2) @ q.abs()).reshape(-1, g, n, d).sum(1) + BF16 * ref_k.abs()
    return (ref_q, 1.01 * b_q + 1e-30), (ref_k, 1.01 * b_k + 1e-30)


def decode(q, k, v, scale: float):
    """o of one query a head, q [heads][d], over k, v [kv_heads][n][d], and the bound of its error."""
    g = q.shape[0] // k.shape[0]
    if k.shape[1] == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    kg, vg = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    s = (kg @ q[..., None])[..., 0] * scale
    p = torch.softmax(s, 1)
    size = float(((kg.abs() @ q.abs()[..., None])[..., 0] * scale).amax())
    eps = 2 * F32 * ((q.shape[1] + 8) * size + k.shape[1] + 64)
    o = (p[:, None] @ vg)[:, 0]
    return o, 1.01 * ((BF16 + eps) * (p[:, None] @ vg.abs())[:, 0] * (1 + BF16) + BF16 * o.abs()) + 1e-30
