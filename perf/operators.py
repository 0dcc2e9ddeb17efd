"""The operators of a frozen backbone's blocks with 4-bit weights, as timed cases.

The blocks whose outputs the activation cache keeps are, one after the other: the norm before a block, the block's products
with weights in microscaled 4-bit floating point (mx4), and the norm after it with the block's gate and the residual scale.
Four kinds of case:

  quant      a matrix to mx4 and back (how weights get into the stored form, and how one looks at them again)
  linear     y = act(x W^T + b) on stored weights, x in bf16 or, with x4, quantised to mx4 in the call
  dx         the gradient of that product into its input, dx = dy W (the weights are frozen and have none)
  norm       p = w_post N(o) + b_post, y = a x + g p, n = w_pre N(y) + b_pre; with grad the gradients of all of these

The stored form, a public format: blocks of 32 along a row; a value is e2m1 (sign, 0 0.5 1 1.5 2 3 4 6), two a byte, the even
column in the low half; a block's scale is the byte s that stands for 2^(s - 127); rows are padded with zeros to a multiple
of 256 columns.  `run` is the operator in elementary torch operations, or the framework's kernels where `own` is true.
"""
import math

import torch

own = False

DEV = "cuda:0"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a projection's weights into the stored form, as when a backbone is loaded
        dict(name="quant_weights", kind="quant", rows=4096, cols=4096, dtype="f32"),
        # a small matrix whose rows end inside a block
        dict(name="quant_ragged", kind="quant", rows=515, cols=1003, dtype="bf16"),
        # serving: one token through one 4096 x 4096 projection; latency and the reading of the weights
        dict(name="linear_token", kind="linear", x4=False, M=1, K=4096, N=4096, bias=False, gelu=False, out="bf16"),
        # a short ragged batch of sentences through the first half of a feed-forward block of a 1024-wide model
        dict(name="linear_ragged", kind="linear", x4=False, M=333, K=1024, N=4096, bias=True, gelu=True, out="bf16"),
        # sixteen samples of 256 tokens through a 4096-wide projection, activations as they are
        dict(name="linear_prompt", kind="linear", x4=False, M=4096, K=4096, N=4096, bias=False, gelu=False, out="bf16"),
        # the largest: the same tokens through the wide half of a feed-forward block, activations in mx4 too
        dict(name="linear_prompt_x4", kind="linear", x4=True, M=4096, K=4096, N=16384, bias=True, gelu=True, out="bf16"),
        # the way back through the 4096-wide projection, where norms and gates below it are tuned
        dict(name="dx_prompt", kind="dx", M=4096, K=4096, N=4096, out="bf16"),
        # the way back through a small layer with odd sizes, gradient kept in 32 bits
        dict(name="dx_ragged", kind="dx", M=517, K=775, N=1001, out="f32"),
        # serving: the norms around one block for one token
        dict(name="norm_token", kind="norm", grad=False, layer=False, rows=1, d=4096, dtype="bf16", gate=1, post=True, pre=True),
        # a long prompt's norms, root-mean-square form, a scalar gate
        dict(name="norm_prompt", kind="norm", grad=False, layer=False, rows=16384, d=4096, dtype="bf16", gate=1, post=True, pre=True),
        # their gradients on the tokens of one batch of that width
        dict(name="norm_grad", kind="norm", grad=True, layer=False, rows=4096, d=4096, dtype="bf16", gate=1, post=True, pre=True),
        # layer norms with biases, a gate for each channel, 32 sentences of 768-wide states in 32 bits, ragged
        dict(name="norm_grad_layer", kind="norm", grad=True, layer=True, rows=2723, d=768, dtype="f32", gate=2, post=True, pre=True),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: two times in three a multiple of 64, as models have them, else any."""
    w = _log_int(rng, lo, hi)
    return max(64, (w + 32) // 64 * 64) if rng.random() < 2 / 3 else w


def draw(rng):
    kind = rng.choice(("quant", "linear", "linear", "linear", "dx", "norm", "norm"))
    if kind == "quant":
        return dict(kind=kind, rows=_log_int(rng, 1, 8192), cols=_width(rng, 20, 8192), dtype=rng.choice(("bf16", "f32")))
    if kind in ("linear", "dx"):
        most = 4096 ** 3 * (4 if kind == "linear" else 1)
        while True:
            M, K, N = _log_int(rng, 1, 8192), _width(rng, 32, 8192), _width(rng, 32, 16384)
            if M * K * N <= most:
                break
        out = rng.choice(("bf16", "bf16", "f32"))
        if kind == "dx":
            return dict(kind=kind, M=M, K=K, N=N, out=out)
        return dict(kind=kind, x4=rng.random() < 0.5, M=M, K=K, N=N, bias=rng.random() < 0.5, gelu=rng.random() < 0.5, out=out)
    while True:
        rows, d = _log_int(rng, 1, 16384), _width(rng, 48, 8192)
        grad = rng.random() < 0.5
        if rows * d <= 16384 * 4096 // (3 if grad else 1):
            break
    post, pre = rng.choice(((True, True), (True, True), (True, False), (False, True)))
    return dict(kind="norm", grad=grad, layer=rng.random() < 0.5, rows=rows, d=d, dtype=rng.choice(("bf16", "f32")),
                gate=rng.choice((0, 1, 2)), post=post, pre=pre)


# ---- the stored form in elementary operations ------------------------------------------------------------------------------
def _pad256(n):
    return (n + 255) // 256 * 256


def _to_values(x):
    """x rounded to mx4 along its last axis (a multiple of 32): the e2m1 values and the blocks' scales 2^e.  64 bits, because a
    value's place next to a border decides its code."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(-127, 125)
    e = torch.where(top > 0, e, torch.full_like(e, -127))
    v = torch.ldexp(b, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.sign(v) * torch.clamp(torch.round(a / step) * step, max=6.0), e


def _padded(x):
    cols = x.shape[-1]
    out = torch.zeros(*x.shape[:-1], _pad256(cols), dtype=x.dtype, device=x.device)
    out[..., :cols] = x
    return out


def _store(w):
    """(codes, scales) of w in the stored form."""
    q, e = _to_values(_padded(w))
    grid = torch.tensor(GRID, dtype=torch.float64, device=w.device)
    c = torch.searchsorted(grid, q.abs()) + 8 * (q < 0)
    c = c.reshape(w.shape[0], -1, 2).to(torch.uint8)
    return (c[..., 0] | (c[..., 1] << 4)).contiguous(), (e.reshape(w.shape[0], -1) + 127).to(torch.uint8).contiguous()


def _load(codes, scales, cols, dtype=torch.float32):
    """The values that a stored matrix stands for."""
    table = torch.tensor(GRID + tuple(-g for g in GRID), dtype=dtype, device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1, 32).long()
    s = torch.ldexp(torch.ones((), dtype=dtype, device=codes.device), scales.to(torch.int32) - 127)
    return (table[c] * s[..., None]).reshape(codes.shape[0], -1)[:, :cols]


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _rng(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _activations(g, rows, cols):
    """Hidden states: unit normal, one channel in 64 eight times as large, as backbones have them."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    return x * (1 + 7 * (torch.rand(cols, generator=g, device=DEV) < 1 / 64))


def _rows(x, dtype):
    """x as a program holds it whose rows have to start on 16 bytes: a view of rows padded to a multiple of 8."""
    store = torch.zeros(x.shape[0], (x.shape[1] + 7) // 8 * 8, dtype=dtype, device=DEV)
    store[:, :x.shape[1]] = x.to(dtype)
    return store[:, :x.shape[1]]


def _empty(rows, cols, dtype):
    return torch.empty(rows, (cols + 7) // 8 * 8, dtype=dtype, device=DEV)[:, :cols]


def _weights(g, N, K):
    return torch.randn(N, K, generator=g, device=DEV) / math.sqrt(K) * torch.exp(torch.randn(N, 1, generator=g, device=DEV) / 2)


def _inputs(case, seed):
    """The inputs of a case, by name."""
    g = _rng(seed)
    kind = case["kind"]
    if kind == "quant":
        return dict(x=_weights(g, case["rows"], case["cols"]).to(DTYPES[case["dtype"]]))
    if kind in ("linear", "dx"):
        M, K, N = case["M"], case["K"], case["N"]
        codes, scales = _store(_weights(g, N, K))
        x = _rows(_activations(g, M, K if kind == "linear" else N), torch.bfloat16)
        bias = torch.randn(N, generator=g, device=DEV) / 4 if case.get("bias") else None
        return dict(x=x, codes=codes, scales=scales, bias=bias)
    rows, d, dt = case["rows"], case["d"], DTYPES[case["dtype"]]
    near = lambda n, at: at + 0.1 * torch.randn(n, generator=g, device=DEV)  # noqa: E731
    t = dict(x=(2 * _activations(g, rows, d)).to(dt), o=_activations(g, rows, d).to(dt), res=near(1, 0.9),
             gate={0: None, 1: near(1, 0.5), 2: near(d, 0.5)}[case["gate"]],
             w_post=near(d, 1.0) if case["post"] else None, b_post=near(d, 0.0) if case["post"] and case["layer"] else None,
             w_pre=near(d, 1.0) if case["pre"] else None, b_pre=near(d, 0.0) if case["pre"] and case["layer"] else None)
    if case["grad"]:
        # gradients lean the same way as the states here and there, so that sums over tokens do not all but cancel
        t["dy"] = (torch.randn(rows, d, generator=g, device=DEV) + 0.1 * t["x"].float()).to(dt)
        t["dn"] = (torch.randn(rows, d, generator=g, device=DEV) + 0.2 * t["o"].float()).to(dt) if case["pre"] else None
    return t


EPS = 1e-5


def prepare(case, seed):
    s = dict(case, **_inputs(case, seed))
    kind = case["kind"]
    # where results go: a program that runs layer after layer keeps these buffers, as it keeps handles of its layers
    if kind == "quant":
        s["codes"] = torch.empty(case["rows"], _pad256(case["cols"]) // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(case["rows"], _pad256(case["cols"]) // 32, dtype=torch.uint8, device=DEV)
        s["back"] = torch.empty_like(s["x"])
    elif kind in ("linear", "dx"):
        s["y"] = _empty(case["M"], case["N"] if kind == "linear" else case["K"], DTYPES[case["out"]])
    elif not case["grad"]:
        s["y"] = torch.empty_like(s["x"])
        s["n"] = torch.empty_like(s["x"]) if case["pre"] else None
    else:
        s["dx"], s["do"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["dparams"] = {k: torch.empty_like(s[k]) for k in PARAMS if s[k] is not None}
    if own:
        from paper_2408_10746_amd import runtime
        if kind in ("linear", "dx"):
            s["layer_handle"] = runtime.Mx4Linear(s["codes"], s["scales"], case["K"], bias=s.get("bias"))
        elif kind == "norm":
            s["layer_handle"] = runtime.BlockNorm(case["d"], layer=case["layer"], eps=EPS, **{k: s[k] for k in PARAMS})
    return s


PARAMS = ("w_post", "b_post", "gate", "res", "w_pre", "b_pre")


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2408_10746_amd import runtime
    kind = s["kind"]
    if kind == "quant":
        runtime.mx4_quantize(s["x"], s["codes"], s["scales"])
        runtime.mx4_dequantize(s["codes"], s["scales"], s["back"])
        return s["back"]
    layer = s["layer_handle"]
    if kind == "linear":
        layer.forward(s["x"], s["y"], gelu=s["gelu"], x4=s["x4"])
        return s["y"]
    if kind == "dx":
        layer.input_grad(s["x"], s["y"])
        return s["y"]
    if not s["grad"]:
        layer.forward(s["x"], s["o"], s["y"], s["n"])
        return (s["y"], s["n"]) if s["pre"] else (s["y"],)
    layer.backward(s["x"], s["o"], s["dy"], s["dn"], s["dx"], s["do"], s["dparams"])
    return s["dx"], s["do"], s["dparams"]


def _plain(s):
    kind = s["kind"]
    if kind == "quant":
        q, e = _to_values(_padded(s["x"]))
        return torch.ldexp(q, e).reshape(s["rows"], -1)[:, :s["cols"]].to(s["x"].dtype)
    if kind == "linear":
        x = s["x"].float()
        if s["x4"]:
            q, e = _to_values(_padded(x))
            x = torch.ldexp(q.float(), e).reshape(s["M"], -1)[:, :s["K"]]
        y = x @ _load(s["codes"], s["scales"], s["K"]).t()
        if s["bias"] is not None:
            y = y + s["bias"]
        if s["gelu"]:
            y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
        return y.to(s["y"].dtype)
    if kind == "dx":
        return (s["x"].float() @ _load(s["codes"], s["scales"], s["K"])).to(s["y"].dtype)
    x, o, dt = s["x"].float(), s["o"].float(), s["x"].dtype
    a, gate = s["res"], s["gate"] if s["gate"] is not None else 1.0
    oh, orstd = _normed(o, s["layer"]) if s["post"] else (o, None)
    p = oh * s["w_post"] if s["post"] else o
    if s["b_post"] is not None:
        p = p + s["b_post"]
    y = a * x + gate * p
    yh, yrstd = _normed(y, s["layer"]) if s["pre"] else (None, None)
    if not s["grad"]:
        if not s["pre"]:
            return (y.to(dt),)
        n = yh * s["w_pre"]
        if s["b_pre"] is not None:
            n = n + s["b_pre"]
        return y.to(dt), n.to(dt)
    gy, dn, d = s["dy"].float(), None, {}
    if s["pre"]:
        dn = s["dn"].float()
        gy = gy + _norm_back(dn * s["w_pre"], yh, yrstd, s["layer"])
        d["w_pre"] = _total(dn * yh, 0)
        if s["b_pre"] is not None:
            d["b_pre"] = _total(dn, 0)
    d["res"] = _total(gy * x, None)
    if s["gate"] is not None:
        d["gate"] = _total(gy * p, 0 if s["gate"].numel() > 1 or s["d"] == 1 else None)
    gp = gy * gate
    if s["post"]:
        d["w_post"] = _total(gp * oh, 0)
        if s["b_post"] is not None:
            d["b_post"] = _total(gp, 0)
        do = _norm_back(gp * s["w_post"], oh, orstd, s["layer"])
    else:
        do = gp
    return (a * gy).to(dt), do.to(dt), d


def _total(t, axis):
    """A sum over many tokens of terms that largely cancel: in 64 bits, rounded once."""
    return (t.sum(dtype=torch.float64).reshape(1) if axis is None else t.sum(axis, dtype=torch.float64)).float()


def _normed(v, layer):
    if layer:
        v = v - v.mean(-1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * rstd, rstd


def _norm_back(g, h, rstd, layer):
    back = g - h * (g * h).mean(-1, keepdim=True)
    return rstd * (back - g.mean(-1, keepdim=True) if layer else back)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "quant":
        n, size = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        # into the stored form and back: values read and written once, the stored form written and read once
        return {"bytes": 2.0 * n * size + 2.0 * n * 17 / 32, "flops": 4.0 * n}
    if kind in ("linear", "dx"):
        M, K, N, size = case["M"], case["K"], case["N"], 2 if case["out"] == "bf16" else 4
        into, out = (K, N) if kind == "linear" else (N, K)
        return {"bytes": 2.0 * M * into + N * K * 17 / 32 + size * M * out, "flops": 2.0 * M * K * N}
    n, size = case["rows"] * case["d"], 2 if case["dtype"] == "bf16" else 4
    arrays = (5 + case["pre"]) if case["grad"] else (3 + case["pre"])
    return {"bytes": float(arrays * n * size), "flops": (30.0 if case["grad"] else 12.0) * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _nearest(x):
    """x in mx4 by its definition: every value to the nearest of the grid, of two as near the one with the even code."""
    cols = x.shape[1]
    b = torch.zeros(x.shape[0], (cols + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    b[:, :cols] = x.double()
    b = b.reshape(x.shape[0], -1, 32)
    top = b.abs().amax(2)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2)
    scale = torch.where(scale * 8 <= top, scale * 2, torch.where(scale * 4 > top, scale / 2, scale))  # the logarithm's own rounding
    scale = torch.where(top > 0, scale, 1.0)[..., None]
    a = b.abs() / scale
    best, far = torch.zeros_like(a), a.clone()
    for code in range(1, 8):
        off = (a - GRID[code]).abs()
        better = (off < far) | ((off == far) & (code % 2 == 0))
        best, far = torch.where(better, GRID[code], best), torch.where(better, off, far)
    return (torch.sign(b) * best * scale).reshape(x.shape[0], -1)[:, :cols]


def exact(case, seed):
    t = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quant":
        return _nearest(t["x"])
    if kind in ("linear", "dx"):
        K = case["K"]
        grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
        w = torch.zeros(case["N"], t["codes"].shape[1] * 2, dtype=torch.float64, device=DEV)
        for half in (0, 1):
            c = (t["codes"].to(torch.int64) >> (4 * half)) & 15
            w[:, half::2] = grid[c & 7] * (1 - 2 * (c >> 3))
        w = (w * torch.exp2(t["scales"].double() - 127).repeat_interleave(32, 1))[:, :K]
        if kind == "dx":
            return t["x"].double() @ w.contiguous()
        x = _nearest(t["x"].float()) if case["x4"] else t["x"].double()
        y = torch.nn.functional.linear(x, w, None if t["bias"] is None else t["bias"].double())
        return torch.nn.functional.gelu(y) if case["gelu"] else y
    # the forward pass as it is defined; its gradients by differentiating that
    v = {k: (None if t[k] is None else t[k].double().requires_grad_(case["grad"])) for k in ("x", "o") + PARAMS}

    def norm(z, w, b):
        if case["layer"]:
            var, mean = torch.var_mean(z, dim=1, correction=0, keepdim=True)
        else:
            var, mean = z.square().mean(1, keepdim=True), 0.0
        z = (z - mean) / torch.sqrt(var + EPS) * w
        return z if b is None else z + b

    p = norm(v["o"], v["w_post"], v["b_post"]) if case["post"] else v["o"]
    y = v["res"] * v["x"] + (p if v["gate"] is None else v["gate"] * p)
    n = norm(y, v["w_pre"], v["b_pre"]) if case["pre"] else None
    if not case["grad"]:
        return (y, n) if case["pre"] else (y,)
    into = {k: z for k, z in v.items() if z is not None}
    outs, grads = ([y, n], [t["dy"].double(), t["dn"].double()]) if case["pre"] else ([y], [t["dy"].double()])
    got = dict(zip(into, torch.autograd.grad(outs, list(into.values()), grads)))
    return got["x"], got["o"], {k: got[k] for k in PARAMS if k in got}
