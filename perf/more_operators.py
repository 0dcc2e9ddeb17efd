"""Attention of a backbone's blocks, as timed cases: over whole packed prompts with its gradients, over a 4-bit cache one token
at a time, and that cache's writing and reading back.

Between the projections of a block (their 4-bit products and the norms around them are timed apart) stands attention.  Four kinds
of case:

  attn    o = softmax(scale q k^T) v over sequences of different lengths packed one after the other, grouped heads, causal or not
  grad    the same and then the gradients of q, k and v, given that of o: a training step's two calls
  store   keys and values of `rows` tokens into the 4-bit cache, each to a slot of its own, and back out of it
  decode  one query a sequence over that sequence's cached keys and values, found through a table of pages

A head's values are cached in blocks of 32, e2m1 (sign, 0 0.5 1 1.5 2 3 4 6) with one scale 2^(s - 127) a block, s a byte: the
public microscaled 4-bit format.  `run` is the operator in elementary torch operations, or the framework's kernels where `own`
is true.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sentence through one layer of a 768-wide encoder: the smallest call, latency
        dict(name="attn_sentence", kind="attn", batch=1, lo=19, hi=19, heads=12, kv_heads=12, d=64, causal=False),
        # a ragged batch of 32 sentences through the same layer
        dict(name="attn_encoder_ragged", kind="attn", batch=32, lo=1, hi=128, heads=12, kv_heads=12, d=64, causal=False),
        # sixteen samples of 256 tokens through a 4096-wide decoder's layer, as the first epoch runs them
        dict(name="attn_decoder_batch", kind="attn", batch=16, lo=256, hi=256, heads=32, kv_heads=32, d=128, causal=True),
        # one long prompt, grouped heads
        dict(name="attn_prompt", kind="attn", batch=1, lo=8192, hi=8192, heads=32, kv_heads=8, d=128, causal=True),
        # the way there and back through the encoder's layer on the ragged batch
        dict(name="grad_encoder_ragged", kind="grad", batch=32, lo=1, hi=128, heads=12, kv_heads=12, d=64, causal=False),
        # eight ragged samples of 256 to 1024 tokens through the decoder's layer
        dict(name="grad_decoder_ragged", kind="grad", batch=8, lo=256, hi=1024, heads=32, kv_heads=32, d=128, causal=True),
        # the largest: two long samples of odd lengths, grouped heads
        dict(name="grad_long", kind="grad", batch=2, lo=4001, hi=6143, heads=32, kv_heads=8, d=128, causal=True),
        # serving: the newest token of each of 48 sequences into the cache of one layer and back; latency
        dict(name="store_tokens", kind="store", rows=48, kv_heads=5, d=80, page=16, prompt=False, dtype="f32"),
        # a long prompt's keys and values
        dict(name="store_prompt", kind="store", rows=8192, kv_heads=8, d=128, page=64, prompt=True, dtype="bf16"),
        # serving one short conversation, every query head with keys of its own: latency
        dict(name="decode_one", kind="decode", batch=1, lo=700, hi=700, heads=32, kv_heads=32, d=128, page=16),
        # serving 64 conversations of very different lengths, grouped heads
        dict(name="decode_batch", kind="decode", batch=64, lo=1, hi=4096, heads=32, kv_heads=8, d=128, page=64),
        # four books: few rows, a long axis
        dict(name="decode_long", kind="decode", batch=4, lo=60001, hi=65536, heads=32, kv_heads=8, d=128, page=128),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """(query heads, key and value heads, values a head)"""
    kv = rng.choice((1, 2, 3, 4, 5, 8, 8, 12, 16, 32))
    group = rng.choice([g for g in (1, 1, 2, 3, 4, 4, 7, 8, 16) if kv * g <= 64])
    return kv * group, kv, rng.choice((64, 128, 64, 128, 8 * rng.randint(1, 16)))


def draw(rng):
    kind = rng.choice(("attn", "attn", "grad", "grad", "store", "decode", "decode"))
    page = rng.choice((8, 16, 16, 32, 64, 128, 256))
    if kind == "store":
        while True:
            _, kv, d = _heads(rng)
            rows = _log_int(rng, 1, 32768)
            if rows * kv * d <= 8192 * 8 * 128:
                return dict(kind=kind, rows=rows, kv_heads=kv, d=d, page=page, prompt=rows > 256 or rng.random() < 0.3, dtype=rng.choice(("bf16", "f32")))
    most = {"attn": 2 ** 25 * 4096, "grad": 2 ** 24 * 4096, "decode": 4 * 60000 * 4096}[kind]
    while True:
        heads, kv, d = _heads(rng)
        batch, hi = _log_int(rng, 1, 64), _log_int(rng, 1, {"attn": 8192, "grad": 6144, "decode": 65536}[kind])
        lo = rng.choice((hi, max(1, hi // 2), min(hi, 1), 0))
        case = dict(kind=kind, batch=batch, lo=lo, hi=hi, heads=heads, kv_heads=kv, d=d)
        # no more than the largest listed cases cost, counted in query-key pairs and in what the cache holds
        lens = _lens(case)
        if kind == "decode":
            if sum(lens) * max(heads * d, 4 * kv * d) <= most and max(lens) > 0:
                return dict(case, page=page)
        else:
            case["causal"] = rng.random() < 0.6
            if _pairs(lens, case["causal"]) * heads * d <= most and batch * kv <= 512 and sum(lens) * heads * d <= 2 ** 16 * 4096 and max(lens) > 0:
                return case


def _lens(case):
    """The sequences' lengths, lo and hi among them: a matter of the case, not of the seed, because the work depends on them."""
    batch, lo, hi = case["batch"], case["lo"], case["hi"]
    rng = random.Random(f"{batch} {lo} {hi}")
    lens = [hi, lo][:batch] + [rng.randint(lo, hi) for _ in range(batch - 2)]
    rng.shuffle(lens)
    return lens


def _pairs(lens, causal):
    return sum(n * (n + 1) // 2 if causal else n * n for n in lens)


# ---- the stored form in elementary operations ------------------------------------------------------------------------------
def _to_codes(x):
    """x [..., d] to e2m1 codes [..., blocks, 32] and scale bytes [..., blocks].  64 bits, because a value's place next to a border
    decides its code."""
    d = x.shape[-1]
    b = torch.zeros(*x.shape[:-1], (d + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    b[..., :d] = x
    b = b.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(-127, 125)
    e = torch.where(top > 0, e, torch.full_like(e, -127))
    v = torch.ldexp(b, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.clamp(torch.round(a / step) * step, max=6.0)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    return (torch.searchsorted(grid, q) + 8 * (v < 0)).to(torch.uint8), (e[..., 0] + 127).to(torch.uint8)


def _from_codes(codes, scales, d):
    """The values that codes stand for, in 32 bits (which hold them exactly)."""
    table = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float32, device=codes.device)
    s = torch.ldexp(torch.ones((), dtype=torch.float32, device=codes.device), scales.to(torch.int32) - 127)
    return (table[codes.long()] * s[..., None]).flatten(-2)[..., :d]


def _pack(codes):
    """Two codes a byte, the even value in the low half."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _rng(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _projected(g, rows, heads, d, dtype, spread=1.0):
    """Queries, keys or values of `heads` heads: normal, heads of different size, one value in 64 of a head four times as large."""
    x = torch.randn(rows, heads, d, generator=g, device=DEV)
    x *= spread * torch.exp(torch.randn(heads, 1, generator=g, device=DEV) / 4)
    x *= 1 + 3 * (torch.rand(heads, d, generator=g, device=DEV) < 1 / 64)
    return x.reshape(rows, heads * d).to(dtype)


def _inputs(case, seed):
    """The inputs of a case, by name."""
    g, kind, d, bf16 = _rng(seed), case["kind"], case["d"], torch.bfloat16
    if kind == "store":
        rows, kv, page = case["rows"], case["kv_heads"], case["page"]
        pages = (rows + page - 1) // page + 3
        if case["prompt"]:  # one sequence's tokens in order, its pages anywhere
            at = torch.arange(rows, device=DEV)
            slots = torch.randperm(pages, generator=g, device=DEV)[at // page] * page + at % page
        else:  # tokens of as many sequences
            slots = torch.randperm(pages * page, generator=g, device=DEV)[:rows]
        k, v = (_projected(g, rows, kv, d, DTYPES[case["dtype"]]) for _ in range(2))
        return dict(k=k, v=v, slots=slots, pages=pages)
    lens = _lens(case)
    rows, heads, kv = sum(lens), case["heads"], case["kv_heads"]
    if kind == "decode":
        page = case["page"]
        held = [(n + page - 1) // page for n in lens]
        order = torch.randperm(sum(held) + 3, generator=g, device=DEV).to(torch.int32)
        table = torch.full((len(lens), max(held)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(held):
            table[b, :n] = order[at:at + n]
            at += n
        where = torch.cat([torch.arange(n, device=DEV) for n in lens])
        row = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV))
        slots = table[row, where // page].long() * page + where % page
        return dict(q=_projected(g, len(lens), heads, d, bf16, 1.5), k=_projected(g, rows, kv, d, bf16), v=_projected(g, rows, kv, d, bf16),
                    table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), slots=slots, pages=sum(held) + 3)
    t = dict(q=_projected(g, rows, heads, d, bf16, 1.5), k=_projected(g, rows, kv, d, bf16), v=_projected(g, rows, kv, d, bf16))
    if kind == "grad":
        t["do"] = _projected(g, rows, heads, d, bf16)
    return t


def prepare(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    s = dict(case, **t)
    if kind in ("attn", "grad"):
        s["seqs"] = _lens(case)
        at = [0]
        for n in s["seqs"]:
            at.append(at[-1] + n)
        s["offsets"] = torch.tensor(at, dtype=torch.int32, device=DEV)
    # where results go: a program that runs layer after layer keeps these buffers, as it keeps handles of its layers
    if kind == "store":
        s["k_back"], s["v_back"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    else:
        s["o"] = torch.empty_like(s["q"])
    if kind == "grad":
        s["dq"], s["dk"], s["dv"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])
        s["lse"] = torch.empty(case["heads"], s["q"].shape[0], dtype=torch.float32, device=DEV)
    if own:
        from paper_2408_10746_amd import runtime
        if kind in ("attn", "grad"):
            s["attention"] = runtime.Attention(case["heads"], case["d"], kv_heads=case["kv_heads"], causal=case["causal"])
        else:
            s["cache"] = runtime.Kv4Cache(s["pages"], case["page"], case["kv_heads"], case["d"], device=DEV)
            if kind == "decode":
                s["cache"].write(s["k"], s["v"], s["slots"])
    elif kind == "decode":
        # the cache as the plain form holds it: codes two a byte and scale bytes, a slot's heads next to each other
        n, kv, d = s["pages"] * case["page"], case["kv_heads"], case["d"]
        for name in ("k", "v"):
            codes = torch.zeros(n, kv, (d + 31) // 32, 16, dtype=torch.uint8, device=DEV)
            scales = torch.zeros(n, kv, (d + 31) // 32, dtype=torch.uint8, device=DEV)
            for at in range(0, t[name].shape[0], 1 << 15):
                c, e = _to_codes(t[name][at:at + (1 << 15)].reshape(-1, kv, d))
                codes[s["slots"][at:at + (1 << 15)]], scales[s["slots"][at:at + (1 << 15)]] = _pack(c), e
            s[name + "_cache"] = codes, scales
        s["seqs"] = _lens(case)
    if kind == "decode":
        del s["k"], s["v"], s["slots"]
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    kind = s["kind"]
    if kind == "attn":
        s["attention"].forward(s["q"], s["k"], s["v"], s["offsets"], s["o"])
        return s["o"]
    if kind == "grad":
        s["attention"].forward(s["q"], s["k"], s["v"], s["offsets"], s["o"], s["lse"])
        s["attention"].backward(s["q"], s["k"], s["v"], s["offsets"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"])
        return s["o"], s["dq"], s["dk"], s["dv"]
    if kind == "store":
        s["cache"].write(s["k"], s["v"], s["slots"])
        s["cache"].read(s["slots"], s["k_back"], s["v_back"])
        return s["k_back"], s["v_back"]
    s["cache"].attend(s["q"], s["table"], s["lens"], s["o"])
    return s["o"]


def _by_head(x, heads):
    return x.float().reshape(x.shape[0], heads, -1).transpose(0, 1)


def _plain(s):
    kind, d = s["kind"], s["d"]
    if kind == "store":
        back = []
        for x in (s["k"], s["v"]):
            codes, scales = _to_codes(x.reshape(-1, s["kv_heads"], d))
            n = s["pages"] * s["page"]
            held = torch.empty(n, *codes.shape[1:3], 16, dtype=torch.uint8, device=DEV), torch.empty(n, *scales.shape[1:], dtype=torch.uint8, device=DEV)
            held[0][s["slots"]], held[1][s["slots"]] = _pack(codes), scales
            back.append(_from_codes(_unpack(held[0][s["slots"]]), held[1][s["slots"]], d).reshape(x.shape).to(x.dtype))
        return tuple(back)
    heads, kv, scale = s["heads"], s["kv_heads"], 1 / math.sqrt(d)
    group = heads // kv
    if kind == "decode":
        for b, n in enumerate(s["seqs"]):
            if n == 0:
                s["o"][b] = 0
                continue
            where = torch.arange(n, device=DEV)
            slots = s["table"][b, where // s["page"]].long() * s["page"] + where % s["page"]
            k, v = (_from_codes(_unpack(codes[slots]), scales[slots], d).transpose(0, 1) for codes, scales in (s["k_cache"], s["v_cache"]))
            p = _softmax(s["q"][b].float().reshape(kv, group, d) @ k.transpose(1, 2) * scale)
            s["o"][b] = (p @ v).reshape(-1).to(s["o"].dtype)
        return s["o"]
    at = 0
    for n in s["seqs"]:
        rows = slice(at, at + n)
        at += n
        q, k, v = _by_head(s["q"][rows], heads), _by_head(s["k"][rows], kv), _by_head(s["v"][rows], kv)
        do = _by_head(s["do"][rows], heads) if kind == "grad" else None
        wide = heads * n * n <= 1 << 28  # all heads at once, or a group after the other where their scores would take gigabytes
        for h in ([slice(0, kv)] if wide else [slice(i, i + 1) for i in range(kv)]):
            hq = slice(h.start * group, h.stop * group)
            parts = _attend(q[hq], k[h], v[h], scale, s["causal"], None if do is None else do[hq])
            for name, part in zip(("o", "dq", "dk", "dv"), parts):
                of = hq if name in ("o", "dq") else h
                s[name][rows, of.start * d:of.stop * d] = part.transpose(0, 1).reshape(n, -1).to(s[name].dtype)
    return s["o"] if kind == "attn" else (s["o"], s["dq"], s["dk"], s["dv"])


def _softmax(scores):
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _attend(q, k, v, scale, causal, do):
    """o, and given do the gradients of q, k and v, of [heads][n][d] queries and [kv heads][n][d] keys and values."""
    if q.shape[1] == 0:
        return (q,) if do is None else (q, q, k, v)
    group = q.shape[0] // k.shape[0]
    kg, vg = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    scores = q @ kg.transpose(1, 2) * scale
    if causal:
        at = torch.arange(q.shape[1], device=q.device)
        scores = torch.where(at[None, :] <= at[:, None], scores, -math.inf)
    p = _softmax(scores)
    del scores
    o = p @ vg
    if do is None:
        return (o,)
    dv = p.transpose(1, 2) @ do
    dp = do @ vg.transpose(1, 2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    shared = lambda t: t.reshape(-1, group, *t.shape[1:]).sum(1)  # noqa: E731
    return o, ds @ kg, shared(ds.transpose(1, 2) @ q), shared(dv)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    kind, d, kv = case["kind"], case["d"], case["kv_heads"]
    held = 17 * ((d + 31) // 32)  # bytes of one head's values in the cache
    if kind == "store":
        n = 2 * case["rows"] * kv
        return {"bytes": 2.0 * n * (d * (2 if case["dtype"] == "bf16" else 4) + held), "flops": 4.0 * n * d}
    lens, heads = _lens(case), case["heads"]
    if kind == "decode":
        return {"bytes": 2.0 * sum(lens) * kv * held + 4.0 * len(lens) * heads * d, "flops": 4.0 * sum(lens) * heads * d}
    pairs = _pairs(lens, case["causal"])
    if kind == "attn":
        return {"bytes": 2.0 * sum(lens) * d * (2 * heads + 2 * kv), "flops": 4.0 * pairs * heads * d}
    return {"bytes": 2.0 * sum(lens) * d * (4 * heads + 4 * kv), "flops": 14.0 * pairs * heads * d}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _nearest(x):
    """x [..., d] in the stored form by its definition: every value to the nearest of its block's grid, of two as near the one with
    the even code."""
    d = x.shape[-1]
    b = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    some = torch.where(top > 0, top, 1.0)
    scale = torch.exp2(torch.floor(torch.log2(some)) - 2)
    scale = torch.where(scale * 8 <= some, scale * 2, torch.where(scale * 4 > some, scale / 2, scale))  # the logarithm's own rounding
    a = b.abs() / scale
    best, far = torch.zeros_like(a), a.clone()
    for code in range(1, 8):
        off = (a - GRID[code]).abs()
        better = (off < far) | ((off == far) & (code % 2 == 0))
        best, far = torch.where(better, GRID[code], best), torch.where(better, off, far)
    return (torch.sign(b) * best * scale).flatten(-2)[..., :d]


def exact(case, seed):
    t, kind, d, kv = _inputs(case, seed), case["kind"], case["d"], case["kv_heads"]
    if kind == "store":
        return tuple(_nearest(t[x].reshape(-1, kv, d)).reshape(t[x].shape) for x in ("k", "v"))
    heads = case["heads"]
    group, grad = heads // kv, kind == "grad"
    out = {x: torch.zeros(t[x].shape, dtype=torch.float64, device=DEV) for x in (("q", "k", "v") if grad else ())}
    o = torch.zeros(t["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, n in enumerate(_lens(case)):
        rows = slice(at, at + n)
        mine = slice(b, b + 1) if kind == "decode" else rows
        at += n
        if n == 0:
            continue
        for h in range(kv):  # one key and value head with its queries after the other
            cols, qcols = slice(h * d, (h + 1) * d), slice(h * group * d, (h + 1) * group * d)
            q = t["q"][mine, qcols].double().unflatten(1, (group, d)).permute(1, 0, 2).requires_grad_(grad)
            k, v = ((_nearest(t[x][rows, cols]) if kind == "decode" else t[x][rows, cols].double()).requires_grad_(grad) for x in ("k", "v"))
            z = torch.matmul(q, k.t().contiguous()) / d ** 0.5
            if case.get("causal"):
                z = z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -math.inf)
            r = torch.matmul(torch.softmax(z, -1), v)
            del z
            o[mine, qcols] = r.detach().permute(1, 0, 2).flatten(1)
            if grad:
                do = t["do"][rows, qcols].double().unflatten(1, (group, d)).permute(1, 0, 2)
                gq, gk, gv = torch.autograd.grad(r, (q, k, v), do)
                out["q"][rows, qcols], out["k"][rows, cols], out["v"][rows, cols] = gq.permute(1, 0, 2).flatten(1), gk, gv
    return (o, out["q"], out["k"], out["v"]) if grad else o
