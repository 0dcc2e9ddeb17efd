"""GPU: attention over the 4-bit cache where scores are infinite or no number: the softmax over such scores is none, and is not taken for one over
no tokens; and what a call allocates."""
import math

import pytest
import torch

from oracle import attn_oracle as ao
from paper_2408_10746_amd import binding as pb
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("page", [8, 16])
@pytest.mark.parametrize("kv,batch,n", [(2, 3, 40), (2, 3, 700), (2, 3, 9000), (8, 80, 1500)])
def test_scores_that_are_all_minus_infinity_are_tokens_all_the_same(kv, batch, n, page):
    """Sequence 0: no tokens.  1: all tokens' scores are -inf for one query head, the others' as they are.  2: pages outside the cache but for the
    last one, whose scores are -inf for that head, and the pages before hold none."""
    heads, d, pages = 2 * kv, 64, -(-n // page)
    g = torch.Generator(device="cuda").manual_seed(n + page)
    k, v = (torch.randn(n, kv * d, generator=g, device="cuda").to(BF) for _ in range(2))
    k[:, 5] = k[:, 5].abs() + 1
    c = rt.Kv4Cache(pages, page, kv, d)
    at = torch.arange(n, device="cuda")
    c.write(k, v, at)
    kb, vb = torch.empty(n, kv * d, device="cuda"), torch.empty(n, kv * d, device="cuda")
    c.read(at, kb, vb)
    assert bool((kb[:, 5] > 0).all())
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(batch, 1)
    table[2, :-1] = -1
    lens = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    lens[0] = 0
    q = (torch.randn(batch, heads * d, generator=g, device="cuda") / 8).to(BF)
    q[1:3, 5] = -math.inf
    o = torch.full_like(q, 3.0)
    c.attend(q, table, lens, o)
    assert not o[0].any()
    assert o[1:3, :d].isnan().all() and o[1:3, d:].isfinite().all()
    for b in range(1, batch):
        s = slice((pages - 1) * page, n) if b == 2 else slice(0, n)
        by = lambda t: t[s].double().reshape(-1, kv, d).transpose(0, 1)  # noqa: E731
        x = q[b].double().reshape(heads, d)
        if b < 3:
            x[0] = 0
        ref, bound = ao.decode(x, by(kb), by(vb), d ** -0.5)
        off = (o[b].double().reshape(heads, d) - ref).abs()
        first = int(b < 3)
        assert bool((off[first:] <= bound[first:]).all()), b


@pytest.mark.parametrize("batch,pages", [(64, 64), (4096, 2), (2, 1000), (1, 10)])
def test_attending_takes_no_more_scratch_than_its_call(batch, pages):
    """What the call itself asks for, and not room for every smaller one."""
    heads, kv, d = 32, 8, 128
    c = rt.Kv4Cache(4, 16, kv, d)
    q, o = torch.zeros(batch, heads * d, device="cuda", dtype=BF), torch.empty(batch, heads * d, device="cuda", dtype=BF)
    table, lens = torch.zeros(batch, pages, dtype=torch.int32, device="cuda"), torch.full((batch,), 5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    c.attend(q, table, lens, o)
    assert torch.cuda.max_memory_allocated() - before <= pb.pac_kv4_attend_bytes(c._at(), heads, batch, pages) + 512  # (the allocator's granularity)
    assert not o.any()
