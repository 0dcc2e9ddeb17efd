"""GPU parity of the 4-bit key and value cache: what is written and read back against oracle/block_oracle.py, to the bit, and attention over it
against oracle/attn_oracle.py (64 bits) on the values that the cache holds, each result within what the stated roundings may make there (p
and o to bf16, scores and sums in 32 bits)."""
import math

import numpy as np
import pytest
import torch

from oracle import attn_oracle as ao
from oracle import block_oracle as bo
from paper_2408_10746_amd import binding as pb
from paper_2408_10746_amd import runtime as rt

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def states(seed, rows, cols, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g, device="cuda").float())
    return x.to(dtype)


def stored(x, d):
    """The values that the heads of x become."""
    h = x.float().cpu().numpy().reshape(-1, d)
    return torch.from_numpy(bo.values(*bo.quantize(h), d).reshape(x.shape)).cuda()


def same(a, b):
    """Equal to the bit, NaN to NaN."""
    return torch.equal(a.double().nan_to_num(7e37), b.double().nan_to_num(7e37))


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("rows,kv,page", [(1, 1, 8), (37, 3, 16), (130, 2, 64)])
def test_written_and_read_back(rows, kv, page, d, dtype):
    pages = rows // page + 3
    c = rt.Kv4Cache(pages, page, kv, d)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(rows))[:rows].cuda()
    k, v = states(d, rows, kv * d, dtype), states(d + 1, rows, kv * d, dtype)
    kb, vb = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    c.write(k, v, slots)
    c.read(slots, kb, vb)
    assert same(kb, stored(k, d)) and same(vb, stored(v, d))


def test_what_blocks_of_any_kind_become():
    """Zeros, the least and largest values, ties, infinities and NaN, a block each."""
    d, kv = 128, 1
    x = torch.zeros(12, d, device="cuda")
    x[1], x[2] = 1e-45, 3.4e38
    x[3] = torch.arange(d, device="cuda") / 16 - 4
    x[4, 5], x[5, 70], x[6, 127] = math.inf, math.nan, -math.inf
    x[7] = 2.0 ** -126 * torch.linspace(-1, 1, d, device="cuda")
    x[8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda").repeat(16)
    x[9] = -x[8]
    x[10], x[11] = 7.9, -0.0
    c = rt.Kv4Cache(2, 8, kv, d)
    slots = torch.arange(12, device="cuda") + 2
    k, v = torch.empty_like(x), torch.empty_like(x)
    c.write(x, x.flip(0).contiguous(), slots)
    c.read(slots, k, v)
    assert same(k, stored(x, d)) and same(v, stored(x, d).flip(0))
    assert k[4, :32].isnan().all() and not k[4, 32:].isnan().any() and torch.equal(torch.signbit(k[11]), torch.signbit(x[11]))


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 40])
def test_any_stride_and_alignment(d, dtype):
    """Views at odd places, of odd strides; k and v side by side in one matrix; nothing beside the rows is written."""
    rows, kv = 19, 2
    for lead, gap in ((1, 3), (8, 8), (4, 4)):
        wide = 2 * kv * d + 2 * lead + gap
        x = states(d + lead, rows, wide, dtype)
        k, v = x[:, lead:lead + kv * d], x[:, lead + kv * d + gap:lead + 2 * kv * d + gap]
        c = rt.Kv4Cache(3, 8, kv, d)
        slots = torch.randperm(24, generator=torch.Generator().manual_seed(1))[:rows].cuda()
        c.write(k, v, slots)
        back = torch.full_like(x, 3.0)
        kb, vb = back[:, lead:lead + kv * d], back[:, lead + kv * d + gap:lead + 2 * kv * d + gap]
        c.read(slots, kb, vb)
        assert same(kb, stored(k.contiguous(), d)) and same(vb, stored(v.contiguous(), d))
        keep = torch.ones(wide, dtype=torch.bool)
        keep[lead:lead + kv * d] = keep[lead + kv * d + gap:lead + 2 * kv * d + gap] = False
        assert (back[:, keep.cuda()] == 3).all()


def test_slots_outside_the_cache_are_left_out():
    pages, page, kv, d = 4, 8, 2, 64
    c = rt.Kv4Cache(pages, page, kv, d)
    k, v = states(0, 8, kv * d), states(1, 8, kv * d)
    slots = torch.tensor([3, -1, 31, 32, 1 << 40, -(1 << 62), (1 << 63) - 1, 0], device="cuda")
    c.write(states(2, 32, kv * d), states(3, 32, kv * d), torch.arange(32, device="cuda"))
    before = c.data.clone()
    only = torch.tensor([False, True, False, True, True, True, True, False], device="cuda")
    c.write(k[only].contiguous(), v[only].contiguous(), slots[only].contiguous())
    assert torch.equal(before, c.data)
    c.write(k, v, slots)
    kb, vb = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    c.read(slots, kb, vb)
    assert (kb[only] == 3).all() and (vb[only] == 3).all()
    assert same(kb[~only], stored(k, d)[~only]) and same(vb[~only], stored(v, d)[~only])
    # the slots that no row went to hold what they held
    rest = torch.tensor([s for s in range(32) if s not in (3, 31, 0)], device="cuda")
    kr, vr = torch.empty(29, kv * d, device="cuda"), torch.empty(29, kv * d, device="cuda")
    c.read(rest, kr, vr)
    assert same(kr, stored(states(2, 32, kv * d), d)[rest]) and same(vr, stored(states(3, 32, kv * d), d)[rest])


def filled(seed, lens, kv, d, page, spare=2, special=None):
    """A cache with sequences of those lengths in pages at random; what else is in its pages is NaN (no value)."""
    held = [-(-n // page) for n in lens]
    pages = sum(held) + spare
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = rt.Kv4Cache(pages, page, kv, d)
    c.data.fill_(255)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(held + [1])), -1, dtype=torch.int32, device="cuda")
    at, slots = 0, []
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        where = torch.arange(lens[b], device="cuda")
        slots.append(table[b, where // page].long() * page + where % page if lens[b] else where)
        at += n
    slots, rows = torch.cat(slots), sum(lens)
    k, v = (torch.randn(rows, kv * d, generator=g, device="cuda").to(BF) for _ in range(2))
    c.write(k, v, slots)
    kb, vb = torch.empty(rows, kv * d, device="cuda"), torch.empty(rows, kv * d, device="cuda")
    c.read(slots, kb, vb)
    return c, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), kb.double(), vb.double()


def check(o, q, lens, kb, vb, kv, d, scale, drop=None):
    at = 0
    for b, n in enumerate(lens):
        s = torch.arange(at, at + n, device="cuda")
        at += n
        if drop is not None:
            s = s[drop(b, torch.arange(n)).cuda()]
        heads = lambda t: t[s].reshape(-1, kv, d).transpose(0, 1)  # noqa: E731
        ref, bound = ao.decode(q[b].double().reshape(-1, d), heads(kb), heads(vb), scale)
        off = (o[b].double().reshape(-1, d) - ref).abs()
        assert torch.isfinite(o[b]).all() and bool((off <= bound).all()), (b, n, float((off / bound).nan_to_num(0).amax()))


CASES = [(1, 1, 128, 8, [1]), (4, 4, 64, 16, [1, 2, 3, 4, 5]), (8, 2, 128, 16, [0, 31, 32, 33, 0]), (32, 8, 128, 64, [700, 1, 0, 129]), (6, 2, 32, 8, [15, 16, 17, 250]),
         (5, 5, 80, 16, [300, 77]), (7, 1, 96, 32, [513, 31]), (16, 1, 40, 8, [100]), (17, 1, 64, 16, [90, 270]), (48, 1, 128, 128, [1000]),
         (33, 3, 72, 8, [41, 260]), (2, 2, 8, 256, [255, 256, 257]), (12, 12, 64, 65536, [20, 3000]), (4, 1, 104, 16, [2049]), (64, 64, 24, 32, [66])]


@pytest.mark.parametrize("heads,kv,d,page,lens", CASES, ids=str)
def test_attend(heads, kv, d, page, lens):
    c, table, ln, kb, vb = filled(heads + d, lens, kv, d, page)
    q = states(3, len(lens), heads * d) / 8
    o = torch.full_like(q, 3.0)
    c.attend(q, table, ln, o)
    check(o, q, lens, kb, vb, kv, d, d ** -0.5)


@pytest.mark.parametrize("heads,kv,d,page,lens", [(8, 1, 128, 64, [20000]), (4, 4, 64, 16, [9000, 17, 5000]), (32, 8, 128, 256, [33333, 70000])])
def test_long_caches(heads, kv, d, page, lens):
    """Many splits of one sequence, joined; short ones beside long ones."""
    c, table, ln, kb, vb = filled(d, lens, kv, d, page)
    q = states(5, len(lens), heads * d) / 4
    o = torch.empty_like(q)
    c.attend(q, table, ln, o)
    check(o, q, lens, kb, vb, kv, d, d ** -0.5)
    for scale in (3.0, 1e-3):
        c.attend(q, table, ln, o, scale=scale)
        check(o, q, lens, kb, vb, kv, d, scale)


@pytest.mark.parametrize("d,page", [(128, 8), (64, 16), (96, 64)])
def test_pages_outside_the_cache_hold_no_tokens(d, page):
    lens, heads, kv = [5 * page + 3, 700, 3 * page], 4, 2
    c, table, ln, kb, vb = filled(1, lens, kv, d, page)
    table[0, 1], table[0, 5], table[1, 0], table[2, :] = -1, c.pages, 2 ** 31 - 1, -2 ** 31
    q, o = states(2, 3, heads * d) / 8, torch.empty(3, heads * d, device="cuda", dtype=BF)
    c.attend(q, table, ln, o)
    gone = {0: (1, 5), 1: (0,), 2: tuple(range(3))}
    check(o, q, lens, kb, vb, kv, d, d ** -0.5, drop=lambda b, t: ~torch.isin(t // page, torch.tensor(gone[b])))
    assert not o[2].any()


def test_lengths_outside_the_table():
    """Negative ones are 0, others end with the table; a table without pages."""
    c, table, ln, kb, vb = filled(2, [64, 48], 2, 64, 16)  # whole pages: every place that a length reaches has been written
    q, o = states(3, 2, 256) / 8, torch.empty(2, 256, device="cuda", dtype=BF)
    c.attend(q, table, torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda"), o)
    check(o, q, [64, 0], kb, vb, 2, 64, 0.125)
    c.attend(q, table, torch.tensor([-2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), o)
    check(o[1:], q[1:], [48], kb[64:], vb[64:], 2, 64, 0.125)
    assert not o[0].any()
    o.fill_(3.0)
    c.attend(q, table[:, :0], ln, o)
    assert not o.any()


def test_tables_and_queries_with_strides():
    """A slice of a wider table; queries and results as columns of wider matrices."""
    lens = [100, 33, 7]
    c, table, ln, kb, vb = filled(4, lens, 2, 64, 8)
    wide = torch.full((3, table.shape[1] + 9), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    wide[:, 4:4 + table.shape[1]] = table
    m = states(6, 3, 256 + 16 + 256) / 8
    keep = m.clone()
    q, o = m[:, :256], m[:, 264:264 + 256]
    c.attend(q, wide[:, 4:4 + table.shape[1]], ln, o)
    check(o, q, lens, kb, vb, 2, 64, 0.125)
    rest = torch.ones(m.shape[1], dtype=torch.bool)
    rest[264:264 + 256] = False
    assert torch.equal(m[:, rest.cuda()], keep[:, rest.cuda()])


def test_sequences_may_share_pages():
    c, table, ln, kb, vb = filled(7, [48, 0], 1, 128, 16)
    table[1] = table[0]
    ln = torch.tensor([48, 20], dtype=torch.int32, device="cuda")
    q, o = states(1, 2, 256) / 8, torch.empty(2, 256, device="cuda", dtype=BF)
    c.attend(q, table, ln, o)
    check(o[:1], q[:1], [48], kb, vb, 1, 128, 128 ** -0.5)
    check(o[1:], q[1:], [20], kb, vb, 1, 128, 128 ** -0.5)


def test_tokens_without_a_value_reach_their_sequence_only():
    """NaN in one sequence's cache, and in what lies behind the ends of all."""
    lens, kv, d, page = [50, 60, 45], 2, 64, 16
    c, table, ln, kb, vb = filled(8, lens, kv, d, page)
    q, o, p = states(4, 3, 256) / 8, torch.empty(3, 256, device="cuda", dtype=BF), torch.empty(3, 256, device="cuda", dtype=BF)
    c.attend(q, table, ln, o)
    x = torch.zeros(1, kv * d, device="cuda")
    x[0, 3] = math.nan
    at = 33
    slot = (table[1, at // page].long() * page + at % page)[None]
    c.write(x, x, slot)
    c.attend(q, table, ln, p)
    assert torch.equal(o[0], p[0]) and torch.equal(o[2], p[2])
    assert p[1, :128].isnan().all() and torch.equal(o[1, 128:].isnan(), p[1, 128:].isnan())  # head 0's two queries, the other head none


def test_a_cache_past_32_bits():
    """Bytes, slots and pages above 2^32: the last pages of a cache of 9 GB."""
    kv, d, page = 8, 128, 1024
    pages = (9 << 30) // (kv * 272 * page // 2)
    c = rt.Kv4Cache(pages, page, kv, d)
    assert c.data.numel() > 2 ** 32
    n = 1500
    table = torch.tensor([[pages - 1, 0], [pages // 2, pages - 2]], dtype=torch.int32, device="cuda")
    where = torch.arange(n, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    kb, vb = [], []
    for b in range(2):
        k, v = (torch.randn(n, kv * d, generator=g, device="cuda").to(BF) for _ in range(2))
        slots = table[b, where // page].long() * page + where % page
        c.write(k, v, slots)
        c.read(slots, k, v)
        kb.append(k.double()), vb.append(v.double())
        assert same(k[::500], stored(k[::500].contiguous(), d))  # what is stored is stored again as it is
    ln = torch.full((2,), n, dtype=torch.int32, device="cuda")
    q, o = states(1, 2, 16 * d) / 8, torch.empty(2, 16 * d, device="cuda", dtype=BF)
    c.attend(q, table, ln, o)
    check(o, q, [n, n], torch.cat(kb), torch.cat(vb), kv, d, d ** -0.5)


def test_same_bits_streams_and_graphs():
    """A step of serving (the newest token's keys and values into the cache, attention over it): again, on a stream of its own, captured and
    replayed with eager work between, lengths and slots growing on the device."""
    lens, kv, heads, d, page = [300, 17, 2000], 2, 8, 128, 16
    c, table, ln, kb, vb = filled(9, [n + 8 for n in lens], kv, d, page)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q, k, v = states(1, 3, heads * d) / 8, states(2, 3, kv * d), states(3, 3, kv * d)
    o, slots = torch.empty_like(q), torch.empty(3, dtype=torch.int64, device="cuda")

    def step(out):
        at = ln.long()
        slots.copy_(table.gather(1, (at // page)[:, None])[:, 0].long() * page + at % page)
        c.write(k, v, slots)
        ln.add_(1)
        c.attend(q, table, ln, out)

    data = c.data.clone()

    def reset():
        c.data.copy_(data)
        ln.copy_(torch.tensor(lens, dtype=torch.int32))

    want = []
    for _ in range(4):
        step(o)
        want.append(o.clone())
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(o)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o, want[0])
    reset()
    g, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(g):
        step(out)
    reset()
    for turn in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[turn]), turn
        c.attend(q, table, ln, o)
        assert torch.equal(o, out)


def test_the_bindings_functions_are_the_layers_calls():
    lens, kv, heads, d, page = [300, 17], 2, 8, 64, 16
    c, table, ln, kb, vb = filled(9, lens, kv, d, page)
    q, o, p = states(1, 2, heads * d) / 8, torch.empty(2, heads * d, device="cuda", dtype=BF), torch.empty(2, heads * d, device="cuda", dtype=BF)
    c.attend(q, table, ln, o, scale=0.2)
    st, s = torch.cuda.current_stream().cuda_stream, pb.pac_kv4(c.data.data_ptr(), c.pages, page, kv, d)
    need = pb.pac_kv4_attend_workspace_bytes(s, heads, 2, table.shape[1])
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    pb.pac_kv4_attend(s, heads, 0.2, 2, table.data_ptr(), table.shape[1], table.stride(0), ln.data_ptr(), q.data_ptr(), heads * d, p.data_ptr(), heads * d,
                      ws.data_ptr(), need, st)
    assert torch.equal(o, p)
    e = rt.Kv4Cache(4, page, kv, d)
    f = pb.pac_kv4(e.data.data_ptr(), 4, page, kv, d)
    k, v, slots = states(2, 9, kv * d), states(3, 9, kv * d), torch.arange(9, device="cuda")
    pb.pac_kv4_write(f, 9, slots.data_ptr(), k.data_ptr(), kv * d, v.data_ptr(), kv * d, pb.PAC_BF16, st)
    kr, vr, k2, v2 = (torch.empty_like(k) for _ in range(4))
    pb.pac_kv4_read(f, 9, slots.data_ptr(), kr.data_ptr(), kv * d, vr.data_ptr(), kv * d, pb.PAC_BF16, st)
    e.read(slots, k2, v2)
    assert same(kr, stored(k, d)) and torch.equal(kr, k2) and torch.equal(vr, v2)


def test_runtime_refuses():
    c, table, ln, _, _ = filled(0, [20, 5], 2, 64, 16)
    q, o = states(1, 2, 256), torch.empty(2, 256, device="cuda", dtype=BF)
    k, v, slots = states(2, 3, 128), states(3, 3, 128), torch.arange(3, device="cuda")
    c.attend(q, table, ln, o)
    for args in ((q.float(), table, ln, o), (q[:, :100], table, ln, o), (q, table.long(), ln, o), (q, table[:1], ln, o), (q, table, ln.long(), o),
                 (q, table, ln[:1], o), (q, table, ln, o.float()), (q, table, ln, o[:1]), (q, table.t(), ln, o), (q, table, ln.cpu(), o)):
        with pytest.raises(ValueError):
            c.attend(*args)
    for args in ((k, v, slots.int()), (k, v[:2], slots), (k, v.float(), slots), (k[:, :64], v, slots), (k.half(), v.half(), slots), (k, v, slots.cpu())):
        with pytest.raises(ValueError):
            c.write(*args)
        with pytest.raises(ValueError):
            c.read(args[2], args[0], args[1])
    with pytest.raises(pb.PacError):
        c.attend(q, table, ln, q)
    with pytest.raises(pb.PacError):
        c.attend(q, table, ln, o, scale=-1.0)
    with pytest.raises(pb.PacError):  # three query heads over two
        c.attend(q[:, :192].contiguous(), table, ln, o[:, :192].contiguous())
    for args in ((-1, 16, 2, 64), (4, 12, 2, 64), (4, 16, 0, 64), (4, 16, 2, 60)):
        with pytest.raises(ValueError):
            rt.Kv4Cache(*args)
    assert rt.Kv4Cache(0, 16, 2, 64).data.numel() == 0 and np.isfinite(float(o.float().sum()))


def test_prompt_then_tokens():
    """A run of the operators together: a prompt through causal attention, its keys and values into the cache, then token after token; each answer
    against 64-bit attention over what the cache holds, and near the prompt's own attention over all tokens at full precision."""
    heads, kv, d, page, n, more = 8, 2, 64, 16, 75, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n + more, h * d, generator=g, device="cuda").to(BF) for h in (heads, kv, kv))
    att, whole = rt.Attention(heads, d, kv_heads=kv, causal=True), torch.empty_like(q)
    att.forward(q, k, v, rt.packed_offsets([n + more]), whole)
    c = rt.Kv4Cache(12, page, kv, d)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(0))[:6].to(torch.int32).cuda()[None]
    slot = lambda t: table[0, t // page].long() * page + t % page  # noqa: E731
    first = torch.empty(n, heads * d, device="cuda", dtype=BF)
    att.forward(q[:n], k[:n], v[:n], rt.packed_offsets([n]), first)
    assert torch.equal(first, whole[:n])  # a longer prompt's rows
    c.write(k[:n], v[:n], slot(torch.arange(n, device="cuda")))
    for t in range(n, n + more):
        c.write(k[t:t + 1], v[t:t + 1], slot(torch.tensor([t], device="cuda")))
        o = torch.empty(1, heads * d, device="cuda", dtype=BF)
        c.attend(q[t:t + 1], table, torch.tensor([t + 1], dtype=torch.int32, device="cuda"), o)
        kb, vb = torch.empty(t + 1, kv * d, device="cuda"), torch.empty(t + 1, kv * d, device="cuda")
        c.read(slot(torch.arange(t + 1, device="cuda")), kb, vb)
        check(o, q[t:t + 1], [t + 1], kb.double(), vb.double(), kv, d, d ** -0.5)
        # 4 bits lose about a tenth of a value; the answer stays that near
        far = float((o.double() - whole[t:t + 1].double()).norm() / whole[t:t + 1].double().norm())
        assert far < 0.5, far


@pytest.mark.parametrize("batch", [2, 63, 64, 65, 130])
def test_sequences_of_any_lengths_in_any_order(batch):
    """Long ones are started first, 64 sequences at a time: each is answered once, also those of one length, without tokens (a negative length)
    and with all that the table holds (a length past it)."""
    heads, kv, d, page, most = 2, 1, 32, 16, 16384
    g = torch.Generator().manual_seed(batch)
    lens = torch.randint(1, most, (batch,), generator=g)
    lens[torch.rand(batch, generator=g) < 0.6] //= 40
    lens[torch.rand(batch, generator=g) < 0.2] = 1023
    lens[1], lens[batch // 2] = most, 0
    lens = lens.tolist()
    c, table, ln, kb, vb = filled(batch, lens, kv, d, page)
    ln[1], ln[batch // 2] = most + 12345, -7
    q = states(6, batch, heads * d) / 4
    o = torch.full_like(q, 3.0)
    c.attend(q, table, ln, o)
    check(o, q, lens, kb, vb, kv, d, d ** -0.5)


@pytest.mark.parametrize("batch,kv,d,page,most", [(64, 8, 32, 16, 700), (128, 4, 64, 8, 300), (520, 1, 96, 32, 129), (1020, 1, 40, 16, 2000)])
def test_one_workgroup_for_every_sequence_and_head(batch, kv, d, page, most):
    """As many sequences by heads as fill the card without a split, of all lengths and in any order."""
    heads = 2 * kv
    g = torch.Generator().manual_seed(batch)
    lens = (torch.rand(batch, generator=g) ** 3 * most).long()
    lens[batch // 3], lens[5] = most, 0
    lens = lens.tolist()
    c, table, ln, kb, vb = filled(batch, lens, kv, d, page)
    ln[5] = -1
    q = states(8, batch, heads * d) / 4
    o = torch.full_like(q, 3.0)
    c.attend(q, table, ln, o)
    check(o, q, lens, kb, vb, kv, d, d ** -0.5)
