"""CPU-only checks of runtime's layers over attention and the 4-bit cache: what is refused before a device is asked for."""
import pytest

torch = pytest.importorskip("torch")
from paper_2408_10746_amd import runtime as rt  # noqa: E402


def test_offsets():
    assert rt.packed_offsets([3, 0, 5], "cpu").tolist() == [0, 3, 3, 8] and rt.packed_offsets([], "cpu").tolist() == [0]
    for bad in ([3, -1], [1 << 30, 1 << 30]):
        with pytest.raises(ValueError):
            rt.packed_offsets(bad, "cpu")


@pytest.mark.parametrize("kw", [dict(heads=0), dict(d=0), dict(d=12), dict(d=136), dict(kv_heads=3), dict(kv_heads=0), dict(scale=0.0), dict(scale=float("nan")),
                                dict(heads=1 << 32), dict(d=1 << 33)])
def test_attentions_that_are_refused(kw):
    with pytest.raises(ValueError):
        rt.Attention(**dict(dict(heads=4, d=64, kv_heads=2), **kw))


def test_attention_on_the_host_is_refused():
    a, x = rt.Attention(2, 8), torch.zeros(3, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        a.forward(x, x, x, rt.packed_offsets([3], "cpu"), x)
    with pytest.raises(ValueError):
        a.backward(x, x, x, rt.packed_offsets([3], "cpu"), x, torch.zeros(2, 3), x, x, x, x)


@pytest.mark.parametrize("args", [(-1, 16, 2, 64), (1 << 31, 16, 2, 64), (4, 0, 2, 64), (4, 12, 2, 64), (4, 1 << 17, 2, 64), (4, 16, 0, 64), (4, 16, 2, 60), (4, 16, 2, 136),
                                  (4, 1 << 32, 2, 64), (4, 16, 2, 64)])
def test_caches_that_are_refused(args):
    """Sizes, and memory that is not a GPU's (the last)."""
    with pytest.raises(ValueError):
        rt.Kv4Cache(*args, device="cpu")


def test_a_scale_past_what_scores_are_taken_times_is_refused():
    rt.Attention(4, 64, scale=2.35e38)
    with pytest.raises(ValueError):
        rt.Attention(4, 64, scale=2.36e38)


@pytest.mark.parametrize("kw", [dict(heads=4 - (1 << 32)), dict(kv_heads=2 - (1 << 32)), dict(d=64 - (1 << 32))])
def test_sizes_that_32_bits_would_turn_into_others_are_refused(kw):
    with pytest.raises(ValueError):
        rt.Attention(**dict(dict(heads=4, d=64, kv_heads=2), **kw))


@pytest.mark.parametrize("name,args", [("pages", ((1 << 64) + 4, 16, 2, 64)), ("pages", (4 - (1 << 64), 16, 2, 64)), ("page", (4, 16 - (1 << 32), 2, 64)),
                                       ("kv_heads", (4, 16, 2 - (1 << 32), 64)), ("d", (4, 16, 2, 64 - (1 << 32)))])
def test_cache_sizes_that_fewer_bits_would_turn_into_others_are_refused(name, args):
    with pytest.raises(ValueError, match=f"^{name}: {args[('pages', 'page', 'kv_heads', 'd').index(name)]} is "):
        rt.Kv4Cache(*args, device="cpu")
