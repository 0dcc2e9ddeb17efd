"""CPU-only checks of runtime's layers over the backbone's blocks: what is refused before a device is asked for."""
import pytest

torch = pytest.importorskip("torch")
from paper_2408_10746_amd import runtime as rt  # noqa: E402


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 256])
def test_sizes_past_32_bits_are_refused_not_cut_off(n):
    codes, scales = rt.mx4_empty(2, 256, "cpu")
    x = torch.zeros(1).expand(2, n)
    for bad in (lambda: rt.mx4_empty(2, n, "cpu"), lambda: rt.BlockNorm(n), lambda: rt._stored(codes, scales, 2, n, codes.device),
                lambda: rt.mx4_quantize(x, codes, scales), lambda: rt.mx4_dequantize(codes, scales, x)):
        with pytest.raises(ValueError):
            bad()
