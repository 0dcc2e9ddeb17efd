"""Which of packed attention's kernels a call takes, for tests that are meant for one of them (tests/test_attn_kernels.py holds this to the library's
launches)."""


def few(heads: int, d: int, batch: int, rows: int, causal: bool) -> bool:
    """Forward and dq: 32 rows a workgroup, whose wavefronts deal the keys among them, instead of 128."""
    most = (160 if causal else 72) if d > 64 else (256 if causal else 128)
    return (rows // 128 + batch) * heads <= most and rows >= 128 * batch


def workgroups(heads: int, d: int, batch: int, rows: int, causal: bool) -> int:
    return (rows // (32 if few(heads, d, batch, rows, causal) else 128) + batch) * heads
