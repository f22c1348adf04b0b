"""Sizes and pointers that the rollout-side entry points refuse before anything is launched (CPU)."""
from test_rollout_host_logic import _product, _quantize, _sample, binding  # noqa: F401


def test_sizes_beyond_the_documented_limits(binding):  # noqa: F811
    B = binding
    assert _sample(B, V=2 ** 30 + 1, ld=2 ** 31) == -2 and _sample(B, T=0, V=2 ** 30, ld=2 ** 30) == 0
    for name, stride in (("M", {}), ("N", {"ldc": 2 ** 31}), ("K", {"lda": 2 ** 31, "ldb": 2 ** 31})):
        assert _product(B, **{name: 2 ** 30 + 1}, **stride) == -2
    # tiles of 128 columns and 16 rows (128 with the transposed form) count in 31 bits
    assert _quantize(B, rows=2 ** 36, cols=1, ld=1, ldq=1, sk=2 ** 36) == -2
    assert _quantize(B, rows=2 ** 38, cols=1, ld=1, q=None, qt=0x60000, st=0x70000, ldqt=2 ** 38) == -2


def test_words_off_their_alignment(binding):  # noqa: F811
    B = binding
    for name in ("tau", "k", "p", "m", "ids", "lp", "status"):
        assert _sample(B, **{name: 0x60002}) == -7
    assert _sample(B, K=4, ti=0x60002, tp=0x70000) == -7 and _sample(B, K=4, ti=0x60000, tp=0x70001) == -7
    assert _quantize(B, status=0x50002) == -7 and _product(B, status=0x60002) == -7
