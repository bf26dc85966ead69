"""Frequencies of rotary positions for longer contexts against their formulas in Python's own floating point numbers."""
import math

import numpy as np
import pytest

from paper_2602_00294_amd import _binding as bnd


@pytest.mark.parametrize("pairs,base,original,factor", [(64, 1e4, 4096.0, 16.0), (64, 5e5, 8192.0, 8.0), (20, 1e4, 4096.0, 8.0),
                                                        (1, 1e4, 100.0, 4.0), (33, 1e6, 1.0, 2.0), (8, 2.0, 1e6, 1.0)])
def test_by_turns_in_between(pairs, base, original, factor):
    """32 turns and more in `original` tokens as they are, one and fewer divided by the factor, and in between the
    share (turns - 1) / 31 of the first and the rest of the second, each rounded to float32 once."""
    f, s = bnd.rotary_frequencies(pairs, base, "by_turns", factor, original, device="cpu")
    want = []
    for i in range(pairs):
        x = base ** (-i / pairs)
        keep = min(1.0, max(0.0, (original * x / (2.0 * math.pi) - 1.0) / 31.0))
        want.append(keep * x + (1.0 - keep) * x / factor)
    assert np.allclose(f.numpy(), want, rtol=2.0 ** -24 * (1 + 1e-6), atol=0.0)
    assert math.isclose(s, 0.1 * math.log(factor) + 1.0, rel_tol=2.0 ** -24)


def test_a_scaled_base_that_is_no_number_is_refused():
    """base * factor^(pairs / (pairs - 1)) beyond 64 bits would leave all pairs but the first unturned."""
    with pytest.raises(bnd.SataError):
        bnd.rotary_frequencies(64, 1e300, "base", 1e300, device="cpu")
    with pytest.raises(bnd.SataError):
        bnd.rotary_frequencies(2, 1e10, "base", 1e200, device="cpu")


def test_too_many_pairs_take_no_memory():
    import tracemalloc
    tracemalloc.start()
    with pytest.raises(bnd.SataError):
        bnd.rotary_frequencies(1 << 24, device="cpu")
    peak = tracemalloc.get_traced_memory()[1]
    tracemalloc.stop()
    assert peak < 1 << 20
