"""A base that stretching takes past the largest double."""

import math
import os

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_31145_amd", "libsekv.so")


@pytest.fixture(scope="module")
def S():
    if not os.path.exists(LIB):
        from paper_2606_31145_amd.build import build
        build()
    from paper_2606_31145_amd import sekv
    return sekv


@pytest.mark.parametrize("R,base,factor", [(4, 10.0, 1e160), (64, 1e300, 1e10), (4096, 1.7e308, 2.0)])
def test_a_base_past_the_largest_double_is_refused(S, R, base, factor):
    with pytest.raises(S.SekvError) as ei:
        S.rotary_frequencies(R, base, "base", factor=factor)
    assert ei.value.status == S.SEKV_ERR_UNSUPPORTED


def test_a_base_just_below_it(S):
    f, _ = S.rotary_frequencies(64, 1e300, "base", factor=1e7)
    want = [1e300 ** (-2 * i / 64) * 1e7 ** (-2 * i / 62) for i in range(32)]
    assert all(math.isclose(a, b, rel_tol=1e-12) for a, b in zip(f.tolist(), want))
