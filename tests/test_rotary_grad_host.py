"""Refusals of sekv.rotate where a gradient would be lost, before any device call."""

import os

import pytest
import torch

from tests.rotary_common import frequencies

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_31145_amd", "libsekv.so")


@pytest.fixture(scope="module")
def S():
    if not os.path.exists(LIB):
        from paper_2606_31145_amd.build import build
        build()
    from paper_2606_31145_amd import sekv
    return sekv


def test_out_is_refused_where_it_would_lose_a_gradient(S):
    r, pos = S.Rotary(frequencies(64)), torch.arange(4, dtype=torch.int32)
    x = torch.randn(4, 2, 64)
    leaf = x.clone().requires_grad_()
    for a, out in ((leaf, x), (x, leaf), (leaf, leaf)):
        with pytest.raises(ValueError, match="out: no gradient"):
            S.rotate(a, pos, r, out=out)
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            S.rotate(a, pos, r, out=out)
    with pytest.raises(ValueError, match="GPU"):
        S.rotate(leaf, pos, r)
