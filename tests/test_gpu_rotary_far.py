"""Angles at the end of what a double can hold: turned as ever up to 2^50 quarter turns, no number from there on."""

import math

import pytest
import torch

from tests.page4_common import Case4
from tests.rotary_common import bound, turned

pytestmark = pytest.mark.gpu

LIMIT = 2.0 ** 50 * math.pi / 2
POS = torch.tensor([2 ** 30, -2 ** 30, 1, -1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_angles_up_to_the_limit_and_past_it(S, layout, dtype):
    """Frequencies so that one position's angles lie on both sides of the limit; a step of the quotient beside it counts
    to either."""
    near = LIMIT / 2.0 ** 30
    f = torch.tensor([near * x for x in (2.0 ** -20, 0.001, 0.1, 0.4, 0.49, 0.9, 0.999, 1.001)] +
                     [1.1 * near, 1e7, 1e9, 1e17, 2.1e19, 1e300, math.inf, math.nan], dtype=torch.float64)
    x = torch.randn((len(POS), 3, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    got = S.rotate(x.cuda(), POS.cuda(), S.Rotary(f.cuda(), layout=layout)).cpu()
    far = ~((POS.double()[:, None] * f).abs() < LIMIT)                      # [tokens][pairs]
    assert far[2].tolist() == [False] * 11 + [True] * 5 and 0 < far[0].sum() < 16
    R = 32
    pair = torch.cat((far, far), -1) if layout == "half" else far.repeat_interleave(2, -1)
    pair = torch.cat((pair, torch.zeros(len(POS), 64 - R, dtype=torch.bool)), -1)[:, None].expand_as(got)
    assert torch.equal(got.isnan(), pair)
    want = turned(x, POS, f, layout)
    tol = bound(x, want.nan_to_num(), dtype)
    assert ((got.double() - want).abs() <= tol)[~pair].all()


def test_a_key_turned_too_far_is_stored_as_no_number(S):
    c = Case4("bf16", [6], [6], dim=64, kv_heads=1, group=1)
    f = torch.full((32,), 1e-3, dtype=torch.float64)
    f[20] = 1e18                                                            # pairs of both blocks of a row
    cache = c.cache(S)
    S.page_append_rotary(c.dims(S), cache, S.Rotary(f.cuda()), None, c.k.cuda(), c.v.cuda(), c.tok_start(), c.workspace(S))
    E = cache.k_scale.cpu()[int(c.table[0, 0]), 0, :6]
    assert (E[0] != 255).all() and (E[1:] == 255).all()                     # position 0 has no angle
    assert torch.equal(cache.v_scale.cpu(), c.stored(c.k, c.v)["v"][1])
