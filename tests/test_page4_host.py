"""4-bit pages on the CPU: refusals, and the format's definition."""

import ctypes
import os

import pytest
import torch

from tests.page4_common import Case4, decode4, encode4, two

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_31145_amd", "libsekv.so")


@pytest.fixture(scope="module")
def S():
    if not os.path.exists(LIB):
        from paper_2606_31145_amd.build import build
        build()
    from paper_2606_31145_amd import sekv
    return sekv


OK = 0x100000     # aligned, and never dereferenced: each call below is refused on the host


def _dims(S, **kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=40, max_pages=8,
                dtype="bf16", page_dtype="e2m1", softmax_scale=0.125)
    base.update(kw)
    return S.make_page_dims(**base)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_dims_are_taken(S, dtype, dim):
    S.check_page_dims(_dims(S, dtype=dtype, head_dim=dim))
    assert S.page_workspace_size(_dims(S, dtype=dtype, head_dim=dim), 9) > 256


def test_pages_are_refused(S):
    d = _dims(S)
    for ks, vs in ((None, None), (OK, None), (None, OK), (OK + 4, OK), (OK, OK + 8)):
        p = S.PagesStruct(OK, OK, ks, vs, OK, OK)
        assert S.LIB.sekv_page_append(d, p, OK, OK, 128, 128, OK, 4, OK, 1 << 20, None) == S.SEKV_ERR_INVALID_ARG
        assert S.LIB.sekv_page_read(d, p, OK, OK, 4, OK, 1 << 20, None) == S.SEKV_ERR_INVALID_ARG
        assert S.LIB.sekv_page_attend(d, p, OK, 512, OK, 4, OK, None, OK, 1 << 30, None) == S.SEKV_ERR_INVALID_ARG
    for dt in (4, -1, 77):
        with pytest.raises(S.SekvError) as ei:
            S.check_page_dims(_dims(S, page_dtype=dt))
        assert ei.value.status == S.SEKV_ERR_UNSUPPORTED
    with pytest.raises(S.SekvError):
        S.check_page_dims(_dims(S, dtype=3, page_dtype=3))          # tokens are never 4-bit
    assert ctypes.sizeof(S.PagesStruct) == 48


def test_binding_checks_tensors(S):
    c = Case4("bf16", [20, 5], [3, 1])
    pd, ts = c.dims(S), c.tok_start("cpu")
    cache = c.cache(S, "cpu")
    with pytest.raises(ValueError, match="GPU"):
        S.page_append(pd, cache, c.k, c.v, ts, None)
    for name, bad in (("k_pages", cache.k_pages[..., :16]), ("v_pages", cache.v_pages.view(torch.int8)),
                      ("k_scale", cache.k_scale[..., 0]), ("v_scale", cache.v_scale.to(torch.int32))):
        other = c.cache(S, "cpu")
        setattr(other, name, bad)
        with pytest.raises(ValueError, match=name):
            S.page_read(pd, other, 4, None)
    cache.k_scale = None
    with pytest.raises((ValueError, S.SekvError)):
        S.page_read(pd, cache, 4, None)
    e = S.PageCache.empty(pd, c.table, torch.tensor(c.lens, dtype=torch.int32), "cpu")
    assert e.k_pages.shape == (c.n_pages, 2, 16, 32) and e.v_scale.shape == (c.n_pages, 2, 16, 2)
    assert e.k_pages.dtype == torch.uint8 and (e.k_scale == 127).all()
    e.struct(pd)


def test_format_definition():
    """Half a step at most, the smallest exponent, ties to the even code, zeros' signs, blocks apart."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(200, 64, generator=g) * torch.exp(4 * torch.randn(200, 1, generator=g))
    c, E = encode4(x)
    y, s = decode4(c, E), two(E.long() - 127).repeat_interleave(32, -1)
    err, u = (y - x.double()).abs() / s, (x.double() / s).abs()
    step = torch.where(u < 2, 0.5, torch.where(u < 4, 1.0, 2.0))
    assert (err <= step / 2).all()
    top = u.unflatten(-1, (-1, 32)).amax(-1)
    assert ((top <= 6) & (top > 3)).all()
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4)
    want = torch.tensor([0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0] * 4).double()
    assert torch.equal(decode4(*encode4(ties[None]))[0], want)
    z = torch.zeros(1, 64)
    z[0, 1] = -0.0
    z[0, 40] = float("nan")
    c, E = encode4(z)
    assert c[0, 0] == 0x80 and E.tolist() == [[127, 255]]
    assert encode4(torch.full((1, 32), 3.4e38))[1].item() == 252
    assert (decode4(*encode4(torch.full((1, 32), -3.4e38))) == -6 * 2.0 ** 125).all()
    assert encode4(torch.full((1, 32), 1e-40))[1].item() == 2
