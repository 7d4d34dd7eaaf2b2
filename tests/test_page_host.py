"""The paged token store on the CPU: refusals come from the host, before any device call; the
storage format's definition against torch's own 8-bit type."""

import ctypes
import os

import pytest
import torch

from tests.page_common import Case, decode_rows, e4m3_grid, encode_rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_31145_amd", "libsekv.so")


@pytest.fixture(scope="module")
def S():
    if not os.path.exists(LIB):
        from paper_2606_31145_amd.build import build
        build()
    from paper_2606_31145_amd import sekv
    return sekv


def _dims(S, **kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=40, max_pages=8,
                dtype="bf16", softmax_scale=0.125)
    base.update(kw)
    return S.make_page_dims(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), 1), (dict(batch=4097), 2), (dict(n_q_heads=0), 1), (dict(n_kv_heads=0), 1),
    (dict(n_q_heads=9), 1), (dict(n_q_heads=6), 2), (dict(n_q_heads=32), 2), (dict(n_q_heads=8192, n_kv_heads=4096), 2),
    (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(page_size=0), 2), (dict(page_size=8), 2), (dict(page_size=24), 2),
    (dict(page_size=2048), 2), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(n_pages=1 << 27), 2),
    (dict(max_pages=(1 << 26) + 1), 2), (dict(dtype=2), 2), (dict(dtype="bf16", page_dtype="f32"), 2),
    (dict(dtype="f32", page_dtype="bf16"), 2), (dict(window=-1), 1), (dict(softmax_scale=0.0), 1),
    (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1), (dict(softmax_scale=1e-40), 2),
    (dict(softmax_scale=1e40), 2),
])
def test_bad_dims_are_refused(S, kw, status):
    d = _dims(S, **kw)
    with pytest.raises(S.SekvError) as ei:
        S.check_page_dims(d)
    assert ei.value.status == status
    with pytest.raises(S.SekvError):
        S.page_workspace_size(d, 4)


def test_reserved_fields_and_counts_are_refused(S):
    d = _dims(S)
    d.reserved[1] = 3
    with pytest.raises(S.SekvError):
        S.check_page_dims(d)
    with pytest.raises(S.SekvError):
        S.page_workspace_size(_dims(S), -1)
    with pytest.raises(S.SekvError):
        S._check(S.LIB.sekv_check_page_dims(None))


@pytest.mark.parametrize("kw", [dict(), dict(dtype="f32"), dict(page_dtype="e4m3"), dict(batch=0),
                                dict(page_size=16, n_pages=1000, max_pages=300), dict(page_size=1024)])
def test_good_dims_have_a_workspace(S, kw):
    S.check_page_dims(_dims(S, **kw))
    assert S.page_workspace_size(_dims(S, **kw), 0) >= 256
    assert S.page_workspace_size(_dims(S, **kw), 100) >= 256


OK = 0x100000     # aligned, and never dereferenced: each call below is refused on the host


def _append(S, d, **kw):
    a = dict(pages=S.PagesStruct(OK, OK, None, None, OK, OK), k=OK, v=OK, ks=2 * 64, vs=2 * 64, ts=OK, n=4, ws=OK,
             nb=1 << 20)
    a.update(kw)
    return S.LIB.sekv_page_append(ctypes.byref(d), ctypes.byref(a["pages"]) if a["pages"] else None, a["k"], a["v"],
                                  a["ks"], a["vs"], a["ts"], a["n"], a["ws"], a["nb"], None)


def _read(S, d, **kw):
    a = dict(pages=S.PagesStruct(OK, OK, None, None, OK, OK), k=OK, v=OK, n=4, ws=OK, nb=1 << 20)
    a.update(kw)
    return S.LIB.sekv_page_read(ctypes.byref(d), ctypes.byref(a["pages"]) if a["pages"] else None, a["k"], a["v"],
                                a["n"], a["ws"], a["nb"], None)


def _attend(S, d, **kw):
    a = dict(pages=S.PagesStruct(OK, OK, None, None, OK, OK), q=OK, qs=8 * 64, ts=OK, n=4, out=OK, lse=OK, ws=OK,
             nb=1 << 30)
    a.update(kw)
    return S.LIB.sekv_page_attend(ctypes.byref(d), ctypes.byref(a["pages"]) if a["pages"] else None, a["q"], a["qs"],
                                  a["ts"], a["n"], a["out"], a["lse"], a["ws"], a["nb"], None)


def _pages(S, **kw):
    f = dict(k=OK, v=OK, k_scale=None, v_scale=None, table=OK, seq_len=OK)
    f.update(kw)
    return S.PagesStruct(f["k"], f["v"], f["k_scale"], f["v_scale"], f["table"], f["seq_len"])


@pytest.mark.parametrize("call", [_append, _read, _attend])
def test_page_arguments_are_refused(S, call):
    d, q = _dims(S), _dims(S, page_dtype="e4m3")
    for kw in (dict(k=None), dict(v=None), dict(table=None), dict(seq_len=None), dict(k=OK + 8), dict(v=OK + 4),
               dict(table=OK + 2), dict(seq_len=OK + 1), dict(k_scale=OK), dict(v_scale=OK)):
        assert call(S, d, pages=_pages(S, **kw)) == S.SEKV_ERR_INVALID_ARG, kw
    for kw in (dict(), dict(k_scale=OK), dict(v_scale=OK), dict(k_scale=OK, v_scale=OK + 8)):
        assert call(S, q, pages=_pages(S, **kw)) == S.SEKV_ERR_INVALID_ARG, kw
    assert call(S, d, pages=None) == S.SEKV_ERR_INVALID_ARG
    assert call(S, d, n=-1) == S.SEKV_ERR_INVALID_ARG
    assert call(S, d, ws=None) == S.SEKV_ERR_WORKSPACE
    assert call(S, d, ws=OK + 128) == S.SEKV_ERR_WORKSPACE
    assert call(S, d, nb=128) == S.SEKV_ERR_WORKSPACE
    assert call(S, _dims(S, head_dim=80)) == S.SEKV_ERR_UNSUPPORTED


def test_row_arguments_are_refused(S):
    d = _dims(S)
    for kw in (dict(k=None), dict(v=None), dict(k=OK + 8), dict(v=OK + 2), dict(ts=None), dict(ts=OK + 2),
               dict(ks=2 * 64 - 8), dict(vs=2 * 64 + 4), dict(ks=0), dict(vs=-128)):
        assert _append(S, d, **kw) == S.SEKV_ERR_INVALID_ARG, kw
    for kw in (dict(k=None), dict(v=None), dict(k=OK + 8), dict(v=OK + 8)):
        assert _read(S, d, **kw) == S.SEKV_ERR_INVALID_ARG, kw
    for kw in (dict(q=None), dict(q=OK + 8), dict(qs=8 * 64 - 8), dict(qs=8 * 64 + 1), dict(ts=None), dict(out=None),
               dict(out=OK + 8), dict(lse=OK + 2)):
        assert _attend(S, d, **kw) == S.SEKV_ERR_INVALID_ARG, kw
    assert _append(S, d, n=(1 << 31) - 1) == S.SEKV_ERR_UNSUPPORTED
    assert _attend(S, d, n=(1 << 31) - 1, nb=1 << 62) == S.SEKV_ERR_UNSUPPORTED


def test_nothing_to_do_is_no_error(S):
    for d in (_dims(S, batch=0), _dims(S)):
        n = 4 if d.batch == 0 else 0
        assert _append(S, d, n=n) == 0 and _read(S, d, n=n) == 0 and _attend(S, d, n=n) == 0


def test_binding_checks_tensors(S):
    """Types, sizes, strides and devices are checked before the library is called."""
    c = Case("bf16", "e4m3", [20, 5], [3, 1])
    pd, cache, ts = c.dims(S), c.cache(S, "cpu"), c.tok_start("cpu")
    with pytest.raises(ValueError, match="GPU"):
        S.page_append(pd, cache, c.k, c.v, ts, None)
    with pytest.raises(ValueError, match="k:"):
        S.page_append(pd, cache, c.k.float(), c.v, ts, None)
    with pytest.raises(ValueError, match="v:"):
        S.page_append(pd, cache, c.k, c.v[:2], ts, None)
    with pytest.raises(ValueError, match="one after another"):
        S.page_append(pd, cache, c.k.transpose(0, 1).contiguous().transpose(0, 1), c.v, ts, None)
    with pytest.raises(ValueError, match="tok_start"):
        S.page_attend(pd, cache, c.q, ts[:2], None)
    with pytest.raises(ValueError, match="tok_start"):
        S.page_attend(pd, cache, c.q, ts.long(), None)
    with pytest.raises(ValueError, match="q:"):
        S.page_attend(pd, cache, c.q[:, :4], ts, None)
    cache.k_scale = None
    with pytest.raises((ValueError, S.SekvError)):
        S.page_read(pd, cache, 4, None)
    cache = c.cache(S, "cpu")
    cache.page_table = cache.page_table[:, :1]
    with pytest.raises(ValueError, match="page_table"):
        S.page_read(pd, cache, 4, None)
    cache = c.cache(S, "cpu")
    cache.k_pages = cache.k_pages.view(torch.uint8)
    with pytest.raises(ValueError, match="k_pages"):
        S.page_read(pd, cache, 4, None)


def test_format_definition_against_torch():
    """The grid is torch's float8_e4m3fn, and encoding by search is its rounding."""
    codes = torch.arange(127, dtype=torch.uint8)
    assert torch.equal(codes.view(torch.float8_e4m3fn).double(), e4m3_grid())
    x = torch.randn(64, 64, generator=torch.Generator().manual_seed(5)) * 3
    c, E = encode_rows(x)
    y = x * torch.pow(2.0, 127.0 - E.float())[:, None]
    assert torch.equal(c, y.to(torch.float8_e4m3fn).view(torch.uint8))
    assert ((y.abs().amax(-1) <= 448) & (y.abs().amax(-1) > 224)).all()
    # half a step: 2^-4 of the value, or 2^-10 of the scale
    err = (decode_rows(c, E) - x.double()).abs()
    assert (err <= torch.maximum(2.0 ** -4 * x.double().abs(),
                                 2.0 ** -10 * torch.pow(2.0, E.double() - 127)[:, None])).all()
