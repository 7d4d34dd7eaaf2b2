"""Rotary positions on the CPU: frequencies against their formulas, and refusals before any device call."""

import ctypes
import math
import os

import pytest
import torch

from tests.page4_common import Case4
from tests.rotary_common import frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_31145_amd", "libsekv.so")


@pytest.fixture(scope="module")
def S():
    if not os.path.exists(LIB):
        from paper_2606_31145_amd.build import build
        build()
    from paper_2606_31145_amd import sekv
    return sekv


# a power and a handful of products in double
TOL = 1e-13


@pytest.mark.parametrize("R,base", [(2, 10.0), (16, 10000.0), (48, 10000.0), (128, 500000.0), (4096, 1.5)])
def test_plain_and_linear(S, R, base):
    f, scale = S.rotary_frequencies(R, base)
    want = frequencies(R, base)
    assert f.dtype == torch.float64 and scale == 1.0
    assert torch.allclose(f, want, rtol=TOL, atol=0)
    f, scale = S.rotary_frequencies(R, base, "linear", factor=8.0)
    assert scale == 1.0 and torch.allclose(f, want / 8, rtol=TOL, atol=0)


@pytest.mark.parametrize("R", [4, 64, 128])
def test_base(S, R):
    """The first pair stays, the last one's frequency is divided by the factor, the others lie on one power."""
    f, scale = S.rotary_frequencies(R, 10000.0, "base", factor=4.0)
    want = frequencies(R, 10000.0)
    assert scale == 1.0 and f[0] == 1.0
    assert abs(f[-1] * 4.0 / want[-1] - 1) < 1e-12
    ratio = f[1:] / f[:-1]
    assert torch.allclose(ratio, ratio[:1].expand_as(ratio), rtol=1e-12, atol=0)


def test_bands(S):
    R, base, factor, trained, low, high = 128, 500000.0, 8.0, 8192.0, 1.0, 4.0
    f, scale = S.rotary_frequencies(R, base, "bands", factor=factor, trained=trained, low=low, high=high)
    assert scale == 1.0
    kinds = set()
    for got, f0 in zip(f.tolist(), frequencies(R, base).tolist()):
        turns = trained * f0 / (2 * math.pi)
        if turns > high:
            want = f0
            kinds.add("kept")
        elif turns < low:
            want = f0 / factor
            kinds.add("stretched")
        else:
            t = (turns - low) / (high - low)
            want = (1 - t) * f0 / factor + t * f0
            kinds.add("mixed")
        assert abs(got / want - 1) < 1e-11
    assert kinds == {"kept", "stretched", "mixed"}


@pytest.mark.parametrize("factor", [1.0, 4.0, 40.0])
def test_ramp(S, factor):
    R, base, trained, low, high = 64, 10000.0, 4096.0, 1.0, 32.0
    f, scale = S.rotary_frequencies(R, base, "ramp", factor=factor, trained=trained, low=low, high=high)
    assert abs(scale - (0.1 * math.log(factor) + 1)) < 1e-15
    pair = lambda turns: R * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))    # noqa: E731
    lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), R - 1)
    for i, (got, f0) in enumerate(zip(f.tolist(), frequencies(R, base).tolist())):
        t = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert abs(got / ((1 - t) * f0 + t * f0 / factor) - 1) < 1e-11
    assert f[0] == 1.0


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=4098), dict(base=1.0),
                                dict(base=math.inf), dict(base=math.nan), dict(scaling="linear", factor=0.5),
                                dict(scaling="base", factor=math.nan), dict(scaling="base", rot_dim=2, factor=2.0),
                                dict(scaling="bands", factor=2.0), dict(scaling="ramp", factor=2.0, trained=-1.0),
                                dict(scaling="bands", factor=2.0, trained=100.0, low=4.0, high=4.0),
                                dict(scaling="ramp", factor=2.0, trained=100.0, low=0.0)])
def test_frequencies_are_refused(S, kw):
    a = dict(rot_dim=64, base=10000.0)
    a.update(kw)
    with pytest.raises(S.SekvError):
        S.rotary_frequencies(**a)


def test_null_pointers_of_frequencies(S):
    spec, scale = S.RotarySpec(16, 0, 10.0, 1.0, 0.0, 1.0, 2.0), ctypes.c_double()
    assert S.LIB.sekv_rotary_frequencies(None, OK, ctypes.byref(scale)) == S.SEKV_ERR_INVALID_ARG
    assert S.LIB.sekv_rotary_frequencies(ctypes.byref(spec), None, ctypes.byref(scale)) == S.SEKV_ERR_INVALID_ARG
    assert S.LIB.sekv_rotary_frequencies(ctypes.byref(spec), OK, None) == S.SEKV_ERR_INVALID_ARG
    spec.scaling = 5
    assert S.LIB.sekv_rotary_frequencies(ctypes.byref(spec), OK, ctypes.byref(scale)) == S.SEKV_ERR_INVALID_ARG
    with pytest.raises(KeyError):
        S.rotary_frequencies(16, 10.0, "other")


OK = 0x100000     # aligned, and never dereferenced: each call below is refused on the host


def _rotary(S, **kw):
    a = dict(rot_dim=64, layout=0, freq=OK, scale=1.0)
    a.update(kw)
    return S.RotaryStruct(a["rot_dim"], a["layout"], a["freq"], a["scale"])


BAD_ROTARY = [(dict(rot_dim=0), 2), (dict(rot_dim=8), 2), (dict(rot_dim=24), 2), (dict(rot_dim=80), 2), (dict(rot_dim=-16), 2),
              (dict(layout=2), 1), (dict(layout=-1), 1), (dict(freq=None), 1), (dict(freq=OK + 4), 1), (dict(scale=0.0), 1),
              (dict(scale=-1.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1), (dict(scale=1e-31), 2),
              (dict(scale=1e31), 2)]


def _rotate(S, **kw):
    a = dict(r=_rotary(S), n=4, heads=8, d=64, dt=1, x=OK, xs=512, y=OK + (1 << 20), ys=512, p=OK, t=0)
    a.update(kw)
    return S.LIB.sekv_rotate(a["r"], a["n"], a["heads"], a["d"], a["dt"], a["x"], a["xs"], a["y"], a["ys"], a["p"], a["t"], None)


def _append(S, **kw):
    d = S.make_page_dims(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=40, max_pages=8,
                         dtype="bf16", page_dtype="e2m1", softmax_scale=0.125)
    a = dict(d=d, pages=S.PagesStruct(OK, OK, OK, OK, OK, OK), r=_rotary(S), q=OK, qs=512, o=OK + (1 << 20), os=512, k=OK,
             v=OK, ks=128, vs=128, p=None, ts=OK, n=4, ws=OK, nb=256)
    a.update(kw)
    return S.LIB.sekv_page_append_rotary(a["d"], a["pages"], a["r"], a["q"], a["qs"], a["o"], a["os"], a["k"], a["v"],
                                         a["ks"], a["vs"], a["p"], a["ts"], a["n"], a["ws"], a["nb"], None)


@pytest.mark.parametrize("kw,status", BAD_ROTARY)
def test_rotary_is_refused(S, kw, status):
    assert _rotate(S, r=_rotary(S, **kw)) == status
    assert _append(S, r=_rotary(S, **kw)) == status


def test_rotate_arguments_are_refused(S):
    for kw in (dict(r=None), dict(n=-1), dict(heads=0), dict(x=None), dict(y=None), dict(x=OK + 8), dict(y=OK + 4),
               dict(xs=504), dict(ys=516), dict(xs=0), dict(ys=-512), dict(p=None), dict(p=OK + 2), dict(t=2), dict(t=-1),
               dict(y=OK, ys=1024)):
        assert _rotate(S, **kw) == S.SEKV_ERR_INVALID_ARG, kw
    for kw in (dict(d=96), dict(d=32), dict(dt=2), dict(dt=3), dict(heads=4097)):
        assert _rotate(S, **kw) == S.SEKV_ERR_UNSUPPORTED, kw
    assert _rotate(S, n=0) == S.SEKV_OK and _rotate(S, n=0, x=None, y=None, p=None) == S.SEKV_OK


def test_append_arguments_are_refused(S):
    for kw in (dict(d=None), dict(pages=None), dict(r=None), dict(q=None), dict(o=None), dict(q=OK + 8), dict(o=OK + 8), dict(qs=504),
               dict(os=516), dict(o=OK, os=1024), dict(k=None), dict(v=None), dict(k=OK + 8), dict(ks=120), dict(vs=132),
               dict(p=OK + 1), dict(ts=None), dict(ts=OK + 2), dict(n=-1)):
        assert _append(S, **kw) == S.SEKV_ERR_INVALID_ARG, kw
    for kw in (dict(ws=None), dict(ws=OK + 128), dict(nb=255)):
        assert _append(S, **kw) == S.SEKV_ERR_WORKSPACE, kw
    assert _append(S, n=(1 << 31) - 1) == S.SEKV_ERR_UNSUPPORTED
    assert _append(S, n=0) == S.SEKV_OK


def test_binding_checks_tensors(S):
    c = Case4("bf16", [20, 5], [3, 1])
    pd, cache, ts = c.dims(S), c.cache(S, "cpu"), c.tok_start("cpu")
    r, pos = S.Rotary(frequencies(64)), torch.arange(4, dtype=torch.int32)
    assert r.rot_dim == 64
    with pytest.raises(AttributeError):
        r.freq = frequencies(64)                         # the C view holds the address of the one it was made of
    for bad in (frequencies(64).float(), frequencies(64)[None], [1.0]):
        with pytest.raises(ValueError, match="freq"):
            S.Rotary(bad)
    with pytest.raises(KeyError):
        S.Rotary(frequencies(64), "other")
    with pytest.raises(ValueError, match="GPU"):
        S.rotate(c.q, pos, r)
    with pytest.raises(ValueError, match="positions"):
        S.rotate(c.q, pos[:3], r)
    with pytest.raises(ValueError, match="positions"):
        S.rotate(c.q, pos.long(), r)
    with pytest.raises(ValueError, match="positions"):
        S.rotate(c.q, None, r)
    for bad in (c.q.half(), c.q[0], c.q.tolist()):
        with pytest.raises(ValueError, match="x:"):
            S.rotate(bad, pos, r)
    with pytest.raises(ValueError, match="one after another"):
        S.rotate(c.q.transpose(0, 1).contiguous().transpose(0, 1), pos, r)
    with pytest.raises(ValueError, match="GPU"):
        S.page_append_rotary(pd, cache, r, c.q, c.k, c.v, ts, None)
    for kw, match in ((dict(k=c.k.float()), "k:"), (dict(v=c.v[:2]), "v:"), (dict(q=c.q[:, :4]), "q:"),
                      (dict(positions=pos[:2]), "positions"), (dict(q=None, q_out=c.q), "q_out"),
                      (dict(tok_start=ts[:2]), "tok_start")):
        a = dict(q=c.q, k=c.k, v=c.v, tok_start=ts)
        a.update(kw)
        with pytest.raises(ValueError, match=match):
            S.page_append_rotary(pd, cache, r, ws=None, **a)
    for name in "qkv":                                   # no tensor, and one of other dimensions
        for bad, error in ((getattr(c, name).tolist(), TypeError), (getattr(c, name)[0], ValueError)):
            a = dict(q=c.q, k=c.k, v=c.v, tok_start=ts)
            a[name] = bad
            with pytest.raises(error, match=f"{name}:"):
                S.page_append_rotary(pd, cache, r, ws=None, **a)
    cache.page_table = None
    with pytest.raises(TypeError, match="page_table"):
        S.page_append_rotary(pd, cache, r, c.q, c.k, c.v, ts, None)
