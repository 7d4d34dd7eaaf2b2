"""8-bit rows whose values decode past the type, seen by some queries of a tile and not by others: the ones that
do not see them keep their results."""

import math

import pytest
import torch

from tests.gpu_common import banner
from tests.test_gpu_page_unseen import SHAPES, _case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _run(S, c):
    out, lse = S.page_attend(c.dims(S), c.cache(S), c.q.cuda(), c.tok_start(), c.workspace(S), want_lse=True)
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("exponent,code", [(247, 0x78), (247, 0xf8), (250, 0x70), (254, 0x40), (255, 0x38)])
def test_values_that_decode_past_the_type(S, dtype, news, group, dim, exponent, code):
    """A token of the chunk, or one at the edge of some queries' windows, whose values decode to infinity or
    to no number: the queries that do not see it have the results they have without it."""
    lens, window = [200, 77], 60
    for b, t in ((0, lens[0] - 1 - news[0] // 2), (0, lens[0] - news[0] - window + 1), (1, lens[1] - 1)):
        if t < 0:
            continue
        banner(f"overflow {dtype} {news} {group} {dim} {exponent} {code} token {t} of {b}")
        c = _case(dtype, news, group, dim, window)
        ref, rl, tol, ltol = c.attend()
        page, slot = int(c.table[b, t // c.page]), t % c.page
        codes, e = c.codes["v"]
        codes[page, :, slot], e[page, :, slot] = code, exponent
        out, lse = _run(S, c)
        for i in range(c.total):
            sb = 0 if i < c.start[1] else 1
            p = lens[sb] - news[sb] + i - c.start[sb]
            if sb == b and p - window < t <= p:
                assert not torch.isfinite(out[i]).any(), (b, t, i)
            else:
                assert ((out[i].double() - ref[i]).abs() <= tol[i]).all(), (b, t, i)
            assert ((lse[i].double() - rl[i]).abs() <= ltol[i]).all(), (b, t, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
def test_the_largest_values_stored_and_attended(S, dtype, news, group, dim):
    """A token whose values are the type's largest, appended with its chunk: stored as 256 * 2^120, which is
    past the type; the tokens before it do not see it."""
    c = _case(dtype, news, group, dim, 0)
    b, i = 0, news[0] // 2
    cache, ws = c.cache(S), c.workspace(S)
    v = c.v.clone()
    v[c.start[b] + i] = torch.finfo(v.dtype).max
    S.page_append(c.dims(S), cache, c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    want, wl = (x.cpu() for x in S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True))
    S.page_append(c.dims(S), cache, c.k.cuda(), v.cuda(), c.tok_start(), ws)
    out, lse = (x.cpu() for x in S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True))
    # both results lie within the plain form's bound of the stored rows, so within twice it of each other
    for name in "kv":
        pool, scale = (cache.k_pages, cache.k_scale) if name == "k" else (cache.v_pages, cache.v_scale)
        c.pools[name] = pool.cpu().double() * 2.0 ** (scale.cpu().double() - 127)[..., None]
        c.pools[name].clamp_(-1e4, 1e4)                      # the large token's rows: their queries are not compared
    _, _, tol, ltol = c.attend()
    sees = torch.zeros(c.total, dtype=torch.bool)
    sees[c.start[b] + i:c.start[b + 1]] = True
    assert not torch.isfinite(out[sees]).any()
    assert ((out.double() - want.double()).abs() <= 2 * tol)[~sees].all()
    assert ((lse.double() - wl.double()).abs() <= 2 * ltol).all()
    assert torch.isfinite(want).all() and ws.status() == 0 and math.isfinite(float(wl.sum()))
