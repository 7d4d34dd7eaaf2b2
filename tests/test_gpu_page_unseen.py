"""Rows of 8-bit pages that a query does not see, with exponent bytes that the store itself never writes
(slots that nobody filled): they do not reach the query."""

import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _case(dtype, news, group, dim, window, lens=(200, 77), page=32):
    """A case whose page 0 is nobody's: it stands in where a block holds no key."""
    c = Case(dtype, "e4m3", list(lens), list(news), group=group, dim=dim, page=page, window=window,
             seed=zlib.crc32(repr((dtype, news, group, dim)).encode()))
    used = set(c.table[c.table < c.n_pages].tolist())
    if 0 in used:
        free = next(p for p in range(c.n_pages) if p not in used)
        c.table[c.table == 0] = free
        for name in "kv":
            for x in (*c.codes[name], c.pools[name]):
                x[[0, free]] = x[[free, 0]]
    return c


def _seen_by_any(c):
    """[n_pages][page]: some query sees the row."""
    seen = torch.zeros((c.n_pages, c.page), dtype=torch.bool)
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        if nq:
            first = max(0, n - nq - c.window + 1) if c.window else 0
            p, s = c.rows(b)
            seen[p[first:], s[first:]] = True
    return seen


def _run(S, c):
    cache, ws = c.cache(S), c.workspace(S)
    out, lse = S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True)
    return out.cpu(), lse.cpu(), ws.status()


SHAPES = [([1, 1], 4, 128), ([6, 3], 4, 64), ([9, 2], 4, 128), ([40, 6], 4, 128), ([150, 33], 1, 128), ([150, 33], 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("exponent,code", [(255, 0), (255, 0x55), (254, 0x7e), (255, 0x7f), (0, 0x7e)])
def test_rows_that_nobody_sees(S, dtype, news, group, dim, window, exponent, code):
    """Every row that no query sees holds the exponent byte and the code: the results are those without it."""
    banner(f"unseen {dtype} {news} {group} {dim} {window} {exponent} {code}")
    c = _case(dtype, news, group, dim, window)
    ref, rl, tol, ltol = c.attend()
    hidden = ~_seen_by_any(c)
    assert hidden[0].all() and hidden.any(1).sum() > 2
    for name in "kv":
        codes, e = c.codes[name]
        codes.masked_fill_(hidden[:, None, :, None], code)
        e.masked_fill_(hidden[:, None], exponent)
    out, lse, status = _run(S, c)
    assert ((out.double() - ref).abs() <= tol).all()
    assert ((lse.double() - rl).abs() <= ltol).all()
    assert status == 0
