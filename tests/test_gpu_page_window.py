"""Page-table entries that lie before every window: a server takes such pages back, so they are neither
read nor flagged, and what the pages hold by then does not matter."""

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


STORES = [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")]


@pytest.mark.parametrize("dtype,store", STORES)
@pytest.mark.parametrize("entry", [-1, 2 ** 31 - 1])
@pytest.mark.parametrize("lens,news,window,group,page,kv_heads", [
    ([200, 130], [1, 1], 100, 4, 16, 2),               # first visible keys 100 and 30: inside a step of 64 keys
    ([200, 130], [12, 5], 100, 4, 16, 2),              # narrow tiles, two for one sequence
    ([700, 301], [150, 40], 100, 2, 16, 2),            # tiles of 128 rows
    ([700], [150], 37, 8, 32, 1),                      # several of them, each with a first key of its own
    ([1111, 63], [1, 1], 17, 1, 16, 3),
    ([5000], [6], 2048, 8, 64, 1),                     # a window that is cut into chunks
])
def test_pages_behind_the_window_were_taken_back(S, dtype, store, entry, lens, news, window, group, page, kv_heads):
    banner(f"window {dtype} {store} {entry} {lens} {news} {window}")
    c = Case(dtype, store, lens, news, window=window, group=group, page=page, kv_heads=kv_heads, dim=128,
             seed=zlib.crc32(repr((dtype, store, lens, news)).encode()))
    ref, rl, tol, ltol = c.attend()
    gone = 0
    for b, (n, nq) in enumerate(zip(lens, news)):
        first = max(0, n - nq - window + 1)              # the first key that a query of the sequence sees
        c.table[b, :first // page] = entry
        gone += first // page
    assert gone
    cache, ws = c.cache(S), c.workspace(S)
    out, lse = S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True)
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    assert ((lse.cpu().double() - rl).abs() <= ltol).all()
    assert ws.status() == 0
    # the page of the first visible key itself is needed
    b = max(range(len(lens)), key=lambda i: lens[i] - news[i])
    at = (lens[b] - news[b] - window + 1) // page
    cache.page_table[b, at] = -1
    S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws)
    assert ws.status() == 8
