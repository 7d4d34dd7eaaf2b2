"""Tables that cannot be, in the calls that store and read: wrong answers are allowed, silence is not."""

import pytest
import torch

from tests.page_common import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


@pytest.mark.parametrize("store", ["same", "e4m3"])
@pytest.mark.parametrize("start", [[0, 2, 1, 3], [0, 1, 2, 9], [2, 1, 0, 0], [-1, 1, 2, 3], [0, 3, 1, 1], [4, 4, 4, 4]])
def test_append_flags_wrong_offsets(S, store, start):
    c = Case("bf16", store, [90, 30, 77], [1, 1, 1], dim=64, page=16, seed=1)
    cache, ws = c.cache(S), c.workspace(S)
    ts = torch.tensor(start, dtype=torch.int32, device="cuda")
    S.page_append(c.dims(S), cache, c.k.cuda(), c.v.cuda(), ts, ws)
    assert ws.status() == 8
    S.page_append(c.dims(S), cache, c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    assert ws.status() == 0


def test_append_flags_wrong_offsets_of_many_sequences(S):
    n = 700
    c = Case("bf16", "e4m3", [20] * n, [1] * n, dim=64, page=16, kv_heads=1, group=1, seed=2)
    cache, ws, k, v = c.cache(S), c.workspace(S), c.k.cuda(), c.v.cuda()
    S.page_append(c.dims(S), cache, k, v, c.tok_start(), ws)
    assert ws.status() == 0
    ts = c.tok_start()
    ts[613] = 100
    S.page_append(c.dims(S), cache, k, v, ts, ws)
    assert ws.status() == 8


def test_offsets_may_leave_rows_out_on_both_sides(S):
    """Rows before the first sequence's and behind the last one's are nobody's: not stored, not flagged."""
    c = Case("bf16", "same", [9, 5], [3, 2], dim=64, page=16, seed=3)
    cache, ws = c.cache(S), S.Workspace(None, "cuda", nbytes=S.page_workspace_size(c.dims(S), c.total + 3))
    k, v = (torch.cat([torch.full_like(x[:2], 7.0), x, torch.full_like(x[:1], 7.0)]).cuda() for x in (c.k, c.v))
    S.page_append(c.dims(S), cache, k, v, c.tok_start() + 2, ws)
    other = c.cache(S)
    S.page_append(c.dims(S), other, c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    assert torch.equal(cache.k_pages, other.k_pages) and torch.equal(cache.v_pages, other.v_pages)
    q = torch.cat([torch.zeros_like(c.q[:2]), c.q, torch.zeros_like(c.q[:1])]).cuda()
    out = torch.full_like(q, -3.0)
    S.page_attend(c.dims(S), cache, q, c.tok_start() + 2, ws, out=out)
    want, _ = S.page_attend(c.dims(S), other, c.q.cuda(), c.tok_start(), ws)
    assert torch.equal(out[2:-1], want) and (out[:2] == -3.0).all() and (out[-1:] == -3.0).all()
    assert ws.status() == 0


@pytest.mark.parametrize("store", ["same", "e4m3"])
def test_read_flags_a_negative_length(S, store):
    c = Case("bf16", store, [40, 20], [0, 0], dim=64, page=16)
    cache, ws = c.cache(S), c.workspace(S)
    want, _ = S.page_read(c.dims(S), cache, 48, ws)
    assert ws.status() == 0
    cache.seq_len[0] = -1
    keys, _ = S.page_read(c.dims(S), cache, 48, ws)
    assert ws.status() == 8 and not keys[0].any() and torch.equal(keys[1], want[1])
