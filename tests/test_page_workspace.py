"""The paged store's calls refuse a workspace that is not on the pages' device: the kernels write to it."""

from types import SimpleNamespace

import pytest
import torch

from tests.page_common import Case


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _ws(device):
    t = torch.empty(1 << 20, dtype=torch.uint8, device=device)
    return SimpleNamespace(tensor=t, ptr=t.data_ptr(), nbytes=t.numel())


def test_a_workspace_elsewhere_is_refused(S):
    with pytest.raises(ValueError, match="workspace is on meta"):
        S._page_ws(_ws("meta"), torch.device("cpu"))
    ws = _ws("cpu")
    assert S._page_ws(ws, torch.device("cpu")) == (ws.ptr, ws.nbytes)


@pytest.mark.gpu
def test_every_call_refuses_it(S):
    c = Case("bf16", "e4m3", [20, 5], [3, 1])
    pd, cache, ts, ws = c.dims(S), c.cache(S), c.tok_start(), _ws("cpu")
    for call in (lambda: S.page_append(pd, cache, c.k.cuda(), c.v.cuda(), ts, ws),
                 lambda: S.page_attend(pd, cache, c.q.cuda(), ts, ws), lambda: S.page_read(pd, cache, 20, ws)):
        with pytest.raises(ValueError, match="workspace is on cpu"):
            call()
