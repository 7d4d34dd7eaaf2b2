"""build_layer_paged on another stream, given as an object or as a handle, with the default stream busy;
and lengths that the builder's dims do not hold."""

import pytest
import torch

from tests.page_common import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _setup(S, lens, max_tokens):
    c = Case("bf16", "e4m3", lens, [0] * len(lens), kv_heads=2, group=4, dim=64, page=16, seed=7)
    bd = S.make_build_dims(batch=c.B, n_kv_heads=2, head_dim=64, max_tokens=max_tokens, rank=16, sketch=24, min_span=8,
                           window=32, dtype="bf16")
    g = torch.Generator().manual_seed(4)
    H = torch.rand((c.B, max_tokens), generator=g).cuda()
    H[:, ::37] += 4.0
    omega = torch.randn((64, 24), generator=g).cuda()
    return c, bd, H, omega


FIELDS = ("anchor_k", "anchor_v", "sum_k", "sum_v", "span_len", "factors", "block_off", "block_rank")


@pytest.mark.parametrize("handle", [False, True])
def test_on_another_stream(S, handle):
    c, bd, H, omega = _setup(S, [700, 433], 700)
    cache, ws = c.cache(S), c.workspace(S)
    want, _, _ = S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-3                        # work of the default stream that the call need not wait for
    got, seg, layout = S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws, stream=st.cuda_stream if handle else st)
    st.synchronize()
    for f in FIELDS:
        assert torch.equal(got[f].cpu(), want[f].cpu()), f
    assert layout["n_spans"].tolist() == seg["n_spans"].tolist()
    torch.cuda.synchronize()
    assert ws.status() == 0


@pytest.mark.parametrize("lens", [[700, 433], [433, 700]])
def test_lengths_past_the_builder_are_refused(S, lens):
    """A sequence longer than the builder's max_tokens, or of negative length, would lose tokens silently."""
    c, bd, H, omega = _setup(S, lens, 699)
    cache, ws = c.cache(S), c.workspace(S)
    with pytest.raises(ValueError, match="max_tokens"):
        S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws)
    cache.seq_len[lens.index(700)] = -1
    with pytest.raises(ValueError, match="max_tokens"):
        S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws)
    cache.seq_len[lens.index(700)] = 699
    S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws)
    assert ws.status() == 0
