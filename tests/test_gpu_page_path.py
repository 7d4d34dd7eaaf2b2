"""The paged token store as it is used: prompts in chunks, read back for the builder, decode steps on the
built cache; captured graphs whose tables change between replays; workspaces shared between calls; offsets
past 2^31."""

import math

import numpy as np
import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import TORCH, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _within(out, lse, c):
    ref, rl, tol, ltol = c.attend()
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    some = rl > -math.inf
    assert torch.equal(lse.cpu() > -math.inf, some)
    assert ((lse.cpu().double() - rl).abs()[some] <= ltol[some]).all()




@pytest.mark.parametrize("dtype,store", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
def test_prompt_in_chunks_then_build_then_decode(S, dtype, store):
    """Chunks are appended and attended to one after another, each result within its bound; the rows read
    back are what was stored; the builder on the pages gives the bytes that it gives on those rows; and a
    decode step runs on what it built."""
    Hkv, G, d, page, n_max = 2, 4, 64, 16, 700
    lens_end, steps = [700, 433], [[256, 200], [256, 1], [187, 200], [1, 32]]
    g = torch.Generator().manual_seed(3)
    dt = TORCH[dtype]
    rows = {n: torch.randn((2, n_max, Hkv, d), generator=g).to(dt) for n in "kv"}
    qs = torch.randn((2, n_max, Hkv * G, d), generator=g).to(dt)
    pd_kw = dict(batch=2, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=90, max_pages=44,
                 dtype=dtype, page_dtype="e4m3" if store == "e4m3" else None, softmax_scale=d ** -0.5)
    pd = S.make_page_dims(**pd_kw)
    table = torch.randperm(88, generator=g).int().reshape(2, 44)
    cache = S.PageCache.empty(pd, table.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda"))
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, 512))
    done = [0, 0]
    for new in steps:
        start = torch.tensor([0, new[0], new[0] + new[1]], dtype=torch.int32, device="cuda")
        done = [done[b] + new[b] for b in range(2)]
        cache.seq_len.copy_(torch.tensor(done, dtype=torch.int32))
        k, v, q = (torch.cat([t[b, done[b] - new[b]:done[b]] for b in range(2)]).cuda() for t in (rows["k"], rows["v"], qs))
        S.page_append(pd, cache, k, v, start, ws)
        out, lse = S.page_attend(pd, cache, q, start, ws, want_lse=True)
        # the plain form on the rows as they are stored
        c = Case(dtype, store, done, new, kv_heads=Hkv, group=G, dim=d, page=page)
        c.table, c.n_pages, c.max_pages, c.scale = table, 90, 44, d ** -0.5
        c.q, c.total = q.cpu(), sum(new)
        for name, pool, scale in (("k", cache.k_pages, cache.k_scale), ("v", cache.v_pages, cache.v_scale)):
            x = pool.cpu().double() if scale is None else pool.cpu().to(torch.float64) * 2.0 ** (scale.cpu().double() - 127)[..., None]
            c.pools[name] = x
        _within(out, lse, c)
    assert done == lens_end and ws.status() == 0
    keys, values = S.page_read(pd, cache, n_max, ws)
    for b in range(2):
        p, s = table[b].long()[torch.arange(done[b]) // page], torch.arange(done[b]) % page
        for got, name in ((keys, "k"), (values, "v")):
            assert torch.equal(got[b, :, :done[b]].cpu().double(), c.pools[name][p, :, s].transpose(0, 1))
            assert not got[b, :, done[b]:].any()
    # builder on the pages and on the rows
    H = torch.rand((2, n_max), generator=g).cuda()
    H[:, ::37] += 4.0
    bd = S.make_build_dims(batch=2, n_kv_heads=Hkv, head_dim=d, max_tokens=n_max, rank=16, sketch=24, min_span=8,
                           window=32, dtype=dtype)
    omega = torch.randn((d, 24), generator=g).cuda()
    a, _, la = S.build_layer_paged(bd, pd, cache, H, omega, ws)
    b_, _, lb = S.build_layer(bd, keys, values, H, cache.seq_len, omega, ws)
    assert la["n_spans"].tolist() == lb["n_spans"].tolist() and ws.status() == 0
    for f in ("anchor_k", "anchor_v", "sum_k", "sum_v", "span_len", "factors", "block_off", "block_rank"):
        assert torch.equal(a[f].cpu(), b_[f].cpu()), f
    # a decode step on it (the same workspace: the step lays it out anew)
    dims = S.make_dims(batch=2, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, rank=16, top_k=4,
                       max_anchors=la["max_anchors"], max_spans=la["max_spans"], max_span_len=la["max_span_len"],
                       dtype=dtype, softmax_scale=d ** -0.5)
    t = dict(a, q=qs[:, -1].contiguous().cuda())
    step_ws = S.Workspace(dims)
    sel, want = S.decode_step(dims, S.DeviceCache(t, dtype), step_ws)
    assert torch.isfinite(want).all() and step_ws.status() == 0
    if ws.nbytes >= S.workspace_size(dims):
        for _ in range(2):                                # step and page calls in turn on one workspace
            sel2, got = S.decode_step(dims, S.DeviceCache(t, dtype), ws)
            assert torch.equal(sel, sel2) and torch.equal(want, got)
            again, l2 = S.page_attend(pd, cache, q, start, ws, want_lse=True)
            assert torch.equal(again, out) and torch.equal(l2, lse)
        assert ws.status() == 0
    with pytest.raises(ValueError):
        S.build_layer_paged(S.make_build_dims(batch=1, n_kv_heads=Hkv, head_dim=d, max_tokens=n_max, rank=16, sketch=24,
                                              min_span=8, window=32, dtype=dtype), pd, cache, H, omega, ws)


@pytest.mark.parametrize("store", ["same", "e4m3"])
def test_captured_calls_follow_the_tables(S, store):
    """append and attend in one graph: replayed after the tables and inputs changed, with eager calls between,
    every replay gives the eager result.  Two graphs share a workspace, one after the other."""
    banner(f"graph {store}")
    B, Hkv, G, d, page = 3, 2, 4, 128, 16
    pd = S.make_page_dims(batch=B, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=400,
                          max_pages=130, dtype="bf16", page_dtype="e4m3" if store == "e4m3" else None,
                          softmax_scale=d ** -0.5)
    g = torch.Generator().manual_seed(9)
    table = torch.randperm(390, generator=g).int().reshape(B, 130).cuda()
    cache = S.PageCache.empty(pd, table, torch.ones(B, dtype=torch.int32, device="cuda"))
    prompt = torch.randn((B * 2000, Hkv, d), generator=g).bfloat16().cuda()
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, B * 2000))
    cache.seq_len.fill_(2000)
    S.page_append(pd, cache, prompt, prompt.flip(0).contiguous(), torch.tensor([0, 2000, 4000, 6000], dtype=torch.int32,
                                                                               device="cuda"), ws)
    graphs = []
    for n in (B, 40):                                     # one token each; a ragged chunk
        x = {k: torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda") for k, h in (("q", Hkv * G), ("k", Hkv), ("v", Hkv))}
        x["start"] = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        x["out"] = torch.empty_like(x["q"])
        x["lse"] = torch.empty((n, Hkv * G), device="cuda")

        def run(x=x):
            S.page_append(pd, cache, x["k"], x["v"], x["start"], ws)
            S.page_attend(pd, cache, x["q"], x["start"], ws, out=x["out"], lse=x["lse"])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            run()
        graphs.append((gr, x))
    lens, starts = [2000] * B, {B: [[0, 1, 2, 3], [0, 1, 2, 3], [0, 1, 1, 2]], 40: [[0, 1, 33, 34], [0, 40, 40, 40], [0, 0, 17, 39]]}
    for turn in range(3):
        for gr, x in graphs:
            n = x["q"].shape[0]
            st = starts[n][turn]
            lens = [ln + st[b + 1] - st[b] for b, ln in enumerate(lens)]
            if turn == 2:
                lens[0] = 31                              # a sequence starts anew
            cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
            x["start"].copy_(torch.tensor(st, dtype=torch.int32))
            for k in "qkv":
                x[k].copy_(torch.randn(x[k].shape, generator=g).bfloat16())
            x["out"].fill_(-3.0)
            gr.replay()
            got, gl = x["out"].clone(), x["lse"].clone()
            want = torch.full_like(got, -3.0)
            wl = torch.empty_like(gl)
            S.page_append(pd, cache, x["k"], x["v"], x["start"], ws)
            S.page_attend(pd, cache, x["q"], x["start"], ws, out=want, lse=wl)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(gl[:st[-1]], wl[:st[-1]])
            assert torch.isfinite(got).all() and (got[st[-1]:] == -3.0).all()
    assert ws.status() == 0


def test_graphs_of_different_shapes_share_a_workspace(S):
    """Captured calls of other head counts and types in turn on one workspace: each finds its counters zero."""
    banner("graphs of shapes")
    cases = [Case("bf16", "e4m3", [3000, 900], [1, 2], dim=128, kv_heads=2, group=8, page=16, seed=1),
             Case("f32", "same", [1500], [1], dim=64, kv_heads=7, group=1, page=16, seed=2),
             Case("bf16", "same", [700, 2600], [150, 300], dim=64, kv_heads=3, group=2, page=32, seed=3)]
    ws = S.Workspace(None, "cuda", nbytes=max(S.page_workspace_size(c.dims(S), sum(c.news)) for c in cases))
    parts = []
    for c in cases:
        cache, q, ts = c.cache(S), c.q.cuda(), c.tok_start()
        own = c.workspace(S)
        want = S.page_attend(c.dims(S), cache, q, ts, own, want_lse=True)
        out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
        S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
        parts.append((gr, cache, q, ts, out, lse, want, own))
    for turn in (0, 1, 2, 1, 0, 2, 2, 0):
        gr, cache, q, ts, out, lse, want, own = parts[turn]
        out.fill_(7.0)
        lse.fill_(7.0)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), turn
    assert ws.status() == 0


def test_wrong_tables_leave_nothing_behind(S):
    """tok_start that descends or passes n_tokens, and a negative or too long seq_len: flagged, and the next
    call on the workspace is right."""
    c = Case("bf16", "e4m3", [900, 300, 77], [1, 1, 1], dim=128, page=16, kv_heads=2, seed=1)
    cache, ws, q = c.cache(S), c.workspace(S), c.q.cuda()
    want, wl = S.page_attend(c.dims(S), cache, q, c.tok_start(), ws, want_lse=True)
    assert ws.status() == 0
    lens = cache.seq_len.clone()
    for start, sl in (([0, 2, 1, 3], None), ([0, 1, 2, 9], None), ([2, 1, 0, 0], None), (None, [-5, 300, 77]),
                      (None, [900, c.max_pages * c.page + 1, 77])):
        ts = c.tok_start() if start is None else torch.tensor(start, dtype=torch.int32, device="cuda")
        if sl is not None:
            cache.seq_len.copy_(torch.tensor(sl, dtype=torch.int32))
        S.page_attend(c.dims(S), cache, q, ts, ws)
        assert ws.status() == 8, (start, sl)
        cache.seq_len.copy_(lens)
        out, lse = S.page_attend(c.dims(S), cache, q, c.tok_start(), ws, want_lse=True)
        assert torch.equal(out, want) and torch.equal(lse, wl) and ws.status() == 0


def test_offsets_past_2_31(S):
    """A pool of more than 2^32 bytes and 2^31 elements whose last pages are used."""
    Hkv, d, page = 8, 128, 64
    n_pages = (1 << 31) // (Hkv * page * d) + 24
    pd = S.make_page_dims(batch=1, n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=n_pages,
                          max_pages=8, dtype="bf16", softmax_scale=d ** -0.5)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, n_pages // 2, 5, n_pages - 9, 1, 2]], dtype=torch.int32)
    k = torch.empty((n_pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    n, new = 380, 380
    cache = S.PageCache(k, v, table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    g = torch.Generator().manual_seed(2)
    x = torch.randn((3, new, Hkv, d), generator=g).bfloat16()
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, new))
    ts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    S.page_append(pd, cache, x[0].cuda(), x[1].cuda(), ts, ws)
    keys, values = S.page_read(pd, cache, n, ws)
    assert torch.equal(keys[0].cpu(), x[0].transpose(0, 1)) and torch.equal(values[0].cpu(), x[1].transpose(0, 1))
    out, _ = S.page_attend(pd, cache, x[2].cuda(), ts, ws)
    one, _ = S.page_attend(pd, cache, x[2][-1:].cuda(), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), ws)
    K, V, Q = (t.double() for t in x)
    s = torch.einsum("qhd,khd->hqk", Q, K) * d ** -0.5
    s.masked_fill_(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
    w = torch.softmax(s, -1)
    ref = torch.einsum("hqk,khd->qhd", w, V)
    # a weight and the result are rounded to bfloat16 (2^-8 each); the float terms are below 2^-12
    tol = (2.0 ** -8 + 2.0 ** -12) * torch.einsum("hqk,khd->qhd", w, V.abs()) + 2.0 ** -8 * ref.abs() + 1e-6
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    assert ((one.cpu().double() - ref[-1:]).abs() <= tol[-1:]).all()
    assert ws.status() == 0


@pytest.mark.parametrize("batch", [1, 64, 65, 200, 257, 1100])
def test_many_sequences(S, batch):
    """More sequences than lanes: the same results as each sequence by itself."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 260, batch)]
    news = [int(min(n, x)) for n, x in zip(lens, rng.choice([0, 1, 1, 1, 5, 40], batch))]
    c = Case("bf16", "e4m3", lens, news, kv_heads=2, group=4, dim=64, page=16, seed=batch)
    out, lse = S.page_attend(c.dims(S), c.cache(S), c.q.cuda(), c.tok_start(), c.workspace(S), want_lse=True)
    _within(out, lse, c)


def test_two_streams_with_their_own_workspaces(S):
    c = Case("bf16", "same", [3000, 900], [1, 33], dim=128, kv_heads=2, page=32, seed=5)
    cache, q, ts = c.cache(S), c.q.cuda(), c.tok_start()
    want, wl = S.page_attend(c.dims(S), cache, q, ts, c.workspace(S), want_lse=True)
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in range(2)]
    ws = [c.workspace(S) for _ in st]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, w in zip(st, ws):
            got.append(S.page_attend(c.dims(S), cache, q, ts, w, want_lse=True, stream=s))
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want) and torch.equal(l, wl)
