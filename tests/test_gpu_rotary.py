"""Rotary positions on the GPU against the plain form in 64 bits: rows turned by themselves within the bound of their
roundings, keys stored on the way bit for bit, and the calls in use."""

import math
import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import TORCH, Case, encode_rows
from tests.page4_common import Case4, decode4, encode4
from tests.rotary_common import bound, frequencies, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _rotary(S, R, base=10000.0, **kw):
    f = frequencies(R, base)
    return S.Rotary(f.cuda(), **kw), f


def _check(got, x, pos, f, layout, scale=1.0, transpose=False):
    want = turned(x, pos, f, layout, scale, transpose)
    got = got.cpu()
    err, tol = (got.double() - want).abs(), bound(x, want, x.dtype, scale)
    banner(f"  error / bound {(err / tol).max().item() if err.numel() else 0:.3f}")
    assert (err <= tol).all()
    R = 2 * len(f)
    assert torch.equal(got[..., R:], x[..., R:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,R", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 64), (128, 112), (128, 16)])
def test_rotate(S, dtype, layout, dim, R):
    g = torch.Generator().manual_seed(zlib.crc32(repr((dtype, layout, dim, R)).encode()))
    r, f = _rotary(S, R, layout=layout)
    for n, heads in ((1, 1), (1, 9), (17, 3), (33, 8), (250, 1), (1000, 5)):
        banner(f"rotate {dtype} {layout} {dim} {R} {n} {heads}")
        x = torch.randn((n, heads, dim), generator=g).to(TORCH[dtype])
        pos = torch.randint(-1000, 200000, (n,), generator=g).int()
        pos[0] = 0
        for transpose in (False, True):
            _check(S.rotate(x.cuda(), pos.cuda(), r, transpose=transpose), x, pos, f, layout, transpose=transpose)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions_and_wide_frequencies(S, layout):
    """Positions over all of int32, frequencies from 2^-40 to 700 a position: angles past 2^40."""
    f = torch.cat([torch.exp2(torch.linspace(-40, 9, 60, dtype=torch.float64)), torch.tensor([math.pi / 2, math.pi, 2 * math.pi, 700.0], dtype=torch.float64)])
    r = S.Rotary(f.cuda(), layout=layout)
    pos = torch.cat([torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131072, 12345679, -99]), torch.arange(2 ** 20, 2 ** 20 + 500)]).int()
    x = torch.randn((len(pos), 2, 128), generator=torch.Generator().manual_seed(1))
    _check(S.rotate(x.cuda(), pos.cuda(), r), x, pos, f, layout)


def test_scale_and_scaled_frequencies(S):
    g = torch.Generator().manual_seed(2)
    x, pos = torch.randn((40, 4, 128), generator=g), torch.randint(0, 131072, (40,), generator=g).int()
    for scaling, kw in (("linear", dict(factor=4.0)), ("base", dict(factor=4.0)),
                        ("bands", dict(factor=8.0, trained=8192.0, low=1.0, high=4.0)),
                        ("ramp", dict(factor=16.0, trained=4096.0))):
        f, scale = S.rotary_frequencies(96, 10000.0, scaling, **kw)
        r = S.Rotary(f.cuda(), scale=scale)
        _check(S.rotate(x.cuda(), pos.cuda(), r), x, pos, f, "half", scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place_strided_and_other_streams(S, dtype, layout):
    """Slices of one projection's output, turned in place: the bits of the call on rows by themselves; nothing beside
    them changes."""
    g = torch.Generator().manual_seed(3)
    r, f = _rotary(S, 64, layout=layout)
    qkv = torch.randn((333, 14, 64), generator=g).to(TORCH[dtype]).cuda()
    pos = torch.randint(0, 99999, (333,), generator=g).int().cuda()
    q = qkv[:, 2:10]
    want = S.rotate(q.contiguous(), pos, r)
    assert torch.equal(S.rotate(q, pos, r), want)
    keep = qkv.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    assert S.rotate(q, pos, r, out=q, stream=st) is q
    st.synchronize()
    assert torch.equal(q, want)
    assert torch.equal(qkv[:, :2], keep[:, :2]) and torch.equal(qkv[:, 10:], keep[:, 10:])
    wide = torch.full((333, 20, 64), 5.0, dtype=TORCH[dtype], device="cuda")
    S.rotate(keep[:, 2:10], pos, r, out=wide[:, 3:11])
    assert torch.equal(wide[:, 3:11], want) and (wide[:, :3] == 5).all() and (wide[:, 11:] == 5).all()
    assert S.rotate(q[:0], pos[:0], r).shape == (0, 8, 64)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_values_that_are_not_finite_stay_in_their_pair(S, layout):
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.ones((4, 2, 128), dtype=dtype)
        x[0, 0, 5], x[1, 1, 100], x[2, 0, 70], x[3, 1, 127] = math.nan, math.inf, -math.inf, math.nan
        f = frequencies(96)
        got = S.rotate(x.cuda(), torch.tensor([3, 5, 7, 9], dtype=torch.int32).cuda(), S.Rotary(f.cuda(), layout=layout)).cpu()
        want = turned(x, torch.tensor([3, 5, 7, 9]), f, layout)
        assert torch.equal(torch.isfinite(got), torch.isfinite(want)) and torch.equal(got.isnan(), want.isnan())
        assert (~torch.isfinite(got)).sum() == 6                # two of a pair twice, and two behind rot_dim


def test_transpose_is_the_gradient(S):
    """Of sum(u * rotate(x)): the formula's, and differences of the call itself, which is linear: a step of 1."""
    g = torch.Generator().manual_seed(4)
    for layout in ("half", "interleaved"):
        f = frequencies(48)
        r = S.Rotary(f.cuda(), layout=layout, scale=1.25)
        x, u = torch.randn((9, 3, 64), generator=g), torch.randn((9, 3, 64), generator=g)
        pos = torch.randint(0, 5000, (9,), generator=g).int()
        grad = S.rotate(u.cuda(), pos.cuda(), r, transpose=True).cpu()
        leaf = x.double().requires_grad_()
        R, a = 48, pos.double()[:, None] * f
        c, s = 1.25 * a.cos()[:, None], 1.25 * a.sin()[:, None]
        p, q = (leaf[..., :R // 2], leaf[..., R // 2:R]) if layout == "half" else (leaf[..., 0:R:2], leaf[..., 1:R:2])
        y = torch.stack((p * c - q * s, q * c + p * s), -2 if layout == "half" else -1).flatten(-2)
        (torch.cat((y, leaf[..., R:]), -1) * u.double()).sum().backward()
        assert ((grad.double() - leaf.grad).abs() <= bound(u, leaf.grad, u.dtype, 1.25)).all()
        at = S.rotate(x.cuda(), pos.cuda(), r).cpu().double()
        for j in range(0, 64, 5):
            step = x.clone()
            step[..., j] += 1.0
            h = step[..., j].double() - x[..., j].double()
            moved = S.rotate(step.cuda(), pos.cuda(), r).cpu().double()
            diff = ((moved - at) * u.double()).sum(-1) / h
            # both results are rounded to float, 2^-24 of each value
            tol = (2.0 ** -24 * 1.01 * (moved.abs() + at.abs()) * u.double().abs()).sum(-1) / h.abs() + 2.0 ** -23 * grad[..., j].abs() + 1e-12
            assert ((grad[..., j].double() - diff).abs() <= tol).all()


def test_more_rows_than_2_31_values(S):
    n, heads, d = 264000, 64, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((n, heads, d), dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=g)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    r, f = _rotary(S, 128)
    tail = x[-20:].cpu()
    out = S.rotate(x, pos, r, out=x)
    _check(out[-20:], tail, pos[-20:].cpu(), f, "half")


# ---- keys on their way into the pages -------------------------------------------------------------

STORES = [("bf16", "same"), ("bf16", "e4m3"), ("bf16", "e2m1"), ("f32", "same"), ("f32", "e4m3"), ("f32", "e2m1")]


def _case(dtype, store, lens, news, **kw):
    return Case4(dtype, lens, news, **kw) if store == "e2m1" else Case(dtype, store, lens, news, **kw)


def _positions(c):
    """Each token's own place; tokens of nobody at 0."""
    p = torch.zeros(c.total, dtype=torch.int64)
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        p[c.start[b]:c.start[b + 1]] = torch.arange(n - nq, n)
    return p


def _expected(c, k):
    """Pools after rows k (float32) and c.v are stored."""
    want = {n: [x if x is None else x.clone() for x in c.codes[n]] for n in "kv"}
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        for i in range(nq):
            p = n - nq + i
            page, slot = int(c.table[b, p // c.page]) if p >= 0 else -1, p % c.page
            if not 0 <= page < c.n_pages:
                continue
            for name, src in (("k", k), ("v", c.v)):
                x = src[c.start[b] + i]
                if c.store == "same" and not isinstance(c, Case4):
                    want[name][0][page, :, slot] = x.to(c.k.dtype)
                else:
                    w = encode4(x) if isinstance(c, Case4) else encode_rows(x)
                    want[name][0][page, :, slot], want[name][1][page, :, slot] = w
    return want


def _check_pools(cache, want):
    for name, pool, scale in (("k", cache.k_pages, cache.k_scale), ("v", cache.v_pages, cache.v_scale)):
        got = pool.cpu()
        got = got.view(torch.uint8) if got.dtype == torch.float8_e4m3fn else got
        assert torch.equal(got, want[name][0]), name
        if scale is not None:
            assert torch.equal(scale.cpu(), want[name][1]), name


APPENDS = [
    dict(lens=[1], news=[1]),
    dict(lens=[40, 7, 0, 33], news=[1, 1, 0, 1], page=16),
    dict(lens=[17, 300, 64], news=[17, 123, 0], page=32, kv_heads=3, group=1),
    dict(lens=[5, 1000], news=[5, 777], page=128, dim=128, kv_heads=1, group=8, strided=True),
    dict(lens=[9, 31], news=[4, 31], page=16, dim=128),
    dict(lens=[1100], news=[1050], page=1024, kv_heads=2, strided=True, tail=5),
    dict(lens=[3, 5], news=[6, 2], dim=128),              # three tokens stand before the sequence
]


@pytest.mark.parametrize("dtype,store", STORES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kw", APPENDS, ids=lambda k: "-".join(map(str, k["lens"])))
def test_append(S, dtype, store, layout, kw):
    """Keys are stored from the turned values rounded to float, values as sekv_page_append stores them, queries have
    sekv_rotate's bits; what belongs to nobody is left alone."""
    banner(f"append turned {dtype} {store} {layout} {kw}")
    c = _case(dtype, store, **kw, seed=zlib.crc32(repr((dtype, store, str(kw))).encode()))
    R = c.d if c.total % 2 else c.d - 16
    r, f = _rotary(S, R, 500000.0, layout=layout, scale=1.0 if c.B > 1 else 1.25)
    scale = 1.0 if c.B > 1 else 1.25
    given = torch.randint(0, 100000, (c.total,), generator=torch.Generator().manual_seed(1)).int()
    for positions in (None, given):
        where = _positions(c) if positions is None else given
        cache, ws = c.cache(S), c.workspace(S)
        wide = torch.empty((c.total, c.Hkv * (c.G + 2) + 1, c.d), dtype=TORCH[dtype], device="cuda")
        Hq, Hkv = c.Hkv * c.G, c.Hkv
        wide[:, :Hq], wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:Hq + 2 * Hkv] = c.q.cuda(), c.k.cuda(), c.v.cuda()
        out = torch.full((c.total, Hq, c.d), 3.0, dtype=TORCH[dtype], device="cuda")
        got = S.page_append_rotary(c.dims(S), cache, r, wide[:, :Hq], wide[:, Hq:Hq + Hkv], wide[:, Hq + Hkv:Hq + 2 * Hkv],
                                   c.tok_start(), ws, q_out=out, positions=None if positions is None else positions.cuda())
        torch.cuda.synchronize()
        assert got is out
        _check_pools(cache, _expected(c, turned(c.k, where, f, layout, scale).float()))
        n = c.start[-1]
        assert torch.equal(out[:n], S.rotate(c.q.cuda(), where.int().cuda(), r)[:n]) and (out[n:] == 3.0).all()
        assert ws.status() == (8 if c.news[0] > c.lens[0] else 0)
        # without queries, and queries in place
        again = c.cache(S)
        assert S.page_append_rotary(c.dims(S), again, r, None, c.k.cuda(), c.v.cuda(), c.tok_start(), ws,
                                    positions=None if positions is None else positions.cuda()) is None
        assert torch.equal(again.k_pages.view(torch.uint8), cache.k_pages.view(torch.uint8))
        S.page_append_rotary(c.dims(S), again, r, wide[:, :Hq], c.k.cuda(), c.v.cuda(), c.tok_start(), ws, q_out=wide[:, :Hq],
                             positions=None if positions is None else positions.cuda())
        assert torch.equal(wide[:n, :Hq], out[:n])
        assert torch.equal(wide[:, Hq:Hq + Hkv], c.k.cuda())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append_in_float_is_rotate_then_append(S, layout):
    c = Case4("f32", [300, 77], [120, 77], dim=128, kv_heads=3, group=2, page=32, seed=3)
    r, _ = _rotary(S, 96, layout=layout)
    a, b, ws = c.cache(S), c.cache(S), c.workspace(S)
    S.page_append_rotary(c.dims(S), a, r, None, c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    S.page_append(c.dims(S), b, S.rotate(c.k.cuda(), _positions(c).int().cuda(), r), c.v.cuda(), c.tok_start(), ws)
    for x, y in zip(a._tensors(), b._tensors()):
        assert torch.equal(x, y)


@pytest.mark.parametrize("store", ["same", "e4m3", "e2m1"])
def test_append_leaves_bad_places_alone(S, store):
    c = _case("bf16", store, [40, 3], [10, 3])
    c.table[0, 1], c.table[0, 2] = -1, c.n_pages
    r, f = _rotary(S, 64)
    cache, ws = c.cache(S), c.workspace(S)
    out = S.page_append_rotary(c.dims(S), cache, r, c.q.cuda(), c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    _check_pools(cache, _expected(c, turned(c.k, _positions(c), f).float()))
    assert torch.equal(out, S.rotate(c.q.cuda(), _positions(c).int().cuda(), r))    # a query needs no place
    assert ws.status() == 8 and ws.status() == 0
    for start in ([0, 9, 4], [0, 3, 99], [-2, 3, 13]):
        out.fill_(3.0)
        S.page_append_rotary(c.dims(S), cache, r, c.q.cuda(), c.k.cuda(), c.v.cuda(),
                             torch.tensor(start, dtype=torch.int32, device="cuda"), ws, q_out=out)
        assert ws.status() == 8, start


def test_values_that_are_not_finite_are_stored_as_nan(S):
    c = Case4("bf16", [6], [6], dim=64, kv_heads=1, group=1)
    c.k[2, 0, 3], c.k[4, 0, 40] = math.inf, math.nan      # halves: with 35 and 8
    r, _ = _rotary(S, 64)
    cache, ws = c.cache(S), c.workspace(S)
    S.page_append_rotary(c.dims(S), cache, r, None, c.k.cuda(), c.v.cuda(), c.tok_start(), ws)
    E = cache.k_scale.cpu()[int(c.table[0, 0]), 0]
    assert (E == 255).tolist() == [[False] * 2] * 2 + [[True] * 2] + [[False] * 2] + [[True] * 2] + [[False] * 2] + \
        (c.codes["k"][1][int(c.table[0, 0]), 0, 6:] == 255).tolist()


def test_captured_calls_follow_the_tables(S):
    """Turning, storing and attending in one graph, replayed after lengths, positions and inputs changed, with eager
    calls between: every replay gives the eager result."""
    B, Hkv, G, d, page = 3, 2, 4, 128, 16
    pd = S.make_page_dims(batch=B, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=400,
                          max_pages=130, dtype="bf16", page_dtype="e2m1", softmax_scale=d ** -0.5)
    g = torch.Generator().manual_seed(9)
    table = torch.randperm(390, generator=g).int().reshape(B, 130).cuda()
    cache = S.PageCache.empty(pd, table, torch.full((B,), 1500, dtype=torch.int32, device="cuda"))
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, B * 1500))
    r, _ = _rotary(S, 128)
    prompt = torch.randn((B * 1500, Hkv, d), generator=g).bfloat16().cuda()
    S.page_append_rotary(pd, cache, r, None, prompt, prompt.flip(0).contiguous(),
                         torch.tensor([0, 1500, 3000, 4500], dtype=torch.int32, device="cuda"), ws)
    n = 40
    x = {k: torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda") for k, h in (("q", Hkv * G), ("k", Hkv), ("v", Hkv))}
    start, pos = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    turned_q, out, back = (torch.empty_like(x["q"]) for _ in range(3))
    lse = torch.empty((n, Hkv * G), device="cuda")

    def run(turned_q, out, lse, back):
        S.page_append_rotary(pd, cache, r, x["q"], x["k"], x["v"], start, ws, q_out=turned_q, positions=pos)
        S.page_attend(pd, cache, turned_q, start, ws, out=out, lse=lse)
        S.rotate(turned_q, pos, r, out=back, transpose=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(turned_q, out, lse, back)
    torch.cuda.current_stream().wait_stream(side)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        run(turned_q, out, lse, back)
    lens = [1500] * B
    for st in ([0, 1, 33, 34], [0, 40, 40, 40], [0, 0, 17, 39], [0, 1, 2, 3]):
        lens = [ln + st[b + 1] - st[b] for b, ln in enumerate(lens)]
        cache.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        start.copy_(torch.tensor(st, dtype=torch.int32))
        pos.copy_(torch.randint(0, 4000, (n,), generator=g).int())
        for k in "qkv":
            x[k].copy_(torch.randn(x[k].shape, generator=g).bfloat16())
        for t in (turned_q, out, lse, back):
            t.fill_(-3.0)
        gr.replay()
        got = [t.clone() for t in (turned_q, out, lse, back)]
        pools = [t.clone() for t in cache._tensors()]
        want = [torch.full_like(t, -3.0) for t in (turned_q, out, lse, back)]
        run(*want)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for a, b in zip(pools, cache._tensors()):
            assert torch.equal(a, b)
        assert (got[0][st[-1]:] == -3.0).all() and torch.isfinite(got[1].float()).all()
    assert ws.status() == 0


@pytest.mark.parametrize("dtype,store", STORES)
def test_prompt_in_chunks_then_build_then_decode(S, dtype, store):
    """The path of a layer: chunks are turned, stored and attended to one after another, each result within its bound;
    the rows read back become the span cache; and a decode step with a turned query runs on it."""
    Hkv, G, d, page, n_max = 2, 4, 64, 16, 300
    steps = [[156, 100], [100, 1], [43, 100], [1, 32]]
    g = torch.Generator().manual_seed(3)
    dt = TORCH[dtype]
    rows = {n: torch.randn((2, n_max, Hkv, d), generator=g).to(dt) for n in "kv"}
    qs = torch.randn((2, n_max, Hkv * G, d), generator=g).to(dt)
    pd = S.make_page_dims(batch=2, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=44, max_pages=20,
                          dtype=dtype, page_dtype=None if store == "same" else store, softmax_scale=d ** -0.5)
    table = torch.randperm(40, generator=g).int().reshape(2, 20)
    cache = S.PageCache.empty(pd, table.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda"))
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, 300))
    f, scale = S.rotary_frequencies(64, 10000.0, "ramp", factor=4.0, trained=128.0)
    r = S.Rotary(f.cuda(), scale=scale)
    done = [0, 0]
    for new in steps:
        start = torch.tensor([0, new[0], new[0] + new[1]], dtype=torch.int32, device="cuda")
        done = [done[b] + new[b] for b in range(2)]
        cache.seq_len.copy_(torch.tensor(done, dtype=torch.int32))
        k, v, q = (torch.cat([t[b, done[b] - new[b]:done[b]] for b in range(2)]).cuda() for t in (rows["k"], rows["v"], qs))
        q = S.page_append_rotary(pd, cache, r, q, k, v, start, ws)
        out, lse = S.page_attend(pd, cache, q, start, ws, want_lse=True)
        c = Case(dtype, "same", done, new, kv_heads=Hkv, group=G, dim=d, page=page)
        c.table, c.n_pages, c.max_pages, c.scale = table, 44, 20, d ** -0.5
        c.q, c.total = q.cpu(), sum(new)
        for name, pool, e in (("k", cache.k_pages, cache.k_scale), ("v", cache.v_pages, cache.v_scale)):
            x = pool.cpu()
            c.pools[name] = x.double() if store == "same" else decode4(x, e.cpu()) if store == "e2m1" else \
                x.double() * 2.0 ** (e.cpu().double() - 127)[..., None]
        ref, rl, tol, ltol = c.attend()
        assert ((out.cpu().double() - ref).abs() <= tol).all() and ((lse.cpu().double() - rl).abs() <= ltol).all()
    assert done == [300, 233] and ws.status() == 0
    keys, values = S.page_read(pd, cache, n_max, ws)
    for b in range(2):
        where = torch.arange(done[b])
        want = turned(rows["k"][b, :done[b]], where, f, "half", scale).float()
        want = want.to(dt).double() if store == "same" else decode4(*encode4(want)) if store == "e2m1" else None
        if want is not None:
            assert torch.equal(keys[b, :, :done[b]].cpu().double(), want.transpose(0, 1))
    H = torch.rand((2, n_max), generator=g).cuda()
    H[:, ::37] += 4.0
    bd = S.make_build_dims(batch=2, n_kv_heads=Hkv, head_dim=d, max_tokens=n_max, rank=16, sketch=24, min_span=8,
                           window=32, dtype=dtype)
    a, _, la = S.build_layer_paged(bd, pd, cache, H, torch.randn((d, 24), generator=g).cuda(), ws)
    dims = S.make_dims(batch=2, n_q_heads=Hkv * G, n_kv_heads=Hkv, head_dim=d, rank=16, top_k=max(1, min(64, la["max_spans"])),
                       max_anchors=la["max_anchors"], max_spans=la["max_spans"], max_span_len=la["max_span_len"],
                       dtype=dtype, softmax_scale=d ** -0.5)
    q = S.rotate(qs[:, -1].contiguous().cuda(), cache.seq_len, r)
    _, got = S.decode_step(dims, S.DeviceCache(dict(a, q=q), dtype), S.Workspace(dims))
    assert torch.isfinite(got).all()
