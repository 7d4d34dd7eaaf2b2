"""Keys and queries turned on their way into the pages: batches of more sequences than a wave has lanes, prompts whose
tokens' heads are one wave's, and calls of more waves than a launch starts."""

import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import TORCH, Case, encode_rows
from tests.page4_common import Case4, encode4
from tests.rotary_common import bound, frequencies, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _places(c):
    """(token, page, slot, position) of the tokens that have a place, and a position for every token."""
    where, rows = torch.zeros(c.total, dtype=torch.int64), []
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        t = torch.arange(c.start[b], c.start[b + 1])
        p = n - nq + torch.arange(nq)
        where[t] = p
        ok = p >= 0
        rows.append(torch.stack((t[ok], c.table[b].long()[p[ok] // c.page], p[ok] % c.page), -1))
    return torch.cat(rows).unbind(-1), where


def _stored(c, k, places):
    """Pools after rows k (float32) and c.v are stored there."""
    t, page, slot = places
    want = {}
    for name, x in (("k", k), ("v", c.v.float())):
        codes, E = (y if y is None else y.clone() for y in c.codes[name])
        if isinstance(c, Case4):
            new = encode4(x)
        elif c.store == "e4m3":
            new = encode_rows(x)
        else:
            new = (x.to(c.k.dtype),)
        codes[page, :, slot] = new[0][t]
        if E is not None:
            E[page, :, slot] = new[1][t]
        want[name] = (codes, E)
    return want


def _check(S, c, layout, given, R, seed=0, queries=True, in_place=False):
    r, f = S.Rotary(frequencies(R, 500000.0).cuda(), layout=layout), frequencies(R, 500000.0)
    places, where = _places(c)
    pos = None
    if given:
        where = torch.randint(-100, 200000, (c.total,), generator=torch.Generator().manual_seed(seed))
        pos = where.int().cuda()
    cache, ws = c.cache(S), c.workspace(S)
    q = c.q.cuda() if queries else None
    out = None if not queries else q if in_place else torch.full(q.shape, 3.0, dtype=q.dtype, device="cuda")
    S.page_append_rotary(c.dims(S), cache, r, q, c.k.cuda(), c.v.cuda(), c.tok_start(), ws, q_out=out, positions=pos)
    torch.cuda.synchronize()
    want = _stored(c, turned(c.k, where, f, layout).float(), places)
    for name, pool, scale in (("k", cache.k_pages, cache.k_scale), ("v", cache.v_pages, cache.v_scale)):
        got = pool.cpu()
        got = got.view(torch.uint8) if got.dtype == torch.float8_e4m3fn else got
        assert torch.equal(got, want[name][0]), name
        assert scale is None or torch.equal(scale.cpu(), want[name][1]), name
    assert ws.status() == 0
    if not queries:
        return
    mine = torch.zeros(c.total, dtype=torch.bool)
    mine[c.start[0]:c.start[-1]] = True
    q_want = turned(c.q, where, f, layout)
    got = out.cpu()
    assert ((got.double() - q_want).abs() <= bound(c.q, q_want, c.q.dtype))[mine].all()
    left = c.q if in_place else torch.full(c.q.shape, 3.0, dtype=c.q.dtype)
    assert torch.equal(got[~mine], left[~mine])              # rows of nobody


def _many(dtype, store, batch, seed, dim=64):
    """Empty sequences at the start, in runs over several steps of a search by 64, and at the end; rows of nobody on both
    sides."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, 20, (batch,), generator=g).tolist()
    news = torch.tensor([0, 0, 1, 1, 2, 7])[torch.randint(0, 6, (batch,), generator=g)].tolist()
    news = [min(a, b) for a, b in zip(lens, news)]
    for a, b in ((0, batch // 13 + 1), (batch // 3, batch // 3 + batch // 5 + 2), (batch - batch // 9 - 1, batch)):
        news[a:b] = [0] * (b - a)
    news[batch // 2], lens[batch // 2] = 33, 40
    new = Case4 if store == "e2m1" else lambda d, *a, **kw: Case(d, store, *a, **kw)
    c = new(dtype, lens, news, kv_heads=1, group=4 if batch < 1000 else 1, dim=dim, page=16, tail=9, seed=seed)
    c.start = [s + 4 for s in c.start]                       # of nine rows of nobody four come first
    return c


@pytest.mark.parametrize("batch,store", [(b, s) for b in (64, 65, 128, 129, 300) for s in ("e2m1", "e4m3", "same")] +
                         [(4095, "e2m1"), (4095, "same"), (4096, "e2m1"), (4096, "same")])
def test_many_sequences(S, batch, store):
    banner(f"many sequences {batch} {store}")
    for dtype, layout, given in (("bf16", "half", False), ("f32", "interleaved", True)):
        c = _many(dtype, store, batch, batch, 64 if batch % 2 else 128)
        _check(S, c, layout, given, 48, in_place=given)


@pytest.mark.parametrize("batch", [65, 300, 4096])
def test_many_wrong_offsets_are_flagged(S, batch):
    c = _many("bf16", "e2m1", batch, 7)
    r = S.Rotary(frequencies(64).cuda())
    for at, to in ((batch // 2, c.total + 5), (batch // 2 + 1, 0), (0, -3), (batch, c.total + 1), (batch // 4, -1)):
        start = c.tok_start()
        start[at] = to
        cache, ws = c.cache(S), c.workspace(S)
        S.page_append_rotary(c.dims(S), cache, r, c.q.cuda(), c.k.cuda(), c.v.cuda(), start, ws)
        assert ws.status() == 8, (at, to)


# (dtype, head_dim, KV heads, tokens): heads a wave stores are 3 and 2 of 5, 2 2 1 of 5, 2 of 3 and 1, all 5, 2 2 2 1 of 7
HEADS = [("bf16", 128, 5, 2099), ("bf16", 64, 5, 2099), ("bf16", 128, 3, 2099), ("f32", 128, 5, 2099), ("f32", 64, 7, 1051)]


@pytest.mark.parametrize("store", ["e2m1", "e4m3", "same"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,dim,heads,n", HEADS)
def test_several_heads_a_wave(S, dtype, dim, heads, n, store, layout):
    """Long prompts: a wave stores several heads of its tokens, the next one's rows on their way meanwhile; the last wave's
    tokens and heads are fewer."""
    banner(f"several heads {dtype} {dim} {heads} {n} {store} {layout}")
    rows = 64 // (dim // (8 if dtype == "bf16" else 4))
    groups = -(-n // rows)
    assert -(-1024 // groups) < heads and n % rows           # fewer parts than heads: one has several
    new = Case4 if store == "e2m1" else lambda d, *a, **kw: Case(d, store, *a, **kw)
    a = n // 3
    c = new(dtype, [a + 100, n - a], [a, n - a], kv_heads=heads, group=1, dim=dim, page=32, strided=True,
            seed=zlib.crc32(repr((dtype, dim, heads, store)).encode()))
    for given in (False, True):
        _check(S, c, layout, given, dim - 16, seed=3, queries=given)


def test_more_query_waves_than_a_launch_starts(S):
    """2^21 workgroups of four waves, a token each, and 1400 tokens more."""
    n = (1 << 23) + 1400
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((n, 1, 64), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    pos, f = torch.arange(n, dtype=torch.int32, device="cuda"), frequencies(64)
    r = S.Rotary(f.cuda())
    out = S.rotate(x, pos, r)
    for at in (0, (1 << 23) - 700, n - 1400):
        rows = slice(at, at + 1400)
        assert torch.equal(out[rows], S.rotate(x[rows], pos[rows], r))
    tail = x[-500:].cpu()
    want = turned(tail, pos[-500:].cpu(), f)
    assert ((out[-500:].cpu().double() - want).abs() <= bound(tail, want, tail.dtype)).all()


def test_more_key_waves_than_a_launch_starts(S):
    """The same of keys, eight tokens a wave."""
    n, page = (1 << 26) + 4000, 1024
    n_pages = -(-n // page)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.empty((n, 1, 64), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    f = frequencies(64)
    r = S.Rotary(f.cuda())

    def store(rows, at):
        """Pools after rows `at` on of one sequence are its only new tokens."""
        pd = S.make_page_dims(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, page_size=page, n_pages=n_pages,
                              max_pages=n_pages, dtype="bf16", page_dtype="e2m1", softmax_scale=0.125)
        cache = S.PageCache.empty(pd, torch.arange(n_pages, dtype=torch.int32, device="cuda")[None],
                                  torch.tensor([at + len(rows)], dtype=torch.int32, device="cuda"))
        ws = S.Workspace(None, "cuda", nbytes=256)
        S.page_append_rotary(pd, cache, r, None, rows, rows, torch.tensor([0, len(rows)], dtype=torch.int32, device="cuda"), ws)
        assert ws.status() == 0
        return cache
    whole = store(x, 0)
    flat = [t.flatten(0, 2) for t in (whole.k_pages, whole.v_pages, whole.k_scale, whole.v_scale)]
    for at in (0, (1 << 26) - 2000, n - 4000):
        part = store(x[at:at + 4000], at)
        for a, b in zip(flat, (part.k_pages, part.v_pages, part.k_scale, part.v_scale)):
            assert torch.equal(a[at:at + 4000], b.flatten(0, 2)[at:at + 4000])
    tail = x[-300:].cpu()
    codes, E = encode4(turned(tail, torch.arange(n - 300, n), f).float())
    assert torch.equal(flat[0][n - 300:n].cpu(), codes[:, 0]) and torch.equal(flat[2][n - 300:n].cpu(), E[:, 0])
