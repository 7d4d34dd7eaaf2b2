"""4-bit pages on the GPU against the plain form in 64 bits: what is stored and read back bit for bit,
attention within the bound that its roundings allow (Case.attend; the stored values are exact in either type)."""

import math
import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import TORCH
from tests.page4_common import Case4, decode4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _seed(*a):
    return zlib.crc32(repr(a).encode())


def _strided(c, name):
    """The same strided view of one device tensor."""
    x = getattr(c, name)
    if x.is_contiguous():
        return x.to("cuda")
    base = torch.as_strided(x, (x.shape[0], x.stride(0) // c.d, c.d), (x.stride(0), c.d, 1), 0).to("cuda")
    at = x.storage_offset() // c.d
    return base[:, at:at + x.shape[1]]


def _check_pools(cache, want):
    for name, pool, scale in (("k", cache.k_pages, cache.k_scale), ("v", cache.v_pages, cache.v_scale)):
        E = scale.cpu()
        assert torch.equal(E, want[name][1]), name
        nan = (E == 255).repeat_interleave(16, -1)          # the codes of such a block stand for nothing
        assert torch.equal(pool.cpu().masked_fill(nan, 0), want[name][0].masked_fill(nan, 0)), name


def _check_append(S, c, bits=0):
    cache, ws = c.cache(S), c.workspace(S)
    S.page_append(c.dims(S), cache, _strided(c, "k"), _strided(c, "v"), c.tok_start(), ws)
    torch.cuda.synchronize()
    _check_pools(cache, c.stored(c.k, c.v))
    assert ws.status() == bits


APPENDS = [
    dict(lens=[1], news=[1]),
    dict(lens=[40, 7, 0, 33], news=[1, 1, 0, 1], page=16),
    dict(lens=[17, 300, 64], news=[17, 123, 0], page=32, kv_heads=3, group=1),
    dict(lens=[5, 1000], news=[5, 777], page=128, dim=128, kv_heads=1, group=8, strided=True),
    dict(lens=[9, 31], news=[4, 31], page=16, dim=128),
    dict(lens=[2100], news=[2050], page=1024, kv_heads=2, strided=True, tail=5),
    dict(lens=[3, 5], news=[6, 2]),                       # three tokens stand before the sequence
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", APPENDS, ids=lambda k: "-".join(map(str, k["lens"])))
def test_append(S, dtype, kw):
    banner(f"append e2m1 {dtype} {kw}")
    _check_append(S, Case4(dtype, **kw, seed=_seed(dtype, str(kw))), 8 if kw["news"][0] > kw["lens"][0] else 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_append_of_extreme_blocks(S, dtype, dim):
    """Zeros, subnormals, the largest values, infinities and NaN in one block of a row and not the others, ties
    of the rounding, blocks just at and above 6 * 2^n, every exponent."""
    banner(f"extreme e2m1 {dtype} {dim}")
    c = Case4(dtype, [512], [512], dim=dim, kv_heads=1, group=1)
    big = torch.finfo(TORCH[dtype]).max
    x = c.k.float()
    x[0] = 0.0
    x[1] = -0.0
    x[2] = 1e-40
    x[3, 0, :4] = torch.tensor([big, -big, 1.0, 0.0])
    x[4, 0, 5] = math.inf
    x[5, 0, dim - 1] = math.nan
    x[6] = math.nan
    x[7, 0, 32:] = -math.inf
    t = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    x[8] = torch.cat([t, -t, t * 1.0078125, t * 0.9921875] * (dim // 32))      # ties, and one bfloat16 step beside them
    x[9] = 6.0
    x[10] = 6.03125
    x[11] = 2.0 ** -126
    x[12] = 6 * 2.0 ** 125
    x[13] = 2.0 ** -124 * torch.arange(dim) / dim
    g = torch.Generator().manual_seed(4)
    n = torch.arange(-126, 128).double()
    x[20:20 + len(n), 0] = (torch.randn((len(n), dim), generator=g).clamp(-1, 1) * torch.exp2(n)[:, None]).float()
    c.k = x.to(TORCH[dtype])
    c.v = c.k.flip(0).contiguous()
    _check_append(S, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_leaves_bad_places_alone(S, dtype):
    banner(f"bad places e2m1 {dtype}")
    c = Case4(dtype, [40, 3], [10, 3])
    c.table[0, 1], c.table[0, 2] = -1, c.n_pages
    _check_append(S, c, bits=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(lens=[1]), dict(lens=[33, 0, 200], page=32, kv_heads=3, group=1),
                                dict(lens=[5, 1000], page=128, dim=128, kv_heads=1), dict(lens=[9, 31]),
                                dict(lens=[2100], page=1024, dim=128)], ids=lambda k: "-".join(map(str, k["lens"])))
def test_read(S, dtype, kw):
    banner(f"read e2m1 {dtype} {kw}")
    c = Case4(dtype, news=[0] * len(kw["lens"]), **kw, seed=_seed(dtype, str(kw)))
    cache, ws = c.cache(S), c.workspace(S)
    for rows in sorted({1, max(c.lens) - 3, max(c.lens), max(c.lens) + 21}):
        if rows < 1:
            continue
        keys = torch.full((c.B, c.Hkv, rows, c.d), -7.0, dtype=TORCH[dtype], device="cuda")
        values = keys.clone()
        S.page_read(c.dims(S), cache, rows, ws, keys=keys, values=values)
        for name, got in (("k", keys), ("v", values)):
            want = torch.full(got.shape, -7.0, dtype=torch.float64)
            for b in range(c.B):
                for g in range(c.Hkv):
                    n = min(c.lens[b], rows)
                    want[b, g, :n] = c.dense(name, b, g)[0][:n]
            assert torch.equal(got.cpu().double(), want), (rows, name)
    assert ws.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_every_code_and_exponent(S, dtype):
    """All codes under all exponents that are stored, and blocks of NaN."""
    c = Case4(dtype, [256], [0], dim=128, page=256, kv_heads=1, group=1)
    pair = torch.arange(64) * 37 % 256
    for name in "kv":
        for t in range(256):
            E = torch.tensor([min(max(t, 2), 252), 254 - min(max(t, 2), 252), 127, 255])
            c.put(name, int(c.table[0, 0]), t, ((pair + t) % 256).to(torch.uint8), E.to(torch.uint8))
    keys, values = S.page_read(c.dims(S), c.cache(S), 256, c.workspace(S))
    for got, name in ((keys, "k"), (values, "v")):
        want = c.dense(name, 0, 0)[0]
        got = got[0, 0].cpu().double()
        assert torch.equal(got.isnan(), want.isnan()) and want.isnan().sum() == 256 * 32
        assert torch.equal(got.nan_to_num(), want.nan_to_num())


def test_read_skips_bad_pages(S):
    c = Case4("bf16", [40, 20], [0, 0])
    c.table[0, 1], c.table[1, 0] = c.n_pages, -5
    ws = c.workspace(S)
    keys, values = S.page_read(c.dims(S), c.cache(S), 48, ws)
    assert ws.status() == 8
    for got, name in ((keys, "k"), (values, "v")):
        for b, g in ((0, 0), (0, 1), (1, 0), (1, 1)):
            x, ok = c.dense(name, b, g)
            x[~ok] = 0.0
            assert torch.equal(got[b, g, :c.lens[b]].cpu().double(), x)
            assert not got[b, g, c.lens[b]:].any()


def _attend(S, c):
    ws = c.workspace(S)
    out = torch.full((c.total, c.Hkv * c.G, c.d), 3.0, dtype=TORCH[c.dtype], device="cuda")
    lse = torch.full((c.total, c.Hkv * c.G), 5.0, dtype=torch.float32, device="cuda")
    S.page_attend(c.dims(S), c.cache(S), _strided(c, "q"), c.tok_start(), ws, out=out, lse=lse)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), ws.status()


def _check_attend(S, c, bits=0):
    out, lse, status = _attend(S, c)
    ref, rl, tol, ltol = c.attend()
    n = c.start[-1]
    err, lerr = (out.double() - ref).abs()[:n], (lse.double() - rl)[:n]
    ratio = (err / tol[:n].clamp(min=1e-300)).max().item() if n else 0.0
    empty = rl[:n] == -math.inf
    assert torch.equal(lse[:n] == -math.inf, empty)
    lratio = (lerr[~empty].abs() / ltol[:n][~empty]).max().item() if (~empty).any() else 0.0
    banner(f"  error / bound: out {ratio:.3f}, lse {lratio:.3f}")
    assert ratio <= 1.0 and lratio <= 1.0
    assert not out[:n][empty].any()
    assert (out[n:] == 3.0).all() and (lse[n:] == 5.0).all()       # rows behind the last sequence
    assert status == bits


ATTENDS = [
    dict(lens=[1], news=[1]),
    dict(lens=[2, 1, 0, 65], news=[1, 1, 0, 1], group=1, kv_heads=3),
    dict(lens=[63, 64, 65, 129], news=[1, 1, 1, 1], group=8, kv_heads=1),
    dict(lens=[1000, 3, 517], news=[1, 1, 1], dim=128, page=64),
    dict(lens=[300, 40], news=[4, 2], group=4, dim=128, page=32, strided=True),
    dict(lens=[300, 17, 90], news=[5, 17, 0], group=8, dim=64, page=16),
    dict(lens=[200, 160], news=[33, 160], group=4, dim=128, page=16, tail=3),
    dict(lens=[131], news=[131], group=1, kv_heads=2, page=128),
    dict(lens=[3, 70], news=[5, 90], group=2),                             # rows before the first token
    dict(lens=[700], news=[150], group=2, dim=128, page=256, window=100),
    dict(lens=[260, 99], news=[1, 20], group=4, window=1),
    dict(lens=[600, 90, 40], news=[1, 3, 40], group=4, dim=128, window=65, page=32),
    dict(lens=[5000], news=[1], group=4, kv_heads=1, dim=128, page=64),
    dict(lens=[2500, 31], news=[20, 31], group=4, kv_heads=1, dim=64, page=16, strided=True),
    dict(lens=[70, 41], news=[1, 37], group=4, dim=128, spread=8.0),       # weights of one entry almost
    dict(lens=[2000] + [30] * 7, news=[40] + [1] * 7, group=4, kv_heads=1, dim=128),   # one wide tile among narrow ones
    dict(lens=[3000], news=[4], group=4, kv_heads=4, page=1024, dim=64),
    dict(lens=[1500, 1400], news=[12, 3], group=4, kv_heads=1, dim=128, page=64, window=700),
    dict(lens=[900, 64], news=[64, 64], group=1, kv_heads=4, dim=128, page=32),
    dict(lens=[777], news=[200], group=8, kv_heads=1, dim=64, page=64),
    # no more tokens than sequences: one each, and all of them in a few
    dict(lens=[9000, 5000, 7777, 8192, 6001, 9000, 9000, 8999], news=[1] * 8, kv_heads=8, dim=128, page=64),
    dict(lens=[4100, 3900, 4097, 4000] * 5, news=[1] * 20, kv_heads=4, group=8, dim=64, page=16),
    dict(lens=[700] + [20] * 39, news=[40] + [0] * 39, group=4, dim=128, page=32),
    dict(lens=[700, 90] + [20] * 58, news=[40, 17] + [0] * 57 + [1], group=8, kv_heads=1, dim=64, page=16, window=300),
    dict(lens=[60, 900] + [0] * 9, news=[5, 6] + [0] * 9, group=8, kv_heads=3, dim=128, page=16),
    # wide tiles behind narrow ones and none: of 64 sequences they start first, of 65 in order
    dict(lens=[50] * 40 + [700] + [0] * 20 + [400, 30, 600], news=[1] * 40 + [100] + [0] * 20 + [40, 1, 150], kv_heads=3, dim=128),
    dict(lens=[50] * 40 + [700] + [0] * 21 + [400, 30, 600], news=[1] * 40 + [100] + [0] * 21 + [40, 1, 150], kv_heads=3, dim=64),
    dict(lens=[900, 800, 1000], news=[1, 0, 333], kv_heads=4, group=2, dim=64, window=300),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", ATTENDS, ids=lambda k: f"{k['lens']}{k['news']}".replace(" ", ""))
def test_attend(S, dtype, kw):
    banner(f"attend e2m1 {dtype} {kw}")
    _check_attend(S, Case4(dtype, **kw, seed=_seed(dtype, str(kw))))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_skips_bad_pages(S, dtype):
    for news in ([1, 1], [70, 5]):
        c = Case4(dtype, [200, 40], news, dim=128, page=16, seed=3)
        c.table[0, 2], c.table[0, 5], c.table[1, 0] = -1, c.n_pages, 2 ** 31 - 1
        _check_attend(S, c, bits=8)


FEW = [0] * 70       # empty sequences beside: no more tokens than sequences
SHAPES = [([1, 1], 4, 128), ([40, 6] + FEW, 4, 128), ([9, 2] + FEW, 8, 64), ([6, 3], 4, 64), ([9, 2], 4, 128), ([40, 6], 4, 128), ([150, 33], 1, 128), ([150, 33], 1, 64)]


def _hidden(c):
    """[n_pages][page]: no query sees the row."""
    seen = torch.zeros((c.n_pages, c.page), dtype=torch.bool)
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        if nq:
            first = max(0, n - nq - c.window + 1) if c.window else 0
            p, s = c.rows(b)
            seen[p[first:], s[first:]] = True
    return ~seen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("exponent,code", [(255, 0), (255, 0xff), (254, 0x77), (253, 0xf7), (0, 0x77)])
def test_rows_that_nobody_sees(S, dtype, news, group, dim, window, exponent, code):
    """Every row that no query sees holds bytes that decode to NaN or infinities: the results are those without."""
    banner(f"unseen e2m1 {dtype} {news} {group} {dim} {window} {exponent} {code}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32, window=window,
              seed=_seed(dtype, news, group, dim))
    used = set(c.table[c.table < c.n_pages].tolist())
    if 0 in used:                                    # page 0 stands in where a block holds no key
        free = next(p for p in range(c.n_pages) if p not in used)
        c.table[c.table == 0] = free
        for name in "kv":
            for x in (*c.codes[name], c.pools[name]):
                x[[0, free]] = x[[free, 0]]
    hidden = _hidden(c)
    assert hidden[0].all() and hidden.any(1).sum() > 2
    for name in "kv":
        c.codes[name][0].masked_fill_(hidden[:, None, :, None], code)
        c.codes[name][1].masked_fill_(hidden[:, None, :, None], exponent)
    _check_attend(S, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("window", [0, 60])
def test_nan_blocks_reach_those_who_see_them(S, dtype, news, group, dim, window):
    """One block of NaN in a value row that some of a chunk's queries see: the others have their value, and so
    have the other columns of those who see it.  In a key row all columns of those who see it are NaN."""
    banner(f"nan block {dtype} {news} {group} {dim} {window}")
    lens = [200, 77] + [0] * (len(news) - 2)
    for which in "vk":
        for b, t in ((0, lens[0] - 1 - news[0] // 2), (1, lens[1] - news[1]), (0, lens[0] - news[0] - 30)):
            if t < 0:
                continue
            c = Case4(dtype, lens, news, group=group, dim=dim, page=32, window=window, seed=_seed(news, group))
            ref, rl, tol, ltol = c.attend()
            page, slot = int(c.table[b, t // 32]), t % 32
            c.codes[which][1][page, :, slot, 1] = 255
            out, lse, _ = _attend(S, c)
            for i in range(c.total):
                sb = 0 if i < c.start[1] else 1
                p = lens[sb] - news[sb] + i - c.start[sb]
                sees = sb == b and t <= p and (not window or t > p - window)
                if sees and which == "k":
                    assert out[i].isnan().all(), (which, b, t, i)
                    continue
                cols = torch.ones(dim, dtype=torch.bool)
                if sees:
                    assert out[i, :, 32:64].isnan().all(), (which, b, t, i)
                    cols[32:64] = False
                assert ((out[i].double() - ref[i]).abs() <= tol[i])[:, cols].all(), (which, b, t, i)
                assert ((lse[i].double() - rl[i]).abs() <= ltol[i]).all(), (which, b, t, i)


def _two(n):
    return torch.exp2(n.double())


QUERIES = {                                              # factors of the queries [tokens][heads][dim], of the keys' exponents
    "one large value": (lambda x, g: x * torch.where(torch.arange(x.shape[-1]) == 5, 1000.0, 1.0), 0),
    "many sizes": (lambda x, g: x * _two(torch.randint(-14, 3, x.shape, generator=g)), 0),
    "one size a block": (lambda x, g: x * _two(torch.randint(-30, 3, x.shape[:-1] + (x.shape[-1] // 32, 1), generator=g)
                                               .expand(*x.shape[:-1], x.shape[-1] // 32, 32).flatten(-2)), 0),
    "tiny": (lambda x, g: x * 2.0 ** -100, 100),
    "some rows tiny": (lambda x, g: x * _two(-110 * torch.randint(0, 2, x.shape[:2] + (1,), generator=g)), 0),
    "huge": (lambda x, g: x * 2.0 ** 100, -100),
    "zeros": (lambda x, g: x * 0.0, 0),
    "zeros in blocks": (lambda x, g: x * (torch.arange(x.shape[-1]) >= 32), 0),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("kind", list(QUERIES))
def test_queries_of_all_sizes(S, dtype, news, group, dim, kind):
    """Float queries are written as six pieces of a block of 32, each off by half a step of the last: what is left of a
    value is below 2^-24 of the block's largest, and a score off by that times the block's keys besides the case's bound.
    That bound takes roundings as relative; a weight, or its product with a value, that falls below 2^-126 has no bits
    there and is off by up to 2^-126 itself: over n keys 2^-126 (n + sum |v|)."""
    banner(f"queries {kind} {dtype} {news} {group} {dim}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32, seed=_seed(kind, news, dim))
    make, up = QUERIES[kind]
    c.q = make(c.q.double(), torch.Generator().manual_seed(7)).to(TORCH[dtype])
    if up:
        c.codes["k"][1].copy_((c.codes["k"][1].int() + up).clamp(2, 252).to(torch.uint8))
        c.pools["k"] = decode4(*c.codes["k"])
    ref, rl, tol, ltol = c.attend()
    for b, n in enumerate(c.lens):
        for g in range(c.Hkv if c.news[b] else 0):
            K = c.dense("k", b, g)[0].abs().unflatten(-1, (-1, 32)).sum(-1).amax(0)
            V = c.dense("v", b, g)[0].abs()
            h = slice(g * c.G, (g + 1) * c.G)
            rows = slice(c.start[b], c.start[b + 1])
            tol[rows, h] += 2.0 ** -126 * (n + V.sum(0))
            if dtype == "f32":
                err = (c.q[rows, h].double().unflatten(-1, (-1, 32)).abs().amax(-1) @ K) * 2.0 ** -24 * c.scale
                ltol[rows, h] += err
                tol[rows, h] += 2 * err[..., None] * V.amax(0)
    out, lse, status = _attend(S, c)
    ratio, lratio = ((out.double() - ref).abs() / tol).max().item(), ((lse.double() - rl).abs() / ltol).max().item()
    banner(f"  error / bound: out {ratio:.3f}, lse {lratio:.3f}")
    assert ratio <= 1.0 and lratio <= 1.0 and status == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
def test_queries_of_no_number(S, dtype, news, group, dim):
    """NaN, and an infinity beside it, in some heads' queries: their results are NaN and all others as without."""
    banner(f"queries nan {dtype} {news} {group} {dim}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32, seed=_seed(news, dim))
    ref, rl, tol, ltol = c.attend()
    bad = torch.rand(c.q.shape[:2], generator=torch.Generator().manual_seed(3)) < 0.3
    bad[0, 0], bad[-1, -1] = True, False
    c.q[..., 3][bad] = math.nan
    c.q[..., 40][bad] = -math.inf
    out, lse, _ = _attend(S, c)
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    assert ((out.double() - ref).abs() <= tol)[~bad].all() and ((lse.double() - rl).abs() <= ltol)[~bad].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
def test_infinite_queries(S, dtype, news, group, dim):
    """Infinities in some heads' queries against keys above 0: all scores -inf give zeros, any of inf no number."""
    banner(f"queries inf {dtype} {news} {group} {dim}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32, seed=_seed(news, dim))
    codes, E = c.codes["k"]
    codes[..., 1] = codes[..., 1] & 0x7f | 0x10             # value 3 of a row: positive, not 0
    c.pools["k"] = decode4(codes, E)
    ref, rl, tol, ltol = c.attend()
    pick = torch.rand(c.q.shape[:2], generator=torch.Generator().manual_seed(3))
    pick[0, 0] = 0.0
    low, high = pick < 0.2, pick > 0.8
    c.q[..., 3][low] = -math.inf
    c.q[..., 3][high] = math.inf
    out, lse, _ = _attend(S, c)
    assert not out[low].any() and (lse[low] == -math.inf).all()
    assert out[high].isnan().all() and not torch.isfinite(lse[high]).any()
    rest = ~low & ~high
    assert ((out.double() - ref).abs() <= tol)[rest].all() and ((lse.double() - rl).abs() <= ltol)[rest].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
def test_scores_past_two_to_the_26(S, dtype, news, group, dim):
    """Scores too large for the fused step are done row by row: one key wins, and its value comes back."""
    banner(f"large scores e2m1 {dtype} {news} {group} {dim}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32, seed=_seed(news, dim))
    for name in "k":
        c.codes[name][1].fill_(127 + 24)
        c.pools[name] = decode4(*c.codes[name])
    out, lse, status = _attend(S, c)
    assert status == 0
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        for g in range(c.Hkv):
            K, V = c.dense("k", b, g)[0], c.dense("v", b, g)[0]
            for i in range(nq):
                s = (c.q[c.start[b] + i, g * c.G:(g + 1) * c.G].double() @ K[:n - nq + i + 1].T) * c.scale
                top = s.topk(min(2, s.shape[1]), -1)
                for h in range(c.G):
                    # a score is off by at most 2 d 2^-24 of its summed magnitude
                    mag = (c.q[c.start[b] + i, g * c.G + h].double().abs() @ K[:n - nq + i + 1].abs().T).max() * c.scale
                    slack = 4 * c.d * 2.0 ** -24 * mag + 40
                    if s.shape[1] > 1 and top.values[h, 0] - top.values[h, 1] < slack:
                        continue
                    want = V[top.indices[h, 0]]
                    got = out[c.start[b] + i, g * c.G + h].double()
                    assert ((got - want).abs() <= 2.0 ** -8 * want.abs()).all()
                    assert abs(lse[c.start[b] + i, g * c.G + h].double() - top.values[h, 0]) <= slack


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_again_and_on_another_stream(S, dtype):
    c = Case4(dtype, [3000, 70, 9], [1, 33, 2], dim=128, kv_heads=1, group=4, page=16, seed=11)
    cache, ws, q, ts = c.cache(S), c.workspace(S), c.q.cuda(), c.tok_start()
    a, la = S.page_attend(c.dims(S), cache, q, ts, ws, want_lse=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b, lb = S.page_attend(c.dims(S), cache, q, ts, ws, want_lse=True, stream=st)
    st.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_many_items_repeat_and_replay(S):
    """More items than run at once: the same bits call after call, on a workspace that other shapes use between, and in a
    captured graph whose lengths change."""
    c = Case4("bf16", [4000 + 7 * b for b in range(40)], [1] * 40, dim=64, kv_heads=8, group=2, page=64, seed=6)
    d = Case4("bf16", [900, 31], [1, 1], dim=64, kv_heads=8, group=2, page=64, seed=7)
    cache, q, ts, ws = c.cache(S), c.q.cuda(), c.tok_start(), c.workspace(S)
    other = d.cache(S), d.q.cuda(), d.tok_start()
    want = S.page_attend(c.dims(S), cache, q, ts, ws, want_lse=True)
    ref, rl, tol, ltol = c.attend()
    assert ((want[0].cpu().double() - ref).abs() <= tol).all() and ((want[1].cpu().double() - rl).abs() <= ltol).all()
    small = S.page_attend(d.dims(S), *other[:2], other[2], ws, want_lse=True)
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
    lens = cache.seq_len.clone()
    for turn in range(6):
        got = S.page_attend(c.dims(S), cache, q, ts, ws, want_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        got = S.page_attend(d.dims(S), *other[:2], other[2], ws, want_lse=True)
        assert torch.equal(got[0], small[0]) and torch.equal(got[1], small[1])
        cache.seq_len.copy_(lens - 500 * turn)
        out.fill_(7.0)
        gr.replay()
        eager = S.page_attend(c.dims(S), cache, q, ts, ws, want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        cache.seq_len.copy_(lens)
    assert ws.status() == 0


def test_one_workspace_for_all_storages(S):
    """Captured calls on 4-bit, 8-bit and plain pages in turn on one workspace, with eager ones between."""
    from tests.page_common import Case
    cases = [Case4("bf16", [3000, 900], [1, 2], dim=128, kv_heads=2, group=8, page=16, seed=1),
             Case("bf16", "e4m3", [1500], [1], dim=64, kv_heads=7, group=1, page=16, seed=2),
             Case4("f32", [700, 1600], [40, 120], dim=64, kv_heads=3, group=2, page=32, seed=3)]
    ws = S.Workspace(None, "cuda", nbytes=max(S.page_workspace_size(c.dims(S), sum(c.news)) for c in cases))
    parts = []
    for c in cases:
        cache, q, ts, own = c.cache(S), c.q.cuda(), c.tok_start(), c.workspace(S)
        want = S.page_attend(c.dims(S), cache, q, ts, own, want_lse=True)
        out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
        S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
        parts.append((gr, c, cache, q, ts, out, lse, want))
    for turn in (0, 1, 2, 1, 0, 2, 2, 0):
        gr, c, cache, q, ts, out, lse, want = parts[turn]
        for eager in (False, True):
            out.fill_(7.0)
            lse.fill_(7.0)
            if eager:
                S.page_attend(c.dims(S), cache, q, ts, ws, out=out, lse=lse)
            else:
                gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), (turn, eager)
    assert ws.status() == 0


def test_offsets_past_2_32(S):
    """A pool of more than 2^32 bytes, 2^31 values and 2^28 exponent bytes whose last pages are used."""
    Hkv, d, page = 8, 128, 64
    n_pages = (1 << 32) // (Hkv * page * d // 2) + 24
    pd = S.make_page_dims(batch=1, n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=d, page_size=page, n_pages=n_pages,
                          max_pages=8, dtype="f32", page_dtype="e2m1", softmax_scale=d ** -0.5)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, n_pages // 2, 5, n_pages - 9, 1, 2]], dtype=torch.int32)
    cache = S.PageCache.empty(pd, table.cuda(), torch.tensor([380], dtype=torch.int32, device="cuda"))
    x = torch.randn((3, 380, Hkv, d), generator=torch.Generator().manual_seed(2))
    ws = S.Workspace(None, "cuda", nbytes=S.page_workspace_size(pd, 380))
    ts = torch.tensor([0, 380], dtype=torch.int32, device="cuda")
    S.page_append(pd, cache, x[0].cuda(), x[1].cuda(), ts, ws)
    keys, values = S.page_read(pd, cache, 380, ws)
    from tests.page4_common import encode4
    K, V = (decode4(*encode4(t)) for t in x[:2])
    assert torch.equal(keys[0].cpu().double(), K.transpose(0, 1)) and torch.equal(values[0].cpu().double(), V.transpose(0, 1))
    out, _ = S.page_attend(pd, cache, x[2].cuda(), ts, ws)
    one, _ = S.page_attend(pd, cache, x[2][-1:].cuda(), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), ws)
    s = torch.einsum("qhd,khd->hqk", x[2].double(), K) * d ** -0.5
    mag = torch.einsum("qhd,khd->hqk", x[2].double().abs(), K.abs()).amax(-1) * d ** -0.5
    s.masked_fill_(torch.ones(380, 380, dtype=torch.bool).triu(1), -math.inf)
    w = torch.softmax(s, -1)
    ref = torch.einsum("hqk,khd->qhd", w, V)
    # as Case.attend's bound: scores 2 d 2^-24 of their magnitude, sums of 380 keys, and the result's rounding
    err = 4 * d * 2.0 ** -24 * mag + 2.0 ** -22 * (2 + s.nan_to_num(neginf=0).abs().amax(-1)) + 760 * 2.0 ** -24
    tol = err.T[..., None] * torch.einsum("hqk,khd->qhd", w, V.abs()) * 1.01 + 2.0 ** -24 * ref.abs()
    assert ((out.cpu().double() - ref).abs() <= tol).all()
    assert ((one.cpu().double() - ref[-1:]).abs() <= tol[-1:]).all()
    assert ws.status() == 0


@pytest.mark.parametrize("batch", [65, 300])
def test_many_sequences(S, batch):
    g = torch.Generator().manual_seed(batch)
    lens = torch.randint(0, 200, (batch,), generator=g).tolist()
    pick = torch.tensor([0, 1, 1, 1, 5, 40])[torch.randint(0, 6, (batch,), generator=g)].tolist()
    c = Case4("bf16", lens, [min(a, b) for a, b in zip(lens, pick)], kv_heads=2, group=4, dim=64, page=16, seed=batch)
    _check_attend(S, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_builder_on_4_bit_pages(S, dtype):
    """build_layer_paged gives the bytes that build_layer gives on the rows that page_read returns."""
    c = Case4(dtype, [500, 331], [0, 0], dim=64, page=16, seed=8)
    cache, ws = c.cache(S), c.workspace(S)
    g = torch.Generator().manual_seed(3)
    H = torch.rand((2, 512), generator=g).cuda()
    H[:, ::37] += 4.0
    bd = S.make_build_dims(batch=2, n_kv_heads=2, head_dim=64, max_tokens=512, rank=16, sketch=24, min_span=8, window=32,
                           dtype=dtype)
    omega = torch.randn((64, 24), generator=g).cuda()
    keys, values = S.page_read(c.dims(S), cache, 512, ws)
    a, _, la = S.build_layer_paged(bd, c.dims(S), cache, H, omega, ws)
    b, _, lb = S.build_layer(bd, keys, values, H, cache.seq_len, omega, ws)
    assert la["n_spans"].tolist() == lb["n_spans"].tolist() and ws.status() == 0
    for f in ("anchor_k", "anchor_v", "sum_k", "sum_v", "span_len", "factors", "block_off", "block_rank"):
        assert torch.equal(a[f], b[f]), f
