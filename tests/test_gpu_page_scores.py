"""Scores of any size that a float holds: the largest one's weight is one, whatever its magnitude."""

import math
import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import HALF_STEP, Case, decode_rows, encode_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


STORES = [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")]


def _reference(c):
    """out, lse, sums of weight times magnitude, and the largest sum of the products' magnitudes that makes a
    score, in float64; the maximum is taken off first, because a sum near it would lose what the others add."""
    shape = (c.total, c.Hkv * c.G)
    out, size = (torch.zeros(shape + (c.d,), dtype=torch.float64) for _ in range(2))
    lse, mag = (torch.full(shape, -math.inf, dtype=torch.float64) for _ in range(2))
    for b, (n, nq) in enumerate(zip(c.lens, c.news)):
        for h in range(c.Hkv * c.G):
            K, V = (c.dense(name, b, h // c.G)[0] for name in "kv")
            q = c.q[c.start[b]:c.start[b + 1], h].double()
            x = (q @ K.T) * c.scale
            x[torch.arange(n) > torch.arange(n - nq, n)[:, None]] = -math.inf
            top = x.amax(-1, keepdim=True)
            w = torch.exp(x - top)
            total = w.sum(-1, keepdim=True)
            r = slice(c.start[b], c.start[b + 1])
            out[r, h], size[r, h] = w @ V / total, w @ V.abs() / total
            lse[r, h] = (top + torch.log(total))[:, 0]
            mag[r, h] = (q.abs() @ K.abs().T).amax(-1) * c.scale
    return out, lse, size, mag


@pytest.mark.parametrize("dtype,store", STORES)
@pytest.mark.parametrize("lens,news,group,dim", [([70, 9], [1, 1], 4, 64), ([900, 300], [9, 5], 4, 128), ([700], [300], 1, 128),
                                                 ([3000, 1], [1, 1], 1, 128)])
@pytest.mark.parametrize("scale,sign", [(1e30, 1), (1e30, -1), (1e12, 1), (1e9, -1), (1e7, 1), (1e3, -1), (0.3, 1), (1e-30, 1)])
def test_scores_of_any_size(S, dtype, store, lens, news, group, dim, scale, sign):
    """A key's score is its first element, exactly, so that only the weights and the output are rounded."""
    banner(f"scores {dtype} {store} {lens} {news} {scale} {sign}")
    c = Case(dtype, store, lens, news, kv_heads=2, group=group, dim=dim, page=16, scale=scale,
             seed=zlib.crc32(repr((dtype, store, lens, scale)).encode()))
    g = torch.Generator().manual_seed(5)
    x = torch.zeros_like(c.pools["k"])
    x[..., 0] = torch.randint(1, 120, x.shape[:-1], generator=g).double()
    if store == "e4m3":
        c.codes["k"] = encode_rows(x)
        c.pools["k"] = decode_rows(*c.codes["k"])
    else:
        c.codes["k"] = (x.to(c.codes["k"][0].dtype), None)
        c.pools["k"] = x
    c.q = torch.randn(c.q.shape, generator=g).to(c.q.dtype)
    c.q[..., 0] = float(sign)
    cache, ws = c.cache(S), c.workspace(S)
    out, lse = (t.cpu().double() for t in S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True))
    ref, z, size, _ = _reference(c)
    half = HALF_STEP[dtype]
    n = max(lens)
    # a weight's argument is a difference of products with a scale that is rounded to float (2^-24 of it) twice: what
    # such a difference decides stays far from the next score, or its size is small; then exp2, sums, division
    span = 120.0 * scale * 2.0 ** -22 if 120.0 * scale < 2.0 ** 20 else 0.0
    err = 2 * span + 2 * n * 2.0 ** -24 + 2.0 ** -22 + (half if dtype == "bf16" else 0.0)
    assert torch.isfinite(out).all() and ws.status() == 0
    assert ((out - ref).abs() <= 1.01 * (err * size + half * ref.abs()) + 1e-38).all()
    # lse: the scale's rounding, two products', a constant's and a sum's, 2^-24 each, make less than 2^-21
    assert ((lse - z).abs() <= 2.0 ** -21 * z.abs().clamp(min=1) + span + (n + 4) * 2.0 ** -24).all()
    assert math.isfinite(float(z.sum()))


@pytest.mark.parametrize("dtype,store", STORES)
@pytest.mark.parametrize("news,group", [([1, 1], 4), ([20, 6], 4), ([150, 33], 1)])
@pytest.mark.parametrize("low", [-1e5, -3e8, -1e10, -1e20])
def test_a_maximum_far_below_the_next(S, dtype, store, news, group, low):
    """The first 200 keys' scores are far below the others': they weigh nothing, whatever their own sums were."""
    c = Case(dtype, store, [900, 477], news, kv_heads=2, group=group, dim=128, page=16, scale=1.0,
             seed=zlib.crc32(repr((dtype, store, news, low)).encode()))
    g = torch.Generator().manual_seed(6)
    for b in range(2):
        p, s = c.rows(b)
        x = torch.zeros((c.lens[b], c.Hkv, c.d), dtype=torch.float64)
        x[..., 0] = torch.randint(-4, 5, x.shape[:-1], generator=g).double()
        x[:200, :, 0] = low * torch.randint(1, 3, (200, c.Hkv), generator=g).double()
        if store == "e4m3":
            codes, e = encode_rows(x)
            c.codes["k"][0][p, :, s], c.codes["k"][1][p, :, s] = codes, e
            c.pools["k"][p, :, s] = decode_rows(codes, e)
        else:
            c.codes["k"][0][p, :, s] = x.to(c.codes["k"][0].dtype)
            c.pools["k"][p, :, s] = c.codes["k"][0][p, :, s].double()
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 1.0
    cache, ws = c.cache(S), c.workspace(S)
    out, lse = (t.cpu().double() for t in S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True))
    ref, z, size, _ = _reference(c)
    half, n = HALF_STEP[dtype], 900
    # scores of at most 4: arguments within 6 * 2^-23, then exp2, sums, division as above
    err = 12 * 2.0 ** -23 + 2 * n * 2.0 ** -24 + 2.0 ** -22 + (half if dtype == "bf16" else 0.0)
    assert ((out - ref).abs() <= 1.01 * (err * size + half * ref.abs()) + 1e-38).all() and ws.status() == 0
    assert ((lse - z).abs() <= 2.0 ** -21 * z.abs().clamp(min=1) + 6 * 2.0 ** -23 + (n + 4) * 2.0 ** -24).all()


@pytest.mark.parametrize("dtype,store", STORES)
@pytest.mark.parametrize("news,group", [([1, 1], 4), ([20, 6], 4), ([150, 33], 1)])
@pytest.mark.parametrize("spread", [1e6, 1e10, 1e15])
def test_large_queries(S, dtype, store, news, group, spread):
    """Queries far outside any softmax's usual range: the results stay averages of values."""
    c = Case(dtype, store, [400, 77], news, group=group, dim=128, page=32, spread=spread, seed=zlib.crc32(repr((news, spread)).encode()))
    cache, ws = c.cache(S), c.workspace(S)
    out, lse = (t.cpu().double() for t in S.page_attend(c.dims(S), cache, c.q.cuda(), c.tok_start(), ws, want_lse=True))
    _, z, _, mag = _reference(c)
    # a score: d products and their order of additions, 2 d 2^-24 of the magnitudes, and three roundings behind;
    # weights follow it as far as exp lets them, so what remains to check of them is that they are weights
    assert torch.isfinite(out).all() and ws.status() == 0
    assert ((lse - z).abs() <= (2 * c.d + 8) * 2.0 ** -24 * mag + 2.0 ** -21 * z.abs().clamp(min=1) + 410 * 2.0 ** -24).all()
    for b in range(2):
        for h in range(c.Hkv):
            top = c.dense("v", b, h)[0].abs().amax()
            r = out[c.start[b]:c.start[b + 1], h * group:(h + 1) * group]
            assert (r.abs() <= top * (1 + 2.0 ** -6)).all() and (r.abs().amax(-1) > 0).all()
            last = c.start[b + 1] - 1, h * group             # where one key outweighs the rest, its value comes out
            x = (c.dense("k", b, h)[0] @ c.q[last].double()) * c.scale
            first, second = torch.topk(x, 2)[0].tolist()
            if first - second > 4 * (2 * c.d + 8) * 2.0 ** -24 * float(mag[last]) + 30:
                want = c.dense("v", b, h)[0][x.argmax()]
                assert ((out[last] - want).abs() <= 2.0 ** -7 * want.abs() + 1e-9 * top).all()
