"""Float queries over 4-bit pages count with all their bits: attention stays within the bound that its roundings allow
where values of a query are of sizes far apart, and the large ones meet keys that hold zeros there."""

import zlib

import pytest
import torch

from tests.gpu_common import banner
from tests.page_common import TORCH
from tests.page4_common import Case4, decode4, encode4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2606_31145_amd import sekv
    return sekv


def _keys(c, x):
    """Keys of the whole pool, stored in 4 bits."""
    c.codes["k"] = encode4(x)
    c.pools["k"] = decode4(*c.codes["k"])


def _zeros_under(c, at):
    """Values `at` of every key become zeros; the others and their exponents stay."""
    codes, E = c.codes["k"]
    keep = torch.where(torch.arange(c.d) % 32 == at, 0, 15)
    codes &= (keep[0::2] + 16 * keep[1::2]).to(torch.uint8)
    c.pools["k"] = decode4(codes, E)


def _outlier(up):
    """A value of every block 2^up times the others; keys are zeros there."""
    def make(c, g):
        c.q = c.q.double() * torch.where(torch.arange(c.d) % 32 == 5, 2.0 ** up, 1.0)
        _zeros_under(c, 5)
    return make


def _channels(spread):
    """Keys with a scale of its own for each channel, queries with its inverse: the keys' small channels end as zeros."""
    def make(c, g):
        s = torch.exp(spread * torch.randn((1, c.Hkv, 1, c.d), generator=g, dtype=torch.float64))
        _keys(c, torch.randn(c.codes["k"][0].shape[:-1] + (c.d,), generator=g).double() * s)
        c.q = c.q.double() * (2.0 / s[0, :, 0]).repeat_interleave(c.G, 0)
    return make


def _far(c, g):
    """A block's only key value that is no zero is some 2^104, its query value some 2^-105 beside others of 1."""
    x = torch.zeros(c.codes["k"][0].shape[:-1] + (c.d,), dtype=torch.float64)
    x[..., 7::32] = 2.0 ** 104 * torch.randn(x[..., 7::32].shape, generator=g).double()
    _keys(c, x)
    c.q = c.q.double() * torch.where(torch.arange(c.d) % 32 == 7, 2.0 ** -105, 1.0)


KINDS = {"2^12": _outlier(12), "2^24": _outlier(24), "2^60": _outlier(60), "channels 1.5": _channels(1.5), "channels 3": _channels(3.0),
         "far apart": _far}
FEW = [0] * 70       # empty sequences beside: no more tokens than sequences
SHAPES = [([1, 1], 4, 128), ([1, 1], 4, 64), ([9, 2] + FEW, 8, 64), ([9, 2], 4, 128), ([40, 6], 4, 128), ([150, 33], 1, 128),
          ([150, 33], 1, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news,group,dim", SHAPES)
@pytest.mark.parametrize("kind", list(KINDS))
def test_values_of_sizes_far_apart(S, dtype, news, group, dim, kind):
    """Case.attend's bound as it stands: a score is off by its own products' roundings, however large the values are that
    meet zeros.  It takes roundings as relative; a weight, or its product with a value, that falls below 2^-126 has no bits
    there and is off by up to 2^-126 itself: over n keys 2^-126 (n + sum |v|)."""
    banner(f"far sizes {kind} {dtype} {news} {group} {dim}")
    c = Case4(dtype, [200, 77] + [0] * (len(news) - 2), news, group=group, dim=dim, page=32,
              seed=zlib.crc32(repr((kind, news, group, dim)).encode()))
    KINDS[kind](c, torch.Generator().manual_seed(7))
    c.q = c.q.to(TORCH[dtype])
    ref, rl, tol, ltol = c.attend()
    assert torch.isfinite(ref).all()
    for b, n in enumerate(c.lens):
        for g in range(c.Hkv if c.news[b] else 0):
            tol[c.start[b]:c.start[b + 1], g * c.G:(g + 1) * c.G] += 2.0 ** -126 * (n + c.dense("v", b, g)[0].abs().sum(0))
    ws = c.workspace(S)
    out, lse = S.page_attend(c.dims(S), c.cache(S), c.q.cuda(), c.tok_start(), ws, want_lse=True)
    ratio, lratio = ((out.cpu().double() - ref).abs() / tol).max().item(), ((lse.cpu().double() - rl).abs() / ltol).max().item()
    banner(f"  error / bound: out {ratio:.3f}, lse {lratio:.3f}")
    assert ratio <= 1.0 and lratio <= 1.0 and ws.status() == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 40])
def test_largest_and_smallest_floats(S, dim, n):
    """Queries of one value from the largest float to the smallest, against keys of +-1: scores that softmax_scale brings to
    ordinary sizes, or as near as it goes."""
    banner(f"largest and smallest {dim} {n}")
    big = torch.finfo(torch.float32).max
    for size, scale in ((big, 2.0 ** -99), (-big, 2.0 ** -99), (2.0 ** -90, 2.0 ** 88), (1.5 * 2.0 ** -99, 2.0 ** 98),
                        (1.0000001 * 2.0 ** -99, 2.0 ** 99), (2.0 ** -120, 2.0 ** 90), (2.0 ** -149, 2.0 ** 90)):
        c = Case4("f32", [90], [n], kv_heads=1, group=4, dim=dim, page=32, scale=scale, seed=3)
        g = torch.Generator().manual_seed(2)
        _keys(c, torch.randint(0, 2, c.codes["k"][0].shape[:-1] + (dim,), generator=g).double() * 2 - 1)
        c.q = torch.zeros(c.q.shape)
        c.q[..., 35] = size
        ref, rl, tol, ltol = c.attend()
        scores_up = scale * abs(size) * 1.4427       # in base 2
        out, lse = S.page_attend(c.dims(S), c.cache(S), c.q.cuda(), c.tok_start(), c.workspace(S), want_lse=True)
        out, lse = out.cpu().double(), lse.cpu().double()
        banner(f"  {size:g}: scores up to {scores_up:g}")
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        if scores_up < 2.0 ** 20:
            assert ((out - ref).abs() <= tol).all() and ((lse - rl).abs() <= ltol).all(), size
        else:                                                   # the largest score's keys alone count
            assert ((lse - rl).abs() <= 2.0 ** -20 * rl.abs()).all(), size
