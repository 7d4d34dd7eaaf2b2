"""4-bit pages in plain form and 64 bits (CPU), and cases for their tests."""

import torch

from tests.page_common import Case

BLOCK = 32
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)    # by code: the format's definition


def two(n):
    """2^n in 64 bits, exact."""
    return torch.ldexp(torch.ones((), dtype=torch.float64), n.to(torch.int32))


def encode4(x):
    """(bytes of two codes, exponent bytes of blocks) of rows x [..., d], from the definition, in float64."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    a = x.abs().amax(-1)
    limit = 6.0 * two(torch.arange(2, 253) - 127)
    E = (torch.searchsorted(limit, torch.nan_to_num(a).contiguous()) + 2).clamp(max=252)  # the first limit >= a
    E = torch.where(a > 0, E, torch.full_like(E, 127))
    odd = ~torch.isfinite(x).all(-1)
    y = torch.nan_to_num(x).abs() * two(127 - E)[..., None]
    hi = torch.searchsorted(GRID, y.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    dl, dh = (y - GRID[lo]).abs(), (GRID[hi] - y).abs()
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi) + 8 * torch.signbit(x).long()
    E = torch.where(odd, torch.full_like(E, 255), E)
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), E.to(torch.uint8)


def decode4(codes, E):
    """Rows in float64; a block of exponent 255 is NaN."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    v = GRID[c % 8] * torch.where(c >= 8, -1.0, 1.0).double()
    s = torch.where(E == 255, torch.nan, two(E.long() - 127))
    return (v.unflatten(-1, (-1, BLOCK)) * s[..., None]).flatten(-2)


class Case4(Case):
    """A case whose pages hold 4 bits a value."""

    def __init__(self, dtype, lens, news, **kw):
        super().__init__(dtype, "same", lens, news, **kw)
        for name in "kv":
            self.codes[name] = encode4(self.pools[name])
            self.pools[name] = decode4(*self.codes[name])

    def dims(self, S, **kw):
        return super().dims(S, **dict(dict(page_dtype="e2m1"), **kw))

    def cache(self, S, dev="cuda"):
        t = {n: [x.to(dev).clone() for x in self.codes[n]] for n in "kv"}
        return S.PageCache(t["k"][0], t["v"][0], self.table.to(dev),
                           torch.tensor(self.lens, dtype=torch.int32, device=dev), t["k"][1], t["v"][1])

    def put(self, name, page, slot, codes, E):
        """Bytes at a place of a pool (all heads), and what they stand for."""
        c, e = self.codes[name]
        c[page, :, slot], e[page, :, slot] = codes, E
        self.pools[name][page, :, slot] = decode4(c[page, :, slot], e[page, :, slot])

    def stored(self, k, v):
        """{name: (codes, exponents)} of the pools after k, v [n_tokens][Hkv][d] are appended."""
        want = {n: [x.clone() for x in self.codes[n]] for n in "kv"}
        for b, (n, nq) in enumerate(zip(self.lens, self.news)):
            for i in range(nq):
                p = n - nq + i
                page, slot = int(self.table[b, p // self.page]) if p >= 0 else -1, p % self.page
                if not 0 <= page < self.n_pages:
                    continue
                for name, src in (("k", k), ("v", v)):
                    want[name][0][page, :, slot], want[name][1][page, :, slot] = encode4(src[self.start[b] + i])
        return want
