"""The paged token store in plain form and 64 bits (CPU), and cases for its tests."""

import math

import torch

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # a rounding, relative to the value


def e4m3_grid():
    """Every non-negative finite e4m3 value, by code (float64): the format's definition."""
    v = [(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)]
    return torch.tensor(v, dtype=torch.float64)


def encode_rows(x):
    """(codes uint8, exponents uint8) of rows x [..., d], from the definition, in float64."""
    x = x.double()
    fin = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    a = fin.amax(-1)
    limit = 448.0 * torch.pow(torch.tensor(2.0, dtype=torch.float64), torch.arange(1, 248).double() - 127)
    E = torch.where(a > 0, torch.searchsorted(limit, a.contiguous()) + 1, 127)     # the first limit >= a
    y = x * torch.pow(torch.tensor(2.0, dtype=torch.float64), (127 - E).double())[..., None]
    grid = e4m3_grid()
    ya = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y))
    hi = torch.searchsorted(grid, ya.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = ya - grid[lo], grid[hi] - ya
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = torch.where(torch.isfinite(y), code, torch.full_like(code, 127))
    code = code + 128 * (torch.signbit(x) & torch.isfinite(x)).long()
    return code.to(torch.uint8), E.to(torch.uint8)


def decode_rows(codes, E):
    c = codes.long()
    grid = torch.cat([e4m3_grid(), torch.tensor([math.nan], dtype=torch.float64)])
    v = grid[c & 127] * torch.where(c >= 128, -1.0, 1.0).double()
    return v * torch.pow(torch.tensor(2.0, dtype=torch.float64), E.double() - 127.0)[..., None]


class Case:
    """Pages (host copies) and new tokens of a ragged batch."""

    def __init__(self, dtype, store, lens, news, *, kv_heads=2, group=4, dim=64, page=16, window=0, seed=0,
                 scale=None, strided=False, spread=1.0, tail=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.store, self.lens, self.news = dtype, store, list(lens), list(news)
        self.Hkv, self.G, self.d, self.page, self.window = kv_heads, group, dim, page, window
        self.B = len(lens)
        self.scale = dim ** -0.5 if scale is None else scale
        per = [-(-max(n, 0) // page) for n in lens]
        self.n_pages, self.max_pages = sum(per) + 2, max(per + [1]) + 1
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((self.B, self.max_pages), 2 ** 31 - 1, dtype=torch.int32)   # never to be read
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n].int()
            at += n
        self.start = [0]
        for q in news:
            self.start.append(self.start[-1] + q)
        self.total = self.start[-1] + tail               # rows behind the last sequence
        dt = TORCH[dtype]
        shape = (self.n_pages, kv_heads, page, dim)
        self.pools, self.codes = {}, {}
        for name in "kv":
            x = torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn((1, kv_heads, 1, dim), generator=g))
            if store == "e4m3":
                self.codes[name] = encode_rows(x)
                self.pools[name] = decode_rows(*self.codes[name])
            else:
                self.codes[name] = (x.to(dt), None)
                self.pools[name] = x.to(dt).double()
        Hq = kv_heads * group
        pad = 3 if strided else 0                        # other heads between the tokens
        wide = (spread * torch.randn((self.total, Hq + 2 * kv_heads + pad, dim), generator=g)).to(dt)
        self.q, self.k, self.v = wide[:, :Hq], wide[:, Hq:Hq + kv_heads], wide[:, Hq + kv_heads:Hq + 2 * kv_heads]
        if not strided:
            self.q, self.k, self.v = (t.contiguous() for t in (self.q, self.k, self.v))

    # ---- on the device -------------------------------------------------------------------

    def dims(self, S, **kw):
        a = dict(batch=self.B, n_q_heads=self.Hkv * self.G, n_kv_heads=self.Hkv, head_dim=self.d,
                 page_size=self.page, n_pages=self.n_pages, max_pages=self.max_pages, dtype=self.dtype,
                 page_dtype="e4m3" if self.store == "e4m3" else None, window=self.window, softmax_scale=self.scale)
        a.update(kw)
        return S.make_page_dims(**a)

    def cache(self, S, dev="cuda"):
        t = {}
        for name in "kv":
            c, e = self.codes[name]
            t[name] = (c.view(torch.float8_e4m3fn) if e is not None else c).to(dev).clone()
            t[name + "e"] = None if e is None else e.to(dev).clone()
        return S.PageCache(t["k"], t["v"], self.table.to(dev), torch.tensor(self.lens, dtype=torch.int32, device=dev),
                           t["ke"], t["ve"])

    def tok_start(self, dev="cuda"):
        return torch.tensor(self.start, dtype=torch.int32, device=dev)

    def workspace(self, S, dev="cuda"):
        return S.Workspace(None, dev, nbytes=S.page_workspace_size(self.dims(S), self.total))

    # ---- plain form ----------------------------------------------------------------------

    def rows(self, b, n=None):
        """(page, slot) of the first tokens of a sequence."""
        t = torch.arange(self.lens[b] if n is None else n)
        return self.table[b].long()[t // self.page], t % self.page

    def dense(self, name, b, g):
        p, s = self.rows(b)
        ok = (p >= 0) & (p < self.n_pages)
        return self.pools[name][p.clamp(0, self.n_pages - 1), g, s], ok

    def attend(self):
        """out, lse in float64, and bounds on what roundings may move out and lse by.

        Bound: a score is a sum of d products in float, off by at most d 2^-24 sum |q k| scale, twice
        that with the unit's own order of additions; the exponent's argument and the maximum are each
        rounded in base 2 (2^-23 |s| together); a weight then moves by twice the score's error after
        the division, by 2^-23 in exp2, and with bfloat16 by a rounding of 2^-8; the sums over n keys
        add n 2^-24 (weights) and n 2^-24 (values).  out's own rounding comes on top."""
        Hq = self.Hkv * self.G
        out = torch.zeros((self.total, Hq, self.d), dtype=torch.float64)
        lse = torch.full((self.total, Hq), -math.inf, dtype=torch.float64)
        tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
        half = HALF_STEP[self.dtype]
        for b, (n, nq) in enumerate(zip(self.lens, self.news)):
            for g in range(self.Hkv if nq and n > 0 else 0):
                K, ok = self.dense("k", b, g)
                V, _ = self.dense("v", b, g)
                for i in range(nq):
                    p = n - nq + i
                    lo = max(0, p - self.window + 1) if self.window else 0
                    see = torch.arange(lo, max(lo, p + 1))
                    see = see[ok[see]]
                    if not len(see):
                        continue
                    r = self.start[b] + i
                    q = self.q[r, g * self.G:(g + 1) * self.G].double()
                    s = (q @ K[see].T) * self.scale
                    mag = (q.abs() @ K[see].abs().T).amax(-1) * self.scale
                    z = torch.logsumexp(s, -1)
                    w = torch.exp(s - z[:, None])
                    o = w @ V[see]
                    h = slice(g * self.G, (g + 1) * self.G)
                    out[r, h], lse[r, h] = o, z
                    err_s = 2 * self.d * 2.0 ** -24 * mag + 2.0 ** -23 * s.abs().amax(-1)
                    err_w = 2 * err_s + 2 * len(see) * 2.0 ** -24 + 2.0 ** -22
                    if self.dtype == "bf16":
                        err_w = err_w + half
                    tol[r, h] = err_w[:, None] * (w @ V[see].abs()) * 1.01 + half * o.abs() * 1.01 + 1e-38
                    ltol[r, h] = err_s + (len(see) + 4) * 2.0 ** -24 + 2.0 ** -22 * z.abs().clamp(min=1)
        return out, lse, tol, ltol
