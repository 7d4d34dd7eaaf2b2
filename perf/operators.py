"""The operators over paged key/value storage whose speed counts, as a serving program calls them.

Before a layer has its span cache, a prompt arrives in chunks.  Each chunk's keys and values are
stored in pages as they come (`append`), the chunk's queries attend to everything stored so far
(`attend`; a decode step is a chunk of one token), and in the end the stored rows are read back
densely for the builder (`read`).

Storage: pools [n_pages][Hkv][page][d]; token t of sequence b is slot t mod page of page
table[b][t div page].  Rows (one token of one head) are held as they are, or as e4m3 codes with one
exponent byte: value = code * 2^(E - 127), E the smallest that brings the row's largest magnitude
to at most 448.  Query i of a sequence's n_q new tokens, with n tokens stored, stands at position
p = n - n_q + i and sees the keys max(0, p - window + 1) .. p.

Values: channels differ in scale as real keys do, rows in length, and scores spread by about two
units, so that the softmax is neither flat nor a single entry.  Lengths and page tables that are
ragged are a case's own, the same for every seed, so that outputs of two seeds have the same shapes.
"""

import math
import random

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4, "e4m3": 1}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, batch=1, context=32768, ragged=False, new=1, mix="same", kv_heads=8, group=4,
             dim=128, page=64, dtype="bf16", store="same", window=0, lse=False, fused=False)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one token of a short fp32 context, where latency is all
        _case("attend_1_2k_f32", "attend", context=2048, kv_heads=2, group=2, dim=64, page=16, dtype="f32"),
        # a full batch decoding: 32 users with up to 32K tokens each
        _case("attend_1_32k_b32", "attend", batch=32, ragged=True),
        # four users at 128K, 8-bit pages: the bytes halved
        _case("attend_1_128k_b4_e4m3", "attend", batch=4, context=131072, store="e4m3"),
        # six drafted tokens checked at once for 16 users, a sliding window, eight query heads a KV head
        _case("attend_6_b16_window", "attend", batch=16, context=12289, ragged=True, new=6, kv_heads=4, group=8,
              page=32, store="e4m3", window=4096, lse=True, fused=True),
        # one chunk of a long prompt's prefill
        _case("attend_2048_32k", "attend", new=2048, page=128, fused=True),
        # a serving step as it comes: single tokens beside ragged chunks, small pages, 8-bit storage
        _case("attend_mixed_e4m3", "attend", batch=13, context=9001, ragged=True, new=257, mix="mixed", page=16,
              store="e4m3", lse=True, fused=True),
        # chunks of a small fp32 model without query-head groups, under a window
        _case("attend_chunk_mha_f32", "attend", batch=2, context=3001, ragged=True, new=333, kv_heads=12, group=1,
              dim=64, page=32, dtype="f32", window=1000, lse=True),
        # one new token of each of 32 users stored in 8 bits: latency
        _case("append_1_b32_e4m3", "append", batch=32, ragged=True, store="e4m3", fused=True),
        # the keys and values of four 8K chunks stored in 8 bits
        _case("append_8k_b4_e4m3", "append", batch=4, new=8192, store="e4m3", fused=True),
        # ragged chunks of an fp32 model, stored as they are
        _case("append_ragged_f32", "append", batch=3, context=20011, ragged=True, new=5001, mix="ragged", kv_heads=12,
              group=1, dim=64, page=16, dtype="f32"),
        # four 128K prompts read back for the builder from 8-bit pages
        _case("read_128k_b4_e4m3", "read", batch=4, context=131072, store="e4m3"),
        # ragged prompts of an fp32 model with head dimension 64, small pages
        _case("read_ragged_e4m3_f32", "read", batch=3, context=20011, ragged=True, dim=64, page=16, dtype="f32",
              store="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "read"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, group, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 4, 4, 8]), rng.choice([64, 128, 128])
    batch = _log_int(rng, 1, 40)
    new = 1 if rng.random() < 0.35 else _log_int(rng, 2, 2048)
    # stored rows within 2^30 values, the products of a chunk within a fixed number of operations
    top = (1 << 30) // (batch * heads * dim)
    if kind == "attend":
        top = min(top, int((4e11 if dtype == "bf16" else 2e10) / (4.0 * batch * heads * group * dim * new)))
    context = _log_int(rng, min(64, max(1, top)), max(1, min(131072, top)))
    c = _case("", kind, batch=batch, context=context, ragged=rng.random() < 0.6, new=min(new, context),
              mix=rng.choice(["same", "ragged", "mixed"]), kv_heads=heads, group=group, dim=dim,
              page=rng.choice([16, 32, 64, 128]), dtype=dtype, store=rng.choice(["same", "e4m3"]),
              window=_log_int(rng, 1, context) if kind == "attend" and rng.random() < 0.25 else 0,
              lse=kind == "attend" and rng.random() < 0.5, fused=rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(case):
    """(stored tokens, new tokens) of each sequence, the new ones among the stored."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n, q = int(case["context"]), int(case["new"])
    lens = [max(1, int(n * rng.uniform(0.2, 1.0))) if case["ragged"] and b else n for b in range(case["batch"])]
    news = []
    for b, length in enumerate(lens):
        x = q
        if case["mix"] == "ragged" and b:
            x = rng.randint(0, q)
        if case["mix"] == "mixed" and b:
            x = rng.choice([1, 1, rng.randint(1, q)])
        news.append(min(x, length))
    return lens, news


def _visible(case):
    """Per sequence: (pairs of a new token and a key that it sees, keys seen by any new token)."""
    w, out = case["window"], []
    for n, q in zip(*_lengths(case)):
        if not q:
            out.append((0, 0))
            continue
        first = n - q
        if not w:
            out.append((q * first + q * (q + 1) // 2, n))
            continue
        full = max(0, n - max(first, w - 1))          # tokens that see a whole window
        rest = q - full
        out.append((full * w + rest * (first + 1) + rest * (rest - 1) // 2, n - max(0, first - w + 1)))
    return out


def work(case):
    lens, news = _lengths(case)
    Hq, Hkv, d, e = case["kv_heads"] * case["group"], case["kv_heads"], case["dim"], BYTES[case["dtype"]]
    row = d + 1 if case["store"] == "e4m3" else d * e
    new = sum(news)
    if case["kind"] == "append":
        return {"bytes": 2.0 * new * Hkv * (d * e + row), "flops": 2.0 * new * Hkv * d}
    if case["kind"] == "read":
        return {"bytes": 2.0 * sum(lens) * Hkv * (d * e + row), "flops": 2.0 * sum(lens) * Hkv * d}
    seen = _visible(case)
    return {"bytes": 2.0 * sum(k for _, k in seen) * Hkv * row + new * Hq * (2 * d * e + (4 if case["lse"] else 0)),
            "flops": 4.0 * sum(p for p, _ in seen) * Hq * d}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _pow2(n):
    """2^n in 32 bits from its bits, -126 <= n <= 127: the library's power is not exact everywhere."""
    return ((n + 127).to(torch.int32) << 23).view(torch.float32)


def _pow2_codes(x):
    """Rows of x in 32 bits as (e4m3 codes, exponent bytes)."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                  # a = m 2^e, m in [0.5, 1)
    e = e - 9 + (m > 0.875)                                # the smallest with a <= 448 * 2^e
    byte = torch.where(a > 0, (e + 127).clamp(1, 247), torch.full_like(e, 127))
    codes = (x * _pow2(127 - byte)[..., None]).to(torch.float8_e4m3fn)
    return codes, byte.to(torch.uint8)


def _values(shape, gen, channel, dtype, row=0.3):
    """Normal rows: a scale of its own for each channel and each row."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= channel
    x *= torch.exp(row * torch.randn(shape[:-1] + (1,), generator=gen, device=DEV))
    return x.to(dtype)


def prepare(case, seed):
    lens, news = _lengths(case)
    B, Hkv, G, d, ps = case["batch"], case["kv_heads"], case["group"], case["dim"], case["page"]
    Hq, dt, quant = Hkv * G, TORCH[case["dtype"]], case["store"] == "e4m3"
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    per = [-(-n // ps) for n in lens]
    n_pages, max_pages = sum(per) + 3, max(per)
    order = list(range(n_pages))
    random.Random(17).shuffle(order)
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    start = [0]
    for q in news:
        start.append(start[-1] + q)
    s = dict(case=case, lens=lens, news=news, max_new=max(news), n_pages=n_pages, table=table.to(DEV),
             seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV),
             tok_start=torch.tensor(start, dtype=torch.int32, device=DEV))
    channel = torch.exp(0.5 * torch.randn((1, Hkv, 1, d), generator=gen, device=DEV))
    if case["kind"] == "append":
        shape = (n_pages, Hkv, ps, d)
        for name in ("k", "v"):
            s[name + "_pages"] = torch.zeros(shape, dtype=torch.float8_e4m3fn if quant else dt, device=DEV)
            s[name + "_scale"] = torch.full(shape[:-1], 127, dtype=torch.uint8, device=DEV) if quant else None
    else:
        for name in ("k", "v"):
            x = _values((n_pages, Hkv, ps, d), gen, channel if name == "k" else 1.0, torch.float32 if quant else dt)
            s[name + "_pages"], s[name + "_scale"] = _pow2_codes(x) if quant else (x, None)
            del x
    total = start[-1]
    if case["kind"] != "read":
        ch = channel.reshape(Hkv, d)
        qkv = torch.empty((total, Hq + 2 * Hkv, d), dtype=dt, device=DEV)
        qkv[:, :Hq] = _values((total, Hq, d), gen, (2.0 / ch).repeat_interleave(G, 0), dt, 0.0)
        qkv[:, Hq:Hq + Hkv] = _values((total, Hkv, d), gen, ch, dt)
        qkv[:, Hq + Hkv:] = _values((total, Hkv, d), gen, 1.0, dt)
        parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        # a program with one projection hands over slices of its output, others three tensors
        s["q"], s["k"], s["v"] = parts if case["fused"] else [p.contiguous() for p in parts]
    else:
        s["keys"], s["values"] = (torch.zeros((B, Hkv, max(lens), d), dtype=dt, device=DEV) for _ in "kv")
    if own:
        from paper_2606_31145_amd import sekv
        s["dims"] = sekv.make_page_dims(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_size=ps,
                                        n_pages=n_pages, max_pages=max_pages, dtype=case["dtype"],
                                        page_dtype="e4m3" if quant else None, window=case["window"],
                                        softmax_scale=d ** -0.5)
        s["cache"] = sekv.PageCache(s["k_pages"], s["v_pages"], s["table"], s["seq_len"], s["k_scale"], s["v_scale"])
        s["ws"] = sekv.Workspace(None, DEV, nbytes=sekv.page_workspace_size(s["dims"], total))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_2606_31145_amd import sekv
    kind = s["case"]["kind"]
    if kind == "append":
        sekv.page_append(s["dims"], s["cache"], s["k"], s["v"], s["tok_start"], s["ws"])
        return _stored(s)
    if kind == "read":
        keys, values = sekv.page_read(s["dims"], s["cache"], s["keys"].shape[2], s["ws"], keys=s["keys"],
                                      values=s["values"])
        return {"keys": keys, "values": values}
    out, lse = sekv.page_attend(s["dims"], s["cache"], s["q"], s["tok_start"], s["ws"], want_lse=s["case"]["lse"])
    return {"out": out, "lse": lse} if s["case"]["lse"] else {"out": out}


def _stored(s):
    r = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["k_scale"] is not None:
        r.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return r


def _raw(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _dense(s, name, rows):
    """The first `rows` stored rows of every sequence in 32 bits, [B][Hkv][rows][d]."""
    ps, table = s["case"]["page"], s["table"]
    t = torch.arange(rows, device=DEV)
    page = table[:, (t // ps).clamp(max=table.shape[1] - 1)].clamp(min=0).long()      # [B][rows]
    pages = s[name + "_pages"]
    x = _raw(pages)[page, :, t % ps].view(pages.dtype).float()                          # [B][rows][Hkv][d]
    if s[name + "_scale"] is not None:
        x = x * _pow2(s[name + "_scale"][page, :, t % ps].int() - 127)[..., None]
    return x.transpose(1, 2)


def _plain(s):
    case = s["case"]
    lens = s["seq_len"].long()
    start = s["tok_start"].long()
    news = start[1:] - start[:-1]
    if case["kind"] == "append":
        tok = torch.arange(s["k"].shape[0], device=DEV)
        b = torch.searchsorted(start, tok, right=True) - 1
        pos = lens[b] - news[b] + tok - start[b]
        page, slot = s["table"][b, pos // case["page"]].long(), pos % case["page"]
        for name in ("k", "v"):
            if s["k_scale"] is None:
                s[name + "_pages"][page, :, slot] = s[name]
            else:
                codes, byte = _pow2_codes(s[name].float())
                _raw(s[name + "_pages"])[page, :, slot] = _raw(codes)
                s[name + "_scale"][page, :, slot] = byte
        return _stored(s)
    if case["kind"] == "read":
        rows = s["keys"].shape[2]
        there = (torch.arange(rows, device=DEV) < lens[:, None])[:, None, :, None]
        for name, to in (("k", s["keys"]), ("v", s["values"])):
            torch.where(there, _dense(s, name, rows).to(to.dtype), to, out=to)
        return {"keys": s["keys"], "values": s["values"]}
    B, Hkv, G, d = case["batch"], case["kv_heads"], case["group"], case["dim"]
    N, Q, total = max(s["lens"]), s["max_new"], s["q"].shape[0]
    i = torch.arange(Q, device=DEV)
    tok = (start[:-1, None] + i).clamp(max=total - 1)                                   # [B][Q]
    q = s["q"][tok].float().view(B, Q, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, d)
    x = q @ _dense(s, "k", N).transpose(2, 3)
    x *= d ** -0.5
    x = x.view(B, Hkv, G, Q, N)
    j = torch.arange(N, device=DEV)
    p = (lens - news)[:, None] + i                                                      # [B][Q]
    seen = (j <= p[..., None]) & (j < lens[:, None, None])
    if case["window"]:
        seen &= j > p[..., None] - case["window"]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    x = x.sub_(m).exp_()
    total_p = x.sum(-1, keepdim=True)
    v = _dense(s, "v", N)
    v = torch.where((j < lens[:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    o = (x.view(B, Hkv, G * Q, N) @ v).view(B, Hkv, G, Q, d)
    o = torch.where(total_p > 0, o / total_p, torch.zeros_like(o))
    real = i < news[:, None]                                                            # [B][Q]
    r = {"out": o.permute(0, 3, 1, 2, 4).reshape(B, Q, Hkv * G, d)[real].to(s["q"].dtype)}
    if case["lse"]:
        r["lse"] = (m + total_p.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, Q, Hkv * G)[real]
    return r


# ---------------------------------------------------------------------------
# the same from the definition in 64 bits
# ---------------------------------------------------------------------------

def _two(n):
    """2^n in 64 bits."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _row_code(x):
    """e4m3 values and exponent of rows, in 64 bits, from the format's own grid."""
    a = x.abs().amax(-1)
    e = torch.zeros_like(a, dtype=torch.int64)
    big = a > 0
    e[big] = torch.ceil(torch.log2(a[big] / 448.0)).long()
    e = torch.where(big & (a > 448.0 * _two(e)), e + 1, e)           # where the logarithm was rounded
    e = torch.where(big & (a <= 448.0 * _two(e - 1)), e - 1, e).clamp(min=-126)
    y = x * _two(-e)[..., None]
    step = _two(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)    # three bits behind the first
    return torch.round(y / step) * step, (e + 127).to(torch.uint8)


def _stored_row(s, name, b, g):
    """Rows of one sequence and head in 64 bits."""
    n, ps = s["lens"][b], s["case"]["page"]
    at = s["table"][b, :-(-n // ps)].long()
    x = s[name + "_pages"][at, g] if s[name + "_scale"] is None else _raw(s[name + "_pages"])[at, g].view(torch.float8_e4m3fn)
    x = x.double()
    if s[name + "_scale"] is not None:
        x = x * _two(s[name + "_scale"][at, g].long() - 127)[..., None]
    return x.reshape(-1, x.shape[-1])[:n]


def exact(case, seed):
    s = prepare(case, seed)
    Hkv, G, ps = case["kv_heads"], case["group"], case["page"]
    start = s["tok_start"].tolist()
    if case["kind"] == "append":
        r = {}
        for name in ("k", "v"):
            pool = s[name + "_pages"].double()
            byte = s[name + "_scale"]
            for b, (n, q) in enumerate(zip(s["lens"], s["news"])):
                pos = torch.arange(n - q, n, device=DEV)
                rows = s["table"][b].long()[pos // ps], pos % ps
                x = s[name][start[b]:start[b] + q].double()
                if byte is not None:
                    x, e = _row_code(x)
                    byte[rows[0], :, rows[1]] = e
                pool[rows[0], :, rows[1]] = x
            r[name + "_pages"] = pool
            if byte is not None:
                r[name + "_scale"] = byte
        return r
    if case["kind"] == "read":
        r = {"keys": s["keys"].double(), "values": s["values"].double()}
        for b in range(case["batch"]):
            for g in range(Hkv):
                r["keys"][b, g, :s["lens"][b]] = _stored_row(s, "k", b, g)
                r["values"][b, g, :s["lens"][b]] = _stored_row(s, "v", b, g)
        return r
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, q) in enumerate(zip(s["lens"], s["news"])):
        if not q:
            continue
        pos = torch.arange(n - q, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)
        hidden = j > pos
        if case["window"]:
            hidden |= j < pos - case["window"] + 1
        for g in range(Hkv):
            K, V = _stored_row(s, "k", b, g), _stored_row(s, "v", b, g)
            for h in range(g * G, (g + 1) * G):
                x = s["q"][start[b]:start[b] + q, h].double() @ K.t().contiguous() / math.sqrt(case["dim"])
                x[hidden] = -math.inf
                z = torch.logsumexp(x, -1)
                lse[start[b]:start[b] + q, h] = z
                out[start[b]:start[b] + q, h] = torch.exp(x - z[:, None]) @ V
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
