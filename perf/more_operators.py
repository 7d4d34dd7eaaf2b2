"""Rotary positions, storing with the rotation on the way, and 4-bit pages, as a serving program calls them.

Keys and queries come from the projections without their positions.  Each chunk's keys are rotated
and stored in pages, its queries rotated beside them (`store`; without rotation a plain append), the
queries attend to everything stored so far (`attend`; a decode step is a chunk of one token), the
stored rows are read back densely for the builder (`read`), and rows of any number of heads are
rotated by themselves (`rotate`; transposed: the gradient's way back).

Rotation: pair i of a token at position p turns by the angle a = p f_i,
  x' = s (x cos a - y sin a),  y' = s (y cos a + x sin a),
pairs (i, i + R/2) in the half layout, (2 i, 2 i + 1) in the interleaved one, over the first R values
of a head; the others stay.  Angles are formed in 64 bits: a position of 131072 times a frequency
leaves 32 bits nothing behind the point.  What is stored in fewer bits than 32 is rotated in 64 and
rounded to 32 before it is stored, so that values next to a border of the format fall on one side.

4-bit storage: a row is held as blocks of 32 values with one exponent byte each,
value = code * 2^(E - 127), codes 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, two a byte, the earlier value
in the low half; E the smallest of 2 .. 252 that brings the block's largest magnitude to at most 6.
8-bit storage: e4m3 codes with one exponent byte a row, the largest at most 448.  Pools, page tables
and positions as the paged store has them: token t of sequence b is slot t mod page of page
table[b][t div page]; query i of a sequence's n_q new tokens, with n stored, stands at n - n_q + i and
sees the keys max(0, p - window + 1) .. p.

Pools in 4 bits come back as the bytes that hold the codes, which have to be equal.
Lengths and page tables that are ragged are a case's own, the same for every seed, so that outputs of
two seeds have the same shapes.
"""

import math
import random

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 32


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, batch=1, context=32768, ragged=False, new=1, mix="same", kv_heads=8, group=4,
             dim=128, page=64, dtype="bf16", store="e2m1", window=0, lse=False, fused=False, layout="half", rot_dim=128,
             base=500000.0, stretch=1.0, scale=1.0, given=False, back=False)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest attention: one token of a short context of a small model, where latency is all
        _case("attend_1_2k_e2m1", "attend", context=2048, kv_heads=2, group=2, dim=64, page=16),
        # a full batch decoding: 32 users with up to 32K tokens each, a quarter of bfloat16's bytes
        _case("attend_1_32k_b32_e2m1", "attend", batch=32, ragged=True),
        # four users at 128K
        _case("attend_1_128k_b4_e2m1", "attend", batch=4, context=131072),
        # one chunk of a long prompt's prefill over 4-bit pages
        _case("attend_2048_32k_e2m1", "attend", new=2048, page=128, fused=True),
        # float tokens: single ones beside ragged chunks under a window, small pages, the log-sum-exp kept
        _case("attend_mixed_f32_e2m1", "attend", batch=7, context=5003, ragged=True, new=129, mix="mixed", kv_heads=4,
              group=2, page=16, dtype="f32", window=3001, lse=True),
        # a decode step's storing: one token of each of 32 users, keys and queries rotated in one call
        _case("store_1_b32_e2m1", "store", batch=32, context=8192, ragged=True, fused=True),
        # four 8K chunks rotated and stored in 4 bits, queries beside them
        _case("store_8k_b4_e2m1", "store", batch=4, context=8192, new=8192, fused=True),
        # ragged chunks of an fp32 model: half of each head interleaved, positions of the caller's own, 8-bit rows
        _case("store_ragged_f32_e4m3", "store", batch=3, context=20011, ragged=True, new=5001, mix="ragged", kv_heads=12,
              group=1, dim=64, page=16, dtype="f32", store="e4m3", layout="interleaved", rot_dim=32, base=10000.0,
              given=True),
        # the queries of a decode step of 32 users: latency
        _case("rotate_1_b32", "rotate", batch=32, ragged=True),
        # a 32K prompt's queries, frequencies stretched by 8 and the attention's factor
        _case("rotate_32k", "rotate", new=32768, stretch=8.0, scale=1.2079, fused=True),
        # the gradient's way back through a small fp32 model's chunk, a part of each head
        _case("rotate_back_f32", "rotate", batch=5, context=4099, ragged=True, new=4099, mix="ragged", kv_heads=12,
              group=1, dim=64, dtype="f32", layout="interleaved", rot_dim=48, base=10000.0, back=True),
        # four 128K prompts read back for the builder
        _case("read_128k_b4_e2m1", "read", batch=4, context=131072),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "store", "store", "rotate", "read"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, group, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 4, 4, 8]), rng.choice([64, 128, 128])
    batch = _log_int(rng, 1, 40)
    new = 1 if rng.random() < 0.35 else _log_int(rng, 2, 2048 if kind == "attend" else 8192)
    # stored rows within 2^30 values, a call's tokens within 2^27, a chunk's products within a number of operations
    new = max(1, min(new, (1 << 27) // (batch * heads * group * dim)))
    top = (1 << 30) // (batch * heads * dim)
    if kind == "attend":
        top = min(top, int((4e11 if dtype == "bf16" else 2e10) / (4.0 * batch * heads * group * dim * new)))
    context = _log_int(rng, min(64, max(1, top)), max(1, min(131072, top)))
    c = _case("", kind, batch=batch, context=context, ragged=rng.random() < 0.6, new=min(new, context),
              mix=rng.choice(["same", "ragged", "mixed"]), kv_heads=heads, group=group, dim=dim,
              page=rng.choice([16, 32, 64, 128]), dtype=dtype, fused=rng.random() < 0.5,
              window=_log_int(rng, 1, context) if kind == "attend" and rng.random() < 0.25 else 0,
              lse=kind == "attend" and rng.random() < 0.5)
    if kind in ("store", "rotate"):
        c.update(layout=rng.choice(["half", "interleaved"]), rot_dim=rng.choice([dim, dim, 16 * rng.randint(1, dim // 16)]),
                 base=rng.choice([10000.0, 500000.0]), stretch=rng.choice([1.0, 1.0, 4.0, 32.0]),
                 scale=rng.choice([1.0, 1.0, 1.1386]), given=rng.random() < 0.3)
    if kind == "store":
        c["store"] = rng.choice(["e2m1", "e2m1", "e4m3", "same"])
        if c["store"] == "e2m1" and rng.random() < 0.25:
            c["layout"] = "none"                             # appended as they are
    if kind == "rotate":
        c["back"] = rng.random() < 0.4
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


def _row_bytes(case):
    d = case["dim"]
    return {"e2m1": d // 2 + d // BLOCK, "e4m3": d + 1, "same": d * BYTES[case["dtype"]]}[case["store"]]


def work(case):
    lens, news = _lengths(case)
    Hq, Hkv, d, e = case["kv_heads"] * case["group"], case["kv_heads"], case["dim"], BYTES[case["dtype"]]
    row, new, R = _row_bytes(case), sum(news), case["rot_dim"]
    if case["kind"] == "rotate":
        return {"bytes": 2.0 * new * Hq * d * e, "flops": 3.0 * new * Hq * R}
    if case["kind"] == "store":
        if case["layout"] == "none":
            return {"bytes": 2.0 * new * Hkv * (d * e + row), "flops": 2.0 * new * Hkv * d}
        return {"bytes": 2.0 * new * Hkv * (d * e + row) + 2.0 * new * Hq * d * e,
                "flops": 2.0 * new * Hkv * d + 3.0 * new * (Hkv + Hq) * R}
    if case["kind"] == "read":
        return {"bytes": 2.0 * sum(lens) * Hkv * (d * e + row), "flops": 2.0 * sum(lens) * Hkv * d}
    seen = _visible(case)
    return {"bytes": 2.0 * sum(k for _, k in seen) * Hkv * row + new * Hq * (2 * d * e + (4 if case["lse"] else 0)),
            "flops": 4.0 * sum(p for p, _ in seen) * Hq * d}


# ---------------------------------------------------------------------------
# the two formats, in 32 bits
# ---------------------------------------------------------------------------

def _pow2(n):
    """2^n in 32 bits from its bits, -126 <= n <= 127: the library's power is not exact everywhere."""
    return ((n + 127).to(torch.int32) << 23).view(torch.float32)


def _codes_e4m3(x):
    """Rows of x in 32 bits as (e4m3 codes, exponent bytes)."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                  # a = m 2^e, m in [0.5, 1)
    e = e - 9 + (m > 0.875)                                # the smallest with a <= 448 * 2^e
    byte = torch.where(a > 0, (e + 127).clamp(1, 247), torch.full_like(e, 127))
    codes = (x * _pow2(127 - byte)[..., None]).to(torch.float8_e4m3fn)
    return codes, byte.to(torch.uint8)


def _codes_e2m1(x):
    """Rows of x in 32 bits as (bytes of two 4-bit codes, exponent bytes of blocks)."""
    x = x.unflatten(-1, (-1, BLOCK))
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)
    e = e - 3 + (m > 0.75)                                 # the smallest with a <= 6 * 2^e
    byte = torch.where(a > 0, (e + 127).clamp(2, 252), torch.full_like(e, 127))
    y = (x * _pow2(127 - byte)[..., None]).abs().clamp(max=6.0)
    # the number of the code: steps of 0.5 up to 2, of 1 up to 4, of 2 up to 6, ties to the even one
    c = torch.where(y < 2, torch.round(2 * y), torch.where(y < 4, torch.round(y) + 2, torch.round(0.5 * y) + 4))
    c = (c.to(torch.uint8) | (torch.signbit(x).to(torch.uint8) << 3)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), byte.to(torch.uint8)


def _values_e2m1(codes):
    """The numbers that bytes of two codes stand for, without their scale."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    m = (c & 7).float()
    v = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2, 2 * m - 8))
    return torch.where(c > 7, -v, v)


_CODES = {"e4m3": _codes_e4m3, "e2m1": _codes_e2m1}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _values(shape, gen, channel, dtype, row=0.3):
    """Normal rows: a scale of its own for each channel and each row."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= channel
    x *= torch.exp(row * torch.randn(shape[:-1] + (1,), generator=gen, device=DEV))
    return x.to(dtype)


def prepare(case, seed):
    lens, news = _lengths(case)
    B, Hkv, G, d, ps, R = case["batch"], case["kv_heads"], case["group"], case["dim"], case["page"], case["rot_dim"]
    Hq, dt, kind, store = Hkv * G, TORCH[case["dtype"]], case["kind"], case["store"]
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    per = [-(-n // ps) for n in lens]
    n_pages, max_pages = sum(per) + 3, max(per)
    start = [0]
    for q in news:
        start.append(start[-1] + q)
    total = start[-1]
    s = dict(case=case, lens=lens, news=news, max_new=max(news), tok_start=torch.tensor(start, dtype=torch.int32, device=DEV),
             seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV))
    if kind != "rotate":
        order = list(range(n_pages))
        random.Random(17).shuffle(order)
        table = torch.full((B, max_pages), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        s["table"] = table.to(DEV)
    channel = torch.exp(0.5 * torch.randn((1, Hkv, 1, d), generator=gen, device=DEV))
    shape = (n_pages, Hkv, ps, d)
    for name in "kv" if kind != "rotate" else "":
        if kind == "store":
            if store == "same":
                s[name + "_pages"], s[name + "_scale"] = torch.zeros(shape, dtype=dt, device=DEV), None
            else:
                s[name + "_pages"], s[name + "_scale"] = _CODES[store](torch.zeros(shape, device=DEV))
        else:
            s[name + "_pages"], s[name + "_scale"] = _CODES[store](_values(shape, gen, channel if name == "k" else 1.0,
                                                                           torch.float32))
    if kind in ("store", "rotate"):
        f = case["base"] ** (-torch.arange(0, R, 2, dtype=torch.float64) / R) / case["stretch"]
        s["freq"] = f.to(DEV)
        own_place = torch.cat([torch.arange(n - q, n) for n, q in zip(lens, news)])
        # a caller's own: behind a common prefix that is stored elsewhere
        s["positions"] = (own_place + 1001 if case["given"] else own_place).to(torch.int32).to(DEV)
    if kind != "read":
        ch = channel.reshape(Hkv, d)
        qkv = torch.empty((total, Hq + 2 * Hkv, d), dtype=dt, device=DEV)
        qkv[:, :Hq] = _values((total, Hq, d), gen, (2.0 / ch).repeat_interleave(G, 0), dt, 0.0)
        qkv[:, Hq:Hq + Hkv] = _values((total, Hkv, d), gen, ch, dt)
        qkv[:, Hq + Hkv:] = _values((total, Hkv, d), gen, 1.0, dt)
        parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        # a program with one projection hands over slices of its output, others three tensors
        s["q"], s["k"], s["v"] = parts if case["fused"] else [p.contiguous() for p in parts]
        if kind != "attend":
            s["q_out"] = torch.zeros((total, Hq, d), dtype=dt, device=DEV)
    else:
        s["keys"], s["values"] = (torch.zeros((B, Hkv, max(lens), d), dtype=dt, device=DEV) for _ in "kv")
    if own:
        from paper_2606_31145_amd import sekv
        if kind in ("store", "rotate") and case["layout"] != "none":
            s["rotary"] = sekv.Rotary(s["freq"], layout=case["layout"], scale=case["scale"])
        if kind != "rotate":
            s["dims"] = sekv.make_page_dims(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_size=ps,
                                            n_pages=n_pages, max_pages=max_pages, dtype=case["dtype"],
                                            page_dtype=None if store == "same" else store, window=case["window"],
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
    case = s["case"]
    if case["kind"] == "rotate":
        return {"q_out": sekv.rotate(s["q"], s["positions"], s["rotary"], out=s["q_out"], transpose=case["back"])}
    if case["kind"] == "store":
        if case["layout"] == "none":
            sekv.page_append(s["dims"], s["cache"], s["k"], s["v"], s["tok_start"], s["ws"])
        else:
            sekv.page_append_rotary(s["dims"], s["cache"], s["rotary"], s["q"], s["k"], s["v"], s["tok_start"], s["ws"],
                                    q_out=s["q_out"], positions=s["positions"] if case["given"] else None)
        return _stored(s)
    if case["kind"] == "read":
        keys, values = sekv.page_read(s["dims"], s["cache"], s["keys"].shape[2], s["ws"], keys=s["keys"],
                                      values=s["values"])
        return {"keys": keys, "values": values}
    out, lse = sekv.page_attend(s["dims"], s["cache"], s["q"], s["tok_start"], s["ws"], want_lse=case["lse"])
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _stored(s):
    r = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["k_scale"] is not None:
        r.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    if s["case"]["layout"] != "none":
        r["q_out"] = s["q_out"]
    return r


def _raw(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _turned(s, x, positions, wide):
    """x [n][heads][d] rotated: angles in 64 bits, products in 64 (wide) or 32, the result in 32."""
    case = s["case"]
    R, t = case["rot_dim"], torch.float64 if wide else torch.float32
    a = positions.double()[:, None] * s["freq"]
    c, n = (case["scale"] * a.cos()).to(t)[:, None], (case["scale"] * a.sin()).to(t)[:, None]
    if case["back"]:
        n = -n
    y = x.to(t)
    half = case["layout"] == "half"
    u, v = (y[..., :R // 2], y[..., R // 2:R]) if half else (y[..., 0:R:2], y[..., 1:R:2])
    p, q = u * c - v * n, v * c + u * n
    turned = torch.cat((p, q), -1) if half else torch.stack((p, q), -1).flatten(-2)
    return torch.cat((turned, y[..., R:]), -1).float()


def _dense(s, name, rows):
    """The first `rows` stored rows of every sequence in 32 bits, [B][Hkv][rows][d]."""
    ps, table = s["case"]["page"], s["table"]
    t = torch.arange(rows, device=DEV)
    page = table[:, (t // ps).clamp(max=table.shape[1] - 1)].clamp(min=0).long()      # [B][rows]
    x = _values_e2m1(s[name + "_pages"][page, :, t % ps])                               # [B][rows][Hkv][d]
    scale = _pow2(s[name + "_scale"][page, :, t % ps].int() - 127)
    return (x.unflatten(-1, (-1, BLOCK)) * scale[..., None]).flatten(-2).transpose(1, 2)


def _plain(s):
    case = s["case"]
    if case["kind"] == "rotate":
        s["q_out"].copy_(_turned(s, s["q"], s["positions"], False))
        return {"q_out": s["q_out"]}
    lens = s["seq_len"].long()
    start = s["tok_start"].long()
    news = start[1:] - start[:-1]
    if case["kind"] == "store":
        tok = torch.arange(s["k"].shape[0], device=DEV)
        b = torch.searchsorted(start, tok, right=True) - 1
        pos = lens[b] - news[b] + tok - start[b]
        page, slot = s["table"][b, pos // case["page"]].long(), pos % case["page"]
        turn = case["layout"] != "none"
        where = s["positions"] if case["given"] else pos
        for name in ("k", "v"):
            x = _turned(s, s["k"], where, True) if name == "k" and turn else s[name].float()
            if s["k_scale"] is None:
                s[name + "_pages"][page, :, slot] = x.to(s["k"].dtype)
            else:
                codes, byte = _CODES[case["store"]](x)
                _raw(s[name + "_pages"])[page, :, slot] = _raw(codes)
                s[name + "_scale"][page, :, slot] = byte
        if turn:
            s["q_out"].copy_(_turned(s, s["q"], where, False))
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

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _two(n):
    """2^n in 64 bits."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _row_e4m3(x):
    """e4m3 values of rows, in 64 bits, from the format's own grid."""
    a = x.abs().amax(-1)
    e = torch.zeros_like(a, dtype=torch.int64)
    big = a > 0
    e[big] = torch.ceil(torch.log2(a[big] / 448.0)).long()
    e = torch.where(big & (a > 448.0 * _two(e)), e + 1, e)           # where the logarithm was rounded
    e = torch.where(big & (a <= 448.0 * _two(e - 1)), e - 1, e).clamp(min=-126)
    y = x * _two(-e)[..., None]
    step = _two(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)    # three bits behind the first
    return torch.round(y / step) * step


def _stored_row(s, name, b, g):
    """Rows of one sequence and head in 64 bits."""
    n, ps = s["lens"][b], s["case"]["page"]
    at = s["table"][b, :-(-n // ps)].long()
    c = s[name + "_pages"][at, g].reshape(-1, s["case"]["dim"] // 2)[:n]
    grid = torch.tensor([v * sign for sign in (1, -1) for v in _E2M1], dtype=torch.float64, device=DEV)
    x = torch.empty((n, s["case"]["dim"]), dtype=torch.float64, device=DEV)
    x[:, 0::2], x[:, 1::2] = grid[(c % 16).long()], grid[torch.div(c, 16, rounding_mode="floor").long()]
    byte = s[name + "_scale"][at, g].reshape(-1, s["case"]["dim"] // BLOCK)[:n]
    return x * _two(byte.long() - 127).repeat_interleave(BLOCK, -1)


def _turned_64(s, x):
    """Rows rotated as complex numbers in 64 bits."""
    case = s["case"]
    R, x = case["rot_dim"], x.double()
    re, im = (torch.arange(R // 2), torch.arange(R // 2) + R // 2) if case["layout"] == "half" else \
        (torch.arange(0, R, 2), torch.arange(1, R, 2))
    re, im = re.to(DEV), im.to(DEV)
    angle = torch.outer(s["positions"].double(), s["freq"]) * (-1.0 if case["back"] else 1.0)
    z = torch.complex(x[..., re], x[..., im]) * torch.polar(torch.full_like(angle, case["scale"]), angle)[:, None]
    out = x.clone()
    out[..., re], out[..., im] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    Hkv, G, ps = case["kv_heads"], case["group"], case["page"]
    start = s["tok_start"].tolist()
    if case["kind"] == "rotate":
        return {"q_out": _turned_64(s, s["q"])}
    if case["kind"] == "store":
        turn, store = case["layout"] != "none", case["store"]
        # bytes of two 4-bit codes and exponent bytes are whole numbers, held to the plain form's by themselves
        r = {"k_pages": None, "v_pages": None}
        if store != "same":
            r.update(k_scale=None, v_scale=None)
        if store != "e2m1":
            for name in ("k", "v"):
                pool = s[name + "_pages"].double()
                x = _turned_64(s, s["k"]) if name == "k" and turn else s[name].double()
                x = _row_e4m3(x) if store == "e4m3" else x
                for b, (n, q) in enumerate(zip(s["lens"], s["news"])):
                    pos = torch.arange(n - q, n, device=DEV)
                    pool[s["table"][b].long()[pos // ps], :, pos % ps] = x[start[b]:start[b] + q]
                r[name + "_pages"] = pool
        if turn:
            r["q_out"] = _turned_64(s, s["q"])
        return None if all(x is None for x in r.values()) else r
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
