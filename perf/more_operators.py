"""Softmax-attention layers between recurrent ones: cases, inputs, plain forms and exact values.

Hybrid models put a softmax-attention layer after every few recurrent layers. A server calls, per such layer:

  rotary positions of q and k          kind "rotary": both layouts, part of the head, long contexts
  a cache of 8-bit keys and values     kind "write": new tokens are quantised into the pages of their rows, and
      what the touched pages then stand for is read back (checks, hand-off to another cache)
  attention over that cache            kind "attend": one token a row, drafted tokens, prompts

The cache is a pool of pages of 32 tokens, uint8 [pages, kv heads, 64 d + 16]. A (page, head) holds the 32 key
rows of d codes, the 32 value rows, then two FP32 scales (keys, values) and 8 unused bytes. A code c stands for
(c - 128) * scale. Of a token's row the 16-byte chunk m lies at chunk m ^ h, h = (t & 7) ^ ((t & 1) << 2) for
token t of the page, masked to the chunks of a row.

`run` computes the plain form, or with `own` calls the framework's entry points.
"""
import math

import torch

own = False

DEVICE = "cuda"
PAGE = 32


def _rotary(name, batch, tokens, heads, kv_heads, d, part, far, **more):
    return {"name": name, "kind": "rotary", "batch": batch, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "d": d,
            "part": part, "far": far, "dtype": "bf16", "interleaved": False, "fused": True, "scaling": "none", **more}


def _write(name, batch, tokens, kv_heads, d, held, **more):
    return {"name": name, "kind": "write", "batch": batch, "tokens": tokens, "kv_heads": kv_heads, "d": d, "held": held,
            "dtype": "bf16", "ragged": False, **more}


def _attend(name, batch, tokens, length, heads, kv_heads, d, **more):
    return {"name": name, "kind": "attend", "batch": batch, "tokens": tokens, "length": length, "heads": heads,
            "kv_heads": kv_heads, "d": d, "dtype": "bf16", "ragged": False, "window": 0, **more}


def listed():
    return [
        # one token of one request, a small layer: the cost of a call
        _rotary("rotary b1 t1 h4 d64", 1, 1, 4, 4, 64, 64, 2048, dtype="fp32", interleaved=True, fused=False),
        # the drafted tokens of a half-full batch, a quarter of the head rotated
        _rotary("rotary b61 t5 h16/2 d256", 61, 5, 16, 2, 256, 64, 131072),
        # prompts, scaled for long contexts
        _rotary("rotary b4 t2048 h32/8 d128", 4, 2048, 32, 8, 128, 128, 262144, scaling="yarn"),
        # one token of one request, a small layer: the cost of a call
        _write("write b1 t1 kv4 d64", 1, 1, 4, 64, 40, dtype="fp32"),
        # a decode batch: a token into the open page of every row, whose scale may grow
        _write("write b256 t1 kv8 d128", 256, 1, 8, 128, 255),
        # prompts of different lengths
        _write("write b8 t2000 kv8 d128", 8, 2000, 8, 128, 100, ragged=True),
        # one token of one request, a short context, FP32: the cost of a call
        _attend("attend b1 n1000 h4 d64", 1, 1, 1000, 4, 4, 64, dtype="fp32"),
        # a decode batch of different contexts: the cache's bytes
        _attend("attend b256 n4096 h32/8 d128", 256, 1, 4096, 32, 8, 128, ragged=True),
        # one long context alone: few rows, a long axis
        _attend("attend b1 n131071 h32/8 d128", 1, 1, 131071, 32, 8, 128),
        # the drafted tokens of a half-full batch
        _attend("attend b61 t5 n2048 h16/2 d256", 61, 5, 2048, 16, 2, 256, ragged=True),
        # a piece of a long prompt
        _attend("attend b1 t4096 n32768 h32/8 d128", 1, 4096, 32768, 32, 8, 128),
        # short prompts of different lengths, each token seeing the last 512
        _attend("attend b16 t1000 n1500 h32/16 d128", 16, 1000, 1500, 32, 16, 128, ragged=True, window=512),
    ]


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rotary", "write", "attend", "attend", "attend"])
    heads, kv_heads, d = rng.choice([(4, 4, 64), (8, 2, 64), (12, 4, 128), (32, 8, 128), (32, 8, 128), (32, 16, 128),
                                     (24, 8, 128), (16, 2, 256), (16, 16, 128)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind == "rotary":
        tokens = rng.choice([1, rng.randrange(2, 9), _log_int(rng, 9, 8192)])
        batch = _log_int(rng, 1, min(256, 8192 // tokens))
        part = rng.choice([d, d, d // 2, d // 4])
        return _unnamed(_rotary("", batch, tokens, heads, kv_heads, d, part, _log_int(rng, 16384, 1 << 20), dtype=dtype,
                                interleaved=rng.random() < 0.5, fused=rng.random() < 0.7,
                                scaling=rng.choice(["none", "linear", "ntk", "yarn"])))
    if kind == "write":
        tokens = rng.choice([1, rng.randrange(2, 9), _log_int(rng, 9, 8192)])
        batch = _log_int(rng, 1, min(256, 16000 // tokens))
        return _unnamed(_write("", batch, tokens, kv_heads, d, rng.randrange(0, 300), dtype=dtype, ragged=rng.random() < 0.5))
    form = rng.choice(["one", "one", "few", "prompt"])
    window = rng.choice([0, 0, 0, _log_int(rng, 100, 4000)])
    if form == "prompt":
        tokens = _log_int(rng, 9, 4096)
        length = tokens + rng.choice([0, 0, _log_int(rng, 1, 28000)])
        most = 2_000_000_000 // (tokens * length * heads)  # scores, under the largest listed case's
        if dtype == "fp32":
            most //= 4
        batch = _log_int(rng, 1, min(16, max(1, most)))
    else:
        tokens = 1 if form == "one" else rng.randrange(2, 9)
        length = _log_int(rng, 16, 16384)
        batch = _log_int(rng, 1, min(256, max(1, 500_000_000 // (length * kv_heads * d))))
    return _unnamed(_attend("", batch, tokens, length, heads, kv_heads, d, dtype=dtype, ragged=rng.random() < 0.7, window=window))


def _shortest(case):
    """The shortest context of a ragged batch: its rows hold this many tokens .. length, uniformly."""
    return max(case["tokens"], (case["length"] + 3) // 4) if case["ragged"] else case["length"]


def work(case):
    B, T, Hk, d = case["batch"], case["tokens"], case["kv_heads"], case["d"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rotary":
        rows = B * T * (case["heads"] + Hk)
        return {"bytes": 2.0 * rows * d * es, "flops": 3.0 * rows * case["part"]}
    if case["kind"] == "write":
        # tokens read, their codes written, the touched pages' codes read and their values written
        new = B * T * (0.75 if case["ragged"] else 1.0)
        touched = new + B * (min(case["held"], PAGE - 1) / 2.0)
        return {"bytes": 2.0 * Hk * d * (new * (es + 1) + touched * (1 + es)), "flops": 2.0 * Hk * d * (3 * new + touched)}
    n = 0.5 * (_shortest(case) + case["length"])
    new = T * 0.75 if case["ragged"] and T > 8 else T
    reach = case["window"] or math.inf
    keys = min(n, reach + new - 1)  # tokens of the cache that a row of the batch reads
    pairs = sum(min(reach, n - i) for i in range(int(new)))  # the last query sees n tokens, the one before it n - 1
    bytes_ = B * Hk * keys * (2 * d + 8 / PAGE) + B * (new + T) * case["heads"] * d * es
    return {"bytes": bytes_, "flops": 4.0 * B * case["heads"] * pairs * d}


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    return gen


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    {"rotary": _prepare_rotary, "write": _prepare_write, "attend": _prepare_attend}[case["kind"]](case, gen, state)
    return state


def _frequencies(case):
    """(radians per position of each pair, factor of the rotated part), in 64 bits."""
    r, base, factor, trained = case["part"], 10000.0, 8.0, 4096
    i = torch.arange(r // 2, dtype=torch.float64, device=DEVICE)
    if case["scaling"] == "ntk":
        base *= factor ** (r / (r - 2))
    f = base ** (-2 * i / r)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] != "yarn":
        return f, 1.0
    # pairs that turn over 32 times within the trained length stay, those under once are stretched, a ramp between
    at = [r * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32.0, 1.0)]
    low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
    keep = 1 - ((i - low) / max(high - low, 0.001)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0


def _prepare_rotary(case, gen, s):
    B, T, H, Hk, d = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["d"]
    # q, k and v of a token come out of one projection, or alone
    x = torch.randn(B, T, H + 2 * Hk, d, generator=gen, device=DEVICE).to(_type(case))
    q, k = x[:, :, :H], x[:, :, H:H + Hk]
    s["q"], s["k"] = (q, k) if case["fused"] else (q.contiguous(), k.contiguous())
    start = torch.randint(0, max(1, case["far"] - T), (B, 1), generator=gen, device=DEVICE)
    s["positions"] = (start + torch.arange(T, device=DEVICE)).to(torch.int32)
    s["freq"], s["scale"] = _frequencies(case)


def _chunk_order(d):
    """order[t, p]: the logical chunk of 16 codes that lies at chunk p of token t's row, and the other way round."""
    t = torch.arange(PAGE, device=DEVICE)[:, None]
    return torch.arange(d // 16, device=DEVICE) ^ (((t & 7) ^ ((t & 1) << 2)) & (d // 16 - 1))


def _swap(rows, d):
    """Rows [..., 32, d] from their order in a page to their own, or back."""
    c = rows.reshape(*rows.shape[:-1], d // 16, 16)
    return c.gather(-2, _chunk_order(d)[..., None].expand(c.shape)).reshape(rows.shape)


def _quantise(x, scale):
    """Codes of x under a scale: rne(x * (1 / scale)) + 128, within 1 .. 255; a scale of 0 holds zeros."""
    inv = torch.where(scale > 0, torch.ones_like(scale) / torch.where(scale > 0, scale, 1.0), 0.0)
    return ((x * inv).round().clamp(-127, 127) + 128).to(torch.uint8)


def _scale_of(amax):
    s = amax / torch.full_like(amax, 127.0)
    return torch.where(s >= torch.finfo(torch.float32).tiny, s, 0.0)


def _pool(pages, Hk, d, gen):
    """A pool of written pages: keys with a few large channels, values without."""
    pool = torch.zeros(pages, Hk, 2 * PAGE * d + 16, dtype=torch.uint8, device=DEVICE)
    spread = torch.rand(Hk, 1, d, generator=gen, device=DEVICE) + 0.5
    spread[:, :, ::17] *= 3.0
    step = max(1, (1 << 26) // (Hk * PAGE * d))
    for at in range(0, pages, step):
        part = pool[at:at + step]
        n = part.shape[0]
        for which in (0, 1):
            x = torch.randn(n, Hk, PAGE, d, generator=gen, device=DEVICE)
            if which == 0:
                x = x * spread
            scale = _scale_of(x.abs().amax((-1, -2)))
            part[..., which * PAGE * d:(which + 1) * PAGE * d] = _swap(_quantise(x, scale[..., None, None]), d).reshape(n, Hk, -1)
            part[..., 2 * PAGE * d + 4 * which:2 * PAGE * d + 4 * which + 4] = scale[..., None].view(torch.uint8)
    return pool


def _tables(pool, B, W, gen):
    return torch.randperm(pool.shape[0], generator=gen, device=DEVICE)[:B * W].reshape(B, W).to(torch.int32)


def _prepare_write(case, gen, s):
    B, T, Hk, d, held = case["batch"], case["tokens"], case["kv_heads"], case["d"], case["held"]
    W = (held + T + PAGE - 1) // PAGE
    s["pool"] = _pool(B * W + 3, Hk, d, gen)
    s["pages"] = _tables(s["pool"], B, W, gen)
    x = torch.randn(B, T, 2 * Hk, d, generator=gen, device=DEVICE).to(_type(case))
    s["k"], s["v"] = x[:, :, :Hk].contiguous(), x[:, :, Hk:]  # k comes rotated, v out of the projection
    s["start"] = torch.randint(0, held + 1, (B,), generator=gen, device=DEVICE, dtype=torch.int32)
    s["new"] = torch.randint((T + 1) // 2, T + 1, (B,), generator=gen, device=DEVICE, dtype=torch.int32) if case["ragged"] else None
    new = s["new"] if case["ragged"] else torch.full_like(s["start"], T)
    # the touched pages, read back: from the start of the open page
    s["first"], s["lengths"] = s["start"] - s["start"] % PAGE, s["start"] + new
    s["read"] = T + PAGE - 1


def _prepare_attend(case, gen, s):
    B, T, H, Hk, d, n = (case[x] for x in ("batch", "tokens", "heads", "kv_heads", "d", "length"))
    W = (n + PAGE - 1) // PAGE
    s["pool"] = _pool(B * W + 3, Hk, d, gen)
    s["pages"] = _tables(s["pool"], B, W, gen)
    s["q"] = (1.5 * torch.randn(B, T, H, d, generator=gen, device=DEVICE)).to(_type(case))
    s["lengths"] = torch.full((B,), n, device=DEVICE, dtype=torch.int32)
    s["new"] = None
    if case["ragged"]:
        s["lengths"] = torch.randint(_shortest(case), n + 1, (B,), generator=gen, device=DEVICE, dtype=torch.int32)
        if T > 8:  # prompts of different lengths in one batch
            s["new"] = torch.randint((T + 1) // 2, T + 1, (B,), generator=gen, device=DEVICE, dtype=torch.int32)


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2608_27513_gb300 as damp

    case = s["case"]
    if case["kind"] == "rotary":
        q, k = damp.rotary(s["q"], s["k"], s["positions"], s["freq"], interleaved=case["interleaved"], scale=s["scale"])
        return {"q": q, "k": k}
    layout = damp.CacheLayout(case.get("heads", case["kv_heads"]), case["kv_heads"], case["d"])
    if case["kind"] == "write":
        damp.cache_append(layout, s["pool"], s["k"], s["v"], s["pages"], s["start"], lengths=s["new"])
        k, v = damp.cache_read(layout, s["pool"], s["pages"], s["lengths"], s["read"], start=s["first"], dtype=_type(case))
        return {"k": k, "v": v}
    return {"o": damp.cache_attend(layout, s["pool"], s["q"], s["pages"], s["lengths"], q_lengths=s["new"],
                                   window=case["window"] or None)}


def _run_plain(s):
    return {"rotary": _plain_rotary, "write": _plain_write, "attend": _plain_attend}[s["case"]["kind"]](s)


def _rotate(x, cos, sin, interleaved, to):
    r = 2 * cos.shape[-1]
    part, rest = x[..., :r].to(cos.dtype), x[..., r:]
    if interleaved:
        a, b = part[..., 0::2], part[..., 1::2]
        out = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = part.chunk(2, -1)
        out = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((out.to(to), rest.to(to)), -1)


def _plain_rotary(s):
    angle = s["positions"].double()[..., None, None] * s["freq"]  # 64 bits: 2^20 radians leave 32 bits nothing of the turn
    cos, sin = ((f(angle) * s["scale"]).float() for f in (torch.cos, torch.sin))
    return {n: _rotate(s[n], cos, sin, s["case"]["interleaved"], s[n].dtype) for n in ("q", "k")}


def _scales(records, d):
    """FP32 scales [..., 2] of records [..., 64 d + 16]."""
    return records[..., 2 * PAGE * d:2 * PAGE * d + 8].contiguous().view(torch.float32)


def _values(records, which, d, to):
    """What the codes of records [..., Hk, 64 d + 16] stand for, [..., Hk, 32, d]."""
    rows = records[..., which * PAGE * d:(which + 1) * PAGE * d].reshape(*records.shape[:-1], PAGE, d)
    return (_swap(rows, d).to(to) - 128) * _scales(records, d)[..., which, None, None].to(to)


def _written(s, to):
    """The pages that the new tokens go to, as the append leaves them: (rows, pages, codes and scales by which), and
    where. Computed in type `to`."""
    case = s["case"]
    B, T, Hk, d = s["k"].shape
    pool, start = s["pool"], s["start"].long()
    new = s["new"].long() if s["new"] is not None else torch.full_like(start, T)
    P = (T + PAGE - 2) // PAGE + 1  # pages that T tokens can touch
    first = start // PAGE
    page = first[:, None] + torch.arange(P, device=DEVICE)  # [B, P]
    live = (page * PAGE < (start + new)[:, None]) & (new > 0)[:, None]
    at = s["pages"].long().gather(1, page.clamp(max=s["pages"].shape[1] - 1))
    records = pool[torch.where(live, at, 0)]  # [B, P, Hk, record]
    position = page[..., None] * PAGE + torch.arange(PAGE, device=DEVICE)  # [B, P, 32]
    token = position - start[:, None, None]
    is_new, is_old = (token >= 0) & (token < new[:, None, None]), token < 0
    result = []
    for which, x in enumerate((s["k"], s["v"])):
        row = torch.arange(B, device=DEVICE)[:, None, None]
        x = x[row, token.clamp(0, T - 1)].to(to).transpose(2, 3)  # [B, P, Hk, 32, d]
        x = torch.where(is_new[:, :, None, :, None], x, 0.0)
        scale = x.abs().amax((-1, -2)) / torch.full((), 127.0, dtype=to, device=DEVICE).expand(B, P, Hk)
        scale = torch.where(scale >= torch.finfo(torch.float32).tiny, scale, 0.0)
        before = _scales(records, d)[..., which].to(to)  # an open page keeps its scale or takes a larger one
        before = torch.where(is_old.any(-1)[..., None], before, 0.0)
        scale = torch.maximum(scale, before)
        inv = torch.where(scale > 0, torch.ones_like(scale) / torch.where(scale > 0, scale, 1.0), 0.0)
        rows = records[..., which * PAGE * d:(which + 1) * PAGE * d].reshape(B, P, Hk, PAGE, d)
        old = _swap(rows, d)
        grown = (before != scale)[..., None, None] & is_old[:, :, None, :, None]
        code = torch.where(grown, ((old.to(to) - 128) * (before * inv)[..., None, None]).round() + 128, old.to(to))
        code = torch.where(is_new[:, :, None, :, None], (x * inv[..., None, None]).round().clamp(-127, 127) + 128, code)
        result.append((code, scale))
    return result, live, at, case


def _read_back(s, values, lengths, T, first):
    """Tokens first .. first + T - 1 of each row, zeros past its length, from values(page numbers) [B, P, Hk, 32, d]."""
    B = s["pages"].shape[0]
    position = first.long()[:, None] + torch.arange(T, device=DEVICE)  # from the start of a page
    x = values.transpose(2, 3).reshape(B, -1, *values.shape[2:3], values.shape[-1])  # [B, P * 32, Hk, d]
    at = (position - first.long()[:, None]).clamp(max=x.shape[1] - 1)
    x = x[torch.arange(B, device=DEVICE)[:, None], at]
    return torch.where((position < lengths.long()[:, None])[..., None, None], x, 0.0)


def _plain_write(s):
    d, pool = s["k"].shape[-1], s["pool"]
    (k, v), live, at, _ = _written(s, torch.float32)
    records = pool[torch.where(live, at, 0)]
    for which, (code, scale) in enumerate((k, v)):
        records[..., which * PAGE * d:(which + 1) * PAGE * d] = _swap(code.to(torch.uint8), d).flatten(-2)
        records[..., 2 * PAGE * d + 4 * which:2 * PAGE * d + 4 * which + 4] = scale[..., None].contiguous().view(torch.uint8)
    pool[at[live]] = records[live]
    records = pool[torch.where(live, at, 0)]
    return {n: _read_back(s, _values(records, i, d, torch.float32), s["lengths"], s["read"], s["first"]).to(_type(s["case"]))
            for i, n in enumerate(("k", "v"))}


def _attention(s, pool, table, q, lengths, new, to):
    """softmax(q k^T / sqrt(d)) v over the tokens that a query sees, for the rows of a batch, in type `to`."""
    B, T, H, d = q.shape
    Hk, window = s["case"]["kv_heads"], s["case"]["window"]
    records = pool[table.long()]  # [B, W, Hk, record]
    N = records.shape[1] * PAGE
    k, v = (_values(records, i, d, to).transpose(1, 2).reshape(B, Hk, N, d) for i in (0, 1))
    del records
    at = lengths.long()[:, None] - new.long()[:, None] + torch.arange(T, device=DEVICE)  # [B, T]
    j = torch.arange(N, device=DEVICE)
    seen = (j <= at[..., None]) & (j >= 0)
    if window:
        seen &= j > at[..., None] - window
    seen &= (torch.arange(T, device=DEVICE) < new[:, None])[..., None]
    rows = q.to(to).reshape(B, T, Hk, H // Hk, d).permute(0, 2, 3, 1, 4)  # [B, Hk, G, T, d]
    p = (rows.reshape(B, Hk, -1, d) @ k.transpose(-1, -2)).reshape(B, Hk, H // Hk, T, N)
    p.mul_(1.0 / math.sqrt(d)).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    p.div_(p.sum(-1, keepdim=True).clamp(min=torch.finfo(to).tiny))
    o = (p.reshape(B, Hk, -1, N) @ v).reshape(B, Hk, H // Hk, T, d)
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, H, d)


def _new_of(s):
    return s["new"] if s["new"] is not None else torch.full_like(s["lengths"], s["q"].shape[1])


def _plain_attend(s):
    return {"o": _attention(s, s["pool"], s["pages"], s["q"], s["lengths"], _new_of(s), torch.float32).to(s["q"].dtype)}


def exact(case, seed):
    """The definitions in 64 bits: whole turns and codes as they are, everything else without rounding."""
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        angle = s["positions"].double()[..., None, None] * s["freq"]
        z = torch.polar(torch.full_like(angle, s["scale"]), angle)  # a pair turns as a complex number
        out = {}
        for n in ("q", "k"):
            x, r = s[n].double().contiguous(), case["part"]
            pairs = x[..., :r].reshape(*x.shape[:-1], *((r // 2, 2) if case["interleaved"] else (2, r // 2)))
            pairs = pairs if case["interleaved"] else pairs.transpose(-1, -2)
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
            x[..., :r] = (turned if case["interleaved"] else turned.transpose(-1, -2)).reshape(x[..., :r].shape)
            out[n] = x
        return out
    if case["kind"] == "write":
        both = _written(s, torch.float64)[0]
        return {n: _read_back(s, (code - 128) * scale[..., None, None], s["lengths"], s["read"], s["first"])
                for n, (code, scale) in zip(("k", "v"), both)}
    # a row of the batch and a KV head at a time
    new, G, d, out = _new_of(s), case["heads"] // case["kv_heads"], case["d"], torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, (length, n) in enumerate(zip(s["lengths"].tolist(), new.tolist())):
        W = (length + PAGE - 1) // PAGE
        at = torch.arange(length - n, length, device=DEVICE)[:, None]
        j = torch.arange(length, device=DEVICE)
        hidden = (j > at) | (j <= at - case["window"]) if case["window"] else j > at
        for h in range(case["kv_heads"]):
            records = s["pool"][s["pages"][b, :W].long(), h]
            k, v = (_values(records[:, None], i, d, torch.float64).reshape(-1, d)[:length] for i in (0, 1))
            x = torch.einsum("tgd,jd->gtj", s["q"][b, :n, h * G:(h + 1) * G].double(), k) / math.sqrt(d)
            x = x.masked_fill_(hidden, -math.inf)
            p = x.sub_(x.amax(-1, keepdim=True)).exp_()
            o = torch.einsum("gtj,jd->tgd", p, v) / p.sum(-1).transpose(0, 1)[..., None]
            out[b, :n, h * G:(h + 1) * G] = o
    return {"o": out}
