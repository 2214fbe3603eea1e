"""Serving operators around a pool of recurrent states: cases, inputs, plain forms and exact values.

Three operators, in the forms that a server of linear-attention models calls them:

  linear attention with a decay per head   S_t = e^{g_t} S_{t-1} + k_t v_t^T,  o_t = S_t^T q_t
      kind "lin_prefill" (a chunk of a prompt) and "lin_decode" (one token), FP32 states in a slot pool
  slots of a state pool                    every layer's pool in one call
      kind "copy" (save, fork, reorder), "compact" (live slots into the lowest numbers), "free"
  verification of drafted tokens           kind "verify": accept a prefix of the draft against the
      target's probabilities, draw the next token from the residual, from given random numbers

`run` computes the plain form, or with `own` calls the framework's entry points.
"""
import math

import torch

own = False

DEVICE = "cuda"
#: Packed slot of one layer at 32 heads, d = 128, 10 FP16 key channels: 32 heads x 4 records of 4896 bytes.
PACKED_SLOT = 32 * 4 * 4896
#: Packed slot of the smallest configuration: 4 heads x 2 records of 2528 bytes (d = 64, 8 FP16 channels).
SMALL_SLOT = 4 * 2 * 2528


def listed():
    return [
        # one request of the smallest layer: the cost of a call
        {"name": "lin decode b1 h4 d64", "kind": "lin_decode", "batch": 1, "slots": 4, "heads": 4, "qk_heads": 4, "d_k": 64,
         "d_v": 64, "dtype": "fp32", "gate": "head"},
        # a full decode batch: the state's bytes
        {"name": "lin decode b256 h32 d128", "kind": "lin_decode", "batch": 256, "slots": 256, "heads": 32, "qk_heads": 32,
         "d_k": 128, "d_v": 128, "dtype": "bf16", "gate": "token"},
        # the drafted tokens of a half-full batch, run as a chunk
        {"name": "lin chunk b61 t5", "kind": "lin_prefill", "batch": 61, "slots": 128, "heads": 32, "qk_heads": 16,
         "d_k": 128, "d_v": 128, "dtype": "bf16", "gate": "token", "tokens": 5, "ragged": True},
        # a batch of short prompts of different lengths, grouped heads
        {"name": "lin prompts b64 t256", "kind": "lin_prefill", "batch": 64, "slots": 64, "heads": 32, "qk_heads": 16,
         "d_k": 128, "d_v": 128, "dtype": "bf16", "gate": "token", "tokens": 256, "ragged": True},
        # one long prompt alone: few rows, many tokens
        {"name": "lin prompt b1 t16381", "kind": "lin_prefill", "batch": 1, "slots": 8, "heads": 32, "qk_heads": 32,
         "d_k": 128, "d_v": 128, "dtype": "bf16", "gate": "head", "tokens": 16381, "ragged": False},
        # one request's state saved before a draft, a small layer: the cost of a call
        {"name": "copy 1 slot", "kind": "copy", "layers": 1, "slots": 8, "slot_bytes": SMALL_SLOT, "moves": 1, "sources": 1},
        # every layer of a prompt's state forked into 64 samples
        {"name": "fork 1 to 64, 10 layers", "kind": "copy", "layers": 10, "slots": 128, "slot_bytes": PACKED_SLOT, "moves": 64,
         "sources": 1},
        # a half-empty pool of 256 slots closed up
        {"name": "compact 131 of 256, 10 layers", "kind": "compact", "layers": 10, "slots": 256, "slot_bytes": PACKED_SLOT,
         "live": 131},
        # finished requests of every layer
        {"name": "free 37, 10 layers", "kind": "free", "layers": 10, "slots": 256, "slot_bytes": PACKED_SLOT, "moves": 37},
        # one request, four drafted tokens
        {"name": "verify b1 d4 v32000", "kind": "verify", "batch": 1, "drafts": 4, "vocab": 32000, "dtype": "fp32",
         "spread": 0.5, "greedy_every": 0},
        # a half-full batch, an odd vocabulary, some greedy requests
        {"name": "verify b61 d5 v100003", "kind": "verify", "batch": 61, "drafts": 5, "vocab": 100003, "dtype": "bf16",
         "spread": 0.5, "greedy_every": 8},
        # a full batch with a large vocabulary
        {"name": "verify b256 d3 v151552", "kind": "verify", "batch": 256, "drafts": 3, "vocab": 151552, "dtype": "bf16",
         "spread": 0.8, "greedy_every": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lin_decode", "lin_prefill", "lin_prefill", "copy", "compact", "free", "verify", "verify"])
    if kind in ("lin_decode", "lin_prefill"):
        d = rng.choice([64, 128, 128, 128])
        heads = rng.choice([4, 8, 16, 24, 32])
        case = {"kind": kind, "heads": heads, "qk_heads": heads // rng.choice([1, 2, 4]), "d_k": d, "d_v": d,
                "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "gate": rng.choice(["token", "token", "head"])}
        if kind == "lin_decode":
            case["batch"] = _log_int(rng, 1, 256)
        else:
            case["tokens"] = _log_int(rng, 2, 16381)
            most = 16384 * 32 // (case["tokens"] * heads * (2 if case["dtype"] == "fp32" else 1))
            case["batch"] = _log_int(rng, 1, min(64, max(1, most)))
            case["ragged"] = rng.random() < 0.5
        case["slots"] = case["batch"] + rng.randrange(0, 9)
        return case
    if kind in ("copy", "compact", "free"):
        slot_bytes = rng.choice([SMALL_SLOT, PACKED_SLOT, 32 * 4 * 5056, 4 * 64 * 64 * 4])
        layers = _log_int(rng, 1, 10)
        slots = rng.randrange(16, 257)
        case = {"kind": kind, "layers": layers, "slots": slots, "slot_bytes": slot_bytes}
        if kind == "compact":
            case["live"] = rng.randrange(1, slots)
        else:
            case["moves"] = _log_int(rng, 1, slots // 2)
            if kind == "copy":
                case["sources"] = rng.choice([1, case["moves"], max(1, case["moves"] // 2)])
        return case
    vocab = _log_int(rng, 8000, 151552)
    drafts = rng.randrange(1, 9)
    return {"kind": kind, "batch": _log_int(rng, 1, 256 * 9 // (2 * drafts + 3)), "drafts": drafts, "vocab": vocab,
            "dtype": rng.choice(["bf16", "bf16", "fp32"]) if vocab < 70000 else "bf16", "spread": rng.choice([0.3, 0.5, 0.8]),
            "greedy_every": rng.choice([0, 0, 8])}


def work(case):
    kind = case["kind"]
    if kind in ("lin_decode", "lin_prefill"):
        B, H, Hq, dk, dv = case["batch"], case["heads"], case["qk_heads"], case["d_k"], case["d_v"]
        es = 2 if case["dtype"] == "bf16" else 4
        T = case.get("tokens", 1)
        # ragged rows hold T/4 .. T tokens, uniformly; outputs past a row's length are written (zeros)
        tokens = B * T * (0.625 if case.get("ragged") else 1.0)
        bytes_ = 2.0 * B * H * dk * dv * 4 + tokens * (2 * Hq * dk * es + H * dv * es) + B * T * H * dv * 4
        bytes_ += tokens * H * 4 if case["gate"] == "token" else H * 4
        # a token against the state (read and update) and its half of a 64-token chunk
        pair = 0.5 * (min(T, 64) + 1) * 2 * (dk + dv) if T > 1 else 2 * (dk + dv)
        return {"bytes": bytes_, "flops": tokens * H * (4.0 * dk * dv + pair)}
    each = float(case["layers"] * case["slot_bytes"]) if "layers" in case else 0.0
    if kind == "copy":
        return {"bytes": each * (case["moves"] + case["sources"]), "flops": 0}
    if kind == "free":
        return {"bytes": each * case["moves"], "flops": 0}
    if kind == "compact":  # the expected number of live slots above the new end
        return {"bytes": 2 * each * max(1.0, case["live"] * (1 - case["live"] / case["slots"])), "flops": 0}
    B, D, V = case["batch"], case["drafts"], case["vocab"]
    es = 2 if case["dtype"] == "bf16" else 4
    greedy = B // case["greedy_every"] if case["greedy_every"] else 0
    # log-normal ratios of spread s agree with probability 2 Phi(-s/2); the rows after the first
    # rejection are not needed; a greedy request needs its first row at least
    agree = math.erfc(case["spread"] / (2 * math.sqrt(2)))
    rows = sum(2 * agree**i for i in range(D)) + agree**D
    need = (B - greedy) * V * (rows * es + 4) + greedy * V * es
    return {"bytes": need, "flops": 6.0 * rows * B * V}


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    return gen


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    if case["kind"] in ("lin_decode", "lin_prefill"):
        _prepare_lin(case, gen, state)
    elif case["kind"] == "verify":
        _prepare_verify(case, gen, state)
    else:
        _prepare_slots(case, gen, state)
    return state


def _prepare_lin(case, gen, state):
    B, H, Hq, dk, dv = case["batch"], case["heads"], case["qk_heads"], case["d_k"], case["d_v"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lead = (B,) if case["kind"] == "lin_decode" else (B, case["tokens"])

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32)

    q, k = normal(*lead, Hq, dk), normal(*lead, Hq, dk)
    state["q"] = (q / q.norm(dim=-1, keepdim=True)).to(dt)
    state["k"] = (k / k.norm(dim=-1, keepdim=True)).to(dt)
    state["v"] = normal(*lead, H, dv).to(dt)
    # heads from slow (half-lives of hundreds of tokens) to fast decay
    bias = torch.linspace(-6.0, 0.5, H, device=DEVICE)
    rates = bias if case["gate"] == "head" else bias + normal(*lead, H)
    state["g"] = -torch.nn.functional.softplus(rates)
    state["pool"] = 0.3 * normal(case["slots"], H, dk, dv)
    state["slot_idx"] = torch.randperm(case["slots"], generator=gen, device=DEVICE)[:B].to(torch.int32)
    state["lengths"] = None
    if case.get("ragged"):
        T = case["tokens"]
        state["lengths"] = torch.randint((T + 3) // 4, T + 1, (B,), generator=gen, device=DEVICE, dtype=torch.int32)


def _prepare_slots(case, gen, state):
    n = case["slots"]
    state["pools"] = [torch.randint(0, 256, (n, case["slot_bytes"]), generator=gen, device=DEVICE, dtype=torch.uint8)
                      for _ in range(case["layers"])]
    order = torch.randperm(n, generator=gen, device=DEVICE).to(torch.int32)
    if case["kind"] == "copy":
        m, s = case["moves"], case["sources"]
        state["dst"] = order[s:s + m].contiguous()
        state["src"] = order[:s].repeat_interleave(-(-m // s))[:m].contiguous()
    elif case["kind"] == "free":
        state["idx"] = order[:case["moves"]].contiguous()
    else:
        state["slot_idx"] = order[:case["live"]].contiguous()


def _prepare_verify(case, gen, state):
    B, D, V = case["batch"], case["drafts"], case["vocab"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32)

    target = 2.5 * normal(B, D + 1, V)
    draft = (target[:, :D] + case["spread"] * normal(B, D, V)).to(dt)
    state["target"] = target.to(dt)
    del target
    state["draft"] = draft
    temperature = torch.full((B,), 1.0, device=DEVICE)
    if case["greedy_every"]:
        temperature[::case["greedy_every"]] = 0.0
    state["temperature"] = temperature
    race = torch.empty(B, D, V, device=DEVICE).exponential_(generator=gen)
    state["tokens"] = (draft.float() - race.log()).argmax(-1).to(torch.int32)  # drawn from softmax(draft)
    state["u"] = torch.rand(B, D, generator=gen, device=DEVICE)
    state["noise"] = torch.empty(B, V, device=DEVICE).exponential_(generator=gen)


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2608_27513_gb300 as damp

    case = s["case"]
    kind = case["kind"]
    if kind in ("lin_decode", "lin_prefill"):
        layout = damp.Layout(case["heads"], case["qk_heads"], case["d_k"], case["d_v"], 0)
        if kind == "lin_decode":
            o = damp.lin_decode_step(layout, s["pool"], s["q"], s["k"], s["v"], s["g"], slot_idx=s["slot_idx"])
        else:
            o = damp.lin_prefill_chunk(layout, s["pool"], s["q"], s["k"], s["v"], s["g"], lengths=s["lengths"],
                                       slot_idx=s["slot_idx"])
        return {"o": o, "pool": s["pool"]}
    if kind == "copy":
        damp.copy_slots(s["pools"], s["src"], s["dst"])
        return {"pools": s["pools"]}
    if kind == "free":
        damp.zero_slots(s["pools"], s["idx"])
        return {"pools": s["pools"]}
    if kind == "compact":
        return {"slot_idx": damp.compact_slots(s["pools"], s["slot_idx"]), "pools": s["pools"]}
    tokens, count = damp.verify_drafts(s["target"], s["tokens"], s["u"], s["noise"], draft_logits=s["draft"],
                                       temperature=s["temperature"])
    return {"tokens": tokens, "count": count}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "lin_decode":
        return _plain_decode(s)
    if kind == "lin_prefill":
        return _plain_prefill(s)
    if kind == "verify":
        return _plain_verify(s)
    return _plain_slots(s)


def _plain_decode(s):
    pool, idx = s["pool"], s["slot_idx"].long()
    group = s["v"].shape[-2] // s["q"].shape[-2]
    q = s["q"].float().repeat_interleave(group, -2)
    k = s["k"].float().repeat_interleave(group, -2)
    S = pool[idx] * s["g"].exp()[..., None, None] + k[..., None] * s["v"].float()[..., None, :]
    pool[idx] = S
    return {"o": (S * q[..., None]).sum(-2), "pool": pool}


def _segment_sums(g):
    """D[i, j] = sum of g over (j, i] for j <= i, -inf above the diagonal; summed, not differenced."""
    n = g.shape[-1]
    below = torch.ones(n, n, dtype=torch.bool, device=g.device).tril(-1)
    D = torch.where(below, g[..., :, None], 0.0).cumsum(-2)
    return torch.where(below.logical_or(torch.eye(n, dtype=torch.bool, device=g.device)), D, -math.inf)


def _plain_prefill(s):
    pool, idx = s["pool"], s["slot_idx"].long()
    B, T, H, dv = s["v"].shape
    group, dk = H // s["q"].shape[2], s["q"].shape[3]
    C = 64
    N = -(-T // C)
    live = torch.ones(B, T, 1, dtype=torch.bool, device=pool.device)
    if s["lengths"] is not None:
        live = (torch.arange(T, device=pool.device) < s["lengths"][:, None])[..., None]
    g = torch.where(live, s["g"], 0.0)  # [B, T, H] from [B, T, H] or [H]

    def chunks(x):  # [B, T, H, d] -> [B, H, N, C, d], zeros past a row's length
        x = torch.where(live[..., None], x.float(), 0.0)
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, N * C - T))
        return x.reshape(B, N, C, x.shape[2], x.shape[3]).permute(0, 3, 1, 2, 4)

    q = chunks(s["q"]).repeat_interleave(group, 1)
    k = chunks(s["k"]).repeat_interleave(group, 1)
    v = chunks(s["v"])
    g = chunks(g[..., None])[..., 0]
    L = _segment_sums(g).exp()
    o = ((q @ k.transpose(-1, -2)) * L) @ v
    added = (k * L[..., -1, :, None]).transpose(-1, -2) @ v  # what each chunk adds to the state
    # states at the chunk borders, from the first state and what the chunks before added
    total = torch.nn.functional.pad(g.sum(-1), (1, 0))
    W = _segment_sums(total).exp()
    states = torch.cat([pool[idx][:, :, None], added], 2).reshape(B, H, N + 1, dk * dv)
    states = (W @ states).reshape(B, H, N + 1, dk, dv)
    o = o + (q * g.cumsum(-1).exp()[..., None]) @ states[:, :, :N]
    pool[idx] = states[:, :, N]
    o = o.permute(0, 2, 3, 1, 4).reshape(B, N * C, H, dv)[:, :T]
    return {"o": torch.where(live[..., None], o, 0.0), "pool": pool}


def _plain_slots(s):
    pools, kind = s["pools"], s["case"]["kind"]
    if kind == "copy":
        src, dst = s["src"].long(), s["dst"].long()
        for pool in pools:
            pool[dst] = pool[src]
        return {"pools": pools}
    if kind == "free":
        idx = s["idx"].long()
        for pool in pools:
            pool[idx] = 0
        return {"pools": pools}
    # live slots at or above the new end move, in order, into the free slots below it
    idx = s["slot_idx"].long()
    n = idx.shape[0]
    taken = torch.zeros(pools[0].shape[0], dtype=torch.bool, device=idx.device)
    taken[idx] = True
    holes = (~taken[:n]).nonzero()[:, 0]
    movers = taken[n:].nonzero()[:, 0] + n
    to = torch.arange(taken.shape[0], device=idx.device)
    to[movers] = holes
    for pool in pools:
        pool[holes] = pool[movers]
    return {"slot_idx": to[idx].to(torch.int32), "pools": pools}


def _plain_verify(s):
    target, draft, x = s["target"].float(), s["draft"].float(), s["tokens"].long()
    B, D = x.shape
    greedy = s["temperature"] == 0
    scale = torch.where(greedy, 1.0, 1.0 / s["temperature"])[:, None, None]

    def softmax(z):
        e = ((z - z.amax(-1, keepdim=True)) * scale).exp()
        return e / e.sum(-1, keepdim=True)

    p, q = softmax(target), softmax(draft)
    best = target.argmax(-1)
    px, qx = (z[:, :D].gather(-1, x[..., None])[..., 0] for z in (p, q))
    ok = torch.where(greedy[:, None], x == best[:, :D], s["u"] * qx < px)
    a = ok.long().cumprod(-1).sum(-1)  # accepted tokens
    row = torch.arange(B, device=x.device)
    pa = p[row, a]
    residual = (pa - q[row, a.clamp(max=D - 1)]).clamp(min=0)
    residual = torch.where(((a < D) & (residual.amax(-1) > 0))[:, None], residual, pa)
    token = torch.where(greedy, best[row, a], (residual / s["noise"]).argmax(-1))
    at = torch.arange(D + 1, device=x.device)
    out = torch.where(at < a[:, None], torch.nn.functional.pad(x, (0, 1)), -1)
    out = torch.where(at == a[:, None], token[:, None], out)
    return {"tokens": out.to(torch.int32), "count": (a + 1).to(torch.int32)}


def exact(case, seed):
    """The linear-attention recurrence token by token in 64 bits; the other operators return whole numbers only."""
    if case["kind"] not in ("lin_decode", "lin_prefill"):
        return None
    s = prepare(case, seed)
    group = case["heads"] // case["qk_heads"]
    q, k, v = (s[n].double() for n in ("q", "k", "v"))
    if case["kind"] == "lin_decode":
        q, k, v = q[:, None], k[:, None], v[:, None]
    B, T, H, _ = v.shape
    alpha = s["g"].double().exp()
    alpha = alpha.expand(B, T, H) if alpha.dim() == 1 else alpha.reshape(B, T, H)
    pool = s["pool"].double()
    idx = s["slot_idx"].long()
    S = pool[idx].reshape(B, H // group, group, q.shape[-1], v.shape[-1])
    o = torch.zeros_like(v)
    length = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, device=v.device)
    for t in range(T):
        on = (t < length)[:, None, None, None, None]
        vt = v[:, t].reshape(B, H // group, group, 1, -1)
        new = S * alpha[:, t].reshape(B, H // group, group, 1, 1) + k[:, t, :, None, :, None] * vt
        S = torch.where(on, new, S)
        out = torch.matmul(q[:, t, :, None, None, :], S)[..., 0, :]
        o[:, t] = torch.where(on[..., 0], out, 0.0).reshape(B, H, -1)
    pool[idx] = S.reshape(B, H, q.shape[-1], v.shape[-1])
    return {"o": o if case["kind"] == "lin_prefill" else o[:, 0], "pool": pool}
