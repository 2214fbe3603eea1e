"""Plain 64-bit references of the serving operators (linear attention with a decay per
head, slots, verification of drafts), written from their formulas in torch float64."""
import math

import torch

EPS = 2.0 ** -24  # unit roundoff of FP32


def lin(S, q, k, v, g, lengths=None):
    """S_t = e^{g_t} S_{t-1} + k_t v_t^T, o_t = S_t^T q_t, token by token in float64.

    S [B, H, d_k, d_v]; q, k [B, T, H_qk, d_k]; v [B, T, H, d_v]; g [B, T, H] or [H].
    Returns o, S and the same computed from absolute values, which bound what the
    roundings of an FP32 evaluation are relative to."""
    B, T, H, dv = v.shape
    group = H // q.shape[2]
    length = torch.full((B,), T) if lengths is None else lengths.cpu().clamp(0, T)
    on = (torch.arange(T)[None] < length[:, None]).to(v.device)
    zero = lambda x: torch.where(on[:, :, None, None], x.double(), 0.0)
    q, k, v = zero(q).repeat_interleave(group, 2), zero(k).repeat_interleave(group, 2), zero(v)
    g = g.double().expand(B, T, H)
    # a gate below -200 is 0 in FP32 (e^-200 is 1e-87)
    a = torch.where(on[:, :, None], torch.where(g < -200, 0.0, g.exp()), 1.0)
    S, Sa = S.double(), S.double().abs()
    o, oa = torch.zeros_like(v), torch.zeros_like(v)
    for t in range(T):
        at = a[:, t, :, None, None]
        S = S * at + k[:, t, :, :, None] * v[:, t, :, None, :]
        Sa = Sa * at + (k[:, t, :, :, None] * v[:, t, :, None, :]).abs()
        o[:, t] = torch.einsum("bhk,bhkv->bhv", q[:, t], S)
        oa[:, t] = torch.einsum("bhk,bhkv->bhv", q[:, t].abs(), Sa)
    return o, S, oa, Sa


def check_lin(got, want, absolute, T, d_k, what):
    """The FP32 result against float64.  A term passes at most T decays (each a rounded
    exponential of two units, and a rounded product or sum) and d_k sums, so an element is
    within (3 T + d_k + 8) units of its absolute-value sum; rounding errors of random sign
    add up to the square root of that in the norm, within a factor of two (and 8)."""
    n = 3 * T + d_k
    err = (got.double() - want).abs()
    worst = (err - (n + 8) * EPS * absolute).max().item()
    assert worst <= 0, f"{what}: an element is {worst:g} outside its bound"
    norm, limit = err.norm().item(), (8 + 2 * math.sqrt(n)) * EPS * absolute.norm().item()
    assert norm <= limit, f"{what}: error norm {norm:g}, limit {limit:g}"


def compact(slot_idx, num_slots):
    """The new slot numbers of a compaction (python lists)."""
    live = sorted({s for s in slot_idx if 0 <= s < num_slots})
    n = len(live)
    free = [s for s in range(n) if s not in set(live)]
    to = {s: s for s in live if s < n}
    to.update(zip([s for s in live if s >= n], free))
    return [to.get(s, -1) for s in slot_idx]


def _clean(z):
    z = torch.where(z.isnan(), -math.inf, z.double())
    return z.clamp(max=torch.finfo(torch.float32).max)


def _softmax(z, t):
    z = _clean(z)
    m = z.max()
    if m == -math.inf:
        return torch.zeros_like(z)
    e = ((z - m) / t).exp()
    return e / e.sum()


def verify_row(target, draft, tokens, u, noise, t=1.0):
    """One request in float64: (tokens, margin), the margin the smallest relative distance
    of a decision from turning out otherwise."""
    out, margin = [], math.inf
    V = target.shape[-1]
    for i in range(len(tokens) + 1):
        z = _clean(target[i])
        if not t > 0:
            best = int(z.argmax()) if z.max() > -math.inf else -1  # torch: the first maximum on ties
            best = int((z == z.max()).nonzero()[0]) if best >= 0 else -1
            if i < len(tokens) and tokens[i] == best:
                out.append(best)
                continue
            return out + ([best] if best >= 0 else []), margin
        p = _softmax(target[i], t)
        r = p
        if i < len(tokens):
            x = tokens[i]
            if draft is None:
                q = torch.zeros_like(p)
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                q = _softmax(draft[i], t)
            if 0 <= x < V and p.sum() > 0:
                lhs, rhs = float(u[i]) * float(q[x]), float(p[x])
                if rhs > 0:  # a token without a probability is rejected whatever u is
                    margin = min(margin, abs(lhs - rhs) / max(lhs, rhs))
                if lhs < rhs:
                    out.append(x)
                    continue
            r = (p - q).clamp(min=0)
            if r.max() <= 0:
                r = p
        if p.sum() == 0:
            return out, margin
        # a residual p - q carries the rounding of p
        score = torch.where(r > 0, r / noise.double(), -1.0)
        top = score.topk(min(2, V))
        if V > 1 and top.values[1] > 0:
            a, b = top.indices[0], top.indices[1]
            loss = max(float(p[a] / r[a]), float(p[b] / r[b]))
            margin = min(margin, float(1 - top.values[1] / top.values[0]) / loss)
        return out + [int(top.indices[0])], margin
    raise AssertionError("not reached")
