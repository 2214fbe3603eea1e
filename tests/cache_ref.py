"""Plain references of the softmax-attention layers' operators, written from their definitions:
rotary positions and attention in float64, the 8-bit cache bit for bit in FP32 steps."""
import math

import numpy as np
import torch

PAGE = 32


def rotary(x, positions, freq, interleaved, scale):
    """x [B, T, H, d] float64; positions [B, T]; freq float64 [r / 2]."""
    r = 2 * len(freq)
    t = positions.double()[:, :, None, None] * freq.double()
    c, s = scale * t.cos(), scale * t.sin()
    out = x.double().clone()
    first = slice(0, r, 2) if interleaved else slice(0, r // 2)
    second = slice(1, r, 2) if interleaved else slice(r // 2, r)
    a, b = x.double()[..., first], x.double()[..., second]
    out[..., first] = a * c - b * s
    out[..., second] = b * c + a * s
    return out


def byte_of(t, e, d):
    """Where the code of value e of token t lies in the rows of a record."""
    h = ((t % 8) ^ (4 * (t % 2))) % (d // 16)
    return t * d + 16 * ((e // 16) ^ h) + e % 16


_order = {}


def order(d):
    if d not in _order:
        _order[d] = np.array([[byte_of(t, e, d) for e in range(d)] for t in range(PAGE)])
    return _order[d]


class Cache:
    """The pool as codes [2][pages, Hk, 32, d] and scales [2][pages, Hk] (keys, values)."""

    def __init__(self, pool, d):
        raw = pool.cpu().numpy()
        self.d = d
        at = order(d)
        self.codes = [raw[:, :, w * PAGE * d:(w + 1) * PAGE * d][:, :, at].copy() for w in (0, 1)]
        self.scales = [raw[:, :, 2 * PAGE * d + 4 * w:2 * PAGE * d + 4 * w + 4].copy().view(np.float32)[..., 0] for w in (0, 1)]
        self.rest = raw[:, :, 2 * PAGE * d + 8:].copy()

    def append(self, k, v, pages, start, lengths=None):
        f = np.float32
        B, T, Hk, d = k.shape
        num = self.codes[0].shape[0]
        for b in range(B):
            n = T if lengths is None else max(0, min(int(lengths[b]), T))
            s0 = int(start[b])
            if s0 < 0 or n == 0:
                continue
            for page in range(s0 // PAGE, (s0 + n - 1) // PAGE + 1):
                slot = int(pages[b, page]) if page < pages.shape[1] else -1
                if not 0 <= slot < num:
                    continue
                lo, hi = max(s0, page * PAGE), min(s0 + n, (page + 1) * PAGE)
                t0, t1 = lo - page * PAGE, hi - page * PAGE
                for w, x in enumerate((k, v)):
                    x = x[b, lo - s0:hi - s0].float().cpu().numpy().transpose(1, 0, 2)  # [Hk, n, d]
                    top = np.where(np.isfinite(x), np.abs(x), 0).max((1, 2))
                    before = self.scales[w][slot].copy() if t0 else np.zeros(Hk, f)
                    s = top / f(127)
                    s = np.where(s < np.finfo(f).tiny, f(0), s)
                    s = np.maximum(s, before)
                    with np.errstate(all="ignore"):
                        r = np.where(s > 0, f(1) / s, f(0)).astype(f)
                        y = (x * r[:, None, None]).astype(f)
                        y = np.where(np.isnan(y), f(0), np.clip(np.rint(y), -127, 127))
                        if t0:
                            old = self.codes[w][slot, :, :t0].astype(f) - 128
                            again = np.rint(old * (before * r)[:, None, None]) + 128
                            grown = (s != before)[:, None, None]
                            self.codes[w][slot, :, :t0] = np.where(grown, again, old + 128).astype(np.uint8)
                    self.codes[w][slot, :, t0:t1] = (y + 128).astype(np.uint8)
                    self.scales[w][slot] = s

    def pool(self):
        P, Hk = self.scales[0].shape
        d = self.d
        raw = np.zeros((P, Hk, 2 * PAGE * d + 16), np.uint8)
        for w in (0, 1):
            rows = np.zeros((P, Hk, PAGE * d), np.uint8)
            rows[:, :, order(d)] = self.codes[w]
            raw[:, :, w * PAGE * d:(w + 1) * PAGE * d] = rows
            raw[:, :, 2 * PAGE * d + 4 * w:2 * PAGE * d + 4 * w + 4] = self.scales[w][..., None].view(np.uint8)
        raw[:, :, 2 * PAGE * d + 8:] = self.rest
        return torch.from_numpy(raw)

    def values(self, w, table, dtype=torch.float64):
        """[len(table) * 32, Hk, d]: what the codes of the pages stand for."""
        t = torch.as_tensor(table).long()
        c = torch.from_numpy(self.codes[w])[t].to(dtype) - 128
        s = torch.from_numpy(self.scales[w])[t].to(dtype)
        return (c * s[:, :, None, None]).transpose(1, 2).reshape(-1, c.shape[1], self.d)


def attend(cache, q, pages, lengths, q_lengths=None, scale=None, window=None, num_pages=None):
    """(o, (A, X, top)): the outputs in float64, the same from |v|, the largest scale sum_i |q_i k_i| of a query,
    and the largest magnitude that a value of the row's cache can stand for."""
    B, T, H, d = q.shape
    Hk = cache.scales[0].shape[1]
    G = H // Hk
    num = cache.scales[0].shape[0]
    scale = d ** -0.5 if scale is None else scale
    o, A, X, most = (torch.zeros(B, T, H, d, dtype=torch.float64) for _ in range(4))
    for b in range(B):
        n = T if q_lengths is None else max(0, min(int(q_lengths[b]), T))
        L = max(0, min(int(lengths[b]), pages.shape[1] * PAGE))
        table = pages[b, :(L + PAGE - 1) // PAGE].cpu()
        good = (table >= 0) & (table < num)
        k, v = (cache.values(w, torch.where(good, table, 0))[:L] for w in (0, 1))
        if good.any():
            most[b] = 127.0 * float(cache.scales[1][table[good].long()].max())
        at = torch.arange(L - n, L)[:, None]
        j = torch.arange(L)
        seen = (j <= at) & good.repeat_interleave(PAGE)[:L]
        if window:
            seen &= j > at - window
        for h in range(H):
            x = q[b, :n, h].double().cpu()
            z = (x @ k[:, h // G].T) * scale
            z = z.masked_fill(~seen, -math.inf)
            top = z.amax(-1, keepdim=True) if L else torch.zeros(n, 1)
            p = (z - torch.where(top > -math.inf, top, 0.0)).exp()
            total = p.sum(-1, keepdim=True)
            p = torch.where(total > 0, p / total, 0.0)
            o[b, :n, h] = p @ v[:, h // G]
            A[b, :n, h] = p @ v[:, h // G].abs()
            big = (x.abs() @ k[:, h // G].abs().T * scale).masked_fill(~seen, 0)
            X[b, :n, h] = big.amax(-1, keepdim=True) if L else 0.0
    return o, (A, X, most)


def check_attend(got, want, bounds, keys, d, what):
    """A computed output against float64.

    A logit is a sum of d exact products, each partial sum within 2^-23 of sum |q k| (tensor cores cut,
    they do not round), plus three FP32 roundings and ex2's 2^-22: the weights are within
    e = 2 ((d + 8) 2^-23 X + 2^-22) of theirs relative to each other (numerator and denominator).  FP32 queries
    are two FP16 parts (2^-22).  A weight is rounded to FP16 (2^-11 eps, half a step: 2^-11) or to two
    parts (2^-21), and the sum over the keys adds (keys + 64) 2^-23 (a rescaling per page among them).  BF16
    outputs are rounded by half a step, 2^-8.

    FP16 has an absolute step too: weights enter as p s / 2^e 2^10, 2^e at most twice the largest scale s, and are
    rounded to a multiple of 2^-24, off by 2^-25.  In an output that is 2^-25 2^-10 2^e 127 <= 2^-34 of the
    largest value for each key (the sum of the weights is 1 at least before it divides)."""
    A, X, most = bounds
    bf = got.dtype == torch.bfloat16
    got = got.double().cpu()
    e = 2 * ((d + 8) * 2.0 ** -23 + (0 if bf else 2.0 ** -21)) * X + 2.0 ** -21
    limit = A * (e + (2.0 ** -11 if bf else 2.0 ** -20) + (keys + 64) * 2.0 ** -23) + (2.0 ** -8 if bf else 2.0 ** -24) * want.abs()
    limit = limit + keys * 2.0 ** -34 * most
    err = (got - want).abs()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    worst = (err - limit).max().item() if err.numel() else 0.0
    assert worst <= 0, f"{what}: an element is {worst:g} outside its bound (error {err.max().item():g})"
    # roundings of random sign: the norm is within their root mean square (a third of the squares' bound), doubled
    norm = err.norm().item()
    rms = ((2.0 ** -8 if bf else 2.0 ** -24) * want.norm() + (2.0 ** -11 if bf else 2.0 ** -20) * A.norm()
           + 2.0 ** -23 * (8 + 2 * math.sqrt(d + keys)) * (A * (1 + X)).norm() + keys * 2.0 ** -34 * most.norm()).item()
    assert norm <= rms, f"{what}: error norm {norm:g}, limit {rms:g}"
