"""Verification of drafted tokens on the GPU against a float64 evaluation of its rule, over
vocabularies, draft counts, types, temperatures and excluded tokens, and the distribution
of the emitted tokens against the target's."""
import math

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
#: Decisions closer than this (relative) may fall either way in FP32: a probability is
#: within a few units (2^-24) of its value, and an exponent of size 30 adds 30 of them.
MARGIN = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_27513_gb300 import build
    build.build()
    torch.cuda.init()
    assert damp.device_status() == 0
    yield
    assert damp.device_status() == 0


def _inputs(B, D, V, dtype, seed=0, spread=0.7, scale=2.0, ld=None):
    gen = torch.Generator(device=DEV).manual_seed(seed + 17 * V + D)
    n = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    ld = V if ld is None else ld
    target = scale * n(B, D + 1, ld)
    draft = (target[:, :D] + spread * n(B, D, ld)).to(dtype)
    race = torch.empty(B, D, V, device=DEV).exponential_(generator=gen)
    tokens = (draft[..., :V].float() - race.log()).argmax(-1).to(torch.int32)
    u = torch.rand(B, D, generator=gen, device=DEV)
    noise = torch.empty(B, V, device=DEV).exponential_(generator=gen)
    return target.to(dtype), draft, tokens, u, noise


def _check(target, tokens, u, noise, draft=None, temperature=None, draft_len=None, vocab=None, least=0.9):
    B, D = tokens.shape
    V = target.shape[-1] if vocab is None else vocab
    out, count = damp.verify_drafts(target, tokens, u, noise, draft_logits=draft, temperature=temperature,
                                    draft_len=draft_len, vocab=vocab)
    out, count = out.cpu(), count.cpu()
    t_, d_, x_, u_, n_ = (None if z is None else z.cpu() for z in (target, draft, tokens, u, noise))
    clear = 0
    for b in range(B):
        L = D if draft_len is None else max(0, min(D, int(draft_len[b])))
        want, margin = R.verify_row(t_[b, :, :V], None if d_ is None else d_[b, :, :V], x_[b, :L].tolist(), u_[b], n_[b],
                                    1.0 if temperature is None else float(temperature[b]))
        if margin < MARGIN:
            continue
        clear += 1
        assert out[b].tolist() == want + [-1] * (D + 1 - len(want)), (b, want, out[b].tolist())
        assert int(count[b]) == len(want)
    assert clear >= least * B
    return out, count


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 1000, 4097, 32000, 100003])
def test_vocabularies(V, dtype):
    _check(*[x for x in _order(_inputs(6, 3, V, dtype))])


def _order(x):
    target, draft, tokens, u, noise = x
    return target, tokens, u, noise, draft


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [0, 1, 2, 5, 8, 16])
@pytest.mark.parametrize("B", [1, 3, 70])
def test_draft_counts(D, B, dtype):
    _check(*_order(_inputs(B, D, 1501, dtype, seed=1, spread=0.4)))


def test_many_requests():
    _check(*_order(_inputs(400, 2, 515, torch.bfloat16, seed=2)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_temperatures(dtype):
    target, draft, tokens, u, noise = _inputs(24, 4, 3001, dtype, seed=3)
    temp = torch.tensor([0.0, 0.3, 0.7, 1.0, 1.7, 5.0, 0.05, -1.0] * 3, device=DEV)
    greedy = target[:, :4].float().argmax(-1).to(torch.int32)
    tokens = torch.where((temp <= 0)[:, None], greedy, tokens)
    tokens[0, 2] = 5
    _check(target, tokens, u, noise, draft, temperature=temp)


def test_greedy_ties_take_the_lowest_index():
    target = torch.zeros(3, 3, 5000, device=DEV)
    target[0, 0, [4000, 17, 300]] = 2.0
    target[0, 1, [4999, 4998]] = 1.0
    target[1] = -1.0
    tokens = torch.tensor([[17, 4998], [0, 1], [3, 3]], dtype=torch.int32, device=DEV)
    out, count = damp.verify_drafts(target, tokens, torch.zeros(3, 2, device=DEV), torch.ones(3, 5000, device=DEV),
                                    temperature=torch.zeros(3, device=DEV))
    assert out.tolist() == [[17, 4998, 0], [0, 0, -1], [0, -1, -1]] and count.tolist() == [3, 2, 1]


def test_drafts_without_probabilities():
    target, _, tokens, u, noise = _inputs(40, 3, 37, torch.float32, seed=4)
    _check(target, tokens, 0.2 * u, noise)


def test_ragged_drafts_and_padded_rows():
    for dtype in (torch.bfloat16, torch.float32):
        target, draft, tokens, u, noise = _inputs(30, 4, 999, dtype, seed=5, spread=0.3, ld=1024)
        target[..., 999:], draft[..., 999:] = 50.0, 50.0  # padding of the vocabulary is not read
        n = torch.tensor([0, 1, 2, 3, 4, 9, -2, 4, 4, 4] * 3, dtype=torch.int32, device=DEV)
        _check(target, tokens, u, noise, draft, draft_len=n, vocab=999)


def test_excluded_tokens():
    """-inf, NaN and the type's lowest value exclude tokens; +inf takes every probability."""
    for dtype in (torch.bfloat16, torch.float32):
        target, draft, tokens, u, noise = _inputs(32, 3, 2003, dtype, seed=6, spread=0.3)
        gen = torch.Generator(device=DEV).manual_seed(7)
        off = torch.rand(target.shape, generator=gen, device=DEV) < 0.9
        target[off] = -math.inf
        draft[off[:, :3]] = math.nan
        target[5, 1], draft[5, 1] = torch.finfo(dtype).min, torch.finfo(dtype).min
        target[6, 0, 77], draft[6, 0, 77] = math.inf, math.inf
        tokens[6, 0] = 77
        tokens[off[:, :3].gather(-1, tokens[..., None].long())[..., 0] & (u < 0.5)] = 3
        _check(target, tokens, u, noise, draft)


LOW = -(2.0 ** 20) / math.log2(math.e)  # where a row's exponents leave the fast sums


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["-1e4", "-1e9", "lowest", "few -1e9", "shift -200", "log-probabilities", "shift -1e9", "border"])
@pytest.mark.parametrize("T", [1.0, 0.1, 3.0])
@pytest.mark.parametrize("B,V", [(6, 20011), (40, 999)])
def test_low_logits(B, V, T, kind, dtype):
    """Tokens masked with large negative numbers, logits far below 0, whole rows of masked tokens."""
    target, draft, tokens, u, noise = _inputs(B, 3, V, dtype, seed=13, spread=0.3, scale=2.0 * T)
    gen = torch.Generator(device=DEV).manual_seed(V)
    value = {"-1e4": -1e4, "-1e9": -1e9, "few -1e9": -1e9, "lowest": torch.finfo(dtype).min}.get(kind)
    if value is not None:
        off = torch.rand(B, 1, V, generator=gen, device=DEV) < (0.01 if kind.startswith("few") else 0.99)
        off[1] = True  # every token masked: all are equally likely
        off[2, :, :V // 2] = True
        target.masked_fill_(off, value), draft.masked_fill_(off, value)
    elif kind == "log-probabilities":
        target, draft = (z.float().log_softmax(-1).to(dtype) for z in (target, draft))
    else:
        down = {"shift -200": -200.0, "shift -1e9": -1e9, "border": LOW * T}[kind]
        target, draft = (target.float() + down).to(dtype), (draft.float() + down).to(dtype)
        if kind == "border":  # rows above, across and below
            target[0], draft[0] = target[0] + 300, draft[0] + 300
            target[1], draft[1] = target[1] - 300, draft[1] - 300
    race = torch.empty(B, 3, V, device=DEV).exponential_(generator=gen)
    tokens = ((draft.float() - draft.float().amax(-1, keepdim=True)) / T - race.log()).argmax(-1).to(torch.int32)
    _check(target, tokens, u, noise, draft, temperature=torch.full((B,), T, device=DEV))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_low_logits_take_no_longer(dtype):
    """Masked tokens, shifted logits and log-probabilities at a low temperature are as many bytes and
    operations as other logits; a quarter more time is left for the clock and the memory."""
    B, D, V = 32, 3, 65536
    target, draft, tokens, u, noise = _inputs(B, D, V, dtype, seed=14)
    off = torch.rand(B, 1, V, device=DEV) < 0.999
    low = {"as they are": (target, draft, 1.0), "shift -200": (target - 200, draft - 200, 1.0),
           "log-probabilities": (target.float().log_softmax(-1).to(dtype), draft.float().log_softmax(-1).to(dtype), 0.1)}
    for value in (-1e4, -1e9, torch.finfo(dtype).min):
        low[value] = (target.masked_fill(off, value), draft.masked_fill(off, value), 1.0)
    u = torch.zeros_like(u)  # every draft with a probability is accepted: all rows are read
    time = {}
    for name, (t, d, temp) in low.items():
        x = d.argmax(-1).to(torch.int32)
        args = dict(draft_logits=d, temperature=torch.full((B,), temp, device=DEV))
        graph = torch.cuda.CUDAGraph()
        assert bool((damp.verify_drafts(t, x, u, noise, **args)[1] == D + 1).all())
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            for _ in range(20):
                damp.verify_drafts(t, x, u, noise, **args)
        best = math.inf
        for _ in range(7):
            start, end = torch.cuda.Event(True), torch.cuda.Event(True)
            start.record(), graph.replay(), end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        time[name] = best
    assert all(t <= 1.25 * time["as they are"] for t in time.values()), time


def test_rows_that_exclude_every_token():
    target, draft, tokens, u, noise = _inputs(6, 2, 700, torch.bfloat16, seed=8, spread=0.0)
    target[0] = -math.inf
    target[1, 1] = math.nan
    target[2, 2] = -math.inf
    draft[3] = -math.inf        # the draft says nothing: q is 0, the target decides
    temp = torch.tensor([1.0, 1.0, 1.0, 1.0, 0.0, 1.0], device=DEV)
    target[4] = -math.inf
    u = torch.zeros_like(u)     # 0 q < p accepts whatever has a probability
    out, count = _check(target, tokens, u, noise, draft, temperature=temp)
    assert count.tolist()[:5] == [0, 1, 2, 3, 0]


def test_tokens_out_of_range_are_rejected_and_reported():
    target, draft, tokens, u, noise = _inputs(4, 2, 900, torch.float32, seed=9)
    tokens[0, 0], tokens[1, 1], tokens[2, 0] = 900, -1, 1 << 30
    _check(target, tokens, 0 * u, noise, draft)
    assert damp.device_status() == damp.DEV_BAD_TOKEN


@pytest.mark.parametrize("with_draft", [True, False])
def test_emitted_tokens_follow_the_target(with_draft):
    """The first two tokens of many requests on one context: their joint frequencies are the
    target's, p_0(x) p_1(y) (the second row does not depend on the first token here), within
    five standard deviations of each cell and of the pair of counts."""
    n, V, D = 200000, 6, 2
    gen = torch.Generator(device=DEV).manual_seed(10)
    row = torch.randn(1, D + 1, V, generator=gen, device=DEV)
    target = row.expand(n, D + 1, V).contiguous()
    draft = (row[:, :D] + torch.randn(1, D, V, generator=gen, device=DEV)).expand(n, D, V).contiguous()
    if with_draft:
        race = torch.empty(n, D, V, device=DEV).exponential_(generator=gen)
        tokens = (draft - race.log()).argmax(-1).to(torch.int32)
    else:
        tokens = torch.full((n, D), 2, dtype=torch.int32, device=DEV)
    u = torch.rand(n, D, generator=gen, device=DEV)
    noise = torch.empty(n, V, device=DEV).exponential_(generator=gen)
    out, count = damp.verify_drafts(target, tokens, u, noise, draft_logits=draft if with_draft else None)
    p = row[0].double().softmax(-1).cpu()
    first = out[:, 0].cpu().bincount(minlength=V).double() / n
    assert bool(((first - p[0]).abs() <= 5 * (p[0] * (1 - p[0]) / n).sqrt()).all())
    two = out[count >= 2].cpu()
    m = two.shape[0]
    second = two[:, 1].bincount(minlength=V).double() / m
    assert bool(((second - p[1]).abs() <= 5 * (p[1] * (1 - p[1]) / m).sqrt()).all())


def test_pairs_of_emitted_tokens_follow_the_target():
    """Of requests whose first draft was accepted, the first token and the second are independent (the
    second row does not depend on the first token here) and the second follows the target's p_1: every
    cell of their table is within five standard deviations, and the first token's frequencies among
    all requests times its acceptance, min(p_0, q_0), too."""
    n, V, D = 400000, 6, 2
    gen = torch.Generator(device=DEV).manual_seed(15)
    row = torch.randn(1, D + 1, V, generator=gen, device=DEV)
    near = row[:, :D] + torch.randn(1, D, V, generator=gen, device=DEV)
    target, draft = row.expand(n, D + 1, V).contiguous(), near.expand(n, D, V).contiguous()
    race = torch.empty(n, D, V, device=DEV).exponential_(generator=gen)
    tokens = (draft - race.log()).argmax(-1).to(torch.int32)
    u = torch.rand(n, D, generator=gen, device=DEV)
    noise = torch.empty(n, V, device=DEV).exponential_(generator=gen)
    out, count = damp.verify_drafts(target, tokens, u, noise, draft_logits=draft)
    p, q = row[0].double().softmax(-1).cpu(), near[0].double().softmax(-1).cpu()
    two = out[count >= 2].cpu().long()
    table = (V * two[:, 0] + two[:, 1]).bincount(minlength=V * V).double().view(V, V) / n
    want = torch.minimum(p[0], q[0])[:, None] * p[1][None, :]
    assert bool(((table - want).abs() <= 5 * (want * (1 - want) / n).sqrt()).all())


def test_repeatable_on_another_stream_and_in_a_graph():
    target, draft, tokens, u, noise = _inputs(9, 3, 20001, torch.bfloat16, seed=11)
    run = lambda **kw: damp.verify_drafts(target, tokens, u, noise, draft_logits=draft, **kw)
    a, n = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b, m = run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, l = run()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(n, m) and torch.equal(a, c) and torch.equal(n, l)


def test_offsets_past_32_bits():
    B, D, V = 9000, 1, 130001  # 2.3e9 target logits
    gen = torch.Generator(device=DEV).manual_seed(12)
    target = torch.zeros(B, D + 1, V, dtype=torch.bfloat16, device=DEV)
    target[-1].normal_(generator=gen)
    tokens = torch.zeros(B, D, dtype=torch.int32, device=DEV)
    u, noise = torch.ones(B, D, device=DEV) * 0.999, torch.ones(B, V, device=DEV)
    noise[-1].exponential_(generator=gen)
    tokens[-1, 0] = int(target[-1, 0].argmax())
    out, count = damp.verify_drafts(target, tokens, u, noise)
    want, margin = R.verify_row(target[-1].cpu(), None, tokens[-1].tolist(), u[-1].cpu(), noise[-1].cpu())
    assert margin > MARGIN and out[-1].tolist() == want + [-1] * (2 - len(want)) and int(count[-1]) == len(want)
