"""The speculative-decoding example end to end: with greedy requests its tokens are those of
one-token decoding, and with warm ones it runs on mixed layers, frees and compacts."""
import os
import sys

import pytest
import torch

import paper_2608_27513_gb300 as damp

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_27513_gb300 import build
    build.build()
    torch.cuda.init()
    assert damp.device_status() == 0
    yield
    assert damp.device_status() == 0


def _server(kinds, batch, seed):
    from speculative_serving import Server
    s = Server(kinds, slots=batch, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lengths = torch.randint(2, 50, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    s.prompt(torch.randint(0, s.vocab, (batch, 50), generator=gen, device="cuda"), lengths)
    return s


def test_greedy_speculation_gives_the_tokens_of_plain_decoding():
    """The first logit gap of random weights is far above the rounding between a chunk and steps."""
    B, rounds = 6, 5
    cold = torch.zeros(B, device="cuda")
    fast, plain = _server(("lin", "lin"), B, 1), _server(("lin", "lin"), B, 1)
    out = [[] for _ in range(B)]
    for _ in range(rounds):
        tokens, count = fast.round(3, cold)
        for b in range(B):
            out[b] += tokens[b, :int(count[b])].tolist()
    steps = torch.cat([plain.step(cold) for _ in range(max(len(o) for o in out))], 1)
    for b in range(B):
        assert out[b] == steps[b, :len(out[b])].tolist()


@pytest.mark.parametrize("kinds", [("lin", "gdn", "lin"), ("gdn", "lin")])
def test_mixed_layers_finish_and_compact(kinds):
    B = 7
    s = _server(kinds, B, 2)
    temperature = torch.full((B,), 0.8, device="cuda")
    for _ in range(2):
        tokens, count = s.round(4, temperature)
        assert bool(((count >= 1) & (count <= 5)).all())
        at = torch.arange(5, device="cuda")[None]
        assert bool((tokens[at >= count[:, None]] == -1).all()) and bool((tokens[at < count[:, None]] >= 0).all())
    done = torch.tensor([True, False, False, True, False, False, False], device="cuda")
    kept = [p[s.slot_idx[~done].long()].clone() for p in s.pools]
    s.finish(done)
    assert sorted(s.slot_idx.tolist()) == list(range(5))
    for p, k in zip(s.pools, kept):
        assert torch.equal(p[s.slot_idx.long()], k)
    tokens, count = s.round(4, temperature[~done].contiguous())
    assert tokens.shape == (5, 5) and bool((count >= 1).all())


def test_requests_without_a_token_stay_where_they_were():
    """Logits that are no numbers exclude every token: nothing is accepted or drawn, and the next
    round goes on from the same token and state.  Prompt lengths are held to 1 .. T."""
    from speculative_serving import Server
    B = 4
    temperature = torch.full((B,), 0.8, device="cuda")
    s = Server(("lin", "lin"), slots=B, seed=3)
    prompts = torch.randint(0, s.vocab, (B, 20), generator=s.gen, device="cuda")
    s.prompt(prompts, torch.tensor([0, 1, 20, 33], dtype=torch.int32, device="cuda"))
    assert s.last[:, 0].tolist() == prompts[range(B), [0, 0, 19, 19]].tolist()
    s.round(3, temperature)
    head, last, states = s.head, s.last.clone(), [p[s.slot_idx.long()].clone() for p in s.pools]
    s.head = torch.full_like(head, float("nan"))
    tokens, count = s.round(3, temperature)
    assert not count.any() and bool((tokens == -1).all()) and torch.equal(s.last, last)
    assert all(torch.equal(p[s.slot_idx.long()], t) for p, t in zip(s.pools, states))
    s.head = head
    tokens, count = s.round(3, temperature)
    assert bool((count >= 1).all()) and bool((tokens[:, 0] >= 0).all())
