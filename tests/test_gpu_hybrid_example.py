"""The serving example with softmax-attention layers between the recurrent ones."""
import os
import sys

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(autouse=True)
def _status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


def _server(kinds, batch, seed):
    from speculative_serving import Server
    s = Server(kinds, slots=batch, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lengths = torch.randint(2, 50, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    s.prompt(torch.randint(0, s.vocab, (batch, 50), generator=gen, device="cuda"), lengths)
    return s, lengths


@pytest.mark.parametrize("kinds", [("lin", "attn", "gdn"), ("attn", "lin"), ("attn", "attn")])
def test_hybrid_layers_speculate_finish_and_compact(kinds):
    B = 6
    s, lengths = _server(kinds, B, 4)
    held = (lengths - 1).tolist()
    temperature = torch.full((B,), 0.8, device="cuda")
    for _ in range(3):
        tokens, count = s.round(4, temperature)
        held = [h + c for h, c in zip(held, count.tolist())]
        assert bool(((count >= 1) & (count <= 5)).all()) and s.held.tolist() == held
    done = torch.tensor([False, True, False, False, True, False], device="cuda")
    kept = [p[s.slot_idx[~done].long()].clone() for p in s.pools]
    s.finish(done)
    assert sorted(s.slot_idx.tolist()) == list(range(4))
    for p, k in zip(s.pools, kept):
        assert torch.equal(p[s.slot_idx.long()], k)
    tokens, count = s.round(3, temperature[~done].contiguous())
    assert tokens.shape == (4, 4) and bool((count >= 1).all())


def test_the_attention_layer_is_attention_over_its_cache():
    """A chunk of a layer against the formulas: rotary positions in 64 bits, the cache as it stands."""
    from speculative_serving import AttentionLayer, D_HEAD, HEADS, QK_HEADS
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = AttentionLayer(128, 4, gen, "cuda")
    slots, held = torch.tensor([2, 0], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for T in (37, 1, 6):
        x = torch.randn(2, T, 128, generator=gen, device="cuda")
        out = layer.run(x, slots, held)
        q = (x @ layer.wqkv).view(2, T, -1, D_HEAD)[:, :, :HEADS]
        positions = held[:, None] + torch.arange(T, device="cuda")
        q = R.rotary(q, positions, layer.freq, False, layer.scale).float()
        held = held + T
        pages = slots[:, None] * layer.PAGES + torch.arange(layer.PAGES, device="cuda")
        o, _ = R.attend(R.Cache(layer.cache, D_HEAD), q, pages.cpu(), held.tolist())
        want = x.double() + o.reshape(2, T, -1).cuda() @ layer.wo.double()
        # q is rounded once more than in the layer, logits and outputs are FP32: 2^-14 of the values at most
        assert (out.double() - want).abs().max().item() < 2.0 ** -14 * want.abs().max().item()
