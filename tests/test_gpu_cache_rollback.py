"""Tokens of an 8-bit cache that are taken back: what a rejected draft leaves in an open page, and how a copy of that
page undoes it; the serving example, whose outputs must not depend on what was rejected."""
import os
import sys

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests.test_gpu_cache import BF, DEV, gen, i32, randn

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(autouse=True)
def clean_status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


def test_a_copy_of_the_open_page_takes_a_draft_back():
    layout = damp.CacheLayout(2, 2, 128)
    g = gen(1)
    B, W, held = 3, 4, [5, 31, 64]
    pool = damp.new_cache(layout, B * W + B, DEV)
    pages = torch.arange(B * W, device=DEV, dtype=torch.int32).reshape(B, W)
    k, v = (randn(g, B, 70, 2, 128, dtype=BF) for _ in range(2))
    damp.cache_append(layout, pool, k, v, pages, i32([0] * B), lengths=i32(held))
    never = pool.clone()
    kept, vkept = k[:, 64:66].contiguous(), v[:, 64:66].contiguous()
    damp.cache_append(layout, never, kept, vkept, pages, i32(held))
    # the draft: the first two tokens, then three with larger values
    draft, vdraft = torch.cat((kept, 9 * k[:, :3]), 1), torch.cat((vkept, 9 * v[:, :3]), 1)
    open_pages, saved = pages.gather(1, i32(held)[:, None].long() // damp.CACHE_PAGE)[:, 0].contiguous(), i32(range(B * W, B * W + B))
    damp.copy_slots([pool], open_pages, saved)
    damp.cache_append(layout, pool, draft, vdraft, pages, i32(held))
    after = i32([h + 2 for h in held])
    dirty = damp.cache_read(layout, pool, pages, after, 96)
    damp.copy_slots([pool], saved, open_pages)
    damp.cache_append(layout, pool, kept, vkept, pages, i32(held))
    for got, want, left in zip(damp.cache_read(layout, pool, pages, after, 96), damp.cache_read(layout, never, pages, after, 96), dirty):
        assert torch.equal(got, want)
        assert not torch.equal(left, want)  # (without the copy: the draft's scale, and the codes rounded to it)


@pytest.mark.parametrize("kinds", [("attn", "lin"), ("lin", "attn", "gdn"), ("attn", "attn")])
def test_a_round_leaves_no_trace_of_rejected_tokens(kinds):
    """Every round's states and caches against a run over the accepted tokens alone, bit for bit."""
    from speculative_serving import AttentionLayer, Server
    B = 6
    s = Server(kinds, slots=B, seed=3)
    s.embed *= torch.exp(randn(gen(2), s.vocab, 1))  # tokens of very different sizes
    lengths = torch.randint(2, 50, (B,), generator=gen(5), device=DEV, dtype=torch.int32)
    s.prompt(torch.randint(0, s.vocab, (B, 50), generator=gen(6), device=DEV), lengths)
    temperature = torch.full((B,), 0.8, device=DEV)

    def tokens_held():
        out = []
        for layer in s.layers:
            if isinstance(layer, AttentionLayer):
                pages = s.slot_idx[:, None] * layer.PAGES + torch.arange(layer.PAGES, dtype=torch.int32, device=DEV)
                out += damp.cache_read(layer.layout, layer.cache, pages, s.held, layer.PAGES * damp.CACHE_PAGE)
            else:
                out.append(layer.pool[s.slot_idx.long()])
        return out

    rejected = 0
    for _ in range(6):
        before, held, last = [p.clone() for p in s.pools], s.held, s.last
        tokens, count = s.round(4, temperature)
        rejected += int((5 - count).sum())
        after, now = tokens_held(), [p.clone() for p in s.pools]
        for p, b in zip(s.pools, before):
            p.copy_(b)
        s.held = held
        s.logits(torch.cat((last, tokens[:, :-1].clamp(min=0)), 1), lengths=count)
        s.held = held + count
        for a, b in zip(after, tokens_held()):
            assert torch.equal(a, b)
        for p, n in zip(s.pools, now):
            p.copy_(n)
    assert rejected > 0
