"""Speculative decoding of a small recurrent language model on libdamp.

A model of linear-attention layers (decay per head on FP32 states, or GDN on the packed state)
with random weights serves a batch of requests:

  prompt    the prompts, of different lengths, run as one chunk per layer
  round     copy_slots saves every layer's state; the first layer alone drafts D tokens, step by
            step; copy_slots takes its state back; all layers run the drafted tokens as one chunk;
            verify_drafts accepts a prefix and draws the next token; copy_slots takes the states
            back and the chunk runs once more over the accepted tokens, whose numbers
            (verify_drafts' counts) are the chunk's lengths on the device
  end       zero_slots frees finished requests, compact_slots closes the pools up

    python examples/speculative_serving.py [--layers lin,gdn,lin] [--batch 8] [--drafts 4]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2608_27513_gb300 as damp

D_HEAD, HEADS, QK_HEADS = 64, 4, 2


class Layer:
    """One linear-attention layer: its weights, its state pool and the calls on it."""

    def __init__(self, kind, width, slots, gen, device):
        n = lambda *s: torch.randn(*s, generator=gen, device=device)
        self.kind = kind
        self.wq, self.wk = (n(width, QK_HEADS * D_HEAD) / width ** 0.5 for _ in range(2))
        self.wv, self.wo = n(width, HEADS * D_HEAD) / width ** 0.5, n(HEADS * D_HEAD, width) / 16
        self.wg, self.wb = (n(width, HEADS) / width ** 0.5 for _ in range(2))
        if kind == "lin":
            self.layout = damp.Layout(HEADS, QK_HEADS, D_HEAD, D_HEAD, 0)
            self.pool = damp.new_fp32_state(self.layout, slots, device)
        else:  # packed DAMP state, 8 FP16 channels
            self.layout = damp.Layout(HEADS, QK_HEADS, D_HEAD, D_HEAD, 8)
            self.pool = damp.new_state(self.layout, slots, device)
            self.perm = torch.arange(D_HEAD, dtype=torch.uint8, device=device).repeat(HEADS, 1)

    def run(self, x, slot_idx, lengths=None):
        """x [B, T, width] -> x + the layer's output; the state of slot_idx moves on (row b by lengths[b])."""
        B, T, _ = x.shape
        unit = lambda z: torch.nn.functional.normalize(z.view(B, T, QK_HEADS, D_HEAD), dim=-1)
        q, k, v = unit(x @ self.wq), unit(x @ self.wk), (x @ self.wv).view(B, T, HEADS, D_HEAD)
        g = -torch.nn.functional.softplus(x @ self.wg - 2)
        ops = [t.contiguous() for t in (q, k, v, g)]
        if self.kind == "gdn":
            ops.append(torch.sigmoid(x @ self.wb).contiguous())
        one = T == 1 and lengths is None
        if one:
            ops = [t[:, 0].contiguous() for t in ops]
        if self.kind == "lin":
            call = damp.lin_decode_step if one else damp.lin_prefill_chunk
            state = (self.pool,)
        else:
            call = damp.gdn_decode_step if one else damp.gdn_prefill_chunk
            state = (self.pool, self.perm)
        o = call(self.layout, *state, *ops, slot_idx=slot_idx, **({} if one else {"lengths": lengths}))
        return x + o.reshape(B, T, HEADS * D_HEAD) @ self.wo


class Server:
    """Requests in the first half of the slots, their saved states in the second half."""

    def __init__(self, kinds=("lin", "lin"), vocab=2000, width=128, slots=16, seed=0, device="cuda"):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.slots, self.vocab, self.device = slots, vocab, device
        self.embed = torch.randn(vocab, width, generator=self.gen, device=device)
        self.head = torch.randn(width, vocab, generator=self.gen, device=device) * (4.0 / width ** 0.5)
        self.layers = [Layer(k, width, 2 * slots, self.gen, device) for k in kinds]
        self.pools = [layer.pool for layer in self.layers]
        self.slot_idx = torch.empty(0, dtype=torch.int32, device=device)

    def logits(self, tokens, depth=None, lengths=None):
        """Logits [B, T, vocab] of tokens [B, T]; the states of the first `depth` layers move on."""
        x = self.embed[tokens.long()]
        for layer in self.layers[:depth]:
            x = layer.run(x, self.slot_idx, lengths)
        return torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.head

    def prompt(self, tokens, lengths):
        """Admits requests: prompts [B, T], row b of lengths[b] (1 .. T) tokens; all but the last token run."""
        B = tokens.shape[0]
        lengths = lengths.clamp(1, tokens.shape[1])
        self.slot_idx = torch.arange(B, dtype=torch.int32, device=self.device)
        damp.zero_slots(self.pools, self.slot_idx)
        self.logits(tokens, lengths=lengths - 1)
        self.last = tokens.gather(1, lengths.long()[:, None] - 1).to(torch.int32)

    def saved(self):
        return self.slot_idx + self.slots

    def draw(self, logits, temperature):
        noise = torch.empty_like(logits).exponential_(generator=self.gen)
        warm = torch.softmax(logits / temperature.clamp(min=1e-3)[:, None], -1)
        return torch.where(temperature[:, None] > 0, warm / noise, logits).argmax(-1).to(torch.int32)[:, None]

    def round(self, drafts, temperature):
        """One round for every request: (tokens [B, drafts + 1], count [B])."""
        B, saved = self.slot_idx.shape[0], self.saved()
        damp.copy_slots(self.pools, self.slot_idx, saved)
        token, drafted, q = self.last, [], []
        for _ in range(drafts):
            q.append(self.logits(token, depth=1))
            token = self.draw(q[-1][:, 0], temperature)
            drafted.append(token)
        damp.copy_slots(self.pools[:1], saved, self.slot_idx)
        chunk = torch.cat([self.last] + drafted, 1)
        target = self.logits(chunk)
        u = torch.rand(B, drafts, generator=self.gen, device=self.device)
        noise = torch.empty(B, self.vocab, device=self.device).exponential_(generator=self.gen)
        tokens, count = damp.verify_drafts(target, torch.cat(drafted, 1), u, noise, draft_logits=torch.cat(q, 1),
                                           temperature=temperature)
        damp.copy_slots(self.pools, saved, self.slot_idx)
        self.logits(chunk, lengths=count)
        # logits that exclude every token give none (count 0): the request stays where it was
        last = tokens.gather(1, (count.long()[:, None] - 1).clamp(min=0))
        self.last = torch.where(count[:, None] > 0, last, self.last)
        return tokens, count

    def step(self, temperature):
        """One token without drafts, for comparison: tokens [B, 1]."""
        self.last = self.draw(self.logits(self.last)[:, 0], temperature)
        return self.last

    def finish(self, done):
        """Frees the requests of the mask `done` and closes the pools up."""
        damp.zero_slots(self.pools, self.slot_idx[done].contiguous())
        self.slot_idx = damp.compact_slots(self.pools, self.slot_idx[~done].contiguous())
        self.last = self.last[~done].contiguous()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", default="lin,gdn,lin")
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=6)
    a = ap.parse_args()
    from paper_2608_27513_gb300 import build
    build.build()
    s = Server(a.layers.split(","), slots=a.batch)
    lengths = torch.randint(3, 40, (a.batch,), generator=s.gen, device=s.device, dtype=torch.int32)
    prompts = torch.randint(0, s.vocab, (a.batch, 40), generator=s.gen, device=s.device)
    s.prompt(prompts, lengths)
    temperature = torch.full((a.batch,), 0.7, device=s.device)
    for r in range(a.rounds):
        tokens, count = s.round(a.drafts, temperature)
        print(f"round {r}: {count.tolist()} tokens per request, first request {tokens[0].tolist()}")
        if r == a.rounds // 2:
            done = torch.zeros(a.batch, dtype=torch.bool, device=s.device)
            done[::3] = True
            s.finish(done)
            temperature = temperature[~done].contiguous()
            print(f"finished {int(done.sum())} requests; slots now {s.slot_idx.tolist()}")
    assert damp.device_status() == 0


if __name__ == "__main__":
    main()
