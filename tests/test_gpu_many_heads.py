"""Layouts with so many heads that (head x query heads) passes 32 bits, on the GPU: the row-absmax
step takes them to the chunk kernel, in which every head is computed from its own operands alone,
so that a layer of H heads gives bit for bit what the same heads give in narrower calls."""
import pytest
import torch

import paper_2608_27513_gb300 as damp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_27513_gb300 import build
    build.build()
    torch.cuda.init()
    assert damp.device_status() == 0
    yield
    assert damp.device_status() == 0


@pytest.mark.parametrize("kind", ["gdn", "kda"])
def test_row_absmax_step(kind):
    H, d, parts = 46400, 128, 4
    gen = torch.Generator(device=DEV).manual_seed(0)
    n = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    ops = dict(q=n(1, H, d).bfloat16() / 11, k=n(1, H, d).bfloat16() / 11, v=n(1, H, d).bfloat16(),
               g=-torch.rand(1, H, *((d,) if kind == "kda" else ()), generator=gen, device=DEV),
               beta=torch.rand(1, H, generator=gen, device=DEV))
    S = n(1, H, d, d)

    def run(h0, h1, chunk):
        L = damp.Layout(h1 - h0, h1 - h0, d, d, 10, damp.LO_S8_ABSMAX_ROW)
        perm = torch.arange(d, dtype=torch.uint8, device=DEV).repeat(h1 - h0, 1)
        pool = damp.new_state(L, 1)
        damp.quantize_state(L, S[:, h0:h1].contiguous(), perm, pool)
        part = {name: t[:, h0:h1].contiguous() for name, t in ops.items()}
        if chunk:
            part = {name: t[:, None] for name, t in part.items()}
        o = getattr(damp, f"{kind}_prefill_chunk" if chunk else f"{kind}_decode_step")(L, pool, perm, **part)
        return o.reshape(h1 - h0, d), pool.reshape(h1 - h0, -1)

    o, after = run(0, H, False)
    for i in range(parts):
        h0, h1 = H // parts * i, H // parts * (i + 1)
        o1, after1 = run(h0, h1, True)
        assert torch.equal(o[h0:h1], o1) and torch.equal(after[h0:h1], after1), (h0, h1)
