"""The serving operators on the host: the C ABI and the Python binding reject bad arguments
before anything is enqueued, and the rule of the draft verification's reference."""
import ctypes

import pytest
import torch

import paper_2608_27513_gb300 as damp
from paper_2608_27513_gb300 import _lib, build
from tests import serving_ref as R
from tests.test_abi_host import FakeBuffers

OK, NULL, SHAPE, ALIGN, ALIAS, FORMAT = range(6)


@pytest.fixture(scope="module")
def L():
    build.build()
    return _lib.lib()


@pytest.fixture(scope="module")
def fb():
    return FakeBuffers(n=12, size=1 << 22)


def _p(fb, i, off=0):
    return ctypes.c_void_p(fb.ptrs[i] + off)


def test_lin_rejects_bad_arguments(L, fb):
    def call(chunk, **over):
        lay = dict(num_heads=2, num_qk_heads=2, d_k=64, d_v=64, k_hi=999, lo_format=77, model_heads=0, head_map=None)
        lay.update(over.pop("lay", {}))
        c = _lib.DampLayout(*lay.values())
        a = dict(layout=ctypes.byref(c), state=_p(fb, 0), num_slots=4, slot_idx=None, batch=2, T=3, lengths=None, q=_p(fb, 1),
                 k=_p(fb, 2), v=_p(fb, 3), g=_p(fb, 4), per_head=0, o=_p(fb, 5), dtype=0, ws=None, ws_bytes=0, stream=None)
        a.update(over)
        if chunk:
            return L.damp_lin_prefill_chunk(*a.values())
        return L.damp_lin_decode_step(*(x for n, x in a.items() if n not in ("T", "lengths", "ws", "ws_bytes")))

    for chunk in (False, True):
        assert call(chunk, batch=0) == OK          # nothing enqueued; k_hi and lo_format are ignored
        assert call(chunk, batch=-1) == SHAPE
        assert call(chunk, layout=None) == NULL
        for name in ("state", "q", "k", "v", "g", "o"):
            assert call(chunk, **{name: None}) == NULL, name
        for name, i in (("state", 0), ("q", 1), ("k", 2), ("v", 3)):
            assert call(chunk, **{name: _p(fb, i, 8)}) == ALIGN, name
        for name, i in (("g", 4), ("o", 5), ("slot_idx", 6)):
            assert call(chunk, **{name: _p(fb, i, 2)}) == ALIGN, name
        assert call(chunk, dtype=2) == FORMAT
        assert call(chunk, num_slots=1) == SHAPE   # fewer slots than rows without slot_idx
        assert call(chunk, num_slots=0, slot_idx=_p(fb, 6)) == SHAPE
        for lay in (dict(d_k=96), dict(d_v=48), dict(d_v=2048), dict(num_qk_heads=3), dict(head_map=fb.ptrs[7]),
                    dict(model_heads=4)):
            assert call(chunk, lay=lay) == SHAPE, lay
        assert call(chunk, o=_p(fb, 0, 64)) == ALIAS
        assert call(chunk, o=_p(fb, 3)) == ALIAS
        assert call(chunk, v=_p(fb, 0)) == ALIAS
        assert call(chunk, slot_idx=_p(fb, 5, 16)) == ALIAS
    assert call(True, T=0) == OK
    assert call(True, T=-1) == SHAPE
    assert call(True, lengths=_p(fb, 7, 1)) == ALIGN
    assert call(True, lengths=_p(fb, 5)) == ALIAS
    # one long row of few heads is split: its scratch
    lay, T = dict(d_k=64, d_v=128), 640
    c = _lib.DampLayout(2, 2, 64, 128, 0, 0, 0, None)
    need = L.damp_lin_prefill_workspace(ctypes.byref(c), 1, T, 0)
    if need:  # (the split goes by the number of SMs, which is not known without a GPU)
        assert call(True, lay=lay, T=T, batch=1) == NULL
        assert call(True, lay=lay, T=T, batch=1, ws=_p(fb, 6), ws_bytes=need - 1) == SHAPE
        assert call(True, lay=lay, T=T, batch=1, ws=_p(fb, 6, 4), ws_bytes=need) == ALIGN
        assert call(True, lay=lay, T=T, batch=1, ws=_p(fb, 5, 64), ws_bytes=need) == ALIAS
    assert L.damp_lin_prefill_workspace(ctypes.byref(c), 0, T, 0) == 0
    assert L.damp_lin_prefill_workspace(ctypes.byref(c), 1, 5, 0) == 0
    assert L.damp_lin_prefill_workspace(None, 1, T, 0) == 0


def test_slots_reject_bad_arguments(L, fb):
    def call(op, ptrs=None, sizes=(1024, 64), slots=8, a=None, b=None, n=4, n_pools=None):
        ptrs = [fb.ptrs[0], fb.ptrs[1]] if ptrs is None else ptrs
        pools = (ctypes.c_void_p * max(1, len(ptrs)))(*ptrs)
        nb = (ctypes.c_int64 * max(1, len(sizes)))(*sizes)
        n_pools = len(ptrs) if n_pools is None else n_pools
        a = _p(fb, 2) if a is None else a
        b = _p(fb, 3) if b is None else b
        if op == "zero":
            return L.damp_zero_slots(pools, nb, n_pools, slots, b, n, None)
        if op == "copy":
            return L.damp_copy_slots(pools, nb, n_pools, slots, a, b, n, None)
        return L.damp_compact_slots(pools, nb, n_pools, slots, a, n, b, None)

    nul = ctypes.c_void_p(0)
    for op in ("copy", "zero", "compact"):
        assert call(op, n=0) == OK
        assert call(op, n=-1) == SHAPE
        assert call(op, n_pools=-1) == SHAPE
        assert call(op, n_pools=1025) == SHAPE
        assert call(op, slots=0) == SHAPE
        assert call(op, slots=1 << 31) == SHAPE
        assert call(op, sizes=(1024, 24)) == SHAPE
        assert call(op, sizes=(0, 64)) == SHAPE
        assert call(op, ptrs=[fb.ptrs[0], fb.ptrs[1] + 8]) == ALIGN
        assert call(op, ptrs=[fb.ptrs[0], 0]) == NULL
        assert call(op, b=nul) == NULL
        assert call(op, b=_p(fb, 3, 2)) == ALIGN
        assert call(op, ptrs=[fb.ptrs[0], fb.ptrs[0] + 512]) == ALIAS
        assert call(op, b=_p(fb, 0, 16)) == ALIAS
    for op in ("copy", "compact"):
        assert call(op, a=nul) == NULL
        assert call(op, a=_p(fb, 2, 1)) == ALIGN
        assert call(op, a=_p(fb, 1)) == ALIAS
        assert call(op, n=4097) == SHAPE
    assert call("compact", slots=(1 << 18) + 1, sizes=(16, 16)) == SHAPE
    assert call("compact", b=_p(fb, 2, 4)) == ALIAS
    assert call("copy", ptrs=[], n_pools=0) == OK


def test_verify_rejects_bad_arguments(L, fb):
    def call(**over):
        a = dict(target=_p(fb, 0), draft=_p(fb, 1), dtype=0, stride=100, vocab=100, tokens=_p(fb, 2), lens=_p(fb, 3), D=3,
                 u=_p(fb, 4), noise=_p(fb, 5), temperature=_p(fb, 6), batch=2, out=_p(fb, 7), count=_p(fb, 8), stream=None)
        a.update(over)
        return L.damp_verify_drafts(*a.values())

    assert call(batch=0) == OK
    assert call(batch=-1) == SHAPE
    assert call(D=-1) == SHAPE
    assert call(vocab=0) == SHAPE
    assert call(vocab=(1 << 30) + 1, stride=1 << 31) == SHAPE
    assert call(stride=99) == SHAPE
    assert call(stride=1 << 62) == SHAPE
    assert call(dtype=2) == FORMAT
    for name in ("target", "tokens", "u", "noise", "out", "count"):
        assert call(**{name: None}) == NULL, name
    for name, i in (("target", 0), ("draft", 1), ("noise", 5)):
        assert call(**{name: _p(fb, i, 8)}) == ALIGN, name
    for name, i in (("tokens", 2), ("lens", 3), ("u", 4), ("temperature", 6), ("out", 7), ("count", 8)):
        assert call(**{name: _p(fb, i, 2)}) == ALIGN, name
    assert call(out=_p(fb, 0)) == ALIAS
    assert call(count=_p(fb, 7, 4)) == ALIAS
    assert call(count=_p(fb, 5, 4)) == ALIAS


class _NoCompute:
    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        if name in ("damp_status_string", "damp_slot_bytes", "damp_validate_layout"):
            return getattr(self.real, name)
        raise AssertionError(f"{name} was called")


@pytest.fixture()
def no_compute(monkeypatch, L):
    monkeypatch.setattr(damp, "lib", lambda: _NoCompute(L))


def test_binding_rejects_missized_tensors(no_compute):
    lay = damp.Layout(4, 2, 64, 64, 0)
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    state = z(5, 4, 64, 64)
    good = dict(q=z(3, 2, 64), k=z(3, 2, 64), v=z(3, 4, 64), g=z(3, 4))
    bad = [dict(q=z(3, 4, 64)), dict(k=z(3, 2, 32)), dict(v=z(3, 4, 63)), dict(g=z(3, 3)), dict(g=z(3)), dict(g=z(3, 4, 64)),
           dict(g=z(3, 4, dt=torch.float64)), dict(q=None), dict(v=None), dict(o=z(3, 4, 32)),
           dict(slot_idx=z(3, dt=torch.int64)), dict(slot_idx=z(4, dt=torch.int32)), dict(num_slots=6), dict(num_slots=2)]
    for b in bad:
        with pytest.raises(ValueError):
            damp.lin_decode_step(lay, state, **{**good, **b})
    with pytest.raises(TypeError):
        damp.lin_decode_step(lay, state, **{**good, "q": z(3, 2, 64, dt=torch.bfloat16)})
    with pytest.raises(TypeError):
        damp.lin_decode_step(lay, state, **{n: t.half() if n != "g" else t for n, t in good.items()})
    with pytest.raises(ValueError):
        damp.lin_decode_step(lay, z(5, 4, 64, 32), **good)
    with pytest.raises(ValueError):  # not on the GPU
        damp.lin_decode_step(lay, state, **good)
    with pytest.raises(ValueError):
        damp.lin_prefill_chunk(lay, state, **good)
    with pytest.raises(ValueError):
        damp.lin_prefill_chunk(lay, state, **{n: t[:, None] for n, t in good.items()}, lengths=z(2, dt=torch.int32))


def test_slots_binding_rejects_missized_tensors(no_compute):
    i = torch.zeros(3, dtype=torch.int32)
    pool = torch.zeros(4, 32, dtype=torch.uint8)
    for call in (lambda: damp.copy_slots([], i, i), lambda: damp.copy_slots(pool, i, i[:2]), lambda: damp.zero_slots(pool, i),
                 lambda: damp.compact_slots(pool, i.long()), lambda: damp.compact_slots(pool, i), lambda: damp.copy_slots(pool, None, i),
                 lambda: damp.zero_slots(pool, i[None])):
        with pytest.raises(ValueError):
            call()


def test_verify_binding_rejects_missized_tensors(no_compute):
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    good = dict(target_logits=z(2, 4, 50), draft_tokens=z(2, 3, dt=torch.int32), u=z(2, 3), noise=z(2, 50),
                draft_logits=z(2, 3, 50))
    for b in (dict(target_logits=z(2, 50)), dict(target_logits=None), dict(draft_tokens=z(2, 4, dt=torch.int32)),
              dict(draft_tokens=z(2, 3)), dict(u=z(2, 4)), dict(noise=z(2, 49)), dict(draft_logits=z(2, 4, 50)),
              dict(draft_logits=z(2, 3, 50, dt=torch.bfloat16)), dict(vocab=51), dict(vocab=0), {}):
        with pytest.raises(ValueError):
            damp.verify_drafts(**{**good, **b})
    with pytest.raises(TypeError):
        damp.verify_drafts(**{**good, "target_logits": z(2, 4, 50, dt=torch.float16)})


def test_reference_rule_keeps_the_targets_distribution():
    """Summed over the drafted token and the accept decision, the rule emits token t with
    probability q(t) min(1, p(t)/q(t)) + (1 - sum min(p, q)) r(t)/sum r = p(t): checked from
    the reference's decisions on a grid of uniforms, and its residual race in the mean."""
    gen = torch.Generator().manual_seed(0)
    V = 5
    target, draft = torch.randn(2, V, generator=gen), torch.randn(1, V, generator=gen)
    p, q = target[0].double().softmax(-1), draft[0].double().softmax(-1)
    n = 400
    ones = torch.ones(V)
    for x in range(V):
        took = sum(R.verify_row(target, draft, [x], torch.tensor([(i + 0.5) / n]), ones)[0][0] == x and
                   len(R.verify_row(target, draft, [x], torch.tensor([(i + 0.5) / n]), ones)[0]) == 2 for i in range(n))
        assert abs(took / n - min(1.0, float(p[x] / q[x]))) <= 1.0 / n
    residual = (p - q).clamp(min=0)
    x = int((p / q).argmin())
    hits = torch.zeros(V)
    for _ in range(4000):
        noise = torch.empty(V).exponential_(generator=gen)
        hits[R.verify_row(target, draft, [x], torch.tensor([0.999999]), noise)[0][0]] += 1
    want = residual / residual.sum()
    assert bool(((hits / 4000 - want).abs() <= 5 * (want * (1 - want) / 4000).sqrt() + 1e-9).all())
