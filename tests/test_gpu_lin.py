"""Linear attention with a decay per head on the GPU against the recurrence in float64:
the single-token step and chunks of every length class, head layouts, types, gates
(none, resets, fast), ragged lengths with garbage past them, slots and streams."""
import math

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import serving_ref as R

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


def _inputs(B, T, H, Hqk, dk, dv, dtype, gate, seed=0, slots=None):
    gen = torch.Generator(device=DEV).manual_seed(seed + 1000 * T + dk)
    n = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    slots = B + 2 if slots is None else slots
    g = {"token": lambda: -torch.nn.functional.softplus(n(B, T, H) + torch.linspace(-6, 2, H, device=DEV)),
         "head": lambda: -torch.linspace(0.001, 0.8, H, device=DEV),
         "zero": lambda: torch.zeros(B, T, H, device=DEV),
         "fast": lambda: -40.0 * torch.rand(B, T, H, generator=gen, device=DEV),
         "grow": lambda: 0.02 * n(B, T, H),
         "reset": lambda: torch.where(torch.rand(B, T, H, generator=gen, device=DEV) < 0.1, -math.inf,
                                      -0.05 * torch.rand(B, T, H, generator=gen, device=DEV)),
         "lowest": lambda: torch.where(torch.rand(B, T, H, generator=gen, device=DEV) < 0.1,
                                       torch.finfo(torch.float32).min, -0.3)}[gate]()
    q, k = n(B, T, Hqk, dk), n(B, T, Hqk, dk)
    pool = n(slots, H, dk, dv)
    idx = torch.randperm(slots, generator=gen, device=DEV)[:B].to(torch.int32)
    return dict(q=(q / dk ** 0.5).to(dtype), k=(k / dk ** 0.5).to(dtype), v=n(B, T, H, dv).to(dtype), g=g), pool, idx


def _check_chunk(B, T, H, Hqk, dk, dv, dtype, gate, lengths=None, seed=0):
    ops, pool, idx = _inputs(B, T, H, Hqk, dk, dv, dtype, gate, seed)
    L = damp.Layout(H, Hqk, dk, dv, 0)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    o_ref, S_ref, oa, Sa = R.lin(pool[idx.long()], **ops, lengths=n)
    if n is not None:  # what stands past a row's length must not matter
        past = torch.arange(T, device=DEV)[None] >= n.clamp(0, T)[:, None]
        for name in ("q", "k", "v"):
            ops[name][past] = math.nan
        if ops["g"].dim() == 3:
            ops["g"][past] = math.nan
    before = pool.clone()
    o = damp.lin_prefill_chunk(L, pool, **ops, lengths=n, slot_idx=idx)
    R.check_lin(o, o_ref, oa, T, dk, "o")
    R.check_lin(pool[idx.long()], S_ref, Sa, T, dk, "S")
    others = torch.ones(pool.shape[0], dtype=torch.bool, device=DEV)
    others[idx.long()] = False
    assert torch.equal(pool[others], before[others])
    if n is not None:
        assert not o[past].any()
        still = idx[n <= 0].long()
        assert torch.equal(pool[still], before[still])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 200, 321])
def test_chunk_lengths(T, dtype):
    _check_chunk(2, T, 4, 2, 128, 128, dtype, "token")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hqk,dk,dv", [(4, 4, 64, 64), (3, 1, 32, 96), (2, 2, 128, 1024), (6, 2, 64, 32), (2, 1, 128, 160),
                                         (1, 1, 32, 32), (8, 8, 128, 64), (2, 1, 64, 128), (2, 2, 128, 256)])
def test_chunk_layouts(H, Hqk, dk, dv, dtype):
    _check_chunk(2, 70, H, Hqk, dk, dv, dtype, "token", seed=1)


@pytest.mark.parametrize("gate", ["head", "zero", "fast", "grow", "reset", "lowest"])
@pytest.mark.parametrize("T", [7, 150])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_gates(gate, T, d):
    _check_chunk(2, T, 4, 4, d, d, torch.bfloat16, gate, seed=2)
    _check_chunk(2, T, 4, 4, d, d, torch.float32, gate, seed=3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [5, 64, 130])
def test_ragged_rows_ignore_what_stands_past_them(T, dtype):
    _check_chunk(7, T, 2, 1, 128, 128, dtype, "token", lengths=[T, 0, 1, T // 2, T + 9, -3, T - 1], seed=4)
    _check_chunk(7, T, 2, 1, 64, 64, dtype, "head", lengths=[T, 0, 1, T // 2, T + 9, -3, T - 1], seed=5)


@pytest.mark.parametrize("H, dk, dv", [(40, 128, 128), (24, 128, 192), (33, 64, 128)])
def test_rows_of_many_lengths_in_any_order(H, dk, dv):
    """More blocks than SMs: rows of equal lengths, empty ones, longer ones than the chunk."""
    _check_chunk(9, 150, H, H, dk, dv, torch.bfloat16, "token", lengths=[1, 150, 0, 64, 65, 150, -3, 129, 200])


@pytest.mark.parametrize("B", [255, 256, 257])
def test_many_rows_of_many_lengths(B):
    _check_chunk(B, 70, 3, 3, 64, 64, torch.bfloat16, "token", lengths=[(37 * b) % 73 - 1 for b in range(B)])


@pytest.mark.parametrize("B,H,T", [(1, 2, 3000), (3, 5, 1111), (1, 32, 2049)])
def test_long_prompts_of_few_rows(B, H, T):
    _check_chunk(B, T, H, H, 128, 128, torch.bfloat16, "token", seed=6)
    _check_chunk(B, T, H, H, 128, 128, torch.bfloat16, "head", lengths=[T - 700] + [T] * (B - 1), seed=7)


@pytest.mark.parametrize("dtype,H,Hqk,dk,dv", [(torch.float32, 2, 1, 128, 128), (torch.float32, 2, 2, 64, 64), (torch.bfloat16, 3, 3, 32, 64),
                                               (torch.bfloat16, 2, 2, 128, 96), (torch.bfloat16, 2, 1, 128, 128),
                                               (torch.bfloat16, 2, 2, 64, 192)])
@pytest.mark.parametrize("T", [700, 1111])
def test_long_rows_end_in_every_segment(T, dtype, H, Hqk, dk, dv):
    """Few rows and many tokens are split into segments: rows that end in the first one, at the borders
    of segments (multiples of 8 or 64 tokens), in their middle, and nowhere."""
    for lengths in ([T, 0, 1, T // 2, T - 1], [T // 2, 64, 65, T // 3, T], [8 * (T // 16), 8 * (T // 24) + 1, 320, 384, 8 * (T // 8)]):
        _check_chunk(5, T, H, Hqk, dk, dv, dtype, "token", lengths=lengths, seed=20)
    _check_chunk(3, T, H, Hqk, dk, dv, dtype, "head", lengths=[T - 200, T + 5, -1], seed=21)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [None, [900, 500, 900, 31]])
def test_bad_slots_of_long_rows_are_skipped_and_reported(lengths, dtype):
    H, d, T = 2, 128, 900
    ops, pool, _ = _inputs(4, T, H, H, d, d, dtype, "token", seed=22, slots=4)
    idx = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device=DEV)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    before = pool.clone()
    o_ref, S_ref, oa, Sa = R.lin(pool[[2, 0]], **{name: t[[0, 3]] for name, t in ops.items()}, lengths=None if n is None else n[[0, 3]])
    o = torch.full((4, T, H, d), 7.0, device=DEV)
    damp.lin_prefill_chunk(damp.Layout(H, H, d, d, 0), pool, **ops, o=o, lengths=n, slot_idx=idx)
    assert damp.device_status() == damp.DEV_BAD_SLOT
    R.check_lin(o[[0, 3]], o_ref, oa, T, d, "o")
    R.check_lin(pool[[2, 0]], S_ref, Sa, T, d, "S")
    assert torch.equal(pool[[1, 3]], before[[1, 3]]) and bool((o[1:3] == 7.0).all())


def test_many_rows_fill_the_gpu():
    _check_chunk(40, 130, 8, 4, 128, 128, torch.bfloat16, "token", lengths=[(37 * i) % 131 for i in range(40)], seed=8)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hqk,dk,dv", [(4, 4, 64, 64), (3, 1, 32, 96), (2, 2, 128, 1024), (6, 2, 64, 32), (32, 16, 128, 128),
                                         (1, 1, 32, 32), (5, 5, 128, 160)])
@pytest.mark.parametrize("gate", ["token", "head", "reset"])
def test_decode_step(H, Hqk, dk, dv, dtype, gate):
    B = 5
    ops, pool, idx = _inputs(B, 1, H, Hqk, dk, dv, dtype, gate, seed=9)
    o_ref, S_ref, oa, Sa = R.lin(pool[idx.long()], **ops)
    one = {n: (t if t.dim() == 1 else t[:, 0].contiguous()) for n, t in ops.items()}
    before = pool.clone()
    o = damp.lin_decode_step(damp.Layout(H, Hqk, dk, dv, 0), pool, **one, slot_idx=idx)
    R.check_lin(o, o_ref[:, 0], oa[:, 0], 1, dk, "o")
    R.check_lin(pool[idx.long()], S_ref, Sa, 1, dk, "S")
    others = torch.ones(pool.shape[0], dtype=torch.bool, device=DEV)
    others[idx.long()] = False
    assert torch.equal(pool[others], before[others])


@pytest.mark.parametrize("H,Hqk", [(46400, 46400), (66000, 33000)])
@pytest.mark.parametrize("T", [1, 3])
def test_head_counts_whose_product_passes_32_bits(H, Hqk, T):
    ops, pool, idx = _inputs(1, T, H, Hqk, 32, 32, torch.float32, "token", seed=17, slots=1)
    o_ref, S_ref, oa, Sa = R.lin(pool, **ops)
    L = damp.Layout(H, Hqk, 32, 32, 0)
    if T == 1:
        o = damp.lin_decode_step(L, pool, **{n: t[:, 0].contiguous() for n, t in ops.items()})[:, None]
    else:
        o = damp.lin_prefill_chunk(L, pool, **ops)
    R.check_lin(o, o_ref, oa, T, 32, "o")
    R.check_lin(pool, S_ref, Sa, T, 32, "S")


def _check_not_finite(got, want, absolute, T, dk, what):
    """Values that are not finite stand where the recurrence has them and nowhere else (an
    infinity may have become a NaN); the others are held to their bounds."""
    finite = want.isfinite()
    assert torch.equal(got.isfinite(), finite), what
    R.check_lin(got[finite], want[finite], absolute[finite], T, dk, what)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 9, 17, 64, 150, 700])
@pytest.mark.parametrize("H,dk,dv", [(2, 128, 128), (3, 64, 64), (2, 128, 192), (2, 64, 128)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_reach_no_earlier_output(H, dk, dv, T, dtype, bad):
    """A row with values of v that are not finite in the first, the last and some other tokens, one
    with a key, one with a query, one with a state that is not, and one without any."""
    ops, pool, idx = _inputs(6, T, H, H, dk, dv, dtype, "token", seed=18)
    n = torch.tensor([T, T, T, max(1, T // 2), T, T], dtype=torch.int32, device=DEV)
    ops["v"][0, T - 1, 0, 3] = ops["v"][0, T // 2, 1, dv - 1] = ops["v"][0, T // 3, 0, 40] = bad
    ops["v"][0, 0, 1, 33] = bad
    ops["k"][1, T // 2, 0, 5] = bad
    ops["q"][2, T // 2, 1, 6] = bad
    ops["v"][3, int(n[3]):] = bad  # past the row's length
    pool[idx[4].long(), 0, 7, 8] = bad
    o_ref, S_ref, oa, Sa = R.lin(pool[idx.long()], **ops, lengths=n)
    o = damp.lin_prefill_chunk(damp.Layout(H, H, dk, dv, 0), pool, **ops, lengths=n, slot_idx=idx)
    _check_not_finite(o, o_ref, oa, T, dk, "o")
    _check_not_finite(pool[idx.long()], S_ref, Sa, T, dk, "S")
    assert bool(o[5].isfinite().all()) and bool(pool[idx[5].long()].isfinite().all())


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, 0), (torch.float32, 0), (torch.bfloat16, 16), (torch.float32, 16),
                                     (torch.float32, 130)])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("where", ["S", "v", "k", "overflow"])
def test_infinities_stay_infinities_token_by_token(where, d, dtype, T):
    """T = 0: the single-token step.  Gates whose decays are rounded up and down."""
    H, n = 2, max(T, 1)
    ops, pool, idx = _inputs(2, n, H, H, d, d, dtype, "token", seed=19)
    ops["g"] = -0.02 * torch.rand(2, n, H, device=DEV, generator=torch.Generator(device=DEV).manual_seed(19))
    ops["k"], ops["q"] = ops["k"].abs(), ops["q"].abs() + 1e-3  # no difference of two infinities
    if where == "S":
        pool[idx[0].long(), :, 3, 5], pool[idx[0].long(), 1, 7, 6] = math.inf, -math.inf
    elif where == "overflow":  # beyond the largest finite value after the first token
        pool[idx[0].long(), :, 3, 5] = 3.4e38
        ops["k"][0, 0, :, 3], ops["v"][0, 0, :, 5] = 1.0, 2e38
    else:
        ops[where][0, n // 2, :, 5] = math.inf
        if where == "k":
            ops["v"] = ops["v"].abs()
    o_ref, S_ref, _, _ = R.lin(pool[idx.long()], **ops)
    if where == "overflow":  # float64 does not overflow
        S_ref[0, :, 3, 5] = math.inf
    L = damp.Layout(H, H, d, d, 0)
    if T:
        o = damp.lin_prefill_chunk(L, pool, **ops, slot_idx=idx)
    else:
        o = damp.lin_decode_step(L, pool, **{name: t[:, 0].contiguous() for name, t in ops.items()}, slot_idx=idx)[:, None]
    for got, want in ((pool[idx.long()], S_ref), (o, o_ref)):
        if where == "overflow" and got is o:
            continue  # q.S may overflow in one order of its terms and not in another
        for test in (torch.isposinf, torch.isneginf, torch.isnan):
            assert torch.equal(test(got), test(want)), test
        assert got.isinf().any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [0, 1, 5, 16, 40, 150])
@pytest.mark.parametrize("gate", [100.0, math.inf, math.nan])
def test_gates_beyond_the_largest_number(gate, T, dtype):
    """e^g is infinite in FP32 from g = 89 on: the state of that head becomes infinite with its
    signs (T = 0: the single-token step), or a NaN for a gate that is one; the other head is untouched.
    On the tensor cores the gates are summed first, and with the later decays e^100 is in range again."""
    H, d, n = 2, 64, max(T, 1)
    if gate == 100.0 and T > 16 and dtype == torch.bfloat16:
        pytest.skip("the sum of the gates is in range")
    ops, pool, idx = _inputs(2, n, H, H, d, d, dtype, "token", seed=23)
    ops["g"][0, n // 2, 1] = gate
    o_ref, S_ref, oa, Sa = R.lin(pool[idx.long()], **{**ops, "g": torch.where(ops["g"] > 89, math.inf, ops["g"])})
    L = damp.Layout(H, H, d, d, 0)
    if T:
        o = damp.lin_prefill_chunk(L, pool, **ops, slot_idx=idx)
    else:
        o = damp.lin_decode_step(L, pool, **{name: t[:, 0].contiguous() for name, t in ops.items()}, slot_idx=idx)[:, None]
    S = pool[idx.long()]
    for test in (torch.isposinf, torch.isneginf, torch.isnan) if T <= 16 else ():
        assert torch.equal(test(S), test(S_ref))
    _check_not_finite(o, o_ref, oa, n, d, "o")
    _check_not_finite(S, S_ref, Sa, n, d, "S")
    assert not S[0, 1].isfinite().any() and bool(S[0, 0].isfinite().all())


def test_steps_after_a_chunk_continue_it():
    B, T, H, d = 3, 90, 4, 128
    ops, pool, idx = _inputs(B, T, H, H, d, d, torch.bfloat16, "token", seed=10)
    L = damp.Layout(H, H, d, d, 0)
    o_ref, S_ref, oa, Sa = R.lin(pool[idx.long()], **ops)
    cut = lambda a, b: {n: t[:, a:b].contiguous() for n, t in ops.items()}
    o = [damp.lin_prefill_chunk(L, pool, **cut(0, 70), slot_idx=idx),
         damp.lin_prefill_chunk(L, pool, **cut(70, 87), slot_idx=idx)]
    o += [damp.lin_decode_step(L, pool, **{n: t[:, 0].contiguous() for n, t in cut(t, t + 1).items()}, slot_idx=idx)[:, None]
          for t in range(87, 90)]
    R.check_lin(torch.cat(o, 1), o_ref, oa, T, d, "o")
    R.check_lin(pool[idx.long()], S_ref, Sa, T, d, "S")


@pytest.mark.parametrize("T", [1, 40])
def test_bad_slots_are_skipped_and_reported(T):
    H, d = 2, 128
    ops, pool, _ = _inputs(4, T, H, H, d, d, torch.bfloat16, "token", seed=11, slots=4)
    idx = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device=DEV)
    before = pool.clone()
    o_ref, S_ref, oa, Sa = R.lin(pool[[2, 0]], **{n: t[[0, 3]] for n, t in ops.items()})
    o = torch.full((4, T, H, d), 7.0, device=DEV)
    damp.lin_prefill_chunk(damp.Layout(H, H, d, d, 0), pool, **ops, o=o, slot_idx=idx)
    assert damp.device_status() == damp.DEV_BAD_SLOT
    R.check_lin(o[[0, 3]], o_ref, oa, T, d, "o")
    R.check_lin(pool[[2, 0]], S_ref, Sa, T, d, "S")
    assert torch.equal(pool[[1, 3]], before[[1, 3]]) and bool((o[1:3] == 7.0).all())


def test_offsets_past_32_bits():
    H, d = 32, 128
    slots = 4200  # 2.2e9 state values
    pool = torch.zeros(slots, H, d, d, device=DEV)
    L = damp.Layout(H, H, d, d, 0)
    for T in (1, 40):
        ops, small, _ = _inputs(2, T, H, H, d, d, torch.bfloat16, "token", seed=12, slots=2)
        idx = torch.tensor([slots - 1, 3], dtype=torch.int32, device=DEV)
        pool[idx.long()] = small
        o_ref, S_ref, oa, Sa = R.lin(small, **ops)
        o = damp.lin_prefill_chunk(L, pool, **ops, slot_idx=idx)
        R.check_lin(o, o_ref, oa, T, d, "o")
        R.check_lin(pool[idx.long()], S_ref, Sa, T, d, "S")
    one = {n: t[:, 0].contiguous() for n, t in ops.items()}
    pool[idx.long()] = small
    o_ref, S_ref, oa, Sa = R.lin(small, **{n: t[:, :1] for n, t in ops.items()})
    o = damp.lin_decode_step(L, pool, **one, slot_idx=idx)
    R.check_lin(o, o_ref[:, 0], oa[:, 0], 1, d, "o")
    R.check_lin(pool[idx.long()], S_ref, Sa, 1, d, "S")


def test_results_repeat_bit_for_bit_and_on_another_stream():
    B, T, H, d = 3, 600, 4, 128
    ops, pool, idx = _inputs(B, T, H, H, d, d, torch.bfloat16, "token", seed=13)
    L = damp.Layout(H, H, d, d, 0)
    a, b = pool.clone(), pool.clone()
    o1 = damp.lin_prefill_chunk(L, a, **ops, slot_idx=idx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2 = damp.lin_prefill_chunk(L, b, **ops, slot_idx=idx, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(o1, o2) and torch.equal(a, b)


def test_a_graph_replays_the_step_and_the_chunk():
    B, H, d = 4, 4, 128
    L = damp.Layout(H, H, d, d, 0)
    for T in (1, 200):
        ops, pool, idx = _inputs(B, T, H, H, d, d, torch.bfloat16, "token", seed=14)
        start = pool.clone()
        run = lambda: damp.lin_prefill_chunk(L, pool, **ops, slot_idx=idx)
        o1 = run().clone()
        end = pool.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o2 = run()
        pool.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, o2) and torch.equal(pool, end)


@pytest.mark.parametrize("T,d", [(9, 128), (70, 128), (70, 64), (9, 32)])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_outputs_of_any_alignment_and_nothing_beside_them(T, d, offset):
    """o needs 4-byte alignment only, and no call writes before or after o or the slots."""
    B, H, poison = 5, 2, 12345.0
    ops, pool, _ = _inputs(B, T, H, H, d, d, torch.bfloat16, "token", seed=15, slots=B)
    n = torch.tensor([T, 0, 3, T - 1, T // 2], dtype=torch.int32, device=DEV)
    o_ref, S_ref, oa, Sa = R.lin(pool, **ops, lengths=n)
    raw = torch.full((64 + offset + B * T * H * d + 64,), poison, device=DEV)
    o = raw[64 + offset:64 + offset + B * T * H * d].view(B, T, H, d)
    held = torch.full((B + 2, H, d, d), poison, device=DEV)
    held[1:-1] = pool
    damp.lin_prefill_chunk(damp.Layout(H, H, d, d, 0), held[1:-1], **ops, o=o, lengths=n)
    R.check_lin(o, o_ref, oa, T, d, "o")
    R.check_lin(held[1:-1], S_ref, Sa, T, d, "S")
    assert not o[torch.arange(T, device=DEV)[None] >= n[:, None]].any()
    assert bool((raw[:64 + offset] == poison).all() and (raw[-64:] == poison).all())
    assert bool((held[[0, -1]] == poison).all())


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, 3000), (torch.float32, 1500)])
def test_constant_slow_gates_keep_their_digits(dtype, T):
    """One gate for all tokens loses the same rounding every time: the error of a head that
    remembers up to 3000 tokens stays that of as many random roundings, sqrt(3000 / 3) = 32 units
    of 2^-24."""
    H, d = 2, 64
    ops, pool, idx = _inputs(1, T, H, H, d, d, dtype, "token", seed=16)
    ops["g"] = torch.tensor([-3e-4, -2.7e-3], device=DEV)
    o_ref, S_ref, _, _ = R.lin(pool[idx.long()], **ops)
    o = damp.lin_prefill_chunk(damp.Layout(H, H, d, d, 0), pool, **ops, slot_idx=idx)
    limit = 32 * R.EPS
    assert (o.double() - o_ref).norm() <= limit * o_ref.norm()
    assert (pool[idx.long()].double() - S_ref).norm() <= limit * S_ref.norm()


def test_empty_calls():
    L = damp.Layout(2, 2, 64, 64, 0)
    pool = damp.new_fp32_state(L, 3)
    z = lambda *s: torch.zeros(*s, device=DEV)
    o = damp.lin_prefill_chunk(L, pool, z(2, 0, 2, 64), z(2, 0, 2, 64), z(2, 0, 2, 64), z(2, 0, 2))
    assert o.shape == (2, 0, 2, 64)
    o = damp.lin_decode_step(L, pool, z(0, 2, 64), z(0, 2, 64), z(0, 2, 64), z(0, 2))
    assert o.shape == (0, 2, 64) and not pool.any()
