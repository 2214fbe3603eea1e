"""Slots of state pools on the GPU: copy (fork, reorder, overlapping lists), free and
compact, byte for byte against indexing, over pool sizes, counts and bad entries."""
import random

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


def _pool(slots, nbytes, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed + nbytes)
    return torch.randint(0, 256, (slots, nbytes), generator=gen, device=DEV, dtype=torch.uint8)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _expect_copy(pool, src, dst):
    want = pool.clone()
    keep = [(s, d) for s, d in zip(src, dst) if 0 <= s < pool.shape[0] and 0 <= d < pool.shape[0]]
    if keep:
        s, d = zip(*keep)
        want[list(d)] = pool[list(s)]
    return want


SIZES = [16, 48, 4096, 20224, 626688 + 16]


@pytest.mark.parametrize("nbytes", SIZES)
@pytest.mark.parametrize("n", [1, 2, 7, 64, 150])
@pytest.mark.parametrize("how", ["disjoint", "fork", "permute", "rotate", "mixed"])
def test_copy(nbytes, n, how):
    slots = 2 * n + 3
    rng = random.Random(n * 31 + nbytes)
    order = rng.sample(range(slots), slots)
    src, dst = order[:n], order[n:2 * n]
    if how == "fork":
        src = [order[-1]] * n
    elif how == "permute":
        dst = rng.sample(src, n)
    elif how == "rotate":
        dst = src[1:] + src[:1]
    elif how == "mixed":  # runs of one source, sources that are destinations, pairs to skip
        src = [rng.choice(order[:max(1, n // 2)]) for _ in range(n)]
        dst = rng.sample(range(slots), n)
        src[n // 2] = -1
        dst[n // 3] = -5
    pools = [_pool(slots, nbytes, 1), _pool(slots, 32, 2), _pool(slots, 20224, 3)]
    want = [_expect_copy(p, src, dst) for p in pools]
    damp.copy_slots(pools, _i32(src), _i32(dst))
    for p, w in zip(pools, want):
        assert torch.equal(p, w)


def test_copy_of_many_entries():
    for n in (1000, 2049, 4096):
        slots = n + 5
        rng = random.Random(n)
        src, dst = [rng.randrange(slots) for _ in range(n)], rng.sample(range(slots), n)
        pool = _pool(slots, 272, 4)
        want = _expect_copy(pool, src, dst)
        damp.copy_slots(pool, _i32(src), _i32(dst))
        assert torch.equal(pool, want)
    with pytest.raises(damp.DampError):
        damp.copy_slots(pool, torch.zeros(4097, dtype=torch.int32, device=DEV), torch.zeros(4097, dtype=torch.int32, device=DEV))


def test_many_pools_and_other_types():
    slots, n = 9, 4
    L = damp.Layout(4, 2, 64, 64, 8)
    pools = [_pool(slots, 16 * (1 + i % 5), i) for i in range(70)]
    pools += [torch.randn(slots, 4, 64, 64, device=DEV), damp.new_state(L, slots, DEV).random_(0, 256)]
    src, dst = [8, 8, 0, 3], [1, 0, 3, 8]
    want = [_expect_copy(p, src, dst) for p in pools]
    damp.copy_slots(pools, _i32(src), _i32(dst))
    assert all(torch.equal(p, w) for p, w in zip(pools, want))
    for w in want:
        w[[2, 7]] = 0
    damp.zero_slots(pools, _i32([7, -1, 2]))
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


def test_bad_entries_are_skipped_and_reported():
    pool = _pool(5, 4096)
    before = pool.clone()
    damp.copy_slots(pool, _i32([0, 5, 1]), _i32([9, 2, 3]))
    assert damp.device_status() == damp.DEV_BAD_SLOT
    before[3] = before[1]
    assert torch.equal(pool, before)
    damp.zero_slots(pool, _i32([5, 4, 1 << 30]))
    assert damp.device_status() == damp.DEV_BAD_SLOT
    before[4] = 0
    assert torch.equal(pool, before)
    assert damp.compact_slots(pool, _i32([4, 77, -1])).tolist() == [0, -1, -1]
    assert damp.device_status() == damp.DEV_BAD_SLOT
    before[0] = before[4]
    assert torch.equal(pool, before)


@pytest.mark.parametrize("nbytes", [16, 20224, 626688])
@pytest.mark.parametrize("n", [0, 1, 37, 300])
def test_zero(nbytes, n):
    slots = 333 if nbytes < 100000 else 301
    pools = [_pool(slots, nbytes), _pool(slots, 48)]
    idx = random.Random(n).sample(range(slots), n)
    want = [p.clone() for p in pools]
    for w in want:
        w[idx] = 0
    damp.zero_slots(pools, _i32(idx))
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


@pytest.mark.parametrize("slots,live", [(1, 1), (2, 1), (31, 9), (32, 32), (33, 20), (64, 1), (256, 131), (256, 255), (1000, 500),
                                        (70000, 3000)])
def test_compact(slots, live):
    rng = random.Random(slots + live)
    idx = rng.sample(range(slots), live)
    rows = idx + [-1, -7]
    rng.shuffle(rows)
    if live > 3:
        rows.append(idx[2])  # two requests on one slot move together
    pools = [_pool(slots, 48), _pool(slots, 1040)]
    before = [p.clone() for p in pools]
    out = damp.compact_slots(pools, _i32(rows)).tolist()
    assert out == R.compact(rows, slots)
    for p, b in zip(pools, before):
        pairs = [(s, d) for s, d in zip(rows, out) if d >= 0]
        assert torch.equal(p[[d for _, d in pairs]], b[[s for s, _ in pairs]])
        untouched = sorted(set(range(slots)) - {d for _, d in pairs})
        assert torch.equal(p[untouched], b[untouched])


def test_compact_edges():
    pool = _pool(40, 32)
    before = pool.clone()
    assert damp.compact_slots(pool, _i32([-1, -1])).tolist() == [-1, -1]          # nothing lives
    assert damp.compact_slots(pool, _i32([39])).tolist() == [0]
    before[0] = before[39]
    full = list(range(40))
    random.Random(1).shuffle(full)
    assert damp.compact_slots(pool, _i32(full)).tolist() == full                   # nothing moves
    assert torch.equal(pool, before)
    assert damp.compact_slots(pool, _i32([])).tolist() == []
    huge = torch.zeros(1 << 18, 16, dtype=torch.uint8, device=DEV)
    assert damp.compact_slots(huge, _i32([262143, 5, 262142])).tolist() == R.compact([262143, 5, 262142], 1 << 18)
    with pytest.raises(damp.DampError):
        damp.compact_slots(torch.zeros((1 << 18) + 1, 16, dtype=torch.uint8, device=DEV), _i32([3]))


def test_offsets_past_32_bits():
    nbytes = (1 << 30) + 16
    pool = torch.zeros(6, nbytes, dtype=torch.uint8, device=DEV)
    pool[5].random_(0, 256)
    last = pool[5].clone()
    damp.copy_slots(pool, _i32([5, 5]), _i32([0, 4]))
    assert torch.equal(pool[0], last) and torch.equal(pool[4], last) and not pool[1:4].any()
    damp.zero_slots(pool, _i32([5, 0]))
    assert not pool[5].any() and not pool[0].any() and torch.equal(pool[4], last)


def test_free_lists_up_to_the_last_32_bit_length():
    pool = _pool(4, 16)
    want = pool.clone()
    want[[1, 2]] = 0
    idx = torch.full(((1 << 31) - 1,), -1, dtype=torch.int32, device=DEV)
    idx[65535 * 32768 - 1], idx[-1] = 1, 2  # the last entry of a full launch, and the last of all
    damp.zero_slots(pool, idx)
    assert torch.equal(pool, want)


def test_another_stream_and_a_graph():
    pools = [_pool(20, 20224, 1), _pool(20, 4096, 2)]
    src, dst, live = _i32([3, 4, 5]), _i32([4, 5, 3]), _i32([19, 3, 18, 0])
    want = [_expect_copy(p, [3, 4, 5], [4, 5, 3]) for p in pools]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    damp.copy_slots(pools, src, dst, stream=side)
    out = damp.compact_slots(pools, live, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert out.tolist() == R.compact([19, 3, 18, 0], 20)
    new = out.tolist()
    for p, w in zip(pools, want):
        assert torch.equal(p[new], w[[19, 3, 18, 0]])
    start = [p.clone() for p in pools]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        damp.copy_slots(pools, src, dst)
        damp.zero_slots(pools, src)
    graph.replay()
    torch.cuda.synchronize()
    for p, s in zip(pools, start):
        w = _expect_copy(s, [3, 4, 5], [4, 5, 3])
        w[[3, 4, 5]] = 0
        assert torch.equal(p, w)
