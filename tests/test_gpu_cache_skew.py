"""Batches in which one row is far longer than the others: no call may take the time that one SM needs for it."""
import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import cache_ref as R
from tests.test_gpu_cache import BF, DEV, filled, gen, i32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


def batch(rows, T, long, short):
    """Row 7 has a context of its own, the others share theirs."""
    layout = damp.CacheLayout(16, 8, 64)
    pool, some = filled(layout, 1, long // R.PAGE, 1)
    pages = some.repeat(rows, 1)
    lengths = i32(short + torch.arange(rows) % 50)
    lengths[7] = long
    return layout, pool, pages, lengths, randn(gen(rows), rows, T, 16, 64, dtype=BF)


@pytest.mark.parametrize("T,window", [(20, None), (20, 600)])
def test_one_long_row_among_many(T, window):
    layout, pool, pages, lengths, q = batch(180, T, 6400, 200)
    q_lengths = i32([T - b % 3 for b in range(180)])
    o = damp.cache_attend(layout, pool, q, pages, lengths, q_lengths=q_lengths, window=window)
    at = torch.tensor([0, 6, 7, 8, 100, 179])
    want, bounds = R.attend(R.Cache(pool, 64), q[at], pages[at].cpu(), lengths[at].tolist(), q_lengths=q_lengths[at].tolist(), window=window)
    R.check_attend(o[at], want, bounds, 6400, 64, "a long row")


def test_one_long_row_takes_no_long_time():
    """Against the long row alone (whose work is spread) and the others alone.  Both together need at most the sum; one
    SM would need many times that for the long row's items alone.  Twice the sum is allowed."""
    layout, pool, pages, lengths, q = batch(180, 9, 65536, 200)
    rest = lengths.clone()
    rest[7] = 200

    def time(*a):
        for _ in range(2):
            damp.cache_attend(layout, pool, *a)
        best = float("inf")
        for _ in range(5):
            s, e = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            s.record()
            for _ in range(5):
                damp.cache_attend(layout, pool, *a)
            e.record()
            torch.cuda.synchronize()
            best = min(best, s.elapsed_time(e))
        return best

    both, one, others = time(q, pages, lengths), time(q[7:8], pages[7:8], lengths[7:8]), time(q, pages, rest)
    assert both <= 2 * (one + others), (both, one, others)
