"""The bounded waits of attention over the 8-bit cache, made to run out without a fault or a hang: in every second
range of the work barriers expect more bytes than are copied and give up after 10 ms.  No output is made of parts that a
range did not leave: what is not right stays as it was or becomes NaN."""
import time

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests.test_gpu_cache import BF, filled, gen, i32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


# a CTA per item; ranges of a few rows; one block of rows, two, items in parts and whole
@pytest.mark.parametrize("queries", [False, True])
@pytest.mark.parametrize("B,T,H,Hk,W", [(3, 1, 8, 2, 8), (2, 1, 8, 2, 300), (2, 3, 8, 2, 200), (3, 9, 8, 2, 40), (3, 70, 8, 2, 40),
                                        (2, 70, 16, 2, 100), (20, 60, 8, 2, 12)])
def test_waits_run_out(queries, B, T, H, Hk, W):
    layout = damp.CacheLayout(H, Hk, 128)
    pool, pages = filled(layout, B, W, T)
    q = randn(gen(T), B, T, H, 128, dtype=BF)
    lengths = i32([32 * W - 5 * b for b in range(B)])
    good = damp.cache_attend(layout, pool, q, pages, lengths)
    assert damp.device_status() == 0
    kept = pool.clone()
    stale = torch.ones(1 << 26, dtype=BF, device="cuda")  # what the workspace may hold
    del stale
    o = torch.full_like(q, 7.0)
    t0 = time.perf_counter()
    damp.test_cache_attend_wait_timeout(layout, pool, q, pages, lengths, o, queries=queries)
    many = T * (H // Hk) > 16
    status = damp.device_status()
    assert time.perf_counter() - t0 < 2.0  # not the 2 s of an ordinary call
    right = (o == good).all(-1)
    if queries and not many:  # queries are read without a barrier
        assert status == 0 and right.all()
    else:
        assert status == damp.DEV_WAIT_TIMEOUT and not right.all()
    assert (right | (o == 7.0).all(-1) | o.isnan().all(-1)).all()
    assert torch.equal(pool, kept)
    assert torch.equal(damp.cache_attend(layout, pool, q, pages, lengths), good)
