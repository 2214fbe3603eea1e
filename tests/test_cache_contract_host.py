"""The softmax-attention layers' calls on the host, beyond their refusals of bad arguments."""
import ctypes

import pytest

import paper_2608_27513_gb300 as damp
from paper_2608_27513_gb300 import _lib, build
from tests.test_abi_host import FakeBuffers

OK, NULL, SHAPE, ALIGN, ALIAS, FORMAT = range(6)


@pytest.fixture(scope="module")
def L():
    build.build()
    return _lib.lib()


def test_wait_test_hook_accepts_only_its_instances(L):
    """The test of the bounded waits runs d = 128 and BF16 alone, with the checks of the call that it tests."""
    fb = FakeBuffers(n=8, size=1 << 22)
    need = L.damp_cache_attend_workspace(ctypes.byref(_lib.DampCacheLayout(8, 2, 128)), 2, 1, 2, 0)
    assert need <= 1 << 22

    def call(layout=(8, 2, 128), batch=2, T=1, dtype=0, queries=0, **over):
        a = dict(layout=ctypes.byref(_lib.DampCacheLayout(*layout)), cache=fb[0], num_pages=8, pages=fb[1], table=2, batch=batch, T=T,
                 lengths=fb[2], q_lengths=None, q=fb[3], q_stride=layout[0] * layout[2], scale=0.125, window=0, o=fb[4], dtype=dtype,
                 ws=fb[5], ws_bytes=need, queries=queries, stream=None)
        a.update(over)
        return L.damp_test_cache_attend_wait_timeout(*a.values())

    assert call(batch=0) == OK and call(T=0, queries=1) == OK
    assert call(layout=(8, 2, 64), batch=0) == SHAPE and call(layout=(8, 2, 256)) == SHAPE and call(dtype=1) == SHAPE
    assert call(dtype=2) == SHAPE and call(layout=(8, 3, 128)) == SHAPE and call(layout=(8, 2, 96)) == SHAPE
    assert call(q=None) == NULL and call(o=fb[3]) == ALIAS


def test_workspace_sizes_are_kept_up_to_a_limit(L):
    """A server's batches, prompt lengths and tables vary without end; equal layouts share what is kept."""
    layout, twin = damp.CacheLayout(8, 2, 64), damp.CacheLayout(8, 2, 64)
    for T in range(1, 5001):
        key = (0, 3, T, 70 + T % 7, 0)
        assert damp._attend_workspace(layout, key) == L.damp_cache_attend_workspace(layout._shared[1], *key[1:])
        assert twin._shared[2][key] == layout._shared[2][key]
        assert len(layout._shared[2]) <= 1024
