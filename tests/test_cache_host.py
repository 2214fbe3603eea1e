"""The softmax-attention layers' operators on the host: the C ABI and the Python binding reject bad
arguments before anything is enqueued; the cache's layout and the rotary frequencies."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_27513_gb300 as damp
from paper_2608_27513_gb300 import _lib, build
from tests import cache_ref as R
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


def layout(H=4, Hk=2, d=64):
    return ctypes.byref(_lib.DampCacheLayout(H, Hk, d))


def test_page_bytes(L):
    for H, Hk, d in ((4, 2, 64), (32, 8, 128), (16, 2, 256)):
        assert L.damp_cache_page_bytes(layout(H, Hk, d)) == Hk * (64 * d + 16)
        assert damp.CacheLayout(H, Hk, d).record_bytes == 64 * d + 16
    for bad in ((4, 3, 64), (4, 0, 64), (0, 1, 64), (4, 2, 32), (4, 2, 96), (4, 2, 512), (4, -2, 64), (1 << 17, 1, 64)):
        assert L.damp_cache_page_bytes(layout(*bad)) == 0
    assert L.damp_cache_page_bytes(None) == 0


def test_rotary_rejects_bad_arguments(L, fb):
    def call(**over):
        a = dict(q=_p(fb, 0), q_stride=256, heads=4, k=_p(fb, 1), k_stride=128, kv_heads=2, d=64, dtype=0, positions=_p(fb, 2),
                 per_row=0, batch=3, T=5, freq=_p(fb, 3), r=64, inter=0, scale=1.0, q_out=_p(fb, 4), k_out=_p(fb, 5), stream=None)
        a.update(over)
        return L.damp_rotary(*a.values())

    assert call(batch=0) == OK and call(T=0) == OK
    for name in ("q", "k", "positions", "freq", "q_out", "k_out"):
        assert call(**{name: None}) == NULL, name
    for over in (dict(batch=-1), dict(T=-1), dict(d=0), dict(d=1025), dict(r=0), dict(r=63), dict(r=66), dict(heads=0), dict(heads=1025),
                 dict(kv_heads=-1), dict(kv_heads=1025), dict(q_stride=255), dict(k_stride=127), dict(q_stride=1 << 60),
                 dict(batch=1 << 16, T=1 << 16)):
        assert call(**over) == SHAPE, over
    assert call(dtype=2) == FORMAT
    for name, i, off in (("q", 0, 1), ("k_out", 5, 1), ("positions", 2, 2), ("freq", 3, 4)):
        assert call(**{name: _p(fb, i, off)}) == ALIGN, name
    assert call(q_out=_p(fb, 0), q_stride=300) == ALIAS   # in place, but not contiguous
    assert call(q_out=_p(fb, 0, 2)) == ALIAS
    assert call(q_out=_p(fb, 1)) == ALIAS
    assert call(k_out=_p(fb, 4, 64)) == ALIAS
    assert call(k_out=_p(fb, 3)) == ALIAS
    assert call(q_out=_p(fb, 2)) == ALIAS


def test_cache_rejects_bad_arguments(L, fb):
    base = dict(layout=layout(), cache=_p(fb, 0), num_pages=8, pages=_p(fb, 1), table=2, batch=3, T=5)

    def append(**over):
        a = dict(base, start=_p(fb, 2), lengths=None, k=_p(fb, 3), k_stride=128, v=_p(fb, 4), v_stride=128, dtype=0, stream=None)
        a.update(over)
        return L.damp_cache_append(*a.values())

    def read(**over):
        a = dict(base, start=None, lengths=_p(fb, 2), k=_p(fb, 3), v=_p(fb, 4), dtype=0, stream=None)
        a.update(over)
        return L.damp_cache_read(*a.values())

    need = L.damp_cache_attend_workspace(layout(), 3, 5, 200, 0)
    assert need > 0 and need <= 1 << 22

    def attend(**over):
        a = dict(base, table=200, lengths=_p(fb, 2), q_lengths=None, q=_p(fb, 3), q_stride=256, scale=0.125, window=0, o=_p(fb, 4), dtype=0,
                 ws=_p(fb, 5), ws_bytes=need, stream=None)
        a.update(over)
        return L.damp_cache_attend(*a.values())

    for f, optional in ((append, ("lengths",)), (read, ("start",)), (attend, ("q_lengths",))):
        assert f(batch=0) == OK and f(T=0) == OK
        assert f(layout=None) == NULL
        for bad in ((4, 3, 64), (4, 2, 96), (0, 1, 64)):
            assert f(layout=layout(*bad)) == SHAPE
        for over in (dict(num_pages=0), dict(num_pages=1 << 31), dict(table=0), dict(table=(1 << 25) + 1), dict(batch=-1),
                     dict(batch=4097), dict(T=-1)):
            assert f(**over) == SHAPE, over
        assert f(dtype=2) == FORMAT
        for name in ("cache", "pages"):
            assert f(**{name: None}) == NULL
        assert f(cache=_p(fb, 0, 8)) == ALIGN and f(pages=_p(fb, 1, 2)) == ALIGN
        for name in optional:
            assert f(**{name: _p(fb, 6, 2)}) == ALIGN
    for name in ("start", "k", "v"):
        assert append(**{name: None}) == NULL
    for over in (dict(k_stride=127), dict(v_stride=120), dict(k_stride=132), dict(k_stride=1 << 60), dict(T=(1 << 31) - 1, batch=4096)):
        assert append(**over) == SHAPE, over
    assert append(k=_p(fb, 3, 8)) == ALIGN and append(start=_p(fb, 2, 1)) == ALIGN
    for name in ("k", "v", "start", "lengths", "pages"):
        assert append(**{name: _p(fb, 0, 64)}) == ALIAS
    for name in ("lengths", "k", "v"):
        assert read(**{name: None}) == NULL
    assert read(v=_p(fb, 4, 8)) == ALIGN
    for over in (dict(k=_p(fb, 0)), dict(v=_p(fb, 3)), dict(lengths=_p(fb, 3)), dict(pages=_p(fb, 4)), dict(start=_p(fb, 4))):
        assert read(**over) == ALIAS, over
    assert read(batch=4096, T=(1 << 31) - 1) == SHAPE
    for name in ("lengths", "q", "o", "ws"):
        assert attend(**{name: None}) == NULL
    for over in (dict(q_stride=255), dict(q_stride=260), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                 dict(window=-1), dict(ws_bytes=need - 1), dict(T=1 << 27), dict(table=1 << 25, T=128)):
        assert attend(**over) == SHAPE, over
    for name, i in (("q", 3), ("o", 4), ("ws", 5)):
        assert attend(**{name: _p(fb, i, 8)}) == ALIGN
    for over in (dict(o=_p(fb, 3)), dict(o=_p(fb, 0)), dict(o=_p(fb, 5, 16)), dict(ws=_p(fb, 0)), dict(q_lengths=_p(fb, 4)), dict(ws=_p(fb, 2))):
        assert attend(**over) == ALIAS, over
    for a in ((None, 3, 5, 200, 0), (layout(4, 3, 64), 3, 5, 200, 0), (layout(), 0, 5, 200, 0), (layout(), 3, 0, 200, 0), (layout(), 4097, 1, 200, 0),
              (layout(), 3, 5, 0, 0)):
        assert L.damp_cache_attend_workspace(*a) == 0
    # few rows of short tables need none
    assert L.damp_cache_attend_workspace(layout(), 1, 1, 4, 0) == 0
    assert attend(batch=0, ws=None, ws_bytes=0) == OK


def test_binding_rejects_bad_tensors(L):
    lay = damp.CacheLayout(4, 2, 64)
    pool = torch.zeros(6, 2, lay.record_bytes, dtype=torch.uint8)
    pages = torch.zeros(3, 2, dtype=torch.int32)
    n = torch.zeros(3, dtype=torch.int32)
    q, k = torch.zeros(3, 5, 4, 64), torch.zeros(3, 5, 2, 64)
    freq, _ = damp.rotary_frequencies(64, device="cpu")
    pos = torch.zeros(3, 5, dtype=torch.int32)
    bad = [
        lambda: damp.cache_append(lay, pool, k, k, pages, n),                       # not on the GPU
        lambda: damp.cache_append(lay, pool[:, :1], k, k, pages, n),
        lambda: damp.cache_append(lay, pool[0], k, k, pages, n),
        lambda: damp.cache_append(lay, pool, k[0], k, pages, n),
        lambda: damp.cache_append(lay, pool, None, k, pages, n),
        lambda: damp.cache_append(lay, pool, k, k, pages[0], n),
        lambda: damp.cache_append(lay, pool, k, k, pages, None),
        lambda: damp.cache_read(lay, pool, pages, None, 4),
        lambda: damp.cache_read(lay, pool, pages, n, -1),
        lambda: damp.cache_read(lay, pool, None, n, 4),
        lambda: damp.cache_attend(lay, pool, q, pages, n),
        lambda: damp.cache_attend(lay, pool, q[0], pages, n),
        lambda: damp.cache_attend(lay, pool, q, pages, None),
        lambda: damp.cache_attend(lay, pool, q, pages, n, window=0),
        lambda: damp.rotary(q, k, pos, freq),
        lambda: damp.rotary(q[0], k, pos, freq),
        lambda: damp.rotary(q, k, pos, None),
        lambda: damp.rotary(q, k, pos[0, 0], freq),
        lambda: damp.rotary_frequencies(63),
        lambda: damp.rotary_frequencies(64, factor=0.5),
        lambda: damp.rotary_frequencies(64, base=1.0),
        lambda: damp.rotary_frequencies(64, scaling="other"),
        lambda: damp.rotary_frequencies(2, scaling="ntk"),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(str(i))
    for f in (lambda: damp.cache_append(lay, pool, k.half(), k.half(), pages, n), lambda: damp.cache_attend(lay, pool, q.double(), pages, n),
              lambda: damp.rotary(q.half(), k.half(), pos, freq), lambda: damp.cache_read(lay, pool, pages, n, 4, dtype=torch.float16)):
        with pytest.raises(TypeError):
            f()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_record_is_a_permutation_without_conflicts(d):
    """Every byte of the rows once; and the 16-byte columns of a 128-byte line that the kernels' accesses hit."""
    at = R.order(d)
    assert sorted(at.reshape(-1)) == list(range(32 * d))
    column = lambda t, m: R.byte_of(t, 16 * m, d) // 16 % 8
    if d >= 128:
        for m in range(d // 16):  # eight tokens, one chunk
            assert len({column(t, m) for t in range(8)}) == 8
        for t in range(0, 8, 2):  # a pair of tokens, four chunks
            for j in range(d // 64):
                assert len({column(x, 4 * j + c) for x in (t, t + 1) for c in range(4)}) == 8
        for e in (0, 1):          # tokens 2c + e, two chunks
            for g in range(0, 8, 2):
                assert len({column(2 * c + e, m) for c in range(4) for m in (g, g + 1)}) == 8


def test_rotary_frequencies():
    f, s = damp.rotary_frequencies(128, device="cpu")
    assert f.dtype == torch.float64 and s == 1.0 and f[0] == 1.0
    assert torch.allclose(f, torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(damp.rotary_frequencies(128, scaling="linear", factor=4.0, device="cpu")[0], f / 4)
    n, _ = damp.rotary_frequencies(128, scaling="ntk", factor=8.0, device="cpu")
    assert n[0] == 1.0 and math.isclose(n[-1], f[-1] / 8, rel_tol=1e-12)
    y, s = damp.rotary_frequencies(128, scaling="yarn", factor=8.0, trained=4096, device="cpu")
    assert math.isclose(s, 0.1 * math.log(8.0) + 1)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(y[turns > 34], f[turns > 34])
    assert torch.allclose(y[turns < 0.9], f[turns < 0.9] / 8, rtol=1e-15)
    assert (y <= f).all() and (y >= f / 8).all() and (y[1:] < y[:-1]).all()
    assert damp.rotary_frequencies(2, device="cpu")[0].tolist() == [1.0]


def test_reference_append_bounds():
    """The reference's own codes: within half a step, and half a step more for each growth of the scale."""
    rng = np.random.default_rng(1)
    pool = torch.zeros(2, 1, 64 * 64 + 16, dtype=torch.uint8)
    ref = R.Cache(pool, 64)
    x = torch.from_numpy(rng.standard_normal((1, 32, 1, 64)).astype(np.float32))
    pages = torch.tensor([[1]])
    for t in range(32):
        ref.append(x[:, t:t + 1], x[:, t:t + 1], pages, [t])
    got = ref.values(0, [1])[:, 0]
    step = float(ref.scales[0][1, 0])
    assert step == np.float32(x.abs().max()) / np.float32(127)
    growths = sum(1 for t in range(1, 32) if x[0, t].abs().max() > x[0, :t].abs().max())
    assert (got - x[0, :, 0].double()).abs().max() <= step * (0.5 + 0.5 * growths) * (1 + 1e-5)
    assert torch.equal(R.Cache(ref.pool(), 64).pool(), ref.pool())


def test_layouts_are_copied_and_pickled():
    import copy
    import pickle
    A = damp.CacheLayout(8, 2, 128)
    for B in (copy.deepcopy(A), copy.copy(A), pickle.loads(pickle.dumps(A)), pickle.loads(pickle.dumps({"attn": A}))["attn"]):
        assert B == A and hash(B) == hash(A) and B.c().num_kv_heads == 2 and B.record_bytes == A.record_bytes


def test_binding_refuses_sizes_past_32_bits(L):
    """A size that does not fit the C call's 32 bits is refused, not cut off."""
    many = (1 << 32) + 1
    q = torch.empty((1, many, 1, 2), dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="tokens"):
        damp._token_rows("q", q, q.shape, torch.bfloat16, q.get_device())
    A = damp.CacheLayout(4, 2, 64)
    pool = torch.empty((3, 2, A.record_bytes), dtype=torch.uint8, device="meta")
    pages = torch.empty((1, many), dtype=torch.int32, device="meta")
    with pytest.raises(ValueError, match="pages"):
        damp._cache(A, pool, pages, 1, pool.get_device(), torch.int32, torch.uint8)


def test_sizes_near_the_limits_are_refused(L, fb):
    """Sums of 32-bit indices in the kernels stay below 2^31."""
    append = [layout(4, 1), _p(fb, 0), 8, _p(fb, 1), 2, 1, (1 << 31) - 8, _p(fb, 2), None, _p(fb, 3), 64, _p(fb, 4), 64, 0, None]
    assert L.damp_cache_append(*append) == SHAPE
    tiles, table = 6, 1 << 25  # 6 tiles of 16 rows, 3 batch rows, 2 KV heads: 1.2e9 pages
    need = L.damp_cache_attend_workspace(layout(), 3, 8 * tiles, table, 0)
    attend = [layout(), _p(fb, 0), 8, _p(fb, 1), table, 3, 8 * tiles, _p(fb, 2), None, _p(fb, 3), 256, 0.125, 0, _p(fb, 4), 0, _p(fb, 5), need, None]
    assert L.damp_cache_attend(*attend) == SHAPE
