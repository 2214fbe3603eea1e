"""Attention over records of the 8-bit cache that cache_append did not write, or only in part: what a code stands for
is (c - 128) times its scale whatever the kernel, a scale of 0 included."""
import math

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import cache_ref as R
from tests.test_gpu_cache import BF, DEV, F32, filled, gen, i32, randn, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def clean_status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


def scales_of(pool, d):
    """The scales [pages, Hk, 2] of a pool, a view."""
    return pool[..., 64 * d:64 * d + 8].view(torch.float32)


# one token, drafts in one block of rows, prompts in one and in two
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk,d", [(8, 2, 64), (8, 2, 128), (16, 2, 256)])
@pytest.mark.parametrize("T", [1, 6, 30, 90])
def test_scale_zero_stands_for_zeros(dtype, H, Hk, d, T):
    """Pages as new_cache and zero_slots leave them (codes 0, scales 0), and any codes under a scale of 0 of the keys, of
    the values or of both."""
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, 3, 9, d + T)
    g = gen(T)
    codes = lambda n: torch.randint(0, 256, (n, Hk, 64 * d), generator=g, device=DEV, dtype=torch.uint8)
    at = pages.long()
    pool[at[0, 1]] = 0
    damp.zero_slots([pool], pages[0, 5:7].contiguous())
    pool[at[1, 2:6], :, :64 * d] = codes(4)
    s = scales_of(pool, d)
    s[at[1, 2], :, 0] = 0
    s[at[1, 3], :, 1] = 0
    s[at[1, 4]] = 0
    s[at[1, 5], 0] = 0  # one head alone
    pool[at[2]] = 0  # nothing was ever written
    q = 1.5 * randn(g, 3, T, H, d)
    run_attend(layout, pool, pages, q.to(dtype), [288, 280, 200], "scales of 0")
    run_attend(layout, pool, pages, q.to(dtype), [250, 288, 100], "scales of 0, a window", window=100)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 20, 70])
def test_zeros_appended_behind_tokens_that_nothing_wrote(dtype, T):
    """start lies inside a zeroed page: the tokens before it stand for zeros, also where the tokens after it are zeros
    and the scale stays 0; and as many tokens decode as read back."""
    layout = damp.CacheLayout(8, 2, 128)
    pool = damp.new_cache(layout, 8, DEV)
    pages = i32([[0, 1, 2], [3, 4, 5]])
    g = gen(T)
    k, v = randn(g, 2, 50, 2, 128), randn(g, 2, 50, 2, 128)
    k[0, :12] = 0  # the rest of the page that start lies in
    v[0, :12] = 0
    v[1, :, 0] = 0
    start = [20, 9]
    damp.cache_append(layout, pool, k, v, pages, i32(start))
    q = randn(g, 2, T, 8, 128)
    held = [70, 59]
    run_attend(layout, pool, pages, q.to(dtype), held, "zeros behind unwritten tokens")
    kr, vr = damp.cache_read(layout, pool, pages, i32(held), 96, dtype=F32)
    ref = R.Cache(pool, 128)
    for w, got in enumerate((kr, vr)):
        for b in range(2):
            want = ref.values(w, pages[b].cpu(), torch.float32)
            want[held[b]:] = 0
            assert torch.equal(got[b].cpu(), want)
            assert not got[b, :start[b]].any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk,d", [(8, 2, 64), (8, 2, 128), (16, 2, 256), (32, 1, 128)])
@pytest.mark.parametrize("T,window", [(2, None), (6, None), (30, None), (90, None), (90, 40), (6, 60), (1, 60)])
def test_unseen_values_change_nothing(dtype, H, Hk, d, T, window):
    """A page whose values are larger by 1e30, in the middle of a context: the queries before it and those whose window
    has left it behind give the same bits as without it, the others its values."""
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, 3, 10, d + T)
    large = pool.clone()
    q = (1.5 * randn(gen(T), 3, T, H, d)).to(dtype)
    held, at = [260, 255 + max(T, 4) // 2, 286], [8, 8, 6 if window else 8]
    for b in range(3):
        scales_of(large, d)[pages[b, at[b]].long(), :, 1] *= 1e30
    seen = torch.zeros(3, T, dtype=torch.bool)
    for b in range(3):
        for t in range(T):
            last = held[b] - T + t
            first = max(0, last - window + 1) if window else 0
            seen[b, t] = first < 32 * (at[b] + 1) and last >= 32 * at[b]
    wide = torch.cat((pages, torch.full((3, 70), -1, dtype=torch.int32, device=DEV)), 1)
    for table in (pages, wide):
        a = damp.cache_attend(layout, large, q, table, i32(held), window=window)
        b = damp.cache_attend(layout, pool, q, table, i32(held), window=window)
        assert not seen.all()
        assert torch.equal(a[~seen], b[~seen]) and b[~seen].any(-1).all()
        want, bounds = R.attend(R.Cache(large, d), q, pages.cpu(), held, window=window)
        R.check_attend(a, want, bounds, max(held), d, "large values")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 6, 40])
def test_every_bad_page_is_reported(dtype, T):
    """Entries outside the pool at both ends of their range."""
    layout = damp.CacheLayout(8, 2, 64)
    pool, pages = filled(layout, 1, 4, T)
    q = randn(gen(1), 1, T, 8, 64).to(dtype)
    for bad in (-2**31, -2**31 + 1, -1, pool.shape[0], 2**31 - 1):
        table = pages.clone()
        table[0, 2] = bad
        o = damp.cache_attend(layout, pool, q, table, i32([128]))
        assert damp.device_status() == damp.DEV_BAD_SLOT, bad
        want, bounds = R.attend(R.Cache(pool, 64), q, table.cpu(), [128])
        R.check_attend(o, want, bounds, 128, 64, "bad pages")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("scale,qsize,ksize", [(3e38, 1e-30, 1e-9), (1e-44, 1e30, 1e13), (1.2e-38, 1e20, 1e17)])
def test_extreme_scales(dtype, T, scale, qsize, ksize):
    """The largest and the smallest factors of q.k, with logits of ordinary size."""
    layout = damp.CacheLayout(4, 2, 64)
    pool, pages = damp.new_cache(layout, 3, DEV), i32([[2, 0, 1]])
    g = gen(T)
    k, v = ksize * randn(g, 1, 96, 2, 64), randn(g, 1, 96, 2, 64)
    damp.cache_append(layout, pool, k, v, pages, i32([0]))
    q = qsize * randn(g, 1, T, 4, 64)
    run_attend(layout, pool, pages, q.to(dtype), [96], "extreme scales", scale=torch.tensor(scale, dtype=F32).item())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk,d", [(8, 2, 64), (8, 2, 128), (16, 2, 256)])
@pytest.mark.parametrize("T", [1, 6, 30, 90])
def test_large_logits_pick_one_token(dtype, H, Hk, d, T):
    """Logits far apart, up to sizes of which FP32 holds no unit any more: the largest takes all.

    A logit is within (d + 8) 2^-23 of sum |q k| (and FP32 queries' two parts, 2^-21); where the largest leads by
    more than twice that and by 40, the other weights are below e^-40 of its own, and the output is its value: a weight in
    FP16 (2^-11; two parts 2^-20), rounded to BF16 (2^-8) or FP32 (2^-24), its exponential and the inverse (2^-20).
    The others add e^-40 of the largest value each, to values of 0 as well."""
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, 2, 9, d + T)
    held = [288, 250]
    ref = R.Cache(pool, d)
    eps = (2.0 ** -11 + 2.0 ** -8 if dtype == BF else 2.0 ** -20 + 2.0 ** -24) + 2.0 ** -20
    few = dtype == F32 or T * (H // Hk) <= 16  # 16 rows at a time: up to FP32's range; else up to 2^60
    for size in (300.0, 1e4, 1e6, 1e9, 1e13, 1e16) + ((1e20, 1e30, 1e36) if few else ()):
        q = (size * randn(gen(T), 2, T, H, d)).to(dtype)
        o = damp.cache_attend(layout, pool, q, pages, i32(held)).double().cpu()
        assert torch.isfinite(o).all(), size
        sure = 0
        for b in range(2):
            k, v = (ref.values(w, pages[b].cpu())[:held[b]] for w in (0, 1))
            unseen = torch.arange(held[b]) > torch.arange(held[b] - T, held[b])[:, None]
            for h in range(H):
                x = q[b, :, h].double().cpu()
                z = (x @ k[:, h // (H // Hk)].T * d ** -0.5).masked_fill(unseen, float("-inf"))
                reach = (x.abs() @ k[:, h // (H // Hk)].abs().T * d ** -0.5).amax(-1)
                two, at = z.topk(2, -1)
                clear = two[:, 0] - two[:, 1] > 40 + 2 * reach * ((d + 8) * 2.0 ** -23 + 2.0 ** -21)
                sure += int(clear.sum())
                want = v[at[:, 0], h // (H // Hk)]
                rest = held[b] * math.exp(-40) * v.abs().max()
                assert ((o[b, :, h] - want).abs()[clear] <= eps * want.abs()[clear] + rest).all(), size
        assert sure > T * H  # of 2 T H; more than half


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("T,window", [(6, None), (30, None), (90, None), (90, 40), (30, 70)])
def test_unseen_keys_change_nothing(dtype, d, T, window):
    """As test_unseen_values_change_nothing with keys larger by 1e12: bits of the queries that do not see them."""
    layout = damp.CacheLayout(8, 2, d)
    pool, pages = filled(layout, 2, 10, d + T)
    large, at, held = pool.clone(), [8, 6], [255 + max(T, 4) // 2, 286]
    for b in range(2):
        scales_of(large, d)[pages[b, at[b]].long(), :, 0] *= 1e12
    q = (1.5 * randn(gen(T), 2, T, 8, d)).to(dtype)
    last = torch.tensor(held)[:, None] - T + torch.arange(T)
    first = (last - (window - 1)).clamp(min=0) if window else torch.zeros_like(last)
    page = torch.tensor(at)[:, None]
    seen = (first < 32 * (page + 1)) & (last >= 32 * page)
    a, b = (damp.cache_attend(layout, x, q, pages, i32(held), window=window) for x in (large, pool))
    assert not seen.all() and torch.equal(a[~seen], b[~seen]) and b[~seen].any(-1).all()
    assert torch.isfinite(a).all()
