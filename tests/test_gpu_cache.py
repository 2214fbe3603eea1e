"""Softmax-attention layers on the GPU: rotary positions, the 8-bit cache written and read back,
attention over it, against plain references."""
import math

import pytest
import torch

import paper_2608_27513_gb300 as damp
from tests import cache_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device=DEV)


@pytest.fixture(autouse=True)
def clean_status():
    damp.device_status()
    yield
    assert damp.device_status() == 0


# ---- rotary ----

def check_rotary(got, x, positions, freq, interleaved, scale):
    """cos and sin are within 2^-31 of a half turn (pi 2^-31) and 2 units of FP32 (2^-22) each, the two
    products and their sum within two units more; then the type's rounding."""
    want = R.rotary(x, positions, freq, interleaved, scale)
    r = 2 * len(freq)
    eps = 2.0 ** -8 if got.dtype == BF else 2.0 ** -24
    pair = R.rotary(x.double().abs(), torch.zeros_like(positions), freq, interleaved, 1.0)
    reach = torch.zeros_like(pair)
    first = slice(0, r, 2) if interleaved else slice(0, r // 2)
    second = slice(1, r, 2) if interleaved else slice(r // 2, r)
    reach[..., first] = reach[..., second] = pair[..., first] + pair[..., second]
    err = (got.double() - want).abs()
    assert (err - eps * want.abs() - scale * 2.0 ** -21 * reach).max().item() <= 0
    assert torch.equal(got[..., r:], x[..., r:])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,H,Hk,d,r", [(1, 1, 4, 4, 64, 64), (3, 5, 6, 2, 128, 128), (2, 700, 5, 1, 256, 64), (2, 3, 3, 1, 80, 34),
                                          (1, 9, 2, 2, 6, 2), (4, 300, 4, 0, 128, 96), (1, 2, 1, 1, 1024, 1024)])
def test_rotary(dtype, interleaved, B, T, H, Hk, d, r):
    g = gen(B + T + d + r)
    q, k = randn(g, B, T, H, d, dtype=dtype), randn(g, B, T, Hk, d, dtype=dtype) if Hk else None
    freq, scale = damp.rotary_frequencies(r, base=500000.0, scaling="yarn", factor=4.0, trained=1024, device=DEV)
    start = torch.randint(-5, 1 << 20, (B,), generator=g, device=DEV)
    pos = (start[:, None] + torch.arange(T, device=DEV)).to(torch.int32)
    qo, ko = damp.rotary(q, k, pos, freq, interleaved=interleaved, scale=scale)
    check_rotary(qo, q, pos, freq, interleaved, scale)
    if Hk:
        check_rotary(ko, k, pos, freq, interleaved, scale)
    else:
        assert ko is None
    # positions per row, and in place
    q2, k2 = q.clone(), None if k is None else k.clone()
    damp.rotary(q2, k2, start.to(torch.int32), freq, interleaved=interleaved, scale=scale, q_out=q2, k_out=k2)
    assert torch.equal(q2, qo) and (k is None or torch.equal(k2, ko))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_rotary_of_slices(dtype, pad):
    """q and k as slices of a projection, with an odd row length too."""
    B, T, H, Hk, d = 2, 33, 4, 2, 64
    flat = randn(gen(pad), B, T, (H + 2 * Hk) * d + pad, dtype=dtype)
    q, k = flat[..., :H * d].unflatten(-1, (H, d)), flat[..., H * d:(H + Hk) * d].unflatten(-1, (Hk, d))
    keep = flat.clone()
    freq, _ = damp.rotary_frequencies(d, device=DEV)
    pos = torch.arange(B * T, device=DEV, dtype=torch.int32).reshape(B, T)
    got = damp.rotary(q, k, pos, freq)
    want = damp.rotary(q.contiguous(), k.contiguous(), pos, freq)
    for a, b, x in zip(got, want, (q, k)):
        assert torch.equal(a, b)
        check_rotary(a, x, pos, freq, False, 1.0)
    assert torch.equal(flat, keep)


def test_rotary_far_positions():
    """The angle keeps its fraction of a turn at the largest positions, forward and back."""
    freq, _ = damp.rotary_frequencies(128, device=DEV)
    pos = i32([[2**31 - 1, -2**31, 2**30 + 12345, 0]])
    q = randn(gen(3), 1, 4, 2, 128)
    out, _ = damp.rotary(q, None, pos, freq)
    # 64 bits hold the angle to 2^-53 of 2^31 radians, 2^-22, for a pair of at most 5 each; the kernel's own
    # part is as in check_rotary, 2^-21 of |a| + |b|
    want = R.rotary(q, pos, freq, False, 1.0)
    assert q.abs().max() < 5
    assert (out.double() - want).abs().max().item() < 10 * (2.0 ** -22 + 2.0 ** -21)
    assert torch.equal(out[0, 3], q[0, 3])
    back, _ = damp.rotary(out, None, torch.where(pos == -2**31, pos, -pos), freq)
    assert (back - q)[0, [0, 2]].abs().max().item() < 2 * 10 * 2.0 ** -21


def test_rotary_empty():
    freq, _ = damp.rotary_frequencies(64, device=DEV)
    q = torch.empty(0, 4, 2, 64, device=DEV)
    assert damp.rotary(q, None, i32(torch.empty(0, 4)), freq)[0].shape == q.shape


# ---- the cache ----

def tables(g, pool_pages, B, W):
    return torch.randperm(pool_pages, generator=g, device=DEV)[:B * W].reshape(B, W).to(torch.int32)


def filled(layout, B, W, seed, extra=3, spread=True):
    """A pool with written pages, and its tables."""
    g = gen(seed)
    pool = damp.new_cache(layout, B * W + extra, DEV)
    pages = tables(g, B * W + extra, B, W)
    T, Hk, d = W * R.PAGE, layout.num_kv_heads, layout.d
    k, v = randn(g, B, T, Hk, d), randn(g, B, T, Hk, d)
    if spread:
        k[..., ::17] *= 4.0
        v *= torch.exp(randn(g, B, T // R.PAGE, 1, 1, 1)).repeat_interleave(R.PAGE, 1).reshape(B, T, 1, 1)
    damp.cache_append(layout, pool, k, v, pages, torch.zeros(B, dtype=torch.int32, device=DEV))
    return pool, pages


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hk", [1, 3])
def test_append_bits(dtype, d, Hk):
    """Calls of many lengths into open pages: the pool bit for bit, and what it is read back as."""
    layout = damp.CacheLayout(Hk, Hk, d)
    g = gen(d + Hk)
    B, W = 5, 5
    pool = torch.randint(0, 256, (B * W + 2, Hk, 64 * d + 16), generator=g, device=DEV, dtype=torch.uint8)  # stale pages
    pool[..., 64 * d:64 * d + 8] = 0
    pages = tables(g, B * W + 2, B, W)
    ref = R.Cache(pool, d)
    held = torch.zeros(B, dtype=torch.int64)
    for step, T in enumerate([1, 1, 7, 33, 1, 8, 9, 40, 2]):
        n = torch.randint(0, T + 1, (B,)) if step % 2 else None
        k, v = (randn(g, B, T, Hk, d) * math.exp(step % 3) for _ in range(2))
        k[:, :, :, 3] *= 10.0
        k, v = k.to(dtype), v.to(dtype)
        lengths = None if n is None else i32(n)
        damp.cache_append(layout, pool, k, v, pages, i32(held), lengths=lengths)
        ref.append(k, v, pages.cpu(), held, n)
        assert torch.equal(pool.cpu(), ref.pool()), step
        held = held + (T if n is None else n)
    assert held.max() <= W * R.PAGE
    for out, start in ((BF, None), (F32, i32([0, 31, 32, 5, 100]))):
        T = W * R.PAGE
        got = damp.cache_read(layout, pool, pages, i32(held), T, start=start, dtype=out)
        for w in (0, 1):
            assert got[w].dtype == out and got[w].shape == (B, T, Hk, d)
            for b in range(B):
                full = ref.values(w, pages[b].cpu(), torch.float32)  # one FP32 product, then the type's rounding
                full[int(held[b]):] = 0
                s = 0 if start is None else int(start[b])
                want = torch.zeros(T, Hk, d)
                want[:T - s] = full[s:]
                assert torch.equal(got[w][b].cpu(), want.to(out)), (out, w, b)


def test_append_slices_and_streams():
    layout = damp.CacheLayout(4, 2, 128)
    g = gen(1)
    x = randn(g, 3, 70, 8, 128, dtype=BF)
    k, v = x[:, :, 4:6], x[:, :, 6:]
    pool, other = damp.new_cache(layout, 12, DEV), damp.new_cache(layout, 12, DEV)
    pages = tables(g, 12, 3, 4)
    zero = i32([0, 0, 0])
    damp.cache_append(layout, pool, k.contiguous(), v.contiguous(), pages, zero)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    damp.cache_append(layout, other, k, v, pages, zero, stream=s)
    q = x[:, 69:, :4]
    o2 = damp.cache_attend(layout, other, q, pages, i32([70] * 3), stream=s)
    r2 = damp.cache_read(layout, other, pages, i32([70] * 3), 70, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(pool, other)
    assert torch.equal(o2, damp.cache_attend(layout, pool, q.contiguous(), pages, i32([70] * 3)))
    assert torch.equal(r2[1], damp.cache_read(layout, pool, pages, i32([70] * 3), 70)[1])


@pytest.mark.parametrize("T", [3, 40])
def test_append_extremes(T):
    """Values that are not finite, zero blocks, the smallest and largest magnitudes."""
    layout = damp.CacheLayout(2, 2, 64)
    for fill in (0.0, 1e-41, 1.2e-36, 3e38, float("nan"), float("inf")):
        pool = damp.new_cache(layout, 4, DEV)
        ref = R.Cache(pool, 64)
        pages = i32([[2, 0], [3, 1]])
        k = randn(gen(T), 2, T, 2, 64)
        v = torch.full_like(k, fill)
        v[:, :, 1] = k[:, :, 0]
        v[0, 1, 1, 5] = fill
        start = [0, 20]
        damp.cache_append(layout, pool, k, v, pages, i32(start))
        ref.append(k, v, pages.cpu(), start)
        assert damp.device_status() == (0 if math.isfinite(fill) else damp.DEV_NOT_FINITE)
        assert torch.equal(pool.cpu(), ref.pool()), fill
        o = damp.cache_attend(layout, pool, k, pages, i32([T, 20 + T]))
        assert torch.isfinite(o).all() or fill == 3e38


def test_bad_pages_and_tokens():
    """Bad pages are neither written nor read; the rest of the call is done."""
    layout = damp.CacheLayout(2, 1, 64)
    pool, _ = filled(layout, 1, 6, 5, extra=0)
    ref = R.Cache(pool, 64)
    pages = i32([[0, 99, 2], [-1, 3, -7], [4, 5, 1]])
    g = gen(2)
    k, v = randn(g, 3, 50, 1, 64), randn(g, 3, 50, 1, 64)
    start = [10, 20, 90]  # the last one runs out of its table
    damp.cache_append(layout, pool, k, v, pages, i32(start))
    assert damp.device_status() == damp.DEV_BAD_SLOT
    ref.append(k, v, pages.cpu(), start)
    assert torch.equal(pool.cpu(), ref.pool())
    damp.cache_append(layout, pool, k, v, pages, i32([-1, -50, -2**31]))
    assert damp.device_status() == damp.DEV_BAD_SLOT
    assert torch.equal(pool.cpu(), ref.pool())
    n = i32([60, 70, 2**31 - 1])
    kr, _ = damp.cache_read(layout, pool, pages, n, 96, dtype=F32)
    assert damp.device_status() == damp.DEV_BAD_SLOT
    assert not kr[0, 32:].any() and not kr[1, :32].any() and not kr[1, 64:].any() and kr[2, 95].any()
    q = randn(g, 3, 4, 2, 64)
    o = damp.cache_attend(layout, pool, q, pages, n)
    assert damp.device_status() == damp.DEV_BAD_SLOT
    want, bounds = R.attend(ref, q, pages, n)
    R.check_attend(o, want, bounds, 96, 64, "bad pages")
    assert not damp.cache_attend(layout, pool, q, i32([[-1] * 3] * 3), n).any()
    assert damp.device_status() == damp.DEV_BAD_SLOT


# ---- attention ----

def run_attend(layout, pool, pages, q, lengths, what, **more):
    """Against the reference, with the table as it is (a CTA per item where it is short) and with a long one, most of
    whose entries hold no token (the work cut into ranges)."""
    want, bounds = R.attend(R.Cache(pool, layout.d), q, pages.cpu(), lengths, **more)
    kw = {n: i32(x) if n == "q_lengths" and x is not None else x for n, x in more.items()}
    wide = torch.cat((pages, torch.full((pages.shape[0], 70), -1, dtype=torch.int32, device=DEV)), 1)
    for table in (pages, wide):
        o = damp.cache_attend(layout, pool, q, table, i32(lengths), **kw)
        R.check_attend(o, want, bounds, int(max(lengths)), layout.d, what)
    return o


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 1, 64), (8, 2, 128), (6, 2, 128), (16, 2, 256), (40, 1, 128), (3, 3, 256)])
def test_attend_single_tokens(dtype, H, Hk, d):
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, 7, 9, H + d)
    q = 1.5 * randn(gen(d), 7, 1, H, d)
    run_attend(layout, pool, pages, q.to(dtype), [1, 31, 32, 33, 0, 288, 200], "single tokens")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (9, 3, 128), (16, 2, 256)])
@pytest.mark.parametrize("T,W,window", [(2, 2, None), (5, 9, None), (5, 9, 40), (70, 3, None), (33, 6, 17), (150, 7, 1), (150, 7, 64),
                                        (260, 11, None)])
def test_attend_many_tokens(dtype, H, Hk, d, T, W, window):
    """Drafts and prompts, ragged: fewer queries than T, a context shorter than its queries, none at all."""
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, 4, W, T + d)
    q = 1.5 * randn(gen(T), 4, T, H, d)
    full = W * R.PAGE
    run_attend(layout, pool, pages, q.to(dtype), [T, full, 0, full - 3], "prompts", window=window)
    run_attend(layout, pool, pages, q.to(dtype), [full, T // 2, full - 1, min(full, 40)], "ragged", window=window,
               q_lengths=[T - 1, T, 0, 1])


@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (8, 1, 256)])
@pytest.mark.parametrize("window", [None, 100])
def test_attend_many_items(H, Hk, d, window):
    """More items than the GPU has ranges: whole ones, ones that end and begin in a range, rows of no query."""
    B, T, W = 40, 150, 9
    layout = damp.CacheLayout(H, Hk, d)
    pool, pages = filled(layout, B, W, d)
    g = gen(H)
    q = 1.5 * randn(g, B, T, H, d)
    n = torch.randint(0, W * R.PAGE + 1, (B,)).tolist()
    new = torch.randint(0, T + 1, (B,)).tolist()
    run_attend(layout, pool, pages, q.to(BF), n, "many items", window=window, q_lengths=new)
    run_attend(layout, pool, pages, q[:, :4].to(BF).contiguous(), n, "many drafts", window=window)


def test_attend_very_many_items():
    """So many items that ranges end with items though the table is long."""
    layout = damp.CacheLayout(16, 8, 64)
    B = 170
    pool, some = filled(layout, 10, 3, 4)
    pages = some[torch.arange(B, device=DEV) % 10].contiguous()  # rows that share their pages
    g = gen(8)
    q = randn(g, B, 40, 16, 64, dtype=BF)
    n, new = torch.randint(0, 97, (B,)).tolist(), torch.randint(0, 41, (B,)).tolist()
    run_attend(layout, pool, pages, q, n, "very many items", q_lengths=new)


@pytest.mark.parametrize("H,T", [(65, 1), (65, 3), (67, 9), (200, 2), (3, 50)])
def test_attend_groups(H, T):
    """Groups of query heads that are no powers of two, one KV head."""
    layout = damp.CacheLayout(H, 1, 64)
    pool, pages = filled(layout, 3, 4, H)
    q = randn(gen(T), 3, T, H, 64)
    for dtype in (BF, F32):
        run_attend(layout, pool, pages, q.to(dtype), [128, 55, 9], f"group of {H}", window=70)


def test_attend_many_tokens_of_slices_and_bad_pages():
    """Prompts whose queries are slices of a projection; bad pages in the middle, at the end and everywhere."""
    layout = damp.CacheLayout(4, 2, 128)
    pool, pages = filled(layout, 4, 6, 9)
    x = randn(gen(1), 4, 100, 8, 128, dtype=BF)
    pages[0, 2], pages[1, 5], pages[2] = -1, 1 << 20, -5
    q = x[:, :, 1:5]
    n = [190, 170, 192, 100]
    o = damp.cache_attend(layout, pool, q, pages, i32(n))
    assert damp.device_status() == damp.DEV_BAD_SLOT
    want, bounds = R.attend(R.Cache(pool, 128), q, pages.cpu(), n)
    R.check_attend(o, want, bounds, 192, 128, "slices and bad pages")
    assert not o[2].any()


def test_attend_clamps_lengths():
    layout = damp.CacheLayout(4, 2, 64)
    pool, pages = filled(layout, 3, 2, 8)
    q = randn(gen(1), 3, 3, 4, 64, dtype=BF)
    long = randn(gen(2), 3, 80, 4, 64, dtype=BF)
    a = damp.cache_attend(layout, pool, long, pages, i32([2**31 - 1, -5, 64]), q_lengths=i32([2**31 - 1, 3, -1]))
    b = damp.cache_attend(layout, pool, long, pages, i32([64, 0, 64]), q_lengths=i32([80, 3, 0]))
    assert torch.equal(a, b) and not b[0, :16].any() and b[0, 16:].any(dim=-1).all() and not b[1:].any()
    a = damp.cache_attend(layout, pool, q, pages, i32([2**31 - 1, -5, 64]), q_lengths=i32([2**31 - 1, 3, -1]))
    b = damp.cache_attend(layout, pool, q, pages, i32([64, 0, 64]), q_lengths=i32([3, 3, 0]))
    assert torch.equal(a, b) and not b[1:].any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attend_long_context(dtype):
    """A long axis over many ranges of the GPU, one row and two."""
    layout = damp.CacheLayout(8, 2, 128)
    for B, W, n in ((1, 1100, [35177]), (2, 500, [16000, 77])):
        pool, pages = filled(layout, B, W, B)
        q = 2.0 * randn(gen(9), B, 1, 8, 128)
        run_attend(layout, pool, pages, q.to(dtype), n, "long")
        run_attend(layout, pool, pages, q.to(dtype), n, "long", window=9000)


def test_attend_sums_of_long_rows_are_rounded():
    """FP32 sums over many pages in one place do not drift: the error's norm against 64 bits.

    Roundings are of random sign, so their squares add up.  In units of 2^-24 of the output: two additions a page,
    relative to a sum whose square is half of the last one's on average (1 page^-1); the sum of the weights, one a
    page, a third of the square (1/3 page^-1); ex2 and the two parts of a weight, 4 units each (2^-22); the scores,
    d / 16 + 4 additions and products of ln 2 times their size in powers of two, which is below 1 here.  Doubled."""
    B, T, Hk, d, W = 4, 640, 8, 64, 250  # more items than the GPU has ranges: whole rows in one of them
    layout = damp.CacheLayout(Hk, Hk, d)
    pool, pages = filled(layout, B, W, 3, spread=False)
    q = 0.25 * randn(gen(4), B, T, Hk, d)
    o = damp.cache_attend(layout, pool, q, pages, i32([W * R.PAGE] * B))
    cache, n = R.Cache(pool, d), W * R.PAGE
    unseen = torch.arange(n, device=DEV) > torch.arange(n - T, n, device=DEV)[:, None]
    err = size = 0.0
    for b in range(B):
        k, v = (cache.values(w, pages[b].cpu()).to(DEV) for w in (0, 1))
        for h in range(Hk):
            p = (q[b, :, h].double() @ k[:, h].T * d ** -0.5).masked_fill(unseen, -math.inf).softmax(-1)
            want = p @ v[:, h]
            err += (o[b, :, h].double() - want).square().sum().item()
            size += want.square().sum().item()
    limit = 2 * 2.0 ** -24 * math.sqrt(W * 4 / 3 + 4 ** 2 + 4 ** 2 + d / 16 + 4)
    assert math.sqrt(err / size) <= limit, f"error norm {math.sqrt(err / size):g}, limit {limit:g}"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1, 40])
def test_attend_scales(dtype, T):
    """Sharp and flat softmaxes, large and tiny values and queries."""
    layout = damp.CacheLayout(4, 2, 128)
    g = gen(5)
    for size, vsize, scale in ((30.0, 1.0, None), (1e-3, 1e-20, None), (1e4, 1e30, 1e-5), (1e-30, 1e-33, 1e29)):
        pool = damp.new_cache(layout, 10, DEV)
        pages = tables(g, 10, 2, 5)
        k, v = randn(g, 2, 160, 2, 128), vsize * randn(g, 2, 160, 2, 128)
        v[:, 32:64] *= 1e-4
        v[:, 96:128] = 0
        damp.cache_append(layout, pool, k, v, pages, i32([0, 0]))
        q = size * randn(g, 2, T, 4, 128)
        run_attend(layout, pool, pages, q.to(dtype), [160, 101], f"{size} {vsize}", scale=scale)


@pytest.mark.parametrize("T", [1, 6, 40])
def test_attend_not_finite(T):
    """A query that is not finite reaches its own output alone; stale scales and codes of pages that hold
    no token reach none."""
    layout = damp.CacheLayout(8, 2, 128)
    pool, pages = filled(layout, 2, 4, 3)
    q = randn(gen(4), 2, T, 8, 128, dtype=BF)
    n = i32([70, 90])
    good = damp.cache_attend(layout, pool, q, pages, n)
    bad = q.clone()
    bad[0, T - 1, 3, 7] = float("nan")
    bad[1, 0, 5, 0] = float("inf")
    dirty = pool.clone()
    dirty[pages[:, 3].long()] = 255  # codes of 127, scales that are NaN
    o = damp.cache_attend(layout, dirty, bad, pages, n)
    hit = torch.zeros(2, T, 8, dtype=torch.bool, device=DEV)
    hit[0, T - 1, 3] = hit[1, 0, 5] = True
    assert torch.equal(o[~hit], good[~hit])
    assert not torch.isfinite(o[hit]).any()


def test_attend_graphs_share_nothing():
    """Two captured calls replayed in turn and together, with inputs that change between replays."""
    layout = damp.CacheLayout(8, 2, 128)
    pool, pages = filled(layout, 3, 40, 6)
    q1, q2 = randn(gen(1), 3, 1, 8, 128, dtype=BF), randn(gen(2), 3, 50, 8, 128, dtype=BF)
    n1, n2 = i32([1280, 900, 3]), i32([1280, 60, 700])
    damp.cache_attend(layout, pool, q1, pages, n1)
    damp.cache_attend(layout, pool, q2, pages, n2)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        o1 = damp.cache_attend(layout, pool, q1, pages, n1)
    with torch.cuda.graph(g2):
        o2 = damp.cache_attend(layout, pool, q2, pages, n2)
    for step in range(3):
        n1.copy_(i32([1280 - 7 * step, 100 + step, 900]))
        q2.mul_(-0.5)
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            g1.replay()
        with torch.cuda.stream(torch.cuda.Stream()):
            g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, damp.cache_attend(layout, pool, q1, pages, n1))
        assert torch.equal(o2, damp.cache_attend(layout, pool, q2, pages, n2))


def test_attend_is_repeatable_and_leaves_its_inputs():
    layout = damp.CacheLayout(32, 8, 128)
    pool, pages = filled(layout, 5, 30, 7)
    q = randn(gen(1), 5, 4, 32, 128, dtype=BF)
    n = i32([960, 1, 500, 33, 64])
    keep = pool.clone(), q.clone(), pages.clone(), n.clone()
    a = damp.cache_attend(layout, pool, q, pages, n)
    for _ in range(3):
        assert torch.equal(a, damp.cache_attend(layout, pool, q, pages, n))
    for x, y in zip(keep, (pool, q, pages, n)):
        assert torch.equal(x, y)


def test_attend_large_batch():
    """As many rows as a call takes, most of them short."""
    layout = damp.CacheLayout(2, 1, 64)
    B = 4096
    pool, some = filled(layout, 8, 4, 2)
    pages = some[torch.arange(B, device=DEV) % 8].contiguous()  # rows that share their pages
    n = (torch.arange(B, device=DEV) * 37 % 128).to(torch.int32)
    q = randn(gen(3), B, 1, 2, 64)
    o = damp.cache_attend(layout, pool, q, pages, n)
    at = torch.tensor([0, 1, 777, 2048, 4094, 4095])
    want, bounds = R.attend(R.Cache(pool, 64), q[at], pages[at].cpu(), n[at].tolist())
    R.check_attend(o[at], want, bounds, 128, 64, "large batch")
    with pytest.raises(damp.DampError, match="SHAPE"):
        damp.cache_attend(layout, pool, torch.zeros(B + 1, 1, 2, 64, device=DEV), pages.repeat(2, 1)[:B + 1].contiguous(), i32(torch.zeros(B + 1)))


def test_attend_far_pages():
    """Records beyond 2^31 bytes of a pool."""
    layout = damp.CacheLayout(2, 1, 256)
    pages_total = (2**32 + 2**28) // layout.record_bytes
    pool = torch.zeros(pages_total, 1, layout.record_bytes, dtype=torch.uint8, device=DEV)
    pages = i32([[pages_total - 1, 131000, pages_total // 2 + 1]])
    g = gen(1)
    k, v = randn(g, 1, 90, 1, 256), randn(g, 1, 90, 1, 256)
    damp.cache_append(layout, pool, k, v, pages, i32([0]))
    small = pool[pages[0].long()].contiguous()
    assert small.any(dim=2).all()
    q = randn(g, 1, 3, 2, 256)
    a = damp.cache_attend(layout, pool, q, pages, i32([90]))
    assert torch.equal(a, damp.cache_attend(layout, small, q, i32([[0, 1, 2]]), i32([90])))
    assert torch.equal(damp.cache_read(layout, pool, pages, i32([90]), 90)[0], damp.cache_read(layout, small, i32([[0, 1, 2]]), i32([90]), 90)[0])


# ---- together ----

def test_layer_together():
    """A layer as a server runs it: a prompt in two pieces, single tokens, a draft of which a part is kept, a
    fork whose open page is copied; every step against attention over what the cache holds."""
    H, Hk, d, B, W = 8, 2, 128, 2, 8
    layout = damp.CacheLayout(H, Hk, d)
    freq, scale = damp.rotary_frequencies(64, scaling="linear", factor=2.0, device=DEV)
    pool = damp.new_cache(layout, 2 * B * W, DEV)
    pages = torch.arange(B * W, device=DEV, dtype=torch.int32).reshape(B, W)
    g = gen(11)
    held = torch.zeros(B, dtype=torch.int64)

    def step(T, pages, held, n=None):
        x = randn(g, B, T, H + 2 * Hk, d, dtype=BF)
        q, k = damp.rotary(x[:, :, :H], x[:, :, H:H + Hk], i32(held), freq, scale=scale)
        lengths = None if n is None else i32(n)
        damp.cache_append(layout, pool, k, x[:, :, H + Hk:], pages, i32(held), lengths=lengths)
        held = held + (T if n is None else torch.tensor(n))
        run_attend(layout, pool, pages, q, held.tolist(), f"step of {T}", q_lengths=n)
        return held

    held = step(45, pages, held, [45, 17])
    held = step(64, pages, held, [50, 64])
    for _ in range(3):
        held = step(1, pages, held)
    held = step(5, pages, held) - torch.tensor([2, 4])  # rejected drafts are written over
    held = step(1, pages, held)
    # row 0 is forked into row 1: full pages shared, the open one copied
    full = int(held[0]) // R.PAGE
    own = torch.arange(B * W, 2 * B * W, device=DEV, dtype=torch.int32)[:W]
    forked = torch.stack((pages[0], torch.cat((pages[0, :full], own[full:]))))
    damp.copy_slots([pool], forked[0, full:full + 1].contiguous(), forked[1, full:full + 1].contiguous())
    held = torch.stack((held[0], held[0]))
    before = pool[pages[0, :full].long()].clone()
    for _ in range(3):
        held = step(1, forked, held)
    assert torch.equal(before, pool[pages[0, :full].long()])
    assert not torch.equal(pool[forked[0, full].long()], pool[forked[1, full].long()])


def test_layer_captured():
    """The three calls of a decode step in one graph, replayed over growing lengths."""
    H, Hk, d, B = 4, 2, 64, 3
    layout = damp.CacheLayout(H, Hk, d)
    freq, _ = damp.rotary_frequencies(d, device=DEV)
    pool, pages = filled(layout, B, 4, 1)
    x = randn(gen(2), B, 1, H + 2 * Hk, d, dtype=BF)
    start = i32([30, 5, 63])
    twin = pool.clone()

    def calls(pool):
        q, k = damp.rotary(x[:, :, :H], x[:, :, H:H + Hk], start, freq)
        damp.cache_append(layout, pool, k, x[:, :, H + Hk:], pages, start)
        return damp.cache_attend(layout, pool, q, pages, start + 1)

    calls(pool.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = calls(pool)
    for t in range(5):
        x.copy_(randn(gen(20 + t), B, 1, H + 2 * Hk, d, dtype=BF))
        graph.replay()
        assert torch.equal(o, calls(twin))
        assert torch.equal(pool, twin)
        start += 1
