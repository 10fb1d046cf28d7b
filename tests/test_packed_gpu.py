"""The cache held in 4 bits and the page book on the GPU, against plain formulas: rounding and appending, attention over what the cache
stands for, copies of its pages, steps of the book, and all of them together as a generator uses them.

Tolerances.  Codes, scale bytes, values that the cache stands for and all numbers of pages are exact: K is turned in 64 bits, where the
reference here and the kernel differ by a few 2^-53 of a product, so only values that lie nearer to a border than 2^-40 could go either way, and
none of the seeds has one (it is asserted).  q_out is the rotation of veda_cache_append, byte for byte.  The attention's bounds are those of
the tests of the unpacked cache: its values are exact bf16 numbers, products and sums are in fp32.  One thing more: many of these values are 0, so
a result can consist of weights alone that are far below the row's largest.  Exponentials below 2^-126 come out as 0, and so may their products
with a value; the largest exponential of a row is at least 1 (the reference is never above its maximum), so that is at most 2^-126 (1 + |v|) of
the result for each key: keys * 2^-126 (1 + max |v|)."""
import heapq
import math
import random

import numpy as np
import pytest
import torch

from paper_2605_30325_amd import veda
from tests.test_streaming_gpu import BF16, F32, IDS, TYPES, Setup, attention, close, dev, frequencies, make_rope, normal

pytestmark = pytest.mark.gpu
GRID = np.asarray([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---- rounding -----------------------------------------------------------------------------------------------------------

def rounded(x):
    """Codes [..., d], scale bytes [..., d / 32] and values [..., d] of rows in 64 bits, by looking at all candidates; and how near the
    nearest border is, relative to the block's power."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    ok = np.isfinite(b).all(-1)
    top = np.where(ok, np.abs(np.where(np.isfinite(b), b, 0.0)).max(-1), 1.0)
    s = np.full(top.shape, 252, np.int64)
    for e in range(251, 1, -1):
        s[top < 7.0 * 2.0 ** (e - 127)] = e
    a = np.abs(np.where(ok[..., None], b, 0.0)) / 2.0 ** (s[..., None] - 127.0)
    order = [0, 2, 4, 6, 1, 3, 5, 7]                               # of two that are equally near, the even one
    code = np.asarray(order)[np.abs(a[..., None] - GRID[order]).argmin(-1)]
    border = (GRID[1:] + GRID[:-1]) / 2
    gap = np.abs(a[..., None] - border).min(-1)
    sign = np.signbit(b) & ok[..., None]
    value = np.where(ok[..., None], np.where(sign, -1.0, 1.0) * GRID[code] * 2.0 ** (s[..., None] - 127.0), np.nan)
    code = np.where(ok[..., None], code + 8 * sign, 0)
    return code.reshape(x.shape), np.where(ok, s, 255), value.reshape(x.shape), gap.reshape(x.shape)


def unpacked(cache, pool):
    """Codes [pages, heads, tokens, d] and scale bytes of a pool, on the host."""
    c = cache.codes(pool).cpu().numpy()
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1), cache.scales(pool).cpu().numpy()


def values(cache, pool):
    """What a pool stands for, float64 on the host."""
    code, s = unpacked(cache, pool)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    p = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127.0))
    return v * np.repeat(p, 32, -1)


def packed_pool(x, page):
    """Pool bytes [pages, heads, page * (d / 2 + d / 32)] of values [pages, heads, page, d]."""
    code, s, _, _ = rounded(x)
    c = (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)
    return np.concatenate([c.reshape(*c.shape[:2], -1), s.astype(np.uint8).reshape(*s.shape[:2], -1)], -1)


def turned(x, positions, dims, halves, amplitude=1.0, **scheme):
    """x [rows, heads, d] turned by positions [rows, axes], in 64 bits."""
    f, axis = frequencies(dims, **scheme)
    rot, x = sum(dims), np.asarray(x, np.float64)
    angle = positions[:, axis].astype(np.float64) * f
    c, s = amplitude * np.cos(angle)[:, None], amplitude * np.sin(angle)[:, None]
    i0 = np.arange(rot // 2) if halves else 2 * np.arange(rot // 2)
    i1 = i0 + rot // 2 if halves else i0 + 1
    y = x.copy()
    y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
    return y


def one_page(rows, d, dtype, heads=1, page=256):
    """A cache of one sequence and its batch of `rows` new rows."""
    pages = -(-rows // page)
    cache = veda.PackedCache(pages, page, heads, d, dtype)
    table = torch.arange(pages, dtype=torch.int32, device=dev()).view(1, -1)
    return cache, veda.CacheBatch(table, torch.tensor([rows], dtype=torch.int32, device=dev()), torch.tensor([0, rows], dtype=torch.int32, device=dev()), rows)


def check_rows(cache, pool, want, out=None):
    """The first rows of a cache of one sequence, in page order, against values [rows, heads, d] in 64 bits; returns the least gap to a border."""
    rows = want.shape[0]
    code, s, value, gap = rounded(want)
    got, got_s = unpacked(cache, pool)
    got, got_s = (x.swapaxes(1, 2).reshape(-1, *x.shape[1:2], x.shape[3])[:rows] for x in (got, got_s))
    np.testing.assert_array_equal(got_s, s)
    np.testing.assert_array_equal(got, code)
    if out is not None:
        np.testing.assert_array_equal(out.double().cpu().numpy(), value)
        np.testing.assert_array_equal(np.signbit(out.double().cpu().numpy())[~np.isnan(value)], np.signbit(value)[~np.isnan(value)])
    return gap


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_rounding(dtype, d):
    """Every border, its neighbours, and blocks of all magnitudes; K without a rope and V alike."""
    top = torch.finfo(dtype).max
    rows = []
    for e in list(range(-149, 128, 3)) + [-126, -125, -124, 124, 125, 126, 127]:
        g = torch.Generator().manual_seed(e + 1000)
        x = (torch.randn(d, generator=g, dtype=torch.float64) * 2.0 ** e).clamp(-top, top)
        rows.append(x)
        edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.96875, 7.0, 0.0, -0.0, 0.5, 4.0, 3.0, 5.0], dtype=torch.float64)
        for lead in (6.0, 6.96875, 7.0, 3.5, 0.2):
            y = torch.cat([edge, -edge])
            y[15] = lead
            y = torch.cat([y.clamp(-lead, lead)] * (d // 32)) * 2.0 ** e
            for nudge in (0.0, 2.0 ** -7, -2.0 ** -7, 2.0 ** -23, -2.0 ** -23):
                rows.append((y * (1 + nudge)).clamp(-top, top))
    rows += [torch.zeros(d, dtype=torch.float64), -torch.zeros(d, dtype=torch.float64), torch.full((d,), top, dtype=torch.float64)]
    x = torch.stack(rows).to(dtype)[:, None].to(dev())
    cache, batch = one_page(x.shape[0], d, dtype)
    k_out, v_out = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    veda.veda_packed_append(cache, batch, x, -x, k_out=k_out, v_out=v_out)
    want = x.double().cpu().numpy()
    check_rows(cache, cache.k, want, k_out)
    check_rows(cache, cache.v, -want, v_out)
    np.testing.assert_array_equal(values(cache, cache.k).swapaxes(1, 2).reshape(-1, 1, d)[:x.shape[0]], rounded(want)[2])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_blocks_that_are_not_finite(dtype, bad):
    x = normal((40, 2, 128), dtype, 3)
    for r in range(40):
        if r % 3:
            x[r, r % 2, (37 * r) % 128] = bad
    cache, batch = one_page(40, 128, dtype, heads=2, page=64)
    k_out, v_out = torch.empty_like(x), torch.empty_like(x)
    veda.veda_packed_append(cache, batch, x, x, k_out=k_out, v_out=v_out)
    want = x.double().cpu().numpy()
    check_rows(cache, cache.k, want, k_out)
    check_rows(cache, cache.v, want, v_out)
    assert int((cache.scales(cache.k) == 255).sum()) == 26


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("halves", [False, True], ids=["interleaved", "halves"])
@pytest.mark.parametrize("d,dims", [(128, (128,)), (64, (64,)), (128, (44, 42, 42)), (128, (64,)), (128, (34,)), (64, (2,)), (64, (6, 4)), (64, (24, 20, 20))])
def test_turned_keys_are_rounded_once(dtype, halves, d, dims):
    scheme = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="parts", factor=16.0, trained=4096.0)][(d + len(dims) + halves) % 3]
    rope = make_rope(d, dims, halves, **scheme)
    amp = rope.frequencies()[1]
    rows, heads = 70, 3
    k, v, q = (normal((rows, heads, d), dtype, 20 + i) for i in range(3))
    pos = (100003 + torch.arange(rows * len(dims)) * 977 % 40009).reshape(rows, -1).to(torch.int32)
    cache, batch = one_page(rows, d, dtype, heads=heads, page=32)
    k_out, v_out = torch.empty_like(k), torch.empty_like(v)
    q_out = veda.veda_packed_append(cache, batch, k, v, rope, pos.to(dev()), q, k_out=k_out, v_out=v_out)
    want = turned(k.double().cpu().numpy(), pos.numpy(), dims, halves, amp, **scheme)
    gap = rounded(want)[3]
    assert gap[..., :sum(dims)].min() > 2.0 ** -40 or dims == (2,)
    check_rows(cache, cache.k, want, k_out)
    check_rows(cache, cache.v, v.double().cpu().numpy(), v_out)
    plain = veda.Cache(cache.pages, 32, heads, d, dtype)
    assert torch.equal(q_out, veda.veda_cache_append(plain, batch, k, v, rope, pos.to(dev()), q))
    if len(dims) == 1:      # positions of their own
        q_own = veda.veda_packed_append(cache, batch, k, v, rope, None, q)
        check_rows(cache, cache.k, turned(k.double().cpu().numpy(), np.arange(rows)[:, None], dims, halves, amp, **scheme))
        assert torch.equal(q_own, veda.veda_cache_append(plain, batch, k, v, rope, None, q))


def test_a_turn_that_leaves_fp32():
    # sqrt 2 times the largest number: finite in 64 bits, so its code is the largest magnitude
    rope = make_rope(64, (64,), False)
    x = torch.full((4, 1, 64), torch.finfo(F32).max, device=dev())
    cache, batch = one_page(4, 64, F32, page=16)
    pos = torch.tensor([[0], [1], [2], [3]], dtype=torch.int32)
    veda.veda_packed_append(cache, batch, x, x, rope, pos.to(dev()))
    check_rows(cache, cache.k, turned(x.double().cpu().numpy(), pos.numpy(), (64,), False))


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_appends_go_where_the_table_says(dtype, d):
    """Ragged sequences, holes, rows at negative positions, rows of no sequence, more rows than max_new: the right bytes, and no others."""
    t = Setup([5, 0, 1, 40, 3], [0, 7, 300, 33, 60], 4, 2, d, dtype, page=32, holes=[(3, 1, -1), (4, 1, 10 ** 6)], seed=4)
    t.len[0], t.batch.kv_len[0] = 3, 3                    # two rows of the first sequence lie before its start
    t.batch.max_new = 39
    run = 32 * (d // 2 + d // 32)
    big = torch.randint(0, 256, (2, t.k.shape[0], 2 * 2 * run), dtype=torch.uint8, device=dev())
    k, v = (x[:, :2 * run].unflatten(1, (2, run)) for x in big)      # pages with room between them
    cache = veda.PackedCache(t.k.shape[0], 32, 2, d, dtype, k=k, v=v)
    before = big.clone()
    rows_k, rows_v = t.qkv[:, 4:6], t.qkv[:, 4:6].flip(2).contiguous()
    q_out, outs = torch.full((t.rows, 4, d), 3.0, dtype=dtype, device=dev()), torch.full((2, t.rows, 2, d), 4.0, dtype=dtype, device=dev())
    veda.veda_packed_append(cache, t.batch, rows_k, rows_v, q=t.q, q_out=q_out, k_out=outs[0], v_out=outs[1])
    want = before.clone()
    wk, wv = (x[:, :2 * run].unflatten(1, (2, run)) for x in want)
    written = torch.zeros(t.rows, dtype=torch.bool)
    for s, n in enumerate(t.new):
        for i in range(min(n, 39)):
            p, row = t.len[s] - n + i, int(t.start[s]) + i
            page = int(t.table[s, p // 32]) if p >= 0 else -1
            assert torch.equal(q_out[row], t.q[row])
            if not 0 <= page < t.k.shape[0]:
                continue
            written[row] = True
            for pool, src in ((wk, rows_k), (wv, rows_v)):
                code, sc, _, _ = rounded(src[row].double().cpu().numpy())
                cache.codes(pool)[page, :, p % 32] = torch.from_numpy((code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)).to(dev())
                cache.scales(pool)[page, :, p % 32] = torch.from_numpy(sc.astype(np.uint8)).to(dev())
    assert torch.equal(big, want)
    for out, src in zip(outs, (rows_k, rows_v)):
        assert bool((out[~written.to(dev())] == 4.0).all())
        np.testing.assert_array_equal(out[written.to(dev())].double().cpu().numpy(), rounded(src[written.to(dev())].double().cpu().numpy())[2])
    assert bool((q_out[int(t.start[-1]):] == 3.0).all())


def test_append_strides_and_places():
    d, rows = 64, 37
    rope = make_rope(d, (64,), True)
    buf = normal((5, rows, 2 * d), BF16, 1)                       # [heads][rows][..]: tokens of a head lie next to each other
    k, v = buf[:3, :, :d].transpose(0, 1), buf[:3, :, d:].transpose(0, 1)
    cache, batch = one_page(rows, d, BF16, heads=3, page=16)
    out = torch.zeros(rows, 6, 2 * d, dtype=BF16, device=dev())
    q = buf[3:, :, :d].transpose(0, 1)
    want_q = veda.veda_packed_append(cache, batch, k.contiguous(), v.contiguous(), rope, None, q.contiguous())
    want = cache.k.clone(), cache.v.clone()
    cache.k.zero_(), cache.v.zero_()
    got = veda.veda_packed_append(cache, batch, k, v, rope, None, q, q, k_out=out[:, ::2, :d], v_out=out[:, 1::2, d:])     # q in place
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want_q)
    assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])
    assert bool((out[:, ::2, d:] == 0).all()) and bool((out[:, 1::2, :d] == 0).all())
    np.testing.assert_array_equal(out[:, 1::2, d:].double().cpu().numpy(), rounded(v.double().cpu().numpy())[2])
    # alone, and without Q
    cache.k.zero_(), cache.v.zero_()
    assert veda.veda_packed_append(cache, batch, k, v, rope, k_out=out[:, ::2, :d].contiguous()) is None
    assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])


@pytest.mark.parametrize("heads", [(1, 1), (300, 1), (8, 200)])
def test_append_many_heads(heads):
    q_heads, kv = heads
    x = normal((9, q_heads + 2 * kv, 64), F32, 7)
    cache, batch = one_page(9, 64, F32, heads=kv, page=16)
    q = veda.veda_packed_append(cache, batch, x[:, q_heads:q_heads + kv], x[:, q_heads + kv:], q=x[:, :q_heads])
    assert torch.equal(q, x[:, :q_heads])
    check_rows(cache, cache.k, x[:, q_heads:q_heads + kv].double().cpu().numpy())
    check_rows(cache, cache.v, x[:, q_heads + kv:].double().cpu().numpy())


# ---- attention ----------------------------------------------------------------------------------------------------------

class Packed(Setup):
    """Setup over a packed cache: k and v are what its pools stand for; bytes that no token has stand for NaN."""

    def __init__(self, new, past, hq, hk, d, dtype, page=16, **more):
        super().__init__(new, past, hq, hk, d, dtype, page, **more)
        live = np.zeros((self.k.shape[0], page), bool)
        for s, n in enumerate(self.len):
            for i in range(-(-n // page)):
                if 0 <= self.table[s, i] < self.k.shape[0]:
                    live[self.table[s, i], :n - i * page] = True
        x = [np.where(live[:, None, :, None], pool.double().cpu().numpy(), np.nan) for pool in (self.k, self.v)]
        k, v = (torch.from_numpy(packed_pool(y, page)).to(dev()) for y in x)
        self.cache = veda.PackedCache(self.k.shape[0], page, hk, d, dtype, k=k, v=v)
        self.look()

    def look(self):
        self.k, self.v = (torch.from_numpy(values(self.cache, pool)) for pool in (self.cache.k, self.cache.v))


def check(t, scale=None, block=1, window=0, sinks=0, q=None, bounds=True):
    q = t.q if q is None else q
    scale = 1.0 / math.sqrt(t.d) if scale is None else scale
    out = torch.full((t.rows, t.hq, t.d), 3.0, dtype=t.dtype, device=dev())
    lse = torch.full((t.hq, t.rows), 5.0, device=dev())
    veda.veda_packed_attn_fwd(t.cache, t.batch, q, scale, block, window, sinks, out, lse)
    used = int(t.start[-1])
    assert bool((out[used:] == 3.0).all()) and bool((lse[:, used:] == 5.0).all())       # rows of no sequence
    if bounds:
        want, want_lse, ob, lb = attention(t, q, scale, block, window, sinks)
        tiny = max(t.len) * 2.0 ** -126 * (1.0 + float(np.nanmax(np.abs(t.v.numpy()))))
        close(out[:used], want[:used], ob[:used] + tiny, t.dtype, "out")
        g, w = lse[:, :used].double().cpu(), want_lse[:, :used]
        assert torch.equal(g == -math.inf, w == -math.inf)
        assert bool(((g - w).nan_to_num(nan=0.0).abs() <= lb[:, :used]).all()), "lse"
    again, again_lse = veda.veda_packed_attn_fwd(t.cache, t.batch, q, scale, block, window, sinks, out.clone(), lse.clone())
    assert torch.equal(again.view(torch.uint8), out.view(torch.uint8)) and torch.equal(again_lse.view(torch.int32), lse.view(torch.int32))   # equal bytes
    return out, lse


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("hq,hk", [(2, 2), (8, 2), (5, 1), (32, 1)])
def test_single_tokens(dtype, d, hq, hk):
    check(Packed([1] * 12, [0, 1, 14, 15, 16, 30, 31, 32, 63, 64, 127, 500], hq, hk, d, dtype, page=16, seed=hq))


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_ragged_chunks_and_pages(dtype, d, page):
    check(Packed([37, 0, 1, 130, 64, 0], [0, 5, 300, 71, 64, 0], 4, 2, d, dtype, page=page, seed=page, extra_width=2))


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("new,past", [([3, 1, 2], [500, 33, 8]), ([17, 5], [300, 90]), ([1, 1, 0, 1], [2999, 1, 8, 640])])
def test_few_rows(dtype, d, new, past):
    check(Packed(new, past, 3, 1, d, dtype, page=64, seed=2))
    check(Packed(new, past, 4, 2, d, dtype, page=16, seed=3), block=4, window=200, sinks=19)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("block,window,sinks", [(0, 0, 0), (1, 1, 0), (1, 7, 2), (1, 64, 4), (1, 100, 70), (16, 48, 0), (50, 0, 0), (50, 75, 33),
                                                (0, 90, 16), (1000, 0, 0), (1, 0, 9), (3, 1 << 30, 1 << 30), (1 << 30, 5, 1)])
def test_masks(dtype, d, block, window, sinks):
    check(Packed([150, 9, 1], [60, 200, 333], 3, 1, d, dtype, page=32, seed=3), block=block, window=window, sinks=sinks)
    check(Packed([5, 9, 1], [60, 200, 333], 3, 1, d, dtype, page=32, seed=4), block=block, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [20, 4])
def test_rows_that_see_nothing(dtype, d, n):
    t = Packed([n, 3], [0, 40], 2, 1, d, dtype, holes=[(1, 0, -1), (1, 1, -1), (1, 2, 99999)], seed=4)
    out, lse = check(t, block=1000, window=100)
    assert bool((out[:n + 3] == 0).all()) and bool((lse[:, :n + 3] == -math.inf).all())
    t = Packed([n, 3], [0, 40], 2, 1, d, dtype, seed=5)                # more rows than tokens: rows at negative positions
    t.len, t.batch.kv_len = [n - 2, 43], torch.tensor([n - 2, 43], dtype=torch.int32, device=dev())
    out, lse = check(t)
    assert bool((out[:2] == 0).all()) and bool((lse[:, :2] == -math.inf).all()) and bool((lse[:, 2:n + 3] > -math.inf).all())
    check(t, block=0)
    check(t, block=7, window=9, sinks=1)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [1, 70])
def test_holes_anywhere(dtype, d, n):
    holes = [(0, 0, -1), (0, 3, -7), (0, 9, 1 << 30), (1, 1, -1), (1, 2, 2 ** 31 - 1)]
    check(Packed([n, n], [300, 90], 4, 1, d, dtype, holes=holes, seed=6))
    check(Packed([n, n], [300, 90], 4, 1, d, dtype, holes=holes, seed=6), window=40, sinks=50)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("byte", [255, 254, 0])
@pytest.mark.parametrize("n", [1, 9, 90])
def test_unseen_values_do_not_matter(dtype, d, byte, n):
    # bytes that stand for NaN, infinities and numbers that are not normal: behind the ends, outside the window and in later tokens
    t = Packed([n, n], [200, 33], 4, 2, d, dtype, page=32, seed=8)
    clean = check(t, window=50, sinks=3)[0].clone()
    seen = torch.zeros(t.cache.pages, t.page, dtype=torch.bool)
    for s in range(2):
        for x in range(t.len[s]):
            if x >= t.past[s] + 1 - 50 or x < 3:
                seen[t.table[s, x // t.page], x % t.page] = True
    hide = (~seen).to(dev())[:, None, :, None]
    for pool in (t.cache.k, t.cache.v):
        t.cache.scales(pool).copy_(torch.where(hide, torch.full_like(t.cache.scales(pool), byte), t.cache.scales(pool)))
        t.cache.codes(pool).copy_(torch.where(hide, torch.full_like(t.cache.codes(pool), 0x77), t.cache.codes(pool)))
    assert torch.equal(check(t, window=50, sinks=3, bounds=False)[0], clean)
    # bad values of the chunk's last token reach the last row alone, and only the channels of their block
    if n > 1:
        page, at = t.table[0, (t.len[0] - 1) // t.page], (t.len[0] - 1) % t.page
        t.cache.scales(t.cache.v)[page, :, at, 1] = 255
        out, _ = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 1.0 / math.sqrt(d), window=50, sinks=3, out=clean.clone())
        assert torch.equal(out[:n - 1], clean[:n - 1]) and torch.equal(out[n:], clean[n:])
        assert bool(torch.isnan(out[n - 1, :, 32:64]).all())
        keep = [c for c in range(d) if not 32 <= c < 64]
        assert torch.equal(out[n - 1][:, keep], clean[n - 1][:, keep])


ALL = [(1, 60), (3, 60), (1, 6000), (3, 9000), (70, 60), (70, 1500), (333, 10)]      # new rows and cached tokens: every kernel, and shared walks


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_every_kernel(dtype, d, n, past):
    check(Packed([n, 2, 0, 1], [past, 5, 0, past // 3], 6, 2, d, dtype, page=32, seed=35))


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_bad_values_that_are_seen(dtype, d, n, past):
    """A block of V that stands for NaN, at keys in tiles that every row sees and in others, with weights of ordinary size and of 0: the rows that
    see it have NaN in its channels, all else keeps its bytes."""
    t = Packed([n, 2], [past, 9], 2, 1, d, dtype, page=32, seed=36)
    q = t.q.clone()
    q[:, :, 0] = 1.0
    for far in (False, True):
        for key in sorted({3, past - 2, past, past + n - 1}):
            page, at = t.table[0, key // 32], key % 32
            codes, scales = t.cache.codes(t.cache.k)[page, 0, at], t.cache.scales(t.cache.k)[page, 0, at]
            kept = codes.clone(), scales.clone()
            if far:                                      # K = (-3 * 2^10, 0 ..): a weight of e^-270 and less
                codes.zero_()
                scales.fill_(137)
                codes[0] = 13
            t.look()
            clean, clean_lse = check(t, q=q)
            vs = t.cache.scales(t.cache.v)[page, 0, at]
            good = vs.clone()
            vs[1] = 255
            out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, q, 1.0 / math.sqrt(d), out=clean.clone(), lse=clean_lse.clone())
            first = max(0, key - past)                   # rows from here on see it
            assert torch.equal(out[:first], clean[:first]) and torch.equal(out[n:], clean[n:]) and torch.equal(lse, clean_lse)
            keep = [c for c in range(d) if not 32 <= c < 64]
            assert torch.equal(out[:, :, keep], clean[:, :, keep])
            assert bool(torch.isnan(out[first:n, :, 32:64]).all()), (far, key)
            vs.copy_(good)
            codes.copy_(kept[0]), scales.copy_(kept[1])


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_bad_keys_that_are_seen(dtype, d, n, past):
    """A block of K that stands for NaN makes the rows that see its key NaN; other rows stay within their bounds, other sequences at their bytes."""
    t = Packed([n, 2], [past, 9], 2, 1, d, dtype, page=32, seed=37)
    clean, clean_lse = check(t)
    want, want_lse, ob, lb = attention(t, t.q, 1.0 / math.sqrt(d), 1, 0, 0)
    for key in sorted({3, past - 2, past, past + n - 1}):
        ks = t.cache.scales(t.cache.k)[t.table[0, key // 32], 0, key % 32]
        good = ks.clone()
        ks[0] = 255
        out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 1.0 / math.sqrt(d), out=clean.clone(), lse=clean_lse.clone())
        first = max(0, key - past)
        assert torch.equal(out[n:], clean[n:]) and torch.equal(lse[:, n:], clean_lse[:, n:])
        assert bool(torch.isnan(out[first:n]).all()) and bool(torch.isnan(lse[:, first:n]).all())
        if first:
            close(out[:first], want[:first], ob[:first], dtype)
            assert bool(((lse[:, :first].double().cpu() - want_lse[:, :first]).abs() <= lb[:, :first]).all())
        ks.copy_(good)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_bad_queries(dtype, d, n, past):
    t = Packed([n, 2], [past, 9], 2, 1, d, dtype, page=32, seed=38)
    clean, clean_lse = check(t)
    for bad in (math.nan, math.inf, -math.inf):
        q = t.q.clone()
        q[0, 1, 3] = bad                       # times codes of either sign, zeros among them
        out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, q, 1.0 / math.sqrt(d), out=clean.clone(), lse=clean_lse.clone())
        assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(lse[1, 0]))
        out[0, 1], lse[1, 0] = clean[0, 1], clean_lse[1, 0]
        assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_logits_that_are_all_minus_infinity(dtype, d, n, past):
    # the softmax over them is 0 / 0; a row that sees no key at all gives zeros
    t = Packed([n, 1, 0, 2], [past, 5, 0, 40], 2, 1, d, dtype, page=32, seed=39, holes=[(3, 0, -1), (3, 1, -1)])
    clean, clean_lse = check(t)
    q = t.q.clone()
    q[:n, 0, :] = 0.0
    q[:n, 0, 0] = -math.inf
    for page in range(-(-(past + n) // 32)):   # K = (1, 0, ..): every logit of head 0 is -inf in channel 0, and 0 elsewhere
        t.cache.codes(t.cache.k)[t.table[0, page], 0] = 0
        t.cache.scales(t.cache.k)[t.table[0, page], 0] = 127
        t.cache.codes(t.cache.k)[t.table[0, page], 0, :, 0] = 2
    out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, q, 0.125, out=clean.clone(), lse=clean_lse.clone())
    assert bool(torch.isnan(out[:n, 0]).all()) and bool((lse[0, :n] == -math.inf).all())
    assert not bool(torch.isnan(out[:n, 1]).any())
    assert bool((out[n + 1:n + 3] == 0).all()) and bool((lse[:, n + 1:n + 3] == -math.inf).all())


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("seqs,n", [(12, 1), (12, 4), (40, 1), (3, 1)])
def test_shared_walks_of_many_streams(dtype, d, seqs, n):
    """Caches cut into few and many parts, which 1, 8 or 16 waves a row join."""
    past = [(i * 577) % 1500 for i in range(seqs)]
    past[0] = 2900
    check(Packed([n if i % 7 != 5 else 0 for i in range(seqs)], past, 16, 8, d, dtype, page=64, seed=90, extra_width=80), window=0)


# Blocks of 17 to 32 rows to a key head: a workgroup for each, and shared walks whose parts 16, 8 or 1 waves a row join.
@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("block,window,sinks", [(1, 0, 0), (0, 0, 0), (16, 48, 0), (1, 100, 70), (3, 5000, 30)])
def test_shared_walks_of_blocks_of_32_rows(dtype, d, block, window, sinks):
    check(Packed([8, 3], [6000, 50], 8, 2, d, dtype, page=64, seed=91), block=block, window=window, sinks=sinks)
    check(Packed([5, 1, 0], [9000, 40, 0], 8, 2, d, dtype, page=64, seed=92, holes=[(0, 3, -1), (0, 90, 10 ** 6), (1, 0, -1)]), block=block, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("seqs,hk,extra", [(12, 4, 40), (40, 8, 80)])
def test_shared_walks_of_many_streams_of_32_rows(dtype, d, seqs, hk, extra):
    past = [(i * 277) % 400 for i in range(seqs)]
    past[0] = 2900
    check(Packed([(8, 5, 1, 0, 7)[i % 5] for i in range(seqs)], past, 4 * hk, hk, d, dtype, page=64, seed=93, extra_width=extra))


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", [(12, 60), (12, 6000)])
@pytest.mark.parametrize("way", [test_bad_values_that_are_seen, test_bad_keys_that_are_seen, test_bad_queries, test_logits_that_are_all_minus_infinity],
                         ids=lambda f: f.__name__[5:])
def test_bad_numbers_in_blocks_of_32_rows(way, dtype, d, n, past):
    way(dtype, d, n, past)


class Bytes(Packed):
    """Pools of any codes, with powers from 2^-5 to 2^0: caches of many heads, whose rows would take long to round on the host."""

    def __init__(self, new, past, hq, hk, d, dtype, page=16, **more):
        Setup.__init__(self, new, past, hq, hk, d, dtype, page, **more)
        g = torch.Generator().manual_seed(more.get("seed", 0))
        run = page * (d // 2 + d // 32)
        k, v = (torch.randint(0, 256, (self.k.shape[0], hk, run), generator=g, dtype=torch.uint8) for _ in range(2))
        live = torch.zeros(self.k.shape[0], page, dtype=torch.bool)
        for s, n in enumerate(self.len):
            for i in range(-(-n // page)):
                live[self.table[s, i], :n - i * page] = True
        for pool in (k, v):
            s = pool[:, :, page * (d // 2):].view(-1, hk, page, d // 32)
            s.copy_(torch.where(live[:, None, :, None], 122 + s % 6, torch.full_like(s, 255)))
        self.cache = veda.PackedCache(self.k.shape[0], page, hk, d, dtype, k=k.to(dev()), v=v.to(dev()))
        self.look()


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("seqs", [70, 130])
@pytest.mark.parametrize("n,group", [(1, 1), (8, 4)])
def test_short_caches_of_many_workgroups(dtype, d, seqs, n, group):
    """More than 256 workgroups, of four waves, and more than 768, of two; 1 and 32 rows to a key head."""
    past = [(i * 37) % 150 for i in range(seqs)]
    past[5], past[seqs - 1] = 640, 900
    new = [n if i % 3 == 0 else i % (n + 1) for i in range(seqs)]
    check(Bytes(new, past, 8 * group, 8, d, dtype, page=32, seed=94))
    check(Bytes(new, past, 8 * group, 8, d, dtype, page=16, seed=95), block=4, window=100, sinks=40)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_shared_walks_joined_by_single_waves(dtype, d):
    # 60 streams of 8 key heads, whose caches come in six parts and less each: a wave a row joins them at d = 64 too
    past = [(i * 77) % 300 for i in range(60)]
    past[7] = 2900
    check(Bytes([1 if i % 7 != 5 else 0 for i in range(60)], past, 16, 8, d, dtype, page=32, seed=97, extra_width=160))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_more_tiles_than_are_looked_up_at_once(dtype):
    # 130 tiles of 32 keys for two waves, which look up 64 each at a time: 4600 workgroups, or the walk would be shared out
    past = [i % 3 for i in range(46)]
    past[3] = 4149
    check(Bytes([1] * 46, past, 100, 100, 64, dtype, page=64, seed=96))


def tall(shared, seed=0):
    """bf16 rows that are cut into blocks of 256: shared out by walks that span workgroups, or many sequences under a wide table."""
    if shared:
        return Packed([64, 3], [6000, 50], 16, 4, 128, BF16, page=64, seed=seed)
    past = [(37 * i) % 211 for i in range(30)]
    past[2] = 900
    return Packed([64 if i % 13 == 2 else i % 3 for i in range(30)], past, 32, 8, 128, BF16, page=64, seed=seed, extra_width=160)


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("block,window,sinks", [(1, 0, 0), (0, 0, 0), (16, 0, 0), (1, 100, 70), (30, 64, 1)])
def test_blocks_of_256_rows(shared, block, window, sinks):
    check(tall(shared, 70), block=block, window=window, sinks=sinks)


def test_blocks_of_256_rows_in_several_rounds():
    # 70 sequences that may have 2048 rows of a key head each, under a table of 5120 keys
    new, past = [1] * 70, [(53 * i) % 97 for i in range(70)]
    new[5], new[31], new[69] = 64, 9, 33
    check(Packed(new, past, 32, 1, 128, BF16, page=64, seed=71, extra_width=80))


@pytest.mark.parametrize("key_heads", [1, 3, 5, 7, 12])
def test_a_window_asks_for_no_more_workspace(key_heads):
    # the binding gives what a call without a window asks for
    t = Packed([256, 1], [20000 // key_heads, 3], key_heads, key_heads, 128, BF16, page=256, seed=72)
    need = veda.veda_packed_attn_workspace_bytes(t.cache, t.batch, t.hq, t.rows)
    for window in (0, 300, 1000, 2500, 5000, 2 ** 30):
        out, _ = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1, 1, window, 0, workspace=torch.empty(need, dtype=torch.uint8, device=dev()))
        assert bool(torch.isfinite(out[:257]).all())


@pytest.mark.parametrize("key_heads", [1, 5, 12])
@pytest.mark.parametrize("window", [300, 2500, 2 ** 30])
def test_windows_in_the_workspace_of_a_call_without_one(key_heads, window):
    # the same calls, against the formula: with blocks of 128 or 256 rows, shared out or not, as the window leaves keys
    check(Packed([256, 1], [20000 // key_heads, 3], key_heads, key_heads, 128, BF16, page=256, seed=72), window=window)


@pytest.mark.parametrize("shared", [True, False])
def test_bad_values_in_blocks_of_256_rows(shared):
    t = tall(shared, 73)
    s = 0 if shared else 2
    r0, n, past = int(t.start[s]), t.new[s], t.past[s]
    clean, clean_lse = check(t)
    want, want_lse, ob, lb = attention(t, t.q, 1.0 / math.sqrt(128), 1, 0, 0)
    for key in (3, past - 2, past, past + 40, past + n - 1):
        page, at, first = t.table[s, key // 64], key % 64, r0 + max(0, key - past)
        others = torch.ones(t.rows, dtype=torch.bool)
        others[first:r0 + n] = False
        vs = t.cache.scales(t.cache.v)[page, :, at]
        good = vs.clone()
        vs[:, 2] = 255
        out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 1.0 / math.sqrt(128), out=clean.clone(), lse=clean_lse.clone())
        keep = [c for c in range(128) if not 64 <= c < 96]
        assert torch.equal(out[others], clean[others]) and torch.equal(out[:, :, keep], clean[:, :, keep]) and torch.equal(lse, clean_lse)
        assert bool(torch.isnan(out[first:r0 + n, :, 64:96]).all())
        vs.copy_(good)
        ks = t.cache.scales(t.cache.k)[page, :, at]
        good = ks.clone()
        ks[:, 1] = 254
        out, lse = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 1.0 / math.sqrt(128), out=clean.clone(), lse=clean_lse.clone())
        away = torch.ones(t.rows, dtype=torch.bool)
        away[r0:r0 + n] = False
        assert torch.equal(out[away], clean[away]) and bool(torch.isnan(out[first:r0 + n]).all()) and bool(torch.isnan(lse[:, first:r0 + n]).all())
        if first > r0:
            close(out[r0:first], want[r0:first], ob[r0:first], BF16)
        ks.copy_(good)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_large_logits(dtype, d):
    t = Packed([5, 140], [400, 100], 4, 2, d, dtype, page=64, seed=11, gain=40.0)
    check(t)
    check(t, scale=1e-6)
    check(t, scale=3.0)
    t = Packed([5, 1], [400, 9100], 4, 2, d, dtype, page=64, seed=12, gain=40.0)
    check(t)
    check(t, scale=3.0)


@pytest.mark.parametrize("n,past", ALL)
@pytest.mark.parametrize("size", [-40, 40])
def test_small_and_large_values(n, past, size):
    """fp32 rows 2^40 times as small or large against keys the other way round: no part of a number is lost on the way."""
    t = Packed([n, 2], [past, 9], 2, 1, 128, F32, page=32, seed=40)
    for pool in (t.cache.k, t.cache.v):
        s = t.cache.scales(pool)
        s.copy_(torch.where(s == 255, s, (s.int() - size).clamp(2, 252).to(torch.uint8)))
    t.look()
    check(t, q=t.q * 2.0 ** size)


@pytest.mark.parametrize("n,past", [(1, 60), (12, 60), (12, 6000), (70, 1500)])
def test_queries_that_end_below_normal_numbers(n, past):
    """fp32 rows around 2^-108 against keys around 2^108.  The least of three bf16 parts ends at 2^-133, so channels below 2^-110 are off by up to 2^-134: with
    |k| below 2^111 that is 128 * 2^-23 * 128^-1/2, under 2^-19, of a logit.  The bound's own term, (128 + 8) * 2^-24 * sum |q k| * 128^-1/2, is that much for sums
    of 2 and some 40 times as much for those of 128 such products, so it needs no more."""
    t = Packed([n, 2], [past, 9], 2, 1, 128, F32, page=32, seed=41)
    s = t.cache.scales(t.cache.k)
    s.copy_(torch.where(s == 255, s, (s.int() + 108).clamp(2, 252).to(torch.uint8)))
    t.look()
    assert float(np.nanmax(np.abs(t.k.numpy()))) < 2.0 ** 111
    check(t, q=t.q * 2.0 ** -108)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_offsets_beyond_32_bits(dtype, d):
    # the sequence's pages lie behind 4.5 GB of each pool, and between pages there is room
    page, hk = 64, 2
    run = page * (d // 2 + d // 32)
    stride = 1 << 20
    pages = 4500
    big = torch.empty(2, pages * stride, dtype=torch.uint8, device=dev())
    k, v = (torch.as_strided(x, (pages, hk, run), (stride, run, 1)) for x in big)
    cache = veda.PackedCache(pages, page, hk, d, dtype, k=k, v=v)
    for new, past in ((1, 700), (90, 300), (1, 9000)):
        t = Packed([new], [past], 4, hk, d, dtype, page=page, seed=13, spare=0)
        width = t.table.shape[1]
        ids = torch.arange(pages - width, pages)
        where = ids[torch.from_numpy(t.table[0]).long()].to(dev())
        cache.k[ids.to(dev())], cache.v[ids.to(dev())] = t.cache.k, t.cache.v
        want = veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1)[0]
        batch = veda.CacheBatch(where.int().view(1, -1), t.batch.kv_len, t.batch.q_start, new)
        assert torch.equal(veda.veda_packed_attn_fwd(cache, batch, t.q, 0.1)[0][:new], want[:new])
        x = normal((t.rows, 2 * hk, d), dtype, 5)
        veda.veda_packed_append(t.cache, t.batch, x[:, :hk], x[:, hk:])
        veda.veda_packed_append(cache, batch, x[:, :hk], x[:, hk:])
        assert torch.equal(cache.k[ids.to(dev())], t.cache.k) and torch.equal(cache.v[ids.to(dev())], t.cache.v)
    veda.veda_packed_copy_pages(cache, [(pages - 1, 0)])
    assert torch.equal(cache.k[0], cache.k[pages - 1]) and torch.equal(cache.v[0], cache.v[pages - 1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,past", ALL)
def test_strided_queries_and_results(dtype, n, past):
    t = Packed([n, 2], [past, 9], 4, 2, 64, dtype, page=32, seed=14)
    want, want_lse = check(t)
    q = torch.zeros(t.rows, 4, 3 * 64, dtype=dtype, device=dev()).transpose(0, 1).contiguous().transpose(0, 1)[..., 64:128]
    q.copy_(t.q)
    out = torch.full((4, t.rows, 128), 3.0, dtype=dtype, device=dev()).transpose(0, 1)[..., :64]
    got, _ = veda.veda_packed_attn_fwd(t.cache, t.batch, q, 0.125, out=out)
    assert torch.equal(got[:n + 2], want[:n + 2])
    assert bool((out.transpose(0, 1)[:, n + 2:] == 3.0).all())


@pytest.mark.parametrize("n,past", ALL)
def test_rows_beyond_max_new_and_odd_lists(n, past):
    # rows from max_new on stay as they were; starts and lengths that point outside are cut
    t = Packed([n, 2], [past, 9], 2, 1, 64, BF16, page=32, seed=15)
    want, _ = check(t)
    t.batch.max_new = 1
    out = torch.full_like(want, 3.0)
    veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.125, out=out)
    assert bool((out[1:n] == 3.0).all()) and bool((out[n + 1:] == 3.0).all())
    wild = veda.CacheBatch(t.batch.page_table, torch.tensor([10 ** 9, -5], dtype=torch.int32, device=dev()),
                           torch.tensor([-3, 10 ** 8, 4], dtype=torch.int32, device=dev()), n)
    veda.veda_packed_attn_fwd(t.cache, wild, t.q, 0.125, out=out)
    x = normal((t.rows, 2, 64), BF16, 1)
    veda.veda_packed_append(t.cache, wild, x[:, :1], x[:, 1:])
    torch.cuda.synchronize()


# ---- copies, streams, graphs --------------------------------------------------------------------------------------------

def test_copies_as_if_one_after_the_other():
    for seed, pages, n in ((1, 9, 40), (2, 700, 1500), (3, 700, 20)):
        cache = veda.PackedCache(pages, 16, 3, 64, BF16)
        for pool in (cache.k, cache.v):
            pool.copy_(torch.randint(0, 256, pool.shape, dtype=torch.uint8))
        rng = random.Random(seed)
        pairs = [(rng.randrange(pages), rng.randrange(pages)) for _ in range(n)]
        want = [x.clone() for x in (cache.k, cache.v)]
        for a, b in pairs:
            for x in want:
                x[b] = x[a]
        veda.veda_packed_copy_pages(cache, pairs)
        assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])
    for bad in ([(0, pages)], [(-1, 0)]):
        with pytest.raises(veda.VedaError):
            veda.veda_packed_copy_pages(cache, bad)
    veda.veda_packed_copy_pages(cache, [])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,past", ALL)
def test_captured_and_on_another_stream(dtype, n, past):
    """A captured append and attention follow the tables, lengths and rows that the buffers hold when they are replayed."""
    t = Packed([n, 2], [past, 40], 4, 2, 64, dtype, page=32, seed=16)
    x = normal((t.rows, 4, 64), dtype, 2)
    rope = make_rope(64, (64,), True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    buffers = {}
    q = t.q.clone()
    with torch.cuda.stream(side):
        veda.veda_cache_attention(t.cache, t.batch, q, x[:, :2], x[:, 2:], 0.125, rope, buffers=buffers)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = veda.veda_cache_attention(t.cache, t.batch, q, x[:, :2], x[:, 2:], 0.125, rope, buffers=buffers)
    for i in range(3):
        q.copy_(normal(q.shape, dtype, 30 + i))
        x.copy_(normal(x.shape, dtype, 40 + i))
        t.batch.kv_len.copy_(torch.tensor([past + n - 5 * i, 42 - i], dtype=torch.int32))
        pools = t.cache.k.clone(), t.cache.v.clone()
        graph.replay()
        torch.cuda.synchronize()
        got, after = out.clone(), (t.cache.k.clone(), t.cache.v.clone())
        t.cache.k.copy_(pools[0]), t.cache.v.copy_(pools[1])
        want, _ = veda.veda_cache_attention(t.cache, t.batch, q, x[:, :2], x[:, 2:], 0.125, rope)
        assert torch.equal(got[:n + 2], want[:n + 2]) and torch.equal(t.cache.k, after[0]) and torch.equal(t.cache.v, after[1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,past", [(12, 60), (12, 6000)])
@pytest.mark.parametrize("way", [test_strided_queries_and_results, test_captured_and_on_another_stream], ids=lambda f: f.__name__[5:])
def test_blocks_of_32_rows_strided_and_captured(way, dtype, n, past):
    way(dtype, n, past)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_captured_calls_that_share_a_workspace(dtype):
    """Calls of different shapes captured into graphs of their own, on one workspace: replayed in any order on one stream, each gives its own result."""
    cases = [Packed([n, 2], [past, 40], 8, 2, 128, dtype, page=64, seed=60 + i) for i, (n, past) in enumerate([(1, 6000), (3, 9000), (70, 1500)])]
    need = max(veda.veda_packed_attn_workspace_bytes(t.cache, t.batch, t.hq, t.rows) for t in cases)
    work = torch.empty(need, dtype=torch.uint8, device=dev())
    want = [veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1)[0] for t in cases]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in cases], [torch.zeros_like(x) for x in want]
    for t, g, out in zip(cases, graphs, outs):
        with torch.cuda.graph(g):
            veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1, out=out, workspace=work)
    for i in (0, 1, 0, 2, 1, 2, 0):
        outs[i].zero_()
        graphs[i].replay()
        work.fill_(255) if i == 1 else None        # what a call leaves in it is of no use to the next
        used = int(cases[i].start[-1])
        assert torch.equal(outs[i][:used], want[i][:used]), i


def test_one_call_of_a_step_is_its_parts():
    t = Packed([40, 3], [100, 9], 4, 2, 128, BF16, page=32, seed=17)
    x = normal((t.rows, 4, 128), BF16, 3)
    rope = make_rope(128, (128,), False)
    out, buffers = veda.veda_cache_attention(t.cache, t.batch, t.q, x[:, :2], x[:, 2:], 0.1, rope)
    k, v = t.cache.k.clone(), t.cache.v.clone()
    q = veda.veda_packed_append(t.cache, t.batch, x[:, :2], x[:, 2:], rope, None, t.q)
    want, _ = veda.veda_packed_attn_fwd(t.cache, t.batch, q, 0.1)
    assert torch.equal(out[:43], want[:43]) and torch.equal(k, t.cache.k) and torch.equal(v, t.cache.v) and set(buffers) == {"out", "ws", "q"}
    plain, _ = veda.veda_cache_attention(t.cache, t.batch, t.q, x[:, :2], x[:, 2:], 0.1)
    assert plain.shape == t.q.shape


def test_refusals_of_the_binding():
    t = Packed([2, 2], [30, 9], 4, 2, 64, BF16, page=32, seed=18)
    x = normal((t.rows, 4, 64), BF16, 3)
    k, v = x[:, :2], x[:, 2:]
    plain = veda.Cache(t.cache.pages, 32, 2, 64, BF16)
    out = torch.zeros_like(x)
    E = (veda.VedaError,)
    for call in (lambda: veda.veda_packed_append(plain, t.batch, k, v), lambda: veda.veda_packed_attn_fwd(plain, t.batch, t.q, 0.1),
                 lambda: veda.veda_packed_copy_pages(plain, [(0, 1)]), lambda: veda.veda_packed_append(t.cache, t.batch, k[:, :1], v),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k.float(), v), lambda: veda.veda_packed_append(t.cache, t.batch, k, v, k_out=out),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k, v, k_out=k), lambda: veda.veda_packed_append(t.cache, t.batch, k, v, v_out=v),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k, v, k_out=out[:, :2], v_out=out[:, :2]),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k, v, k_out=out[:, :1].expand(-1, 2, -1)),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k, v, k_out=out[:, :2].float()),
                 lambda: veda.veda_packed_append(t.cache, t.batch, k, v, q_out=t.q), lambda: veda.veda_packed_append(t.cache, t.batch, k.cpu(), v),
                 lambda: veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1, out=t.q), lambda: veda.veda_packed_attn_fwd(t.cache, t.batch, t.q[:, :3], 0.1),
                 lambda: veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, -0.1), lambda: veda.veda_packed_attn_fwd(t.cache, t.batch, t.q, 0.1, window=-1)):
        with pytest.raises(E):
            call()
    for call in (lambda: veda.veda_cache_append(t.cache, t.batch, k, v), lambda: veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.1)):
        with pytest.raises(Exception):
            call()
    assert not bool(out.any())


# ---- the page book on the GPU -------------------------------------------------------------------------------------------

class Model:
    """The book, one request after the other."""

    def __init__(self, pages, page, seqs, width):
        self.pages, self.page, self.width = pages, page, width
        self.table, self.length, self.free = [[] for _ in range(seqs)], [0] * seqs, list(range(pages))     # free: a heap

    def step(self, rows, max_new, asks):
        page, seen, plan, res = self.page, set(), [], []
        for s, keep, evict, grow in asks:
            ok = 0 <= s < len(self.length) and s not in seen
            if ok:
                seen.add(s)
                keep = min(keep, self.length[s])
                first, last = evict
                ok = keep >= 0 and 0 <= grow <= max_new and keep + grow <= self.width * page and 0 <= first <= last <= keep
                ok = ok and not (grow and keep % page and self.table[s][keep // page] < 0)
            plan.append(keep if ok else None)
            if not ok:
                continue
            have = -(-keep // page)
            for p in self.table[s][have:]:
                if p >= 0:
                    heapq.heappush(self.free, p)
            del self.table[s][have:]
            for x in range(-(-first // page), last // page):
                if self.table[s][x] >= 0:
                    heapq.heappush(self.free, self.table[s][x])
                self.table[s][x] = -1
            self.length[s] = keep
        closed, at = False, 0
        for (s, _, _, grow), keep in zip(asks, plan):
            if keep is None:
                res.append((1, 0, [], at, []))
                continue
            need = -(-(keep + grow) // page) - -(-keep // page)
            closed = closed or (grow > 0 and (need > len(self.free) or at + grow > rows))
            new = 0 if closed else grow
            if new:
                for _ in range(need):
                    self.table[s].append(heapq.heappop(self.free))
                self.length[s] += new
            tokens = [(p, self.table[s][p // page] * page + p % page) for p in range(keep, keep + new)]
            res.append((2 if closed and grow else 0, self.length[s], list(self.table[s]), at, tokens))
            at += new
        return res, at


def check_step(book, model, out, asks, max_new, dense=False):
    seq, keep, evict, grow = ([a[i] for a in asks] for i in range(4))
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())
    for x in (out.positions, out.row_seq, out.slots, out.page_table, out.kv_len, out.q_start, out.status):
        x.fill_(-77)
    veda.veda_pages_step(book, out, t(grow), None if dense else t(seq), t(keep), t(evict).view(-1, 2))
    want, total = model.step(out.rows, max_new, asks)
    status, kv_len, start, table = (x.tolist() for x in (out.status, out.kv_len, out.q_start, out.page_table))
    pos, row_seq, slots = out.positions.tolist(), out.row_seq.tolist(), out.slots.tolist()
    assert start[-1] == total
    h, w = out.frame
    for i, (st, n, pages, at, tokens) in enumerate(want):
        assert (status[i], kv_len[i], start[i]) == (st, n, at), (i, asks[i])
        assert table[i] == pages + [-1] * (book.max_pages - len(pages)), i
        for j, (p, slot) in enumerate(tokens):
            assert slots[at + j] == slot and row_seq[at + j] == i
            assert pos[at + j] == ([p] if out.axes == 1 else [p // (h * w), p // w % h, p % w])
    assert all(x == -77 for x in slots[total:]) and all(x == -77 for x in row_seq[total:]) and bool((out.positions[total:] == -77).all())
    bits = np.unpackbits(book.used.cpu().numpy().view(np.uint8), bitorder="little")
    assert np.array_equal(np.nonzero(bits[:book.pages] == 0)[0], sorted(model.free)) and not bits[book.pages:].any()
    assert book.length.tolist() == model.length
    held = book.table.tolist()
    for s, pages in enumerate(model.table):
        assert held[s][:len(pages)] == pages


SIZES = [(40, 16, 5, 8, 6, 30), (7, 1, 3, 20, 2, 9), (1000, 64, 90, 30, 70, 900), (33, 100, 2, 40, 4, 500), (5000, 16, 300, 64, 200, 700),
         (300000, 3, 2000, 200, 1500, 600), (12, 16, 4, 2 ** 14, 9, 64), (524288, 1, 8192, 40, 8192, 5)]


@pytest.mark.parametrize("pages,page,seqs,width,n,max_new", SIZES)
def test_steps_against_the_model(pages, page, seqs, width, n, max_new):
    rng = random.Random(pages)
    book, model = veda.DevicePages(pages, page, seqs, width), Model(pages, page, seqs, width)
    most = min(max_new * n, 200000)
    for step in range(3 if n > 1000 else 12):
        axes = rng.choice([1, 3])
        out = veda.StepTables(book, n, rng.choice([most, most, most // 2, 0]), max_new, axes=axes, frame=(rng.randint(1, 9), rng.randint(1, 50)))
        order = rng.sample(range(seqs), min(n, seqs))
        asks = []
        for i in range(n):
            s = order[i] if i < len(order) else -1
            if rng.random() < 0.1:
                s = rng.choice([-1, seqs, 2 ** 31 - 1, -2 ** 31] + order[:2])      # padding, and the same sequence again
            have = model.length[s] if 0 <= s < seqs else 0
            keep = rng.choice([have, have, 2 ** 31 - 1, rng.randint(0, have), 0, -1 if rng.random() < 0.2 else have])
            last = rng.randint(0, min(max(keep, 0), have)) if rng.random() < 0.5 else 0
            first = rng.randint(0, last)
            if rng.random() < 0.03:
                first, last = rng.choice([(-1, 0), (last + 1, last), (0, have + 1), (0, 2 ** 31 - 1)])
            grow = rng.choice([0, 1, max_new, rng.randint(0, max_new), max_new + 1 if rng.random() < 0.1 else 1, -1 if rng.random() < 0.1 else 1])
            asks.append((s, keep, (first, last), grow))
        check_step(book, model, out, asks, max_new)


def test_steps_without_lists():
    book, model = veda.DevicePages(50, 16, 6, 9), Model(50, 16, 6, 9)
    out = veda.StepTables(book, 4, 100, 40)
    for grow in ([40, 0, 5, 1], [1, 1, 1, 1], [0, 0, 0, 40], [16, 16, 16, 16]):
        veda.veda_pages_step(book, out, torch.tensor(grow, dtype=torch.int32, device=dev()))
        want, total = model.step(100, 40, [(i, 2 ** 31 - 1, (0, 0), g) for i, g in enumerate(grow)])
        assert out.q_start.tolist()[-1] == total and out.kv_len.tolist() == [w[1] for w in want] and book.length.tolist() == model.length
        assert out.slots.tolist()[:total] == [s for w in want for _, s in w[4]]
    none = veda.StepTables(book, 0, 0, 5)
    none.q_start.fill_(-77)
    veda.veda_pages_step(book, none, torch.zeros(0, dtype=torch.int32, device=dev()))
    assert none.q_start.tolist() == [0]
    # only what every call needs
    import ctypes as C
    few = veda.veda_step_tables(9, out.page_table.data_ptr(), out.kv_len.data_ptr(), out.q_start.data_ptr(), out.status.data_ptr(), None, None, None)
    one = torch.ones(4, dtype=torch.int32, device=dev())
    step = veda.veda_step(4, 100, 40, 3, 5, 5, None, None, None, one.data_ptr())
    before = out.slots.clone()
    assert veda.load().veda_pages_step(book._ref, C.byref(step), C.byref(few), None) == veda.VEDA_OK
    assert out.kv_len.tolist() == [n + 1 for n in model.length[:4]] and torch.equal(out.slots, before)


def test_long_sequences_go_back_whole():
    # more entries to give back than a workgroup has threads, from many sequences at once, again and again
    seqs, width = 40, 700
    book = veda.DevicePages(seqs * width, 16, seqs, width)
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=dev())
    out = veda.StepTables(book, seqs, seqs * width * 16, width * 16)
    for i in range(20):
        veda.veda_pages_step(book, out, t([width * 16] * seqs), None, t([0] * seqs))
        assert out.kv_len.tolist() == [width * 16] * seqs and not out.status.any()
        assert sorted(out.page_table.flatten().tolist()) == list(range(seqs * width))
        veda.veda_pages_step(book, out, t([0] * seqs), None, t([i] * seqs))
        bits = np.unpackbits(book.used.cpu().numpy().view(np.uint8))
        assert bits.sum() == seqs * -(-i // 16) and out.kv_len.tolist() == [i] * seqs


def test_books_with_wild_numbers_stay_inside():
    # lengths beyond the table, pages that are none: nothing outside the book is touched, and steps go on
    book = veda.DevicePages(64, 16, 4, 8)
    book.table.copy_(torch.tensor([2 ** 31 - 1, -5, 64, 3, -2 ** 31, 7, 100, 9], dtype=torch.int32).repeat(4, 1))
    book.length.copy_(torch.tensor([2 ** 31 - 1, -7, 129, 37], dtype=torch.int32))
    out = veda.StepTables(book, 4, 64, 16)
    t = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev())
    veda.veda_pages_step(book, out, t(0, 16, 1, 3), None, t(100, 5, 2 ** 31 - 1, 37), t(0, 90, 0, 0, 0, 0, 0, 0).view(4, 2))
    assert out.status.tolist() == [0, 0, 1, 1] and out.kv_len.tolist() == [100, 16, 0, 0]     # no 129 tokens in 8 pages of 16; an open page that is none
    assert book.length.tolist()[:2] == [100, 16]


def test_a_captured_loop_of_steps():
    """Step, append and attention over a 4-bit cache captured once and replayed for tokens after tokens, against the host's book and eager calls."""
    page, seqs, hk, hq, d = 16, 3, 2, 4, 64
    pages, width, n = 40, 8, 4
    book, host = veda.DevicePages(pages, page, seqs, width), veda.Pages(pages, page, seqs, width)
    cache, twin = (veda.PackedCache(pages, page, hk, d, BF16) for _ in range(2))
    rope = make_rope(d, (24, 20, 20), False)
    out = veda.StepTables(book, n, 64, 20, axes=3, frame=(3, 5))
    grow, seq, keep, evict = (torch.zeros(s, dtype=torch.int32, device=dev()) for s in ((n,), (n,), (n,), (n, 2)))
    qkv = normal((64, hq + 2 * hk, d), BF16, 1)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    buffers = {}

    def step():
        veda.veda_pages_step(book, out, grow, seq, keep, evict)
        return veda.veda_cache_attention(cache, out.batch, q, k, v, 0.125, rope, out.positions, block=15, window=45, sinks=15, buffers=buffers)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    rng = random.Random(5)
    for i in range(9):
        order = rng.sample(range(seqs), 3)
        g = [rng.randint(0, 15) for _ in order]
        kept = [host.length(s) - (rng.randint(0, min(4, host.length(s))) if i % 3 == 2 else 0) for s in order]
        gone = [(15, max(15, x - 45)) if x >= 15 else (0, 0) for x in kept]
        grow.copy_(torch.tensor(g + [0])), seq.copy_(torch.tensor(order + [-1])), keep.copy_(torch.tensor(kept + [0]))
        evict.copy_(torch.tensor(gone + [(0, 0)]))
        qkv.copy_(normal(qkv.shape, BF16, 50 + i))
        graph.replay()
        torch.cuda.synchronize()
        for s, x, (a, b) in zip(order, kept, gone):
            host.truncate(s, x)
            host.evict(s, a, b)
        for s, x, m in zip(order, kept, g):
            assert host.extend(s, x + m).size == 0
        assert out.status.tolist() == [0, 0, 0, 1] and out.q_start.tolist() == [0] + np.cumsum(g).tolist() + [sum(g)]
        table = host.table()
        assert [out.page_table[j, :-(-host.length(s) // page)].tolist() for j, s in enumerate(order)] == \
            [table[s, :-(-host.length(s) // page)].tolist() for s in order]
        total = sum(g)
        tok = [p for x, m in zip(kept, g) for p in range(x, x + m)]
        pos = torch.tensor([[p // 15, p // 5 % 3, p % 5] for p in tok] + [[0, 0, 0]] * (64 - total), dtype=torch.int32, device=dev()).view(64, 3)
        assert torch.equal(out.positions[:total], pos[:total])
        mine = veda.CacheBatch(torch.from_numpy(table[order]).to(dev()), torch.tensor([host.length(s) for s in order], dtype=torch.int32, device=dev()),
                               torch.tensor([0] + np.cumsum(g).tolist(), dtype=torch.int32, device=dev()), 20)
        want, _ = veda.veda_cache_attention(twin, mine, q, k, v, 0.125, rope, pos, block=15, window=45, sinks=15)
        assert torch.equal(got[:total], want[:total]) and torch.equal(cache.k, twin.k) and torch.equal(cache.v, twin.v)
        # the rows' slots are where the appends went
        for r in range(0, total, 7):
            slot = int(out.slots[r])
            at = cache.codes(cache.v)[slot // page, :, slot % page].cpu().numpy()
            code = rounded(v[r].double().cpu().numpy())[0]
            np.testing.assert_array_equal(at, (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8))
    host.close()
