"""Streaming operators on the GPU against plain 64-bit formulas: rotary positions, appends, attention over the paged cache, page
copies, and all of them together as a generator uses them.

Tolerances.  A rounding is off by at most half a step: bf16 2^-8, fp32 2^-24 of the value.
  rope       an angle is 2 pi times a fraction of a turn rounded to fp32 (|fraction| <= 1/2: pi 2^-24 < 2^-22), sine and cosine and the
             amplitude's product add a few 2^-24, two products and a sum three more: 2^-21 (|x0| + |x1|) A holds all; then the output's rounding.
  attention  a logit is a sum of d products in fp32, however ordered: at most (d + 2) 2^-24 S off, S the largest sum of |q_c k_c| scale of
             the row; the exponential's argument (logit minus reference, both up to S log2 e) and the exponential add 4 S 2^-24 and 2^-22.
             The sum over n keys, the rescalings and the division add (n + 64) 2^-24.  All act on probabilities that average |v|, so
             |error| <= A (2 ((d + 8) 2^-24 S + 2^-22) + 2 (n + 64) 2^-24) with A = sum p |v|.  bf16 rounds every probability
             once, 2^-8 A, and the output, 2^-8 |o|; both a little enlarged (1.01) by each other."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2605_30325_amd import veda

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def dev():
    return torch.device("cuda:0")


def normal(shape, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(shape, generator=g)).to(dtype).to(dev())


# ---- rotary positions ---------------------------------------------------------------------------------------------------

def frequencies(dims, base=10000.0, scaling="plain", factor=1.0, trained=0.0, fast=32.0, slow=1.0):
    f, axis = [], []
    for a, w in enumerate(dims):
        for i in range(w // 2):
            x = (base * factor ** (w / (w - 2)) if scaling == "ntk" else base) ** (-2.0 * i / w)
            if scaling == "linear":
                x /= factor
            if scaling == "parts":
                g = min(1.0, max(0.0, (trained * x / (2 * math.pi) - slow) / (fast - slow)))
                x = x * g + x / factor * (1 - g)
            f.append(x)
            axis.append(a)
    return np.asarray(f), axis


def rotated(x, positions, dims, halves, transpose=False, amplitude=1.0, **scheme):
    """x [..., tokens, d] and positions [..., tokens, axes] in 64 bits on the CPU; and the bound of the fp32 rotation."""
    f, axis = frequencies(dims, **scheme)
    x, rot = x.double().cpu(), sum(dims)
    angle = positions.double().cpu()[..., axis] * torch.from_numpy(f)
    c, s = amplitude * torch.cos(angle), amplitude * torch.sin(angle) * (-1.0 if transpose else 1.0)
    i0 = torch.arange(rot // 2) if halves else 2 * torch.arange(rot // 2)
    i1 = i0 + rot // 2 if halves else i0 + 1
    y, bound = x.clone(), torch.zeros_like(x)
    x0, x1 = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = x0 * c - x1 * s, x0 * s + x1 * c
    bound[..., i0] = bound[..., i1] = 2.0 ** -21 * amplitude * (x0.abs() + x1.abs())
    return y, bound


def close(got, want, bound, dtype, what=""):
    step = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    over = (got.double().cpu() - want).abs() - (bound + 1.01 * step * want.abs())
    assert not torch.isnan(over).any() and over.max().item() <= 0.0, f"{what}: {over.max().item():.3e} over the bound"


SCHEMES = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0), dict(scaling="parts", factor=16.0, trained=4096.0)]
KIND = {"plain": veda.VEDA_ROPE_PLAIN, "linear": veda.VEDA_ROPE_LINEAR, "ntk": veda.VEDA_ROPE_NTK, "parts": veda.VEDA_ROPE_BY_PARTS}


def make_rope(d, dims, halves, base=10000.0, scaling="plain", factor=1.0, trained=0.0, **more):
    return veda.Rope(d, dims, base=base, pairs=veda.VEDA_ROPE_HALVES if halves else veda.VEDA_ROPE_INTERLEAVED, scaling=KIND[scaling], factor=factor,
                     trained_len=trained, **more)


@pytest.mark.parametrize("scheme", SCHEMES, ids=lambda s: s.get("scaling", "plain"))
def test_rope_frequencies(scheme):
    rope = make_rope(128, (64, 20, 4), False, **scheme)
    f, amp = rope.frequencies()
    want, _ = frequencies((64, 20, 4), **scheme)
    np.testing.assert_allclose(f, want, rtol=1e-14)
    assert amp == pytest.approx(0.1 * math.log(16.0) + 1.0 if scheme.get("scaling") == "parts" else 1.0, rel=1e-15)
    assert make_rope(64, 8, True, amplitude=1.5).frequencies()[1] == 1.5


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("halves", [False, True], ids=["interleaved", "halves"])
@pytest.mark.parametrize("d,dims", [(128, (128,)), (64, (64,)), (128, (44, 42, 42)), (128, (64,)), (128, (34,)), (64, (2,)), (64, (6, 4)), (8, (8,)),
                                    (40, (20, 10)), (512, (512,)), (504, (250,))])
def test_rope_against_the_formula(dtype, halves, d, dims):
    scheme = SCHEMES[(d + len(dims) + halves) % 4 if 2 not in dims else 0]
    rope = make_rope(d, dims, halves, **scheme)
    amp = rope.frequencies()[1]
    for b, h, n, first in ((1, 1, 1, 0), (2, 3, 17, 1 << 20), (1, 5, 40, -9), (3, 40, 2, 1 << 30)):
        x = normal((b, h, n, d), dtype, n)
        pos = (first + torch.arange(b * n * len(dims)) * 37 % 1013).reshape(b, n, len(dims)).to(torch.int32).to(dev())
        for transpose in (False, True):
            y = veda.veda_rope_apply(rope, x, pos, transpose=transpose)
            want, bound = rotated(x, pos[:, None], dims, halves, transpose, amp, **scheme)
            close(y, want, bound, dtype, f"{b}x{h}x{n} from {first}")


def test_rope_angles_are_not_rounded_to_fp32():
    """Pairs (1, 0) become (cos, sin).  A fraction of a turn that is rounded to fp32 turns them by 2 pi times what that loses, which the
    errors then follow: their slope on it is 1, and 0 where nothing is lost (the other roundings know nothing of it: 100,000 errors of
    about a half step each leave 0.01)."""
    rope = make_rope(128, (128,), False)
    f, _ = rope.frequencies()
    n = 1600
    pos = (torch.arange(n, dtype=torch.int32) * 7919 % 65536).view(1, n, 1)
    x = torch.zeros(1, 1, n, 128, device=dev())
    x[..., 0::2] = 1.0
    y = veda.veda_rope_apply(rope, x, pos.to(dev()))[0, 0].double().cpu().numpy()
    turns = pos.view(n, 1).numpy().astype(np.float64) * (f / 6.283185307179586476925286766559)
    part = turns - np.rint(turns)
    lost = 2 * math.pi * (part - part.astype(np.float32).astype(np.float64))
    c, s = np.cos(2 * math.pi * part), np.sin(2 * math.pi * part)
    err = np.stack([y[:, 0::2] - c, y[:, 1::2] - s])
    follows = np.stack([s * lost, -c * lost])
    assert abs((err * follows).sum() / (follows ** 2).sum()) < 0.25


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rope_strides_sharing_and_in_place(dtype):
    rope = make_rope(64, (32,), True)
    buf = normal((2, 19, 5, 3 * 64), dtype, 5)                       # [b, n, h, (q k v)]
    x = buf[..., 64:128].transpose(1, 2)
    pos = torch.arange(19, dtype=torch.int32, device=dev()) * 1000
    want, bound = rotated(x, pos[:, None], (32,), True)
    out = torch.full((2, 5, 19, 128), 7.0, dtype=dtype, device=dev())
    y = out[..., :64]
    assert veda.veda_rope_apply(rope, x, pos, y) is y
    close(y, want, bound, dtype)
    assert bool((out[..., 64:] == 7.0).all())
    before = buf.clone()
    veda.veda_rope_apply(rope, x, pos.view(1, -1, 1), x)             # in place, positions of all samples
    assert torch.equal(x, y)
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[..., 64:128] = False
    assert torch.equal(buf[keep], before[keep])
    for empty in (x[:0], x[:, :0], x[:, :, :0]):
        assert veda.veda_rope_apply(rope, empty, pos[:empty.shape[2]].view(1, -1, 1)).shape == empty.shape


def test_rope_gradient():
    # the map is linear: <R x, g> = <x, R^T g>, and differences along single channels give R^T g exactly up to rounding
    rope = make_rope(128, (64,), False, scaling="parts", factor=8.0, trained=2048.0)
    x, g = normal((2, 3, 33, 128), F32, 1), normal((2, 3, 33, 128), F32, 2)
    pos = (torch.arange(66, dtype=torch.int32, device=dev()) * 911).view(2, 33, 1)
    dx = veda.veda_rope_apply(rope, g, pos, transpose=True)
    y = veda.veda_rope_apply(rope, x, pos)
    # each product of the two sums carries 2^-21 of its size, the sums of 25,344 terms in 64 bits none
    size = (y.abs() * g.abs()).double().sum().item()
    assert abs((y.double() * g.double()).sum().item() - (x.double() * dx.double()).sum().item()) <= 2.0 ** -20 * 2 * size
    amp = rope.frequencies()[1]
    for c in (0, 1, 62, 63, 64, 127):
        step = torch.zeros_like(x)
        step[..., c] = 0.5
        hi, lo = (veda.veda_rope_apply(rope, x + s * step, pos).double() for s in (1, -1))
        slope = ((hi - lo) * g.double()).sum(-1)            # (R(x + h e) - R(x - h e)) . g / (2 h), 2 h = 1
        # the two results round up to 2^-21 A (|x| + 1) a channel, two channels are met, and x + h itself rounds
        bound = 2 * 2.0 ** -20 * amp * (x.abs().amax(-1) + 2.0).double() * g.abs().amax(-1).double() * 2
        assert bool(((slope - dx[..., c].double()).abs() <= bound).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("transpose", [False, True])
def test_rope_gradient_through_autograd(dtype, transpose):
    rope = make_rope(64, (24, 8), False, scaling="linear", factor=4.0)
    b, h, n = 2, 3, 17
    leaf = normal((b, n, h, 64), dtype, 1).requires_grad_()
    pos = (torch.arange(n * 2, dtype=torch.int32, device=dev()) * 131).view(1, n, 2)
    x = leaf.transpose(1, 2)
    y = veda.veda_rope_apply(rope, x, pos, transpose=transpose)
    with torch.no_grad():
        plain = veda.veda_rope_apply(rope, x, pos, transpose=transpose)
        assert not plain.requires_grad and torch.equal(plain, y) and y.requires_grad
    odd = torch.empty(b * h * n * 64 + 1, dtype=dtype, device=dev())[1:].view(b, h, n, 64).copy_(normal((b, h, n, 64), dtype, 4))
    grads = [normal((b, h, n, 64), dtype, 2), normal((b, n, h, 64), dtype, 3).transpose(1, 2), torch.ones((), dtype=dtype, device=dev()).expand(b, h, n, 64),
             normal((b, h, 64, n), dtype, 5).transpose(2, 3), odd]      # dense, other orders, no strides at all, an odd address
    for g in grads:
        (got,) = torch.autograd.grad(y, leaf, g, retain_graph=True)
        want = veda.veda_rope_apply(rope, g.clone(memory_format=torch.contiguous_format), pos, transpose=not transpose)
        assert torch.equal(got.transpose(1, 2), want)
        exact, bound = rotated(g, pos[:, None], (24, 8), False, not transpose, scaling="linear", factor=4.0)
        close(got.transpose(1, 2), exact, bound, dtype)
    # one head for all: its gradient is the sum over them
    one = normal((b, 1, n, 64), F32, 6).requires_grad_()
    g = normal((b, h, n, 64), F32, 7)
    (got,) = torch.autograd.grad(veda.veda_rope_apply(rope, one.expand(b, h, n, 64), pos, transpose=transpose), one, g)
    exact, bound = rotated(g, pos[:, None], (24, 8), False, not transpose, scaling="linear", factor=4.0)
    close(got, exact.sum(1, keepdim=True), bound.sum(1, keepdim=True) + 3 * 2.0 ** -24 * exact.abs().sum(1, keepdim=True), F32)
    # the gradient's own gradient is the rotation again
    v = normal((b, h, n, 64), dtype, 8).requires_grad_()
    (first,) = torch.autograd.grad(veda.veda_rope_apply(rope, x, pos, transpose=transpose), leaf, v, create_graph=True)
    (second,) = torch.autograd.grad(first, v, normal((b, n, h, 64), dtype, 9))
    assert torch.equal(second, veda.veda_rope_apply(rope, normal((b, n, h, 64), dtype, 9).transpose(1, 2), pos, transpose=transpose))


def test_rope_and_its_gradient_captured():
    # leaves of the graph's own: no eager graph of theirs lives while it is captured
    rope = make_rope(64, (64,), True)
    pos = torch.arange(33, dtype=torch.int32, device=dev())
    g = normal((2, 3, 33, 64), BF16, 1)

    def both(x, g):
        y = veda.veda_rope_apply(rope, x, pos)
        return y, torch.autograd.grad(y, x, g)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(normal((2, 3, 33, 64), BF16, 2).requires_grad_(), g)
    torch.cuda.synchronize()
    x = normal((2, 3, 33, 64), BF16, 3).requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = both(x, g)
    y = y.detach()
    for i in range(3):
        with torch.no_grad():
            x.copy_(normal(x.shape, BF16, 10 + i))
        g.copy_(normal(g.shape, BF16, 20 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, veda.veda_rope_apply(rope, x.detach(), pos)) and torch.equal(dx, veda.veda_rope_apply(rope, g, pos, transpose=True))


def test_rope_into_a_given_tensor_has_no_graph():
    rope = make_rope(64, (64,), True)
    x, pos = normal((1, 2, 5, 64), F32, 0).requires_grad_(), torch.arange(5, dtype=torch.int32, device=dev())
    y = torch.zeros((1, 2, 5, 64), device=dev())
    for args in ((x, y), (x, x), (y, x)):
        with pytest.raises(veda.VedaError, match="gradient"):
            veda.veda_rope_apply(rope, args[0], pos, args[1])
    with torch.no_grad():
        want = veda.veda_rope_apply(rope, x, pos)
        assert torch.equal(veda.veda_rope_apply(rope, x, pos, y), want) and not y.requires_grad
    assert torch.equal(veda.veda_rope_apply(rope, x.detach(), pos, y), want)


def test_rope_refuses_what_does_not_fit():
    rope = make_rope(64, (24, 20, 20), False)
    x, pos = normal((2, 3, 10, 64), F32, 0), torch.zeros((2, 10, 3), dtype=torch.int32, device=dev())
    wrong = [(x[0], pos), (x[..., :32], pos), (x.transpose(2, 3), pos), (x.cpu(), pos), (x, pos[:, :9]), (x, pos.long()), (x, pos[..., :1]), (x, pos.cpu()),
             (x, pos.transpose(0, 1).contiguous().transpose(0, 1)), (x, pos, x[:, :2]), (x, pos, x.bfloat16())]
    for args in wrong:
        with pytest.raises(veda.VedaError):
            veda.veda_rope_apply(rope, *args)
    with pytest.raises(veda.VedaError):      # rows of y on top of each other
        veda.veda_rope_apply(rope, x, pos, x[:, :1].expand(2, 3, 10, 64))
    with pytest.raises(TypeError):
        veda.veda_rope_apply(rope, x.double(), pos)


def test_rope_refuses_rows_that_share_bytes():
    rope = make_rope(64, (64,), True)
    x, pos = normal((2, 3, 4, 64), F32, 0), torch.arange(4, dtype=torch.int32, device=dev())
    room = torch.zeros(4096, device=dev())
    for strides in ((64, 64, 64), (768, 64, 64), (64, 256, 64), (128, 128, 256), (192, 256, 128), (512, 256, 96)):
        with pytest.raises(veda.VedaError):
            veda.veda_rope_apply(rope, x, pos, torch.as_strided(room, x.shape, (*strides, 1)))
    assert not bool(room.any())
    want = veda.veda_rope_apply(rope, x, pos)
    for strides in ((192, 64, 384), (64, 512, 128), (2048, 192, 320)):      # others than [b, h, n]; the last: one axis not within the other
        y = veda.veda_rope_apply(rope, x, pos, torch.as_strided(room, x.shape, (*strides, 1)))
        assert torch.equal(y, want)


# ---- the cache ----------------------------------------------------------------------------------------------------------

class Setup:
    """Sequences of `new` rows behind `past` cached tokens, pages in no order, rows of no sequence before (lead) and behind."""

    def __init__(self, new, past, hq, hk, d, dtype, page=16, holes=(), tail=3, seed=0, extra_width=0, spare=2, gain=1.0, pools=None):
        self.new, self.past, self.hq, self.hk, self.d, self.dtype, self.page = list(new), list(past), hq, hk, d, dtype, page
        self.len = [n + p for n, p in zip(new, past)]
        width = max(1, max(-(-x // page) for x in self.len)) + extra_width
        need = sum(-(-x // page) for x in self.len)
        total = need + spare
        ids = list(range(total))
        random.Random(seed).shuffle(ids)
        table = np.full((len(new), width), -1, np.int32)
        for s, n in enumerate(self.len):
            for i in range(-(-n // page)):
                table[s, i] = ids.pop()
        for s, i, mark in holes:
            table[s, i] = mark
        self.table = table
        if pools is None:
            pools = [normal((total, hk, page, d), dtype, 10 * seed + j + 1) for j in range(2)]
        self.k, self.v = pools
        self.cache = veda.Cache(self.k.shape[0], page, hk, d, dtype, k=self.k, v=self.v)
        self.start = np.cumsum([0] + self.new)
        self.batch = veda.CacheBatch(torch.from_numpy(table).to(dev()), torch.tensor(self.len, dtype=torch.int32, device=dev()),
                                     torch.tensor(self.start, dtype=torch.int32, device=dev()), max_new=max(self.new + [0]))
        self.rows = int(self.start[-1]) + tail
        self.qkv = normal((self.rows, hq + 2 * hk, d), dtype, 10 * seed + 7, gain)
        self.q = self.qkv[:, :hq]

    def keys(self, s):
        """(token numbers, K, V in 64 bits) of the keys that exist, on the CPU."""
        at = [(t, self.table[s, t // self.page], t % self.page) for t in range(self.len[s])]
        at = [x for x in at if 0 <= x[1] < self.k.shape[0]]
        p, o = torch.tensor([x[1] for x in at], dtype=torch.int64), torch.tensor([x[2] for x in at], dtype=torch.int64)
        k, v = (pool.cpu()[p, :, o].double() for pool in (self.k, self.v))
        return torch.tensor([x[0] for x in at], dtype=torch.int64), k, v


def attention(t, q, scale, block, window, sinks):
    """out, lse and the bounds of both, [rows, q_heads, d] and [q_heads, rows], in 64 bits on the CPU."""
    rows, hq, d = q.shape
    out, lse = torch.zeros(rows, hq, d, dtype=torch.float64), torch.zeros(hq, rows, dtype=torch.float64)
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    g = t.hq // t.hk
    for s, n in enumerate(t.new):
        if not n:
            continue
        tok, k, v = t.keys(s)
        r = slice(int(t.start[s]), int(t.start[s + 1]))
        p = t.len[s] - n + torch.arange(n)
        e = (torch.div(p, block, rounding_mode="floor") + 1) * block if block else torch.full_like(p, t.len[s])
        seen = (tok < e[:, None]) & (p >= 0)[:, None]
        if window:
            seen &= (tok >= e[:, None] - window) | (tok < sinks)
        for h in range(hq):
            qh, kh, vh = q[r, h].double().cpu(), k[:, h // g], v[:, h // g]
            x = (qh @ kh.T * scale).masked_fill(~seen, -math.inf)
            big = (qh.abs() @ kh.abs().T * scale).masked_fill(~seen, 0.0).amax(1) if len(tok) else torch.zeros(n, dtype=torch.float64)
            pr = torch.nan_to_num(torch.softmax(x, 1), nan=0.0) if len(tok) else torch.zeros(n, 0, dtype=torch.float64)
            vis = torch.where(seen.any(0)[:, None], vh, 0.0)          # what no row sees may be anything
            out[r, h] = pr @ vis
            lse[h, r] = torch.logsumexp(x, 1) if len(tok) else -math.inf
            count = seen.sum(1).double()
            delta = (d + 8) * 2.0 ** -24 * big + 2.0 ** -22
            mean = pr @ vis.abs()
            ob[r, h] = mean * (2 * delta + 2 * (count + 64) * 2.0 ** -24)[:, None] * 1.01
            if t.dtype == BF16:
                ob[r, h] += 1.01 * 2.0 ** -8 * mean
            lb[h, r] = delta + (count + 64) * 2.0 ** -24 + 2.0 ** -21 * lse[h, r].nan_to_num(neginf=0.0).abs()
    return out, lse, ob, lb


def check_attention(t, scale=None, block=1, window=0, sinks=0, q=None):
    q = t.q if q is None else q
    scale = 1.0 / math.sqrt(t.d) if scale is None else scale
    out = torch.full((t.rows, t.hq, t.d), 3.0, dtype=t.dtype, device=dev())
    lse = torch.full((t.hq, t.rows), 5.0, device=dev())
    veda.veda_cache_attn_fwd(t.cache, t.batch, q, scale, block, window, sinks, out, lse)
    want, want_lse, ob, lb = attention(t, q, scale, block, window, sinks)
    used = int(t.start[-1])
    assert bool((out[used:] == 3.0).all()) and bool((lse[:, used:] == 5.0).all())       # rows of no sequence
    close(out[:used], want[:used], ob[:used], t.dtype, "out")
    g, w = lse[:, :used].double().cpu(), want_lse[:, :used]
    assert torch.equal(g == -math.inf, w == -math.inf)
    assert bool(((g - w).nan_to_num(nan=0.0).abs() <= lb[:, :used]).all()), "lse"
    again, again_lse = veda.veda_cache_attn_fwd(t.cache, t.batch, q, scale, block, window, sinks, out.clone(), lse.clone())
    assert torch.equal(again, out) and torch.equal(again_lse, lse)                       # equal inputs, equal bytes
    return out, lse


TYPES = [(F32, 64), (F32, 128), (BF16, 64), (BF16, 128)]
IDS = ["f32-64", "f32-128", "bf16-64", "bf16-128"]


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("hq,hk", [(2, 2), (8, 2), (5, 1), (32, 1)])
def test_single_tokens(dtype, d, hq, hk):
    # every tile edge: lengths from the token alone on
    t = Setup([1] * 12, [0, 1, 14, 15, 16, 30, 31, 32, 63, 64, 127, 500], hq, hk, d, dtype, page=16, seed=hq)
    check_attention(t)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_ragged_chunks_and_pages(dtype, d, page):
    t = Setup([37, 0, 1, 130, 64, 0], [0, 5, 300, 71, 64, 0], 4, 2, d, dtype, page=page, seed=page, extra_width=2)
    check_attention(t)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("block,window,sinks", [(0, 0, 0), (1, 1, 0), (1, 7, 2), (1, 64, 4), (1, 100, 70), (16, 48, 0), (50, 0, 0), (50, 75, 33),
                                                (0, 90, 16), (1000, 0, 0), (1, 0, 9), (3, 1 << 30, 1 << 30), (1 << 30, 5, 1)])
def test_masks(dtype, d, block, window, sinks):
    t = Setup([150, 9, 1], [60, 200, 333], 3, 1, d, dtype, page=32, seed=3)
    check_attention(t, block=block, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_rows_that_see_nothing(dtype, d):
    # blocks whose end lies far behind the sequence's: the window ends before its first key; and holes instead of pages
    t = Setup([20, 3], [0, 40], 2, 1, d, dtype, holes=[(1, 0, -1), (1, 1, -1), (1, 2, 99999)], seed=4)
    out, lse = check_attention(t, block=1000, window=100)
    assert bool((out[:23] == 0).all()) and bool((lse[:, :23] == -math.inf).all())
    # more rows than tokens: rows at negative positions
    t = Setup([20, 3], [0, 40], 2, 1, d, dtype, seed=5)
    t.len, t.batch.kv_len = [12, 43], torch.tensor([12, 43], dtype=torch.int32, device=dev())
    out, lse = check_attention(t)
    assert bool((out[:8] == 0).all()) and bool((lse[:, :8] == -math.inf).all()) and bool((lse[:, 8:23] > -math.inf).all())
    check_attention(t, block=0)
    check_attention(t, block=7, window=9, sinks=1)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [1, 70])
def test_holes_anywhere(dtype, d, n):
    holes = [(0, 0, -1), (0, 3, -7), (0, 9, 1 << 30), (1, 1, -1), (1, 2, 2 ** 31 - 1)]
    check_attention(Setup([n, n], [300, 90], 4, 1, d, dtype, holes=holes, seed=6))
    check_attention(Setup([n, n], [300, 90], 4, 1, d, dtype, holes=holes, seed=6), window=40, sinks=50)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n", [1, 90])
def test_unseen_values_do_not_matter(dtype, d, bad, n):
    # infinities and NaN behind the ends, in holes' pages, outside the window and in later tokens of the chunk
    t = Setup([n, n], [200, 33], 4, 2, d, dtype, page=32, seed=8)
    clean = check_attention(t, window=50, sinks=3)[0].clone()
    seen = torch.zeros(t.k.shape[0], t.page, dtype=torch.bool)
    for s in range(2):
        for x in range(t.len[s]):
            if x >= t.past[s] + 1 - 50 or x < 3:
                seen[t.table[s, x // t.page], x % t.page] = True
    hide = (~seen).to(dev())[:, None, :, None]
    for pool in (t.k, t.v):
        pool.copy_(torch.where(hide, torch.full_like(pool, bad), pool))
    assert torch.equal(check_attention(t, window=50, sinks=3)[0], clean)
    # a bad value of the chunk's last token reaches the last row alone, and only its channel
    if n > 1:
        page, at = t.table[0, (t.len[0] - 1) // t.page], (t.len[0] - 1) % t.page
        t.v[page, :, at, 5] = bad
        out, _ = veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 1.0 / math.sqrt(d), window=50, sinks=3, out=clean.clone())
        assert torch.equal(out[:n - 1], clean[:n - 1]) and torch.equal(out[n:], clean[n:])
        row = out[n - 1].float()
        assert bool(torch.isnan(row[:, 5]).all()) if math.isnan(bad) else bool((row[:, 5] == bad).all())
        keep = [c for c in range(d) if c != 5]
        assert torch.equal(out[n - 1][:, keep], clean[n - 1][:, keep])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
def test_bad_queries_and_keys_that_are_seen(dtype, n):
    t = Setup([n, 2], [100, 9], 2, 1, 64, dtype, seed=9)
    clean = check_attention(t)[0].clone()
    t.q[0, 1, 3] = math.nan
    out, lse = veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.125, out=clean.clone(), want_lse=True)
    assert bool(torch.isnan(out[0, 1]).all()) and bool(torch.isnan(lse[1, 0]))
    out[0, 1], out[-3:] = clean[0, 1], clean[-3:]
    assert torch.equal(out, clean)


def plain_row(t, s, i, h, q, scale, block=1, window=0, sinks=0):
    """Row i of sequence s, query head h, by the formula in 64 bits with all that infinities do there: (out, lse)."""
    tok, k, v = t.keys(s)
    p = t.len[s] - t.new[s] + i
    e = (p // block + 1) * block if block else t.len[s]
    seen = (tok < e) & ((tok >= e - window) | (tok < sinks) if window else tok >= 0)
    g = h // (t.hq // t.hk)
    x = k[seen, g] @ q[int(t.start[s]) + i, h].double().cpu() * scale
    pr = torch.softmax(x, 0)
    return pr @ v[seen, g], torch.logsumexp(x, 0)


ALL = [(1, 60), (3, 60), (1, 6000), (70, 60), (70, 1500), (333, 10)]      # new rows and cached tokens: every kernel, and shared walks


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
def test_logits_that_are_all_minus_infinity(dtype, d, n, past):
    # the softmax over them is 0 / 0; a row that sees no key at all gives zeros
    t = Setup([n, 1, 0, 2], [past, 5, 0, 40], 2, 1, d, dtype, page=32, seed=35, holes=[(3, 0, -1), (3, 1, -1)])
    q = t.q.clone()
    q[:, 0, 0], q[:, 1, 0] = 1.0, -1.0
    clean, clean_lse = check_attention(t, q=q)
    for page in range(-(-(past + n) // 32)):
        t.k[t.table[0, page], :, :, 0] = -math.inf                 # every key of the first sequence: head 0 is repelled, head 1 attracted
    out, lse = clean.clone(), clean_lse.clone()
    veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125, out=out, lse=lse)
    assert bool(torch.isnan(out[:n, 0]).all()) and bool((lse[0, :n] == -math.inf).all())
    assert bool(torch.isnan(out[:n, 1]).all()) and bool(torch.isnan(lse[1, :n]).all())
    assert bool((out[n + 1:n + 3] == 0).all()) and bool((lse[:, n + 1:n + 3] == -math.inf).all())
    # nothing but the first token is seen: the rows of head 0 are its value
    first = t.table[0, 0]
    t.k[first, :, 0, 0] = 0.5
    q[:, 1] = q[:, 0]
    veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125, out=out, lse=lse)
    want, want_lse = plain_row(t, 0, n - 1, 0, q, 0.125)
    # one weight, divided by itself: a few roundings on its way through products, joining and division; its logit is a sum of d products
    bound = 2.0 ** -20 * want.abs()
    close(out[:n], want.expand(n, 2, d), bound.expand(n, 2, d), dtype)
    big = 0.125 * (q[n - 1, 0].abs().double() @ t.k[first, 0, 0].abs().double()).item()
    assert (lse[0, n - 1].double().cpu() - want_lse).abs() <= (d + 8) * 2.0 ** -24 * big + 2.0 ** -20
    # a window over the repelling ones alone, and one that leaves the first token
    veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125, window=50, out=out, lse=lse)
    assert bool(torch.isnan(out[n - 1]).all()) and bool((lse[:, n - 1] == -math.inf).all())
    veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125, window=50, sinks=1, out=out, lse=lse)
    close(out[n - 1], want.expand(2, d), bound.expand(2, d), dtype)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_bad_values_that_are_seen(dtype, d, n, past, bad):
    """At keys in tiles that every row sees and in tiles that some do not, with weights of ordinary size and with weights that are 0 in
    fp32: the rows that see one are never finite there, and as the formula says where the weight is more than 2^-100; all else keeps its bytes."""
    t = Setup([n, 2], [past, 9], 2, 1, d, dtype, page=32, seed=36)
    last = past + n - 1
    q = t.q.clone()
    q[:, :, 0] = 1.0
    for far in (0.0, -3000.0):               # the logit falls by a hundred or two: a weight of e^-375 at d = 64, and less
        for key in sorted({3, past - 2, past, last}):
            page, at = t.table[0, key // 32], key % 32
            kept = t.k[page, 0, at].clone()
            t.k[page, 0, at, 0] = far
            clean, clean_lse = check_attention(t, q=q)
            good = t.v[page, 0, at, 5].clone()
            t.v[page, 0, at, 5] = bad
            out, lse = veda.veda_cache_attn_fwd(t.cache, t.batch, q, 1.0 / math.sqrt(d), out=clean.clone(), lse=clean_lse.clone())
            first = max(0, key - past)                       # rows from here on see it
            assert torch.equal(out[:first], clean[:first]) and torch.equal(out[n:], clean[n:]) and torch.equal(lse, clean_lse)
            keep = [c for c in range(d) if c != 5]
            assert torch.equal(out[:, :, keep], clean[:, :, keep])
            hit = out[first:n, :, 5].float()
            assert not bool(torch.isfinite(hit).any()), (far, key)
            if far == 0.0 and math.isinf(bad):
                assert bool((hit == bad).all())
            if math.isnan(bad):
                assert bool(torch.isnan(hit).all())
            t.v[page, 0, at, 5], t.k[page, 0, at] = good, kept


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,past", ALL)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_bad_keys_that_are_seen(dtype, d, n, past, bad):
    """A logit of -inf is a weight of 0, one of +inf or NaN makes the row NaN.  Rows of the same sequence that do not see the key stay within
    their bounds, not at their bytes: all rows of a wave move their references where one has outgrown its own, and the quotient
    sum p v / sum p is the same for any reference only up to the roundings that the bounds count (exponential, sums, rescalings)."""
    t = Setup([n, 2], [past, 9], 2, 1, d, dtype, page=32, seed=37)
    last = past + n - 1
    q = t.q.clone()
    q[:, 0, 0], q[:, 1, 0] = 1.0, -1.0
    for key in sorted({3, past - 2, past, last}):
        page, at = t.table[0, key // 32], key % 32
        kept = t.k[page, 0, at].clone()
        clean, clean_lse = check_attention(t, q=q)
        formula, formula_lse, ob, lb = attention(t, q, 1.0 / math.sqrt(d), 1, 0, 0)
        t.k[page, 0, at, 0] = bad
        out, lse = veda.veda_cache_attn_fwd(t.cache, t.batch, q, 1.0 / math.sqrt(d), out=clean.clone(), lse=clean_lse.clone())
        first = max(0, key - past)
        assert torch.equal(out[n:], clean[n:]) and torch.equal(lse[:, n:], clean_lse[:, n:])        # the other sequence
        if first:
            close(out[:first], formula[:first], ob[:first], dtype)
            assert bool(((lse[:, :first].double().cpu() - formula_lse[:, :first]).abs() <= lb[:, :first]).all())
        for h in range(2):
            if math.isnan(bad) or (bad > 0) == (h == 0):
                assert bool(torch.isnan(out[first:n, h]).all()) and bool(torch.isnan(lse[h, first:n]).all())
                continue
            for i in {first, n - 1}:
                want, want_lse = plain_row(t, 0, i, h, q, 1.0 / math.sqrt(d))
                tok, k, v = t.keys(0)
                seen = (tok <= past + i) & (tok != key)
                if not bool(seen.any()):
                    continue
                k, v, qr = k[seen, 0], v[seen, 0], q[i, h].double().cpu()
                mean = torch.softmax(k @ qr / math.sqrt(d), 0) @ v.abs()
                big = (k.abs() @ qr.abs()).max().item() / math.sqrt(d)
                delta, count = (d + 8) * 2.0 ** -24 * big + 2.0 ** -22, int(seen.sum())
                bound = mean * (2 * delta + 2 * (count + 64) * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0.0)) * 1.01
                close(out[i, h], want, bound, dtype)
                assert abs(lse[h, i].item() - want_lse.item()) <= delta + (count + 64) * 2.0 ** -24 + 2.0 ** -21 * abs(want_lse.item())
        t.k[page, 0, at] = kept


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
def test_large_logits(dtype, d):
    # queries forty times as large: one key takes almost all; the reference moves often
    t = Setup([5, 140], [400, 100], 4, 2, d, dtype, page=64, seed=11, gain=40.0)
    check_attention(t)
    check_attention(t, scale=1e-6)
    check_attention(t, scale=3.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,past,hq,hk", [([1] * 3, [0, 37, 700], 4, 2), ([1] * 300, [90] * 300, 1, 1), ([1, 1], [6000, 20], 5, 1),
                                            ([3, 1], [500, 30], 8, 1), ([3, 2], [6000, 100], 16, 2)])
def test_weights_of_few_rows_are_not_rounded_to_bf16(d, new, past, hq, hk):
    """Up to 32 rows of a key head: a weight goes into its product in two bf16 parts.  The first lies below it by at most a step, 2^-7
    of it, and that is rounded by half a step: 2^-15 of the weight, where one part alone is off by 2^-8."""
    t = Setup(new, past, hq, hk, d, BF16, page=32, seed=38)
    out, _ = check_attention(t)
    want, _, ob, _ = attention(t, t.q, 1.0 / math.sqrt(d), 1, 0, 0)
    real, t.v = t.v, t.v.abs()                      # the mean of |v|, of which the bound counts 1.01 * 2^-8
    mean, _, _, _ = attention(t, t.q, 1.0 / math.sqrt(d), 1, 0, 0)
    t.v, used = real, int(t.start[-1])
    close(out[:used], want[:used], (ob - 1.01 * (2.0 ** -8 - 2.0 ** -15) * mean)[:used], BF16)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("n,hq,hk", [(1, 3, 1), (3, 8, 2), (40, 4, 1)])
def test_long_caches_are_split(dtype, d, n, hq, hk):
    # one long sequence beside short and empty ones: splits with and without work, joined
    t = Setup([n, 1, 0, n], [9000, 0, 70, 130], hq, hk, d, dtype, page=128, seed=12)
    assert veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, hq, t.rows) > 0
    check_attention(t)
    check_attention(t, window=5000, sinks=100)
    check_attention(t, block=0)


@pytest.mark.parametrize("dtype,heads,new", [(F32, 300, [40]), (F32, 130, [0, 40, 1]), (BF16, 800, [1, 0, 1]), (F32, 800, [1])])
def test_many_key_heads(dtype, heads, new):
    # 300: more than workgroups that share; single tokens: a workgroup for each
    t = Setup(new, [560] * len(new), heads, heads, 64, dtype, seed=29)
    assert (veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, heads, t.rows) > 0) == (max(new) > 32)
    check_attention(t)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("seqs,far", [(70, 0), (130, 100), (65, 64)])
def test_many_sequences_shared(dtype, d, seqs, far):
    # counted 64 at a time; one long sequence, at the beginning, in the middle or at the end
    past = [(37 * i) % 90 for i in range(seqs)]
    past[far] = 6000
    t = Setup([i % 3 for i in range(seqs)], past, 4, 2, d, dtype, seed=31)
    assert veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, 4, t.rows) > 0
    check_attention(t)
    check_attention(t, window=4500, sinks=10)


@pytest.mark.parametrize("new,past,shared", [
    ([300, 5, 0, 129, 260, 1, 77, 128], [900, 0, 40, 3000, 700, 2100, 1, 513], True), ([128] * 9, [640] * 9, True),
    ([40] * 30 + [600], [30] * 30 + [2000], True),
    ([40] * 63 + [600], [30] * 63 + [2000], False),      # 320 blocks, most of them empty: as they are
])
def test_uneven_blocks(new, past, shared):
    # whole multiples, rests of many blocks in one workgroup, blocks that see no more than themselves
    t = Setup(new, past, 2, 2, 64, F32, seed=30)
    assert (veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, 2, t.rows) > 0) == shared
    check_attention(t)
    check_attention(t, block=64, window=700, sinks=20)


@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,seqs", [(33, 1), (35, 3), (127, 1)])
def test_odd_numbers_of_rows_shared(dtype, d, rows, seqs):
    # odd numbers of rows, key heads and sequences: what is written behind the unfinished sums keeps its alignment
    t = Setup([rows] * seqs, [1500] * seqs, 1, 1, d, dtype, page=64, seed=32)
    assert veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, 1, t.rows) > 0
    check_attention(t)
    check_attention(t, window=900, sinks=5)


def test_pools_beyond_4_gib():
    # 16 KB a page and head: 150,000 pages of each pool are 4.9 GB, and the sequence lies at both ends
    pages, page, hk, d = 150000, 64, 2, 128
    pools = [torch.empty((pages, hk, page, d), dtype=BF16, device=dev()) for _ in range(2)]
    t = Setup([3, 70], [200, 500], 4, hk, d, BF16, page=page, seed=13)
    for pool, small in zip(pools, (t.k, t.v)):
        pool[-small.shape[0]:] = small
    moved = t.table + np.int32(pages - t.k.shape[0]) * (t.table >= 0)
    cache = veda.Cache(pages, page, hk, d, BF16, k=pools[0], v=pools[1])
    batch = veda.CacheBatch(torch.from_numpy(moved.astype(np.int32)).to(dev()), t.batch.kv_len, t.batch.q_start, 70)
    out, _ = veda.veda_cache_attn_fwd(cache, batch, t.q, 0.1)
    want, _ = veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.1)
    assert torch.equal(out[:73], want[:73])
    veda.veda_cache_append(cache, batch, t.qkv[:, 4:6], t.qkv[:, 6:])
    veda.veda_cache_append(t.cache, t.batch, t.qkv[:, 4:6], t.qkv[:, 6:])
    veda.veda_cache_copy_pages(cache, [(pages - 1, 0), (pages - 2, pages // 2)])
    assert torch.equal(pools[0][-t.k.shape[0]:], t.k) and torch.equal(pools[1][-t.k.shape[0]:], t.v)
    assert torch.equal(pools[0][0], t.k[-1]) and torch.equal(pools[1][pages // 2], t.v[-2])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_strided_tensors_and_pools(dtype):
    # K and V pages of one allocation, queries and outputs as slices of wider rows and as [heads, rows, d]
    t = Setup([33, 5], [50, 100], 4, 2, 64, dtype, seed=14)
    want, lse = check_attention(t)
    both = torch.zeros((t.k.shape[0], 2, 2, t.page, 64), dtype=dtype, device=dev())
    both[:, 0], both[:, 1] = t.k, t.v
    cache = veda.Cache(t.k.shape[0], t.page, 2, 64, dtype, k=both[:, 0], v=both[:, 1])
    q = t.q.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((t.rows, 4, 192), 3.0, dtype=dtype, device=dev())
    out, lse2 = veda.veda_cache_attn_fwd(cache, t.batch, q, 0.125, out=wide[..., 64:128], want_lse=True)
    assert torch.equal(out[:38], want[:38]) and torch.equal(lse2[:, :38], lse[:, :38]) and bool((wide[..., :64] == 3.0).all())
    spread = torch.full((2, 3), -1, dtype=torch.int32, device=dev())
    table = torch.cat([t.batch.page_table, spread], 1)[:, :t.batch.page_table.shape[1]]      # rows of a wider table
    out, _ = veda.veda_cache_attn_fwd(cache, veda.CacheBatch(table, t.batch.kv_len, t.batch.q_start, 33), q, 0.125)
    assert torch.equal(out[:38], want[:38])


def test_lists_out_of_range_stay_inside():
    t = Setup([4, 4], [30, 30], 2, 1, 64, F32, seed=15)
    out = torch.full((t.rows, 2, 64), 3.0, device=dev())
    # rows from 6 on are cut off by max_new, lengths are cut to the table's width, starts to the buffer
    odd = veda.CacheBatch(t.batch.page_table, torch.tensor([10 ** 9, -5], dtype=torch.int32, device=dev()),
                          torch.tensor([-3, 9, 2 ** 31 - 1], dtype=torch.int32, device=dev()), max_new=6)
    veda.veda_cache_attn_fwd(t.cache, odd, t.q, 0.1, out=out)
    veda.veda_cache_append(t.cache, odd, t.qkv[:, 2:3], t.qkv[:, 3:4])
    torch.cuda.synchronize()
    assert bool((out[6:9] == 3.0).all()) and bool((out[9:] == 0.0).all()) and not bool((out[:6] == 3.0).any())


# ---- appends ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", TYPES, ids=IDS)
@pytest.mark.parametrize("rope_dims,halves", [(None, False), ("all", True), ("all", False), ("axes", False), ("some", True), ("odd", True), ("odd", False)])
def test_append(dtype, d, rope_dims, halves):
    dims = {None: None, "all": (d,), "axes": (d // 2, d // 4, d // 4), "some": (d // 2,), "odd": (d // 4 + 2,)}[rope_dims]
    rope = None if dims is None else make_rope(d, dims, halves)
    t = Setup([19, 0, 1, 70, 40], [5, 9, 63, 128, 0], 6, 2, d, dtype, page=32, seed=21, holes=[(3, 5, -1)])
    t.batch.kv_len = torch.tensor([24, 9, 64, 198, 25], dtype=torch.int32, device=dev())     # the last: 15 rows at negative positions
    lens, used = [24, 9, 64, 198, 25], int(t.start[-1])
    k, v = t.qkv[:, 6:8], t.qkv[:, 8:]
    axes = 1 if dims is None else len(dims)
    where = torch.cat([lens[s] - n + torch.arange(n) for s, n in enumerate(t.new)] + [torch.zeros(3, dtype=torch.int64)])
    pos = torch.stack([where * (a + 1) + a for a in range(axes)], 1).to(torch.int32).to(dev()) if axes > 1 else None
    k0, v0 = t.k.clone(), t.v.clone()
    q_out = torch.full((t.rows, 6, d), 3.0, dtype=dtype, device=dev())
    veda.veda_cache_append(t.cache, t.batch, k, v, rope, pos, t.q, q_out)
    kw, vw, bound = k0.double().cpu(), v0.double().cpu(), torch.zeros(k0.shape, dtype=torch.float64)
    p = pos.cpu() if pos is not None else where[:, None]
    if rope is None:
        kr, kb = k.double().cpu(), torch.zeros(k.shape, dtype=torch.float64)
        qr, qb = t.q.double().cpu(), torch.zeros(t.q.shape, dtype=torch.float64)
    else:
        (kr, kb), (qr, qb) = (tuple(y.transpose(0, 1) for y in rotated(x.transpose(0, 1), p, dims, halves)) for x in (k, t.q))
    written = torch.zeros(k0.shape[0], t.page, dtype=torch.bool)
    for s, n in enumerate(t.new):
        for i in range(n):
            x, row = lens[s] - n + i, int(t.start[s]) + i
            page = t.table[s, x // t.page] if x >= 0 else -1
            if page < 0:
                continue
            kw[page, :, x % t.page], bound[page, :, x % t.page], vw[page, :, x % t.page] = kr[row], kb[row], v[row].double().cpu()
            written[page, x % t.page] = True
    assert torch.equal(t.v.double().cpu(), vw)
    close(t.k, kw, bound, dtype, "k")
    keep = (~written).to(dev())[:, None, :, None].expand_as(t.k)
    assert torch.equal(t.k[keep], k0[keep])
    close(q_out[:used], qr[:used], qb[:used], dtype, "q")
    assert bool((q_out[used:] == 3.0).all())
    if rope is None:
        assert torch.equal(q_out[:used], t.q[:used])
    # without q, and with q in place: the same bytes
    t.k.copy_(k0)
    veda.veda_cache_append(t.cache, t.batch, k, v, rope, pos)
    close(t.k, kw, bound, dtype, "k alone")
    veda.veda_cache_append(t.cache, t.batch, k, v, rope, pos, t.q, t.q)
    assert torch.equal(t.q[:used], q_out[:used])


def test_append_refuses_what_does_not_fit():
    t = Setup([4], [8], 4, 2, 64, F32, seed=22)
    k, v, rope = t.qkv[:, 4:6], t.qkv[:, 6:], make_rope(64, (24, 20, 20), False)
    pos = torch.zeros((t.rows, 3), dtype=torch.int32, device=dev())
    wrong = [dict(k=k[:, :1]), dict(v=v[:-1]), dict(k=k.bfloat16()), dict(q_out=t.q), dict(rope=rope), dict(positions=pos), dict(rope=rope, positions=pos[:-1]),
             dict(rope=rope, positions=pos.long()), dict(rope=make_rope(128, (128,), True)), dict(q=t.q, q_out=t.q[:, :2]), dict(k=k.cpu())]
    for more in wrong:
        args = dict(k=k, v=v)
        args.update(more)
        with pytest.raises(veda.VedaError):
            veda.veda_cache_append(t.cache, t.batch, **args)
    with pytest.raises(veda.VedaError):
        veda.veda_cache_attn_fwd(t.cache, t.batch, t.q[:, :3], 0.1)
    with pytest.raises(veda.VedaError):
        veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.1, lse=torch.zeros((t.rows, 4), device=dev()))


def test_axes_of_one_entry_have_no_stride():
    # one row, one head: strides of such axes can be anything, and are not looked at
    t = Setup([1], [40], 1, 1, 64, BF16, seed=23, tail=0)
    want, _ = check_attention(t)
    odd = lambda x, *strides: torch.as_strided(x.contiguous(), x.shape, strides)
    q, k, v = odd(t.q, 3, 5, 1), odd(t.qkv[:, 1:2], 1, 7, 1), odd(t.qkv[:, 2:], 9, 1, 1)
    out, _ = veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125, out=odd(torch.zeros(1, 1, 64, dtype=BF16, device=dev()), 11, 1, 1))
    assert torch.equal(out, want)
    veda.veda_cache_append(t.cache, t.batch, k, v, q=q, q_out=odd(torch.zeros(1, 1, 64, dtype=BF16, device=dev()), 3, 2, 1))
    assert torch.equal(t.k[t.table[0, 2], :, 8], k[0]) and torch.equal(t.v[t.table[0, 2], :, 8], v[0])
    x = torch.as_strided(normal((64,), BF16, 1), (1, 1, 1, 64), (3, 5, 7, 1))
    rope = make_rope(64, (64,), True)
    want, bound = rotated(x, torch.tensor([[[5]]]), (64,), True)
    close(veda.veda_rope_apply(rope, x, torch.tensor([5], dtype=torch.int32, device=dev())), want, bound, BF16)
    one = normal((1, 16, 64), F32, 3)
    cache = veda.Cache(1, 16, 1, 64, F32, k=torch.as_strided(one, (1, 1, 16, 64), (3, 5, 64, 1)), v=one[:, None])
    assert cache.pages == 1


def test_one_attention_call_of_a_step_refuses_positions_without_a_rope():
    t = Setup([4], [8], 4, 2, 64, F32, seed=24)
    with pytest.raises(veda.VedaError):
        veda.veda_cache_attention(t.cache, t.batch, t.q, t.qkv[:, 4:6], t.qkv[:, 6:], 0.125, positions=torch.zeros((t.rows, 1), dtype=torch.int32, device=dev()))


def test_buffers_serve_calls_of_one_size():
    t = Setup([4], [100], 4, 2, 64, BF16, seed=25, tail=0)
    q, k, v = t.q, t.qkv[:, 4:6], t.qkv[:, 6:]
    out, b = veda.veda_cache_attention(t.cache, t.batch, q, k, v, 0.125)
    first, held = out.clone(), dict(b)
    pools = t.k.clone(), t.v.clone()
    wide = veda.CacheBatch(torch.nn.functional.pad(t.batch.page_table, (0, 4096), value=-1), t.batch.kv_len, t.batch.q_start, 4)
    assert veda.veda_cache_attn_workspace_bytes(t.cache, wide, 4, 4) > b["ws"].numel()
    for batch, rows in ((wide, 4), (t.batch, 3)):
        with pytest.raises(veda.VedaError, match="other sizes"):
            veda.veda_cache_attention(t.cache, batch, q[:rows], k[:rows], v[:rows], 0.125, buffers=b)
    assert all(b[x] is held[x] for x in held) and torch.equal(t.k, pools[0]) and torch.equal(t.v, pools[1])
    again, _ = veda.veda_cache_attention(t.cache, t.batch, q, k, v, 0.125, buffers=b)
    assert again is out and torch.equal(again, first)


def test_a_refused_first_call_leaves_buffers_that_serve_the_next():
    t = Setup([4], [100], 4, 2, 64, BF16, seed=34, tail=0)
    q, k, v, b = t.q, t.qkv[:, 4:6], t.qkv[:, 6:], {}
    pools = t.k.clone(), t.v.clone()
    for bad in (dict(softmax_scale=-1.0), dict(softmax_scale=0.1, window=-1)):
        with pytest.raises(veda.VedaError):
            veda.veda_cache_attention(t.cache, t.batch, q, k, v, buffers=b, **bad)
    with pytest.raises(veda.VedaError):
        veda.veda_cache_attention(t.cache, t.batch, q[:, :3], k, v, 0.125, buffers=b)
    assert b == {} and torch.equal(t.k, pools[0]) and torch.equal(t.v, pools[1])
    out, _ = veda.veda_cache_attention(t.cache, t.batch, q, k, v, 0.125, buffers=b)
    want, _ = veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.125)
    assert torch.equal(out, want)


def test_attention_refuses_buffers_and_numbers_that_do_not_fit():
    t = Setup([4], [600], 4, 2, 64, F32, seed=26)
    need = veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, 4, t.rows)
    scratch = torch.empty(max(need, 16) * 2, dtype=torch.uint8)
    for more in (dict(workspace=scratch), dict(workspace=scratch.to(dev())[::2]), dict(window=(1 << 32) + 5), dict(block=1 << 32), dict(sinks=1 << 40, window=1), dict(out=t.q)):
        with pytest.raises(veda.VedaError):
            veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.1, **more)
    for pairs in (np.asarray([[1 << 32, 0]]), [[0.0, 1.0]], np.asarray([[0, -1]])):
        with pytest.raises(veda.VedaError):
            veda.veda_cache_copy_pages(t.cache, pairs)


def test_closed_ropes_are_refused():
    t = Setup([4], [8], 4, 2, 64, F32, seed=27)
    rope = make_rope(64, (64,), True)
    rope.close()
    with pytest.raises(veda.VedaError, match="closed"):      # not: no rope
        veda.veda_cache_append(t.cache, t.batch, t.qkv[:, 4:6], t.qkv[:, 6:], rope)
    with pytest.raises(veda.VedaError, match="closed"):
        veda.veda_rope_apply(rope, t.q[None], torch.zeros((1, 4, 1), dtype=torch.int32, device=dev()))


@pytest.mark.parametrize("lens", [[3] * 200, [0, 40, 0, 0, 1, 17] * 30, [300] + [0] * 130])
def test_append_to_many_sequences(lens):
    # even and uneven numbers of new rows: blocks of rows found by division and by counting
    t = Setup(lens, [5] * len(lens), 2, 1, 64, BF16, seed=28)
    k, v = normal((t.rows, 1, 64), BF16, 1), normal((t.rows, 1, 64), BF16, 2)
    want_k, want_v = t.k.clone(), t.v.clone()
    table, start = t.table.tolist(), t.start.tolist()
    for s, n in enumerate(lens):
        for i in range(n):
            page, at = table[s][(5 + i) // t.cache.page_tokens], (5 + i) % t.cache.page_tokens
            want_k[page, :, at], want_v[page, :, at] = k[start[s] + i], v[start[s] + i]
    veda.veda_cache_append(t.cache, t.batch, k, v)
    assert torch.equal(t.k, want_k) and torch.equal(t.v, want_v)


# ---- copies of pages ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,hk,page", [(BF16, 64, 1, 16), (F32, 128, 3, 64), (BF16, 128, 12, 256)])
def test_copies_in_order(dtype, d, hk, page):
    n = 40
    both = normal((n, 2, hk, page, d), dtype, 31)
    cache = veda.Cache(n, page, hk, d, dtype, k=both[:, 0], v=both[:, 1])
    for pairs in ([(3, 4)], [(1, 2), (2, 3), (3, 1), (1, 1)], [(0, 5), (0, 6), (7, 5), (5, 8)], [(i, (i + 1) % n) for i in range(n)],
                  [(9, 10)] * 3, [], [(random.Random(i).randrange(n), random.Random(i + 99).randrange(n)) for i in range(120)]):
        want = both.clone()
        for a, b in pairs:
            want[b] = want[a]
        veda.veda_cache_copy_pages(cache, np.asarray(pairs, np.int32).reshape(-1, 2))
        assert torch.equal(both, want)


def test_more_copies_than_a_launch_holds():
    k, v = normal((2000, 1, 16, 64), BF16, 32), normal((2000, 1, 16, 64), BF16, 33)
    cache, k0, v0 = veda.Cache(2000, 16, 1, 64, BF16, k=k, v=v), k.clone(), v.clone()
    order = np.random.default_rng(0).permutation(2000).astype(np.int32).reshape(-1, 2)
    veda.veda_cache_copy_pages(cache, order)
    src, dst = torch.from_numpy(order[:, 0].astype(np.int64)).to(dev()), torch.from_numpy(order[:, 1].astype(np.int64)).to(dev())
    k0[dst], v0[dst] = k0[src], v0[src]
    assert torch.equal(k, k0) and torch.equal(v, v0)


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 16), (BF16, 128, 64)], ids=["f32", "bf16"])
def test_a_streaming_run(dtype, d, page):
    """Two clips made chunk by chunk, one branched on the way, old frames dropped, pages moved together: every attention against
    the whole history of its clip in 64 bits."""
    hq, hk, frame, sinks, window = 4, 2, 30, 20, 150
    grid_h, grid_w, dims = 5, 6, (d // 2, d // 4, d // 4)
    rope, book = make_rope(d, dims, False), veda.Pages(60, page, 4, 40)
    cache = veda.Cache(60, page, hk, d, dtype)
    for pool in (cache.k, cache.v):
        pool.fill_(math.nan)
    history = {s: [torch.zeros(0, hk, d, dtype=torch.float64) for _ in range(2)] for s in range(4)}
    bufs, steps = {}, 0

    def positions(a, n):
        x = torch.arange(a, a + n)
        return torch.stack([x // frame, x // grid_w % grid_h, x % grid_w], 1).to(torch.int32)

    def step(seqs, news, seed):
        nonlocal steps
        starts = np.cumsum([0] + news)
        for s, n in zip(seqs, news):
            copies = book.extend(s, book.length(s) + n)
            veda.veda_cache_copy_pages(cache, copies)
        table = torch.from_numpy(book.table()[seqs]).to(dev())
        lens = [book.length(s) for s in seqs]
        batch = veda.CacheBatch(table, torch.tensor(lens, dtype=torch.int32, device=dev()), torch.tensor(starts, dtype=torch.int32, device=dev()), max(news))
        rows = int(starts[-1])
        qkv = normal((rows, hq + 2 * hk, d), dtype, seed)
        pos = torch.cat([positions(a - n, n) for a, n in zip(lens, news)]).to(dev())
        out, _ = veda.veda_cache_attention(cache, batch, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], 1.0 / math.sqrt(d), rope, pos,
                                           block=frame, window=window, sinks=sinks, buffers=bufs if rows == 2 * frame else None)
        for i, (s, n) in enumerate(zip(seqs, news)):
            r = slice(int(starts[i]), int(starts[i + 1]))
            step_cast = (lambda x: x.to(dtype).double())       # what the cache holds is rounded once
            kr, qr = (step_cast(rotated(x[r].transpose(0, 1), pos[r].cpu(), dims, False)[0].transpose(0, 1)) for x in (qkv[:, hq:hq + hk], qkv[:, :hq]))
            history[s] = [torch.cat([history[s][0], kr]), torch.cat([history[s][1], qkv[r, hq + hk:].double().cpu()])]
            k, v = history[s]
            tok, p = torch.arange(len(k)), lens[i] - n + torch.arange(n)
            e = (p // frame + 1) * frame
            seen = (tok < e[:, None]) & ((tok >= e[:, None] - window) | (tok < sinks))
            for h in range(hq):
                x = (qr[:, h] @ k[:, h // 2].T / math.sqrt(d)).masked_fill(~seen, -math.inf)
                pr = torch.softmax(x, 1)
                mean = pr @ v[:, h // 2].abs()
                big = (qr[:, h].abs() @ k[:, h // 2].abs().T / math.sqrt(d)).amax(1, keepdim=True)
                # q and k of the call and of the formula may round to different neighbours (their rotations differ by 2^-21): one step
                # of the largest logit's sum each, and the attention's own bound
                unit = 2.0 ** -7 if dtype == BF16 else 2.0 ** -20
                tol = mean * (2 * 2 * unit * big + 2.0 ** -16) + (1.01 * 2.0 ** -8 * (mean + (pr @ v[:, h // 2]).abs()) if dtype == BF16 else 0.0)
                err = (out[r, h].double().cpu() - pr @ v[:, h // 2]).abs()
                assert bool((err <= tol).all()), (steps, s, h, (err - tol).max().item())
        steps += 1

    seed = 100
    for _ in range(3):
        step([0, 1], [frame, frame], seed)
        seed += 1
    step([0], [7], seed)                       # a part of a frame
    book.fork(0, 2)                            # a branch that shares the open page
    history[2] = list(history[0])
    free = book.free_count()
    step([2, 0], [23, 23], seed + 1)           # both write the same tokens' places: one of them on a copy
    assert book.free_count() < free
    for s in (0, 1, 2):                        # frames that nobody will see again
        book.evict(s, sinks, max(sinks, book.length(s) + frame - window))
    step([1, 2], [frame, frame], seed + 2)
    book.truncate(0)                           # one clip ends; its pages are free
    history[0] = [x[:0] for x in history[0]]
    copies = book.compact()
    assert len(copies) > 0
    veda.veda_cache_copy_pages(cache, copies)
    used = book.pages - book.free_count()
    for pool in (cache.k, cache.v):
        pool[used:].fill_(math.nan)
    step([2, 1, 0], [frame, 1, 5], seed + 3)
    step([1], [1], seed + 4)
    step([1, 2], [frame, frame], seed + 5)
    for s in (0, 1, 2):
        book.truncate(s)
    assert book.free_count() == 60


def test_beside_the_tile_sparse_attention():
    """One clip whose chunk is the whole clip: rotated rows through the tile-sparse path with every tile kept, and through the cache."""
    from paper_2605_30325_amd import workloads as wlm
    grid, heads, d = (4, 9, 10), 3, 128
    n = 4 * 9 * 10
    shapes = np.asarray([(4, 4, 4), (1, 8, 8), (16, 2, 2)], np.int32)
    plan = veda.Plan(1, heads, d, grid, shapes, BF16)
    plan.set_option(veda.VEDA_OPT_EXACT_LOGIT_SCALE, 1)
    wl = wlm.custom_workload("streaming", heads, d, "bf16", grid, True, (1, 1), seed=5)
    q, k, v = wlm.make_qkv(wl, dev())
    rope = make_rope(d, (44, 42, 42), False)
    x = torch.arange(n, device=dev())
    pos = torch.stack([x // 90, x // 10 % 9, x % 10], 1).to(torch.int32)
    qr, kr = (veda.veda_rope_apply(rope, y, pos[None]) for y in (q, k))
    qt, vm, _ = veda.veda_tile_layout(plan, qr)
    kt, _, _ = veda.veda_tile_layout(plan, kr, want_mask=False)
    vt, _, _ = veda.veda_tile_layout(plan, v, veda.VEDA_CHANNEL_MAJOR, want_mask=False)
    rp = torch.tensor(np.cumsum([0] + [t for t in plan.tiles for _ in range(t)]), dtype=torch.int32, device=dev())
    ci = torch.cat([torch.arange(t, dtype=torch.int32) for t in plan.tiles for _ in range(t)]).to(dev())
    tiled, _ = veda.veda_sparse_attn_fwd(plan, qt, kt, vt, vm, rp, ci, 1.0 / math.sqrt(d))
    book, cache = veda.Pages(6, 64, 1, 6), veda.Cache(6, 64, heads, d, BF16)
    assert len(book.extend(0, n)) == 0
    batch = veda.CacheBatch(torch.from_numpy(book.table()).to(dev()), torch.tensor([n], dtype=torch.int32, device=dev()),
                            torch.tensor([0, n], dtype=torch.int32, device=dev()), n)
    rows = [y[0].transpose(0, 1) for y in (q, k, v)]
    out, _ = veda.veda_cache_attention(cache, batch, *rows, 1.0 / math.sqrt(d), rope, pos, block=0)
    # both round every probability and the output once: 2^-8 of at most the largest |v| each, on either side
    assert (out.transpose(0, 1).float() - tiled[0].float()).abs().max().item() <= 4 * 2.0 ** -8 * v.abs().max().item()
    assert (out.transpose(0, 1).float() - tiled[0].float()).abs().mean().item() <= 2.0 ** -8 * v.float().abs().mean().item()


def test_captured_and_replayed():
    """Two graphs with their own workspaces over one cache, lengths and pages changed between the replays."""
    hq, hk, d, page, width = 8, 2, 128, 32, 200
    rope = make_rope(d, (d,), True)
    cache = veda.Cache(2 * width, page, hk, d, BF16, k=normal((2 * width, hk, page, d), BF16, 41), v=normal((2 * width, hk, page, d), BF16, 42))
    table = torch.arange(2 * width, dtype=torch.int32, device=dev()).view(2, width)
    lens = torch.tensor([page * width - 40, 77], dtype=torch.int32, device=dev())
    graphs = []
    for new in (1, 20):
        start = torch.tensor([0, new, 2 * new], dtype=torch.int32, device=dev())
        batch = veda.CacheBatch(table, lens, start, new)
        qkv = normal((2 * new, hq + 2 * hk, d), BF16, new)
        ws = torch.empty(veda.veda_cache_attn_workspace_bytes(cache, batch, hq, 2 * new), dtype=torch.uint8, device=dev())
        out, q_out = (torch.zeros((2 * new, hq, d), dtype=BF16, device=dev()) for _ in range(2))

        def call(batch=batch, qkv=qkv, ws=ws, out=out, q_out=q_out):
            veda.veda_cache_append(cache, batch, qkv[:, hq:hq + hk], qkv[:, hq + hk:], rope, None, qkv[:, :hq], q_out)
            veda.veda_cache_attn_fwd(cache, batch, q_out, 0.09, window=3000, sinks=5, out=out, workspace=ws)

        call()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            call()
        graphs.append((g, call, qkv, out))
    for i in range(4):
        lens.copy_(torch.tensor([page * width - 39 + i, 77 + 40 * i], dtype=torch.int32))
        table.copy_(torch.randperm(2 * width, generator=torch.Generator().manual_seed(i)).to(torch.int32).view(2, width))
        for g, call, qkv, out in graphs:
            qkv.copy_(normal(qkv.shape, BF16, 50 + i))
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            got, k, v = out.clone(), cache.k.clone(), cache.v.clone()
            out.zero_()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out) and torch.equal(k, cache.k) and torch.equal(v, cache.v) and bool(got.float().abs().sum() > 0)


def test_two_streams_at_once():
    calls = []
    for seed in (1, 2):
        t = Setup([1, 2], [5000, 900], 8, 2, 128, BF16, page=64, seed=seed)
        want, _ = veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.09)
        calls.append((t, want[:3].clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for t, _, s in calls:
            with torch.cuda.stream(s):
                got.append(veda.veda_cache_attn_fwd(t.cache, t.batch, t.q, 0.09)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o[:3], calls[i % 2][1])


@pytest.mark.parametrize("dtype,d,seqs,new,past", [
    (BF16, 128, 2, 1, 200), (BF16, 64, 300, 1, 90), (F32, 128, 2, 3, 300), (F32, 64, 40, 1, 300), (F32, 128, 2, 40, 100), (F32, 128, 2, 100, 1500),
    (F32, 64, 1, 3, 6000), (BF16, 64, 2, 33, 1200), (BF16, 128, 3, 90, 90)])
def test_every_form_of_the_attention_captured(dtype, d, seqs, new, past):
    # short and shared walks of few and of many rows; those that ask for more LDS than a launch has without asking among them
    t = Setup([new] * seqs, [past] * seqs, 4, 2, d, dtype, page=32, seed=39)
    ws = torch.empty(veda.veda_cache_attn_workspace_bytes(t.cache, t.batch, 4, t.rows), dtype=torch.uint8, device=dev())
    q, out, lse = t.q.clone(), torch.zeros((t.rows, 4, d), dtype=dtype, device=dev()), torch.zeros((4, t.rows), device=dev())

    def call():
        veda.veda_cache_attn_fwd(t.cache, t.batch, q, 0.1, window=past - 7, sinks=9, out=out, lse=lse, workspace=ws)

    call()
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        call()
    for i in range(3):
        q.copy_(normal(q.shape, dtype, 60 + i))
        t.batch.kv_len.copy_(torch.tensor([past + new - 5 * i] * seqs, dtype=torch.int32))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        out.zero_()
        lse.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_lse, lse) and bool(torch.isfinite(got).all()) and bool(got.float().abs().sum() > 0)
