"""The cache held in 4 bits and the page book on the GPU, the parts that need none: refusals at the C entry points and in the binding."""
import ctypes as C

import pytest
import torch

from paper_2605_30325_amd import veda
from tests.test_streaming_cpu import _batch, lib  # noqa: F401

INVALID, UNSUPPORTED, WORKSPACE, OK = veda.VEDA_ERR_INVALID_ARG, veda.VEDA_ERR_UNSUPPORTED, veda.VEDA_ERR_WORKSPACE, veda.VEDA_OK
AT = 1 << 20     # a 16-byte aligned address that no check reads from


def _cache(**more):
    f = dict(pages=8, page_tokens=64, kv_heads=2, head_dim=128, dtype=veda.VEDA_BF16, page_stride=0, k=AT, v=AT)
    f.update(more)
    return veda.veda_packed_cache(*f.values())


def _append(lib, cache, batch, **more):
    s = veda.veda_strides(0, 128, 256)
    f = dict(k=AT, sk=s, v=AT, sv=s, q_heads=4, q=AT, sq=veda.veda_strides(0, 128, 512), q_out=AT, so=veda.veda_strides(0, 128, 512), rope=None,
             positions=None, k_out=2 * AT, sko=s, v_out=3 * AT, svo=s)
    f.update(more)
    return lib.veda_packed_append(None if cache is None else C.byref(cache), None if batch is None else C.byref(batch), *f.values(), None)


def _attend(lib, cache, batch, **more):
    s = veda.veda_strides(0, 128, 512)
    f = dict(q_heads=4, q=AT, sq=s, scale=0.1, visible=veda.veda_visible(1, 0, 0), out=2 * AT, so=s, lse=None, workspace=AT, workspace_bytes=1 << 30)
    f.update(more)
    return lib.veda_packed_attn_fwd(None if cache is None else C.byref(cache), None if batch is None else C.byref(batch), *f.values(), None)


RUN = 2 * 64 * (64 + 4)      # bytes of a page
BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pages=0), INVALID), (dict(kv_heads=0), INVALID), (dict(dtype=2), INVALID),
    (dict(page_stride=-1), INVALID), (dict(page_stride=RUN - 16), INVALID), (dict(page_stride=RUN + 8), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
    (dict(kv_heads=1025), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=512), UNSUPPORTED),
    (dict(k=AT + 8), UNSUPPORTED), (dict(v=AT + 4), UNSUPPORTED),
]
BAD_BATCHES = [
    (dict(seqs=-1), INVALID), (dict(rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(max_pages=0), INVALID), (dict(table_stride=3), INVALID),
    (dict(page_table=None), INVALID), (dict(kv_len=None), INVALID), (dict(q_start=None), INVALID),
    (dict(max_pages=1 << 25, table_stride=1 << 25), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED),
]


@pytest.mark.parametrize("field,status", BAD_CACHES)
def test_bad_caches_are_refused(lib, field, status):
    c = _cache(**field)
    assert _append(lib, c, _batch()) == status
    assert _attend(lib, c, _batch()) == status
    assert lib.veda_packed_copy_pages(C.byref(c), None, 0, None) == status
    assert lib.veda_packed_attn_workspace_bytes(C.byref(c), C.byref(_batch()), 4) == 0


@pytest.mark.parametrize("field,status", BAD_BATCHES)
def test_bad_batches_are_refused(lib, field, status):
    assert _append(lib, _cache(), _batch(**field)) == status
    assert _attend(lib, _cache(), _batch(**field)) == status
    assert lib.veda_packed_attn_workspace_bytes(C.byref(_cache()), C.byref(_batch(**field)), 4) == 0


def test_null_cache_or_batch_is_refused(lib):
    assert _append(lib, None, _batch()) == INVALID and _append(lib, _cache(), None) == INVALID
    assert _attend(lib, None, _batch()) == INVALID and _attend(lib, _cache(), None) == INVALID
    assert lib.veda_packed_copy_pages(None, None, 0, None) == INVALID
    assert lib.veda_packed_attn_workspace_bytes(None, C.byref(_batch()), 4) == 0 and lib.veda_packed_attn_workspace_bytes(C.byref(_cache()), None, 4) == 0


@pytest.mark.parametrize("more,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=-1), INVALID), (dict(q_heads=40000), UNSUPPORTED), (dict(sk=veda.veda_strides(0, -8, 256)), INVALID),
    (dict(so=veda.veda_strides(0, 128, 64)), INVALID), (dict(sv=veda.veda_strides(0, 128, 260)), UNSUPPORTED), (dict(k=AT + 2), UNSUPPORTED),
    (dict(k_out=AT), INVALID), (dict(v_out=AT), INVALID), (dict(k_out=3 * AT), INVALID), (dict(v_out=9 * AT, q_out=9 * AT), INVALID),
    (dict(k_out=9 * AT, q=9 * AT), INVALID), (dict(k_out=2 * AT + 8), UNSUPPORTED),
    (dict(sko=veda.veda_strides(0, 64, 256)), INVALID), (dict(svo=veda.veda_strides(0, 128, 128)), INVALID), (dict(svo=veda.veda_strides(0, 128, 260)), UNSUPPORTED),
])
def test_append_refusals(lib, more, status):
    assert _append(lib, _cache(), _batch(), **more) == status


@pytest.mark.parametrize("more,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q_heads=0), INVALID), (dict(q_heads=3), INVALID), (dict(q_heads=66), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(visible=veda.veda_visible(-1, 0, 0)), INVALID), (dict(visible=veda.veda_visible(1, -1, 0)), INVALID),
    (dict(visible=veda.veda_visible(1, 0, -1)), INVALID), (dict(visible=veda.veda_visible((1 << 30) + 1, 0, 0)), INVALID),
    (dict(so=veda.veda_strides(0, 128, 120)), INVALID), (dict(sq=veda.veda_strides(0, 128, 516)), UNSUPPORTED), (dict(out=AT + 8), UNSUPPORTED),
    (dict(out=AT), INVALID),     # where q is
])
def test_attention_refusals(lib, more, status):
    assert _attend(lib, _cache(), _batch(), **more) == status


@pytest.mark.parametrize("dtype", [veda.VEDA_F32, veda.VEDA_BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_workspaces(lib, dtype, d):
    # whole 16 bytes whatever the rows; one byte too few, none and a crooked one are refused
    asked = 0
    for kv_heads in (1, 2, 3, 7, 12):
        for rows in list(range(1, 40)) + [64, 65, 127, 1000]:
            c = _cache(kv_heads=kv_heads, dtype=dtype, head_dim=d)
            b = _batch(seqs=1, rows=rows, max_new=rows, max_pages=4096, table_stride=4096)
            s = veda.veda_strides(0, d, d * kv_heads)
            need = lib.veda_packed_attn_workspace_bytes(C.byref(c), C.byref(b), kv_heads)
            assert need % 16 == 0
            if not need:
                continue
            asked += 1
            args = dict(q_heads=kv_heads, sq=s, so=s)
            assert _attend(lib, c, b, workspace_bytes=need - 1, **args) == WORKSPACE
            assert _attend(lib, c, b, workspace=None, **args) == INVALID
            assert _attend(lib, c, b, workspace=AT + 4, workspace_bytes=need, **args) == UNSUPPORTED
    assert asked > 150
    assert lib.veda_packed_attn_workspace_bytes(C.byref(_cache()), C.byref(_batch(max_pages=8, table_stride=8)), 4) == 0


def test_empty_calls_do_nothing(lib):
    for more in (dict(seqs=0, page_table=None, kv_len=None, q_start=None), dict(rows=0), dict(max_new=0)):
        assert _append(lib, _cache(), _batch(**more), k=None, v=None) == OK
        assert _attend(lib, _cache(), _batch(**more), q=None, out=None) == OK


def test_grids_beyond_2_32_threads_are_refused(lib):
    assert _append(lib, _cache(), _batch(seqs=1, rows=1 << 28, max_new=1 << 28)) == UNSUPPORTED
    assert _attend(lib, _cache(kv_heads=4), _batch(seqs=1 << 21, rows=1 << 21, max_new=1)) == UNSUPPORTED


def _step(lib, book=None, step=None, out=None):
    b = dict(pages=40, page_tokens=16, max_seqs=5, max_pages=8, table=AT, length=2 * AT, used=3 * AT)
    s = dict(seqs=4, rows=30, max_new=9, axes=1, frame_h=1, frame_w=1, seq=4 * AT, keep=5 * AT, evict=6 * AT, grow=7 * AT)
    o = dict(table_stride=8, page_table=8 * AT, kv_len=9 * AT, q_start=10 * AT, status=11 * AT, positions=12 * AT, row_seq=13 * AT, slots=14 * AT)
    for mine, more in ((b, book), (s, step), (o, out)):
        mine.update(more or {})
    return lib.veda_pages_step(C.byref(veda.veda_device_pages(*b.values())), C.byref(veda.veda_step(*s.values())), C.byref(veda.veda_step_tables(*o.values())), None)


@pytest.mark.parametrize("book,status", [
    (dict(pages=0), INVALID), (dict(page_tokens=0), INVALID), (dict(max_seqs=0), INVALID), (dict(max_pages=0), INVALID), (dict(table=None), INVALID),
    (dict(length=None), INVALID), (dict(used=None), INVALID), (dict(pages=(1 << 19) + 1), UNSUPPORTED), (dict(max_seqs=8193), UNSUPPORTED),
    (dict(page_tokens=(1 << 27) + 1), UNSUPPORTED),
])
def test_bad_books_are_refused(lib, book, status):
    assert _step(lib, book=book) == status


@pytest.mark.parametrize("step,out,status", [
    (dict(seqs=-1), {}, INVALID), (dict(rows=-1), {}, INVALID), (dict(max_new=-1), {}, INVALID), (dict(axes=2), {}, INVALID),
    (dict(axes=3, frame_h=0), {}, INVALID), (dict(axes=3, frame_w=-1), {}, INVALID), (dict(grow=None), {}, INVALID), (dict(seqs=6, seq=None), {}, INVALID),
    (dict(seqs=8193), {}, UNSUPPORTED), (dict(rows=(1 << 30) + 1), {}, UNSUPPORTED), ({}, dict(table_stride=7), INVALID), ({}, dict(page_table=None), INVALID),
    ({}, dict(kv_len=None), INVALID), ({}, dict(q_start=None), INVALID), ({}, dict(status=None), INVALID),
    ({}, dict(kv_len=5 * AT), INVALID), ({}, dict(status=7 * AT), INVALID), (dict(keep=2 * AT), {}, INVALID), (dict(seq=8 * AT), {}, INVALID),
    (dict(evict=3 * AT), {}, INVALID), (dict(grow=14 * AT), {}, INVALID),
])
def test_bad_steps_are_refused(lib, step, out, status):
    assert _step(lib, step=step, out=out) == status


def test_null_books_and_steps_are_refused(lib):
    s, o, b = veda.veda_step(), veda.veda_step_tables(), veda.veda_device_pages()
    for args in ((None, C.byref(s), C.byref(o)), (C.byref(b), None, C.byref(o)), (C.byref(b), C.byref(s), None)):
        assert lib.veda_pages_step(*args, None) == INVALID


def test_the_binding_refuses_what_does_not_fit(monkeypatch):
    cpu = dict(device="cpu")
    with pytest.raises(veda.VedaError):
        veda.PackedCache(4, 16, 2, 64, torch.bfloat16, k=torch.zeros(4, 2, 16 * 34, dtype=torch.uint8))
    with pytest.raises(veda.VedaError):
        veda.PackedCache(4, 16, 2, 64, torch.bfloat16, k=torch.zeros(4, 2, 16 * 32, dtype=torch.uint8), v=torch.zeros(4, 2, 16 * 32, dtype=torch.uint8))
    with pytest.raises(veda.VedaError):
        veda.PackedCache(1 << 32, 16, 2, 64, torch.bfloat16, **cpu)
    cache = veda.PackedCache(4, 16, 2, 64, torch.bfloat16, **cpu)
    assert cache.codes(cache.k).shape == (4, 2, 16, 32) and cache.scales(cache.v).shape == (4, 2, 16, 2)
    cache.scales(cache.v)[3, 1, 15, 1] = 7
    assert int(cache.v.view(-1)[-1]) == 7
    i32 = torch.int32
    batch = veda.CacheBatch(torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32), 1)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    monkeypatch.setattr(veda, "load", lambda: pytest.fail("the library was called"))
    for call in (lambda: veda.veda_packed_append(cache, batch, x, x), lambda: veda.veda_packed_attn_fwd(cache, batch, x, 0.1),
                 lambda: veda.veda_packed_copy_pages(cache, [(0, 1)])):
        with pytest.raises(veda.VedaError, match="current device"):
            call()
    with pytest.raises(veda.VedaError):
        veda.DevicePages(0, 16, 2, 4, **cpu)
    with pytest.raises(veda.VedaError):
        veda.DevicePages(40, 16, 2, 4, table=torch.zeros(2, 4, dtype=i32), length=torch.zeros(2, dtype=i32), used=torch.zeros(1, dtype=i32))
    book = veda.DevicePages(40, 16, 2, 4, **cpu)
    assert book.used.shape == (2,)
    with pytest.raises(veda.VedaError):
        veda.StepTables(book, 3, 10, 4, axes=2)
    with pytest.raises(veda.VedaError):
        veda.StepTables(book, 3, 10, 4, kv_len=torch.zeros(4, dtype=i32))
    out = veda.StepTables(book, 3, 10, 4)
    with pytest.raises(veda.VedaError, match="current device"):
        veda.veda_pages_step(book, out, torch.zeros(3, dtype=i32))
    monkeypatch.setattr(veda, "_on", lambda *a: None)
    for args in ((torch.zeros(2, dtype=i32),), (torch.zeros(3),), (torch.zeros(3, dtype=i32), torch.zeros(3, dtype=torch.int64)),
                 (torch.zeros(3, dtype=i32), None, None, torch.zeros(3, dtype=i32))):
        with pytest.raises(veda.VedaError):
            veda.veda_pages_step(book, out, *args)
    with pytest.raises(veda.VedaError, match="another book"):
        veda.veda_pages_step(veda.DevicePages(40, 16, 2, 5, **cpu), out, torch.zeros(3, dtype=i32))


def test_calls_of_the_other_cache_refuse_this_one(lib, monkeypatch):
    cpu, i32 = dict(device="cpu"), torch.int32
    packed, plain = veda.PackedCache(4, 16, 2, 64, torch.bfloat16, **cpu), veda.Cache(4, 16, 2, 64, torch.bfloat16, **cpu)
    batch = veda.CacheBatch(torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32), 1)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    monkeypatch.setattr(veda, "_on", lambda *a: None)
    monkeypatch.setattr(veda, "_stream_of", lambda *a: 0)
    for call in (lambda: veda.veda_cache_append(packed, batch, x, x), lambda: veda.veda_cache_attn_fwd(packed, batch, x, 0.1),
                 lambda: veda.veda_cache_copy_pages(packed, [(0, 1)]), lambda: veda.veda_cache_attn_workspace_bytes(packed, batch, 2, 3)):
        with pytest.raises(C.ArgumentError):
            call()
    for call in (lambda: veda.veda_packed_append(plain, batch, x, x), lambda: veda.veda_packed_attn_fwd(plain, batch, x, 0.1),
                 lambda: veda.veda_packed_copy_pages(plain, [(0, 1)])):
        with pytest.raises(veda.VedaError, match="4 bits"):
            call()


class Taken:
    """Stands for the library: takes every call, and keeps its name and the masks that it was told."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            seen = [(a.block, a.window, a.sinks) for a in args if isinstance(a, veda.veda_visible)]
            self.calls.append((name, *seen))
            return OK
        return call


@pytest.mark.parametrize("kind", ["packed", "plain"])
def test_masks_are_the_numbers_that_are_given(monkeypatch, kind):
    """Whatever was asked before: numbers that are not whole are refused, with nothing appended, and a tensor's number is read at every call."""
    cpu, i32 = dict(device="cpu"), torch.int32
    cache = (veda.PackedCache if kind == "packed" else veda.Cache)(4, 16, 2, 64, torch.bfloat16, **cpu)
    attend = veda.veda_packed_attn_fwd if kind == "packed" else veda.veda_cache_attn_fwd
    batch = veda.CacheBatch(torch.zeros(1, 2, dtype=i32), torch.zeros(1, dtype=i32), torch.zeros(2, dtype=i32), 1)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    lib = Taken()
    monkeypatch.setattr(veda, "load", lambda: lib)
    monkeypatch.setattr(veda, "_on", lambda *a: None)
    monkeypatch.setattr(veda, "_stream_of", lambda *a: 0)
    masks = lambda: [c[1] for c in lib.calls if len(c) > 1]
    attend(cache, batch, x, 0.1, 7, 3, 2)
    veda.veda_cache_attention(cache, batch, x, x, x, 0.1, block=7, window=3, sinks=2)
    assert masks() == [(7, 3, 2)] * 2
    lib.calls.clear()
    for bad in (dict(block=7.0, window=3, sinks=2), dict(block=7, window=3.0, sinks=2), dict(block=7, window=3, sinks=2.0)):
        with pytest.raises(TypeError):
            attend(cache, batch, x, 0.1, **bad)
        with pytest.raises(TypeError):
            veda.veda_cache_attention(cache, batch, x, x, x, 0.1, **bad)
    assert not [c for c in lib.calls if "append" in c[0] or c[0].endswith("_fwd")]
    t = torch.tensor(5)
    attend(cache, batch, x, 0.1, t, t, t)
    t.fill_(9)
    attend(cache, batch, x, 0.1, t, t, t)
    assert masks() == [(5, 5, 5), (9, 9, 9)]
