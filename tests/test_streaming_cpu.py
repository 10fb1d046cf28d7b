"""Streaming operators, the parts that need no GPU: refusals at the C entry points and in the binding, and the page book against
a plain model of it."""
import ctypes as C
import random
import subprocess

import numpy as np
import pytest
import torch

from paper_2605_30325_amd import veda

INVALID, UNSUPPORTED, WORKSPACE, OK = veda.VEDA_ERR_INVALID_ARG, veda.VEDA_ERR_UNSUPPORTED, veda.VEDA_ERR_WORKSPACE, veda.VEDA_OK
AT = 1 << 20     # a 16-byte aligned address that no check reads from


@pytest.fixture(scope="module")
def lib():
    if not veda.LIB_PATH.exists():
        from paper_2605_30325_amd import build
        build.build()
    return veda.load()


def _cache(**more):
    f = dict(pages=8, page_tokens=64, kv_heads=2, head_dim=128, dtype=veda.VEDA_BF16, page_stride=0, k=AT, v=AT)
    f.update(more)
    return veda.veda_cache(*f.values())


def _batch(**more):
    f = dict(seqs=2, rows=10, max_new=5, max_pages=4, table_stride=4, page_table=AT, kv_len=AT, q_start=AT)
    f.update(more)
    return veda.veda_cache_batch(*f.values())


BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pages=0), INVALID), (dict(kv_heads=0), INVALID), (dict(dtype=2), INVALID),
    (dict(page_stride=-1), INVALID), (dict(page_stride=2 * 64 * 128 - 8), INVALID), (dict(page_stride=2 * 64 * 128 + 4), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(kv_heads=1025), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED),
    (dict(page_tokens=512), UNSUPPORTED), (dict(k=AT + 8), UNSUPPORTED),
]
BAD_BATCHES = [
    (dict(seqs=-1), INVALID), (dict(rows=-1), INVALID), (dict(max_new=-1), INVALID), (dict(max_pages=0), INVALID), (dict(table_stride=3), INVALID),
    (dict(page_table=None), INVALID), (dict(kv_len=None), INVALID), (dict(q_start=None), INVALID),
    (dict(max_pages=1 << 25, table_stride=1 << 25), UNSUPPORTED), (dict(rows=(1 << 30) + 1), UNSUPPORTED),
]


def _append(lib, cache, batch, **more):
    s = veda.veda_strides(0, 128, 256)
    f = dict(k=AT, sk=s, v=AT, sv=s, q_heads=4, q=AT, sq=veda.veda_strides(0, 128, 512), q_out=AT, so=veda.veda_strides(0, 128, 512), rope=None, positions=None)
    f.update(more)
    return lib.veda_cache_append(None if cache is None else C.byref(cache), None if batch is None else C.byref(batch), *f.values(), None)


def _attend(lib, cache, batch, **more):
    s = veda.veda_strides(0, 128, 512)
    f = dict(q_heads=4, q=AT, sq=s, scale=0.1, visible=veda.veda_visible(1, 0, 0), out=2 * AT, so=s, lse=None, workspace=AT, workspace_bytes=1 << 30)
    f.update(more)
    return lib.veda_cache_attn_fwd(None if cache is None else C.byref(cache), None if batch is None else C.byref(batch), *f.values(), None)


@pytest.mark.parametrize("field,status", BAD_CACHES)
def test_bad_caches_are_refused(lib, field, status):
    c = _cache(**field)
    assert _append(lib, c, _batch()) == status
    assert _attend(lib, c, _batch()) == status
    assert lib.veda_cache_copy_pages(C.byref(c), None, 0, None) == status
    assert lib.veda_cache_attn_workspace_bytes(C.byref(c), C.byref(_batch()), 4) == 0


@pytest.mark.parametrize("field,status", BAD_BATCHES)
def test_bad_batches_are_refused(lib, field, status):
    assert _append(lib, _cache(), _batch(**field)) == status
    assert _attend(lib, _cache(), _batch(**field)) == status
    assert lib.veda_cache_attn_workspace_bytes(C.byref(_cache()), C.byref(_batch(**field)), 4) == 0


def test_null_cache_or_batch_is_refused(lib):
    assert _append(lib, None, _batch()) == INVALID and _append(lib, _cache(), None) == INVALID
    assert _attend(lib, None, _batch()) == INVALID and _attend(lib, _cache(), None) == INVALID
    assert lib.veda_cache_copy_pages(None, None, 0, None) == INVALID


@pytest.mark.parametrize("more,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=-1), INVALID), (dict(q_heads=40000), UNSUPPORTED), (dict(sk=veda.veda_strides(0, -8, 256)), INVALID),
    (dict(so=veda.veda_strides(0, 128, 64)), INVALID), (dict(so=veda.veda_strides(0, 64, 512)), INVALID), (dict(so=veda.veda_strides(0, 128, 1024)), INVALID),
    (dict(sv=veda.veda_strides(0, 128, 260)), UNSUPPORTED), (dict(k=AT + 2), UNSUPPORTED),
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


# (rows, heads), strides (row, head) of a result with d = 128, and whether two of its rows share bytes
LAID_OUT = [
    ((10, 4), (128, 128), True), ((10, 4), (256, 128), True), ((10, 4), (384, 128), True), ((10, 4), (512, 128), False), ((10, 4), (128, 1280), False),
    ((10, 4), (128, 1152), True), ((10, 4), (504, 128), True), ((10, 4), (1280, 256), False), ((10, 4), (136, 272), True), ((1, 4), (0, 128), False),
    ((2, 4), (128, 256), False),      # in turn: rows 0 and 1 of head 0, then of head 1
    ((10, 4), (384, 256), True),      # row 2 of head 0 is row 0 of head 3
    ((2, 3), (384, 256), False),      # 0 256 512, 384 640 896: each its own place, no axis within the other
    ((3, 3), (384, 256), False), ((3, 4), (384, 256), True), ((3, 3), (376, 256), True), ((2, 4), (1 << 40, 128), False),
]


@pytest.mark.parametrize("shape,strides,share", LAID_OUT)
def test_results_on_top_of_each_other_are_refused(lib, shape, strides, share):
    # strides that are not refused lead to the next check, which refuses the address: nothing is launched
    rows, heads = shape
    s = veda.veda_strides(0, strides[1], strides[0])
    near = veda.veda_strides(0, 128, 128 * heads)
    c = _cache(kv_heads=1)
    b = _batch(seqs=1, rows=rows, max_new=rows)
    one = veda.veda_strides(0, 128, 128)
    want = INVALID if share else UNSUPPORTED
    assert _attend(lib, c, b, q_heads=heads, q=AT, sq=near, out=AT * 2 + 8, so=s) == want
    assert _append(lib, c, b, sk=one, sv=one, q_heads=heads, q=AT, sq=near, q_out=AT * 2 + 8, so=s) == want


def test_rows_apart_against_all_their_elements(tmp_path):
    """Three axes, by marking every element of every row; the header has no HIP in it."""
    src, exe = tmp_path / "apart.cpp", tmp_path / "apart"
    src.write_text("""
#include <cstdio>
#include "rows_apart.h"
int main() {
    long long v[7];
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6) == 7)
        std::printf("%d\\n", (int)veda::rows_apart({v[0], v[1]}, {v[2], v[3]}, {v[4], v[5]}, v[6]));
}
""")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", str(veda.LIB_PATH.parent / "csrc"), str(src), "-o", str(exe)], check=True)
    rng, cases, want = random.Random(3), [], []
    for _ in range(4000):
        d = rng.choice([4, 8])
        axes = [(rng.randint(1, 5), 2 * rng.randint(0, 24) if rng.random() < 0.7 else d * rng.randint(1, 9)) for _ in range(3)]
        at = [i * axes[0][1] + j * axes[1][1] + k * axes[2][1] + e
              for i in range(axes[0][0]) for j in range(axes[1][0]) for k in range(axes[2][0]) for e in range(d)]
        cases.append(" ".join(str(x) for a in axes for x in a) + f" {d}")
        want.append(int(len(set(at)) < len(at)))
    cases += ["1073741824 128 4096 192 1 0 128", "65535 1000 65535 1001 65535 1002 64", "2 4611686018427387904 1000000 64 32768 9223372036854775800 64"]
    want += [1, 2, 0]
    got = subprocess.run([str(exe)], input="\n".join(cases), capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == want and 1000 < sum(want) < 3000


def test_attention_workspace_refusals(lib):
    c, b = _cache(), _batch(seqs=1, rows=1, max_new=1, max_pages=4096, table_stride=4096)
    need = lib.veda_cache_attn_workspace_bytes(C.byref(c), C.byref(b), 4)
    assert need > 0
    assert _attend(lib, c, b, workspace_bytes=need - 1) == WORKSPACE
    assert _attend(lib, c, b, workspace=None) == INVALID
    assert _attend(lib, c, b, workspace=AT + 4, workspace_bytes=need) == UNSUPPORTED
    # few or many rows over long caches ask for some, short caches for none
    for rows in (1, 8, 9, 16, 17, 64, 65, 1000):
        many = _batch(seqs=1, rows=rows, max_new=rows, max_pages=4096, table_stride=4096)
        need = lib.veda_cache_attn_workspace_bytes(C.byref(c), C.byref(many), 4)
        assert need > 0 and _attend(lib, c, many, workspace_bytes=need - 1) == WORKSPACE
    assert lib.veda_cache_attn_workspace_bytes(C.byref(c), C.byref(_batch(max_pages=8, table_stride=8)), 4) == 0


@pytest.mark.parametrize("dtype", [veda.VEDA_F32, veda.VEDA_BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_workspaces_hold_whole_16_bytes(lib, dtype, d):
    # sums of odd numbers of rows and key heads come before a list that is read 16 bytes at a time: what lies before it, and so the whole,
    # has to be a multiple of 16
    shared = 0
    for kv_heads in range(1, 13):
        for rows in range(33, 128):
            for seqs in (1, 3):
                b = _batch(seqs=seqs, rows=seqs * rows, max_new=rows, max_pages=4096, table_stride=4096)
                need = lib.veda_cache_attn_workspace_bytes(C.byref(_cache(kv_heads=kv_heads, dtype=dtype, head_dim=d)), C.byref(b), kv_heads)
                shared += need > 0
                assert need % 16 == 0, (kv_heads, rows, seqs)
    assert shared > 1000


def test_grids_beyond_2_32_threads_are_refused(lib):
    assert _append(lib, _cache(), _batch(seqs=1, rows=1 << 28, max_new=1 << 28)) == UNSUPPORTED
    assert _append(lib, _cache(), _batch(seqs=1 << 24, rows=1 << 24, max_new=1)) == UNSUPPORTED
    assert _attend(lib, _cache(kv_heads=4), _batch(seqs=1 << 21, rows=1 << 21, max_new=1)) == UNSUPPORTED
    assert _attend(lib, _cache(), _batch(seqs=1, rows=1 << 26, max_new=1, max_pages=4096, table_stride=4096)) == UNSUPPORTED


def test_empty_calls_do_nothing(lib):
    for more in (dict(seqs=0, page_table=None, kv_len=None, q_start=None), dict(rows=0), dict(max_new=0)):
        assert _append(lib, _cache(), _batch(**more), k=None, v=None) == OK
        assert _attend(lib, _cache(), _batch(**more), q=None, out=None) == OK
    assert lib.veda_cache_copy_pages(C.byref(_cache()), None, 0, None) == OK
    same = np.asarray([[3, 3], [5, 5]], np.int32)      # a page onto itself: nothing to launch
    assert lib.veda_cache_copy_pages(C.byref(_cache()), same.ctypes.data_as(C.c_void_p), 2, None) == OK


@pytest.mark.parametrize("pair", [(0, 8), (8, 0), (-1, 3), (3, -1)])
def test_copies_outside_the_pool_are_refused(lib, pair):
    p = np.asarray([[0, 1], pair], np.int32)
    assert lib.veda_cache_copy_pages(C.byref(_cache()), p.ctypes.data_as(C.c_void_p), 2, None) == INVALID
    assert lib.veda_cache_copy_pages(C.byref(_cache()), None, 1, None) == INVALID
    assert lib.veda_cache_copy_pages(C.byref(_cache()), p.ctypes.data_as(C.c_void_p), -1, None) == INVALID


def _config(**more):
    f = dict(head_dim=128, axes=3, axis_dim=(44, 42, 42), pairs=0, scaling=0, base=1e4, factor=1.0, trained_len=0.0, beta_fast=32.0, beta_slow=1.0, amplitude=0.0)
    f.update(more)
    f["axis_dim"] = (C.c_int32 * 3)(*f["axis_dim"])
    return veda.veda_rope_config(*f.values())


@pytest.mark.parametrize("more,status", [
    (dict(axes=0), INVALID), (dict(axes=4), INVALID), (dict(axis_dim=(44, 42, 44)), INVALID), (dict(axis_dim=(43, 42, 42)), INVALID),
    (dict(axis_dim=(0, 42, 42)), INVALID), (dict(pairs=2), INVALID), (dict(scaling=4), INVALID), (dict(base=1.0), INVALID),
    (dict(base=float("nan")), INVALID), (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=2, factor=float("inf")), INVALID),
    (dict(scaling=2, factor=2.0, axis_dim=(2, 42, 42)), INVALID), (dict(scaling=3, factor=2.0), INVALID),
    (dict(scaling=3, factor=2.0, trained_len=4096.0, beta_fast=1.0), INVALID), (dict(amplitude=-1.0), INVALID), (dict(amplitude=float("nan")), INVALID),
    (dict(head_dim=0), INVALID), (dict(head_dim=132), UNSUPPORTED), (dict(head_dim=520), UNSUPPORTED),
])
def test_rope_config_refusals(lib, more, status):
    out = C.c_void_p()
    assert lib.veda_rope_create(C.byref(_config(**more)), C.byref(out)) == status
    assert out.value is None


def test_rope_null_arguments(lib):
    out, s = C.c_void_p(), veda.veda_strides(0, 0, 128)
    assert lib.veda_rope_create(None, C.byref(out)) == INVALID and lib.veda_rope_create(C.byref(_config()), None) == INVALID
    assert lib.veda_rope_frequencies(None, None, None) == INVALID
    assert lib.veda_rope_apply(None, 1, 1, 1, 1, AT, s, AT, 0, 0, AT, s, None) == INVALID
    lib.veda_rope_destroy(None)


# ---- the page book ------------------------------------------------------------------------------------------------------

class Model:
    """Sequences as lists of (page or None), straight from the description."""

    def __init__(self, pages, page, seqs, width):
        self.pages, self.page, self.width = pages, page, width
        self.rows, self.length = [[] for _ in range(seqs)], [0] * seqs

    def held(self, p):
        return sum(r.count(p) for r in self.rows)

    def free(self):
        used = {p for r in self.rows for p in r if p is not None}
        return [p for p in range(self.pages) if p not in used]

    def table(self):
        return np.asarray([[-1 if p is None else p for p in r] + [-1] * (self.width - len(r)) for r in self.rows], np.int32)

    def extend(self, s, tokens):
        row, copies = list(self.rows[s]), []
        free = self.free()
        need = -(-tokens // self.page) - len(row)
        open_page = tokens > self.length[s] and self.length[s] % self.page
        if open_page and row[-1] is None:
            return INVALID
        fresh = open_page and self.held(row[-1]) > 1
        if need + bool(fresh) > len(free):
            return WORKSPACE
        if fresh:
            copies.append((row[-1], free[0]))
            row[-1] = free.pop(0)
        row += free[:need]
        self.rows[s], self.length[s] = row, tokens
        return copies


@pytest.mark.parametrize("seed,page", [(0, 16), (1, 64), (2, 1), (3, 16), (4, 256)])
def test_page_book_against_a_model(lib, seed, page):
    rng = random.Random(seed)
    pages, seqs, width = 24, 5, 12
    book, model = veda.Pages(pages, page, seqs, width), Model(pages, page, seqs, width)
    refused = {"extend": 0, "fork": 0}
    for _ in range(600):
        s, t = rng.randrange(seqs), rng.randrange(seqs)
        n = model.length[s]
        op = rng.choice(["extend"] * 4 + ["fork", "truncate", "evict", "compact"])
        before = book.table()
        if op == "extend":
            tokens = min(width * page, n + rng.choice([0, 1, page - 1, page, 2 * page + 3]))
            want = model.extend(s, tokens)
            if not isinstance(want, list):
                refused["extend"] += 1
                with pytest.raises(veda.VedaError) as e:
                    book.extend(s, tokens)
                assert e.value.status == want and np.array_equal(book.table(), before) and book.length(s) == n
            else:
                assert [tuple(x) for x in book.extend(s, tokens).tolist()] == want
        elif op == "fork":
            if s == t or model.length[t]:
                refused["fork"] += 1
                with pytest.raises(veda.VedaError):
                    book.fork(s, t)
                assert np.array_equal(book.table(), before)
            else:
                book.fork(s, t)
                model.rows[t], model.length[t] = list(model.rows[s]), n
        elif op == "truncate":
            tokens = rng.randint(0, n)
            book.truncate(s, tokens)
            model.rows[s], model.length[s] = model.rows[s][:-(-tokens // page)], tokens
        elif op == "evict":
            a = rng.randint(0, n)
            b = rng.randint(a, n)
            book.evict(s, a, b)
            for i in range(-(-a // page), b // page):
                model.rows[s][i] = None
        else:
            copies = [tuple(x) for x in book.compact().tolist()]
            used = pages - len(model.free())
            sources, targets = [c[0] for c in copies], [c[1] for c in copies]
            assert len(set(targets)) == len(targets) and not set(sources) & set(targets)
            assert all(a >= used > b and model.held(a) and not model.held(b) for a, b in copies)
            move = dict(copies)
            model.rows = [[move.get(p, p) for p in r] for r in model.rows]
            assert sorted({p for r in model.rows for p in r if p is not None}) == list(range(used))
        assert np.array_equal(book.table(), model.table())
        assert [book.length(i) for i in range(seqs)] == model.length and book.free_count() == len(model.free())
    assert refused["extend"] and refused["fork"]
    for s in range(seqs):
        book.truncate(s)
    assert book.free_count() == pages


def test_page_book_refusals(lib):
    out, n = C.c_void_p(), C.c_int32(7)
    for bad in ((0, 16, 1, 1), (1, 0, 1, 1), (1, 16, 0, 1), (1, 16, 1, 0)):
        assert lib.veda_pages_create(*bad, C.byref(out)) == INVALID
    assert lib.veda_pages_create(1, 16, 1, 1 << 27, C.byref(out)) == UNSUPPORTED
    assert lib.veda_pages_create(1, 16, 1, 1, None) == INVALID and out.value is None
    for call in (lib.veda_pages_fork, lib.veda_pages_truncate):
        assert call(None, 0, 0) == INVALID
    assert lib.veda_pages_evict(None, 0, 0, 0) == INVALID and lib.veda_pages_compact(None, None, 0, C.byref(n)) == INVALID
    assert lib.veda_pages_extend(None, 0, 1, None, 0, C.byref(n)) == INVALID
    assert lib.veda_pages_length(None, 0) == -1 and lib.veda_pages_free_count(None) == -1 and not lib.veda_pages_table(None)
    lib.veda_pages_destroy(None)
    book = veda.Pages(4, 16, 2, 3)
    h = book.handle
    assert lib.veda_pages_extend(h, 0, 20, None, 0, C.byref(n)) == OK and n.value == 0     # no copy, no list needed
    assert lib.veda_pages_extend(h, 0, 19, None, 0, C.byref(n)) == INVALID                 # shorter
    assert lib.veda_pages_extend(h, 0, 49, None, 0, C.byref(n)) == INVALID                 # beyond the table
    assert lib.veda_pages_extend(h, 2, 1, None, 0, C.byref(n)) == INVALID and lib.veda_pages_extend(h, -1, 1, None, 0, C.byref(n)) == INVALID
    assert lib.veda_pages_extend(h, 0, 20, None, 0, None) == INVALID
    book.fork(0, 1)
    assert lib.veda_pages_extend(h, 1, 21, None, 0, C.byref(n)) == WORKSPACE and book.length(1) == 20   # a copy, and no room to tell
    assert lib.veda_pages_truncate(h, 0, 21) == INVALID and lib.veda_pages_truncate(h, 0, -1) == INVALID
    assert lib.veda_pages_evict(h, 0, 5, 4) == INVALID and lib.veda_pages_evict(h, 0, 0, 21) == INVALID
    assert lib.veda_pages_length(h, 2) == -1 and lib.veda_pages_length(h, -1) == -1
    assert [tuple(x) for x in book.extend(1, 21).tolist()] == [(1, 2)]
    book.truncate(0)
    assert lib.veda_pages_compact(h, None, 0, C.byref(n)) == WORKSPACE and book.table()[1].tolist() == [0, 2, -1]
    assert [tuple(x) for x in book.compact().tolist()] == [(2, 1)]


def test_a_sequence_cut_inside_an_evicted_page_cannot_grow(lib):
    book = veda.Pages(8, 16, 1, 4)
    book.extend(0, 40)
    book.evict(0, 0, 32)
    book.truncate(0, 20)
    before = book.table()
    with pytest.raises(veda.VedaError) as e:
        book.extend(0, 21)
    assert e.value.status == INVALID and np.array_equal(book.table(), before) and book.length(0) == 20
    assert book.extend(0, 20).size == 0     # as long as it was: nothing to write
    book.truncate(0, 16)
    assert book.extend(0, 30).size == 0 and book.table()[0].tolist() == [-1, 0, -1, -1]


# ---- the binding --------------------------------------------------------------------------------------------------------

def test_binding_refuses_before_the_library(monkeypatch, lib):
    monkeypatch.setattr(veda, "load", lambda: pytest.fail("the library was called"))
    with pytest.raises(veda.VedaError, match="axis_dim"):
        veda.Rope(128, (2, 2, 2, 2))
    with pytest.raises(veda.VedaError, match="close rows"):
        veda.Cache(4, 16, 2, 64, torch.float32, k=torch.zeros(4, 2, 16, 64), v=torch.zeros(4, 16, 2, 64).transpose(1, 2))
    with pytest.raises(veda.VedaError, match="close rows"):
        veda.Cache(4, 16, 2, 64, torch.float32, k=torch.zeros(4, 2, 16, 64))
    table, length, start = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((table.long(), length, start), (table, length[:1], start), (table, length, start[:2]), (table.T.contiguous().T, length, start)):
        with pytest.raises(veda.VedaError):
            veda.CacheBatch(*bad, 1)
    with pytest.raises(veda.VedaError, match="a row for each"):      # one row for all of them
        veda.CacheBatch(table[:1].expand(2, 4), length, start, 1)
    veda.CacheBatch(table[:1].expand(1, 4), length[:1], start[:2], 1)
    for many in (1 << 31, 1 << 32, -(1 << 32)):
        with pytest.raises(veda.VedaError, match="32 bits"):
            veda.CacheBatch(table, length, start, many)
    one = torch.zeros(1, 2, 16, 64)
    with pytest.raises(veda.VedaError, match="pages apart"):         # one page for all of them
        veda.Cache(4, 16, 2, 64, torch.float32, k=one.expand(4, 2, 16, 64), v=one.expand(4, 2, 16, 64))
    with pytest.raises(veda.VedaError, match="32 bits"):
        veda.Pages(4, 16, 1 << 32, 1)
    cache, batch = veda.Cache(4, 16, 2, 64, torch.float32, device="cpu"), veda.CacheBatch(table, length, start, 1)
    x = torch.zeros(3, 2, 64)
    with pytest.raises(veda.VedaError, match="current device"):
        veda.veda_cache_append(cache, batch, x, x)
    with pytest.raises(veda.VedaError, match="current device"):
        veda.veda_cache_attn_fwd(cache, batch, x, 0.1)
    with pytest.raises(veda.VedaError, match="current device"):
        veda.veda_cache_copy_pages(cache, [(0, 1)])


class Recorder:
    """Stands for the library: notes the calls and says that all went well, or what it is told to."""

    def __init__(self):
        self.calls, self.attn = [], OK

    def veda_cache_append(self, *args):
        self.calls.append("append")
        return OK

    def veda_cache_attn_workspace_bytes(self, *args):
        return 64

    def veda_cache_attn_fwd(self, *args):
        self.calls.append("attend")
        return self.attn

    def veda_status_string(self, status):
        return b"status"

    def veda_last_error(self):
        return b""


def _step(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(veda, "load", lambda: rec)
    monkeypatch.setattr(veda, "_on", lambda dev, where: None)
    monkeypatch.setattr(veda, "_stream_of", lambda dev: 0)
    cache = veda.Cache(4, 16, 2, 64, torch.float32, device="cpu")
    batch = veda.CacheBatch(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 3)
    q, k, v = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64), torch.zeros(3, 2, 64)
    return rec, lambda **more: veda.veda_cache_attention(cache, batch, **{**dict(q=q, k=k, v=v, softmax_scale=0.1), **more})


@pytest.mark.parametrize("bad", [
    dict(softmax_scale=0.0), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(window=-1), dict(sinks=1 << 31),
    dict(block=-2), dict(q=torch.zeros(3, 3, 64)), dict(q=torch.zeros(3, 66, 64)), dict(q=torch.zeros(3, 4, 32)),
    dict(q=torch.zeros(3, 0, 64)), dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3 * 4 * 64 + 1)[1:].view(3, 4, 64)), dict(q=torch.zeros(3, 4, 66)[..., :64]), dict(q=torch.zeros(4, 64)),
], ids=lambda bad: "-".join(f"{k}-{tuple(v.shape) if torch.is_tensor(v) else v}" for k, v in bad.items()))
def test_a_refused_first_call_of_a_step_leaves_everything_as_it_was(monkeypatch, bad):
    rec, step = _step(monkeypatch)
    b = {}
    with pytest.raises(veda.VedaError):
        step(buffers=b, **bad)
    assert b == {} and rec.calls == []       # nothing appended either
    out, same = step(buffers=b)
    assert same is b and b["out"] is out and rec.calls == ["append", "attend"]
    assert step(buffers=b)[0] is out


def test_a_failed_first_call_of_a_step_leaves_the_buffers_as_they_were(monkeypatch):
    rec, step = _step(monkeypatch)
    b = {}
    rec.attn = veda.VEDA_ERR_HIP
    with pytest.raises(veda.VedaError):
        step(buffers=b)
    assert b == {}
    rec.attn = OK
    out, _ = step(buffers=b)
    assert step(buffers=b)[0] is out


def test_a_later_call_of_a_step_that_does_not_fit_its_buffers_appends_nothing(monkeypatch):
    rec, step = _step(monkeypatch)
    b = {}
    step(buffers=b)
    held, rec.calls = dict(b), []
    for bad in (dict(q=torch.zeros(3, 2, 64)), dict(softmax_scale=0.0), dict(q=torch.zeros(3, 4, 64).bfloat16())):
        with pytest.raises(veda.VedaError):
            step(buffers=b, **bad)
    assert rec.calls == [] and b.keys() == held.keys() and all(b[x] is held[x] for x in held)


def test_some_buffers_of_a_step_may_be_the_callers(monkeypatch):
    rec, step = _step(monkeypatch)
    for mine in (dict(out=torch.zeros(3, 4, 64)), dict(ws=torch.empty(80, dtype=torch.uint8)), dict(ws=torch.empty(16))):
        b = dict(mine)
        out, _ = step(buffers=b)
        assert out is b["out"] and set(b) == {"out", "ws"} and all(b[x] is mine[x] for x in mine)
        assert step(buffers=b)[0] is out
    rec.calls = []
    for small in (dict(ws=torch.empty(63, dtype=torch.uint8)), dict(out=torch.zeros(3, 4, 64).bfloat16()), dict(out=torch.zeros(2, 4, 64))):
        with pytest.raises(veda.VedaError, match="other sizes"):
            step(buffers=dict(small))
    assert rec.calls == []


def test_numbers_are_not_cut_off_at_32_bits(lib):
    book = veda.Pages(8, 16, 2, 4)
    book.extend(0, 20)
    far = 1 << 32
    for call in (lambda: book.extend(far, 40), lambda: book.extend(0, far + 40), lambda: book.fork(far, 1), lambda: book.fork(0, far + 1),
                 lambda: book.truncate(far, 0), lambda: book.truncate(0, far), lambda: book.evict(far, 0, 16), lambda: book.length(far)):
        with pytest.raises(veda.VedaError, match="32 bits"):
            call()
    assert book.length(0) == 20 and book.length(1) == 0


def test_books_say_no_to_sequences_that_are_not_theirs(lib):
    book = veda.Pages(8, 16, 2, 4)
    for seq in (-1, 2, 1 << 20):
        with pytest.raises(veda.VedaError):      # a length of -1 would go on into the next sum
            book.length(seq)
    assert book.length(1) == 0
    book.close()
    for call in (book.table, book.free_count, lambda: book.length(0), lambda: book.extend(0, 1), lambda: book.truncate(0), book.compact):
        with pytest.raises(veda.VedaError):
            call()


def test_copies_are_pairs(monkeypatch, lib):
    monkeypatch.setattr(veda, "_on", lambda dev, where: None)
    monkeypatch.setattr(veda, "_stream_of", lambda dev: 0)
    cache, seen = veda.Cache(8, 16, 2, 64, torch.float32, device="cpu"), []

    class Listed(Recorder):
        def veda_cache_copy_pages(self, ref, at, n, stream):
            seen.append(np.ctypeslib.as_array(C.cast(at, C.POINTER(C.c_int32)), (n, 2)).tolist() if n else [])
            return OK

    rec = Listed()
    monkeypatch.setattr(veda, "load", lambda: rec)
    for pairs in ([[1, 2], [3, 4]], np.asarray([[1, 2], [3, 4]]), [1, 2, 3, 4]):
        veda.veda_cache_copy_pages(cache, pairs)
        assert seen.pop() == [[1, 2], [3, 4]]
    for none in ([], np.zeros((0, 2), np.int32)):
        veda.veda_cache_copy_pages(cache, none)
        assert seen.pop() == []
    for bad in ([[1, 2, 3, 4], [5, 6, 7, 0]], [1, 2, 3], [[[1, 2]]], 5, np.zeros((2, 3), np.int32)):      # the first: sources and targets
        with pytest.raises(veda.VedaError, match="pairs"):
            veda.veda_cache_copy_pages(cache, bad)
    assert seen == []


def test_counts_and_kinds_are_not_cut_off_either(monkeypatch, lib):
    cache = veda.Cache(4, 16, 2, 64, torch.float32, device="cpu")
    batch = veda.CacheBatch(torch.zeros(1, 4096, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 3)
    assert veda.veda_cache_attn_workspace_bytes(cache, batch, 4, 3) > 0
    for q_heads, rows in (((1 << 32) + 4, 3), (4, (1 << 32) + 3)):
        with pytest.raises(veda.VedaError, match="32 bits"):
            veda.veda_cache_attn_workspace_bytes(cache, batch, q_heads, rows)
    monkeypatch.setattr(veda, "load", lambda: pytest.fail("the library was called"))
    for more in (dict(pairs=1 << 32), dict(scaling=1 << 32)):
        with pytest.raises(veda.VedaError, match="32 bits"):
            veda.Rope(64, 64, **more)
