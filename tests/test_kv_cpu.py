"""The 4-bit key/value cache without a GPU: refusals of every entry point before anything is launched, the book of pages against a
plain Python one, and pins of the numpy statement that the device tests compare with."""
import ctypes as C
import os
import subprocess
import types

import numpy as np
import pytest
import torch

import test_kv_gpu as tg
from oracle import kv_cache as okv
from paper_2310_08041_amd import binding as b

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, PAGES = -1, -2, -4, -6, -7, -9
A = 0x10000                                    # never dereferenced: every call below fails before a launch, or has nothing to do


def cache(heads=2, dim=128, page=64, n_pages=10, pages=A):
    return b._KVCache(heads, dim, page, n_pages, pages)


def batch(rows=4, n_seqs=4, row_start=None, slot=None, n_slots=4, ld=3, table=A, length=A):
    return b._KVBatch(rows, n_seqs, row_start, slot, n_slots, ld, table, length)


BAD_SIZES = [(dict(heads=0), {}), (dict(heads=-1), {}), (dict(dim=96), {}), (dict(page=16), {}), (dict(page=48), {}), (dict(page=512), {}),
             (dict(n_pages=0), {}), (dict(n_pages=1 << 31), {}), ({}, dict(rows=-1)), ({}, dict(rows=1 << 25)), ({}, dict(n_seqs=-1)),
             ({}, dict(n_slots=0)), ({}, dict(ld=0)), ({}, dict(ld=1 << 26)), ({}, dict(rows=3)), ({}, dict(n_slots=3))]
BAD_POINTERS = [(dict(pages=None), {}, NULL), ({}, dict(table=None), NULL), ({}, dict(length=None), NULL), (dict(pages=A + 8), {}, ALIGN),
                ({}, dict(table=A + 2), ALIGN), ({}, dict(row_start=A + 1), ALIGN), ({}, dict(slot=A + 2), ALIGN)]


def append(c=None, t=None, q=A, ldq=512, hq=4, q_out=A, ldqo=512, k=A, ldk=256, v=A, ldv=256, dt=b.BF16, rope=1, f=A, no_c=False, no_t=False):
    c, t = c or cache(), t or batch()
    return b.raw().qllm_kv_append(q, ldq, hq, q_out, ldqo, k, ldk, v, ldv, dt, rope, f, None if no_c else C.byref(c), None if no_t else C.byref(t), None)


def read(c=None, t=None, k=A, ldk=256, v=A, ldv=256, dt=b.BF16):
    c, t = c or cache(), t or batch()
    return b.raw().qllm_kv_read(C.byref(c), C.byref(t), k, ldk, v, ldv, dt, None)


def attend(c=None, t=None, q=A, dt=b.BF16, ldq=512, hq=4, scale=0.1, window=0, out=A, odt=b.BF16, ldo=512, ws=A, ws_bytes=1 << 30):
    c, t = c or cache(), t or batch()
    return b.raw().qllm_kv_attention(q, dt, ldq, hq, C.byref(c), C.byref(t), scale, window, out, odt, ldo, ws, ws_bytes, None)


def test_entry_points_refuse_bad_arguments_before_launching():
    for call in (append, read, attend):
        for ck, tk in BAD_SIZES:
            assert call(cache(**ck), batch(**tk)) == SHAPE, (call, ck, tk)
        for ck, tk, want in BAD_POINTERS:
            assert call(cache(**ck), batch(**tk)) == want, (call, ck, tk)
        assert call(dt=2) == DTYPE
        assert call(t=batch(rows=0, n_seqs=0)) == 0 and call(t=batch(rows=5, n_seqs=0)) == 0
        assert call(t=batch(rows=0, n_seqs=3, row_start=A)) == 0
    assert append(no_c=True) == NULL and append(no_t=True) == NULL
    assert append(k=None) == NULL and append(v=None) == NULL and append(q=None) == NULL and append(q_out=None) == NULL and append(f=None) == NULL
    assert append(rope=3) == DTYPE and append(rope=-1) == DTYPE
    assert append(ldk=255) == SHAPE and append(ldv=255) == SHAPE and append(ldq=511) == SHAPE and append(ldqo=511) == SHAPE and append(hq=0) == SHAPE
    assert append(k=A + 1) == ALIGN and append(q=A + 2, dt=b.F32) == ALIGN and append(f=A + 4) == ALIGN
    assert append(k=None, v=None, q=None, t=batch(rows=0, n_seqs=2, row_start=A)) == 0             # empty tensors have no address
    assert read(ldk=255) == SHAPE and read(ldv=0) == SHAPE and read(k=A + 1) == ALIGN
    assert attend(q=None) == NULL and attend(out=None) == NULL and attend(odt=-1) == DTYPE
    assert attend(hq=3) == SHAPE and attend(hq=0) == SHAPE and attend(ldq=511) == SHAPE and attend(ldo=511) == SHAPE and attend(window=-1) == SHAPE
    assert attend(scale=float("nan")) == SHAPE and attend(scale=float("inf")) == SHAPE
    assert attend(q=A + 1) == ALIGN and attend(out=A + 2, odt=b.F32) == ALIGN and attend(ws=A + 4) == ALIGN
    assert attend(ws=None) == WORKSPACE and attend(ws_bytes=0) == WORKSPACE
    f = b.raw().qllm_kv_attention_workspace_bytes
    assert f(C.byref(cache(pages=None)), C.byref(batch(table=None, length=None)), 4) > 0           # sizes only
    assert f(C.byref(cache()), C.byref(batch()), 5) == SHAPE and f(C.byref(cache(dim=32)), C.byref(batch()), 4) == SHAPE
    assert b.raw().qllm_kv_page_bytes(8, 128, 64) == 8 * 64 * 144 and b.raw().qllm_kv_page_bytes(1, 64, 32) == 32 * 80
    assert b.status_string(PAGES) != b.status_string(-99)


def test_copying_pages_refuses_clashes_and_numbers_out_of_range():
    f = b.raw().qllm_kv_copy_pages

    def copy(src, dst, pages=A, layers=2, stride=10 * 4096, n_pages=10, page_bytes=4096, n=None):
        s, d = np.array(src, np.int32), np.array(dst, np.int32)
        return f(pages, layers, stride, n_pages, page_bytes, s.ctypes.data if s.size else None, d.ctypes.data if d.size else None, s.size if n is None else n, None)

    assert copy([], []) == 0 and copy([3, 4], [3, 4], layers=0) == 0
    assert copy([5, 6], [5, 6]) == 0                                         # nothing to move: nothing is launched
    assert copy([0, 1], [5, 5]) == PAGES                                     # one page copied to twice
    assert copy([0, 5], [5, 6]) == PAGES                                     # a page that is source and destination
    assert copy([0, 5], [5, 5]) == PAGES
    assert copy([10], [1]) == PAGES and copy([-1], [1]) == PAGES and copy([1], [10]) == PAGES and copy([1], [-2]) == PAGES
    assert copy(list(range(10)) + [0], list(range(10)) + [0]) == PAGES       # more pairs than pages
    assert copy([0], [1], pages=None) == NULL and copy([], [], n=1) == NULL and copy([0], [1], n=-1) == SHAPE
    assert copy([0], [1], pages=A + 8) == ALIGN and copy([0], [1], page_bytes=4100, stride=41000) == ALIGN and copy([0], [1], stride=40968) == ALIGN
    assert copy([0], [1], stride=10 * 4096 - 16) == SHAPE and copy([0], [1], stride=-(1 << 40)) == SHAPE
    assert copy([0], [1], n_pages=0) == SHAPE and copy([0], [1], page_bytes=0) == SHAPE and copy([0], [1], layers=-1) == SHAPE


def test_wrappers_refuse_mismatched_tensors():
    """On CPU tensors: every call fails on a shape or type, or at last on "must be a device tensor"."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    kv = b.DeviceKVCache(2, 5, 2, 64, 32, device="cpu")
    t = b.DeviceKVBatch(3, i32(3, 4), i32(3))
    k = torch.zeros((3, 128))
    q = torch.zeros((3, 256))
    f = torch.zeros(32, dtype=torch.float64)
    ws = torch.zeros(1 << 12, dtype=torch.uint8)
    cases = [
        (lambda: b.DeviceKVCache(1, 5, 2, 64, 32, pages=torch.zeros((1, 4, 5120), dtype=torch.uint8)), "pages has shape"),
        (lambda: b.DeviceKVCache(1, 5, 2, 64, 32, pages=torch.zeros((1, 5, 5120))), "pages has dtype"),
        (lambda: b.DeviceKVCache(2, 5, 2, 64, 32, pages=torch.zeros((5, 2, 5120), dtype=torch.uint8).transpose(0, 1)), "contiguous"),
        (lambda: b.DeviceKVBatch(3, i32(3, 4), i32(4)), "length must hold 3"),
        (lambda: b.DeviceKVBatch(3, i32(3, 4).long(), i32(3)), "table has dtype"),
        (lambda: b.DeviceKVBatch(3, i32(3, 8)[:, ::2], i32(3)), "table must be"),
        (lambda: b.DeviceKVBatch(2, i32(3, 4), i32(3)), "as many rows"),
        (lambda: b.DeviceKVBatch(9, i32(3, 4), i32(3), row_start=i32(5)), "4 sequences, but 3 lines"),
        (lambda: b.DeviceKVBatch(9, i32(3, 4), i32(3), row_start=i32(5), slot=i32(3)), "slot must hold 4"),
        (lambda: b.DeviceKVBatch(9, i32(3, 4), i32(3), row_start=i32(0)), "row_start needs"),
        (lambda: b.qllm_kv_append(kv, 2, t, k, k), "layer 2"),
        (lambda: b.qllm_kv_append(kv, 0, t, k[:2], k), "k has shape"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, torch.zeros((3, 64))), "v has shape"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k.bfloat16()), "v has dtype"),
        (lambda: b.qllm_kv_append(kv, 0, t, k.half(), k.half()), "k has dtype"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, q=q), "go together"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, q=q, q_out=q[:, :128], rope=0), "q_out has shape"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, rope=1), "inv_freq is required"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, rope=1, inv_freq=f.float()), "inv_freq has dtype"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, rope=1, inv_freq=f[:8]), "inv_freq must hold"),
        (lambda: b.qllm_kv_append(kv, 0, t, k.t().contiguous().t(), k), "stride 1"),
        (lambda: b.qllm_kv_append(kv, 0, t, k, k, q=q, q_out=q, rope=1, inv_freq=f), "must be a device"),
        (lambda: b.qllm_kv_read(kv, 0, t), "k_out or v_out"),
        (lambda: b.qllm_kv_read(kv, 0, t, k, k.bfloat16()), "v_out has dtype"),
        (lambda: b.qllm_kv_read(kv, 0, t, k), "must be a device"),
        (lambda: b.qllm_kv_attention(q[:, :250], kv, 0, t, 0.1, q, ws), "q has shape"),
        (lambda: b.qllm_kv_attention(q, kv, 0, t, 0.1, q[:, :128], ws), "out has shape"),
        (lambda: b.qllm_kv_attention(q, kv, 0, t, 0.1, q, None), "workspace is required"),
        (lambda: b.qllm_kv_attention(q, kv, 0, t, 0.1, q, ws[::2]), "stride 1"),
        (lambda: b.qllm_kv_attention(q, kv, 0, t, 0.1, q, ws), "must be a device"),
        (lambda: b.qllm_kv_copy_pages(kv, [1, 2], [3]), "of one length"),
        (lambda: b.KVBook(32, np.zeros((2, 3)), np.zeros(2, np.int32), np.zeros(4, np.int32)), "table must be"),
        (lambda: b.KVBook(32, np.zeros((2, 3), np.int32), np.zeros(3, np.int32), np.zeros(4, np.int32)), "length must hold"),
        (lambda: b.qllm_kv_reserve_host(b.KVBook.empty(2, 3, 4, 32), [0, 1], [1]), "counts must be"),
    ]
    for call, text in cases:
        with pytest.raises(ValueError, match=text):
            call()


@pytest.mark.parametrize("layers,n_pages", [(0, 5), (-1, 5), (2, 0)])
def test_a_cache_without_layers_or_pages_is_refused(layers, n_pages):
    with pytest.raises(ValueError, match="a cache of"):
        b.DeviceKVCache(layers, n_pages, 2, 64, 32, device="cpu")


def test_wrappers_refuse_tensors_of_another_device(monkeypatch):
    """A tensor of a device that is not the current one is refused (devices are pretended: there is none here)."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    there = types.SimpleNamespace(is_cuda=True, get_device=lambda: 1)
    here = types.SimpleNamespace(is_cuda=True, get_device=lambda: 0)
    b._check_on_current(a=here, c=None)
    with pytest.raises(ValueError, match="q is on device 1, the call runs on device 0"):
        b._check_on_current(a=here, q=there)


def test_arrays_that_the_library_holds_addresses_of_are_not_replaced():
    """An assignment would leave the C struct with the old array's address, and its memory to the next owner."""
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    book, kv, t = b.KVBook.empty(2, 3, 4, 32), b.DeviceKVCache(1, 5, 2, 64, 32, device="cpu"), b.DeviceKVBatch(3, i32(3, 4), i32(3), slot=i32(3))
    for owner, names in ((book, ("table", "length", "refs")), (kv, ("pages",)), (t, ("table", "length", "row_start", "slot"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(owner, name, getattr(owner, name))
    book.length[:] = 1                                                       # their contents are the caller's
    t.length.add_(1)
    kv.pages.zero_()


def test_lists_that_do_not_fit_are_refused_and_not_wrapped_around():
    """64-bit numbers beyond int32 named line 0, fractions the line below: refused, in any form that a list may come in."""
    book = b.KVBook.empty(2, 3, 4, 32)
    b.qllm_kv_reserve_host(book, [0, 1], [5, 6])
    kv = b.DeviceKVCache(1, 5, 2, 64, 32, device="cpu")
    far = 2 ** 32
    for bad in ([far], (far,), [-far], np.array([far]), np.array([-far]), np.array([far], np.uint64), np.array([2 ** 31]), torch.tensor([far]), [0.5], [1.0],
                np.array([0.5]), torch.tensor([0.0]), [None], ["0"], np.array([True])):
        for call in (lambda: b.qllm_kv_free_host(book, bad), lambda: b.qllm_kv_reserve_host(book, bad, [1]), lambda: b.qllm_kv_reserve_host(book, [1], bad),
                     lambda: b.qllm_kv_copy_pages(kv, bad, [1]), lambda: b.qllm_kv_fork_host(book, bad, [1])):
            with pytest.raises(ValueError, match="whole numbers"):
                call()
    assert book.length.tolist() == [5, 6]
    for good in ([1], (1,), np.array([1]), np.array([1], np.uint8), np.array([0, 1, 2], np.int32)[1::2], torch.tensor([1]), 1, np.int64(1), [np.int64(1)]):
        b.qllm_kv_reserve_host(book, good, 1)
    assert book.length.tolist() == [5, 15]
    b.qllm_kv_free_host(book, [])
    b.qllm_kv_free_host(book, np.array([]))
    for bad in ([[0, 1]], np.zeros((1, 2), np.int32)):
        with pytest.raises(ValueError):
            b.qllm_kv_free_host(book, bad)


# ---------------------------------------------------------------- the book

def same(book, plain):
    assert np.array_equal(book.table, plain.table())
    assert book.length.tolist() == plain.length and book.refs.tolist() == plain.refs()


def test_book_against_a_plain_one():
    """Thousands of random requests: the same pages, lengths, references and copies; a request that cannot be met changes nothing."""
    import copy
    rng = np.random.default_rng(3)
    seen = dict(reserve=0, fork=0, free=0, compact=0, refused=0)
    for trial in range(60):
        lines, per_line, n_pages, page = int(rng.integers(1, 9)), int(rng.integers(1, 9)), int(rng.integers(1, 30)), int(rng.choice([32, 64, 128, 256]))
        book, plain = b.KVBook.empty(lines, per_line, n_pages, page), okv.Book(lines, per_line, n_pages, page)
        for _ in range(60):
            kind = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
            trial_plain = copy.deepcopy(plain)
            before = [a.copy() for a in (book.table, book.length, book.refs)]
            n = int(rng.integers(1, lines + 1))
            ok, copies = True, None
            try:
                if kind == "reserve":
                    slots, counts = rng.integers(0, lines, n), rng.choice([0, 1, 5, page, 2 * page + 3], n)
                    for s, k in zip(slots, counts):
                        ok = ok and trial_plain.reserve(int(s), int(k))
                    b.qllm_kv_reserve_host(book, slots, counts)
                elif kind == "fork":
                    empty = [i for i in range(lines) if plain.length[i] == 0]
                    full = [i for i in range(lines) if plain.length[i]]
                    if not empty or not full:
                        continue
                    children = rng.permutation(empty)[:n]
                    parents = rng.choice(full, children.size)
                    copies = [trial_plain.fork(int(p), int(c)) for p, c in zip(parents, children)]
                    ok = False not in copies
                    src, dst = b.qllm_kv_fork_host(book, parents, children)
                    assert list(zip(src.tolist(), dst.tolist())) == [c for c in copies if c is not None]
                elif kind == "free":
                    slots = rng.integers(0, lines, n)                    # a line may be named twice, or be empty
                    for s in slots:
                        trial_plain.free(int(s))
                    b.qllm_kv_free_host(book, slots)
                else:
                    want = trial_plain.compact()
                    src, dst = b.qllm_kv_compact_host(book)
                    assert (src.tolist(), dst.tolist()) == want
                    assert set(src).isdisjoint(dst) and (book.refs[:int((book.refs > 0).sum())] > 0).all()
                assert ok
                plain = trial_plain
                seen[kind] += 1
            except b.QllmError as e:
                assert not ok and e.status in (SHAPE, PAGES)
                assert all(np.array_equal(x, y) for x, y in zip(before, (book.table, book.length, book.refs)))
                seen["refused"] += 1
            same(book, plain)
    assert all(v > 40 for v in seen.values()), seen


def test_book_refuses_what_contradicts_itself():
    lib = b.raw()
    i32 = lambda *a: np.array(a, np.int32)

    def made():
        book = b.KVBook.empty(4, 4, 6, 32)
        b.qllm_kv_reserve_host(book, [0, 1], [70, 33])               # pages 0, 1, 2 and 3, 4
        return book

    def refused(want, call, *args):
        with pytest.raises(b.QllmError) as e:
            call(*args)
        assert e.value.status == want

    book = made()
    assert book.table[:2].tolist() == [[0, 1, 2, -1], [3, 4, -1, -1]]
    refused(SHAPE, b.qllm_kv_reserve_host, book, [4], [1])
    refused(SHAPE, b.qllm_kv_reserve_host, book, [-1], [1])
    refused(SHAPE, b.qllm_kv_reserve_host, book, [0], [-1])
    refused(SHAPE, b.qllm_kv_reserve_host, book, [0], [59])          # 129 tokens in 4 pages of 32
    refused(SHAPE, b.qllm_kv_reserve_host, book, [0, 0], [2147483647, 2147483647])
    refused(PAGES, b.qllm_kv_reserve_host, book, [2], [64])          # two pages, one is free
    refused(SHAPE, b.qllm_kv_fork_host, book, [0], [1])              # a child that has tokens
    refused(SHAPE, b.qllm_kv_fork_host, book, [0, 1], [2, 2])
    refused(SHAPE, b.qllm_kv_fork_host, book, [0, 2], [2, 3])        # a child that is a parent too
    refused(SHAPE, b.qllm_kv_fork_host, book, [0], [9])
    refused(PAGES, b.qllm_kv_fork_host, book, [0, 1], [2, 3])        # two part pages, one page is free
    refused(SHAPE, b.qllm_kv_free_host, book, [7])
    for spoil in (lambda k: k.table.__setitem__((0, 1), 6), lambda k: k.table.__setitem__((0, 1), -1), lambda k: k.refs.__setitem__(1, 0),
                  lambda k: k.length.__setitem__(0, 200), lambda k: k.length.__setitem__(0, -1)):
        book = made()
        spoil(book)
        refused(PAGES, b.qllm_kv_reserve_host, book, [0], [1])
        refused(PAGES, b.qllm_kv_fork_host, book, [0], [2])
        refused(PAGES, b.qllm_kv_free_host, book, [0])
        refused(PAGES, b.qllm_kv_compact_host, book)
    book = made()
    book.table[1, 0] = 0                                             # two lines, one reference
    refused(PAGES, b.qllm_kv_free_host, book, [0, 1])
    book = made()
    book.refs[2] = 2                                                 # a part page that is shared: appending would write into both lines
    refused(PAGES, b.qllm_kv_reserve_host, book, [0], [1])
    bad = b._KVBook(48, 1, 1, 1, A, A, A)
    assert lib.qllm_kv_compact_host(C.byref(bad), A, A) == SHAPE and lib.qllm_kv_free_host(None, None, 0) == NULL
    assert lib.qllm_kv_reserve_host(C.byref(made().c), None, None, 1) == NULL and lib.qllm_kv_reserve_host(C.byref(made().c), None, None, -1) == SHAPE
    assert lib.qllm_kv_fork_host(C.byref(made().c), i32(0).ctypes.data, i32(2).ctypes.data, 1, None, None) == NULL
    assert lib.qllm_kv_compact_host(C.byref(made().c), None, None) == NULL


@pytest.mark.parametrize("n,ctx,shared,page", [(4, 200, 0, 64), (4, 200, 63, 64), (4, 200, 64, 64), (4, 200, 150, 64), (1, 200, 150, 64), (3, 64, 63, 32), (16, 500, 499, 32)])
def test_bench_counts_tokens_in_shared_pages_once(n, ctx, shared, page):
    """Against the book that the bench's cache stage makes: a token of every entry of every page."""
    import bench
    per_line = -(-ctx // page)
    book = b.KVBook.empty(n, per_line, n * per_line, page)
    if shared:
        b.qllm_kv_reserve_host(book, [0], [shared])
        b.qllm_kv_fork_host(book, [0] * (n - 1), list(range(1, n)))
    b.qllm_kv_reserve_host(book, list(range(n)), [ctx - int(x) for x in book.length])
    places = {(int(book.table[i, t // page]), t % page) for i in range(n) for t in range(ctx)}
    assert bench.kv_tokens(n, ctx, shared, page) == len(places)


# ---------------------------------------------------------------- pins of the numpy statement

def test_statement_of_the_rotation():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 2, 8)).astype(np.float32)
    f = np.array([1.0, 0.1, 0.01, 0.001])
    pos = np.array([0, 1, 2, 1000, 123456])
    halves = okv.rotate(x, pos, f, 1)
    assert np.array_equal(halves[0], x[0])                                                      # position 0 stays
    z = (x[..., :4] + 1j * x[..., 4:].astype(np.float64)) * np.exp(1j * pos[:, None, None] * f)
    assert np.abs(halves - np.concatenate([z.real, z.imag], -1)).max() < 1e-6
    order = [0, 4, 1, 5, 2, 6, 3, 7]
    assert np.array_equal(okv.rotate(x[..., order], pos, f, 2), halves[..., order])             # the same pairs, side by side
    # the score of two tokens goes by their distance alone
    k, q = x[:1, :1], x[1:2, :1]
    score = [(okv.rotate(q, [p + 7], f, 1) * okv.rotate(k, [p], f, 1)).sum() for p in (0, 50, 4000)]
    assert np.ptp(score) < 1e-5


def test_statement_of_the_quantizer(oracle):
    """Against the layer's own Eq. (2), whose alpha is a correctly rounded quotient: within one ulp, and with it at most a step of
    beta and of codes at a border; constant, tiny and one-sided vectors by hand."""
    x = np.random.default_rng(4).standard_normal((400, 64)).astype(np.float32) * 3.0
    codes, alpha, beta = okv.quantize(x)
    c2, a2, b2, _ = oracle.quantize_rows(x, 4)
    assert (np.abs(alpha - a2) <= np.spacing(a2)).all() and (np.abs(beta - b2) <= 1).all()
    assert (codes != c2).mean() < 1e-3 and np.abs(codes.astype(int) - c2).max() <= 1
    back = alpha[:, None].astype(np.float64) * (codes.astype(np.float64) - beta[:, None])
    assert (np.abs(back - x) <= alpha[:, None] * 1.001).all()
    codes, alpha, beta = okv.quantize(np.array([[0.75] * 4, [0.0] * 4, [1e-40, 0, 0, 0], [30.0, 45.0, 31.4, 44.6]], np.float32))
    assert alpha.tolist() == [1.0, 1.0, 1.0, 1.0] and beta.tolist() == [-1, 0, 0, -30]
    assert codes.tolist() == [[0] * 4, [0] * 4, [0] * 4, [0, 15, 1, 15]]


def test_statement_of_the_pages_and_of_attention():
    rng = np.random.default_rng(2)
    heads, dim, page = 2, 64, 32
    raw = np.zeros((4, heads * page * (dim + 16)), np.uint8)
    pages = okv.Pages(raw, heads, dim, page)
    table = np.array([[2, 0, -1]], np.int32)
    length = np.array([40], np.int32)
    k, v = (rng.standard_normal((40, heads, dim)).astype(np.float32) for _ in range(2))
    tok = okv.rows_of(40, np.array([0, 40]), None, length)
    okv.append(pages, table, tok, k, v)
    for h in range(heads):
        for r in (0, 31, 32, 39):
            for value, x in ((0, k), (1, v)):
                got, alpha, _ = pages.get(2 if r < 32 else 0, h, r % 32, value)
                assert np.abs(got - x[r, h]).max() <= 1.01 * alpha                          # half a step, and the zero point's half
    assert not raw[[1, 3]].any() and not raw[0][pages._at(0, 0, 8, 0)[1]]                   # nothing beyond the 40 tokens
    # by hand: code 2j low, 2j + 1 high, behind them the parameters
    assert pages._at(1, 1, 3, 1) == (1, 32 * 80 + (32 + 3) * 32, 32 * 80 + 32 * 64 + 8 * 32 + 12)
    q = rng.standard_normal((40, 6, dim)).astype(np.float32)
    out, absv, err_s, err_o = okv.attention(q, pages, table, tok, length, 0.2, window=9)
    kk = np.array([[pages.get(2 if t < 32 else 0, h, t % 32, 0)[0] for t in range(40)] for h in range(heads)])
    vv = np.array([[pages.get(2 if t < 32 else 0, h, t % 32, 1)[0] for t in range(40)] for h in range(heads)])
    s = np.einsum("rhgd,htd->rhgt", q.reshape(40, heads, 3, dim).astype(np.float64), kk) * 0.2
    dist = np.arange(40)[:, None] - np.arange(40)
    s = np.where((dist >= 0) & (dist < 9), s.transpose(1, 2, 0, 3), -np.inf)
    w = np.exp(s - s.max(-1, keepdims=True))
    ref = np.einsum("hgrt,htd->rhgd", w / w.sum(-1, keepdims=True), vv).reshape(40, 6, dim)
    assert np.abs(out - ref).max() < 1e-12
    assert np.abs(out[0].reshape(heads, 3, dim) - vv[:, None, 0]).max() < 1e-12             # the first token sees itself alone
    assert (absv >= np.abs(out) - 1e-12).all() and (err_s >= 0).all() and err_s.max() < 1e-2 and err_o.max() < 1e-3
    late = okv.attention(q[:3], pages, table, [(0, 0, -1), (1, 5, 3), (2, 0, 0)], length, 0.2)[0]
    assert not late[:2].any() and late[2].any()


def test_limits_of_a_step():
    f = b.raw().qllm_kv_attention_workspace_bytes
    bytes_for = lambda hq, ck={}, **tk: f(C.byref(cache(pages=None, **ck)), C.byref(batch(table=None, length=None, **tk)), hq)
    assert bytes_for(4, rows=(1 << 24) - 1, row_start=A) > 0 and bytes_for(4, rows=1 << 24, row_start=A) == SHAPE
    assert bytes_for(4, n_seqs=(1 << 20) + 1, rows=1 << 21, row_start=A) == SHAPE
    assert bytes_for(1 << 15) > 0 and bytes_for(1 << 16) == SHAPE
    assert bytes_for(64, rows=(1 << 22) - 64, row_start=A) > 0 and bytes_for(64, rows=1 << 22, row_start=A) == SHAPE     # 2^23 tiles of 16 rows
    assert bytes_for(4, rows=1 << 21, row_start=A, n_slots=8, ld=1 << 14) == SHAPE                                 # 2^31 steps of 32 tokens


# ---------------------------------------------------------------- index arithmetic of the kernels, compiled for the host

@pytest.fixture(scope="module")
def index(tmp_path_factory):
    """csrc/kv_index.h as a host library."""
    here = tmp_path_factory.mktemp("kv_index")
    (here / "index.cpp").write_text('''#include "kv_index.h"
using namespace qllm_kv_detail;
extern "C" int32_t entry(int32_t p, int32_t shift, int32_t ld) { return entry_of(p, shift, ld); }
extern "C" int32_t first(int32_t pos, int32_t window) { return first_seen(pos, window); }
extern "C" int32_t block(int32_t b, int32_t last) { return block_begin(b, last); }
''')
    csrc = os.path.join(os.path.dirname(b.__file__), "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", csrc, str(here / "index.cpp"), "-o", str(here / "index.so")], check=True)
    return C.CDLL(str(here / "index.so"))


@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_table_entries_stay_in_their_line_up_to_the_last_position(index, page):
    """The lists of page numbers that the prompts kernel makes (64 blocks of 32 tokens from a tile of 64 on, two tiles and more ahead of
    the last): every entry lies in the line, is that of the block, and blocks behind the last position have none."""
    shift, ld = page.bit_length() - 1, (2 ** 31 - 1) // page
    top = ld * page
    for last in (-1, 0, 31, 32, top - 1, top - 33, top - 2016, top - 2017, top - 4096):
        for tile in {0, 1, max(last, 0) // 64 - 32, max(last, 0) // 64 - 1, max(last, 0) // 64, max(last, 0) // 64 + 4, (2 ** 31 - 1) // 64}:
            if tile < 0:
                continue
            for lane in range(64):
                want = (tile * 2 + lane) * 32                                # exact: no 32 bits here
                p = index.block(tile * 2 + lane, last)
                assert p == (want if want <= last else -1), (last, tile, lane)
                k = index.entry(p, shift, ld)
                assert k == (want // page if want <= last else -1), (last, tile, lane)
    for p in (-1, -32, -page, -2 ** 31, -2 ** 31 + 1, -2016):
        assert index.entry(p, shift, ld) == -1 and index.entry(p, shift, 1) == -1
    assert index.entry(top - 1, shift, ld) == ld - 1 and index.entry(2 ** 31 - 1, shift, ld - 1) == -1 and index.entry(page, shift, 1) == -1


def test_first_token_of_a_window_at_the_ends_of_its_range(index):
    """Rows before the first token, and windows up to the largest (a common way to say "none"), do not wrap around."""
    edges = [0, 1, 2, 3, 31, 32, 1000, 2 ** 24 - 1, 2 ** 24, 2 ** 30, 2 ** 31 - 2 ** 24, 2 ** 31 - 3, 2 ** 31 - 2, 2 ** 31 - 1]
    for pos in edges + [-e for e in edges if e <= 2 ** 24]:
        for window in edges:
            want = max(0, pos - window + 1) if window else 0
            assert index.first(pos, window) == want, (pos, window)


def test_a_scale_that_overflows_in_base_2_is_refused():
    """scale log2 e is what the kernels multiply by: infinite from 2.3587e38 on, although the scale itself is finite."""
    limit = float(np.finfo(np.float32).max) / 1.44269504088896341
    for scale in (1.001 * limit, 2.9e38, 3.3e38, -2.9e38):
        assert attend(scale=scale) == SHAPE and attend(scale=scale, t=batch(rows=0, n_seqs=0)) == SHAPE
    for scale in (0.999 * limit, -0.999 * limit, 0.0, 1e-45):
        assert attend(scale=scale, t=batch(rows=0, n_seqs=0)) == 0


def test_statement_of_attention_with_the_largest_windows():
    """Positions are exact whatever the arrays' type: a window that no line reaches is no window, for rows before the first token too."""
    rng = np.random.default_rng(6)
    pages = okv.Pages(np.zeros((1, 32 * 80), np.uint8), 1, 64, 32)
    table, length, start = np.zeros((1, 1), np.int32), np.array([4], np.int32), np.array([0, 9], np.int32)
    tok = okv.rows_of(9, start, None, length)
    assert [p for _, _, p in tok] == list(range(-5, 4)) and all(type(p) is int for _, _, p in tok)
    k, v = (rng.standard_normal((9, 1, 64)).astype(np.float32) for _ in range(2))
    okv.append(pages, table, tok, k, v)
    q = rng.standard_normal((9, 2, 64)).astype(np.float32)
    want = okv.attention(q, pages, table, tok, length, 0.1)[0]
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 1 << 40):
        assert np.array_equal(okv.attention(q, pages, table, tok, length, 0.1, window)[0], want) and want[5:].any() and not want[:5].any()


# ---------------------------------------------------------------- do the attention tests' bounds have teeth?

def _bits(x, n):
    """float64 rounded to n significant bits."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, n)), e - n)


def mistaken(c, q, scale, window, weight_bits=None, wider=0, newest=0):
    """The statement of attention with a mistake planted: weights times alpha of so many bits, a window of `wider` tokens more, the
    `newest` tokens left out."""
    out = np.zeros(q.shape)
    for r, line, pos in c.tokens:
        hi = min(pos, int(c.length[line]) - 1) - newest
        lo = max(0, pos - (window + wider) + 1) if window else 0
        for h in range(c.heads):
            got = [[c.pages.get(int(c.table[line, t // c.page]), h, t % c.page, value) for t in range(lo, hi + 1)] for value in (0, 1)]
            if not got[0]:
                continue
            k, v = (np.array([x[0] for x in side]) for side in got)
            alpha = np.array([x[1] for x in got[1]])
            for j in range(c.group):
                o = h * c.group + j
                s = float(scale) * (k @ q[r, o].astype(np.float64))
                w = np.exp(s - s.max())
                above = w if weight_bits is None else _bits(w * alpha, weight_bits) / alpha
                out[r, o] = (above @ v) / w.sum()
    return out


@pytest.mark.parametrize("case", tg.CLOSE, ids=str)
def test_close_bounds_reject_planted_mistakes(oracle, case):
    window = case[7]
    c, q, want, bound = tg.close_case(*case)
    scale = np.float32(c.dim ** -0.5)
    share = lambda **k: (np.abs(mistaken(c, q, scale, window, **k) - want) / bound).max()
    assert share() < 1e-3 and share(weight_bits=24) < 0.1                       # nothing planted; float32's own rounding
    if case[0] == "bf16":
        assert share(weight_bits=17) <= 1.0                                     # what the header allows
    assert share(weight_bits=8) > 1.0 and share(newest=1) > 1.0
    if window:
        assert share(wider=1) > 1.0 and share(wider=-1) > 1.0


@pytest.mark.parametrize("case", tg.CLOSE_PROMPTS, ids=str)
def test_close_bounds_of_prompts_reject_planted_mistakes(oracle, case):
    window = case[7]
    c, q, want, bound = tg.close_prompts_case(*case)
    share = lambda **k: (np.abs(mistaken(c, q, np.float32(c.dim ** -0.5), window, **k) - want) / bound).max()
    assert share() < 1e-3 and share(weight_bits=8) <= 1.0                       # what the header allows
    assert share(weight_bits=5) > 1.0 and share(newest=1) > 1.0
    if window:
        assert share(wider=1) > 1.0 and share(wider=-1) > 1.0


@pytest.mark.parametrize("case", tg.CLOSE_PROMPTS, ids=str)
def test_close_bounds_of_two_parts_reject_one(oracle, case):
    c, q, want, bound = tg.two_part_prompts_case(*case)
    share = lambda **k: (np.abs(mistaken(c, q, np.float32(c.dim ** -0.5), case[7], **k) - want) / bound).max()
    assert share(weight_bits=17) <= 1.0 and share(weight_bits=9) > 1.0 and share(weight_bits=8) > 1.0


@pytest.mark.parametrize("case", tg.WINDOWED, ids=str)
def test_exactness_of_float32_rejects_weights_of_16_bits(oracle, case):
    c, q, want, plain = tg.windowed_case(*case)
    scale = np.float32(c.dim ** -0.5)
    off = lambda **k: tg.exactness(mistaken(c, q, scale, case[6], **k), want, plain)
    assert off(weight_bits=24) <= 1.0 and off(weight_bits=16) > 1.0 and off(weight_bits=8) > 1.0
    assert off(wider=1) > 1.0 and off(wider=-1) > 1.0 and off(newest=1) > 1.0


def test_the_workspace_goes_by_the_step_it_is_asked_for():
    """Sizes and whether row_start is there, no addresses; a call whose workspace is for the other kind, or for a larger step that needs
    less, is refused."""
    f = b.raw().qllm_kv_attention_workspace_bytes
    sizes = dict(rows=60, n_seqs=1, n_slots=1, ld=80, table=None, length=None)
    bytes_of = lambda **k: f(C.byref(cache(heads=1, pages=None)), C.byref(batch(**{**sizes, **k})), 64)
    with_rows, without, larger = bytes_of(row_start=A), bytes_of(row_start=None), bytes_of(row_start=A, rows=500)
    assert with_rows == bytes_of(row_start=64 * A) and without > 0 and with_rows > without and with_rows > larger > 0
    call = lambda ws_bytes: attend(cache(heads=1), batch(rows=60, n_seqs=1, n_slots=1, ld=80, row_start=A), hq=64, ldq=64 * 128, ldo=64 * 128, ws_bytes=ws_bytes)
    assert call(with_rows - 1) == WORKSPACE and call(without) == WORKSPACE and call(larger) == WORKSPACE
