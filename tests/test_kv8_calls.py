"""What an 8-bit cache's calls decide on the host (CPU), over a stand-in for the CUDA
runtime and the kernels: where rows go, what failing calls leave, refusals, and
the turns of plans and workspaces over streams."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2602_22603_gb300 as sq
from paper_2602_22603_gb300 import build

HQ, HKV, D, P, PAGES = 8, 2, 64, 16, 200
STORE8, COPY8, READ8, WIDEN8, EVICT8 = range(5)
BLOCKS = 7
Q, OUT, LSE = 1 << 20, 1 << 30, 1 << 32   # never read or written by the stand-in
_lib = None


def lib():
    global _lib
    if _lib is None:
        nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
        cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
        if not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
            cuda = "/usr/local/cuda/include"
        os.makedirs(build.OUT, exist_ok=True)
        out = os.path.join(build.OUT, f"libsq_fake_kv8.{os.getpid()}.so")
        here = os.path.dirname(os.path.abspath(__file__))
        subprocess.run(
            ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Bsymbolic",
             "-I" + cuda, "-I" + build.INCLUDE, "-o", out, os.path.join(here, "fake_kv8.cpp"),
             os.path.join(build.CSRC, "api", "sq_api.cpp"),
             os.path.join(build.CSRC, "host", "core.cpp"), "-ldl"], check=True)
        L = ctypes.CDLL(out)
        os.remove(out)
        for name, (res, args) in sq._SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        L.fake_count.restype = L.fake_races.restype = L.fake_bad.restype = L.fake_page_races.restype = ctypes.c_int64
        L.fake_malloc_limit.argtypes = [ctypes.c_int64]
        _lib = L
    return _lib


@pytest.fixture
def L(monkeypatch):
    monkeypatch.setattr(sq, "_lib", lib())
    lib().fake_reset()
    lib().fake_fail8(-1)
    lib().fake_new_pages()
    yield lib()
    assert lib().fake_bad() == 0


@pytest.fixture(params=[8, 16, 64, 256])
def cache(L, request):
    c = sq.Cache(2, HQ, HKV, D, request.param, PAGES, bits=8)
    yield c
    c.close()


def kv(n, tag, layers=2):
    """Rows whose elements name them (in the low byte): [layers, n, HKV, D]."""
    x = (tag + np.arange(n)) % 256 + 256 * 65
    return np.ascontiguousarray(np.broadcast_to(x[None, :, None, None], (layers, n, HKV, D)).astype(np.uint16))


def append(c, h, n, tag, stream=1):
    k = kv(n, tag)
    c.append_kv(h, n, k.ctypes.data, k.ctypes.data, stream)
    return list(k[0, :, 0, 0] % 256)


def read(c, h, layer=1, n=None):
    n = c.seq_info(h)[0] if n is None else n
    k, v = (np.zeros((n, HKV, D), np.uint16) for _ in range(2))
    sq.sq_read_kv(c.handle, [h], [n], layer, k.ctypes.data, v.ctypes.data, 1)
    assert (k == k[:, :1, :1]).all() and (k == v).all()
    return list(k[:, 0, 0])


def scales(c, h, layer=1):
    """Scale of every block of the sequence's pages (key, head 1)."""
    codes = 2 * PAGES * 2 * HKV * c.P * D
    s = np.ctypeslib.as_array((ctypes.c_float * (codes // D // 8)).from_address(
        sq.sq_pool_ptr(c.handle) + codes)).reshape(2, PAGES, 2, HKV, c.P // 8)
    return [int(x) for p, f in zip(c.page_table(h), c.page_fills(h)) for x in s[layer, p, 0, 1, :-(-f // 8)]]


def store(c, hs, counts, layer, tag, stream=1, positions=None, params=None):
    k = kv(sum(counts), tag, 1)
    sq.sq_qk_norm_rope_store(c.handle, hs, counts, layer, Q, HQ * D, k.ctypes.data, HKV * D, k.ctypes.data,
                             HKV * D, positions, params or sq.norm_rope(), OUT, stream)
    return list(k[0, :, 0, 0] % 256)


def test_pool_bytes():
    cfg = sq.make_config(3, 8, 2, 128, 64, 100)
    with pytest.MonkeyPatch.context() as m:
        m.setattr(sq, "_lib", lib())
        assert sq.sq_pool_bytes_8bit(cfg) == 3 * 100 * 2 * 2 * (64 * 128 + 64 // 8 * 4)
        assert sq.sq_pool_bytes_8bit(sq.make_config(1, 8, 2, 96, 16, 10)) == 0


def test_appended_rows_lie_where_they_belong(cache):
    a, b = cache.seq_new(), cache.seq_new()
    ta = append(cache, a, 13, 1)
    tb = append(cache, b, 3, 100)
    f = cache.fork_aux(b)
    tf = list(tb)
    for i in range(20):
        k = kv(3, 7 * i)
        cache.append_kv_batch([a, b, f], k.ctypes.data, k.ctypes.data, 1)
        for t, x in zip((ta, tb, tf), k[0, :, 0, 0]):
            t.append(x % 256)
    ta += append(cache, a, 300, 50)
    for h, t in ((a, ta), (b, tb), (f, tf)):
        for layer in range(2):
            assert read(cache, h, layer) == t
            assert read(cache, h, layer, 5) == t[-5:]
            # each block's scale was written with its last row
            n, want = len(t), []
            for fill in cache.page_fills(h):
                want += [min(8, fill - at) for at in range(0, fill, 8)]
            assert scales(cache, h, layer) == want


def test_stored_rows_lie_where_they_belong(cache):
    a, b = cache.seq_new(), cache.seq_new()
    ta, tb = append(cache, a, 70, 1), append(cache, b, 3, 2)
    f = cache.fork_aux(b)
    tf = list(tb)
    for counts, tag in (([2, 1, 1], 3), ([300, 0, 70], 5), ([1, 1, 1], 7)):
        cache.extend([a, b, f], counts, 1)
        for _ in range(2):
            new = store(cache, [a, b, f], counts, 1, tag)
        at = 0
        for t, m in zip((ta, tb, tf), counts):
            t += new[at:at + m]
            at += m
        assert [read(cache, h) for h in (a, b, f)] == [ta, tb, tf]
    cache.evict_spans_ragged(a, [(5, 9), (100, 140)], 1)
    ta = ta[:5] + ta[9:100] + ta[140:]
    assert read(cache, a) == ta
    cache.extend([a], [9], 1)
    ta += store(cache, [a], [9], 1, 200)
    assert read(cache, a) == ta
    cache.evict_spans(a, [(0, 3), (33, 34)], 1)
    assert read(cache, a) == ta[3:33] + ta[34:]


def test_failed_appends_leave_nothing(L, cache):
    a = cache.seq_new()
    t = append(cache, a, 21, 1)
    f = cache.fork_aux(a)
    before = [cache.page_table(h) for h in (a, f)], cache.free_pages(), cache.next_pos(a)
    for kind in (STORE8, COPY8):
        L.fake_fail8(kind)
        if kind == COPY8 and cache.page_fills(a)[-1] == cache.P:
            continue
        with pytest.raises(sq.SqError):
            append(cache, a, 300, 9)
        assert ([cache.page_table(h) for h in (a, f)], cache.free_pages(), cache.next_pos(a)) == before
    with pytest.raises(sq.SqError) as e:
        append(cache, a, PAGES * cache.P, 9)
    assert e.value.code == sq.SQ_ERR_CAPACITY   # (of one sequence)
    assert read(cache, a) == t
    L.fake_fail8(EVICT8)
    with pytest.raises(sq.SqError):
        cache.evict_spans(a, [(0, 1)], 1)
    assert ([cache.page_table(h) for h in (a, f)], cache.free_pages(), cache.next_pos(a)) == before
    append(cache, a, 90, 1)
    for m, fail in ((3, lambda: L.fake_fail(BLOCKS)), (100, lambda: L.fake_fail(BLOCKS)),
                    (100, lambda: L.fake_fail8(WIDEN8))):
        fail()
        with pytest.raises(sq.SqError):
            sq.sq_window_attention(cache.handle, [a], [m], 0, Q, OUT, 0, sm_scale=0.1, stream=1)
        sq.sq_window_attention(cache.handle, [a], [m], 0, Q, OUT, 0, sm_scale=0.1, stream=1)


def test_blocks_of_many_tiles_widen_the_pages_that_they_see(L, cache):
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 1000, 1)
    append(cache, b, 40, 2)
    rows = 3 * 128 // (HQ // HKV)   # queries of three tiles
    for n in (rows // 3, rows // 3 + 1, rows):
        sq.sq_window_attention(cache.handle, [a, b], [n, 3], 0, Q, OUT, 0, sm_scale=0.1, stream=1)
        assert L.fake_wide() == 0
    sq.sq_window_attention(cache.handle, [a, b], [rows + 1, 3], 0, Q, OUT, 0, sm_scale=0.1, stream=1)
    assert L.fake_wide() == sum(cache.seq_info(h)[1] for h in (a, b))
    # (whole 64-row boxes of the window's, and the sinks')
    sq.sq_window_attention(cache.handle, [a], [rows + 1], 0, Q, OUT, 20, 2, sm_scale=0.1, stream=1)
    seen = 64 + 1000 - (1000 - rows - 1 - 19) // 64 * 64
    assert 0 < L.fake_wide() <= -(-seen // cache.P) + 2


def test_query_blocks_take_turns_over_streams(L, cache):
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 300, 1)
    append(cache, b, 900, 2)
    for s in (1, 2, 3, 1, 2):
        for h in (a, b):
            sq.sq_window_attention(cache.handle, [h], [100], 0, Q, OUT, 0, sm_scale=0.1, stream=s)
        sq.sq_tree_attention(cache.handle, [a, b], [2, 2], [-1, 0, -1, 0], 0, Q, OUT, sm_scale=0.1, stream=s)
    assert L.fake_races() == 0


def test_no_room_for_widened_pages(L):
    c = sq.Cache(1, HQ, HKV, D, 64, PAGES, bits=8)
    a = c.seq_new()
    k = kv(5000, 1, 1)
    c.append_kv(a, 5000, k.ctypes.data, k.ctypes.data, 1)
    L.fake_malloc_limit(1 << 20)
    with pytest.raises(sq.SqError) as e:
        sq.sq_window_attention(c.handle, [a], [100], 0, Q, OUT, 0, sm_scale=0.1, stream=1)
    assert e.value.code == sq.SQ_ERR_NO_MEMORY
    sq.sq_decode_attention(c.handle, [a], 0, Q, OUT, sm_scale=0.1, stream=1)
    L.fake_malloc_limit(-1)
    sq.sq_window_attention(c.handle, [a], [100], 0, Q, OUT, 0, sm_scale=0.1, stream=1)
    c.close()


def test_refusals(L, cache):
    a = cache.seq_new()
    append(cache, a, 30, 1)
    f = cache.fork_aux(a)
    b = cache.seq_new()

    def code(call, *args, **kw):
        with pytest.raises(sq.SqError) as e:
            call(cache.handle, *args, **kw)
        return e.value.code

    bad, unsupported = sq.SQ_ERR_INVALID_ARG, sq.SQ_ERR_UNSUPPORTED
    assert code(sq.sq_prefill_attention, a, 0, 3, Q, OUT, stream=1) == unsupported
    # rows of a shared page are not stored over
    assert code(sq.sq_qk_norm_rope_store, [a], [1], 0, Q, HQ * D, Q, HKV * D, Q, HKV * D, None, sq.norm_rope(),
                OUT, 1) == bad
    cache.extend([b], [4], 1)
    ok = ([b], [4], 0, Q, HQ * D, Q, HKV * D, Q, HKV * D, None, sq.norm_rope(), OUT, 1)
    for i, x in ((0, [b, b]), (1, [5]), (1, [-1]), (2, 2), (3, Q + 8), (4, HQ * D + 4), (5, 0), (6, HKV * D - 8),
                 (7, Q + 2), (11, Q)):
        args = list(ok)
        args[i] = x
        assert code(sq.sq_qk_norm_rope_store, *args) == bad
    pool = sq.sq_pool_ptr(cache.handle)
    for args in (([a], [31], 0, Q, OUT), ([a], [-1], 0, Q, OUT), ([a, a], None, 0, Q, OUT), ([a], None, 2, Q, OUT),
                 ([a], None, 0, None, OUT), ([a], None, 0, Q, OUT + 4), ([a], None, 0, Q, Q),
                 ([a], None, 0, pool + 16, OUT), ([a], [30], 0, Q, Q + 512)):
        assert code(sq.sq_read_kv, *args, 1) == bad
    assert code(sq.sq_read_kv, [a + (1 << 25)], None, 0, Q, OUT, 1) == sq.SQ_ERR_BAD_HANDLE
    with pytest.raises(ValueError):
        sq.Cache(1, HQ, HKV, D, 16, 10, bits=4)
    assert f != a


def test_rows_of_a_bf16_cache_are_read_as_they_are(L):
    c = sq.Cache(2, HQ, HKV, D, 16, PAGES)
    a = c.seq_new()
    k = kv(50, 3)
    c.append_kv(a, 50, k.ctypes.data, k.ctypes.data, 1)
    out = np.zeros((50, HKV, D), np.uint16), np.zeros((50, HKV, D), np.uint16)
    sq.sq_read_kv(c.handle, [a], [50], 1, out[0].ctypes.data, out[1].ctypes.data, 1)
    assert (out[0] == k[1]).all() and (out[1] == k[1]).all()
    c.close()


def decode(c, hs, stream=1):
    sq.sq_decode_attention(c.handle, hs, 0, Q, OUT, sm_scale=0.1, stream=stream)


def test_rows_that_an_append_writes_are_not_read_ahead_of_it(L):
    """The next token's call on a kept plan, its last page written by an append alone."""
    c = sq.Cache(2, HQ, HKV, D, 64, PAGES, bits=8)
    a = c.seq_new()
    append(c, a, 100, 1)
    first, last = c.page_table(a)
    L.fake_done(1)
    decode(c, [a])
    decode(c, [a])
    assert L.fake_early(first) and L.fake_early(last)
    L.fake_done(0)
    plans = c.stats()["decode_plans_built"]
    for m in (1, 2):
        append(c, a, m, 2)
        decode(c, [a])
        assert c.stats()["decode_plans_built"] == plans
        assert L.fake_early(first) and not L.fake_early(last)
    c.extend([a], [1], 1)
    store(c, [a], [1], 0, 3)
    decode(c, [a])
    assert not L.fake_early(last)
    c.close()


def test_failed_appends_leave_no_plan_with_their_rows(L):
    c = sq.Cache(2, HQ, HKV, D, 64, PAGES, bits=8)
    a = c.seq_new()
    append(c, a, 100, 1)
    for kind in (STORE8, COPY8):
        decode(c, [a])
        decode(c, [a])
        L.fake_fail8(kind)
        with pytest.raises(sq.SqError):
            append(c, a, 1, 2)
        decode(c, [a])
        assert L.fake_rows() == 100
    append(c, a, 1, 2)
    decode(c, [a])
    assert L.fake_rows() == 101
    c.close()


def test_captured_calls_of_many_rows_are_refused(L, cache):
    a = cache.seq_new()
    append(cache, a, 20, 1)
    f = cache.fork_aux(a)
    before = [cache.page_table(h) for h in (a, f)], cache.free_pages(), cache.next_pos(a)
    L.fake_graph(1)
    try:
        x = np.zeros((2, 3, HKV, D), np.uint16)
        for call in (lambda: append(cache, a, 3, 5),
                     lambda: cache.append_kv_batch([a, f], x.ctypes.data, x.ctypes.data, 1)):
            with pytest.raises(sq.SqError) as e:
                call()
            assert e.value.code == sq.SQ_ERR_UNSUPPORTED
    finally:
        L.fake_graph(0)
    assert ([cache.page_table(h) for h in (a, f)], cache.free_pages(), cache.next_pos(a)) == before
    n = 237 * min(cache.P, 64)
    if n > PAGES * cache.P // 2:
        return
    b = cache.seq_new()
    append(cache, b, n, 1)
    L.fake_graph(1)
    try:
        with pytest.raises(sq.SqError) as e:
            read(cache, b)
        assert e.value.code == sq.SQ_ERR_UNSUPPORTED
    finally:
        L.fake_graph(0)


@pytest.mark.parametrize("end", ["release", "append", "extend", "evict", "evict_copy", "two"])
@pytest.mark.parametrize("write", ["append", "store", "evict"])
def test_a_block_of_rows_changes_scale_after_its_readers(L, end, write):
    """A fork on another stream reads a page and gives it up; what its parent then writes
    there, rows of the fork's among those that may be scaled anew, waits for that."""
    c = sq.Cache(2, HQ, HKV, D, 64, PAGES, bits=8)
    a = c.seq_new()
    append(c, a, 100, 1)
    page = c.page_table(a)[1]
    f = c.fork_aux(a)
    g = c.fork_aux(a) if end == "two" else None
    L.fake_new_pages()
    decode(c, [f], 2)
    if end == "release":
        c.release(f, 2)
    elif end == "append":
        append(c, f, 1, 2, 2)
    elif end == "extend":
        c.extend([f], [1], 2)
    elif end == "evict":
        c.evict_spans(f, [(60, 100)], 2)
    elif end == "evict_copy":
        c.evict_spans_ragged(f, [(80, 90)], 2)
    else:
        decode(c, [g], 3)
        c.release(g, 3)
        c.release(f, 2)
    if write == "append":
        append(c, a, 1, 2, 1)
    elif write == "store":
        c.extend([a], [1], 4)
        L.fake_new_pages()
        f = c.fork_aux(a)
        decode(c, [f], 2)
        c.release(f, 2)
        store(c, [a], [1], 0, 3, 1)
    else:
        c.evict_spans_ragged(a, [(70, 71)], 1)
    assert c.page_table(a)[1] == page and L.fake_page_races() == 0
    c.close()


def test_stores_of_the_same_rows_share_an_event(L):
    """Layer after layer: nothing reads their pages ahead until the last store is done,
    other pages stay readable, and other writes between have events of their own."""
    c = sq.Cache(2, HQ, HKV, D, 64, PAGES, bits=8)
    a, b = c.seq_new(), c.seq_new()
    append(c, a, 100, 1)
    append(c, b, 10, 1)
    first, last = c.page_table(a)
    L.fake_done(1)
    c.extend([a], [1], 1)
    store(c, [a], [1], 0, 3)
    decode(c, [a])
    decode(c, [a])
    assert L.fake_early(first) and L.fake_early(last)
    L.fake_done(0)
    for i in range(5):
        store(c, [a], [1], i % 2, 3)
        decode(c, [a])
        assert L.fake_early(first) and not L.fake_early(last)
    store(c, [a], [1], 0, 3, stream=2)
    append(c, b, 1, 4)
    store(c, [a], [1], 1, 3)
    decode(c, [a])
    assert L.fake_early(first) and not L.fake_early(last)
    store(c, [b], [1], 0, 3)   # (the stores before it are not listed page by page)
    decode(c, [a])
    assert not L.fake_early(first) and not L.fake_early(last)
    L.fake_done(1)
    decode(c, [a])
    assert L.fake_early(first) and L.fake_early(last)
    L.fake_done(0)
    c.close()
