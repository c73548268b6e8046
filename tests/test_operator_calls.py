"""What the calls around a model's attention decide on the host (CPU), over a
stand-in for the CUDA runtime and the kernels: rows added and stored in place,
accepted drafts, turns of plans and workspaces over streams, what a failing call
leaves, and what a launch may read ahead of a store."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2602_22603_gb300 as sq
from paper_2602_22603_gb300 import build
from tests import fakelib

HQ, HKV, D, P = 8, 2, 128, 64
NORM, BLOCKS = 6, 7
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
        out = os.path.join(build.OUT, f"libsq_fake_ops.{os.getpid()}.so")
        here = os.path.dirname(os.path.abspath(__file__))
        subprocess.run(
            ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Bsymbolic",
             "-I" + cuda, "-I" + build.INCLUDE, "-o", out, os.path.join(here, "fake_operators.cpp"),
             os.path.join(build.CSRC, "api", "sq_api.cpp"),
             os.path.join(build.CSRC, "host", "core.cpp"), "-ldl"], check=True)
        L = ctypes.CDLL(out)
        os.remove(out)
        for name, (res, args) in sq._SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        L.fake_count.restype = L.fake_races.restype = ctypes.c_int64
        L.fake_malloc_limit.argtypes = [ctypes.c_int64]
        _lib = L
    return _lib


@pytest.fixture
def L(monkeypatch):
    monkeypatch.setattr(sq, "_lib", lib())
    lib().fake_reset()
    return lib()


@pytest.fixture
def cache(L):
    c = sq.Cache(2, HQ, HKV, D, P, 400)
    yield c
    c.close()


def kv(n, tag):
    """Rows whose elements name them: [n, HKV, D] of tag * 1000 + row."""
    return np.ascontiguousarray(np.broadcast_to((tag * 1000 + np.arange(n))[:, None, None], (n, HKV, D))
                                .astype(np.uint16))


def row_tags(c, h, layer):
    """Element 0 of each row's key, head 0, read through the page table."""
    pool = np.ctypeslib.as_array((ctypes.c_uint16 * (2 * 400 * 2 * HKV * P * D)).from_address(
        sq.sq_pool_ptr(c.handle))).reshape(2, 400, 2, HKV, P, D)
    return [int(pool[layer, pg, 0, 0, s, 0]) for pg, f in zip(c.page_table(h), c.page_fills(h))
            for s in range(f)]


def store(c, hs, counts, layer, tag, stream=1, positions=None):
    n = sum(counts)
    k = kv(n, tag)
    sq.sq_qk_norm_rope_store(c.handle, hs, counts, layer, Q, HQ * D, k.ctypes.data, HKV * D, k.ctypes.data,
                             HKV * D, positions, sq.norm_rope(), OUT, stream)


def append(c, h, n, tag, stream=1):
    k = np.stack([kv(n, tag)] * 2)
    c.append_kv(h, n, k.ctypes.data, k.ctypes.data, stream)


def tree(c, hs, counts, stream, parents=None, layer=0, **kw):
    sq.sq_tree_attention(c.handle, hs, counts, parents or [j - 1 for m in counts for j in range(m)], layer, Q,
                         OUT, stream=stream, sm_scale=0.1, **kw)


def window(c, hs, counts, stream, w=100, layer=0, lse=LSE, **kw):
    sq.sq_window_attention(c.handle, hs, counts, layer, Q, OUT, w, 4, lse=lse, sm_scale=0.1, stream=stream, **kw)


def test_rows_are_stored_where_they_belong(cache):
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 70, 1)
    append(cache, b, 3, 2)
    f = cache.fork_aux(b)
    for counts, tag in (([2, 1, 1], 3), ([300, 0, 70], 5), ([1, 1, 1], 7)):
        before = [row_tags(cache, h, 1) for h in (a, b, f)]
        other = [row_tags(cache, h, 0) for h in (a, b, f)]
        cache.extend([a, b, f], counts, 1)
        for _ in range(2):
            store(cache, [a, b, f], counts, 1, tag)
        new = iter(range(tag * 1000, tag * 1000 + sum(counts)))
        for h, old, o, m in zip((a, b, f), before, other, counts):
            assert row_tags(cache, h, 1) == old + [next(new) for _ in range(m)]
            assert row_tags(cache, h, 0)[:len(o)] == o
    assert cache.next_pos(a) == 373 and cache.seq_info(b) == (5, 1)


def test_a_failed_extension_leaves_nothing(L, cache):
    a = cache.seq_new()
    append(cache, a, 70, 1)
    f = cache.fork_aux(a)
    tables = [cache.page_table(h) for h in (a, f)]
    free = cache.free_pages()
    L.fake_fail(fakelib.APPEND_BATCH)   # (the copy of the shared page)
    with pytest.raises(sq.SqError) as e:
        cache.extend([a, f], [5, 400], 1)
    assert e.value.code == sq.SQ_ERR_CUDA
    assert [cache.page_table(h) for h in (a, f)] == tables and cache.free_pages() == free
    assert cache.seq_info(a)[0] == cache.next_pos(f) == 70
    cache.extend([a, f], [5, 400], 1)
    assert cache.seq_info(f)[0] == 470


def test_accepted_rows(cache):
    a = cache.seq_new()
    append(cache, a, 60, 1)
    cache.extend([a], [9], 1)
    for layer in (0, 1):
        store(cache, [a], [9], layer, 4)
    cache.accept_draft(a, 9, [0, 1], 1)          # a prefix: nothing moves
    assert cache.seq_info(a)[0] == cache.next_pos(a) == 62
    assert row_tags(cache, a, 1)[60:] == [4000, 4001]
    cache.extend([a], [9], 1)
    cache.accept_draft(a, 9, [], 1)
    assert cache.seq_info(a)[0] == cache.next_pos(a) == 62 and len(cache.page_table(a)) == 1
    sq.sq_evict_spans_ragged(cache.handle, a, [(3, 5)], 1)
    assert cache.seq_info(a)[0] == 60 and cache.next_pos(a) == 62
    cache.extend([a], [3], 1)
    cache.accept_draft(a, 3, [0, 1, 2], 1)
    assert cache.seq_info(a)[0] == 63 and cache.next_pos(a) == 65


def test_streams_take_turns(L, cache):
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 9000, 1)
    append(cache, b, 5000, 2)
    cache.extend([a, b], [300, 300], 1)
    for _ in range(2):
        for s in (1, 2, 3):
            store(cache, [a, b], [300, 300], 0, 1, s)
            tree(cache, [a, b], [9, 9], s)
            tree(cache, [a], [200], s)
            window(cache, [a, b], [1, 40], s)
            window(cache, [a, b], [1, 1], s, lse=None)
            window(cache, [a], [1], s, w=0)
            cache.prefill_attention(a, 0, 8, Q, OUT, sq.SQ_OUT_BF16, None, 0.1, (), s)
            sq.sq_qk_norm_rope_backward(cache.handle, 5, Q, HQ * D, Q, HKV * D, None, sq.norm_rope(),
                                        Q, Q, OUT, HQ * D, 2 * OUT, HKV * D, LSE, None, s)
    assert L.fake_races() == 0


@pytest.mark.parametrize("kind", [BLOCKS, fakelib.COMBINE, NORM])
def test_after_a_failed_launch(L, cache, kind):
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 9000, 1)
    append(cache, b, 5000, 2)
    cache.extend([a], [300], 1)

    def call(h, s):
        if kind == NORM:
            store(cache, [a], [300], 0, 1, s)
        else:
            tree(cache, [h], [9], s)

    for first in (True, False):
        L.fake_fail(kind)
        with pytest.raises(sq.SqError) as e:
            call(a, 1)
        assert e.value.code == sq.SQ_ERR_CUDA
        for s in (2, 3, 1):
            call(b, s)
            call(a, s)
    assert L.fake_races() == 0
    assert cache.seq_info(a)[0] == 9300


def test_without_room_for_partial_results(L, cache):
    a = cache.seq_new()
    append(cache, a, 9000, 1)
    L.fake_malloc_limit(1 << 20)
    tree(cache, [a], [9], 1)
    assert L.fake_count(fakelib.COMBINE) == 0 and L.fake_count(BLOCKS) == 1
    L.fake_malloc_limit(-1)
    tree(cache, [a], [10], 1)
    assert L.fake_count(fakelib.COMBINE) == 1
    L.fake_malloc_limit(1000)
    with pytest.raises(sq.SqError) as e:   # no room for the weights' partial gradients
        sq.sq_qk_norm_rope_backward(cache.handle, 100, Q, HQ * D, Q, HKV * D, None, sq.norm_rope(), Q, Q, OUT,
                                    HQ * D, 2 * OUT, HKV * D, LSE, None, 1)
    assert e.value.code == sq.SQ_ERR_NO_MEMORY


def test_a_store_is_not_read_ahead(L, cache):
    """A launch may read keys ahead of its dependency wait, but not the pages of a
    store that may still run (the stand-in's events never complete): those are
    listed, or, where they are too many or an earlier store's are not known, nothing
    is read ahead."""
    hs = [cache.seq_new() for _ in range(40)]
    for h in hs:
        cache.extend([h], [130], 1)      # (no copies: nothing written yet)
    call = lambda k=1: tree(cache, hs[:k], [4] * k, 1)  # noqa: E731
    call()
    call()
    assert L.fake_unsafe() == 0          # a plan on the device, nothing outstanding
    store(cache, hs[:1], [4], 0, 1)
    call()
    assert L.fake_unsafe() == 2          # rows 126 .. 129 lie in two pages
    store(cache, hs[:1], [4], 1, 1)
    call()
    assert L.fake_unsafe() == 2
    store(cache, hs[:2], [4, 4], 0, 1)   # other pages: the store before may still run
    call()
    assert L.fake_unsafe() == -1


def test_a_store_to_many_pages_is_not_read_ahead(L, cache):
    hs = [cache.seq_new() for _ in range(40)]
    for h in hs:
        cache.extend([h], [130], 1)
    tree(cache, hs[:1], [4], 1)
    store(cache, hs, [1] * 40, 0, 1)
    tree(cache, hs[:1], [4], 1)
    assert L.fake_unsafe() == -1


def test_calls_without_their_kernels_are_refused(monkeypatch):
    """The stand-in without these launchers links, and the calls say so."""
    monkeypatch.setattr(sq, "_lib", fakelib.lib())
    fakelib.lib().fake_reset()
    c = sq.Cache(1, HQ, HKV, D, P, 20)
    h = c.seq_new()
    c.extend([h], [5], 1)
    for f in (lambda: store(c, [h], [1], 0, 1), lambda: tree(c, [h], [2], 1), lambda: window(c, [h], [2], 1)):
        with pytest.raises(sq.SqError) as e:
            f()
        assert e.value.code == sq.SQ_ERR_UNSUPPORTED
    c.close()
