"""Calls around a model's attention on a stream that is being captured (CPU, over a
stand-in for the runtime): a captured store leaves no event that cannot be asked, and
nothing is asked during a capture."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2602_22603_gb300 as sq
from paper_2602_22603_gb300 import build
from tests.test_operator_calls import D, HKV, HQ, LSE, OUT, P, Q, append, store, tree, window

_lib = None


def lib():
    global _lib
    if _lib is None:
        nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
        cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
        if not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
            cuda = "/usr/local/cuda/include"
        os.makedirs(build.OUT, exist_ok=True)
        out = os.path.join(build.OUT, f"libsq_fake_capture.{os.getpid()}.so")
        here = os.path.dirname(os.path.abspath(__file__))
        subprocess.run(
            ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Bsymbolic",
             "-I" + cuda, "-I" + build.INCLUDE, "-o", out, os.path.join(here, "fake_capture.cpp"),
             os.path.join(build.CSRC, "api", "sq_api.cpp"),
             os.path.join(build.CSRC, "host", "core.cpp"), "-ldl"], check=True)
        L = ctypes.CDLL(out)
        os.remove(out)
        for name, (res, args) in sq._SIGS.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        for name in ("fake_count", "fake_races", "fake_wrong", "fake_captured_uploads"):
            getattr(L, name).restype = ctypes.c_int64
        L.fake_capture.argtypes = L.fake_was_freed.argtypes = [ctypes.c_void_p]
        L.fake_malloc_limit.argtypes = [ctypes.c_int64]
        _lib = L
    return _lib


@pytest.fixture
def L(monkeypatch):
    monkeypatch.setattr(sq, "_lib", lib())
    lib().fake_reset()
    lib().fake_capture_reset()
    return lib()


@pytest.fixture
def cache(L):
    c = sq.Cache(2, HQ, HKV, D, P, 400)
    yield c
    L.fake_capture(None)
    c.close()


def decode_early(c, h, stream):
    before = c.stats()["decode_early_calls"]
    c.decode_attention([h], 0, Q, OUT, sq.SQ_OUT_BF16, 0.1, stream)
    return c.stats()["decode_early_calls"] > before


def test_eager_stores_keep_early_loads(L, cache):
    a = cache.seq_new()
    append(cache, a, 9000, 1)
    cache.extend([a], [4], 1)
    for i in range(100):
        store(cache, [a], [4], i % 2, 1)
    tree(cache, [a], [4], 1)
    tree(cache, [a], [4], 1)
    assert L.fake_unsafe() == 0 and L.fake_wrong() == 0


def test_a_captured_store(L, cache):
    """The stores of a capture run whenever it is replayed: no launch reads ahead of
    its dependency wait from then on, and the events of eager writes still work."""
    a = cache.seq_new()
    append(cache, a, 9000, 1)
    cache.extend([a], [4], 1)
    store(cache, [a], [4], 0, 1)
    for _ in range(2):
        tree(cache, [a], [4], 1)
        decode_early(cache, a, 1)
    for i in range(40):        # (many writes that nobody has asked about)
        store(cache, [a], [4], i % 2, 1)
    L.fake_capture(1)
    for i in range(40):
        store(cache, [a], [4], i % 2, 2)
        cache.decode_attention([a], 0, Q, OUT, sq.SQ_OUT_BF16, 0.1, 1)
    L.fake_capture(None)
    assert L.fake_wrong() == 0
    for i in range(40):
        store(cache, [a], [4], i % 2, 3)
        tree(cache, [a], [4], 1)
        assert L.fake_unsafe() == -1
        assert not decode_early(cache, a, 1)
    assert L.fake_wrong() == 0


def test_captured_attention_of_windows(L, cache):
    """Single tokens of a window take the decode kernel: its plan is not read ahead of
    work that a replay may follow."""
    a = cache.seq_new()
    append(cache, a, 9000, 1)
    for _ in range(2):
        window(cache, [a], [1], 1, lse=None)
    append(cache, a, 1, 1)
    window(cache, [a], [1], 1, lse=None)
    early = cache.stats()["decode_early_calls"]
    L.fake_capture(1)
    window(cache, [a], [1], 1, lse=None)
    L.fake_capture(None)
    assert cache.stats()["decode_early_calls"] == early and L.fake_wrong() == 0
    window(cache, [a], [1], 1, lse=None)
    assert cache.stats()["decode_early_calls"] == early + 1
