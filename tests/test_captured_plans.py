"""What a captured call around a model's attention was given stays as it is for as long
as the cache lives, whatever is called between the graph's runs (CPU, over a stand-in
for the runtime); a call that would have to upload something is refused while its
stream is captured."""
import ctypes

import pytest

import paper_2602_22603_gb300 as sq
from tests.test_captured_calls import L, cache  # noqa: F401
from tests.test_operator_calls import HKV, D, HQ, LSE, OUT, Q, append, kv, store, tree, window


def backward(c, n, stream, weights=LSE):
    sq.sq_qk_norm_rope_backward(c.handle, n, Q, HQ * D, Q, HKV * D, None, sq.norm_rope(), Q, Q, OUT, HQ * D,
                                2 * OUT, HKV * D, weights, None, stream)


def large_store(c, h, layer, stream):
    k = kv(300, 3)
    sq.sq_qk_norm_rope_store(c.handle, [h], [300], layer, Q, HQ * D, k.ctypes.data, HKV * D, k.ctypes.data,
                             HKV * D, None, sq.norm_rope(), OUT, stream)


KINDS = {
    "tree": lambda c, h, s: tree(c, [h], [9], s),
    "window": lambda c, h, s: window(c, [h], [40], s),
    "token": lambda c, h, s: window(c, [h], [1], s, lse=None),
    "prefill": lambda c, h, s: c.prefill_attention(h, 0, 8, Q, OUT, sq.SQ_OUT_BF16, None, 0.1, (), s),
    "store": lambda c, h, s: large_store(c, h, 0, s),
    "backward": lambda c, h, s: backward(c, 20, s),
}


def given(L):  # noqa: F811
    out = (ctypes.c_void_p * 4)()
    L.fake_given(out)
    return list(out)


def sequences(c):
    hs = [c.seq_new() for _ in range(6)]
    for i, h in enumerate(hs):
        append(c, h, 2000 + 64 * i, 1)
        c.extend([h], [300], 1)
    return hs


@pytest.mark.parametrize("kind", [k for k in KINDS if k != "prefill"])
def test_refused_where_it_would_upload(L, cache, kind):  # noqa: F811
    h = sequences(cache)[0]
    L.fake_capture(1)
    with pytest.raises(sq.SqError) as e:
        KINDS[kind](cache, h, 1)
    assert e.value.code == sq.SQ_ERR_UNSUPPORTED
    assert L.fake_wrong() == 0 and L.fake_captured_uploads() == 0
    L.fake_capture(None)
    for _ in range(2):
        KINDS[kind](cache, h, 1)      # (what was refused left nothing behind)
    if kind != "backward":            # made on another stream: no wait for it can be captured
        L.fake_capture(2)
        with pytest.raises(sq.SqError) as e:
            KINDS[kind](cache, h, 2)
        assert e.value.code == sq.SQ_ERR_UNSUPPORTED and L.fake_wrong() == 0
        L.fake_capture(None)
    L.fake_capture(1)
    KINDS[kind](cache, h, 1)
    assert L.fake_wrong() == 0 and L.fake_captured_uploads() == 0


def test_what_needs_no_upload_is_captured(L, cache):  # noqa: F811
    h = sequences(cache)[0]
    L.fake_capture(1)
    store(cache, [h], [200], 0, 1)
    sq.sq_qk_norm_rope(cache.handle, 5, Q, HQ * D, Q, HKV * D, None, sq.norm_rope(), OUT, 2 * OUT, 1)
    backward(cache, 20, 1, None)
    assert L.fake_wrong() == 0 and L.fake_captured_uploads() == 0


@pytest.mark.parametrize("kind", list(KINDS))
def test_a_capture_keeps_its_buffers(L, cache, kind):  # noqa: F811
    hs = sequences(cache)
    for _ in range(2):
        KINDS[kind](cache, hs[0], 1)
    L.fake_capture(1)
    KINDS[kind](cache, hs[0], 1)
    L.fake_capture(None)
    mine = [p for p in given(L) if p]
    assert mine
    plan = given(L)[2 if kind == "store" else 0]
    bytes_of = lambda p: ctypes.string_at(p, 128) if p else b""  # noqa: E731
    before = bytes_of(plan if kind != "backward" else None)
    # calls of the kind on other sequences, streams and sizes
    for i in range(1, 6):
        for s in (1, 2, 3):
            KINDS[kind](cache, hs[i], s)
            tree(cache, [hs[i]], [10 + i], s)
            window(cache, [hs[i]], [1], s, w=50 + i, lse=None)
            backward(cache, 500 * i, s)
    # larger partial results than any so far
    many = cache.seq_new()
    append(cache, many, 8000, 1)
    window(cache, [many], [300], 2, w=0)
    tree(cache, hs, [30] * 6, 2)
    assert L.fake_wrong() == 0 and L.fake_races() == 0
    assert not any(L.fake_was_freed(p) for p in mine)
    assert bytes_of(plan if before else None) == before
    # and the call itself still works, on any stream
    for s in (1, 2, 3):
        KINDS[kind](cache, hs[0], s)
    assert L.fake_wrong() == 0
