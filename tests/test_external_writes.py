"""Rows that sq_extend added and the caller writes itself, through the address that
sq_pool_ptr gives (CPU, over the stand-in): the library does not see such a write, so
no launch may read those sequences' keys ahead of its dependency wait."""
import pytest

import paper_2602_22603_gb300 as sq
from tests.test_operator_calls import LSE, OUT, Q, append, cache, lib, store, tree, window  # noqa: F401
from tests.test_operator_calls import L  # noqa: F401


def decode_early(c, hs):
    """Whether a decode call whose plan is kept may read ahead."""
    c.decode_attention(hs, 0, Q, OUT, sq.SQ_OUT_BF16, 0.1, 1)
    before = c.stats()["decode_early_calls"]
    c.decode_attention(hs, 0, Q, OUT, sq.SQ_OUT_BF16, 0.1, 1)
    return c.stats()["decode_early_calls"] > before


@pytest.mark.parametrize("first", ["address", "rows"])
def test_query_blocks(L, cache, first):  # noqa: F811
    a = cache.seq_new()
    if first == "address":
        sq.sq_pool_ptr(cache.handle)
    cache.extend([a], [130], 1)
    if first == "rows":
        sq.sq_pool_ptr(cache.handle)
    for call in (lambda: tree(cache, [a], [4], 1), lambda: window(cache, [a], [4], 1)):
        for _ in range(3):
            call()
            assert L.fake_unsafe() == -1
    store(cache, [a], [4], 0, 1)     # (the other layer is still the caller's)
    tree(cache, [a], [4], 1)
    assert L.fake_unsafe() == -1


def test_single_tokens(L, cache):  # noqa: F811
    a, b = cache.seq_new(), cache.seq_new()
    append(cache, a, 130, 1)
    append(cache, b, 130, 2)
    sq.sq_pool_ptr(cache.handle)
    assert decode_early(cache, [a]) and decode_early(cache, [a, b])
    cache.extend([b], [1], 1)
    f = cache.fork_aux(b)
    assert not decode_early(cache, [b]) and not decode_early(cache, [a, b])
    assert not decode_early(cache, [f])
    assert decode_early(cache, [a])   # (appended rows are the library's writes)
    append(cache, b, 1, 3)            # the rows before it are the caller's still
    assert not decode_early(cache, [b])


def test_without_the_address_nothing_changes(L, cache):  # noqa: F811
    a = cache.seq_new()
    cache.extend([a], [130], 1)
    assert decode_early(cache, [a])
    for _ in range(2):
        tree(cache, [a], [4], 1)
    assert L.fake_unsafe() == 0
