"""An append to an 8-bit cache that fails after its copies are under way (CPU, over the
stand-in of test_kv8_calls): the pages that it gives back are written by nothing any more."""
import numpy as np
import pytest

import paper_2602_22603_gb300 as sq
from tests.test_kv8_calls import D, HKV, HQ, STORE8, L, kv, read  # noqa: F401 (L: the fixture)


def test_pages_of_an_append_whose_rows_fail(L):  # noqa: F811
    """Forks' copies are enqueued, then the launch that writes the rows fails."""
    n = 5
    c = sq.Cache(1, HQ, HKV, D, 16, 40, bits=8)
    a = c.seq_new()
    k = kv(5, 1, 1)
    c.append_kv(a, 5, k.ctypes.data, k.ctypes.data, 1)
    forks = [c.fork_aux(a) for _ in range(n)]
    before = [c.page_table(h) for h in forks], c.free_pages(), c.next_pos(a)
    x = np.zeros((1, n, HKV, D), np.uint16)
    L.fake_new_pages()
    L.fake_fail8(STORE8)
    with pytest.raises(sq.SqError):
        c.append_kv_batch(forks, x.ctypes.data, x.ctypes.data, 1)
    assert ([c.page_table(h) for h in forks], c.free_pages(), c.next_pos(a)) == before
    # the pages go to another sequence, on another stream
    b = c.seq_new()
    k = kv(39 * 16, 2, 1)
    c.append_kv(b, 39 * 16, k.ctypes.data, k.ctypes.data, 2)
    assert L.fake_page_races() == 0
    assert read(c, b, 0) == list(k[0, :, 0, 0] % 256)
    c.close()
