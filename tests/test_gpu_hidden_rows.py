"""Rows that a query does not see may hold infinities and NaN: windows, sinks,
drafted trees and single tokens over pages whose other rows are poisoned, against
64-bit references within the kernels' error budget."""
import math

import numpy as np
import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.budget import decode_budget
from tests.gpu_harness import assert_budget, row_slots
from tests.test_gpu_blocks import GEOMETRIES, Batch

pytestmark = pytest.mark.gpu
BAD = [math.inf, -math.inf, math.nan]


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def poison(b, h, rows):
    """Infinities and NaN in the K and V rows `rows` (indices) of sequence h."""
    rows = torch.as_tensor(rows, device="cuda", dtype=torch.long)
    page, slot = (x[rows] for x in row_slots(b.c, h))
    for i, bad in enumerate(BAD):
        b.pool[0, page[i::3], 0, :, slot[i::3]] = bad
        b.pool[0, page[i::3], 1, :, slot[i::3]] = BAD[(i + 1) % 3]


def hidden(n, m, window, sinks):
    """Rows of a sequence of n that none of its newest m queries sees."""
    low = n - m - window + 1 if window else 0
    return [j for j in range(n) if j < low and j >= sinks]


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (70, 65), (200, 3)])
def test_single_tokens(Hq, Hkv, D, P, window, sinks):
    b = Batch(Hq, Hkv, D, P, [1, 63, 64, 65, 129, 700], seed=window + P)
    for h, n in zip(b.h, [1, 63, 64, 65, 129, 700]):
        poison(b, h, hidden(n, 1, window, sinks))
    q, out, _ = b.check(None, window=window, sinks=sinks)
    # (the decode kernel, without log-sum-exps: within both kernels' budgets)
    got = torch.full_like(out, float("nan"))
    b.c.window_attention(b.h, None, 0, q, got, window, sinks, out_dtype=sq.SQ_OUT_F32, sm_scale=D ** -0.5)
    assert b.c.sync_status() == sq.SQ_OK
    for i, h in enumerate(b.h):
        k, v = b.rows(h)
        n = k.shape[0]
        see = [j for j in range(n) if j > n - 1 - window or j < sinks]
        assert_rows(got[i], q[i], k[see], v[see], Hq, Hkv, D)
    b.c.close()


def assert_rows(got, q, k, v, Hq, Hkv, D):
    """One query's output over the rows k, v that it sees."""
    G = Hq // Hkv
    z = torch.einsum("ghd,tgd->ght", q.double().view(Hkv, G, -1), k) * D ** -0.5
    w = torch.softmax(z, -1)
    o = torch.einsum("ght,tgd->ghd", w, v)
    dev = torch.stack([torch.einsum("ht,htd->hd", w[g], (v[:, g][None] - o[g][:, None]).abs()) for g in range(Hkv)])
    flat = lambda t: t.reshape(Hq, D).cpu().numpy()  # noqa: E731
    absv = torch.einsum("ght,tgd->ghd", w, v.abs())
    assert_budget(got, flat(o), decode_budget(flat(dev), flat(absv), k.shape[0]))


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(3, 2), (64, 0), (100, 70)])
@pytest.mark.parametrize("f32", [True, False])
def test_prompts_and_tokens(Hq, Hkv, D, P, window, sinks, f32):
    lengths, n_q = [300, 65, 900, 700, 1], [40, 65, 1, 300, 1]
    b = Batch(Hq, Hkv, D, P, lengths, seed=window)
    for h, n, m in zip(b.h, lengths, n_q):
        poison(b, h, hidden(n, m, window, sinks))
    b.check(n_q, window=window, sinks=sinks, f32=f32)
    b.c.close()


def test_pieces_of_a_long_context():
    """Key ranges cut into pieces: a piece in which a row sees nothing as well."""
    b = Batch(8, 2, 128, 64, [20000, 9000], seed=3)
    for h, n, m in zip(b.h, [20000, 9000], [200, 3]):
        poison(b, h, hidden(n, m, 5000, 130))
    b.check([200, 3], window=5000, sinks=130)
    b.c.close()


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,m", [(0, 40), (9, 40), (0, 200)])
def test_a_drafted_token_that_is_not_finite(Hq, Hkv, D, P, window, m):
    """What a draft's infinities touch: itself and its descendants, no other."""
    rng = np.random.RandomState(m + window)
    n, sinks = 333, 2
    b = Batch(Hq, Hkv, D, P, [n], seed=m)
    parents = [int(rng.randint(-1, i)) if i else -1 for i in range(m)]
    anc = []
    for i, p in enumerate(parents):
        anc.append((anc[p] if p >= 0 else []) + [i])
    bad = {m // 3, m // 2, m - 1}
    poison(b, b.h[0], [n - m + i for i in sorted(bad)])
    q = b.queries(m)
    out, _ = b.call([m], q, parents, window, sinks)
    assert b.c.sync_status() == sq.SQ_OK
    k, v = b.rows(b.h[0])
    place = list(range(n - m)) + [n - m + len(a) - 1 for a in anc]
    touched = 0
    for i in range(m):
        see = [j for j in list(range(n - m)) + [n - m + a for a in anc[i]]
               if not window or place[j] > place[n - m + i] - window or place[j] < sinks]
        if bad & {j - n + m for j in see}:
            touched += 1
            continue
        assert_rows(out[i], q[i], k[see], v[see], Hq, Hkv, D)
    assert 3 <= touched < m
    b.c.close()


@pytest.mark.parametrize("P,D", [(8, 64), (64, 128)])
def test_rows_evicted_from_partial_pages(P, D):
    """Hidden slots of pages that a ragged eviction left partial."""
    b = Batch(8, 2, D, P, [700], seed=P)
    h = b.h[0]
    poison(b, h, list(range(100, 131)) + list(range(400, 403)))
    b.c.evict_spans_ragged(h, [(100, 131), (400, 403)])
    torch.cuda.synchronize()
    b.check([30], window=0)
    b.check([30], window=350, sinks=101)
    q, out, _ = b.check(None, window=0)
    got = torch.full_like(out, float("nan"))
    b.c.window_attention(b.h, None, 0, q, got, 0, 0, out_dtype=sq.SQ_OUT_F32, sm_scale=D ** -0.5)
    b.c.decode_attention(b.h, 0, q, out, sq.SQ_OUT_F32, D ** -0.5)
    assert b.c.sync_status() == sq.SQ_OK
    k, v = b.rows(h)
    for o in (got, out):
        assert_rows(o[0], q[0], k, v, 8, 2, D)
    b.c.close()


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 64), (16, 2, 64, 16)])
@pytest.mark.parametrize("m", [20, 200])
def test_what_a_query_sees_is_not_hidden(Hq, Hkv, D, P, m):
    """Values that are not finite reach the queries that see them, and those alone,
    also where hidden ones lie beside them."""
    n, window, sinks = 3000, 100, 3
    b = Batch(Hq, Hkv, D, P, [n], seed=m)
    q = b.queries(m)
    q[m - 1, 1] = math.nan
    seen = n - m // 2                       # a row that the queries from it on see
    page, slot = (t[seen] for t in row_slots(b.c, b.h[0]))
    b.pool[0, page, 1, :, slot, 5] = math.inf     # one column of V
    poison(b, b.h[0], [n - m - 90])         # hidden from all but the first queries
    out, _ = b.call([m], q, None, window, sinks)
    assert b.c.sync_status() == sq.SQ_OK
    k, v = b.rows(b.h[0])
    for i in range(m):
        p = n - m + i
        see = [j for j in range(p + 1) if j > p - window or j < sinks]
        if n - m - 90 in see:
            assert not torch.isfinite(out[i]).any()
            continue
        ok = torch.isfinite(out[i])
        want = torch.ones_like(ok)
        want[:, 5] = seen not in see
        if i == m - 1:
            want[1] = False
        assert torch.equal(ok, want)
        if i != m - 1 and seen not in see:
            assert_rows(out[i], q[i], k[see], v[see], Hq, Hkv, D)
    b.c.close()


@pytest.mark.parametrize("n", [50, 700, 9000])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("m", [1, 4, 100])
def test_nan_is_not_lost(n, what, m):
    """NaN in a query, or in a key or value that it sees, is NaN in its output, also
    where the keys are cut into pieces; a NaN weight in its log-sum-exp too."""
    b = Batch(8, 2, 128, 64, [n + m], seed=n)
    q = b.queries(m)
    if what == "q":
        q[:, 1] = math.nan
    else:
        page, slot = (t[n // 2] for t in row_slots(b.c, b.h[0]))
        b.pool[0, page, 0 if what == "k" else 1, :, slot] = math.nan
    out, lse = b.call([m], q)
    assert b.c.sync_status() == sq.SQ_OK
    nan = torch.zeros(m, 8, dtype=torch.bool, device="cuda")
    nan[:, 1 if what == "q" else slice(None)] = True
    assert torch.equal(torch.isnan(out), nan[:, :, None].expand_as(out))
    assert torch.equal(torch.isnan(lse), nan & (what != "v"))
    got = torch.zeros_like(out)
    b.c.tree_attention(b.h, [m], list(range(-1, m - 1)), 0, q, got, out_dtype=sq.SQ_OUT_F32, sm_scale=0.1)
    assert torch.equal(torch.isnan(got), nan[:, :, None].expand_as(out))
    b.c.close()
