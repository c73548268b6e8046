"""Masked prefill loses no NaN: one in a query, or in a key or value that it sees, is
in its output, also where the keys are cut into pieces whose results are merged."""
import math

import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.gpu_harness import row_slots
from tests.test_gpu_blocks import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("P,D", [(64, 128), (16, 64)])
@pytest.mark.parametrize("n", [50, 700, 9000, 40000])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("m", [1, 4, 100])
def test_nan_is_not_lost(P, D, n, what, m):
    b = Batch(8, 2, D, P, [n + m], seed=n)
    q = b.queries(m)
    if what == "q":
        q[:, 1] = math.nan
    else:
        page, slot = (t[n // 2] for t in row_slots(b.c, b.h[0]))
        b.pool[0, page, 0 if what == "k" else 1, :, slot] = math.nan
    torch.cuda.synchronize()
    out = torch.zeros(q.shape, device="cuda")
    lse = torch.zeros(q.shape[:2], device="cuda")
    b.c.prefill_attention(b.h[0], 0, m, q, out, sq.SQ_OUT_F32, lse, D ** -0.5, [])
    assert b.c.sync_status() == sq.SQ_OK
    nan = torch.zeros(m, 8, dtype=torch.bool, device="cuda")
    nan[:, 1 if what == "q" else slice(None)] = True
    assert torch.equal(torch.isnan(out), nan[:, :, None].expand_as(out))
    assert torch.equal(torch.isnan(lse), nan & (what != "v"))
    b.c.close()


def test_a_row_without_keys_is_zero():
    """A span over all that a query sees: no NaN, zero and minus infinity."""
    b = Batch(8, 2, 128, 64, [400], seed=1)
    q = b.queries(40)
    out = torch.full(q.shape, float("nan"), device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    b.c.prefill_attention(b.h[0], 0, 40, q, out, sq.SQ_OUT_F32, lse, 0.1, [(0, 380)])
    assert b.c.sync_status() == sq.SQ_OK
    assert (out[:20] == 0).all() and torch.isinf(lse[:20]).all() and (lse[:20] < 0).all()
    assert torch.isfinite(out).all() and torch.isfinite(lse[20:]).all()
    b.c.close()
