"""Values of any finite size: attention of query blocks has the finite result that the
definition has also where weights times values pass what 32 bits hold on the way."""
import numpy as np
import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.budget import decode_budget
from tests.gpu_harness import assert_budget, row_slots
from tests.test_gpu_blocks import Batch

pytestmark = pytest.mark.gpu
LARGEST = 3.3895313892515355e38   # of bf16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def large_values(b, h, size):
    """Every value of sequence h times a factor that makes the largest `size`."""
    page, slot = row_slots(b.c, h)
    v = b.pool[0, page, 1, :, slot].float()
    v = (v / v.abs().max() * size).bfloat16()
    b.pool[0, page, 1, :, slot] = v
    torch.cuda.synchronize()


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 64), (16, 2, 64, 16), (4, 4, 64, 64), (6, 2, 128, 256)])
@pytest.mark.parametrize("size", [1e20, 1e28, 1e36, LARGEST])
@pytest.mark.parametrize("n,n_q,window,sharp", [
    (700, [40], 0, 1.0), (700, [300], 100, 4.0), (900, [7], 0, 8.0), (20000, [9], 0, 4.0), (3000, [64], 1000, 8.0)])
def test_finite_where_the_result_is(Hq, Hkv, D, P, size, n, n_q, window, sharp):
    b = Batch(Hq, Hkv, D, P, [n], seed=n)
    large_values(b, b.h[0], size)
    m = n_q[0]
    q = b.queries(m, sharp)
    k, v = b.rows(b.h[0])
    for parents in (None, list(range(-1, m - 1)) if m <= sq.SQ_MAX_DRAFT else None):
        out, lse = b.call(n_q, q, parents, window, 0)
        assert b.c.sync_status() == sq.SQ_OK
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        for i in sorted(set(np.linspace(0, m - 1, min(m, 8)).round().astype(int).tolist())):
            p = n - m + i
            see = torch.arange(n, device="cuda") <= p
            if window:
                see &= torch.arange(n, device="cuda") > p - window
            kk, vv = k[see], v[see] / size
            z = torch.einsum("ghd,tgd->ght", q[i].double().view(Hkv, Hq // Hkv, -1), kk) * D ** -0.5
            w = torch.softmax(z, -1)
            o = torch.einsum("ght,tgd->ghd", w, vv)
            dev = torch.stack([torch.einsum("ht,htd->hd", w[g], (vv[:, g][None] - o[g][:, None]).abs())
                               for g in range(Hkv)])
            absv = torch.einsum("ght,tgd->ghd", w, vv.abs())
            flat = lambda t: t.reshape(Hq, D).cpu().numpy()  # noqa: E731
            assert_budget((out[i].double() / size).float(), flat(o),
                          decode_budget(flat(dev), flat(absv), kk.shape[0]))
    b.c.close()


def test_one_value_for_all():
    """Equal values come back as they are, the largest of them too."""
    b = Batch(8, 2, 128, 64, [5000], seed=2)
    page, slot = row_slots(b.c, b.h[0])
    for value in (LARGEST, -LARGEST, 1e30):
        b.pool[0, page, 1, :, slot] = value
        torch.cuda.synchronize()
        out, _ = b.call([33], b.queries(33, 6.0), None, 3000, 5)
        assert b.c.sync_status() == sq.SQ_OK
        want = torch.full_like(out, value).bfloat16().float()
        assert ((out.double() - want.double()).abs() <= want.double().abs() * 2.0 ** -12).all()
    b.c.close()
