"""Infinities and NaN in a row of the norms with rotation: they reach the elements that
the formulas take them to and no others (an infinity's own element, or its pair, is NaN
since the row's scale is 0; the row's others are 0)."""
import math

import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.test_gpu_norm_rope import inputs, turn

pytestmark = pytest.mark.gpu
CASES = [(128, 0, False), (128, 48, False), (128, 64, True), (64, 16, False), (64, 0, True), (64, 64, False)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("D,rot,inter", CASES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_forward(D, rot, inter, bad):
    q, k, v, w, table, pos, _ = inputs(6, 2, D, D, rot, D + rot, "f32")
    q, k = q.contiguous(), k.contiguous()
    for t in range(D):                   # token t has it in element t of two heads
        q[t, t % 6, t] = bad
        k[t, t % 2, t] = bad
    c = sq.Cache(1, 6, 2, D, 16, 64)
    par = sq.norm_rope(table, rot, 1e-5, *w, interleaved=inter)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    c.qk_norm_rope(q, k, pos if rot else None, par, qo, ko)
    h = c.seq_new()
    c.extend([h], [D])
    q2 = torch.empty_like(q)
    c.qk_norm_rope_store([h], [D], 0, q, k, v, pos if rot else None, par, q2)
    assert c.sync_status() == sq.SQ_OK
    assert torch.equal(q2.view(torch.int16), qo.view(torch.int16))
    for x, o, wt in ((q, qo, w[0]), (k, ko, w[1])):
        y = x.double()
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-5) * wt.double()
        want, _ = turn(y, table, pos, rot, inter)
        assert torch.equal(torch.isnan(o), torch.isnan(want))
        hit = ~torch.isfinite(x).all(-1)
        assert hit.sum() == D
        keep = ~torch.isnan(want) & hit[..., None]
        assert (want[keep] == 0).all() and (o[keep] == 0).all()
        assert torch.isfinite(o[~hit]).all()
    c.close()


@pytest.mark.parametrize("D,rot,inter", CASES)
def test_backward(D, rot, inter):
    """A gradient that is not finite in an element that does not turn: the weights'
    gradients of the others stay finite, and right."""
    q, k, _, w, table, pos, g = inputs(6, 2, D, 40, rot, D + rot, "f32")
    dz = [torch.randn(40, n, D, generator=g, device="cuda").bfloat16() for n in (6, 2)]
    at = D - 3 if rot < D else 5
    for z in dz:
        z[7, 1, at] = math.inf
    c = sq.Cache(1, 6, 2, D, 16, 1)
    par = sq.norm_rope(table, rot, 1e-5, *w, interleaved=inter)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dw = [torch.empty(D, device="cuda") for _ in range(2)]
    c.qk_norm_rope_backward(q, k, pos, par, *dz, dq, dk, *dw)
    assert c.sync_status() == sq.SQ_OK
    for x, z, got in ((q, dz[0], dw[0]), (k, dz[1], dw[1])):
        x = x.double()
        xr = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        dy, _ = turn(z.double(), table, pos, rot, inter, -1.0)
        want = (dy * xr).sum((0, 1))
        fine = torch.isfinite(want)
        assert (~fine).sum() == (1 if rot < D else 2)
        assert torch.equal(torch.isfinite(got), fine)
        size = (dy * xr).abs().sum((0, 1))[fine]
        assert ((got.double()[fine] - want[fine]).abs() <= size * 2.0 ** -16).all()
    c.close()
