"""Masked prefill over a pool whose unwritten slots hold NaN: rows that were added
before their keys and values exist, and never got any, are hidden by a ragged
eviction or by a span, and reach no query.  Against 64-bit references within the
kernel's error budget."""
import numpy as np
import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.budget import decode_budget
from tests.gpu_harness import assert_budget
from tests.test_gpu_blocks import LSE_ABS, Batch

pytestmark = pytest.mark.gpu
PAGES = [8, 16, 32, 64, 128, 256]
HEADS = [(8, 2, 128), (16, 1, 64), (4, 4, 64), (6, 2, 128)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def store(b, h, m):
    """Keys and values of the newest m rows of sequence h."""
    q, k, v = (torch.randn(m, n, b.D, generator=b.g, device="cuda").bfloat16() for n in (b.Hq, b.Hkv, b.Hkv))
    b.c.qk_norm_rope_store([h], [m], 0, q, k, v, None, sq.norm_rope(), torch.empty_like(q))
    torch.cuda.synchronize()


def check(b, h, m, spans=(), sample=16):
    q = b.queries(m)
    out = torch.full(q.shape, float("inf"), device="cuda")
    lse = torch.full(q.shape[:2], float("inf"), device="cuda")
    for again in range(3):     # (a kept plan is read, and keys are loaded, ahead of the launch's wait)
        first = out.clone()
        b.c.prefill_attention(h, 0, m, q, out, sq.SQ_OUT_F32, lse, b.D ** -0.5, list(spans))
        assert b.c.sync_status() == sq.SQ_OK
        assert not again or torch.equal(out, first)
    k, v = b.rows(h)
    n, G = k.shape[0], b.Hq // b.Hkv
    shown = torch.ones(n, dtype=torch.bool, device="cuda")
    for lo, hi in spans:
        shown[lo:hi] = False
    for i in sorted(set(np.linspace(0, m - 1, min(m, sample)).round().astype(int).tolist())):
        see = shown & (torch.arange(n, device="cuda") <= n - m + i)
        kk, vv = k[see], v[see]
        z = torch.einsum("ghd,tgd->ght", q[i].double().view(b.Hkv, G, -1), kk) * b.D ** -0.5
        w = torch.softmax(z, -1)
        o = torch.einsum("ght,tgd->ghd", w, vv)
        dev = torch.stack([torch.einsum("ht,htd->hd", w[g], (vv[:, g][None] - o[g][:, None]).abs())
                           for g in range(b.Hkv)])
        absv = torch.einsum("ght,tgd->ghd", w, vv.abs())
        flat = lambda t: t.reshape(b.Hq, b.D).cpu().numpy()  # noqa: E731
        assert_budget(out[i], flat(o), decode_budget(flat(dev), flat(absv), kk.shape[0]))
        assert (lse[i].double() - torch.logsumexp(z, -1).view(-1)).abs().max() <= LSE_ABS
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("P", PAGES)
def test_evicted_before_they_were_stored(Hq, Hkv, D, P):
    """The last rows of a page leave by a ragged eviction: their slots stay as they
    were."""
    b = Batch(Hq, Hkv, D, P, [200], seed=P, num_pages=200)
    h = b.h[0]
    end = (216 + P - 1) // P * P
    first = end - min(6, P - 2)
    b.c.extend([h], [end + 300 - 200])
    b.c.evict_spans_ragged(h, [(first, end)])
    assert b.c.page_fills(h)[end // P - 1] == first - (end - P)
    store(b, h, first - 200 + 300)
    for m in (5, 44, 300):
        check(b, h, m)
    check(b, h, 44, [(20, 90), (first - 3, first + 2)])
    b.c.close()


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("P", PAGES)
def test_under_a_span(Hq, Hkv, D, P):
    """Rows that a span hides were added and not stored."""
    b = Batch(Hq, Hkv, D, P, [300], seed=P, num_pages=200)
    h = b.h[0]
    b.c.extend([h], [37])
    b.append(h, 130)
    b.c.extend([h], [101])
    b.append(h, 260)
    spans = [(10, 20), (300, 337), (467, 568)]
    for m in (1, 5, 60, 260):
        check(b, h, m, spans)
    f = b.c.fork_aux(h)     # (what its parent's rows hold is its own too)
    b.append(f, 40)
    check(b, f, 40, spans)
    b.c.close()


@pytest.mark.parametrize("P,D", [(16, 64), (64, 128), (256, 128)])
@pytest.mark.parametrize("m", [8, 40, 700])
def test_pieces_of_a_long_context(P, D, m):
    """Key ranges cut into pieces, unwritten rows in most of them."""
    b = Batch(8, 2, D, P, [1000], seed=m, num_pages=700)
    h, spans, n = b.h[0], [], 1000
    for i in range(8):
        extra = 1 + 17 * i
        b.c.extend([h], [extra])
        spans.append((n, n + extra))
        b.append(h, 1000)
        n += extra + 1000
    check(b, h, m, spans)
    b.c.close()
