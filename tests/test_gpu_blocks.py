"""Attention of query blocks on the GPU (sliding windows, sinks, drafted trees)
against 64-bit references, row by row within the error budget of the kernel's
bf16 weights (tests/budget.py): windows and sinks at the edges of 64-key boxes and
of pages, single tokens, ragged batches of prompts and tokens, blocks of one and of
two query tiles, key ranges cut into pieces, trees of every shape, partial pages,
forks, slots past the end that hold NaN, streams, and refusals."""
import math
import random

import numpy as np
import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.budget import decode_budget
from tests.gpu_harness import Pair, assert_budget, row_slots

pytestmark = pytest.mark.gpu
LSE_ABS = 1e-2   # as for sq_prefill_attention


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


class Batch:
    """A cache of one layer of N(0, 1) rows, its sequences, and what they hold."""

    def __init__(self, Hq, Hkv, D, P, lengths, seed=0, k_scale=1.0, num_pages=None):
        pages = num_pages or sum(-(-n // P) for n in lengths) + 40
        g = torch.Generator("cuda").manual_seed(seed)
        # slots nothing was stored to hold NaN
        self.pool = torch.full((1, pages, 2, Hkv, P, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.c = sq.Cache(1, Hq, Hkv, D, P, pages, kv_pool=self.pool)
        self.g, self.Hq, self.Hkv, self.D, self.k_scale = g, Hq, Hkv, D, k_scale
        self.h = [self.c.seq_new() for _ in lengths]
        for h, n in zip(self.h, lengths):
            self.append(h, n)

    def append(self, h, n):
        if n:
            k, v = (torch.randn(1, n, self.Hkv, self.D, generator=self.g, device="cuda") for _ in range(2))
            self.c.append_kv(h, n, (k * self.k_scale).bfloat16(), v.bfloat16())
            torch.cuda.synchronize()

    def rows(self, h):
        page, slot = row_slots(self.c, h)
        r = self.pool[0, page, :, :, slot]
        return r[:, 0].double(), r[:, 1].double()

    def queries(self, n, sharp=1.0):
        return (sharp * torch.randn(n, self.Hq, self.D, generator=self.g, device="cuda")).bfloat16()

    def call(self, n_q, q, parents=None, window=0, sinks=0, f32=True, scale=None, stream=None, hs=None):
        out = torch.full(q.shape, float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:2], float("nan"), device="cuda")
        kw = dict(out_dtype=sq.SQ_OUT_F32 if f32 else sq.SQ_OUT_BF16, lse=lse,
                  sm_scale=self.D ** -0.5 if scale is None else scale, stream=stream)
        hs = hs or self.h
        if parents is None:
            self.c.window_attention(hs, n_q, 0, q, out, window, sinks, **kw)
        else:
            self.c.tree_attention(hs, n_q, parents, 0, q, out, window, sinks, **kw)
        return out, lse

    def check(self, n_q, parents=None, window=0, sinks=0, f32=True, scale=None, sharp=1.0, sample=24):
        counts = [1] * len(self.h) if n_q is None else n_q
        q = self.queries(sum(counts), sharp)
        out, lse = self.call(n_q, q, parents, window, sinks, f32, scale)
        assert self.c.sync_status() == sq.SQ_OK
        scale = self.D ** -0.5 if scale is None else scale
        G, at = self.Hq // self.Hkv, 0
        for h, m in zip(self.h, counts):
            k, v = self.rows(h)
            n = k.shape[0]
            place = torch.arange(n, device="cuda")
            anc = []
            if parents is not None:
                for p in parents[at:at + m]:
                    anc.append((anc[p] if p >= 0 else []) + [len(anc)])
                place[n - m:] = n - m + torch.tensor([len(a) - 1 for a in anc], device="cuda")
            picked = sorted(set(np.linspace(0, m - 1, min(m, sample)).round().astype(int).tolist())) if m else []
            for i in picked:
                see = torch.arange(n, device="cuda") <= n - m + i
                if parents is not None:
                    see[n - m:] = False
                    see[[n - m + a for a in anc[i]]] = True
                if window:
                    see &= (place > place[n - m + i] - window) | (place < sinks)
                kk, vv = k[see], v[see]
                z = torch.einsum("ghd,tgd->ght", q[at + i].double().view(self.Hkv, G, -1), kk) * scale
                w = torch.softmax(z, -1)
                o = torch.einsum("ght,tgd->ghd", w, vv)
                dev = torch.stack([torch.einsum("ht,htd->hd", w[g], (vv[:, g][None] - o[g][:, None]).abs())
                                   for g in range(self.Hkv)])
                absv = torch.einsum("ght,tgd->ghd", w, vv.abs())
                flat = lambda t: t.reshape(self.Hq, self.D).cpu().numpy()  # noqa: E731
                budget = decode_budget(flat(dev), flat(absv), kk.shape[0])
                if not f32:
                    budget = budget * (1 + 2.0 ** -8) + np.abs(flat(o)) * 2.0 ** -8
                got = out[at + i].float()
                if f32:
                    assert_budget(got, flat(o), budget)
                else:
                    assert (np.abs(got.cpu().numpy() - flat(o)) <= budget).all()
                exact = torch.logsumexp(z, -1).view(-1)
                assert (lse[at + i].double() - exact).abs().max() <= LSE_ABS
            at += m
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        return q, out, lse


GEOMETRIES = [(8, 2, 128, 64), (16, 2, 64, 16), (6, 2, 128, 256), (16, 1, 64, 8), (4, 4, 128, 32), (8, 1, 128, 128)]


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (64, 4), (65, 64), (200, 130), (0, 0), (4000, 7)])
def test_single_tokens(Hq, Hkv, D, P, window, sinks):
    b = Batch(Hq, Hkv, D, P, [1, 63, 64, 65, 129, 700], seed=window + P)
    b.check(None, window=window, sinks=sinks)
    b.c.close()


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (64, 4), (65, 64), (200, 130), (0, 0), (4000, 7)])
def test_single_tokens_without_log_sums(Hq, Hkv, D, P, window, sinks):
    """Without log-sum-exps single tokens take the decode kernel: the same rows,
    within both kernels' budgets; sequences without a query in between."""
    b = Batch(Hq, Hkv, D, P, [1, 63, 64, 65, 129, 700, 3000], seed=window + P)
    q, out, _ = b.check(None, window=window, sinks=sinks)
    got = torch.full_like(out, float("nan"))
    kw = dict(out_dtype=sq.SQ_OUT_F32, sm_scale=D ** -0.5)
    b.c.window_attention(b.h, None, 0, q, got, window, sinks, **kw)
    some = torch.full_like(out[:3], float("nan"))
    b.c.window_attention(b.h, [1, 0, 0, 1, 0, 1, 0], 0, q[[0, 3, 5]], some, window, sinks, **kw)
    assert b.c.sync_status() == sq.SQ_OK
    assert torch.isfinite(got).all()
    for i, h in enumerate(b.h):
        k, v = b.rows(h)
        see = torch.arange(k.shape[0], device="cuda")
        see = (see >= k.shape[0] - (window or 1 << 30)) | (see < sinks)
        G = Hq // Hkv
        z = torch.einsum("ghd,tgd->ght", q[i].double().view(Hkv, G, -1), k[see]) * D ** -0.5
        w = torch.softmax(z, -1)
        o = torch.einsum("ght,tgd->ghd", w, v[see]).reshape(Hq, D)
        dev = torch.stack([torch.einsum("ht,htd->hd", w[g], (v[see][:, g][None] - o.view(Hkv, G, D)[g][:, None]).abs())
                           for g in range(Hkv)]).reshape(Hq, D)
        absv = torch.einsum("ght,tgd->ghd", w, v[see].abs()).reshape(Hq, D)
        budget = decode_budget(dev.cpu().numpy(), absv.cpu().numpy(), int(see.sum()))
        assert_budget(got[i], o.cpu().numpy(), budget)
        if i in (0, 3, 5):
            assert_budget(some[(0, 3, 5).index(i)], o.cpu().numpy(), budget)
    b.c.close()


def test_windows_follow_appended_rows():
    """Decode steps: the window moves with every row, also where a plain decode
    plan of the same sequences is kept, and on another stream."""
    b = Batch(8, 2, 128, 64, [300, 64, 1000], seed=77)
    for step in range(5):
        for h in b.h:
            b.append(h, 1)
        q = b.queries(3)
        for window, sinks in ((100, 4), (100, 0), (0, 0), (64, 4)):
            got, ref = (torch.empty(3, 8, 128, device="cuda") for _ in range(2))
            kw = dict(out_dtype=sq.SQ_OUT_F32, sm_scale=0.1)
            b.c.window_attention(b.h, None, 0, q, got, window, sinks, **kw)
            b.c.window_attention(b.h, None, 0, q, ref, window, sinks, lse=torch.empty(3, 8, device="cuda"), **kw)
            torch.cuda.synchronize()
            assert (got - ref).abs().max() <= 1e-2
        b.c.decode_attention(b.h, 0, q, ref, sq.SQ_OUT_F32, 0.1)
        b.c.window_attention(b.h, None, 0, q, got, 0, 9, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, ref)
    assert b.c.sync_status() == sq.SQ_OK
    b.c.close()


@pytest.mark.parametrize("value", [-300.0, -90.0, 60.0, 400.0])
def test_logits_far_from_zero(value):
    """Rows whose logits all lie far below or above zero, and rows that a tile
    without visible keys comes before."""
    b = Batch(8, 2, 64, 64, [900], seed=3)
    page, slot = row_slots(b.c, b.h[0])
    k = b.pool[0, page, 0, :, slot]
    k[..., 0] = 8.0
    b.pool[0, page, 0, :, slot] = k
    q = b.queries(200)
    q[:, :, 0] = value
    parents = None
    for window, sinks in ((100, 0), (100, 3), (0, 0)):
        out, lse = b.call([200], q, parents, window, sinks, scale=0.125)
        assert b.c.sync_status() == sq.SQ_OK
        kk, vv = b.rows(b.h[0])
        at = torch.arange(900, device="cuda")
        see = (at[None] <= at[700:, None]) & ((at[None] > at[700:, None] - (window or 9999)) | (at[None] < sinks))
        z = torch.einsum("nghd,tgd->nght", q.double().view(200, 2, 4, 64), kk) * 0.125
        z = z.masked_fill(~see[:, None, None], -math.inf)
        w = torch.softmax(z, -1)
        o = torch.einsum("nght,tgd->nghd", w, vv).reshape(200, 8, 64)
        assert (out.double() - o).abs().max() <= 1e-2
        ref = torch.logsumexp(z, -1).reshape(200, 8)
        assert ((lse.double() - ref).abs() <= LSE_ABS + ref.abs() * 2.0 ** -20).all()
    b.c.close()


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(3, 2), (64, 0), (100, 70), (0, 0)])
def test_prompts_and_tokens_together(Hq, Hkv, D, P, window, sinks):
    b = Batch(Hq, Hkv, D, P, [300, 1, 517, 90, 128], seed=window + D + 1)
    b.check([300, 1, 131, 0, 64], window=window, sinks=sinks)
    b.check([17, 1, 517, 90, 0], window=window, sinks=sinks, f32=False)
    b.c.close()


@pytest.mark.parametrize("sharp,scale", [(1.0, 0.0), (6.0, None), (20.0, None), (1.0, 1.0)])
def test_scales(sharp, scale):
    b = Batch(8, 2, 128, 64, [900, 300], seed=7)
    b.check([200, 1], window=150, sinks=3, scale=scale, sharp=sharp)
    b.c.close()


def test_long_contexts_are_cut_and_merged():
    b = Batch(8, 2, 128, 64, [9001], seed=11)
    b.check(None, window=0)
    b.check([9], window=7000, sinks=4)
    b.check([40], window=0, sample=8)     # two query tiles
    b.check(None, window=20, sinks=8500)  # sinks in pieces that see no window
    b.c.close()


def tree(rng, m):
    return [-1 if i == 0 or rng.random() < 0.15 else rng.randrange(max(-1, i - 6), i) for i in range(m)]


@pytest.mark.parametrize("Hq,Hkv,D,P", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (4, 2), (70, 0), (1, 300)])
def test_trees(Hq, Hkv, D, P, window, sinks):
    rng = random.Random(window + D + P)
    counts = [1, 33, 0, 64, 7]
    b = Batch(Hq, Hkv, D, P, [n + m for n, m in zip([1, 31, 500, 193, 64], counts)], seed=window + Hq)
    b.check(counts, [p for m in counts for p in tree(rng, m)], window, sinks)
    b.c.close()


@pytest.mark.parametrize("m,kind", [(256, "random"), (256, "chain"), (200, "star"), (256, "binary")])
def test_largest_trees(m, kind):
    parents = {"random": tree(random.Random(m), m), "chain": list(range(-1, m - 1)), "star": [-1] * m,
               "binary": [-1] + [(i - 1) // 2 for i in range(1, m)]}[kind]
    b = Batch(8, 1, 128, 64, [1000 + m], seed=m)
    b.check([m], parents, sample=40)
    b.check([m], parents, window=30, sinks=1, sample=40, f32=False)
    b.c.close()


def test_a_chain_is_causal_attention():
    """A tree without branches gives what the window form and masked prefill give."""
    b = Batch(8, 2, 128, 64, [700, 80], seed=2)
    q = b.queries(60)
    chain = list(range(-1, 29))
    o1, l1 = b.call([30, 30], q, chain * 2, window=50, sinks=2)
    o2, l2 = b.call([30, 30], q, None, window=50, sinks=2)
    torch.cuda.synchronize()
    assert (o1 - o2).abs().max() <= 1e-2 and (l1 - l2).abs().max() <= LSE_ABS
    o3, l3 = b.call([30, 30], q, None)
    o4, l4 = torch.empty_like(o3), torch.empty_like(l3)
    for i, h in enumerate(b.h):
        at = slice(30 * i, 30 * i + 30)
        b.c.prefill_attention(h, 0, 30, q[at].contiguous(), o4[at], sq.SQ_OUT_F32, l4[at], 128 ** -0.5)
    torch.cuda.synchronize()
    assert (o3 - o4).abs().max() <= 1e-2 and (l3 - l4).abs().max() <= LSE_ABS
    b.c.close()


@pytest.mark.parametrize("P,D", [(8, 64), (64, 128), (256, 128)])
def test_partial_pages(P, D):
    """After ragged evictions windows count rows, not slots, and unused slots are
    not seen; queries may lie on both sides of a partial page."""
    b = Batch(8, 2, D, P, [1500, 900, 2 * P + 3], seed=P)
    b.c.evict_spans_ragged(b.h[0], [(3, 40), (700, 731), (1200, 1450)])
    b.c.evict_spans_ragged(b.h[1], [(P, P + 5), (880, 890)])
    for window, sinks in ((1, 0), (30, 5), (64, 64), (500, 0), (0, 0)):
        b.check(None, window=window, sinks=sinks)
        b.check([200, 30, 5], window=window, sinks=sinks)
    for h in b.h:
        b.append(h, 20)
    rng = random.Random(P)
    for window, sinks in ((0, 0), (25, 3), (400, 0)):
        b.check([20, 12, 20], tree(rng, 20) + tree(rng, 12) + tree(rng, 20), window, sinks)
    b.c.close()


def test_forks_and_drafted_tokens_accepted():
    """A drafted step as a server runs it: rows added and stored, the tree
    verified, a path kept; the next tokens attend to what is left, on pages that a
    fork made before still reads."""
    b = Batch(8, 2, 64, 16, [100], seed=21)
    a = b.h[0]
    f = b.c.fork_aux(a)
    par = sq.norm_rope()
    rng = random.Random(4)
    kept, nxt = 100, 100
    before = b.rows(f)
    for step in range(6):
        m = rng.randint(1, 24)
        parents = tree(rng, m)
        b.c.extend([a], [m])
        qkv = torch.randn(m, 12, 64, generator=b.g, device="cuda").bfloat16()
        q = torch.empty(m, 8, 64, dtype=torch.bfloat16, device="cuda")
        b.c.qk_norm_rope_store([a], [m], 0, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], None, par, q)
        b.h = [a]
        b.check([m], parents, window=rng.choice([0, 40]), sinks=2)
        k0, v0 = b.rows(a)
        path = []                                   # from a leaf to the root
        i = rng.randrange(-1, m)
        while i >= 0:
            path.insert(0, i)
            i = parents[i]
        b.c.accept_draft(a, m, path)
        stay = list(range(kept)) + [kept + i for i in path]
        kept, nxt = kept + len(path), nxt + len(path)
        assert b.c.seq_info(a)[0] == kept and b.c.next_pos(a) == nxt
        k1, v1 = b.rows(a)
        assert torch.equal(k0[stay], k1) and torch.equal(v0[stay], v1)
        b.check(None, window=37, sinks=2)
    assert torch.equal(before[0], b.rows(f)[0]) and torch.equal(before[1], b.rows(f)[1])
    # and with partial pages, which stay as they are
    b.c.evict_spans_ragged(a, [(20, 27), (50, 60)])
    fills = b.c.page_fills(a)
    b.append(a, 5)
    k0, _ = b.rows(a)
    n = k0.shape[0]
    b.c.accept_draft(a, 5, [0, 2])
    stay = list(range(n - 5)) + [n - 5, n - 3]
    assert torch.equal(b.rows(a)[0], k0[stay])
    assert b.c.page_fills(a)[:len(fills) - 1] == fills[:-1]
    b.check(None, window=0)
    b.c.close()


def test_a_store_between_layers_is_seen():
    """A store changes no plan: calls that reuse theirs read the rows stored just
    before, every time (several layers, the same plans, back to back)."""
    P, L = 64, 6
    c = sq.Cache(L, 8, 2, 128, P, 40)
    hs = [c.seq_new() for _ in range(3)]
    g = torch.Generator("cuda").manual_seed(5)
    for h in hs:
        k, v = (torch.randn(L, 700, 2, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
        c.append_kv(h, 700, k, v)
    torch.cuda.synchronize()
    par = sq.norm_rope()
    c.extend(hs, [4, 4, 4])
    qkv = torch.randn(L, 12, 12, 128, generator=g, device="cuda").bfloat16()
    chain = [-1, 0, 1, 2] * 3
    outs = []
    for slow in (False, True):
        out = torch.empty(L, 3, 12, 8, 128, device="cuda")
        c.pool_view()[:, :, :, :, :, :].view(torch.int16)[:, c.page_table(hs[0])[-1]] = 0
        torch.cuda.synchronize()
        for rep in range(4):
            for layer in range(L):
                q = torch.empty(12, 8, 128, dtype=torch.bfloat16, device="cuda")
                x = qkv[(layer + rep) % L]
                c.qk_norm_rope_store(hs, [4, 4, 4], layer, x[:, :8], x[:, 8:10], x[:, 10:], None, par, q)
                if slow:
                    torch.cuda.synchronize()
                c.tree_attention(hs, [4, 4, 4], chain, layer, q, out[layer, 0], out_dtype=sq.SQ_OUT_F32)
                c.window_attention(hs, [4, 4, 4], layer, q, out[layer, 1], 100, 2, out_dtype=sq.SQ_OUT_F32)
                if slow:
                    torch.cuda.synchronize()
                c.decode_attention(hs, layer, q[3::4].contiguous(), out[layer, 2, :3], sq.SQ_OUT_F32)
                if slow:
                    torch.cuda.synchronize()
        assert c.sync_status() == sq.SQ_OK
        outs.append(torch.cat([out[:, 0], out[:, 1], out[:, 2, :3]], 1))
    assert torch.equal(*outs)
    c.close()


def test_streams_and_repeats():
    """Calls on three streams take turns with plans and workspaces; results do not
    depend on the order, bit for bit."""
    b = Batch(8, 2, 128, 64, [9000, 3000, 700], seed=31)
    q = b.queries(3)
    qs = b.queries(30)
    parents = tree(random.Random(1), 10) * 3
    first = [t.clone() for t in (*b.call(None, q, window=0), *b.call([10] * 3, qs, parents))]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append((*b.call(None, q, window=0), *b.call([10] * 3, qs, parents)))
    torch.cuda.synchronize()
    assert b.c.sync_status() == sq.SQ_OK
    for g in got:
        for x, y in zip(first, g):
            assert torch.equal(x, y)
    b.c.close()


def test_empty_calls_and_refusals():
    b = Batch(8, 2, 128, 64, [100, 50], seed=1)
    c, q = b.c, b.queries(6)
    out = torch.empty_like(q)
    c.window_attention([], [], 0, q[:0], out[:0], 5)
    c.window_attention(b.h, [0, 0], 0, q[:0], out[:0], 5)
    c.tree_attention(b.h, [0, 0], [], 0, q[:0], out[:0])
    c.accept_draft(b.h[0], 0, [])
    assert c.seq_info(b.h[0])[0] == 100

    def refused(code, f, *a, **kw):
        with pytest.raises(sq.SqError) as e:
            f(*a, **kw)
        assert e.value.code == code

    bad = sq.SQ_ERR_INVALID_ARG
    win, tr = c.window_attention, c.tree_attention
    refused(bad, win, b.h, [5, 1], 1, q, out, 5)                 # layer
    refused(bad, win, b.h, [5, 1], 0, q, out, -1)                # window
    refused(bad, win, b.h, [5, 1], 0, q, out, 5, -1)             # sinks
    refused(bad, win, b.h, [5, 1], 0, q, out, 5, sm_scale=-1.0)
    refused(bad, win, b.h, [5, 1], 0, q, out, 5, sm_scale=float("nan"))
    refused(bad, win, b.h, [5, 1], 0, q, out, 5, out_dtype=3)
    refused(bad, win, b.h, [5, 1], 0, q, q, 5)                   # overlap
    refused(bad, win, [b.h[0], b.h[0]], [5, 1], 0, q, out, 5)    # twice
    refused(sq.SQ_ERR_BAD_HANDLE, win, [b.h[0], b.h[1] + 5], [5, 1], 0, q, out, 5)
    refused(bad, sq.sq_window_attention, c.handle, b.h, [5, 51], 0, q, out, 5)
    refused(bad, sq.sq_window_attention, c.handle, b.h, [5, -1], 0, q, out, 5)
    refused(bad, win, b.h, [5, 1], 0, q.data_ptr() + 2, out, 5)
    with pytest.raises(ValueError):
        win(b.h, [5, 2], 0, q, out, 5)
    refused(bad, tr, b.h, [5, 1], [-1, 0, 2, 0, 0, -1], 0, q, out)    # its own parent
    refused(bad, tr, b.h, [5, 1], [-1, 0, -2, 0, 0, -1], 0, q, out)
    with pytest.raises(ValueError):
        tr(b.h, [5, 1], [-1] * 5, 0, q, out)
    big = b.queries(257)
    b.append(b.h[0], 300)
    refused(bad, tr, b.h[:1], [257], [-1] * 257, 0, big, torch.empty_like(big))
    for path in ([1, 0], [0, 0], [5], [-1]):
        refused(bad, c.accept_draft, b.h[0], 5, path)
    refused(bad, c.accept_draft, b.h[0], 401, [])
    assert c.sync_status() == sq.SQ_OK
    c.close()
