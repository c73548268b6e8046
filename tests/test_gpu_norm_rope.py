"""Norms and rotation of queries and keys on the GPU, forwards (to tensors and
into the cache) and backwards, against 64-bit references: head counts that do not
divide a warp's rows, parts of fused projections, partial rotations, both ways of
pairing, both weight types and none, empty calls, positions at the table's ends,
pages and copy-on-write, and refusals.

Tolerances, set by the arithmetic: a bf16 output is the exact value rounded once
(half a unit in the last place, at most 2^-8 of it) after fp32 errors of a few
2^-24 of the pair's length, 2^-20 allowed; weights' gradients are fp32
sums of n terms, each with a few 2^-24 of its size, added in chains of at most a
few hundred terms, so within 2^-16 of the sum of the terms' sizes."""
import math

import numpy as np
import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.gpu_harness import Pair, row_slots

pytestmark = pytest.mark.gpu
MAX_POS = 3001


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def reference(x, w, eps, table, pos, rot, inter):
    """(rotated rows, length of each element's pair) in 64 bits: x [n, heads, D]."""
    x = x.double()
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    return turn(y, table, pos, rot, inter)


def turn(y, table, pos, rot, inter, sign=1.0):
    size = y.abs().clone()
    out = y.clone()
    if rot:
        c, s = table[pos.long(), :, 0].double()[:, None], sign * table[pos.long(), :, 1].double()[:, None]
        i = torch.arange(rot // 2, device=y.device)
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = torch.hypot(y[..., a], y[..., b])
    return out, size


def assert_rounded(got, exact, size):
    """got is exact rounded to bf16, but for fp32 errors of `size`."""
    err = (got.double() - exact).abs()
    bound = exact.abs() * 2.0 ** -8 + size * 2.0 ** -20 + 1e-30
    assert torch.isfinite(got.float()).all()
    assert (err <= bound).all(), float((err / bound).max())


def inputs(Hq, Hkv, D, n, rot, seed, weights="bf16", extra=0):
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    qkv = (rnd(n, Hq + 2 * Hkv + extra, D) * torch.exp(rnd(n, Hq + 2 * Hkv + extra, 1))).bfloat16()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:Hq + 2 * Hkv]
    dt = torch.float32 if weights == "f32" else torch.bfloat16
    w = (None, None) if weights is None else ((1 + 0.3 * rnd(D)).to(dt), (1 + 0.3 * rnd(D)).to(dt))
    table = sq.rope_table(MAX_POS, rot, 10000.0) if rot else None
    pos = torch.randint(0, MAX_POS, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 1:
        pos[0], pos[-1] = 0, MAX_POS - 1
    return q, k, v, w, table, pos, g


GEOMETRIES = [(8, 2, 128), (6, 2, 128), (64, 8, 64), (5, 5, 64), (16, 1, 128), (3, 1, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", GEOMETRIES)
@pytest.mark.parametrize("rot,inter,weights,n", [
    ("all", False, "bf16", 37), ("all", True, "f32", 9), (16, False, "f32", 130), (48, True, "bf16", 1),
    (48, False, None, 3), (0, False, "bf16", 50), ("all", False, "f32", 0), (32, False, "bf16", 1001)])
def test_forward(Hq, Hkv, D, rot, inter, weights, n):
    rot = D if rot == "all" else rot
    q, k, _, w, table, pos, _ = inputs(Hq, Hkv, D, n, rot, n + D, weights, extra=n % 3)
    c = sq.Cache(1, Hq, Hkv, D, 16, 1)
    par = sq.norm_rope(table, rot, 1e-5, *w, interleaved=inter)
    qo = torch.full((n, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ko = torch.full((n, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.qk_norm_rope(q, k, pos if rot else None, par, qo, ko)
    assert c.sync_status() == sq.SQ_OK
    for x, o, wt in ((q, qo, w[0]), (k, ko, w[1])):
        assert_rounded(o, *reference(x, wt, 1e-5, table, pos, rot, inter))
    c.close()


@pytest.mark.parametrize("Hq,Hkv,D", GEOMETRIES)
@pytest.mark.parametrize("rot,inter,weights,n", [
    ("all", False, "bf16", 37), ("all", True, "f32", 9), (16, False, "f32", 130), (48, True, "bf16", 1),
    (48, False, None, 3), (0, False, "bf16", 50), (32, False, "bf16", 2001)])
def test_backward(Hq, Hkv, D, rot, inter, weights, n):
    rot = D if rot == "all" else rot
    q, k, _, w, table, pos, g = inputs(Hq, Hkv, D, n, rot, n + D, weights)
    c = sq.Cache(1, Hq, Hkv, D, 16, 1)
    par = sq.norm_rope(table, rot, 1e-5, *w, interleaved=inter)
    dz = [torch.randn(n, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv)]
    # the inputs' gradients as parts of one fused gradient
    fused = torch.full((n, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    dq, dk = fused[:, :Hq], fused[:, Hq:Hq + Hkv]
    dw = [torch.full((D,), float("nan"), device="cuda") for _ in range(2)]
    run = lambda: c.qk_norm_rope_backward(q, k, pos if rot else None, par, *dz, dq, dk, *dw)  # noqa: E731
    run()
    assert c.sync_status() == sq.SQ_OK
    first = [t.clone() for t in (*dw, dq, dk)]
    for x, wt, z, dx, dwt in ((q, w[0], dz[0], dq, dw[0]), (k, w[1], dz[1], dk, dw[1])):
        x = x.double()
        wt = torch.ones(D, dtype=torch.float64, device="cuda") if wt is None else wt.double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
        dy, size = turn(z.double(), table, pos, rot, inter, -1.0)
        xn = x * r
        dot = (dy * wt * xn).mean(-1, keepdim=True)
        dots = (size * wt.abs() * xn.abs()).mean(-1, keepdim=True)
        assert_rounded(dx, r * (dy * wt - xn * dot), r * (size * wt.abs() + xn.abs() * dots))
        exact, terms = (dy * xn).sum((0, 1)), (size * xn.abs()).sum((0, 1))
        assert ((dwt.double() - exact).abs() <= terms * 2.0 ** -16).all()
    assert (fused[:, Hq + Hkv:] == 7).all()
    # the same again, bit for bit, and without the weights' gradients
    run()
    for a, b in zip(first, (*dw, dq, dk)):
        assert torch.equal(a, b)
    c.qk_norm_rope_backward(q, k, pos if rot else None, par, *dz, dq, dk)
    assert torch.equal(first[2], dq) and torch.equal(first[3], dk)
    c.close()


def test_backward_of_nothing_zeroes_the_weights():
    c = sq.Cache(1, 4, 2, 64, 16, 1)
    e = lambda h: torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    dw = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    c.qk_norm_rope_backward(e(4), e(2), None, sq.norm_rope(), e(4), e(2), e(4), e(2), *dw)
    assert c.sync_status() == sq.SQ_OK
    assert all((d == 0).all() for d in dw)
    c.close()


def test_backward_against_differences():
    """Central differences of a loss in 64 bits, along random directions, through
    the forward's definition: the kernel's gradients give the same slopes."""
    Hq, Hkv, D, n, rot = 4, 2, 64, 12, 32
    q, k, _, w, table, pos, g = inputs(Hq, Hkv, D, n, rot, 5, "f32")
    c = sq.Cache(1, Hq, Hkv, D, 16, 1)
    par = sq.norm_rope(table, rot, 1e-5, *w)
    dz = [torch.randn(n, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv)]
    dx = [torch.empty(n, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv)]
    dw = [torch.empty(D, device="cuda") for _ in range(2)]
    c.qk_norm_rope_backward(q, k, pos, par, *dz, *dx, *dw)
    assert c.sync_status() == sq.SQ_OK
    for x, wt, z, gx, gw in ((q, w[0], dz[0], dx[0], dw[0]), (k, w[1], dz[1], dx[1], dw[1])):
        loss = lambda xx, ww: (reference(xx, ww, 1e-5, table, pos, rot, False)[0] * z.double()).sum()  # noqa: E731
        for _ in range(4):
            # directions in proportion to the rows, so that a step is small in each
            d = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64) * \
                x.double().pow(2).mean(-1, keepdim=True).sqrt()
            h = 1e-5
            slope = (loss(x.double() + h * d, wt.double()) - loss(x.double() - h * d, wt.double())) / (2 * h)
            mine, size = (gx.double() * d).sum(), (gx.double() * d).abs().sum()
            assert abs(float(slope - mine)) <= 2.0 ** -8 * float(size)
            d = torch.randn(D, generator=g, device="cuda", dtype=torch.float64)
            slope = (loss(x.double(), wt.double() + h * d) - loss(x.double(), wt.double() - h * d)) / (2 * h)
            assert abs(float(slope - (gw.double() * d).sum())) <= 1e-4 * float((gw.double() * d).abs().sum()) + 1e-6
    c.close()


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 64), (6, 3, 64, 8), (16, 1, 128, 256)])
@pytest.mark.parametrize("own_positions", [False, True])
def test_store(Hq, Hkv, D, P, own_positions):
    """Ragged stores at one layer of three: places across pages and after a
    ragged eviction, a forked sequence (copied on write by sq_extend), rows of
    nobody else touched; few rows (with the launch) and many (uploaded)."""
    p = Pair(3, Hq, Hkv, D, P, num_pages=4000 // P + 40, seed=P)
    keep = [p.append(h := p.seq_new(), n) or h for n in (P + 3, 2 * P, 5)]
    hs = list(p.o)
    p.evict(hs[0], [(2, 4)], ragged=True)
    f = p.fork(hs[2])
    hs.append(f)
    for counts in ([1, 1, 1, 1], [3, 0, P + 1, 2], [700, 1, 130, 2 * P]):
        before = p.cache.pool_view().clone()
        held = [p.cache.page_table(h) for h in hs]
        n0 = [p.cache.seq_info(h)[0] for h in hs]
        nxt = [p.cache.next_pos(h) for h in hs]
        p.cache.extend(hs, None if counts == [1] * 4 else counts)
        for h, m in zip(hs, counts):
            p.oracle.append(p.o[h], m)
        p.check_tables()
        n = sum(counts)
        q, k, v, w, table, pos, _ = inputs(Hq, Hkv, D, n, 32, n, "bf16")
        par = sq.norm_rope(table, 32, 1e-6, *w)
        qo = torch.full((n, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        if own_positions:
            pos = torch.tensor([a + i for a, m in zip(nxt, counts) for i in range(m)], dtype=torch.int32,
                               device="cuda")
        for layer in (1, 1):  # (the second finds its places on the device)
            p.cache.qk_norm_rope_store(hs, counts, layer, q, k, v, None if own_positions else pos, par, qo)
        assert p.cache.sync_status() == sq.SQ_OK
        assert_rounded(qo, *reference(q, w[0], 1e-6, table, pos, 32, False))
        exact, size = reference(k, w[1], 1e-6, table, pos, 32, False)
        pool, at = p.cache.pool_view(), 0
        free = torch.ones(pool.shape[1], P, dtype=torch.bool, device="cuda")
        for h, m, old in zip(hs, counts, n0):
            page, slot = row_slots(p.cache, h)
            page, slot = page[old:], slot[old:]
            got = pool[1, page, :, :, slot]                   # [m, 2, Hkv, D]
            assert_rounded(got[:, 0], exact[at:at + m], size[at:at + m])
            assert torch.equal(got[:, 1], v[at:at + m])
            free[page, slot] = False
            at += m
        # what was not stored to is as it was (a copied page's rows aside)
        for h, t in zip(hs, held):
            if p.cache.page_table(h)[:len(t)] != t:
                free[p.cache.page_table(h)[len(t) - 1]] = False
        for layer in range(3):
            mine = free if layer == 1 else torch.ones_like(free)
            if layer != 1:
                for h, t in zip(hs, held):
                    if p.cache.page_table(h)[:len(t)] != t:
                        mine[p.cache.page_table(h)[len(t) - 1]] = False
            same = (pool[layer].view(torch.int16) == before[layer].view(torch.int16)).all(-1).all(2).all(1)
            assert (same | ~mine).all()
    p.close()


def test_extend_copies_a_shared_page_and_keeps_decode_plans():
    """The fork's shared last page is copied before rows are added; a decode plan
    reused after an extension inside a stage reads the new row."""
    p = Pair(2, 4, 2, 64, 64, num_pages=40, seed=3)
    keep = [p.append(p.seq_new(), 70)]
    a = next(iter(p.o))
    f = p.fork(a)
    p.cache.extend([f, a], [2, 1])
    assert p.cache.sync_status() == sq.SQ_OK
    assert p.cache.page_table(a)[0] == p.cache.page_table(f)[0]
    assert p.cache.page_table(a)[1] != p.cache.page_table(f)[1]
    pool = p.cache.pool_view()
    x, y = p.cache.page_table(a)[1], p.cache.page_table(f)[1]
    assert torch.equal(pool[:, x, :, :, :6].view(torch.int16), pool[:, y, :, :, :6].view(torch.int16))
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    outs = [torch.empty(1, 4, 64, device="cuda") for _ in range(3)]
    par = sq.norm_rope()

    def row(h, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        k, v = (torch.randn(1, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
        p.cache.extend([h])
        for layer in range(2):
            p.cache.qk_norm_rope_store([h], None, layer, q, k, v, None, par, torch.empty_like(q))

    def decode(out):
        p.cache.decode_attention([a], 1, q, out, sq.SQ_OUT_F32, 0.125)

    row(a, 1)
    decode(outs[0])
    built = p.cache.stats()["decode_plans_built"]
    row(a, 2)
    decode(outs[1])
    assert p.cache.stats()["decode_plans_built"] == built
    b = sq.Cache(2, 4, 2, 64, 64, 40)       # the same rows, planned anew
    h = b.seq_new()
    n = p.cache.seq_info(a)[0]
    page, slot = row_slots(p.cache, a)
    kv = pool[:, page, :, :, slot]          # [n, L, 2, Hkv, D]
    b.append_kv(h, n, kv[:, :, 0].transpose(0, 1).contiguous(), kv[:, :, 1].transpose(0, 1).contiguous())
    b.decode_attention([h], 1, q, outs[2], sq.SQ_OUT_F32, 0.125)
    torch.cuda.synchronize()
    assert torch.equal(outs[1], outs[2]) and not torch.equal(outs[0], outs[1])
    b.close()
    p.close()


def test_position_outside_the_table_is_reported():
    c = sq.Cache(1, 4, 2, 64, 16, 1)
    q, k, _, w, table, pos, _ = inputs(4, 2, 64, 5, 32, 1)
    par = sq.norm_rope(table, 32, 1e-6, *w)
    qo, ko = torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda"), \
        torch.empty(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (-1, MAX_POS):
        pos[3] = bad
        c.qk_norm_rope(q, k, pos, par, qo, ko)
        assert c.sync_status() == sq.SQ_ERR_DEVICE
    pos[3] = 0
    at0 = qo.clone()
    c.qk_norm_rope(q, k, pos, par, qo, ko)
    assert c.sync_status() == sq.SQ_OK and torch.equal(at0, qo)
    c.close()


def test_rows_of_zeros_and_wide_ranges():
    """A zero row stays zero (eps > 0), and rows near the type's limits neither
    overflow nor vanish beyond what fp32 does to their squares."""
    c = sq.Cache(1, 4, 2, 128, 16, 1)
    q = torch.randn(6, 4, 128, device="cuda")
    q[0] = 0
    q[1] *= 1e15
    q[2] *= 1e-12
    q = q.bfloat16()
    k = q[:, :2].contiguous()
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    c.qk_norm_rope(q, k, None, sq.norm_rope(eps=1e-6), qo, ko)
    assert c.sync_status() == sq.SQ_OK
    assert (qo[0] == 0).all() and (ko[0] == 0).all()
    assert_rounded(qo, *reference(q, None, 1e-6, None, None, 0, False))
    c.close()


def test_refusals():
    c = sq.Cache(2, 4, 2, 64, 16, 40)
    q, k, v, w, table, pos, _ = inputs(4, 2, 64, 8, 32, 1)
    par = sq.norm_rope(table, 32, 1e-6, *w)
    qo = torch.empty(8, 4, 64, dtype=torch.bfloat16, device="cuda")
    ko = torch.empty(8, 2, 64, dtype=torch.bfloat16, device="cuda")

    def refused(code, f, *a, **kw):
        with pytest.raises(sq.SqError) as e:
            f(*a, **kw)
        assert e.value.code == code

    bad = sq.SQ_ERR_INVALID_ARG
    fwd = c.qk_norm_rope
    refused(bad, fwd, q, k, None, par, qo, ko)                       # no positions
    for change in (dict(rot_dim=24), dict(rot_dim=-16), dict(rot_dim=80), dict(eps=float("nan")),
                   dict(eps=-1.0), dict(max_pos=0), dict(rope=None), dict(weight_dtype=2),
                   dict(q_weight=w[0].data_ptr() + 2)):
        p2 = sq.norm_rope(table, 32, 1e-6, *w)
        for name, x in change.items():
            setattr(p2, name, x)
        refused(bad, fwd, q, k, pos, p2, qo, ko)
    h = c.handle
    refused(bad, sq.sq_qk_norm_rope, h, 8, q, 250, k, 128, pos, par, qo, ko)       # row overlaps the next
    refused(bad, sq.sq_qk_norm_rope, h, 8, q, 260, k, 128, pos, par, qo, ko)       # not a multiple of 8
    refused(bad, sq.sq_qk_norm_rope, h, 8, q.data_ptr() + 2, 512, k, 512, pos, par, qo, ko)
    refused(bad, sq.sq_qk_norm_rope, h, -1, q, 512, k, 512, pos, par, qo, ko)
    refused(bad, sq.sq_qk_norm_rope, h, 8, q, 512, k, 512, pos, par, qo, qo)       # outputs overlap
    cq = q.contiguous()
    refused(bad, fwd, cq, k, pos, par, cq, ko)                                     # in place
    with pytest.raises(ValueError):
        fwd(q[:, :, ::2], k, pos, par, qo, ko)
    with pytest.raises(ValueError):
        fwd(q.float(), k, pos, par, qo, ko)
    with pytest.raises(ValueError):
        fwd(q, k[:5], pos, par, qo, ko)
    with pytest.raises(ValueError):
        sq.norm_rope(table, 32, 1e-6, w[0], w[1].float())
    # backward: gradients that overlap each other, other than as turns of one tensor
    dz, dzk = torch.empty_like(qo), torch.empty_like(ko)
    refused(bad, c.qk_norm_rope_backward, q, k, pos, par, dz, dzk, dz, ko)
    one = torch.empty(8, 6, 64, dtype=torch.bfloat16, device="cuda")
    refused(bad, c.qk_norm_rope_backward, q, k, pos, par, dz, dzk, one[:, :4], one[:, 3:5])
    # store
    a = c.seq_new()
    c.extend([a], [8])
    store = c.qk_norm_rope_store
    refused(bad, store, [a], [8], 2, q, k, v, pos, par, qo)          # layer
    refused(bad, store, [a], [8], 0, q, k, v, pos, par, q.contiguous().data_ptr() + 2)
    refused(bad, sq.sq_qk_norm_rope_store, h, [a], [9], 0, q, 512, k, 512, v, 512, pos, par, qo)  # rows it has not
    refused(bad, sq.sq_qk_norm_rope_store, h, [a, a], [4, 4], 0, q, 512, k, 512, v, 512, pos, par, qo)
    refused(sq.SQ_ERR_BAD_HANDLE, store, [a + 1], [8], 0, q, k, v, pos, par, qo)
    with pytest.raises(ValueError):
        store([a], [7], 0, q, k, v, pos, par, qo)
    f = c.fork_aux(a)
    refused(bad, store, [a], [8], 0, q, k, v, pos, par, qo)          # the fork holds the rows too
    c.release(f)
    store([a], [8], 0, q, k, v, pos, par, qo)
    refused(bad, c.extend, [a, a])
    refused(bad, c.extend, [a], [-1])
    refused(sq.SQ_ERR_CAPACITY, c.extend, [a], [16 * 40])
    n = c.seq_info(a)[0]
    b = c.seq_new()
    refused(sq.SQ_ERR_NO_PAGES, c.extend, [b, a], [16 * 20, 16 * 30])   # all or nothing
    assert c.seq_info(a)[0] == n and c.seq_info(b)[0] == 0 and c.free_pages() == 39
    assert c.sync_status() == sq.SQ_OK
    c.close()
