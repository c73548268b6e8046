"""Single tokens over rows of 8 bits at the ends of what queries, keys and values may be:
the results are those of the values that the cache holds."""
import math

import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests import kv8_reference as ref
from tests.test_gpu_kv8 import append, gen, read, rows

pytestmark = pytest.mark.gpu
LARGEST = 240 * 2.0 ** 120   # that a block holds


def cache_of(hq, hkv, d, page, k, v, ctas=0):
    """A cache with one sequence of these rows, and the rows as they are held.  (ctas:
    of a call; of one its warps have many stages.)"""
    n = k.shape[0]
    c = sq.Cache(1, hq, hkv, d, page, -(-n // page) + 4, bits=8, decode_ctas=ctas)
    h = c.seq_new()
    append(c, h, k.bfloat16()[None], v.bfloat16()[None])
    return c, h, *read(c, h)


def single(c, hs, q, scale):
    out = torch.empty(len(hs), c.Hq, c.D, device="cuda")
    c.decode_attention(hs, 0, q, out, sq.SQ_OUT_F32, scale)
    assert c.sync_status() == sq.SQ_OK
    return out.double()


def rising(g, n, hkv, d, step):
    """Keys whose first dimension rises from -n step / 2 by about `step` a row (held with
    4 significant bits, so that it stays for some rows), the others small."""
    k = torch.randn(n, hkv, d, generator=g, device="cuda") * 0.05
    k[..., 0] = ((torch.arange(n, device="cuda") - n / 2) * step)[:, None]
    return k


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 128, 64), (16, 2, 64, 8), (32, 2, 64, 64), (6, 2, 128, 256)])
@pytest.mark.parametrize("n,size", [(1, 1e36), (1, 1e37), (1, LARGEST), (7, 1e37), (100, 1e36), (300, 1e36)])
@pytest.mark.parametrize("step", [0.0, 0.3, 1.5, 6.0])
@pytest.mark.parametrize("ctas", [0, 1])
def test_values_of_any_size(hq, hkv, d, page, n, size, step, ctas):
    """Values up to the largest that are held, one sign a dimension (so that sums are as
    large as they can be), at logits that rise and bring weights above 1."""
    g = gen(1)
    v = (0.5 + 0.5 * torch.rand(n, hkv, d, generator=g, device="cuda")) * size
    v[:, :, ::2] = size
    v *= torch.where(torch.arange(d, device="cuda") % 3 == 0, -1.0, 1.0)
    c, h, k, v = cache_of(hq, hkv, d, page, rising(g, n, hkv, d, step), v, ctas)
    assert n > 1 or size < LARGEST or (v.abs().amax() == LARGEST)
    q = rows(g, 1, hq, d, 0.0) * 0.1
    q[..., 0] = 1.0
    # (in units of the largest: 64 bits have room, the budget's least term has not)
    got = single(c, [h], q, 1.0) / size
    want, weighted, logits = ref.attention(q, k, v / size, 1.0)
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    c.close()


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 128, 64), (32, 2, 64, 8)])
@pytest.mark.parametrize("n", [1, 9, 700])
@pytest.mark.parametrize("size", [2.0 ** 90, 1e30, 2.0 ** 101, 2.0 ** 120, 2.0 ** 126])
def test_logits_far_below_zero(hq, hkv, d, page, n, size):
    """All logits from -size on down: the key nearest to zero has all the weight.  (They
    differ by a fifth and more of the nearest, and fp32 logits by 2^-16 at most.)"""
    g = gen(2)
    k = torch.zeros(n, hkv, d, device="cuda")
    # 1, 1.25, 1.5 or 1.75 times a power of two: held exactly, in blocks that span 2^8
    k[..., 0] = -torch.randint(5, 7 * 64, (n, hkv), generator=g, device="cuda").float()
    k[..., 0] = torch.round(k[..., 0] / 64) * 64 - 64
    best = int(torch.randint(0, n, (1,), generator=g, device="cuda"))
    k[best, :, 0] = -40.0
    v = rows(g, n, hkv, d).float()
    c, h, k, v = cache_of(hq, hkv, d, page, k * 2.0 ** 20, v)
    q = torch.zeros(1, hq, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 60
    got = single(c, [h], q, size / 2.0 ** 60 / (40 * 2.0 ** 20))
    want = v[best].repeat_interleave(hq // hkv, 0)[None]
    # (its weight is a power of two that fp16 holds: one fp32 division and product)
    assert ((got - want).abs() <= want.abs() * 2.0 ** -20).all()
    c.close()


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 128, 64), (16, 2, 64, 16), (32, 2, 64, 64)])
@pytest.mark.parametrize("big,scale", [(2.0 ** 100, 1.0), (2.0 ** 126, 1.0), (2.0 ** 120, 1e30), (1.0, 3e38)])
def test_keys_of_zeros_beside_large_ones(hq, hkv, d, page, big, scale):
    """Queries and keys whose sizes' product passes fp32, in other dimensions: every logit
    is 0."""
    g = gen(3)
    n = 90
    k = torch.zeros(n, hkv, d, device="cuda")
    k[::3, :, d // 2:] = torch.randn(n // 3, hkv, d // 2, generator=g, device="cuda") * 1e37
    c, h, k, v = cache_of(hq, hkv, d, page, k, rows(g, n, hkv, d).float())
    q = torch.zeros(1, hq, d, dtype=torch.bfloat16, device="cuda")
    q[..., :d // 2] = rows(g, 1, hq, d // 2, 0.0) * big
    got = single(c, [h], q, scale)
    want, weighted, logits = ref.attention(torch.zeros_like(q), k, v, 1.0)
    assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    c.close()


def test_large_queries():
    """Logits of ordinary size from large queries and small keys, and the other way."""
    g = gen(4)
    hq, hkv, d, n = 16, 2, 64, 200
    v = rows(g, n, hkv, d).float()
    for e in (-90, -60, -20, 20, 60, 100):
        c, h, k, vv = cache_of(hq, hkv, d, 16, torch.randn(n, hkv, d, generator=g, device="cuda") * 2.0 ** e, v)
        q = torch.randn(1, hq, d, generator=g, device="cuda").bfloat16() * 2.0 ** -e
        got = single(c, [h], q, d ** -0.5)
        want, weighted, logits = ref.attention(q, k, vv, d ** -0.5)
        assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
        c.close()


@pytest.mark.parametrize("size,scale", [(2.0 ** 100, 2.0 ** 100), (2.0 ** 126, 2.0 ** 120), (1.0, 2.0 ** 127),
                                        (2.0 ** -80, 2.0 ** 126)])
def test_large_scales(size, scale):
    """Factors that pass fp32 where logits do not: the largest logit has all the weight
    (and all the same where the keys are too small for a cache to hold)."""
    g = gen(5)
    hq, hkv, d, n = 8, 2, 128, 150
    k = torch.randint(1, 8, (n, hkv, d), generator=g, device="cuda") * (torch.arange(d, device="cuda") == 3)
    k[77, :, 3] = 14
    e = 100 - math.log2(size) - math.log2(scale)   # logits of 2^100 and more
    c, h, k, v = cache_of(hq, hkv, d, 64, k.double() * 2.0 ** e, rows(g, n, hkv, d).float())
    q = torch.full((1, hq, d), size, dtype=torch.bfloat16, device="cuda")
    got = single(c, [h], q, scale)
    if k.any():
        want = v[77].repeat_interleave(hq // hkv, 0)[None]
        assert ((got - want).abs() <= want.abs() * 2.0 ** -20).all()
    else:
        want, weighted, logits = ref.attention(q, k, v, 1.0)
        assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    c.close()


def share_budget(q, k, v, scale, blocks):
    """What a key may be off by beside its own rounding, for each of n keys: fp16's least
    step is 2^-24, where the row's largest product of a weight and a block's scale is 2^7
    or more.  Half a step of a code of at most 448, and a block's largest value is 224
    scales or more: 2^-31 of the largest product of a weight and such a value (and of the
    normaliser 2^-32 of the largest weight, as much of the output)."""
    m, hq, d = q.shape
    g = hq // k.shape[1]
    most = torch.empty(v.shape[:2], dtype=torch.float64, device=v.device)
    for a, b in blocks:
        most[a:b] = v[a:b].abs().amax((0, 2))
    s = torch.einsum("mhd,nhd->mhn", q.double(), k.repeat_interleave(g, 1)) * scale
    w = torch.softmax(s, -1)
    return k.shape[0] * 2.0 ** -31 * (w * most.repeat_interleave(g, 1).T[None]).amax(-1)[..., None]


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 128, 64), (16, 2, 64, 8), (32, 2, 64, 64), (16, 1, 128, 16)])
@pytest.mark.parametrize("gap", [12, 20, 26, 38, 60, 110])
@pytest.mark.parametrize("far", [0.0, 0.5, 1.0, 1.2, 2.0, math.inf])
@pytest.mark.parametrize("ctas", [0, 1])
def test_blocks_of_values_beside_much_larger_ones(hq, hkv, d, page, gap, far, ctas):
    """Blocks whose values are 2^gap of the others', before, between and after those in
    every warp's share, at weights of 2^-(far gap) of theirs: negligible ones (a weight of
    0 too) take nothing from the others, whatever their size."""
    g = gen(int(100 * min(far, 9)) + gap)
    n = 1100
    q = torch.zeros(1, hq, d, dtype=torch.bfloat16, device="cuda")
    q[..., :] = 0.1 * rows(g, 1, hq, d, 0.0)
    q[..., 0] = 1.0
    k = torch.randn(n, hkv, d, generator=g, device="cuda")
    v = torch.randn(n, hkv, d, generator=g, device="cuda") * 2.0 ** -(gap // 2)
    block = torch.arange(n, device="cuda") // 8
    large = (block % 11 == 3) | (block < 2) & (block % 2 == 0)
    k[..., 0] = torch.where(large, -min(far * gap, 3000.0) * math.log(2.0), 0.0)[:, None]
    v = torch.where(large[:, None, None], v * 2.0 ** gap, v)
    c, h, k, v = cache_of(hq, hkv, d, page, k, v, ctas)
    blocks = ref.blocks_of(c.page_fills(h), page)
    for scale in (1.0, 0.25):
        got = single(c, [h], q, scale)
        want, weighted, logits = ref.attention(q, k, v, scale)
        assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d) +
                share_budget(q, k, v, scale, blocks)).all()
    c.close()


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("ctas", [0, 1])
def test_rows_of_a_pass_keep_their_own_references(d, page, ctas):
    """Query heads of one KV head, and of forks that share pages: some attend to large
    values, some to small ones alone, in turns along the context."""
    hq, hkv, n = 8, 1, 900
    g = gen(7)
    k = torch.randn(n, hkv, d, generator=g, device="cuda") * 0.3
    v = torch.randn(n, hkv, d, generator=g, device="cuda")
    part = torch.arange(n, device="cuda") // 40 % 3
    v *= torch.exp2(torch.tensor([-30.0, 0.0, 30.0], device="cuda")[part])[:, None, None]
    for i in range(3):
        k[:, 0, i] = torch.where(part == i, 0.0, -120.0)
    c, h, k, v = cache_of(hq, hkv, d, page, k, v, ctas)
    f = c.fork_aux(h)
    q = 0.1 * rows(g, 2, hq, d, 0.0)
    q[..., :3] = 0
    for i in range(2):
        for j in range(hq):
            q[i, j, (i + j) % 3] = 1.0
    got = single(c, [h, f], q, 1.0)
    blocks = ref.blocks_of(c.page_fills(h), page)
    want, weighted, logits = ref.attention(q, k, v, 1.0)
    assert ((got - want).abs() <= ref.token_budget(want, weighted, logits, d) +
            share_budget(q, k, v, 1.0, blocks)).all()
    c.close()
