"""An 8-bit cache on the GPU: rows stored, read back, shared, evicted, and attended
to, against a restatement in 64 bits and the bf16 cache of the same values."""
import math

import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

GEOMETRIES = [(8, 2, 128, 64), (16, 4, 64, 16), (8, 1, 64, 8), (6, 2, 128, 256), (32, 2, 64, 32), (4, 4, 128, 8)]


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def rows(g, n, heads, d, spread=1.0):
    """bf16 rows whose sizes differ by token and head."""
    x = torch.randn(n, heads, d, generator=g, device="cuda")
    x *= torch.exp(spread * torch.randn(n, heads, 1, generator=g, device="cuda"))
    return x.bfloat16()


def read(cache, h, n=None, layer=0):
    n = cache.seq_info(h)[0] if n is None else n
    k, v = (torch.full((n, cache.Hkv, cache.D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read_kv([h], [n], layer, k, v)
    return k.double(), v.double()


def blocks(cache, h):
    return ref.blocks_of(cache.page_fills(h), cache.P)


def same(got, want):
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


def append(cache, h, k, v):
    """k, v [L, n, Hkv, D]"""
    cache.append_kv(h, k.shape[1], k.contiguous(), v.contiguous())


def scales_of(cache, h, layer=0):
    """Every row's scales of keys and values, [n, Hkv] each."""
    s, pages, out = cache.scale_view()[layer], cache.page_table(h), []
    for p, f in zip(pages, cache.page_fills(h)):
        out.append(s[p].repeat_interleave(8, -1)[..., :f])
    return torch.cat(out, -1).double().permute(0, 2, 1)


def same_scales(got, rows, blocks):
    """Scales [n, hkv] of rows as they are held: the least that they need, or, where the
    largest was rounded down to 448 of it, twice that."""
    for a, b in blocks:
        size = torch.nan_to_num(rows[a:b].abs(), nan=0.0).amax((0, 2))
        want = ref.scale_of(size)
        s = got[a]
        assert (got[a:b] == s).all()
        assert ((s == want) | ((s == 2 * want) & (size == 448 * want))).all()


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
def test_appended_rows(hq, hkv, d, page):
    """Rows that come together, one by one, and in a batch: every block is held as its
    rows with the scale of them together."""
    c = sq.Cache(2, hq, hkv, d, page, 200, bits=8)
    g = gen(1)
    h, other = c.seq_new(), c.seq_new()
    k, v = (torch.stack([rows(g, 75, hkv, d, 2.0) for _ in range(2)]) for _ in range(2))
    append(c, h, k[:, :13], v[:, :13])
    append(c, other, k[:, :5], v[:, :5])
    want = {(l, p): ref.held(x[l, :13].double(), blocks(c, h))[0] for l in range(2) for p, x in enumerate((k, v))}
    for l in range(2):
        for p, got in enumerate(read(c, h, layer=l)):
            same(got, want[l, p])
    for i in range(13, 40):
        kk, vv = (torch.stack([x[:, i], x[:, i - 8]], 1).contiguous() for x in (k, v))
        c.append_kv_batch([h, other], kk, vv)
        for l in range(2):
            for p, x in enumerate((k, v)):
                new = torch.cat([want[l, p], x[l, i:i + 1].double()])
                want[l, p] = ref.held(new, blocks(c, h))[0]
    append(c, h, k[:, 40:], v[:, 40:])
    for l in range(2):
        for p, x in enumerate((k, v)):
            want[l, p], _ = ref.held(torch.cat([want[l, p], x[l, 40:].double()]), blocks(c, h))
            same(read(c, h, layer=l)[p], want[l, p])
            same_scales(scales_of(c, h, l)[p], want[l, p], blocks(c, h))
        same(read(c, h, 9, l)[0], want[l, 0][-9:])
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
@pytest.mark.parametrize("pairs,f32", [(False, False), (True, True)])
def test_stored_rows(hq, hkv, d, page, pairs, f32):
    """The store with norms and rotation: queries as the bf16 cache has them, values
    exactly, keys to half a step of their code."""
    g = gen(2)
    rot = d // 2 if pairs else d
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.float32 if f32 else torch.bfloat16)
         for _ in range(2)]
    table = sq.rope_table(4096, rot)
    params = sq.norm_rope(table, rot, 1e-6, *w, interleaved=pairs)
    c, wide = (sq.Cache(1, hq, hkv, d, page, 400, bits=b) for b in (8, 16))
    for counts in ([1, 1, 1], [37, 1, 0], [300, 8, 70], [1, 7, 2]):
        if page == 8 and max(counts) == 300:
            counts = [1100, 600, 200]   # more blocks than go with a launch
        hs = [[x.seq_new() for _ in counts] for x in (c, wide)]
        pre = [5, 16, 0]
        for cache, h in zip((c, wide), hs):
            kv = rows(gen(3), 16, hkv, d)[None]
            for x, n in zip(h, pre):
                if n:
                    append(cache, x, kv[:, :n], kv[:, :n])
        held0 = [read(c, x) if n else None for x, n in zip(hs[0], pre)]
        n = sum(counts)
        qkv = rows(g, n, hq + 2 * hkv, d, 1.5)
        q, k, v = qkv.split([hq, hkv, hkv], 1)
        outs = []
        for cache, h in zip((c, wide), hs):
            cache.extend(h, counts)
            outs.append(torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda"))
            for _ in range(2):     # (a second store of the same rows changes nothing)
                cache.qk_norm_rope_store(h, counts, 0, q, k, v, None, params, outs[-1])
        assert torch.equal(*outs)
        at = 0
        for x, m, n0, old in zip(hs[0], counts, pre, held0):
            if m == 0:
                continue
            pos = torch.arange(n0, n0 + m, device="cuda")
            x64 = k[at:at + m].double()
            y = x64 / torch.sqrt(x64.square().mean(-1, keepdim=True) + 1e-6) * w[1].double()
            cs = torch.complex(*table[pos].double().unbind(-1))[:, None]
            i = torch.arange(rot // 2, device="cuda") * (2 if pairs else 1)
            j = i + (1 if pairs else rot // 2)
            z = torch.complex(y[..., i], y[..., j]) * cs
            y[..., i], y[..., j] = z.real, z.imag
            got_k, got_v = read(c, x)
            start = torch.zeros(0, hkv, d, device="cuda", dtype=torch.float64) if old is None else old[1]
            want_v, _ = ref.held(torch.cat([start, v[at:at + m].double()]), blocks(c, x))
            same(got_v, want_v)
            sk = scales_of(c, x)[0][n0:]
            # half a step of the code, and fp32: sums of d squares, a root, three factors
            # and a sum of two products (d / 2 + 16 roundings of 2^-24 of a row's size)
            size = y.abs().amax(-1, keepdim=True)
            half = torch.maximum(y.abs() * 2.0 ** -4, sk[..., None] * 2.0 ** -10)
            assert ((got_k[n0:] - y).abs() <= half * (1 + 2.0 ** -12) + size * (d / 2 + 16) * 2.0 ** -24).all()
            same_scales(scales_of(c, x)[0], got_k, blocks(c, x))
            same_scales(scales_of(c, x)[1], got_v, blocks(c, x))
            at += m
        for cache, h in zip((c, wide), hs):
            for x in h:
                cache.release(x)
    assert c.sync_status() == sq.SQ_OK and wide.sync_status() == sq.SQ_OK


def test_sizes_at_the_ends():
    """Blocks of zeros, of the largest and smallest values, infinities and NaN."""
    c = sq.Cache(1, 4, 2, 64, 16, 20, bits=8)
    h = c.seq_new()
    x = torch.zeros(40, 2, 64)
    x[8:16] = torch.randn(8, 2, 64) * 1e38
    x[16:24] = torch.randn(8, 2, 64) * 1e-36
    x[24:32] = torch.randn(8, 2, 64)
    x[25, 0, 3], x[26, 0, 4], x[27, 1, 5] = math.inf, -math.inf, math.nan
    x[32:40] = 448.0
    x[33, 1, 0] = 449.0
    x = x.bfloat16().cuda()
    append(c, h, x[None], x[None])
    want, s = ref.held(x.double(), blocks(c, h))
    for got in read(c, h):
        same(got, want)
    assert torch.equal(scales_of(c, h)[0], s)
    assert s[0, 0] == 2.0 ** -100 and s[33, 0] == 1.0 and s[33, 1] == 1.0   # (449 is 448 in bf16)
    assert c.sync_status() == sq.SQ_OK


def test_scales_at_the_borders():
    """Sizes next to 448 times a power of two, from the smallest scale to the largest."""
    c = sq.Cache(1, 4, 2, 64, 16, 60, bits=8)
    h = c.seq_new()
    sizes = [448.0, 450.0, 446.0, 1.75, 1.7578125, 2.0 ** -100 * 448, 2.0 ** -100 * 450, 2.0 ** -92 * 1.5,
             2.0 ** -106, 2.0 ** -109, 2.0 ** -110, 2.0 ** 127 * 1.75, 2.0 ** 127 * 1.9375, 2.0 ** 127 * 1.9921875]
    x = torch.rand(8 * len(sizes), 2, 64, dtype=torch.float64) * 0.9
    for i, size in enumerate(sizes):
        x[8 * i + i % 8, 0, i] = 1.0
        x[8 * i + 3, 1, 63] = -1.0
        x[8 * i:8 * i + 8] *= size
    x = x.float().bfloat16().cuda()
    append(c, h, x[None], x[None])
    want, s = ref.held(x.double(), blocks(c, h))
    for got in read(c, h):
        same(got, want)
    assert torch.equal(scales_of(c, h)[0], s)
    assert c.sync_status() == sq.SQ_OK


def fill_sequences(c, lengths, seed, garbage=True):
    """Sequences of these lengths, their pages in turns; the pool's other slots hold
    NaN codes and NaN scales."""
    if garbage:
        c.pool_view().view(torch.uint8).fill_(0x7f)
        c.scale_view().fill_(math.nan)
    g = gen(seed)
    hs = [c.seq_new() for _ in lengths]
    left = list(lengths)
    while any(left):
        for i, h in enumerate(hs):
            n = min(left[i], 3 * c.P + 5)
            if n:
                k, v = (torch.stack([rows(g, n, c.Hkv, c.D, 0.7) for _ in range(c.L)]) for _ in range(2))
                append(c, h, k, v)
                left[i] -= n
    return hs


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4), (1, 0), (700, 9)])
def test_single_tokens(hq, hkv, d, page, window, sinks):
    lengths = [1, 8, 63, 64, 65, 700, 2049]
    c = sq.Cache(2, hq, hkv, d, page, sum(-(-n // page) for n in lengths) + 40, bits=8)
    hs = fill_sequences(c, lengths, 5)
    q = rows(gen(6), len(hs), hq, d, 0.5)
    scale = d ** -0.5
    out, half = torch.empty(len(hs), hq, d, device="cuda"), torch.empty_like(q)
    c.window_attention(hs, None, 1, q, out, window, sinks, out_dtype=sq.SQ_OUT_F32, sm_scale=scale)
    c.window_attention(hs, None, 1, q, half, window, sinks, sm_scale=scale)
    assert c.sync_status() == sq.SQ_OK
    assert torch.equal(out.bfloat16(), half)
    for i, (h, n) in enumerate(zip(hs, lengths)):
        k, v = read(c, h, layer=1)
        j = torch.arange(n, device="cuda")
        keep = ((j > n - 1 - window) | (j < sinks) if window else j >= 0)[None]
        want, weighted, logits = ref.attention(q[i:i + 1], k, v, scale, keep)
        assert ((out[i:i + 1].double() - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()


def test_values_of_very_different_sizes():
    """Blocks of values from 2^-60 to 2^40, the large ones far off by their logits or
    near: outputs to fp16 weights' accuracy of what dominates them."""
    hq, hkv, d = 4, 1, 128
    c = sq.Cache(1, hq, hkv, d, 64, 20, bits=8)
    h = c.seq_new()
    g = gen(8)
    n = 512
    k = rows(g, n, 1, d, 0.3)
    v = torch.randn(n, 1, d, generator=g, device="cuda")
    v *= torch.exp2(torch.arange(n, device="cuda").div(8, rounding_mode="floor") % 26 * 4.0 - 60)[:, None, None]
    append(c, h, k[None], v.bfloat16()[None])
    kk, vv = read(c, h)
    for size in (1e-30, 1.0, 1e30):
        q = (rows(g, 1, hq, d) * size).bfloat16()
        out = torch.empty(1, hq, d, device="cuda")
        c.decode_attention([h], 0, q, out, sq.SQ_OUT_F32, d ** -0.5 / size)
        want, weighted, logits = ref.attention(q, kk, vv, d ** -0.5 / size)
        assert ((out.double() - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    assert c.sync_status() == sq.SQ_OK


def wide_twin(c, pages):
    """A bf16 cache of the same geometry whose pool holds the values of c's."""
    codes, scales = c.pool_view(), c.scale_view()
    values = codes.float() * scales.repeat_interleave(8, -1)[..., None]
    pool = values.bfloat16().contiguous()
    return sq.Cache(c.L, c.Hq, c.Hkv, c.D, c.P, pages, kv_pool=pool), pool


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
def test_query_blocks_are_those_of_the_values(hq, hkv, d, page):
    """Prompts, chunks and trees of one tile a sequence or of more than three: bit for
    bit the bf16 cache's outputs over the same values."""
    lengths = [300, 64, 9, 1500]
    pages = sum(-(-n // page) for n in lengths) + 8
    c = sq.Cache(2, hq, hkv, d, page, pages, bits=8)
    hs = fill_sequences(c, lengths, 9)
    twin, _pool = wide_twin(c, pages)
    other = [twin.seq_new() for _ in lengths]
    left = list(lengths)
    while any(left):     # (the same pages)
        for i, h in enumerate(other):
            n = min(left[i], 3 * page + 5)
            twin.extend([h], [n])
            left[i] -= n
    assert [c.page_table(h) for h in hs] == [twin.page_table(h) for h in other]
    scale = d ** -0.5
    tile = 128 // (hq // hkv)
    for counts, window, sinks in (([300, 64, 9, 1500], 0, 0), ([1, 3, 9, 3 * tile + 2], 100, 5),
                                  ([0, 2, 1, min(40, tile)], 0, 0)):
        q = rows(gen(10), sum(counts), hq, d, 0.5)
        outs = [torch.empty_like(q) for _ in range(2)]
        lses = [torch.empty(q.shape[0], hq, device="cuda") for _ in range(2)]
        for cache, h, out, lse in zip((c, twin), (hs, other), outs, lses):
            for _ in range(2):
                cache.window_attention(h, counts, 1, q, out, window, sinks, lse=lse, sm_scale=scale)
        assert torch.equal(*outs) and torch.equal(*lses)
        assert not outs[0].isnan().any()
    counts = [min(17, tile), 1, 5, min(33, tile)]
    parents = [max(-1, j - 1 - j % 3) for m in counts for j in range(m)]
    q = rows(gen(11), sum(counts), hq, d, 0.5)
    outs = [torch.empty_like(q) for _ in range(2)]
    for cache, h, out in zip((c, twin), (hs, other), outs):
        cache.tree_attention(h, counts, parents, 1, q, out, sm_scale=scale)
    assert torch.equal(*outs)
    assert c.sync_status() == sq.SQ_OK and twin.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
@pytest.mark.parametrize("ragged", [False, True])
def test_eviction(hq, hkv, d, page, ragged):
    """Kept rows in the blocks that they are in now, of a sequence alone and of one that
    shares its pages with a fork, which keeps its own."""
    c = sq.Cache(2, hq, hkv, d, page, 1200, bits=8)
    h, = fill_sequences(c, [1003], 12)
    f = c.fork_aux(h)
    kept_f = [read(c, f, layer=l) for l in range(2)]
    g = gen(13)
    for spans in ([(3, 9), (100, 131), (500, 731), (770, 771)], [(0, 1)], [(50, 200), (330, 333)], [(390, 400)]):
        n = c.seq_info(h)[0]
        spans = [(a, min(b, n)) for a, b in spans if a < n]
        before = [read(c, h, layer=l) for l in range(2)]
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        for a, b in spans:
            keep[a:b] = False
        (c.evict_spans_ragged if ragged else c.evict_spans)(h, spans)
        assert c.seq_info(h)[0] == int(keep.sum())
        for l in range(2):
            for p in range(2):
                want, _ = ref.held(before[l][p][keep], blocks(c, h))
                same(read(c, h, layer=l)[p], want)
                same_scales(scales_of(c, h, l)[p], want, blocks(c, h))
                same(read(c, f, layer=l)[p], kept_f[l][p])
        # rows go on behind
        k, v = (torch.stack([rows(g, 11, hkv, d, 1.0) for _ in range(2)]) for _ in range(2))
        old = [read(c, h, layer=l) for l in range(2)]
        append(c, h, k, v)
        for l in range(2):
            for p, x in enumerate((k, v)):
                same(read(c, h, layer=l)[p], ref.held(torch.cat([old[l][p], x[l].double()]), blocks(c, h))[0])
    # both go on, and are attended to together
    append(c, f, k, v)
    q = rows(g, 2, hq, d, 0.5)
    out = torch.empty(2, hq, d, device="cuda")
    c.decode_attention([h, f], 1, q, out, sq.SQ_OUT_F32, d ** -0.5)
    for i, x in enumerate((h, f)):
        kk, vv = read(c, x, layer=1)
        want, weighted, logits = ref.attention(q[i:i + 1], kk, vv, d ** -0.5)
        assert ((out[i:i + 1].double() - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    blk = torch.empty(10, hq, d, dtype=torch.bfloat16, device="cuda")
    q = rows(g, 10, hq, d, 0.5)
    c.window_attention([h, f], [5, 5], 1, q, blk, 300, 4, sm_scale=d ** -0.5)
    for i, x in enumerate((h, f)):
        kk, vv = read(c, x, layer=1)
        n = kk.shape[0]
        p, j = torch.arange(n - 5, n, device="cuda")[:, None], torch.arange(n, device="cuda")
        keep = (j <= p) & ((j > p - 300) | (j < 4))
        want, weighted, logits = ref.attention(q[5 * i:5 * i + 5], kk, vv, d ** -0.5, keep)
        # bf16 weights (2^-8 each way) and the output's own rounding (2^-8 at most)
        off = (blk[5 * i:5 * i + 5].double() - want).abs()
        assert (off <= weighted * 2.0 ** -7 + want.abs() * 2.0 ** -8 +
                weighted * (2.0 * (d + 8) * 2.0 ** -24 * logits)[..., None]).all()
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16)])
def test_eviction_joins_rows_of_very_different_scales(d, page):
    """Blocks of sizes from 2^-90 to 2^90, packed together."""
    c = sq.Cache(1, 4, 2, d, page, 100, bits=8)
    h = c.seq_new()
    g = gen(31)
    n = 640
    x = torch.randn(n, 2, d, generator=g, device="cuda")
    size = torch.randint(-90, 90, (n // 8, 2), generator=g, device="cuda")
    size[::3] = torch.randint(-20, 20, (len(size[::3]), 2), generator=g, device="cuda")
    x = (x * torch.exp2(size.float()).repeat_interleave(8, 0)[..., None]).bfloat16()
    x[17, 0, 5], x[100, 1, 7] = math.nan, math.inf
    append(c, h, x[None], x[None])
    before = read(c, h)
    spans = [(i, i + 5) for i in range(2, n - 10, 13)]
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    for a, b in spans:
        keep[a:b] = False
    c.evict_spans(h, spans)
    for p in range(2):
        want, _ = ref.held(before[p][keep], blocks(c, h))
        same(read(c, h)[p], want)
        same_scales(scales_of(c, h)[p], want, blocks(c, h))
    assert c.sync_status() == sq.SQ_OK


def test_drafted_step():
    """Extension, store, tree, acceptance, then single tokens: the calls of a decode
    step together, in two layers."""
    hq, hkv, d, page = 8, 2, 128, 64
    c = sq.Cache(2, hq, hkv, d, page, 40, bits=8)
    hs = fill_sequences(c, [130, 61], 14)
    g = gen(15)
    params = sq.norm_rope(sq.rope_table(1024, d), d, 1e-6)
    counts, parents = [5, 3], [-1, 0, 0, 1, 2, -1, 0, 1]
    ctx = [c.seq_info(h)[0] for h in hs]
    c.extend(hs, counts)
    for l in range(2):
        q, k, v = rows(g, 8, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
        q_out, out = torch.empty(8, hq, d, dtype=torch.bfloat16, device="cuda"), None
        out = torch.empty_like(q_out)
        c.qk_norm_rope_store(hs, counts, l, q, k, v, None, params, q_out)
        c.tree_attention(hs, counts, parents, l, q_out, out, sm_scale=d ** -0.5)
        at = 0
        for h, m, n0 in zip(hs, counts, ctx):
            kk, vv = read(c, h, layer=l)
            keep = torch.ones(m, n0 + m, dtype=torch.bool, device="cuda")
            for i in range(m):
                line, p = {i}, parents[at + i]
                while p >= 0:
                    line.add(p)
                    p = parents[at + p]
                for j in range(m):
                    keep[i, n0 + j] = j in line
            want, weighted, logits = ref.attention(q_out[at:at + m], kk, vv, d ** -0.5, keep)
            off = (out[at:at + m].double() - want).abs()
            assert (off <= weighted * 2.0 ** -7 + want.abs() * 2.0 ** -8 +
                    weighted * (2.0 * (d + 8) * 2.0 ** -24 * logits)[..., None]).all()
            at += m
    before = read(c, hs[0])
    c.accept_draft(hs[0], 5, [0, 2, 4])
    idx = torch.tensor(list(range(130)) + [130, 132, 134], device="cuda")
    for p in range(2):
        same(read(c, hs[0])[p], ref.held(before[p][idx], blocks(c, hs[0]))[0])
    assert c.sync_status() == sq.SQ_OK


def test_captured_step():
    """A store, single tokens and a query block in a graph, run over new inputs."""
    hq, hkv, d, page = 8, 2, 64, 32
    c = sq.Cache(1, hq, hkv, d, page, 60, bits=8)
    hs = fill_sequences(c, [300, 77], 16)
    params = sq.norm_rope(None, 0, 1e-6)
    c.extend(hs, [2, 2])
    qkv = rows(gen(17), 4, hq + 2 * hkv, d)
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    q_out = torch.empty(4, hq, d, dtype=torch.bfloat16, device="cuda")
    one, blk = torch.empty(2, hq, d, device="cuda"), torch.empty(4, hq, d, device="cuda")
    kb, vb = (torch.empty(4, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        c.qk_norm_rope_store(hs, [2, 2], 0, q, k, v, None, params, q_out)
        c.window_attention(hs, None, 0, q_out[:2], one, 100, 4, out_dtype=sq.SQ_OUT_F32, sm_scale=0.1)
        c.window_attention(hs, [2, 2], 0, q_out, blk, 100, 4, out_dtype=sq.SQ_OUT_F32, sm_scale=0.1)
        c.read_kv(hs, [2, 2], 0, kb, vb)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
    for seed in (18, 19):
        qkv.copy_(rows(gen(seed), 4, hq + 2 * hkv, d))
        torch.cuda.synchronize()
        for x in (q_out, one, blk, kb, vb):
            x.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (q_out, one, blk, kb, vb)]
        with torch.cuda.stream(s):
            step()
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (q_out, one, blk, kb, vb)))
        same(vb.double(), torch.cat([read(c, h, 2)[1] for h in hs]))
    assert c.sync_status() == sq.SQ_OK


def test_streams_take_turns():
    """Two streams with query blocks of different sizes and plans."""
    hq, hkv, d, page = 8, 2, 128, 64
    c = sq.Cache(1, hq, hkv, d, page, 200, bits=8)
    hs = fill_sequences(c, [2000, 5000], 20)
    q = rows(gen(21), 700, hq, d, 0.5)
    want = []
    for h, m in zip(hs, (200, 700)):
        out = torch.empty(m, hq, d, dtype=torch.bfloat16, device="cuda")
        c.window_attention([h], [m], 0, q[:m], out, 0, sm_scale=d ** -0.5)
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        outs = [torch.zeros_like(x) for x in want]
        torch.cuda.synchronize()
        for h, m, s, out in zip(hs, (200, 700), streams, outs):
            c.window_attention([h], [m], 0, q[:m], out, 0, sm_scale=d ** -0.5, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
    assert c.sync_status() == sq.SQ_OK


def test_rows_of_a_bf16_cache():
    c = sq.Cache(2, 8, 2, 64, 16, 90)
    h = c.seq_new()
    k, v = (torch.stack([rows(gen(s), 77, 2, 64) for _ in range(2)]) for s in (1, 2))
    append(c, h, k, v)
    c.evict_spans_ragged(h, [(5, 9), (40, 41)])
    keep = [i for i in range(77) if not (5 <= i < 9 or i == 40)]
    for l in range(2):
        same(read(c, h, layer=l)[0], k[l, keep].double())
        same(read(c, h, 30, l)[1], v[l, keep].double()[-30:])
    assert c.sync_status() == sq.SQ_OK


def test_noalloc_tokens():
    c = sq.Cache(1, 8, 2, 128, 64, 60, bits=8)
    hs = fill_sequences(c, [900, 70], 22)
    q = rows(gen(23), 2, 8, 128, 0.5)
    outs = [torch.empty(2, 8, 128, device="cuda") for _ in range(2)]
    c.decode_attention(hs, 0, q, outs[0], sq.SQ_OUT_F32, 0.1)
    sq.sq_decode_attention_noalloc(c.handle, hs, 0, q, outs[1], sq.SQ_OUT_F32, 0.1)
    assert torch.equal(*outs)
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 64), (16, 4, 64, 16), (8, 1, 64, 8), (32, 2, 128, 32)])
def test_tokens_of_forks(hq, hkv, d, page):
    """Sequences that share pages, more of them than a tile's columns, each grown by rows
    of its own: a block that a fork copies and scales anew leaves the others' as it was."""
    c = sq.Cache(1, hq, hkv, d, page, 3000 // page + 400, bits=8)
    hs = fill_sequences(c, [1500 + page // 2 + 3, 70], 30)
    g = gen(31)
    for i in range(7):
        hs.append(c.fork_aux(hs[0]))
    before = read(c, hs[0])
    for i, h in enumerate(hs):
        if i % 3 != 2:
            k, v = (rows(g, 1 + 3 * i, hkv, d, 1.0)[None] * 2.0 ** (i - 4) for _ in range(2))
            append(c, h, k, v)
    same(read(c, hs[2])[0], before[0])   # (shared, and not grown)
    same(read(c, hs[2])[1], before[1])
    q = rows(gen(32), len(hs), hq, d, 0.5)
    out = torch.empty(len(hs), hq, d, device="cuda")
    for _ in range(2):
        out.fill_(3.0)
        c.decode_attention(hs, 0, q, out, sq.SQ_OUT_F32, d ** -0.5)
    for i, h in enumerate(hs):
        want, weighted, logits = ref.attention(q[i:i + 1], *read(c, h), d ** -0.5)
        assert ((out[i:i + 1].double() - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 8), (4, 4, 64, 256), (16, 1, 64, 64)])
def test_tokens_of_long_contexts(hq, hkv, d, page):
    """Many pieces to a row; one token more at a time on a kept plan."""
    n = 20011
    c = sq.Cache(1, hq, hkv, d, page, n // page + 60, bits=8)
    h = fill_sequences(c, [n], 33)[0]
    g = gen(34)
    for i in range(4):
        q = rows(g, 1, hq, d, 0.5)
        out = torch.empty(1, hq, d, device="cuda")
        c.decode_attention([h], 0, q, out, sq.SQ_OUT_F32, d ** -0.5)
        want, weighted, logits = ref.attention(q, *read(c, h), d ** -0.5)
        assert ((out.double() - want).abs() <= ref.token_budget(want, weighted, logits, d)).all()
        k, v = (rows(g, 1, hkv, d)[None] * 4.0 ** i for _ in range(2))
        append(c, h, k, v)
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16), (128, 8)])
def test_rows_of_nan(d, page):
    """A row of NaN and of infinities counts for the queries that see it, and for no other."""
    hq, hkv, n, bad = 8, 2, 400, 333
    c = sq.Cache(1, hq, hkv, d, page, n // page + 8, bits=8)
    h = c.seq_new()
    g = gen(35)
    k, v = (rows(g, n, hkv, d, 0.5) for _ in range(2))
    v[bad, 0, 3], v[bad, 1, 5] = math.nan, math.inf
    append(c, h, k[None], v[None])
    q = rows(g, n, hq, d, 0.5)
    kk, vv = read(c, h)
    assert vv[bad].isnan().sum() == 2
    for m, window, sinks in ((n, 50, 0), (80, 30, 7), (20, 40, 0)):
        out = torch.empty(m, hq, d, dtype=torch.bfloat16, device="cuda")
        c.window_attention([h], [m], 0, q[:m], out, window, sinks, sm_scale=d ** -0.5)
        i, j = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        keep = (j <= i) & ((j > i - window) | (j < sinks))
        want, weighted, logits = ref.attention(q[:m], kk, torch.nan_to_num(vv, nan=0.0), d ** -0.5, keep)
        sees = keep[:, bad]
        assert out[sees][:, :4, 3].isnan().all() and out[sees][:, 4:, 5].isnan().all()
        off = (out.double() - want).abs()
        fits = off <= (weighted * 2.0 ** -7 + want.abs() * 2.0 ** -8 +
                       weighted * (2.0 * (d + 8) * 2.0 ** -24 * logits)[..., None])
        fits[sees, :4, 3] = fits[sees, 4:, 5] = True
        assert fits.all()
    one = torch.empty(1, hq, d, device="cuda")
    for window, sinks, seen in ((n - bad, 0, True), (n - bad - 1, 0, False), (3, bad + 1, True), (3, bad, False)):
        c.window_attention([h], None, 0, q[:1], one, window, sinks, out_dtype=sq.SQ_OUT_F32, sm_scale=d ** -0.5)
        assert one[0, :4, 3].isnan().all() == seen and one[0, 4:, 5].isnan().all() == seen
        one[0, :4, 3] = one[0, 4:, 5] = 0.0
        assert one.isfinite().all()
    assert c.sync_status() == sq.SQ_OK


def test_calls_of_no_rows():
    c = sq.Cache(1, 8, 2, 64, 16, 20, bits=8)
    hs = fill_sequences(c, [20, 5], 36)
    before = [read(c, h)[0] for h in hs]
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    c.read_kv(hs, [0, 0], 0, none, none)
    c.append_kv(hs[0], 0, none, none)
    c.extend(hs, [0, 0])
    out = torch.full((2, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    c.read_kv(hs, [0, 1], 0, out[:1], out[1:])
    same(out[0].double(), before[1][-1])
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16)])
def test_an_unsignalled_stage_runs_out(d, page):
    """A bounded wait that runs out is reported, and the cache works on."""
    c = sq.Cache(1, 8, 2, d, page, 4000 // page, bits=8)
    h = fill_sequences(c, [3000], 37)[0]
    q = rows(gen(38), 1, 8, d, 0.5)
    outs = [torch.empty(1, 8, d, device="cuda") for _ in range(2)]
    c.decode_attention([h], 0, q, outs[0], sq.SQ_OUT_F32, 0.1)
    assert c.sync_status() == sq.SQ_OK
    sq.sq_debug_set(c.handle, sq.SQ_DEBUG_DROP_DECODE_STAGE)
    c.decode_attention([h], 0, q, outs[1], sq.SQ_OUT_F32, 0.1)
    assert c.sync_status() == sq.SQ_ERR_DEVICE_TIMEOUT
    for _ in range(2):
        outs[1].fill_(3.0)
        c.decode_attention([h], 0, q, outs[1], sq.SQ_OUT_F32, 0.1)
        assert torch.equal(*outs)
    k, v = (rows(gen(39), 5, 2, d)[None] for _ in range(2))
    append(c, h, k, v)
    c.evict_spans(h, [(10, 500)])
    assert read(c, h)[0].isfinite().all() and c.sync_status() == sq.SQ_OK


def all_calls(c, h, seed):
    """Every call of a step over a sequence of 500 rows; what they give."""
    g = gen(seed)
    hq, hkv, d = c.Hq, c.Hkv, c.D
    k, v = (torch.stack([rows(g, 500, hkv, d, 0.7) for _ in range(c.L)]) for _ in range(2))
    append(c, h, k, v)
    layer, outs = c.L - 1, []
    c.extend([h], [9])
    q, k, v = rows(g, 9, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
    q_out = torch.empty(9, hq, d, dtype=torch.bfloat16, device="cuda")
    c.qk_norm_rope_store([h], [9], layer, q, k, v, None, sq.norm_rope(sq.rope_table(600, d), d, 1e-6), q_out)
    outs.append(q_out)
    f = c.fork_aux(h)
    append(c, f, *(rows(g, c.L * 3, hkv, d).view(c.L, 3, hkv, d) for _ in range(2)))
    for x in (h, f):
        for m in (1, 9, 400):
            q = rows(g, m, hq, d, 0.5)
            outs.append(torch.empty_like(q))
            c.window_attention([x], [m], layer, q, outs[-1], 0, sm_scale=d ** -0.5)
    c.release(f)
    c.evict_spans(h, [(13, 77), (300, 301)])
    outs.append(torch.empty(9, hq, d, dtype=torch.bfloat16, device="cuda"))
    c.tree_attention([h], [9], [max(-1, j - 2) for j in range(9)], layer, q_out, outs[-1], sm_scale=d ** -0.5)
    c.accept_draft(h, 9, [0, 2, 4])
    outs += [x.clone() for x in read(c, h, layer=layer)]
    assert c.sync_status() == sq.SQ_OK
    return outs


@pytest.mark.parametrize("hq,hkv,d,page", [(32, 8, 128, 64), (16, 4, 64, 16)])
def test_pages_far_into_a_pool(hq, hkv, d, page):
    """Offsets past 32 bits: the same bits as at a small pool's start."""
    per = 2 * hkv * page * d
    pages = (5 << 30) // (2 * per)
    big, small = (sq.Cache(2, hq, hkv, d, page, n, bits=8) for n in (pages, 900 // page + 60))
    filler = big.seq_new()
    big.extend([filler], [(pages - 900 // page - 60) * page])
    want, got = (all_calls(c, c.seq_new(), 40) for c in (small, big))
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_a_pool_of_the_callers():
    hq, hkv, d, page, pages = 8, 2, 128, 64, 30
    cfg = sq.make_config(2, hq, hkv, d, page, pages)
    pool = torch.full((sq.sq_pool_bytes_8bit(cfg),), 0x7f, dtype=torch.uint8, device="cuda")
    given, own = sq.Cache(2, hq, hkv, d, page, pages, kv_pool=pool, bits=8), sq.Cache(2, hq, hkv, d, page, pages, bits=8)
    assert sq.sq_pool_ptr(given.handle) == pool.data_ptr()
    hs = [c.seq_new() for c in (given, own)]
    want, got = (all_calls(c, h, 41) for c, h in zip((own, given), hs))
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    # rows that the caller writes: the other cache's
    given.pool_view().view(torch.uint8).copy_(own.pool_view().view(torch.uint8))
    given.scale_view().copy_(own.scale_view())
    for x, y in zip(read(given, hs[0]), read(own, hs[1])):
        same(x, y)
    with pytest.raises(sq.SqError):
        sq.Cache(2, hq, hkv, d, page, pages, kv_pool=pool[1:], bits=8)


def test_captured_blocks_of_two_tiles():
    """Graphs of calls that widen pages share the cache's workspace: run in any order,
    also after it has grown, they give what the calls give."""
    hq, hkv, d, page = 8, 2, 64, 32
    c = sq.Cache(1, hq, hkv, d, page, 300, bits=8)
    hs = fill_sequences(c, [900, 300, 5000], 42)
    q = rows(gen(43), 300, hq, d, 0.5)
    outs = [torch.empty(300, hq, d, dtype=torch.bfloat16, device="cuda") for _ in hs]
    s = torch.cuda.Stream()

    def call(i, m=300):
        c.window_attention([hs[i]], [m], 0, q[:m], outs[i][:m], 0, sm_scale=d ** -0.5)

    graphs = []
    with torch.cuda.stream(s):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
            with pytest.raises(sq.SqError) as e:
                call(0)
            assert e.value.code == sq.SQ_ERR_UNSUPPORTED
        for i in range(2):
            call(i)
            s.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                call(i)
        call(2)   # (more pages than the workspace had)
        s.synchronize()
        want = [x.clone() for x in outs]
        for order in ((0, 1), (1, 0, 0, 1)):
            for i in order:
                outs[i].fill_(3.0)
                graphs[i].replay()
                call(2)
            s.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(outs, want))
    assert c.sync_status() == sq.SQ_OK


@pytest.mark.parametrize("hq,hkv,d,page", GEOMETRIES)
@pytest.mark.parametrize("ragged", [False, True])
def test_blocks_of_two_and_three_tiles(hq, hkv, d, page, ragged):
    """Chunks and trees of up to three query tiles a sequence, beside shorter ones, over
    whole and partial pages."""
    tile = 128 // (hq // hkv)
    lengths = [3 * tile + 300, 2 * tile + 70, tile + 1]
    c = sq.Cache(1, hq, hkv, d, page, sum(-(-n // page) for n in lengths) + 40, bits=8)
    hs = fill_sequences(c, lengths, 44)
    if ragged:
        c.evict_spans_ragged(hs[0], [(5, 40), (90, 91), (130, 133)])
    ctx = [c.seq_info(h)[0] for h in hs]
    scale = d ** -0.5

    def check(out, q, i, keep):
        want, weighted, logits = ref.attention(q, *read(c, hs[i]), scale, keep)
        # weights and outputs in bf16 (2^-8 of each, the normaliser's as well), sums as
        # in token_budget
        off = (out.double() - want).abs()
        assert (off <= weighted * 2.0 ** -7 + want.abs() * 2.0 ** -8 +
                weighted * (2.0 * (d + 8) * 2.0 ** -24 * logits)[..., None]).all()

    for counts, window, sinks in (([3 * tile, 2 * tile, 1], 0, 0), ([2 * tile + 1, 2 * tile - 1, tile + 1], 60, 3)):
        q = rows(gen(45), sum(counts), hq, d, 0.5)
        out = torch.full_like(q, 3.0)
        for _ in range(2):
            c.window_attention(hs, counts, 0, q, out, window, sinks, sm_scale=scale)
        at = 0
        for i, m in enumerate(counts):
            p, j = torch.arange(ctx[i] - m, ctx[i], device="cuda")[:, None], torch.arange(ctx[i], device="cuda")[None]
            keep = (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p
            check(out[at:at + m], q[at:at + m], i, keep)
            at += m
    counts = [min(256, 3 * tile), min(256, 2 * tile), 1]
    parents = [max(-1, j - 1 - j % 3) for m in counts for j in range(m)]
    q = rows(gen(46), sum(counts), hq, d, 0.5)
    out = torch.full_like(q, 3.0)
    c.tree_attention(hs, counts, parents, 0, q, out, sm_scale=scale)
    at = 0
    for i, m in enumerate(counts):
        keep = torch.ones(m, ctx[i], dtype=torch.bool)
        own = torch.zeros(m, m, dtype=torch.bool)
        for j in range(m):
            if parents[at + j] >= 0:
                own[j] = own[parents[at + j]]
            own[j, j] = True
        keep[:, ctx[i] - m:] = own
        check(out[at:at + m], q[at:at + m], i, keep.cuda())
        at += m
    assert c.sync_status() == sq.SQ_OK
