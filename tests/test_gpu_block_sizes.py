"""Query blocks and stores at sizes that take the kernels' other ways: more blocks
than SMs, several items on one CTA, small pages with long key ranges cut into
pieces and merged, and pools whose offsets pass 32 bits; against 64-bit references
within the kernels' error budget."""
import random

import pytest
import torch

import paper_2602_22603_gb300 as sq
from tests.gpu_harness import row_slots
from tests.test_gpu_blocks import Batch, tree
from tests.test_gpu_norm_rope import assert_rounded, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("P", [8, 16, 32, 64])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 70)])
def test_long_contexts_on_small_pages(P, Hq, Hkv, D, window, sinks):
    b = Batch(Hq, Hkv, D, P, [7001, 30, 4097], seed=P)
    b.check([9, 2, 30], window=window, sinks=sinks, sample=6)       # one query tile
    b.check([90, 30, 200], window=window, sinks=sinks, sample=6)    # two
    rng = random.Random(P)
    b.check([20, 30, 7], tree(rng, 20) + tree(rng, 30) + tree(rng, 7), window, sinks, sample=6)
    b.c.close()


@pytest.mark.parametrize("P,Hkv,D", [(64, 8, 128), (16, 4, 64), (32, 8, 128), (256, 4, 64)])
@pytest.mark.parametrize("m", [20, 180])
def test_more_blocks_than_processors(P, Hkv, D, m):
    """m = 20: blocks of one query tile, several items to each CTA (dealt out
    beforehand); m = 180: of two, handed out while the kernel runs."""
    rng = random.Random(P + m)
    lengths = [rng.randint(m, 900) for _ in range(48)]
    counts = [rng.randint(m // 2, m) for _ in range(48)]
    counts[7] = counts[11] = 0
    b = Batch(4 * Hkv, Hkv, D, P, lengths, seed=P + m)
    b.check(counts, window=300, sinks=5, sample=2)
    b.check(counts, sum((tree(rng, x) for x in counts), []), sample=2)
    b.c.close()


def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^32 of the pool: stores, and attention of
    single tokens, prompts and trees."""
    Hq, Hkv, D, P, n, m = 32, 8, 128, 64, 700, 90
    pages = (1 << 32) // (2 * Hkv * P * D) + 400
    if torch.cuda.mem_get_info()[0] < 3 * pages * 2 * Hkv * P * D:
        pytest.skip("not enough memory")
    b = Batch(Hq, Hkv, D, P, [0, 0], seed=1, num_pages=pages)
    filler = b.c.seq_new()
    b.c.extend([filler], [(pages - 100) * P])
    for h in b.h:
        b.append(h, n)
    assert min(b.c.page_table(b.h[0])) * 2 * Hkv * P * D > 1 << 32
    b.check(None, window=300, sinks=3)
    b.check([m, 2], window=300, sinks=3)
    b.check([m, 20], tree(random.Random(1), m) + tree(random.Random(2), 20))
    counts = [3, 200]
    b.c.extend(b.h, counts)
    q, k, v, w, table, pos, _ = inputs(Hq, Hkv, D, sum(counts), 64, 5, "bf16")
    q_out = torch.empty_like(q)
    b.c.qk_norm_rope_store(b.h, counts, 0, q, k, v, pos, sq.norm_rope(table, 64, 1e-6, *w), q_out)
    assert b.c.sync_status() == sq.SQ_OK
    exact, size = reference(k, w[1], 1e-6, table, pos, 64, False)
    at = 0
    for h, x in zip(b.h, counts):
        page, slot = (t[-x:] for t in row_slots(b.c, h))
        got = b.pool[0, page, :, :, slot]
        assert_rounded(got[:, 0], exact[at:at + x], size[at:at + x])
        assert torch.equal(got[:, 1], v[at:at + x])
        at += x
    b.c.close()


@pytest.mark.parametrize("P", [16, 64, 256])
def test_stores_between_layers_are_seen_at_64_dimensions(P):
    """Calls that reuse their plans, and load keys ahead of the launch before them,
    read the rows stored just before: back to back as with waits in between, bit
    for bit; contexts cut into pieces, several streams."""
    L, D, lengths, m = 4, 64, [5000, 700, 130], 6
    c = sq.Cache(L, 16, 4, D, P, sum(lengths) // P + 20)
    g = torch.Generator("cuda").manual_seed(P)
    hs = [c.seq_new() for _ in lengths]
    for h, n in zip(hs, lengths):
        c.append_kv(h, n, *(torch.randn(L, n, 4, D, generator=g, device="cuda").bfloat16() for _ in range(2)))
    torch.cuda.synchronize()
    counts, par = [m] * 3, sq.norm_rope()
    c.extend(hs, counts)
    qkv = torch.randn(L, 3 * m, 24, D, generator=g, device="cuda").bfloat16()
    parents = [-1, 0, 0, 1, 1, 4] * 3
    side = torch.cuda.Stream()
    outs = []
    for slow in (True, False):
        out = torch.empty(L, 2, 3 * m, 16, D, device="cuda")
        torch.cuda.synchronize()
        for rep in range(5):
            for layer in range(L):
                x = qkv[(layer + rep) % L]
                q = torch.empty(3 * m, 16, D, dtype=torch.bfloat16, device="cuda")
                stream = side if rep == 3 else torch.cuda.current_stream()
                stream.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(stream):
                    c.qk_norm_rope_store(hs, counts, layer, x[:, :16], x[:, 16:20], x[:, 20:], None, par, q)
                    if slow:
                        torch.cuda.synchronize()
                    kw = dict(out_dtype=sq.SQ_OUT_F32, sm_scale=D ** -0.5)
                    c.tree_attention(hs, counts, parents, layer, q, out[layer, 0], **kw)
                    c.window_attention(hs, counts, layer, q, out[layer, 1], 3000, 2, **kw)
                    if slow:
                        torch.cuda.synchronize()
                torch.cuda.current_stream().wait_stream(stream)
        assert c.sync_status() == sq.SQ_OK
        outs.append(out)
    assert torch.isfinite(outs[0]).all()
    assert torch.equal(*outs)
    c.close()
