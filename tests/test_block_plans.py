"""Plans of attention for query blocks (CPU): what each query sees by the plan's
key tiles and masks, read as the kernel reads them, is what the definition says;
every key tile of a unit is in exactly one item; pages and partial results are in
bounds; partial pages, trees, windows, sinks, odd head groups and page sizes."""
import ctypes
import random

import numpy as np
import pytest

from tests import hostlib

KEYS, ROWS, NO_KEYS, TWO, NO_TREE = 128, 128, 0x7fffffc0, 1 << 30, 0x7fffffff


def plan(c, handles, n_q, parents=None, window=0, sinks=0, ctas=152, part_limit=1 << 27):
    L = hostlib.lib()
    arr = lambda x: (ctypes.c_int32 * max(1, len(x)))(*x)  # noqa: E731
    info = (ctypes.c_int64 * 12)()
    L.sqh_plan_blocks.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int32] + [ctypes.c_void_p] * 2 + \
        [ctypes.c_int32] * 3 + [ctypes.c_int64] + [ctypes.c_void_p] * 7
    args = [c.h, arr(handles), len(handles), arr(n_q), None if parents is None else arr(parents), window,
            sinks, ctas, part_limit, info]
    rc = L.sqh_plan_blocks(*args, *[None] * 6)
    if rc:
        return rc, None
    names = "tiles items merges rows n_words n_pieces BP n_parts one unit_rows max_splits n_ctas".split()
    p = dict(zip(names, list(info)))
    buf = {}
    queries = sum(n_q)
    for name, shape in (("tiles", (p["tiles"], 8)), ("items", (p["items"], 12)), ("merges", (p["merges"], 8)),
                        ("rows", (p["rows"], 2)), ("bits", (queries if p["n_words"] else 0, p["n_words"])),
                        ("tile_pages", (p["tiles"], p["n_pieces"]))):
        buf[name] = np.full(shape, -77, np.int32)
    assert L.sqh_plan_blocks(*args, *[b.ctypes.data for b in buf.values()]) == 0
    buf["bits"] = buf["bits"].view(np.uint32)
    return 0, dict(p, **buf)


def bits_through(x):
    return 0xffffffff if x >= 31 else (0 if x < 0 else (2 << x) - 1)


def kernel_word(p, it, qi, low, top, k):
    """RowMask::word of prefill_kernel.cuh."""
    sink_end, base = int(it[9]), int(it[10])
    if k >= base:
        w = (k - base) >> 5
        return int(p["bits"][it[4] + qi, w]) if w < p["n_words"] else 0
    return bits_through(top - k) & (~bits_through(low - 1 - k) & 0xffffffff | bits_through(sink_end - 1 - k))


def kernel_whole(low, top, sink_end, k):
    return k <= top - 63 and (k >= low or k <= sink_end - 64)


def check(c, P, G, Hkv, handles, n_q, parents=None, window=0, sinks=0, **kw):
    rc, p = plan(c, handles, n_q, parents, window, sinks, **kw)
    assert rc == 0
    BP = ROWS // G
    assert p["BP"] == BP and p["n_pieces"] == KEYS // min(P, 64)
    # the definition, row by row of each sequence, as slots
    want, ends, tables, at = [], [], [], 0
    for h, m in zip(handles, n_q):
        n, fills, table = c.info(h)[1], list(c.page_fill(h)), list(c.page_table(h))
        slots = [q * P + s for q, f in enumerate(fills) for s in range(f)]
        assert len(slots) == n
        ctx, pos, anc = n - m, list(range(n)), None
        if parents is not None:
            anc = []
            for i in range(m):
                par = parents[at + i]
                anc.append((anc[par] if par >= 0 else set()) | {i})
                pos[ctx + i] = ctx + len(anc[i]) - 1
        for i in range(m):
            here = pos[ctx + i]
            seen = set()
            for j in range(n):
                ok = (j < ctx or (j - ctx) in anc[i]) if anc is not None else j <= ctx + i
                if ok and (not window or pos[j] > here - window or pos[j] < sinks):
                    seen.add(slots[j])
            want.append(seen)
        ends += [(len(fills) - 1) * P + fills[-1]] * m if m else []
        tables += [table] * m
        at += m
    # the plan, item by item
    got = [set() for _ in want]
    cover, parts = {}, {}
    last = None
    for it in p["items"].tolist():
        head, two = it[0] & (TWO - 1), bool(it[0] & TWO)
        assert 0 <= head < Hkv and two == (it[5] > BP) and 1 <= it[5] <= 2 * BP
        assert 0 <= it[1] and it[2] >= 1 and it[1] + it[2] <= len(p["tiles"])
        if not p["one"]:
            assert last is None or it[2] <= last + 1   # longest first
            last = it[2] if last is None else min(last, it[2])
        unit = (it[4], it[5], head)
        for t in range(it[1], it[1] + it[2]):
            assert t not in cover.setdefault(unit, set())
            cover[unit].add(t)
        parts.setdefault(unit, []).append(it[3])
        if p["one"]:
            assert it[5] <= BP
        for qi in range(it[5]):
            q = it[4] + qi
            low, top = (p["rows"][q].tolist() if p["rows"].size else (it[8] + qi, it[7] + qi))
            assert it[6] == ends[q]
            for t in range(it[1], it[1] + it[2]):
                key0, flags, key0b = int(p["tiles"][t, 0]), int(p["tiles"][t, 1]), int(p["tiles"][t, 6])
                vis = [int(x) & 0xffffffff for x in p["tiles"][t, 2:6]]
                assert key0 % 64 == 0 and key0b % 64 == 0 and key0b > key0
                if t > it[1]:
                    assert key0 > int(p["tiles"][t - 1, 6])
                if key0b == NO_KEYS:
                    assert vis[2] == vis[3] == 0 and not flags
                assert bool(flags) == all(v == 0xffffffff for v in vis)
                seen = set()
                for w in range(4):
                    k = (key0 if w < 2 else key0b) + 32 * (w & 1)
                    m = vis[w] & kernel_word(p, it, qi, low, top, k) if vis[w] else 0
                    seen |= {k + b for b in range(32) if m >> b & 1}
                if flags and all(kernel_whole(low, top, it[9], k) for k in (key0, key0b)):
                    assert len(seen) == KEYS
                if head == 0:
                    assert not (got[q] & seen)
                    got[q] |= seen
                for i in range(p["n_pieces"]):
                    br = min(P, 64)
                    half = p["n_pieces"] // 2
                    k = key0 + i * br if i < half else key0b + (i - half) * br
                    pg = int(p["tile_pages"][t, i])
                    assert pg == (tables[q][k // P] if k < ends[q] else -1)
    assert got == want
    # the items of one-tile blocks are dealt out: every CTA's chain, each item once
    if p["one"]:
        ctas, seen = kw.get("ctas", 152), []
        assert p["n_ctas"] <= ctas
        for first in range(p["n_ctas"]):
            i = first
            while i >= 0:
                seen.append(i)
                i = int(p["items"][i, 11])
        assert sorted(seen) == list(range(len(p["items"])))
    else:
        assert p["n_ctas"] == len(p["items"]) and (p["items"][:, 11] == -1).all()
    # every head the same tiles; partial results in bounds, each once, and merged
    for (q, m, head), tiles in cover.items():
        assert tiles == cover[(q, m, 0)] and len(cover) % Hkv == 0
    used = [x for v in parts.values() for x in v if x >= 0]
    assert sorted(used) == list(range(p["n_parts"]))
    merged = {(r[3], r[4], r[0]): (r[1], r[2]) for r in p["merges"].tolist()}
    for unit, v in parts.items():
        if len(v) == 1:
            assert v == [-1] and unit not in merged
        else:
            assert sorted(v) == list(range(merged[unit][0], merged[unit][0] + merged[unit][1]))
            assert len(v) <= 64 and len(v) <= p["max_splits"]
            assert p["unit_rows"] >= (unit[1] * G if unit[1] <= BP else 256)
    return p


def tree(rng, m):
    return [-1 if i == 0 or rng.random() < 0.15 else rng.randrange(max(-1, i - 6), i) for i in range(m)]


@pytest.mark.parametrize("seed", range(40))
def test_plans_follow_the_definition(seed):
    rng = random.Random(seed)
    P = rng.choice([8, 16, 32, 64, 128, 256])
    Hkv, G = rng.choice([(2, 4), (1, 3), (3, 1), (2, 16), (1, 8)])
    c = hostlib.HostCache(1, Hkv * G, Hkv, rng.choice([64, 128]), P, 4000)
    handles = [c.seq_new()[1] for _ in range(rng.randint(1, 4))]
    for h in handles:
        assert c.append(h, rng.choice([1, P - 1, P, rng.randint(1, 700)])) == 0
        n = c.info(h)[1]
        if rng.random() < 0.4 and n > 8:
            a, b = sorted(rng.sample(range(n), 2))
            assert c.evict(h, [(a, b)], ragged=True)[0] == 0
    is_tree = rng.random() < 0.5
    n_q = []
    for h in handles:
        if is_tree:
            m = rng.choice([0, 1, rng.randint(1, 70)])
            if m:
                assert c.append(h, m) == 0
        else:
            m = rng.choice([0, 1, rng.randint(0, c.info(h)[1])])
        n_q.append(m)
    parents = [x for m in n_q for x in tree(rng, m)] if is_tree else None
    check(c, P, G, Hkv, handles, n_q, parents, window=rng.choice([0, 1, 2, 63, 64, 65, rng.randint(1, 900)]),
          sinks=rng.choice([0, 1, 4, 64, 130, 5000]), ctas=rng.choice([1, 8, 152]))


@pytest.mark.parametrize("m", [1, 31, 32, 33, 255, 256])
@pytest.mark.parametrize("ctx", [1, 31, 32, 64, 97])
def test_trees_at_word_edges(m, ctx):
    rng = random.Random(m * 1000 + ctx)
    c = hostlib.HostCache(1, 4, 1, 128, 64, 100)
    h = c.seq_new()[1]
    assert c.append(h, ctx + m) == 0
    check(c, 64, 4, 1, [h], [m], tree(rng, m), window=rng.choice([0, 3, 40]), sinks=rng.choice([0, 2]))


def test_long_units_are_cut_and_parts_limited():
    c = hostlib.HostCache(1, 4, 1, 128, 64, 100)
    h = c.seq_new()[1]
    assert c.append(h, 64 * 99 + 3) == 0
    p = check(c, 64, 4, 1, [h], [1], window=6000, sinks=4)
    assert p["n_parts"] > 4 and p["one"]
    assert check(c, 64, 4, 1, [h], [1], window=6000, part_limit=0)["n_parts"] == 0
    # a window of a few rows reads its boxes and the sinks' alone
    p = check(c, 64, 4, 1, [h], [1], window=3, sinks=4)
    assert len(p["tiles"]) == 1 and sorted(p["tile_pages"][0]) == sorted([c.page_table(h)[0], c.page_table(h)[99]])


def test_drafted_rows_across_a_partial_page_are_refused():
    c = hostlib.HostCache(1, 4, 1, 128, 64, 100)
    h = c.seq_new()[1]
    assert c.append(h, 200) == 0
    assert c.evict(h, [(150, 152)], ragged=True)[0] == 0
    # the last page holds 8 rows, the page before it lacks two
    assert plan(c, [h], [8], tree(random.Random(1), 8))[0] == 0
    assert plan(c, [h], [9], tree(random.Random(1), 9))[0] == -8


@pytest.mark.parametrize("D,lengths,window", [
    (128, [30000], 4096), (128, [30000] * 3, 0), (64, [200 * i + 7 for i in range(1, 49)], 4096),
    (128, [60000 // i for i in range(1, 40)], 4096), (64, [5000] * 20, 128)])
def test_even_shares(D, lengths, window):
    """No CTA has much more than its share of the key tiles (a piece costs a few
    tiles' worth more), and short units stay whole."""
    c = hostlib.HostCache(1, 32, 8, D, 64, sum(n // 64 + 1 for n in lengths), max_seqs=64)
    handles = [c.seq_new()[1] for _ in lengths]
    for h, n in zip(handles, lengths):
        assert c.append(h, n) == 0
    rc, p = plan(c, handles, [1] * len(handles), window=window, sinks=4)
    assert rc == 0 and p["one"]
    fixed, load = (2 if D == 128 else 4), []
    for i in range(p["n_ctas"]):
        load.append(0)
        while i >= 0:
            load[-1] += int(p["items"][i, 2]) + fixed
            i = int(p["items"][i, 11])
    assert max(load) <= sum(load) / min(152, p["n_ctas"]) + 4 + 2 * fixed
    if window == 128:
        assert p["n_parts"] == 0


def test_a_unit_of_more_shares_than_a_merge_takes():
    c = hostlib.HostCache(1, 8, 1, 128, 256, 4000)
    h = c.seq_new()[1]
    assert c.append(h, 1000000) == 0
    rc, p = plan(c, [h], [1])
    assert rc == 0 and 50 < p["max_splits"] <= 64
    assert p["items"][:, 2].max() <= 1.1 * len(p["tiles"]) / 60
