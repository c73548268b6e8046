"""Plans of windowed decode (CPU): what each sequence's segments, items, fills and
limits let the kernel read, taken the way the kernel takes them, is each sink and
each row of the window exactly once, at every page size and over partial pages."""
import ctypes
import random

import pytest

from tests import hostlib

STAGE = 64


def plan(monkeypatch, c, handles, n_ctas, window, sinks):
    L = hostlib.lib()
    f = L.sqh_plan_window_decode
    P, I32 = ctypes.c_void_p, ctypes.c_int32
    f.argtypes = [P, P, I32, I32, I32, I32, P, P, ctypes.c_int64]
    monkeypatch.setattr(L, "sqh_plan_decode", lambda h, arr, n, ctas, lay, buf, size: f(
        h, arr, n, ctas, window, sinks, lay, buf, size))
    return c.plan_decode(handles, n_ctas)


@pytest.mark.parametrize("seed", range(60))
def test_windows_and_sinks(monkeypatch, seed):
    rng = random.Random(seed)
    P, Hkv = rng.choice([8, 16, 32, 64, 128, 256]), rng.choice([1, 2, 3])
    c = hostlib.HostCache(1, 4 * Hkv, Hkv, 64, P, 3000)
    handles = [c.seq_new()[1] for _ in range(rng.randint(1, 5))]
    for h in handles:
        assert c.append(h, rng.choice([1, P, P + 1, rng.randint(1, 1500)])) == 0
        n = c.info(h)[1]
        if rng.random() < 0.5 and n > 8:
            a, b = sorted(rng.sample(range(n), 2))
            assert c.evict(h, [(a, b)], ragged=True)[0] == 0
    window, sinks = rng.choice([1, 5, 64, 65, 300, 4000]), rng.choice([0, 1, 4, 64, 130, 900])
    n_ctas = rng.choice([1, 7, 152])
    rc, p = plan(monkeypatch, c, handles, n_ctas, window, sinks)
    assert rc == 0 and len(p["cta_begin"]) - 1 <= n_ctas
    got, loads = {}, 0
    for seg, head, s0, s1 in p["items"]:
        s = p["segs"][seg]
        assert s["n_grp"] == 1 and s["tail"] == 0 and s1 > s0 >= 0
        assert s["n_tok"] == s["grp_lim"][0] <= s["n_pages"] * P
        loads += s1 - s0
        for t in range(s0 * STAGE, s1 * STAGE):
            q, slot = t // P, t % P
            if t >= s["n_tok"] or q >= s["n_pages"]:
                continue
            fill = p["page_fill"][s["page_off"] + q]
            if slot < fill >> 20 or (fill >> 10 & 1023) <= slot < (fill & 1023):
                got.setdefault((s["grp_seq"][0], head), []).append((p["page_ids"][s["page_off"] + q], slot))
    visible = 0
    for i, h in enumerate(handles):
        rows = [(pg, s) for pg, f in zip(c.page_table(h), c.page_fill(h)) for s in range(f)]
        n = len(rows)
        want = [r for j, r in enumerate(rows) if j >= n - window or j < sinks]
        visible += len(want)
        for head in range(Hkv):
            assert sorted(got[(i, head)]) == sorted(want)
    assert p["logical_tokens"] == visible
    full = all(f == P for h in handles for f in c.page_fill(h)[:-1])
    if full:
        assert loads <= Hkv * (visible / STAGE + 5 * len(handles))
