"""Plans of query blocks without partial results (no memory for them): the units stay
whole and are spread over the CTAs by their key tiles."""
import pytest

from tests import hostlib
from tests.test_block_plans import check, plan


@pytest.mark.parametrize("Hkv,D,lengths,ctas", [
    (8, 128, [16000] * 64, 152), (8, 128, [100 + 900 * i for i in range(40)], 152),
    (1, 64, [30000] + [70] * 400, 152), (2, 64, [5000] * 76, 152), (2, 64, [5000] * 77, 152), (8, 128, [900] * 9, 8)])
def test_whole_units_are_spread(Hkv, D, lengths, ctas):
    c = hostlib.HostCache(1, 4 * Hkv, Hkv, D, 64, sum(n // 64 + 1 for n in lengths), max_seqs=512)
    handles = [c.seq_new()[1] for _ in lengths]
    for h, n in zip(handles, lengths):
        assert c.append(h, n) == 0
    rc, p = plan(c, handles, [1] * len(handles), ctas=ctas, part_limit=0)
    assert rc == 0 and p["one"] and p["n_parts"] == 0
    fixed, load, seen = (2 if D == 128 else 4), [], 0
    for i in range(p["n_ctas"]):
        load.append(0)
        while i >= 0:
            load[-1] += int(p["items"][i, 2]) + fixed
            i = int(p["items"][i, 11])
            seen += 1
    assert seen == len(p["items"]) == len(lengths) * Hkv
    assert p["n_ctas"] == min(ctas, seen)
    # the CTA that ends last began its last unit when no CTA was free
    longest = int(p["items"][:, 2].max()) + fixed
    assert max(load) <= sum(load) / ctas + longest


def test_they_still_follow_the_definition():
    c = hostlib.HostCache(1, 8, 2, 128, 64, 2000)
    handles = [c.seq_new()[1] for _ in range(30)]
    for i, h in enumerate(handles):
        assert c.append(h, 64 * i + 5) == 0
    check(c, 64, 4, 2, handles, [1 + i % 5 for i in range(30)], ctas=16, part_limit=0, window=700, sinks=3)
