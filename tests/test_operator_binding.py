"""What the binding of the calls around a model's attention refuses before it hands
an address on: wrong types, sizes, strides and counts."""
import pytest
import torch

import paper_2602_22603_gb300 as sq


@pytest.fixture
def cache():
    c = object.__new__(sq.Cache)     # (no call gets as far as the library)
    c.handle, c.Hq, c.Hkv, c.D = None, 4, 2, 64
    yield c


def rows(n, heads, dtype=torch.bfloat16, dim=64):
    return torch.zeros(n, heads, dim, dtype=dtype)


@pytest.mark.parametrize("q,out,kw", [
    (rows(3, 4, torch.float32), rows(3, 4), {}),                        # type
    (rows(2, 4), rows(3, 4), {}),                                       # too few queries
    (rows(3, 4), rows(2, 4), {}),                                       # too small an output
    (rows(3, 4), rows(3, 4), {"out_dtype": sq.SQ_OUT_F32}),             # half the size it says
    (rows(3, 8)[:, :4], rows(3, 4), {}),                                # rows apart
    (rows(3, 4), rows(3, 8)[:, ::2], {}),
    (rows(3, 4), rows(3, 4), {"lse": torch.zeros(3, 2)}),
    (rows(3, 4), rows(3, 4), {"lse": torch.zeros(3, 4, dtype=torch.float64)}),
])
def test_attention_tensors(cache, q, out, kw):
    with pytest.raises(ValueError):
        cache.window_attention([1, 2], [1, 2], 0, q, out, 4, **kw)
    with pytest.raises(ValueError):
        cache.tree_attention([1, 2], [1, 2], [-1, -1, 0], 0, q, out, **kw)


def test_counts(cache):
    q = rows(3, 4)
    with pytest.raises(ValueError):
        cache.window_attention([1, 2], [3], 0, q, q.clone(), 4)
    with pytest.raises(ValueError):
        cache.window_attention([1, 2], None, 0, q, q.clone(), 4)
    with pytest.raises(ValueError):
        cache.tree_attention([1], [3], [-1, 0], 0, q, q.clone())


@pytest.mark.parametrize("wrong", [
    {"q": rows(3, 2)}, {"k": rows(2, 2)}, {"v": rows(3, 2, torch.float16)}, {"k": rows(3, 2, dim=32)},
    {"q": torch.zeros(3, 256, dtype=torch.bfloat16)}, {"v": rows(3, 2).transpose(1, 2).contiguous().transpose(1, 2)},
    {"positions": torch.zeros(3, dtype=torch.int64)}, {"positions": torch.zeros(2, dtype=torch.int32)},
    {"q_out": rows(3, 8)[:, ::2]}, {"q_out": rows(3, 4, torch.float32)},
])
def test_store_tensors(cache, wrong):
    t = dict(q=rows(3, 4), k=rows(3, 2), v=rows(3, 2), positions=None, q_out=rows(3, 4))
    t.update(wrong)
    with pytest.raises(ValueError):
        cache.qk_norm_rope_store([1], [3], 0, t["q"], t["k"], t["v"], t["positions"], sq.norm_rope(), t["q_out"])
