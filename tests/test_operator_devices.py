"""The binding hands on no address of host memory and no weights of another size than
the head's: what it refuses before the library is reached, and that it takes the rest
(CPU, with stand-ins for tensors on a device)."""
import pytest
import torch

import paper_2602_22603_gb300 as sq


class OnDevice:
    """What the binding asks of a tensor on a CUDA device."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def cache(monkeypatch):
    c = object.__new__(sq.Cache)     # (no call gets as far as the library)
    c.handle, c.Hq, c.Hkv, c.D = None, 4, 2, 64
    c.calls = []
    for name in ("store", "", "backward"):
        name = "sq_qk_norm_rope" + (name and "_" + name)
        monkeypatch.setattr(sq, name, lambda *a, _n=name: c.calls.append(_n))
    for name in ("sq_window_attention", "sq_tree_attention"):
        monkeypatch.setattr(sq, name, lambda *a, _n=name, **k: c.calls.append(_n))
    yield c


def rows(n, heads, dim=64):
    return OnDevice(torch.zeros(n, heads, dim, dtype=torch.bfloat16))


def tensors():
    f = lambda *s: OnDevice(torch.zeros(*s))  # noqa: E731
    return dict(q=rows(3, 4), k=rows(3, 2), v=rows(3, 2), positions=OnDevice(torch.zeros(3, dtype=torch.int32)),
                q_out=rows(3, 4), k_out=rows(3, 2), dq_out=rows(3, 4), dk_out=rows(3, 2), dq=rows(3, 4),
                dk=rows(3, 2), dqw=f(64), dkw=f(64), out=rows(3, 4), lse=f(3, 4))


def calls(c, t, params):
    return {
        "q k v positions q_out": lambda: c.qk_norm_rope_store([1], [3], 0, t["q"], t["k"], t["v"], t["positions"],
                                                              params, t["q_out"]),
        "q k positions q_out k_out": lambda: c.qk_norm_rope(t["q"], t["k"], t["positions"], params, t["q_out"],
                                                            t["k_out"]),
        "q k positions dq_out dk_out dq dk dqw dkw": lambda: c.qk_norm_rope_backward(
            t["q"], t["k"], t["positions"], params, t["dq_out"], t["dk_out"], t["dq"], t["dk"], t["dqw"], t["dkw"]),
        "q out lse": lambda: c.window_attention([1], [3], 0, t["q"], t["out"], 4, lse=t["lse"]),
        "q out  lse": lambda: c.tree_attention([1], [3], [-1, 0, 1], 0, t["q"], t["out"], lse=t["lse"]),
    }


def test_tensors_on_the_device_are_taken(cache):
    for f in calls(cache, tensors(), sq.norm_rope()).values():
        f()
    assert len(cache.calls) == 5


@pytest.mark.parametrize("which", range(5))
def test_tensors_of_the_host_are_refused(cache, which):
    names, _ = list(calls(cache, tensors(), sq.norm_rope()).items())[which]
    for name in names.split():
        t = tensors()
        t[name] = t[name].t
        with pytest.raises(ValueError, match="cuda"):
            list(calls(cache, t, sq.norm_rope()).values())[which]()
    assert not cache.calls


@pytest.mark.parametrize("kind", ["q_weight", "k_weight"])
def test_weights_of_another_size(cache, kind):
    for dtype in (torch.bfloat16, torch.float32):
        for n in (32, 128, 1):
            params = sq.norm_rope(**{kind: OnDevice(torch.zeros(n, dtype=dtype))})
            for f in list(calls(cache, tensors(), params).values())[:3]:
                with pytest.raises(ValueError, match="weight"):
                    f()
        params = sq.norm_rope(**{kind: OnDevice(torch.zeros(64, dtype=dtype))})
        for f in list(calls(cache, tensors(), params).values())[:3]:
            f()
    assert len(cache.calls) == 6
    with pytest.raises(ValueError, match="weight"):
        sq.norm_rope(q_weight=OnDevice(torch.zeros(64)), k_weight=OnDevice(torch.zeros(128)))


def test_parameters_of_the_host(cache):
    with pytest.raises(ValueError, match="cuda"):
        sq.norm_rope(q_weight=torch.zeros(64))
    with pytest.raises(ValueError, match="cuda"):
        sq.norm_rope(torch.zeros(10, 32, 2), 64)
    sq.norm_rope(OnDevice(torch.zeros(10, 32, 2)), 64)
