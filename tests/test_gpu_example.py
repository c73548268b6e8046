"""The drafted-decoding example: the cache that its steps leave (trees verified,
paths accepted) is the one that its answers as prompts give, and the norms' weights
are fitted."""
import importlib.util
import os

import pytest
import torch

import paper_2602_22603_gb300 as sq

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(__file__), os.pardir, "examples", "drafted_decode.py")


@pytest.fixture(scope="module")
def example():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("drafted_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("D,page,window", [(64, 16, 60), (128, 64, 100)])
def test_drafted_answers(example, D, page, window):
    model = example.Decoder(layers=4, Hq=8, Hkv=2, D=D, page=page, seqs=8, window=window)
    g = torch.Generator().manual_seed(D)
    prompts = [torch.randint(0, 8, (n,), generator=g).tolist() for n in (1, 90, 150)]
    handles, history, steps = example.generate(model, prompts, 40, 9)
    made = [len(h) - len(p) for h, p in zip(history, prompts)]
    assert min(made) >= 40 and sum(made) > 3 * steps     # some drafts were taken
    for h, x in zip(handles, history):
        assert model.cache.seq_info(h)[0] == len(x) - 1 == model.cache.next_pos(h)
    # one more token through what the drafts left, and the whole answer as a prompt:
    # 4 layers of bf16 roundings apart (each value some 2^-8 of its size off, a dozen
    # roundings a layer): 2^-8 sqrt(48) = 2.7% of the logits' size, times 3
    model.cache.extend(handles)
    last = torch.tensor([x[-1] for x in history], device="cuda")
    logits = model.forward(handles, None, last, None)
    other, every = model.prompts(history)
    ends = torch.tensor([len(x) for x in history]).cumsum(0) - 1
    want = every[ends.cuda()]
    assert model.cache.sync_status() == sq.SQ_OK
    off = (logits - want).square().mean(-1).sqrt() / want.square().mean(-1).sqrt()
    assert (off < 0.08).all(), off
    # and the tokens are the greedy ones wherever the best logit stands out
    at = 0
    for x, p in zip(history, prompts):
        top = every[at + len(p) - 1:at + len(x) - 1].topk(2, -1)
        clear = (top.values[:, 0] - top.values[:, 1]) > 0.16 * want.square().mean().sqrt()
        assert clear.any()
        got = torch.tensor(x[len(p):], device="cuda")
        assert (got == top.indices[:, 0])[clear].all()
        at += len(x)
    model.cache.close()


def test_norm_weights_are_fitted(example):
    model = example.Decoder(layers=1, Hq=8, Hkv=2, D=64)
    g = torch.Generator("cuda").manual_seed(3)
    q, k, _ = (t.contiguous() for t in model.project(0, torch.randn(100, 512, generator=g, device="cuda").bfloat16()))
    positions = torch.arange(100, dtype=torch.int32, device="cuda")
    want = [1 + 0.2 * torch.randn(64, generator=g, device="cuda") for _ in range(2)]
    target = example.NormRope.apply(model.cache, model.table, q, k, positions, *want)
    losses = example.fit_norms(model, 0, q, k, *target, positions)
    assert losses[-1] < 0.01 * losses[0]
    for got, w in zip(model.norms[0], want):
        assert (got - w).abs().max() < 0.03
    model.cache.close()
