"""Stores, norms and attention around a model in a CUDA graph: its runs take the inputs
as they are then and give what the same calls give outside, also after other calls have
made plans and larger workspaces of their own."""
import pytest
import torch

import paper_2602_22603_gb300 as sq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2602_22603_gb300 import build
    build.build_libsq()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 128, 64), (16, 4, 64, 16)])
def test_a_step_in_a_graph(Hq, Hkv, D, P):
    g = torch.Generator("cuda").manual_seed(P)
    c = sq.Cache(2, Hq, Hkv, D, P, 3 * (30000 // P) + 200, max_seqs=8)
    hs = [c.seq_new() for _ in range(2)]
    for h, n in zip(hs, (20000, 3000)):
        k, v = (torch.randn(2, n, Hkv, D, generator=g, device="cuda").bfloat16() for _ in range(2))
        c.append_kv(h, n, k, v)
    m = [12, 5]
    n = sum(m)
    c.extend(hs, m)
    table = sq.rope_table(64000, D)
    params = sq.norm_rope(table, D, 1e-6, *(torch.rand(D, generator=g, device="cuda") + 0.5 for _ in range(2)))
    qkv = torch.empty(n, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    dz = [torch.empty(n, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv)]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    parents = [-1] + [(i - 1) // 2 for i in range(1, 12)] + [-1, 0, 0, 2, 2]

    def outputs():
        e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
        return dict(q=e(n, Hq, D, dt=torch.bfloat16), tree=e(n, Hq, D), window=e(n, Hq, D), lse=e(n, Hq),
                    token=e(2, Hq, D), dq=e(n, Hq, D, dt=torch.bfloat16), dk=e(n, Hkv, D, dt=torch.bfloat16),
                    dqw=e(D), dkw=e(D))

    def step(o):
        q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
        rule = dict(out_dtype=sq.SQ_OUT_F32, sm_scale=D ** -0.5)
        for layer in range(2):
            c.qk_norm_rope_store(hs, m, layer, q, k, v, None, params, o["q"])
            c.tree_attention(hs, m, parents, layer, o["q"], o["tree"], **rule)
            c.window_attention(hs, m, layer, o["q"], o["window"], 900, 3, lse=o["lse"], **rule)
            c.window_attention(hs, None, layer, o["q"][:2], o["token"], 5000, 3, **rule)
        c.qk_norm_rope_backward(q, k, pos, params, *dz, o["dq"], o["dk"], o["dqw"], o["dkw"])

    def new_inputs():
        for t in (qkv, *dz):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    new_inputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mine = outputs()
    with torch.cuda.stream(s):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
            with pytest.raises(sq.SqError) as e:      # (nothing kept yet, and a capture uploads nothing)
                c.tree_attention(hs, m, parents, 0, mine["q"], mine["tree"], out_dtype=sq.SQ_OUT_F32)
            assert e.value.code == sq.SQ_ERR_UNSUPPORTED
            mine["lse"].add_(1)
        for _ in range(2):
            step(mine)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(mine)
    for rep in range(3):
        new_inputs()
        for t in mine.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = outputs()
        step(want)
        torch.cuda.synchronize()
        assert c.sync_status() == sq.SQ_OK
        for name, t in mine.items():
            assert torch.equal(t, want[name]), (rep, name)
        # other plans and larger workspaces between the runs
        for w in range(10, 16):
            o = torch.empty(n, Hq, D, device="cuda")
            c.window_attention(hs, m, 0, want["q"], o, w, out_dtype=sq.SQ_OUT_F32)
            c.tree_attention(hs, m, parents, 0, want["q"], o, 100 + w, out_dtype=sq.SQ_OUT_F32)
            c.window_attention(hs, None, 0, want["q"][:2], o[:2], w, out_dtype=sq.SQ_OUT_F32)
        big = torch.randn(2 * 2900, Hq, D, generator=g, device="cuda").bfloat16()
        c.window_attention(hs, [2900, 2900], 0, big, torch.empty_like(big), 0)
        many = torch.randn(3000, Hq + Hkv, D, generator=g, device="cuda").bfloat16()
        p2 = torch.zeros(3000, dtype=torch.int32, device="cuda")
        q2, k2 = many.split([Hq, Hkv], 1)
        c.qk_norm_rope_backward(q2, k2, p2, params, q2.contiguous(), k2.contiguous(), torch.empty_like(q2),
                                torch.empty_like(k2), want["dqw"], want["dkw"])
        torch.cuda.synchronize()
    del graph
    c.close()
