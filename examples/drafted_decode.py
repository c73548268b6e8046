"""Drafted decoding over the paged cache.

A small random-init decoder (per-head q/k norms, rotated positions, a sliding
window with sinks on every layer but each fourth) answers a batch of prompts.  A
step drafts a tree of tokens for every sequence by looking its last token up in
the sequence's own history, and one pass through the layers verifies all trees:

    cache.extend                 rows for the drafted tokens
    for each layer:
        cache.qk_norm_rope_store norm, rotate, store the layer's keys and values
        cache.tree_attention     each token over the context and its ancestors
    cache.accept_draft           the verified path stays

Prompts, and steps without drafts, take the same layers with window_attention.
Before that the norm weights of the layers are fitted to given queries and keys,
with qk_norm_rope and its backward pass (fit_norms), as a training program would.

    python examples/drafted_decode.py [--seqs 8] [--tokens 96] [--draft 12]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), os.pardir))
import paper_2602_22603_gb300 as sq  # noqa: E402

EPS = 1e-6


class NormRope(torch.autograd.Function):
    """cache.qk_norm_rope with its gradients."""

    @staticmethod
    def forward(ctx, cache, table, q, k, positions, q_weight, k_weight):
        params = sq.norm_rope(table, table.shape[1] * 2, EPS, q_weight.detach(), k_weight.detach())
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        cache.qk_norm_rope(q, k, positions, params, q_out, k_out)
        ctx.save_for_backward(q, k, positions)
        ctx.call = cache, params
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        (q, k, positions), (cache, params) = ctx.saved_tensors, ctx.call
        dq, dk = torch.empty_like(q), torch.empty_like(k)
        dqw, dkw = (torch.empty(q.shape[-1], device=q.device) for _ in range(2))
        cache.qk_norm_rope_backward(q, k, positions, params, dq_out.contiguous(), dk_out.contiguous(),
                                    dq, dk, dqw, dkw)
        return None, None, dq, dk, None, dqw, dkw


class Decoder:
    """layers of attention with residuals; weights N(0, 1) scaled, seeded."""

    def __init__(self, layers=4, Hq=16, Hkv=4, D=64, vocab=512, page=16, pages=2048, seqs=8, window=256,
                 sinks=4, max_pos=8192, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        width = Hq * D
        def weights(*shape):  # noqa: E306
            return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()
        self.Hq, self.Hkv, self.D, self.layers = Hq, Hkv, D, layers
        self.embed = weights(vocab, width) * width ** 0.5
        self.w_in = [weights((Hq + 2 * Hkv) * D, width) for _ in range(layers)]
        self.w_out = [weights(width, width) for _ in range(layers)]
        self.norms = [[torch.ones(D, device="cuda") for _ in range(2)] for _ in range(layers)]
        self.table = sq.rope_table(max_pos, D)
        self.window = [0 if (i + 1) % 4 == 0 else window for i in range(layers)]
        self.sinks = sinks
        self.cache = sq.Cache(layers, Hq, Hkv, D, page, pages, max_seqs=seqs)

    def project(self, layer, x):
        """q, k, v of the layer: parts of one product."""
        x = x.float()
        x = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)).bfloat16()
        y = (x @ self.w_in[layer].T).view(-1, self.Hq + 2 * self.Hkv, self.D)
        return y.split([self.Hq, self.Hkv, self.Hkv], 1)

    def forward(self, handles, counts, tokens, positions, parents=None):
        """Logits of the newest counts[i] tokens of every sequence, whose rows
        cache.extend has made; parents: they are drafted trees."""
        c = self.cache
        x = self.embed[tokens]
        for layer in range(self.layers):
            q, k, v = self.project(layer, x)
            params = sq.norm_rope(self.table, self.D, EPS, *self.norms[layer])
            q_out, out = (torch.empty(len(x), self.Hq, self.D, dtype=x.dtype, device="cuda") for _ in range(2))
            c.qk_norm_rope_store(handles, counts, layer, q, k, v, positions, params, q_out)
            rule = dict(window=self.window[layer], n_sink=self.sinks, sm_scale=self.D ** -0.5)
            if parents is None:
                c.window_attention(handles, counts, layer, q_out, out, **rule)
            else:
                c.tree_attention(handles, counts, parents, layer, q_out, out, **rule)
            x = x + out.view(len(x), -1) @ self.w_out[layer].T
        return x.float() @ self.embed.float().T

    def prompts(self, prompts):
        """Sequences of these tokens, and the logits of all of them."""
        handles, counts = [self.cache.seq_new() for _ in prompts], [len(p) for p in prompts]
        self.cache.extend(handles, counts)
        tokens = torch.tensor(sum(prompts, []), device="cuda")
        return handles, self.forward(handles, counts, tokens, None)


def fit_norms(model, layer, q, k, q_want, k_want, positions, steps=20, rate=0.3):
    """Gradient steps on the layer's norm weights towards wanted (normed, rotated)
    queries and keys; the losses."""
    weights = [w.requires_grad_() for w in model.norms[layer]]
    losses = []
    for _ in range(steps):
        got = NormRope.apply(model.cache, model.table, q, k, positions, *weights)
        loss = sum((a.float() - b.float()).square().mean() for a, b in zip(got, (q_want, k_want)))
        grads = torch.autograd.grad(loss, weights)
        with torch.no_grad():
            for w, gr in zip(weights, grads):
                w -= rate * gr * len(w)
        losses.append(loss.item())
    model.norms[layer] = [w.detach() for w in weights]
    return losses


def draft(history, most):
    """A tree for a sequence: its last token, then the continuations of that token's
    earlier occurrences, newest first, equal beginnings shared.  Tokens and parents."""
    tokens, parents, child = [history[-1]], [-1], {}
    for at in range(len(history) - 2, -1, -1):
        if history[at] != history[-1]:
            continue
        node = 0
        for tok in history[at + 1:at + 5]:
            if (node, tok) not in child:
                if len(tokens) == most:
                    return tokens, parents
                child[node, tok] = len(tokens)
                tokens.append(tok)
                parents.append(node)
            node = child[node, tok]
    return tokens, parents


def generate(model, prompts, n_tokens, most):
    """Greedy answers by drafted decoding: the sequences' handles and tokens (the
    newest token of each is not in the cache yet), and the steps taken."""
    handles, logits = model.prompts(prompts)
    ends = torch.tensor([len(p) for p in prompts]).cumsum(0) - 1
    history = [p + [t] for p, t in zip(prompts, logits[ends.cuda()].argmax(-1).tolist())]
    steps = 0
    while min(len(h) - len(p) for h, p in zip(history, prompts)) < n_tokens:
        trees = [draft(h, most) for h in history]
        counts = [len(t) for t, _ in trees]
        positions, parents = [], []
        for h, (_, up) in zip(history, trees):
            depth = []
            for p in up:
                depth.append(depth[p] + 1 if p >= 0 else 0)
            positions += [len(h) - 1 + d for d in depth]
            parents += up
        model.cache.extend(handles, counts)
        logits = model.forward(handles, counts, torch.tensor(sum((t for t, _ in trees), []), device="cuda"),
                               torch.tensor(positions, dtype=torch.int32, device="cuda"), parents)
        best, at = logits.argmax(-1).tolist(), 0
        for i, (toks, up) in enumerate(trees):
            path, node = [0], 0
            history[i].append(best[at])
            while True:
                node = next((j for j in range(node + 1, len(toks)) if up[j] == node and
                             toks[j] == history[i][-1]), None)
                if node is None:
                    break
                path.append(node)
                history[i].append(best[at + node])
            model.cache.accept_draft(handles[i], len(toks), path)
            at += len(toks)
        steps += 1
    assert model.cache.sync_status() == sq.SQ_OK
    return handles, history, steps


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--seqs", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=96)
    ap.add_argument("--draft", type=int, default=12)
    args = ap.parse_args()
    model = Decoder(seqs=args.seqs)
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(200, model.Hq * model.D, generator=g, device="cuda").bfloat16()
    want = [1 + 0.2 * torch.randn(model.D, generator=g, device="cuda") for _ in range(2)]
    positions = torch.arange(200, dtype=torch.int32, device="cuda")
    for layer in range(model.layers):
        q, k, _ = (t.contiguous() for t in model.project(layer, x))
        q_want, k_want = NormRope.apply(model.cache, model.table, q, k, positions, *want)
        losses = fit_norms(model, layer, q, k, q_want, k_want, positions)
        print(f"layer {layer}: norm weights fitted, loss {losses[0]:.4f} -> {losses[-1]:.6f}")
    pick = torch.randint(0, 16, (args.seqs, 300), generator=g, device="cuda").tolist()
    generate(model, [p[:20] for p in pick], 4, args.draft)   # (first launches)
    model.cache.close()
    model.cache = sq.Cache(model.layers, model.Hq, model.Hkv, model.D, 16, 2048, max_seqs=args.seqs)
    t0 = time.perf_counter()
    _, history, steps = generate(model, [p[:100 + 20 * i] for i, p in enumerate(pick)], args.tokens, args.draft)
    took = time.perf_counter() - t0
    made = sum(len(h) - 100 - 20 * i for i, h in enumerate(history))
    print(f"{made} tokens in {steps} passes ({made / steps / args.seqs:.2f} a sequence and pass), "
          f"{1e3 * took / steps:.2f} ms a pass")


if __name__ == "__main__":
    main()
