"""Performance cases of the operators around a model's attention over the cache:
per-head norms of queries and keys with the position rotation (stored into the
cache, as plain tensors, and backwards), attention with a sliding window and
sinks, and attention for trees of drafted tokens.

A case is a dict of plain values:

    kind                 store | forward | backward | window | tree
    hq hkv d page        geometry of the cache (one layer of it)
    layout               seed of the case's shape (lengths, trees), not of its values
    rot pairs weights    store, forward, backward: dimensions rotated; whether the
                         rotation pairs neighbours instead of halves; type of the
                         norms' weights
    seqs n_min n_max     store: sequences and the new tokens of each
    n                    forward, backward: tokens
    seqs n_min n_max     window, tree: sequences and their tokens before the queries
    q_min q_max          window: queries of each sequence (its newest tokens)
    drafts_min, _max     tree: drafted tokens of each sequence
    window sinks         window, tree: reach of a query, first tokens that stay visible
                         (window 0: every earlier token)

Queries, keys and values are N(0, 1) in bf16, the query heads of a group at
several sharpnesses (SHARPNESS), as real heads range from near-uniform to
peaked; projections that the norms take have a scale of their own per head.
"""
import math
import random

import torch

own = False

SHARPNESS = (1.0, 1.0, 2.0, 4.0)
MAX_POS = 131072   # rows of the rotation's table
THETA = 500000.0
EPS = 1e-6


def listed():
    big = dict(hq=32, hkv=8, d=128, page=64)     # the 8B-class model
    large = dict(hq=64, hkv=8, d=128, page=64)   # the 70B-class model
    wide = dict(hq=64, hkv=8, d=64, page=32)     # many query heads of few dimensions
    tiny = dict(hq=16, hkv=4, d=64, page=16)     # a small model, small pages
    return [
        # one agent generates a token: the norms, the rotation and the new cache
        # row of one layer, where latency is all
        dict(name="store-decode-1", kind="store", **big, layout=1, seqs=1, n_min=1, n_max=1,
             rot=128, pairs=False, weights="bf16"),
        # a serving batch generates a token each, a part of each head rotated
        dict(name="store-decode-batch150", kind="store", **wide, layout=2, seqs=150, n_min=1,
             n_max=1, rot=32, pairs=True, weights="f32"),
        # three prompts of odd lengths enter the cache together
        dict(name="store-prompts-ragged", kind="store", **big, layout=3, seqs=3, n_min=2501,
             n_max=9001, rot=128, pairs=False, weights="bf16"),
        # training forward of one packed sequence of odd length
        dict(name="forward-4097", kind="forward", **tiny, layout=4, n=4097, rot=64, pairs=False,
             weights="f32"),
        # training backward, with the gradients of both weights
        dict(name="backward-8k", kind="backward", **large, layout=5, n=8192, rot=128, pairs=False,
             weights="bf16"),
        # one agent decodes at the far end of a long context in a windowed layer
        dict(name="window-decode-1", kind="window", **wide, layout=6, seqs=1, n_min=131071,
             n_max=131071, q_min=1, q_max=1, window=128, sinks=4),
        # a batch in mid-trace decodes, some still inside the window
        dict(name="window-decode-batch48", kind="window", **big, layout=7, seqs=48, n_min=200,
             n_max=60000, q_min=1, q_max=1, window=4096, sinks=4),
        # a long prompt's windowed layer
        dict(name="window-prefill-16k", kind="window", **big, layout=8, seqs=1, n_min=0, n_max=0,
             q_min=16384, q_max=16384, window=1024, sinks=4),
        # ragged chunks of several prompts in one call, beside single tokens
        dict(name="window-chunks-ragged", kind="window", **tiny, layout=9, seqs=6, n_min=30,
             n_max=20000, q_min=1, q_max=700, window=1000, sinks=5),
        # one agent verifies a small tree of drafted tokens
        dict(name="tree-1", kind="tree", **big, layout=10, seqs=1, n_min=8191, n_max=8191,
             drafts_min=16, drafts_max=16, window=0, sinks=0),
        # a batch verifies full trees over long contexts
        dict(name="tree-batch8-64", kind="tree", **large, layout=11, seqs=8, n_min=20001,
             n_max=60000, drafts_min=64, drafts_max=64, window=0, sinks=0),
        # the same step in a windowed layer, trees of different sizes
        dict(name="tree-window-batch24", kind="tree", **wide, layout=12, seqs=24, n_min=100,
             n_max=30000, drafts_min=5, drafts_max=33, window=512, sinks=4),
    ]


GEOMETRIES = [
    dict(hq=32, hkv=8, d=128, page=64), dict(hq=32, hkv=8, d=128, page=64),
    dict(hq=64, hkv=8, d=128, page=64), dict(hq=16, hkv=4, d=64, page=16),
    dict(hq=64, hkv=8, d=64, page=32), dict(hq=32, hkv=2, d=64, page=32),
    dict(hq=6, hkv=2, d=128, page=256), dict(hq=8, hkv=8, d=64, page=8),
]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _between(rng, lo, hi):
    return lo if lo == hi else _log(rng, lo, hi)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most:
            return c


def _draw_any(rng):
    kind = rng.choice(["store", "store", "forward", "backward", "window", "window", "window",
                       "tree", "tree"])
    c = dict(kind=kind, **rng.choice(GEOMETRIES), layout=rng.randrange(1 << 20))
    if kind in ("store", "forward", "backward"):
        c.update(rot=rng.choice([c["d"], c["d"], c["d"] // 2, c["d"] // 4, 0, 48]),
                 pairs=rng.random() < 0.3, weights=rng.choice(["bf16", "f32"]))
        if kind == "store":
            a, b = (1, 1) if rng.random() < 0.5 else sorted((_log(rng, 1, 9000), _log(rng, 1, 9000)))
            c.update(seqs=_log(rng, 1, 300 if b == 1 else 8), n_min=a, n_max=b)
        else:
            c.update(n=_log(rng, 1, 16384))
        return c
    a, b = sorted((_log(rng, 1, 131000), _log(rng, 1, 131000)))
    sinks = rng.choice([0, 4, rng.randint(1, 200)])
    if kind == "window":
        window = _log(rng, 1, 8192)
        if rng.random() < 0.5:
            c.update(seqs=_log(rng, 1, 64), q_min=1, q_max=1)
        else:
            x, y = sorted((_log(rng, 1, 16384), _log(rng, 1, 16384)))
            c.update(seqs=_log(rng, 1, 8), q_min=x, q_max=y)
    else:
        window = rng.choice([0, 0, _log(rng, 16, 8192)])
        x, y = sorted((_log(rng, 1, 96), _log(rng, 1, 96)))
        c.update(seqs=_log(rng, 1, 32), drafts_min=x, drafts_max=y)
    c.update(n_min=a, n_max=b, window=window, sinks=sinks)
    if _rows(c) * c["hkv"] * c["d"] * 4 > 6 << 30:
        c.update(seqs=1)
    return c


def _rows(c):
    return sum(n for n, _ in _lengths(c))


def _lengths(c):
    """(rows in the cache, newest of them that the call is about) of each sequence."""
    rng = random.Random(c["layout"])
    if c["kind"] == "store":
        out = []
        for _ in range(c["seqs"]):
            new = _between(rng, c["n_min"], c["n_max"])
            out.append((rng.randint(0, 2 * c["page"]) + new, new))
        return out
    lo, hi = (c["q_min"], c["q_max"]) if c["kind"] == "window" else (c["drafts_min"], c["drafts_max"])
    out = []
    for _ in range(c["seqs"]):
        new = _between(rng, lo, hi)
        before = _between(rng, c["n_min"], c["n_max"])
        out.append((before + new, new))
    return out


def _trees(c):
    """Parents of every sequence's drafted tokens: -1 (the context's last token)
    or an earlier drafted one, mostly a recent one."""
    rng = random.Random(c["layout"] + 1)
    return [[-1 if i == 0 or rng.random() < 0.1 else i - 1 - min(i - 1, int(rng.expovariate(0.4)))
             for i in range(new)] for _, new in _lengths(c)]


def _tables(c):
    """Page ids of each sequence: the sequences grew by turns, four pages a turn,
    each taking the lowest free ids."""
    P, lens = c["page"], [n for n, _ in _lengths(c)]
    tables, free = [[] for _ in lens], 0
    while True:
        grew = False
        for t, n in zip(tables, lens):
            k = min(4, -(-n // P) - len(t))
            t.extend(range(free, free + k))
            free += k
            grew |= k > 0
        if not grew:
            return tables, max(free, 1)


def _starts(c):
    """First position of each sequence's new tokens: far above the rows in the
    cache, most of whose predecessors were evicted."""
    rng = random.Random(c["layout"] + 2)
    return [rng.randint(0, MAX_POS - new) for _, new in _lengths(c)]


# ---- inputs ------------------------------------------------------------------
def _tokens(c):
    return c["n"] if "n" in c else sum(new for _, new in _lengths(c))


def _norm_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    n, d, heads = _tokens(c), c["d"], c["hq"] + 2 * c["hkv"]
    s = dict(qkv=torch.randn(n, heads, d, generator=g, device="cuda"))
    s["qkv"] *= torch.exp(torch.randn(1, heads, 1, generator=g, device="cuda"))
    s["qkv"] = s["qkv"].bfloat16()   # what the fused projection leaves
    dt = torch.float32 if c["weights"] == "f32" else torch.bfloat16
    for w in ("q_weight", "k_weight"):
        s[w] = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt)
    inv = THETA ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64)
                    / max(c["rot"], 1))
    angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * inv
    s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    if c["kind"] == "store":
        pos = [p + i for p, (_, new) in zip(_starts(c), _lengths(c)) for i in range(new)]
        s["positions"] = torch.tensor(pos, dtype=torch.int32).cuda()
    else:
        # packed sequences: positions start again at each
        rng, pos = random.Random(c["layout"] + 3), []
        while len(pos) < n:
            pos.extend(range(min(n - len(pos), _log(rng, 1, 16384))))
        s["positions"] = torch.tensor(pos, dtype=torch.int32).cuda()
    if c["kind"] == "backward":
        for name, h in (("dq_out", c["hq"]), ("dk_out", c["hkv"])):
            s[name] = torch.randn(n, h, d, generator=g, device="cuda").bfloat16()
    if c["kind"] == "store":
        s["pool"] = _pool(c, g)
    return s


def _pool(c, g):
    _, pages = _tables(c)
    return torch.randn(1, pages, 2, c["hkv"], c["page"], c["d"], generator=g, device="cuda",
                       dtype=torch.bfloat16)


def _attention_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    n, group = _tokens(c), c["hq"] // c["hkv"]
    q = torch.randn(n, c["hq"], c["d"], generator=g, device="cuda")
    sharp = torch.tensor([SHARPNESS[h % group % len(SHARPNESS)] for h in range(c["hq"])])
    return dict(pool=_pool(c, g), q=(q * sharp.cuda()[None, :, None]).bfloat16())


def _inputs(c, seed):
    return (_attention_inputs if c["kind"] in ("window", "tree") else _norm_inputs)(c, seed)


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    s["case"] = c
    s["lengths"] = _lengths(c) if c["kind"] in ("store", "window", "tree") else []
    s["new"] = [new for _, new in s["lengths"]]
    hq, hkv = c["hq"], c["hkv"]
    if "qkv" in s:
        s["q"], s["k"], s["v"] = s["qkv"].split([hq, hkv, hkv], dim=1)
    if c["kind"] == "tree":
        s["parents"] = [p for t in _trees(c) for p in t]
    if own:
        import paper_2602_22603_gb300 as sq
        _open(sq, s)
    else:
        _plan(s)
    return s


def _open(sq, s):
    """The cache, its sequences and the buffers that a serving program holds."""
    c, P = s["case"], s["case"]["page"]
    pages = s["pool"].shape[1] if "pool" in s else 1
    cache = sq.Cache(1, c["hq"], c["hkv"], c["d"], P, pages, max_seqs=max(1, len(s["new"])),
                     kv_pool=s.get("pool"))
    s["cache"] = cache
    s["handles"] = [cache.seq_new() for _ in s["lengths"]]
    have = [0] * len(s["handles"])
    while True:
        grow = [(i, min(4 * P, n - h)) for i, ((n, _), h) in enumerate(zip(s["lengths"], have))
                if n > h]
        if not grow:
            break
        cache.extend([s["handles"][i] for i, _ in grow], [k for _, k in grow])
        for i, k in grow:
            have[i] += k
    if "qkv" in s:
        s["params"] = sq.norm_rope(s["rope"], c["rot"], EPS, s["q_weight"], s["k_weight"],
                                   interleaved=c["pairs"])
        n = s["qkv"].shape[0]
        s["q_out"] = torch.empty(n, c["hq"], c["d"], dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.empty(n, c["hkv"], c["d"], dtype=torch.bfloat16, device="cuda")
        if c["kind"] == "backward":
            s["dq"], s["dk"] = torch.empty_like(s["q_out"]), torch.empty_like(s["k_out"])
            s["dqw"], s["dkw"] = (torch.empty(c["d"], device="cuda") for _ in range(2))
    else:
        s["out"] = torch.empty_like(s["q"])


def _plan(s):
    """What the plain forms index with: the page and slot of every row."""
    c, P = s["case"], s["case"]["page"]
    if c["kind"] in ("forward", "backward"):
        return
    tables, _ = _tables(c)
    s["pages"] = [torch.tensor(t, dtype=torch.int64).cuda() for t in tables]
    if c["kind"] == "store":
        page, slot = [], []
        for t, (n, new) in zip(tables, s["lengths"]):
            page.extend(t[j // P] for j in range(n - new, n))
            slot.extend(j % P for j in range(n - new, n))
        s["page"], s["slot"] = torch.tensor(page).cuda(), torch.tensor(slot).cuda()
    if c["kind"] == "tree":
        s["masks"], s["depths"] = [], []
        for tree in _trees(c):
            seen, depth = torch.zeros(len(tree), len(tree), dtype=torch.bool), []
            for i, p in enumerate(tree):
                if p >= 0:
                    seen[i] = seen[p]
                seen[i, i] = True
                depth.append(depth[p] + 1 if p >= 0 else 0)
            s["masks"].append(seen.cuda())
            s["depths"].append(torch.tensor(depth).cuda())


# ---- one pass ----------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_store(s):
    s["cache"].qk_norm_rope_store(s["handles"], s["new"], 0, s["q"], s["k"], s["v"],
                                  s["positions"], s["params"], s["q_out"])
    return s["q_out"], s["pool"]


def _own_forward(s):
    s["cache"].qk_norm_rope(s["q"], s["k"], s["positions"], s["params"], s["q_out"], s["k_out"])
    return s["q_out"], s["k_out"]


def _own_backward(s):
    s["cache"].qk_norm_rope_backward(s["q"], s["k"], s["positions"], s["params"], s["dq_out"],
                                     s["dk_out"], s["dq"], s["dk"], s["dqw"], s["dkw"])
    return s["dq"], s["dk"], s["dqw"], s["dkw"]


def _own_window(s):
    c = s["case"]
    s["cache"].window_attention(s["handles"], s["new"], 0, s["q"], s["out"], c["window"],
                                c["sinks"], sm_scale=c["d"] ** -0.5)
    return s["out"]


def _own_tree(s):
    c = s["case"]
    s["cache"].tree_attention(s["handles"], s["new"], s["parents"], 0, s["q"], s["out"],
                              c["window"], c["sinks"], sm_scale=c["d"] ** -0.5)
    return s["out"]


_OWN = dict(store=_own_store, forward=_own_forward, backward=_own_backward, window=_own_window,
            tree=_own_tree)


def _turned(x, cos, sin, pairs):
    """x with its leading 2 * cos.shape[-1] dimensions rotated."""
    r = 2 * cos.shape[-1]
    if r == 0:
        return x
    if pairs:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_norm(s, x, w):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s[w].float()
    cs = s["rope"][s["positions"].long()][:, None]
    return _turned(x, cs[..., 0], cs[..., 1], s["case"]["pairs"]).bfloat16()


def _plain_store(s):
    q, k = _plain_norm(s, s["q"], "q_weight"), _plain_norm(s, s["k"], "k_weight")
    s["pool"][0, s["page"], 0, :, s["slot"]] = k
    s["pool"][0, s["page"], 1, :, s["slot"]] = s["v"]
    return q, s["pool"]


def _plain_forward(s):
    return _plain_norm(s, s["q"], "q_weight"), _plain_norm(s, s["k"], "k_weight")


def _plain_backward(s):
    out = []
    cs = s["rope"][s["positions"].long()][:, None]
    for x, w, dz in ((s["q"], "q_weight", s["dq_out"]), (s["k"], "k_weight", s["dk_out"])):
        x, w = x.float(), s[w].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        # the rotation's transpose turns the other way
        dy = _turned(dz.float(), cs[..., 0], -cs[..., 1], s["case"]["pairs"])
        xn = x * r
        dn = dy * w
        dx = r * (dn - xn * (dn * xn).mean(-1, keepdim=True))
        out += [dx.bfloat16(), (dy * xn).sum((0, 1))]
    return out[0], out[2], out[1], out[3]


def _plain_attend(s, i, q, keep, rows):
    """Queries q over the cache rows `rows` of sequence i that `keep` allows."""
    c = s["case"]
    page, slot = s["pages"][i][rows // c["page"]], rows % c["page"]
    k = s["pool"][0, page, 0, :, slot].float().transpose(0, 1)      # [hkv, rows, d]
    v = s["pool"][0, page, 1, :, slot].float().transpose(0, 1)
    m = q.shape[0]
    x = q.float().view(m, c["hkv"], -1, c["d"]).transpose(0, 1)     # [hkv, m, group, d]
    z = torch.matmul(x.reshape(c["hkv"], -1, c["d"]), k.transpose(1, 2)) * c["d"] ** -0.5
    z = z.view(c["hkv"], m, -1, rows.numel()).masked_fill(~keep[None, :, None], -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True))
    z = z / z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(c["hkv"], -1, rows.numel()), v)
    return o.view(c["hkv"], m, -1, c["d"]).transpose(0, 1).reshape(m, c["hq"], c["d"]).bfloat16()


def _plain_window(s):
    c, out, at = s["case"], [], 0
    for i, (n, new) in enumerate(s["lengths"]):
        for b in range(0, new, 256):
            m = min(256, new - b)
            at_pos = n - new + b + torch.arange(m, device="cuda")[:, None]
            low = max(0, n - new + b - c["window"] + 1)
            rows = torch.cat([torch.arange(min(c["sinks"], low), device="cuda"),
                              torch.arange(low, n - new + b + m, device="cuda")])
            keep = (rows <= at_pos) & ((rows > at_pos - c["window"]) | (rows < c["sinks"]))
            out.append(_plain_attend(s, i, s["q"][at + b:at + b + m], keep, rows))
        at += new
    return torch.cat(out)


def _plain_tree(s):
    c, out, at = s["case"], [], 0
    for i, (n, new) in enumerate(s["lengths"]):
        ctx, reach = n - new, c["window"] or n + 1
        low = max(0, ctx - reach + 1)
        rows = torch.cat([torch.arange(min(c["sinks"], low), device="cuda"),
                          torch.arange(low, n, device="cuda")])
        at_pos = ctx + s["depths"][i][:, None]
        pos = torch.where(rows < ctx, rows, 0)
        pos[rows >= ctx] = ctx + s["depths"][i]
        keep = (pos > at_pos - reach) | (pos < c["sinks"])
        keep[:, rows >= ctx] &= s["masks"][i]
        out.append(_plain_attend(s, i, s["q"][at:at + new], keep, rows))
        at += new
    return torch.cat(out)


_PLAIN = dict(store=_plain_store, forward=_plain_forward, backward=_plain_backward,
              window=_plain_window, tree=_plain_tree)


# ---- what a pass cannot do without -------------------------------------------
def _seen(c):
    """(cache rows some query sees, visible (query, row) pairs) of all sequences."""
    rows = pairs = 0
    trees = _trees(c) if c["kind"] == "tree" else None
    for i, (n, new) in enumerate(_lengths(c)):
        ctx, reach = n - new, c["window"] or n + 1
        low = max(0, ctx - reach + 1)
        rows += min(c["sinks"], low) + n - low
        if trees is None:
            # query p sees min(p + 1, reach) rows and the sinks before them
            for a, b in ((ctx, min(n, reach)), (max(ctx, reach), n)):
                if a >= b:
                    continue
                if b <= reach:
                    pairs += (b - a) * (a + b + 1) // 2
                    continue
                pairs += (b - a) * reach
                first = a - reach + 1   # rows before the first query's window
                x = min(b - a, max(0, c["sinks"] - first))
                pairs += x * first + x * (x - 1) // 2 + (b - a - x) * c["sinks"]
            continue
        depth = []
        for p in trees[i]:
            depth.append(depth[p] + 1 if p >= 0 else 0)
        for e in depth:
            lo = max(0, ctx + e - reach + 1)
            pairs += max(ctx - lo, 0) + min(c["sinks"], lo, ctx) + min(e + 1, reach)
            pairs += min(max(c["sinks"] - ctx, 0), max(e + 1 - reach, 0))
    return rows, pairs


def work(case):
    c = case
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    if c["kind"] in ("window", "tree"):
        rows, pairs = _seen(c)
        return {"bytes": rows * hkv * d * 4 + _tokens(c) * hq * d * 4,
                "flops": pairs * hq * d * 4}
    n = _tokens(c)
    table = n * (4 + c["rot"] * 4)
    if c["kind"] == "store":
        return {"bytes": n * (hq + 2 * hkv) * d * 4 + table, "flops": n * (hq + hkv) * d * 7}
    if c["kind"] == "forward":
        return {"bytes": n * (hq + hkv) * d * 4 + table, "flops": n * (hq + hkv) * d * 7}
    return {"bytes": n * (hq + hkv) * d * 6 + table, "flops": n * (hq + hkv) * d * 16}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.5e15)


# ---- the definitions in 64 bits ----------------------------------------------
def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if c["kind"] in ("window", "tree"):
        return _exact_attention(c, s)
    pos = s["positions"].long()
    hq, hkv, d, half = c["hq"], c["hkv"], c["d"], c["rot"] // 2
    angle = torch.complex(s["rope"][pos, :, 0].double(), s["rope"][pos, :, 1].double())
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)

    def rotate(x, by):
        y = x.clone()
        z = torch.complex(x[..., first], x[..., second]) * by[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    res = []
    for lo, hi, w, dz in ((0, hq, "q_weight", "dq_out"), (hq, hq + hkv, "k_weight", "dk_out")):
        x, wt = s["qkv"][:, lo:hi].double(), s[w].double()
        rms = torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + EPS)
        if c["kind"] != "backward":
            res.append(rotate(x / rms * wt, angle))
            continue
        dy = rotate(s[dz].double(), angle.conj())
        dot = (dy * wt * x).sum(-1, keepdim=True)
        res.append((dy * wt / rms - x * dot / (d * rms.pow(3)), (dy * x / rms).sum((0, 1))))
    if c["kind"] == "forward":
        return tuple(res)
    if c["kind"] == "backward":
        return res[0][0], res[1][0], res[0][1], res[1][1]
    pool, P, at = s["pool"].double(), c["page"], 0
    for t, (n, new) in zip(_tables(c)[0], _lengths(c)):
        for a in range((n - new) // P * P, n, P):
            lo, hi = max(a, n - new), min(a + P, n)
            b = at + lo - (n - new)
            pool[0, t[a // P], 0, :, lo - a:hi - a] = res[1][b:b + hi - lo].transpose(0, 1)
            pool[0, t[a // P], 1, :, lo - a:hi - a] = \
                s["qkv"][b:b + hi - lo, hq + hkv:].double().transpose(0, 1)
        at += new
    return res[0], pool


def _exact_attention(c, s):
    d, group, P = c["d"], c["hq"] // c["hkv"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    trees = _trees(c) if c["kind"] == "tree" else None
    at = 0
    for i, (t, (n, new)) in enumerate(zip(_tables(c)[0], _lengths(c))):
        ctx = n - new
        # one row of the cache after the other, whole pages at a time
        ids = torch.tensor(t, device="cuda")
        index = torch.arange(n, device="cuda")
        for b in range(0, new, 128):
            e = min(new, b + 128)
            if trees is None:
                place = ctx + torch.arange(b, e, device="cuda")
                see = index[None] <= place[:, None]
                where = index
            else:
                anc, depth = [], []
                for p in trees[i]:
                    anc.append((anc[p] if p >= 0 else []) + [len(anc)])
                    depth.append(len(anc[-1]) - 1)
                where = torch.cat([index[:ctx], ctx + torch.tensor(depth, device="cuda")])
                place = where[ctx + b:ctx + e]
                see = torch.zeros(e - b, n, dtype=torch.bool, device="cuda")
                see[:, :ctx] = True
                for r in range(b, e):
                    see[r - b, [ctx + a for a in anc[r]]] = True
            if c["window"]:
                near = place[:, None] - where[None] < c["window"]
                see &= near | (where < c["sinks"])[None]
            some = see.any(0).nonzero()[:, 0]
            see = see[:, some]
            rows = s["pool"][0, ids[some // P], :, :, some % P]   # [rows, 2, hkv, d]
            for g in range(c["hkv"]):
                key, val = rows[:, 0, g].double(), rows[:, 1, g].double()
                for h in range(g * group, (g + 1) * group):
                    a = s["q"][at + b:at + e, h].double() @ key.T / math.sqrt(d)
                    a = torch.where(see, a, torch.tensor(-math.inf, dtype=a.dtype, device="cuda"))
                    a = torch.exp(a - torch.logsumexp(a, 1, keepdim=True))
                    out[at + b:at + e, h] = a @ val
        at += new
    return out
