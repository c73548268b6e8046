"""Performance cases of a key/value cache held in 8 bits: storing new rows in it
(per-head norms, position rotation, rounding to e4m3 with one power-of-two scale
for every 8 slots of a page and head), attention of single tokens over it, and
attention of query blocks over it (prompt chunks and trees of drafted tokens).

A case is a dict of plain values:

    kind                 store | tokens | chunks | tree
    hq hkv d page        geometry of the cache (one layer of it)
    layout               seed of the case's shape (lengths, trees), not of its values
    rot pairs weights    store: dimensions rotated; whether the rotation pairs
                         neighbours instead of halves; type of the norms' weights
    seqs n_min n_max     sequences and their rows before the new ones
    q_min q_max          new rows of each sequence: the ones stored, or the queries
    window sinks         reach of a query, first tokens that stay visible (window 0:
                         every earlier token)

Keys have channels and tokens of different sizes, values heads and tokens of
different sizes, so that the scales of neighbouring blocks differ.  Rows read
back from the cache are bf16: what their 8 bits stand for has 4 significant bits.
"""
import math
import random

import torch

own = False

SHARPNESS = (0.7, 1.0, 1.4, 2.0)   # of the query heads of a group
MAX_POS = 131072                   # rows of the rotation's table
THETA = 500000.0
EPS = 1e-6
BLOCK = 8                          # slots that share a scale
E4M3_MOST = 448.0
LEAST_SCALE = -100                 # exponent of the smallest scale


def listed():
    big = dict(hq=32, hkv=8, d=128, page=64)     # the 8B-class model
    large = dict(hq=64, hkv=8, d=128, page=64)   # the 70B-class model
    wide = dict(hq=64, hkv=8, d=64, page=32)     # many query heads of few dimensions
    tiny = dict(hq=16, hkv=4, d=64, page=16)     # a small model, small pages
    return [
        # one agent generates a token: its cache row joins a block begun before,
        # whose scale may grow with it; latency is all
        dict(name="store-1", kind="store", **big, layout=1, seqs=1, n_min=1003, n_max=1003,
             q_min=1, q_max=1, rot=128, pairs=False, weights="bf16"),
        # a serving batch generates a token each, a part of each head rotated
        dict(name="store-batch150", kind="store", **wide, layout=2, seqs=150, n_min=1, n_max=4000,
             q_min=1, q_max=1, rot=32, pairs=True, weights="f32"),
        # three prompts of odd lengths enter the cache together
        dict(name="store-prompts-ragged", kind="store", **big, layout=3, seqs=3, n_min=1,
             n_max=100, q_min=2501, q_max=9001, rot=128, pairs=False, weights="bf16"),
        # one agent decodes in a short context: latency
        dict(name="tokens-1-short", kind="tokens", **wide, layout=4, seqs=1, n_min=700, n_max=700,
             q_min=1, q_max=1, window=0, sinks=0),
        # one agent decodes at the far end of a long context
        dict(name="tokens-1-long", kind="tokens", **big, layout=5, seqs=1, n_min=131071,
             n_max=131071, q_min=1, q_max=1, window=0, sinks=0),
        # a serving batch in mid-trace, contexts of very different lengths
        dict(name="tokens-batch48", kind="tokens", **big, layout=6, seqs=48, n_min=200,
             n_max=60000, q_min=1, q_max=1, window=0, sinks=0),
        # long contexts of the larger model
        dict(name="tokens-large-batch16", kind="tokens", **large, layout=7, seqs=16, n_min=20001,
             n_max=60000, q_min=1, q_max=1, window=0, sinks=0),
        # a batch decodes in a windowed layer on small pages
        dict(name="tokens-window-batch64", kind="tokens", **tiny, layout=8, seqs=64, n_min=30,
             n_max=20000, q_min=1, q_max=1, window=2048, sinks=4),
        # a whole prompt attends to itself
        dict(name="chunk-prompt-8k", kind="chunks", **big, layout=9, seqs=1, n_min=0, n_max=0,
             q_min=8191, q_max=8191, window=0, sinks=0),
        # a tool's answer of some hundred tokens joins a long context
        dict(name="chunk-512-over-60k", kind="chunks", **big, layout=10, seqs=1, n_min=60001,
             n_max=60001, q_min=512, q_max=512, window=0, sinks=0),
        # ragged chunks of several prompts in one call, a windowed layer, small pages
        dict(name="chunks-ragged-window", kind="chunks", **tiny, layout=11, seqs=6, n_min=30,
             n_max=20000, q_min=1, q_max=700, window=1000, sinks=5),
        # a batch verifies trees of drafted tokens over long contexts
        dict(name="tree-batch8-16", kind="tree", **large, layout=12, seqs=8, n_min=8001,
             n_max=32000, q_min=16, q_max=16, window=0, sinks=0),
    ]


GEOMETRIES = [
    dict(hq=32, hkv=8, d=128, page=64), dict(hq=32, hkv=8, d=128, page=64),
    dict(hq=64, hkv=8, d=128, page=64), dict(hq=16, hkv=4, d=64, page=16),
    dict(hq=64, hkv=8, d=64, page=32), dict(hq=32, hkv=2, d=64, page=32),
    dict(hq=6, hkv=2, d=128, page=256), dict(hq=8, hkv=8, d=64, page=8),
]


def _log(rng, lo, hi):
    if lo == hi:
        return lo
    return int(round(math.exp(rng.uniform(math.log(max(lo, 0.7)), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most and _rows(c) * c["hkv"] * c["d"] <= 1 << 30:
            return c


def _draw_any(rng):
    kind = rng.choice(["store", "store", "tokens", "tokens", "tokens", "chunks", "chunks", "tree"])
    c = dict(kind=kind, **rng.choice(GEOMETRIES), layout=rng.randrange(1 << 20))
    a, b = sorted((_log(rng, 1, 131000), _log(rng, 1, 131000)))
    x, y = sorted((_log(rng, 1, 9000), _log(rng, 1, 9000)))
    window = rng.choice([0, 0, _log(rng, 1, 8192)])
    if kind == "store":
        if rng.random() < 0.5:
            x = y = 1
        c.update(seqs=_log(rng, 1, 300 if y == 1 else 8), n_min=a // 64, n_max=max(1, b // 64), q_min=x,
                 q_max=y, rot=rng.choice([c["d"], c["d"], c["d"] // 2, c["d"] // 4, 0, 48]),
                 pairs=rng.random() < 0.3, weights=rng.choice(["bf16", "f32"]))
        return c
    if kind == "tokens":
        c.update(seqs=_log(rng, 1, 64), q_min=1, q_max=1)
    elif kind == "chunks":
        c.update(seqs=_log(rng, 1, 8), q_min=x, q_max=y)
    else:
        x, y = sorted((_log(rng, 1, 96), _log(rng, 1, 96)))
        c.update(seqs=_log(rng, 1, 32), q_min=x, q_max=y)
    c.update(n_min=a, n_max=b, window=window, sinks=rng.choice([0, 4, rng.randint(1, 200)]) if window else 0)
    return c


def _rows(c):
    return sum(n for n, _ in _lengths(c))


def _lengths(c):
    """(rows in the cache, newest of them that the call is about) of each sequence."""
    rng, out = random.Random(c["layout"]), []
    for _ in range(c["seqs"]):
        new = _log(rng, c["q_min"], c["q_max"])
        out.append((_log(rng, c["n_min"], c["n_max"]) + new, new))
    return out


def _new(c):
    return sum(new for _, new in _lengths(c))


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


# ---- inputs ------------------------------------------------------------------
def _quantised(x):
    """(codes, scales) of x [..., slots, d]: the smallest power of two for every
    BLOCK slots with which the largest of their elements is at most E4M3_MOST."""
    x = x.view(*x.shape[:-2], -1, BLOCK, x.shape[-1])
    mant, exp = torch.frexp(x.abs().amax((-1, -2)))       # mant in [0.5, 1)
    e = torch.where(mant == 0, LEAST_SCALE, exp - 9 + (mant > 0.875))
    scale = torch.ldexp(torch.ones_like(mant), e.clamp(min=LEAST_SCALE))
    codes = (x / scale[..., None, None]).to(torch.float8_e4m3fn)
    return codes.flatten(-3, -2), scale


def _inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    n, d, hq, hkv, P = _new(c), c["d"], c["hq"], c["hkv"], c["page"]
    _, pages = _tables(c)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {}
    # the cache's rows
    rows = randn(pages, 2, hkv, P, d)
    rows *= torch.exp(0.5 * randn(pages, 2, hkv, P, 1))
    rows[:, 0] *= torch.exp(0.4 * randn(1, hkv, 1, d))    # channels of the keys
    rows[:, 1] *= torch.exp(0.7 * randn(1, hkv, 1, 1))    # heads of the values
    codes, scales = _quantised(rows)
    del rows
    # as the cache holds them: the codes of all pages, then their scales
    s["pool"] = torch.cat([codes.view(torch.uint8).reshape(-1), scales.reshape(-1).view(torch.uint8)])
    s["codes"] = s["pool"][:codes.numel()].view(pages, 2, hkv, P, d)
    s["scales"] = s["pool"][codes.numel():].view(torch.float32).view(pages, 2, hkv, P // BLOCK)
    if c["kind"] != "store":
        sharp = torch.tensor([SHARPNESS[h % (hq // hkv) % len(SHARPNESS)] for h in range(hq)])
        s["q"] = (randn(n, hq, d) * sharp.cuda()[None, :, None]).bfloat16()
        return s
    # what the fused projection leaves, heads at scales of their own
    qkv = randn(n, hq + 2 * hkv, d) * torch.exp(randn(1, hq + 2 * hkv, 1))
    s["qkv"] = (qkv * torch.exp(0.5 * randn(n, 1, 1))).bfloat16()
    s["q"], s["k"], s["v"] = s["qkv"].split([hq, hkv, hkv], dim=1)
    dt = torch.float32 if c["weights"] == "f32" else torch.bfloat16
    for w in ("q_weight", "k_weight"):
        s[w] = (1 + 0.3 * randn(d)).to(dt)
    inv = THETA ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64)
                    / max(c["rot"], 1))
    angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * inv
    s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    # positions far above the rows in the cache, most of whose predecessors were evicted
    rng, pos = random.Random(c["layout"] + 2), []
    for _, new in _lengths(c):
        at = rng.randint(0, MAX_POS - new)
        pos.extend(range(at, at + new))
    s["positions"] = torch.tensor(pos, dtype=torch.int32).cuda()
    return s


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    s["case"] = c
    s["lengths"] = _lengths(c)
    s["new"] = [new for _, new in s["lengths"]]
    if c["kind"] == "tree":
        s["parents"] = [p for t in _trees(c) for p in t]
    if c["kind"] == "store":
        # the rows read back: the new ones and those that may share a block with them
        s["back"] = [min(n, new + BLOCK - 1) for n, new in s["lengths"]]
    if own:
        import paper_2602_22603_gb300 as sq
        _open(sq, s)
    else:
        _plan(s)
    return s


def _open(sq, s):
    """The cache, its sequences and the buffers that a serving program holds."""
    c, P = s["case"], s["case"]["page"]
    cache = sq.Cache(1, c["hq"], c["hkv"], c["d"], P, s["codes"].shape[0], max_seqs=len(s["new"]),
                     kv_pool=s["pool"], bits=8)
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
    if c["kind"] == "store":
        s["params"] = sq.norm_rope(s["rope"], c["rot"], EPS, s["q_weight"], s["k_weight"],
                                   interleaved=c["pairs"])
        s["q_out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["k_back"], s["v_back"] = (torch.empty(sum(s["back"]), c["hkv"], c["d"], dtype=torch.bfloat16,
                                                device="cuda") for _ in range(2))
    else:
        s["out"] = torch.empty_like(s["q"])


def _plan(s):
    """What the plain forms index with: the page and slot of every row."""
    c, P = s["case"], s["case"]["page"]
    tables, _ = _tables(c)
    s["pages"] = [torch.tensor(t, dtype=torch.int64).cuda() for t in tables]
    if c["kind"] == "store":
        # the blocks with new rows: their place, and for every slot the new row that
        # goes there, or -1 (it keeps its row) or -2 (it has none)
        page, block, source, back, at = [], [], [], [], 0
        for t, (n, new), m in zip(tables, s["lengths"], s["back"]):
            for b in range((n - new) // BLOCK, -(-n // BLOCK)):
                page.append(t[b * BLOCK // P])
                block.append(b * BLOCK % P // BLOCK)
                source.append([-2 if j >= n else at + j - (n - new) if j >= n - new else -1
                               for j in range(b * BLOCK, (b + 1) * BLOCK)])
            back.extend((t[j // P], j % P) for j in range(n - m, n))
            at += new
        s["page"], s["block"], s["source"] = (torch.tensor(x).cuda() for x in (page, block, source))
        s["back_page"], s["back_slot"] = torch.tensor(back).cuda().unbind(1)
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
    s["cache"].read_kv(s["handles"], s["back"], 0, s["k_back"], s["v_back"])
    return s["q_out"], s["k_back"], s["v_back"]


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


_OWN = dict(store=_own_store, tokens=_own_window, chunks=_own_window, tree=_own_tree)


def _plain_norm(s, x, w):
    """x normed and rotated, in 32 bits."""
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s[w].float()
    cs = s["rope"][s["positions"].long()][:, None]
    cos, sin, r = cs[..., 0], cs[..., 1], s["case"]["rot"]
    if s["case"]["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_store(s):
    page, block, source = s["page"], s["block"], s["source"]
    codes = s["codes"].view(*s["codes"].shape[:3], -1, BLOCK, s["case"]["d"])
    fresh = (source >= 0)[:, None, :, None]
    some = (source > -2)[:, None, :, None]
    for plane, x in ((0, _plain_norm(s, s["k"], "k_weight")), (1, s["v"].float())):
        old = codes[page, plane, :, block]                 # [blocks, hkv, slots, d]
        scale = s["scales"][page, plane, :, block]
        rows = old.view(torch.float8_e4m3fn).float() * scale[..., None, None]
        rows = torch.where(fresh, x[source.clamp(min=0)].transpose(1, 2), rows)
        now, scale = _quantised(torch.where(some, rows, 0.0))
        codes[page, plane, :, block] = torch.where(some, now.view(torch.uint8).view(old.shape), old)
        s["scales"][page, plane, :, block] = scale[..., 0]
    back = [_plain_rows(s, s["back_page"], s["back_slot"], plane).bfloat16() for plane in (0, 1)]
    return _plain_norm(s, s["q"], "q_weight").bfloat16(), back[0], back[1]


def _plain_rows(s, page, slot, plane):
    """What the 8 bits of rows stand for, [rows, hkv, d]."""
    x = s["codes"][page, plane, :, slot].view(torch.float8_e4m3fn).float()
    return x * s["scales"][page, plane, :, slot // BLOCK][..., None]


def _plain_attend(s, i, q, keep, rows):
    """Queries q over the cache rows `rows` of sequence i that `keep` allows."""
    c = s["case"]
    page, slot = s["pages"][i][rows // c["page"]], rows % c["page"]
    k = _plain_rows(s, page, slot, 0).transpose(0, 1)               # [hkv, rows, d]
    v = _plain_rows(s, page, slot, 1).transpose(0, 1)
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
        reach = c["window"] or n + 1
        for b in range(0, new, 256):
            m = min(256, new - b)
            at_pos = n - new + b + torch.arange(m, device="cuda")[:, None]
            low = max(0, n - new + b - reach + 1)
            rows = torch.cat([torch.arange(min(c["sinks"], low), device="cuda"),
                              torch.arange(low, n - new + b + m, device="cuda")])
            keep = (rows <= at_pos) & ((rows > at_pos - reach) | (rows < c["sinks"]))
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


_PLAIN = dict(store=_plain_store, tokens=_plain_window, chunks=_plain_window, tree=_plain_tree)


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
            near = min(max(reach - ctx, 0), new)           # queries that see all before them
            pairs += near * (2 * ctx + near + 1) // 2 + (new - near) * reach
            first = ctx + near - reach + 1                 # rows before the next one's window
            some = min(new - near, max(0, c["sinks"] - first))
            pairs += some * first + some * (some - 1) // 2 + (new - near - some) * c["sinks"]
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
    c, n = case, _new(case)
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    row = 2 * hkv * d + 2 * hkv * 4 / BLOCK                # a cache row and its share of the scales
    if c["kind"] == "store":
        back = sum(min(m, new + BLOCK - 1) for m, new in _lengths(c))
        return {"bytes": n * (2 * hq + 2 * hkv) * d * 2 + n * (4 + c["rot"] * 4) + back * row
                + back * 2 * hkv * d * 2, "flops": n * (hq + hkv) * d * 7}
    rows, pairs = _seen(c)
    return {"bytes": rows * row + n * hq * d * 4, "flops": pairs * hq * d * 4}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.8e12, w["flops"] / 1.5e15)


# ---- the definitions in 64 bits ----------------------------------------------
def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    if c["kind"] == "store":
        return _exact_store(c, s)
    if work(c)["flops"] * 2 > 6e12:
        return None
    return _exact_attention(c, s)


def _nearest_e4m3(x):
    """The e4m3 value nearest to x (|x| <= 448), ties to an even last digit: 4
    significant bits, and steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_store(c, s):
    hq, hkv, d, half, P = c["hq"], c["hkv"], c["d"], c["rot"] // 2, c["page"]
    pos = s["positions"].long()
    angle = torch.complex(s["rope"][pos, :, 0].double(), s["rope"][pos, :, 1].double())
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)

    def normed(x, w):
        x = x.double()
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / d + EPS) * s[w].double()
        z = torch.complex(x[..., first], x[..., second]) * angle[:, None]
        x[..., first], x[..., second] = z.real, z.imag
        return x

    fresh = torch.stack([normed(s["k"], "k_weight"), s["v"].double()], 2)   # [n, hkv, 2, d]
    back, at = [], 0
    for t, (n, new) in zip(_tables(c)[0], _lengths(c)):
        a, m = (n - new) // BLOCK * BLOCK, min(n, new + BLOCK - 1)
        j = torch.arange(min(a, n - m), n, device="cuda")   # the rows read back, and those of their blocks
        page = torch.tensor(t, device="cuda")[j // P]
        rows = s["codes"][page, :, :, j % P].view(torch.float8_e4m3fn).double()
        rows = (rows * s["scales"][page, :, :, j % P // BLOCK].double()[..., None]).transpose(1, 2)
        rows[-new:] = fresh[at:at + new]
        # one scale for the rows of a block
        tail = rows[a - n:]
        size = tail.abs().amax(-1)                          # [rows, hkv, 2]
        size = torch.cat([size, size.new_zeros(-size.shape[0] % BLOCK, *size.shape[1:])])
        size = size.view(-1, BLOCK, *size.shape[1:]).amax(1).clamp(min=1e-300) / E4M3_MOST
        e = torch.ceil(torch.log2(size)).clamp(min=LEAST_SCALE)
        e = torch.where(torch.exp2(e - 1) >= size, e - 1, e).clamp(min=LEAST_SCALE)
        scale = torch.exp2(e).repeat_interleave(BLOCK, 0)[:tail.shape[0], ..., None]
        rows[a - n:] = _nearest_e4m3(tail / scale) * scale
        back.append(rows[rows.shape[0] - m:])
        at += new
    back = torch.cat(back)
    return normed(s["q"], "q_weight"), back[:, :, 0], back[:, :, 1]


def _exact_attention(c, s):
    d, group, P = c["d"], c["hq"] // c["hkv"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    trees = _trees(c) if c["kind"] == "tree" else None
    at = 0
    for i, (t, (n, new)) in enumerate(zip(_tables(c)[0], _lengths(c))):
        ctx, ids, index = n - new, torch.tensor(t, device="cuda"), torch.arange(n, device="cuda")
        for b in range(0, new, 128):
            e = min(new, b + 128)
            if trees is None:
                where, place = index, ctx + torch.arange(b, e, device="cuda")
                see = index[None] <= place[:, None]
            else:
                line, depth = [], []
                for p in trees[i]:
                    line.append((line[p] if p >= 0 else []) + [len(line)])
                    depth.append(len(line[-1]) - 1)
                where = torch.cat([index[:ctx], ctx + torch.tensor(depth, device="cuda")])
                place = where[ctx + b:ctx + e]
                see = torch.zeros(e - b, n, dtype=torch.bool, device="cuda")
                see[:, :ctx] = True
                for r in range(b, e):
                    see[r - b, [ctx + x for x in line[r]]] = True
            if c["window"]:
                see &= (place[:, None] - where[None] < c["window"]) | (where < c["sinks"])[None]
            some = see.any(0).nonzero()[:, 0]
            see = see[:, some]
            page, slot = ids[some // P], some % P
            rows = s["codes"][page, :, :, slot].view(torch.float8_e4m3fn).double()
            rows *= s["scales"][page, :, :, slot // BLOCK].double()[..., None]   # [rows, 2, hkv, d]
            for h in range(c["hq"]):
                key, val = rows[:, 0, h // group], rows[:, 1, h // group]
                a = s["q"][at + b:at + e, h].double() @ key.T / math.sqrt(d)
                a = torch.where(see, a, torch.tensor(-math.inf, dtype=a.dtype, device="cuda"))
                out[at + b:at + e, h] = torch.exp(a - torch.logsumexp(a, 1, keepdim=True)) @ val
        at += new
    return out
