"""The operators around the linears when drafted tokens are verified, as cases that can be timed and checked.

A model that is served at several bitwidths drafts tokens with the narrow one and verifies them with the wide one.  Four kinds of pass:

  rope    rotary positions of the queries and the keys of some tokens, or the gradient of that
  attend  attention of a tree of drafted tokens over a cache of pages and over the tree itself
  verify  which drafted tokens stand against the target's probabilities, and the token behind them
  append  the keys and values of the tokens that stand go into the cache, all layers at once

`own` chooses between the library's calls and elementary torch operations.
"""
import math
import random

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------------------
def _rope(name, dtype, batch, tokens, heads, kv, dim, rotary, layout, scaling, first, inverse):
    c = {"kind": "rope", "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "rotary": rotary,
         "layout": layout, "scaling": scaling, "first": first, "inverse": inverse}
    return dict(c, name=name) if name else c


def _attend(name, dtype, batch, nodes, heads, kv, dim, shortest, longest, page, branch):
    """page 0: every sequence has one stretch of memory; branch 0: the drafted tokens are a chain."""
    c = {"kind": "attend", "dtype": dtype, "batch": batch, "nodes": nodes, "heads": heads, "kv": kv, "dim": dim, "shortest": shortest,
         "longest": longest, "page": page, "branch": branch}
    return dict(c, name=name) if name else c


def _verify(name, dtype, batch, nodes, words, branch, draft, greedy):
    """greedy: every such sequence takes the target's best token (0: none does)."""
    c = {"kind": "verify", "dtype": dtype, "batch": batch, "nodes": nodes, "words": words, "branch": branch, "draft": draft, "greedy": greedy}
    return dict(c, name=name) if name else c


def _append(name, dtype, layers, batch, nodes, kv, dim, shortest, longest, page, branch):
    c = {"kind": "append", "dtype": dtype, "layers": layers, "batch": batch, "nodes": nodes, "kv": kv, "dim": dim, "shortest": shortest,
         "longest": longest, "page": page, "branch": branch}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence: what every layer of every step asks for
        _rope("rope_one_token", "f16", 1, 1, 32, 8, 128, 128, "half", "plain", 700, False),
        # drafted trees of a batch far into long contexts, part of the head, neighbours as pairs
        _rope("rope_trees_part", "bf16", 24, 27, 64, 8, 128, 96, "interleaved", "yarn", 100000, False),
        # the gradient over whole sequences of a fine-tuning batch
        _rope("rope_gradient", "bf16", 4, 4099, 32, 32, 128, 128, "half", "bands", 0, True),
        # the next token of one conversation, no drafts
        _attend("attend_one_token", "f16", 1, 1, 32, 8, 128, 900, 900, 0, 0),
        # eight drafted tokens in four sequences, every head with keys of its own
        _attend("attend_own_heads", "f16", 4, 8, 32, 32, 128, 1500, 4095, 16, 0),
        # a batch of trees over contexts of very different lengths
        _attend("attend_ragged", "bf16", 24, 13, 64, 8, 128, 37, 16000, 64, 3),
        # a large tree over one long context
        _attend("attend_long", "bf16", 1, 63, 32, 8, 128, 130001, 130001, 256, 4),
        # a chain of five for one conversation, small vocabulary
        _verify("verify_chain", "f16", 1, 6, 32000, 0, True, 0),
        # trees of a batch whose children were named, not drawn; some sequences take the best token
        _verify("verify_trees", "f32", 6, 33, 128256, 3, False, 2),
        # many chains at once, large vocabulary
        _verify("verify_batch", "bf16", 48, 8, 128256, 0, True, 3),
        # one conversation's accepted tokens
        _append("append_one", "f16", 32, 1, 8, 8, 128, 1000, 1000, 16, 2),
        # a batch's accepted tokens
        _append("append_batch", "bf16", 48, 16, 27, 8, 128, 100, 350, 64, 3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "attend", "attend", "verify", "append"])
    dtype = rng.choice(["f16", "bf16"])
    heads, kv = rng.choice([(32, 32), (32, 8), (64, 8), (16, 2), (24, 4), (12, 1), (7, 7), (40, 8)])
    dim = rng.choice([64, 96, 128, 128, 256])
    if kind == "rope":
        dtype = rng.choice(["f16", "bf16", "f32"])
        inverse = rng.random() < 0.4
        batch = rng.randint(1, 24)
        tokens = _log_int(rng, 1, max(1, int((6e7 if dtype == "f32" else 1.2e8) / (batch * (heads + kv) * dim))))
        rotary = rng.choice([dim, dim, dim // 2, dim // 4 * 3])
        return _rope(None, dtype, batch, tokens, heads, kv, dim, rotary, rng.choice(["half", "interleaved"]),
                     rng.choice(["plain", "linear", "ntk", "yarn", "bands"]), rng.choice([0, 5000, 120000]), inverse)
    branch = rng.choice([0, 2, 3, 4])
    if kind == "attend":
        batch, nodes = _log_int(rng, 1, 32), _log_int(rng, 1, 64)
        most = max(16, min(130000, int(1.3e8 / (batch * kv * dim)), int(2.4e10 / (batch * nodes * heads * dim))))
        longest = _log_int(rng, 1, most)
        return _attend(None, dtype, batch, nodes, heads, kv, dim, max(1, int(longest * rng.uniform(0.01, 1.0))), longest,
                       rng.choice([0, 16, 32, 64, 128]), branch)
    if kind == "verify":
        dtype = rng.choice(["f16", "bf16", "f32"])
        words = _log_int(rng, 1000, 152000)
        batch = _log_int(rng, 1, 48)
        nodes = _log_int(rng, 2, max(2, min(64, int(4.8e7 / (batch * words)))))
        draft = rng.random() < 0.5
        return _verify(None, dtype, batch, nodes, words, rng.choice([0, 2]) if draft else branch, draft, rng.choice([0, 0, 2, 3]))
    batch, nodes, longest = _log_int(rng, 1, 16), _log_int(rng, 1, 64), _log_int(rng, 1, 2000)
    layers = rng.randint(1, max(1, min(80, int(3e8 / (batch * (longest + nodes + 64) * kv * dim)))))
    return _append(None, dtype, layers, batch, nodes, kv, dim, max(1, longest // rng.randint(1, 8)), longest, rng.choice([0, 16, 32, 64]), branch)


def _lens(c):
    """Context lengths of a batch: evenly spread over their logarithm."""
    n, lo, hi = c["batch"], c["shortest"], c["longest"]
    return [hi if n == 1 else int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]


def _parents(c):
    """A tree of the drafted tokens, the root first, parents before children, up to `branch` children to a node."""
    n, branch = c["nodes"], c["branch"]
    if branch == 0:
        return list(range(-1, n - 1))
    rng, parents, room = random.Random(n * 100 + branch), [-1], [0]
    children = [0] * n
    for i in range(1, n):
        at = room[min(len(room) - 1, int(rng.random() ** 1.5 * len(room)))]
        parents.append(at)
        children[at] += 1
        if children[at] == branch:
            room.remove(at)
        room.append(i)
    return parents


def _ancestors(parents):
    """Row i: the nodes that node i sees, itself among them."""
    rows = []
    for i, p in enumerate(parents):
        rows.append(([] if p < 0 else rows[p]) + [i])
    return rows


def _kept(c):
    """How many nodes of every sequence go into the cache: from one to the depth of the tree."""
    deepest = max(len(r) for r in _ancestors(_parents(c)))
    return [1 + b * 7 % deepest for b in range(c["batch"])] if c["batch"] > 1 else [(deepest + 1) // 2]


def _pages(c):
    """Tokens to a page, and pages to a sequence; there is room for the drafted tokens behind the longest context."""
    need = c["longest"] + c["nodes"]
    return (need, 1) if c["page"] == 0 else (c["page"], -(-need // c["page"]))


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rope":
        n = c["batch"] * c["tokens"]
        each = n * (c["heads"] + c["kv"])
        return {"bytes": 2 * each * c["dim"] * es + 4 * n, "flops": 3 * each * c["rotary"]}
    if c["kind"] == "attend":
        seen = sum(len(r) for r in _ancestors(_parents(c)))
        b, t, lens = c["batch"], c["nodes"], sum(_lens(c))
        values = 2 * (lens + b * t) * c["kv"] * c["dim"] + 2 * b * t * c["heads"] * c["dim"]
        return {"bytes": values * es + 4 * b * t * c["heads"], "flops": 4 * c["dim"] * c["heads"] * (t * lens + b * seen)}
    if c["kind"] == "verify":
        n = c["batch"] * c["nodes"] * c["words"] * (2 if c["draft"] else 1)
        return {"bytes": n * es + 20 * c["batch"] * c["nodes"], "flops": 4 * n}
    n = 2 * c["layers"] * sum(_kept(c)) * c["kv"] * c["dim"]
    return {"bytes": 2 * n * es, "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------
def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    n = int(seed)
    for k in key:
        n = (n * 1000003 + int(k)) % (2 ** 61 - 1)
    g.manual_seed(n)
    return g


def _normal(g, *shape, dtype):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


_SCALINGS = {   # scaling -> base, factor, length trained on, low, high
    "plain": (10000.0, 1.0, 0, 1.0, 1.0),
    "linear": (10000.0, 4.0, 4096, 1.0, 1.0),
    "ntk": (10000.0, 8.0, 8192, 1.0, 1.0),
    "yarn": (1000000.0, 16.0, 8192, 1.0, 32.0),
    "bands": (500000.0, 8.0, 8192, 1.0, 4.0),
}


def _frequencies(rotary, scaling):
    """Angle per position of every pair, 64 bits, and what the rotated part is multiplied by."""
    base, factor, trained, low, high = _SCALINGS[scaling]
    n = rotary // 2
    if scaling == "ntk":
        base *= factor ** (rotary / (rotary - 2))
    f = [base ** (-2.0 * i / rotary) for i in range(n)]
    scale = 1.0
    if scaling == "linear":
        f = [v / factor for v in f]
    elif scaling == "yarn":
        place = [rotary * math.log(trained / (r * 2 * math.pi)) / (2 * math.log(base)) for r in (high, low)]
        lo, hi = max(math.floor(place[0]), 0), min(math.ceil(place[1]), rotary - 1)
        hi = hi if hi > lo else lo + 0.001
        ramp = [min(max((i - lo) / (hi - lo), 0.0), 1.0) for i in range(n)]
        f = [v * (1 - r) + v / factor * r for v, r in zip(f, ramp)]
        scale = 0.1 * math.log(factor) + 1.0
    elif scaling == "bands":
        out = []
        for v in f:
            turns = trained * v / (2 * math.pi)      # over the length trained on
            s = min(max((turns - low) / (high - low), 0.0), 1.0)
            out.append((1 - s) * v / factor + s * v)
        f = out
    return f, scale


def _cache(c, g, layers, s):
    """A pool of pages with every sequence's pages spread over it, filled, and its table."""
    page, each = _pages(c)
    n = c["batch"] * each
    dtype = _TYPES[c["dtype"]]
    s["k"] = torch.empty(layers, n, page, c["kv"], c["dim"], dtype=dtype, device="cuda")
    s["v"] = torch.empty_like(s["k"])
    for l in range(layers):
        s["k"][l] = _normal(g, n, page, c["kv"], c["dim"], dtype=dtype)
        s["v"][l] = _normal(g, n, page, c["kv"], c["dim"], dtype=dtype)
    order = torch.randperm(n, generator=g, device="cuda") if c["page"] else torch.arange(n, device="cuda")
    s["table"] = order.reshape(c["batch"], each).to(torch.int32)
    lens = _lens(c)
    order = torch.randperm(c["batch"], generator=g, device="cuda")
    s["lens"] = _ints(lens)[order]
    if own:
        import paper_2508_06041_amd as dp
        s["cache"] = dp.Cache(s["k"], s["v"], s["table"])


def prepare(c, seed):
    s = {"case": c}
    dtype = _TYPES[c["dtype"]]
    g = _gen(seed, 1)
    if c["kind"] == "rope":
        b, t, d = c["batch"], c["tokens"], c["dim"]
        # as the projections leave them: queries, keys and values of a token side by side
        qkv = _normal(g, b, t, c["heads"] + 2 * c["kv"], d, dtype=dtype)
        s["q"], s["keys"] = qkv[:, :, :c["heads"]], qkv[:, :, c["heads"]:c["heads"] + c["kv"]]
        first = torch.randint(0, 1 + c["first"], (b, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(t, device="cuda")).to(torch.int32)
        if own:
            import paper_2508_06041_amd as dp
            base, factor, trained, low, high = _SCALINGS[c["scaling"]]
            s["plan"] = dp.dpllm_rope_frequencies(c["rotary"], base, getattr(dp, "DPLLM_ROPE_" + c["scaling"].upper()), factor, trained, low, high)
            s["layout"] = getattr(dp, "DPLLM_ROPE_" + c["layout"].upper())
        else:
            f, s["scale"] = _frequencies(c["rotary"], c["scaling"])
            s["freqs"] = torch.tensor(f, dtype=torch.float64, device="cuda")
    elif c["kind"] == "attend":
        b, t, d = c["batch"], c["nodes"], c["dim"]
        _cache(c, g, 1, s)
        # some directions of the keys are stronger than others, so that few tokens carry most of the weight
        strong = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
        s["q"] = (torch.randn(b, t, c["heads"], d, generator=g, device="cuda") * strong).to(dtype)
        s["k_new"], s["v_new"] = _normal(g, b, t, c["kv"], d, dtype=dtype), _normal(g, b, t, c["kv"], d, dtype=dtype)
        rows = [sum(1 << j for j in r) for r in _ancestors(_parents(c))]
        words = [r - (1 << 64) if r >= 1 << 63 else r for r in rows]
        s["mask"] = torch.tensor(words, dtype=torch.int64, device="cuda").reshape(1, t, 1)
    elif c["kind"] == "verify":
        b, t, v = c["batch"], c["nodes"], c["words"]
        parents = _parents(c)
        s["parents"] = _ints(parents).repeat(b, 1)
        s["temperature"] = torch.rand(b, generator=g, device="cuda") * 0.7 + 0.6
        if c["greedy"]:
            s["temperature"][::c["greedy"]] = 0.0
        s["uniforms"] = torch.rand(b, t, generator=g, device="cuda")
        s["logits"] = torch.empty(b, t, v, dtype=dtype, device="cuda")
        s["draft"] = torch.empty_like(s["logits"]) if c["draft"] else None
        s["tokens"] = torch.zeros(b, t, dtype=torch.int32, device="cuda")
        for i in range(t):
            # few words carry most of the probability, and the draft is near the target
            x = torch.randn(b, v, generator=g, device="cuda") * 2.5
            x[torch.arange(b, device="cuda")[:, None], torch.randint(0, v, (b, 8), generator=g, device="cuda")] += 9.0
            s["logits"][:, i] = x.to(dtype)
            x = x + 0.4 * torch.randn(b, v, generator=g, device="cuda")
            mine = [j for j in range(1, t) if parents[j] == i]
            if c["draft"]:
                s["draft"][:, i] = x.to(dtype)
                w = torch.softmax(x / s["temperature"].clamp(min=0.05)[:, None], dim=1)
                if mine:
                    s["tokens"][:, mine] = torch.multinomial(w, len(mine), replacement=True, generator=g).to(torch.int32)
            elif mine:
                s["tokens"][:, mine] = torch.topk(x, len(mine), dim=1).indices.to(torch.int32)
        s["siblings"] = max(parents.count(p) for p in range(t)) if t > 1 else 1
    else:
        b, t, d, layers = c["batch"], c["nodes"], c["dim"], c["layers"]
        _cache(c, g, layers, s)
        s["k_new"] = torch.empty(layers, b, t, c["kv"], d, dtype=dtype, device="cuda")
        s["v_new"] = torch.empty_like(s["k_new"])
        for l in range(layers):
            s["k_new"][l], s["v_new"][l] = _normal(g, b, t, c["kv"], d, dtype=dtype), _normal(g, b, t, c["kv"], d, dtype=dtype)
        rows, kept = _ancestors(_parents(c)), _kept(c)
        order = torch.randperm(b, generator=g, device="cuda").tolist()
        kept = [kept[i] for i in order]
        paths = []
        for n in kept:
            reach = [r for r in rows if len(r) >= n]
            r = reach[int(torch.randint(0, len(reach), (1,), generator=g, device="cuda"))][:n]
            paths.append(r + [-1] * (t - n))
        s["path"], s["count"] = _ints(paths), _ints(kept)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, c):
    import paper_2508_06041_amd as dp
    if c["kind"] == "rope":
        freqs, scale = s["plan"]
        return dp.dpllm_rope((s["q"], s["keys"]), s["positions"], freqs, scale=scale, layout=s["layout"], inverse=c["inverse"])
    if c["kind"] == "attend":
        lse = torch.empty(c["batch"], c["nodes"], c["heads"], dtype=torch.float32, device="cuda")
        out = dp.dpllm_tree_attention(s["cache"], 0, s["lens"], s["q"], s["k_new"], s["v_new"], mask=s["mask"], lse=lse, max_len=c["longest"])
        return out, lse
    if c["kind"] == "verify":
        return dp.dpllm_verify(s["logits"], s["tokens"], s["uniforms"], s["temperature"], parents=s["parents"], draft=s["draft"],
                               siblings=s["siblings"])
    dp.dpllm_cache_append(s["cache"], s["lens"], s["k_new"], s["v_new"], path=s["path"], count=s["count"])
    return s["k"], s["v"]


def _run_plain(s, c):
    return {"rope": _plain_rope, "attend": _plain_attend, "verify": _plain_verify, "append": _plain_append}[c["kind"]](s, c)


def _plain_rope(s, c):
    angle = s["positions"].double()[:, :, None, None] * s["freqs"]      # far positions: an angle of 32 bits is off by whole degrees
    sin = (torch.sin(angle) * (-s["scale"] if c["inverse"] else s["scale"])).float()
    cos = (torch.cos(angle) * s["scale"]).float()
    outs, r = [], c["rotary"]
    for x in (s["q"], s["keys"]):
        y = x.float()
        if c["layout"] == "half":
            a, b = y[..., :r // 2], y[..., r // 2:r]
            turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
        else:
            a, b = y[..., 0:r:2], y[..., 1:r:2]
            turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
        outs.append(torch.cat([turned, y[..., r:]], dim=-1).to(x.dtype))
    return tuple(outs)


def _plain_attend(s, c):
    b, t, kv, d, n = c["batch"], c["nodes"], c["kv"], c["dim"], c["longest"]
    group = c["heads"] // kv
    old = torch.arange(n, device="cuda") < s["lens"][:, None]                               # [b][n]
    bits = torch.arange(t, device="cuda")
    tree = ((s["mask"] >> bits) & 1).bool().expand(b, t, t)
    seen = torch.cat([old[:, None, :].expand(b, t, n), tree], dim=2)                        # [b][t][n + t]
    k = torch.cat([s["k"][0][s["table"].long()].flatten(1, 2)[:, :n], s["k_new"]], dim=1).float()
    v = torch.cat([s["v"][0][s["table"].long()].flatten(1, 2)[:, :n], s["v_new"]], dim=1).float()
    v = torch.where(torch.cat([old, torch.ones_like(tree[:, 0])], dim=1)[:, :, None, None], v, 0.0)
    q = s["q"].float().reshape(b, t, kv, group, d).permute(0, 2, 3, 1, 4).reshape(b, kv, group * t, d)
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(d))
    x = x.reshape(b, kv, group, t, n + t).masked_fill(~seen[:, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    z = e.sum(dim=-1, keepdim=True)
    o = torch.matmul(e.reshape(b, kv, group * t, n + t), v.permute(0, 2, 1, 3).contiguous()).reshape(b, kv, group, t, d)
    o = torch.where(z > 0, o / z, 0.0).permute(0, 3, 1, 2, 4).reshape(b, t, c["heads"], d)
    lse = (top + torch.log(z)).squeeze(-1).permute(0, 3, 1, 2).reshape(b, t, c["heads"])
    return o.to(s["q"].dtype), lse


def _plain_verify(s, c):
    # 64 bits throughout: the answers are whole numbers, and sums of many small probabilities decide them
    b, t, v = c["batch"], c["nodes"], c["words"]
    at = torch.arange(b, device="cuda")
    greedy = s["temperature"] == 0
    temp = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]

    def chances(rows):                                                                      # [b][v]
        x = rows.double()
        e = torch.exp((x - x.amax(dim=1, keepdim=True)) / temp)
        best = torch.zeros_like(e).scatter_(1, rows.float().argmax(dim=1, keepdim=True), 1.0)
        return torch.where(greedy[:, None], best, e / e.sum(dim=1, keepdim=True))

    node = torch.zeros(b, dtype=torch.int64, device="cuda")
    left = chances(s["logits"][:, 0])                                                       # what is left of the node's distribution
    q = chances(s["draft"][:, 0]) if c["draft"] else None
    depth = torch.ones(b, dtype=torch.int64, device="cuda")
    path = torch.full((b, t), -1, dtype=torch.int64, device="cuda")
    path[:, 0] = 0
    words = torch.full((b, t), -1, dtype=torch.int64, device="cuda")
    u = s["uniforms"].double()
    for i in range(1, t):
        asked = s["parents"][:, i] == node
        word = s["tokens"][:, i].long()
        have = left[at, word]
        if c["draft"]:
            stands = torch.where(greedy, have > 0, u[:, i] * q[at, word] < have)
            less = torch.clamp(left - q, min=0)
        else:
            stands = torch.where(greedy, have > 0, u[:, i] < have)
            less = left.scatter(1, word[:, None], 0.0)
        total = less.sum(dim=1, keepdim=True)
        less = torch.where((total > 0) & ~greedy[:, None], less / torch.where(total > 0, total, 1.0), left)
        left = torch.where((asked & ~stands)[:, None], less, left)
        on = asked & stands
        node = torch.where(on, i, node)
        path[at, depth.clamp(max=t - 1)] = torch.where(on, i, path[at, depth.clamp(max=t - 1)])
        words[at, depth - 1] = torch.where(on, word, words[at, depth - 1])
        depth = depth + on
        left = torch.where(on[:, None], chances(s["logits"][:, i]), left)
        if c["draft"]:
            q = torch.where(on[:, None], chances(s["draft"][:, i]), q)
    run_ = torch.cumsum(left, dim=1)
    over = run_ > u[:, :1] * run_[:, -1:]
    drawn = torch.where(greedy, left.argmax(dim=1), over.to(torch.uint8).argmax(dim=1))
    words[at, depth - 1] = drawn
    return depth.to(torch.int32), path.to(torch.int32), words.to(torch.int32)


def _plain_append(s, c):
    b, t = c["batch"], c["nodes"]
    page = s["k"].shape[2]
    step = torch.arange(t, device="cuda")
    slot = s["lens"].long()[:, None] + step
    where = s["table"].long().gather(1, slot // page)
    keep = (step < s["count"][:, None])[None, :, :, None, None]
    take = s["path"].long().clamp(min=0)
    seq = torch.arange(b, device="cuda")[:, None]
    for mine, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        mine[:, where, slot % page] = torch.where(keep, new[:, seq, take], mine[:, where, slot % page])
    return s["k"], s["v"]


# ---- the same from the definitions in 64 bits --------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] == "verify":
        return None      # whole numbers
    s = prepare(c, seed)
    if c["kind"] == "rope":
        f, scale = _frequencies(c["rotary"], c["scaling"])
        r, outs = c["rotary"], []
        w = torch.polar(torch.full((), scale, dtype=torch.float64, device="cuda"),
                        s["positions"].double()[..., None] * torch.tensor(f, dtype=torch.float64, device="cuda"))
        w = w.conj() if c["inverse"] else w
        for x in (s["q"], s["keys"]):
            y = x.double()
            for h in range(x.shape[2]):
                z = y[:, :, h, :r].reshape(*x.shape[:2], 2, r // 2).transpose(2, 3) if c["layout"] == "half" else \
                    y[:, :, h, :r].reshape(*x.shape[:2], r // 2, 2)
                z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * w)
                y[:, :, h, :r] = (z.transpose(2, 3) if c["layout"] == "half" else z).reshape(*x.shape[:2], r)
            outs.append(y)
        return tuple(outs)
    if c["kind"] == "append":
        k, v = s["k"].clone(), s["v"].clone()
        lens, table, path, count = (s[n].tolist() for n in ("lens", "table", "path", "count"))
        page = k.shape[2]
        for b in range(c["batch"]):
            for i in range(count[b]):
                at = lens[b] + i
                k[:, table[b][at // page], at % page] = s["k_new"][:, b, path[b][i]]
                v[:, table[b][at // page], at % page] = s["v_new"][:, b, path[b][i]]
        return k, v
    rows = _ancestors(_parents(c))
    lens, table = s["lens"].tolist(), s["table"].long()
    group = c["heads"] // c["kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        sees = torch.zeros(c["nodes"], c["nodes"], dtype=torch.bool)
        for i, r in enumerate(rows):
            sees[i, r] = True
        sees = torch.cat([torch.ones(c["nodes"], lens[b], dtype=torch.bool), sees], dim=1).cuda()
        for h in range(c["kv"]):
            k = torch.cat([s["k"][0, table[b], :, h].flatten(0, 1)[:lens[b]], s["k_new"][b, :, h]]).double()
            v = torch.cat([s["v"][0, table[b], :, h].flatten(0, 1)[:lens[b]], s["v_new"][b, :, h]]).double()
            for j in range(h * group, (h + 1) * group):
                x = (s["q"][b, :, j].double() @ k.t().contiguous() / math.sqrt(c["dim"])).masked_fill(~sees, float("-inf"))
                out[b, :, j] = torch.softmax(x, dim=1) @ v
                lse[b, :, j] = torch.logsumexp(x, dim=1)
    return out, lse
