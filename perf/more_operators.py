"""The operators of a decode step over a quantised cache, as cases that can be timed and checked.

Keys and values are held in 8 or 4 bits, with one scale for each token and head.  Five kinds of pass:

  norm    norms of queries and keys for each head with their rotary positions, or the gradient of that
  append  keys and values are quantised as they go into the cache, and read back
  read    a stretch of the cache is read back
  attend  attention of new tokens over such a cache and over one another
  sample  a word is drawn: temperature, top-k, top-p and min-p, from a given uniform number

`own` chooses between the library's calls and elementary torch operations.
"""
import math
import random

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------------------
def _norm(name, dtype, batch, tokens, heads, kv, dim, rotary, layout, weights, each, first, backward):
    """weights: the type of the weights; each: every head has weights of its own."""
    c = {"kind": "norm", "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "rotary": rotary, "layout": layout,
         "weights": weights, "each": each, "first": first, "backward": backward}
    return dict(c, name=name) if name else c


def _append(name, dtype, form, layers, batch, tokens, kv, dim, shortest, longest, page):
    c = {"kind": "append", "dtype": dtype, "form": form, "layers": layers, "batch": batch, "tokens": tokens, "kv": kv, "dim": dim, "shortest": shortest,
         "longest": longest, "page": page}
    return dict(c, name=name) if name else c


def _read(name, dtype, form, layers, batch, kv, dim, shortest, longest, page):
    c = {"kind": "read", "dtype": dtype, "form": form, "layers": layers, "batch": batch, "tokens": 0, "kv": kv, "dim": dim, "shortest": shortest, "longest": longest, "page": page}
    return dict(c, name=name) if name else c


def _attend(name, dtype, form, batch, tokens, heads, kv, dim, shortest, longest, page, branch):
    """page 0: every sequence has one stretch of memory; branch 0: the new tokens are a chain, else a tree with so many children to a node."""
    c = {"kind": "attend", "dtype": dtype, "form": form, "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "shortest": shortest, "longest": longest,
         "page": page, "branch": branch}
    return dict(c, name=name) if name else c


def _sample(name, dtype, rows, words, filters, boost):
    """boost: how far the logits of a few words stand above the others."""
    c = {"kind": "sample", "dtype": dtype, "rows": rows, "words": words, "filters": filters, "boost": boost}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token of one conversation, every layer of every step
        _norm("norm_one_token", "f16", 1, 1, 32, 8, 128, 128, "half", "f16", False, 900, False),
        # a batch of prompts whose heads are turned in part
        _norm("norm_prompts", "bf16", 3, 2111, 40, 8, 128, 96, "interleaved", "bf16", False, 5000, False),
        # fine-tuning: the gradient of whole sequences, weights kept in 32 bits
        _norm("norm_gradient", "bf16", 4, 2049, 32, 8, 128, 128, "half", "f32", False, 0, True),
        # one conversation's token goes into all layers
        _append("append_one", "f16", "e4m3", 32, 1, 1, 8, 128, 900, 900, 16),
        # prompts of a batch go into the cache, 4 bits
        _append("append_prompts", "bf16", "int4", 4, 6, 1023, 8, 128, 0, 300, 64),
        # a lone context is read back in one layer
        _read("read_one", "f16", "int8", 1, 1, 8, 128, 777, 777, 16),
        # the contexts of a batch are moved out of the cache
        _read("read_batch", "bf16", "int4", 2, 24, 8, 128, 37, 8001, 64),
        # the next token of one conversation
        _attend("attend_one_token", "f16", "e4m3", 1, 1, 32, 8, 128, 900, 900, 16, 0),
        # the next token of a batch with contexts of very different lengths
        _attend("attend_batch", "bf16", "int8", 32, 1, 64, 8, 128, 37, 24000, 64, 0),
        # drafted trees over long contexts, 4 bits
        _attend("attend_trees", "f16", "int4", 4, 13, 32, 8, 128, 9000, 65001, 128, 3),
        # one conversation, a small vocabulary, every filter
        _sample("sample_one", "f16", 1, 32000, "all", 12.0),
        # a batch whose sequences have their own settings, a large vocabulary
        _sample("sample_batch", "bf16", 64, 128256, "mixed", 9.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "append", "read", "attend", "attend", "sample"])
    dtype, form = rng.choice(["f16", "bf16"]), rng.choice(["e4m3", "int8", "int4"])
    heads, kv = rng.choice([(32, 32), (32, 8), (64, 8), (16, 2), (24, 4), (12, 1), (7, 7), (40, 8)])
    dim = rng.choice([64, 96, 128, 128, 256])
    page = rng.choice([0, 16, 32, 64, 128])
    if kind == "norm":
        dtype = rng.choice(["f16", "bf16", "f32"])
        batch, backward = rng.randint(1, 16), rng.random() < 0.5
        tokens = _log_int(rng, 1, max(1, int((1.6e7 if dtype == "f32" else 3e7) / (batch * (heads + kv) * dim))))
        return _norm(None, dtype, batch, tokens, heads, kv, dim, rng.choice([0, dim, dim, dim // 2, dim // 4 * 3]), rng.choice(["half", "interleaved"]),
                     rng.choice([dtype, "f32"]), rng.random() < 0.3, rng.choice([0, 5000, 120000]), backward)
    if kind == "append":
        batch, tokens, longest = _log_int(rng, 1, 16), _log_int(rng, 1, 1000), _log_int(rng, 1, 500)
        layers = rng.randint(1, max(1, min(40, int(2e7 / (batch * tokens * kv * dim)))))
        return _append(None, dtype, form, layers, batch, tokens, kv, dim, rng.randint(0, longest), longest, page)
    if kind == "read":
        batch = _log_int(rng, 1, 24)
        longest = _log_int(rng, 1, max(16, min(20000, int(6e7 / (batch * kv * dim)))))
        layers = rng.randint(1, max(1, min(8, int(8e7 / (batch * longest * kv * dim)))))
        return _read(None, dtype, form, layers, batch, kv, dim, rng.randint(0, longest), longest, page)
    if kind == "attend":
        batch, tokens = _log_int(rng, 1, 32), 1 if rng.random() < 0.5 else _log_int(rng, 2, 48)
        longest = _log_int(rng, 1, max(16, min(65000, int(1.3e8 / (batch * kv * dim)), int(8e9 / (batch * tokens * heads * dim)))))
        return _attend(None, dtype, form, batch, tokens, heads, kv, dim, max(1, int(longest * rng.uniform(0.01, 1.0))), longest, page, rng.choice([0, 2, 3, 4]))
    words = _log_int(rng, 1000, 152000)
    return _sample(None, rng.choice(["f16", "bf16", "f32"]), _log_int(rng, 1, max(1, min(64, int(8e6 / words)))), words,
                   rng.choice(["none", "top_k", "top_p", "min_p", "all", "mixed"]), rng.choice([0.0, 9.0, 12.0, 15.0]))


def _lens(c):
    """Lengths of the contexts of a batch: evenly spread over their logarithm, or from none at all to the longest."""
    n, lo, hi = c["batch"], c["shortest"], c["longest"]
    if n == 1:
        return [hi]
    return [int(round(lo * (hi / lo) ** (i / (n - 1)))) if lo > 0 else hi * i // (n - 1) for i in range(n)]


def _parents(c):
    """A tree of the new tokens, the root first, parents before children, up to `branch` children to a node."""
    n, branch = c["tokens"], c["branch"]
    if branch == 0:
        return list(range(-1, n - 1))
    rng, parents, room, children = random.Random(n * 100 + branch), [-1], [0], [0] * n
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


def _pages(c):
    """Tokens to a page, and pages to a sequence; there is room for the new tokens behind the longest context."""
    need = max(1, c["longest"] + c["tokens"])
    return (need, 1) if c["page"] == 0 else (c["page"], -(-need // c["page"]))


def _held(c):
    """Bytes of one head of one token in the cache, its scale among them."""
    return (c["dim"] // 2 if c["form"] == "int4" else c["dim"]) + 4


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "norm":
        n = c["batch"] * c["tokens"]
        each = n * (c["heads"] + c["kv"])
        weights = (c["heads"] + c["kv"] if c["each"] else 2) * c["dim"] * (4 if c["weights"] == "f32" else 2)
        return {"bytes": (3 if c["backward"] else 2) * each * c["dim"] * es + (2 if c["backward"] else 1) * weights + 4 * n, "flops": (12 if c["backward"] else 7) * each * c["dim"]}
    if c["kind"] == "append":
        n = 2 * c["layers"] * c["batch"] * c["tokens"] * c["kv"]
        return {"bytes": n * (2 * c["dim"] * es + 2 * _held(c)), "flops": 4 * n * c["dim"]}
    if c["kind"] == "read":
        n = 2 * c["layers"] * c["kv"]
        return {"bytes": n * (sum(_lens(c)) * _held(c) + c["batch"] * c["longest"] * c["dim"] * es), "flops": n * sum(_lens(c)) * c["dim"]}
    if c["kind"] == "attend":
        seen = sum(len(r) for r in _ancestors(_parents(c)))
        b, t, lens = c["batch"], c["tokens"], sum(_lens(c))
        new = 2 * b * t * (c["kv"] + c["heads"]) * c["dim"]
        return {"bytes": 2 * lens * c["kv"] * _held(c) + new * es + 4 * b * t * c["heads"], "flops": 4 * c["dim"] * c["heads"] * (t * lens + b * seen)}
    return {"bytes": c["rows"] * c["words"] * es + 24 * c["rows"], "flops": 4 * c["rows"] * c["words"]}


# ---- inputs ---------------------------------------------------------------------------------------------------
def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    n = int(seed)
    for k in key:
        n = (n * 1000003 + int(k)) % (2 ** 61 - 1)
    g.manual_seed(n)
    return g


def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


_LEAST = 2.0 ** -100      # heads whose largest value is below this are held as if it were this


def _quantize(x, form):
    """Codes (uint8) and scales of heads x [..., dim], 32 bits.  The scales of int4 are pairs: scale, offset."""
    if form == "e4m3":      # the smallest power of two with which the largest value is at most 448
        m, e = torch.frexp(x.abs().amax(-1).clamp(min=_LEAST))
        scale = torch.ldexp(torch.ones_like(m), e - 9 + (m > 0.875).to(e.dtype))
        return (x / scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), scale
    if form == "int8":
        top = x.abs().amax(-1).clamp(min=_LEAST)
        code = torch.round(x * 127.0 / top[..., None])
        return code.to(torch.int8).view(torch.uint8), top / 127.0
    lo, hi = x.amin(-1), x.amax(-1)
    offset = (lo * 0.5 + hi * 0.5).to(torch.bfloat16).float()
    reach = torch.maximum(hi - offset, offset - lo)
    step = (reach.clamp(min=_LEAST) * 0.125).view(torch.int32)      # upwards to 16 bits
    step = ((step + 0xffff) & -0x10000).view(torch.float32)
    n = torch.floor((x - offset[..., None]) / step[..., None]).clamp(-8, 7).to(torch.int32)
    step = torch.where(reach > 0, step, 0.0)
    nibble = torch.where(n >= 0, n, 8 + (-1 - n)).to(torch.uint8)      # sign and magnitude
    return nibble[..., 0::2] | (nibble[..., 1::2] << 4), torch.stack([step, offset], dim=-1).to(torch.bfloat16)


def _values(codes, scales, form, dtype=torch.float32):
    """What codes and scales stand for."""
    if form == "e4m3":
        return codes.view(torch.float8_e4m3fn).to(dtype) * scales[..., None].to(dtype)
    if form == "int8":
        return codes.view(torch.int8).to(dtype) * scales[..., None].to(dtype)
    nibble = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    level = ((nibble & 7).to(dtype) + 0.5) * (1 - 2 * (nibble >> 3).to(dtype))
    return scales[..., 1:].to(dtype) + scales[..., :1].to(dtype) * level


def _pool(c, g, s, filled):
    """Pages with every sequence's own spread over them, and the table.  Channels differ in size, and those of the keys in their mean."""
    page, each = _pages(c)
    layers, n, kv, d, form = c.get("layers", 1), c["batch"] * each, c["kv"], c["dim"], c["form"]
    size = torch.exp(0.5 * _normal(g, kv, d))
    mean = _normal(g, kv, d)
    for name, middle in (("k", mean), ("v", 0.0 * mean)):
        s[name] = torch.zeros(layers, n, page, kv, d // 2 if form == "int4" else d, dtype=torch.uint8, device="cuda")
        s[name + "_scales"] = torch.zeros(layers, n, page, kv, *((2,) if form == "int4" else ()), dtype=torch.bfloat16 if form == "int4" else torch.float32, device="cuda")
        for l in range(layers if filled else 0):
            s[name][l], s[name + "_scales"][l] = _quantize(_normal(g, n, page, kv, d) * size + middle, form)
    s["size"], s["mean"] = size, mean
    order = torch.randperm(n, generator=g, device="cuda") if c["page"] else torch.arange(n, device="cuda")
    s["table"] = order.reshape(c["batch"], each).to(torch.int32)
    order = torch.randperm(c["batch"], generator=g, device="cuda")
    s["lens"] = _ints(_lens(c))[order]
    if own:
        import paper_2508_06041_amd as dp
        s["cache"] = dp.QuantizedCache(s["k"], s["v"], s["k_scales"], s["v_scales"], getattr(dp, "DPLLM_CACHE_" + form.upper()), s["table"])


def prepare(c, seed):
    s = {"case": c}
    g = _gen(seed, 1)
    dtype = _TYPES[c["dtype"]]
    if c["kind"] == "norm":
        b, t, d = c["batch"], c["tokens"], c["dim"]
        # as the projections leave them: queries, keys and values of a token side by side, heads of different sizes
        qkv = (_normal(g, b, t, c["heads"] + 2 * c["kv"], d) * torch.exp(_normal(g, c["heads"] + 2 * c["kv"], 1))).to(dtype)
        s["x"] = (qkv[:, :, :c["heads"]], qkv[:, :, c["heads"]:c["heads"] + c["kv"]])
        s["w"] = tuple((1.0 + 0.3 * _normal(g, *((n,) if c["each"] else ()), d)).to(_TYPES[c["weights"]]) for n in (c["heads"], c["kv"]))
        first = torch.randint(0, 1 + c["first"], (b, 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(t, device="cuda")).to(torch.int32)
        s["freqs"] = None
        if c["rotary"]:
            s["freqs"] = torch.tensor([500000.0 ** (-2.0 * i / c["rotary"]) for i in range(c["rotary"] // 2)], dtype=torch.float64, device="cuda")
        if c["backward"]:
            s["grads"] = tuple(_normal(g, b, t, n, d, dtype=dtype) for n in (c["heads"], c["kv"]))
        if own:
            import paper_2508_06041_amd as dp
            s["layout"] = getattr(dp, "DPLLM_ROPE_" + c["layout"].upper())
    elif c["kind"] == "append":
        _pool(c, g, s, False)
        shape = c["layers"], c["batch"], c["tokens"], c["kv"], c["dim"]
        s["k_new"], s["v_new"] = torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda")
        for l in range(c["layers"]):
            s["k_new"][l] = (_normal(g, *shape[1:]) * s["size"] + s["mean"]).to(dtype)
            s["v_new"][l] = (_normal(g, *shape[1:]) * s["size"]).to(dtype)
    elif c["kind"] == "read":
        _pool(c, g, s, True)
        s["first"] = torch.zeros(c["batch"], dtype=torch.int32, device="cuda")
    elif c["kind"] == "attend":
        b, t, d = c["batch"], c["tokens"], c["dim"]
        _pool(c, g, s, True)
        s["q"] = _normal(g, b, t, c["heads"], d, dtype=dtype)
        s["k_new"] = (_normal(g, b, t, c["kv"], d) * s["size"] + s["mean"]).to(dtype)
        s["v_new"] = (_normal(g, b, t, c["kv"], d) * s["size"]).to(dtype)
        rows = [sum(1 << j for j in r) for r in _ancestors(_parents(c))]
        s["mask"] = torch.tensor([r - (1 << 64) if r >= 1 << 63 else r for r in rows], dtype=torch.int64, device="cuda").reshape(1, t, 1)
    else:
        n, v = c["rows"], c["words"]
        x = 2.5 * _normal(g, n, v)
        at = torch.randint(0, v, (n, 12), generator=g, device="cuda")
        x.scatter_add_(1, at, c["boost"] + 1.5 * _normal(g, n, 12))
        s["logits"] = x.to(dtype)
        s["uniforms"] = torch.rand(n, generator=g, device="cuda")
        s["temperature"] = torch.rand(n, generator=g, device="cuda") * 0.7 + 0.6
        if c["filters"] == "mixed":
            s["temperature"][::5] = 0.0
        # in a mixed batch every second, third and fourth row has a filter
        has = {f: torch.tensor([c["filters"] in (f, "all") or (c["filters"] == "mixed" and i % every == every - 1) for i in range(n)], device="cuda")
               for f, every in (("top_k", 2), ("top_p", 3), ("min_p", 4))}
        s["top_k"] = torch.where(has["top_k"], torch.randint(1, 100, (n,), generator=g, device="cuda"), 0).to(torch.int32)
        s["top_p"] = torch.where(has["top_p"], 0.8 + 0.19 * torch.rand(n, generator=g, device="cuda"), 1.0)
        s["min_p"] = torch.where(has["min_p"], 0.01 + 0.1 * torch.rand(n, generator=g, device="cuda"), 0.0)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _run_own(s, c):
    import paper_2508_06041_amd as dp
    dtype = _TYPES[c["dtype"]]
    if c["kind"] == "norm":
        if c["backward"]:
            return dp.dpllm_norm_rope_backward(s["x"], s["grads"], s["w"], s["positions"], s["freqs"], eps=1e-6, layout=s["layout"])
        return dp.dpllm_norm_rope(s["x"], s["w"], s["positions"], s["freqs"], eps=1e-6, layout=s["layout"])
    if c["kind"] == "append":
        dp.dpllm_quantized_append(s["cache"], s["lens"], s["k_new"], s["v_new"])
        return dp.dpllm_quantized_read(s["cache"], s["lens"], c["tokens"], dtype=dtype, layers=c["layers"])
    if c["kind"] == "read":
        return dp.dpllm_quantized_read(s["cache"], s["first"], c["longest"], dtype=dtype, count=s["lens"], layers=c["layers"])
    if c["kind"] == "attend":
        lse = torch.empty(c["batch"], c["tokens"], c["heads"], dtype=torch.float32, device="cuda")
        out = dp.dpllm_quantized_attention(s["cache"], 0, s["lens"], s["q"], s["k_new"], s["v_new"], mask=s["mask"], lse=lse, max_len=c["longest"])
        return out, lse
    kept = torch.empty(c["rows"], dtype=torch.int32, device="cuda")
    return dp.dpllm_sample(s["logits"], s["uniforms"], s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], kept=kept), kept


def _run_plain(s, c):
    if c["kind"] == "norm":
        return (_plain_gradient if c["backward"] else _plain_norm)(s, c)
    return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "sample": _plain_sample}[c["kind"]](s, c)


def _sines(s):
    angle = s["positions"].double()[:, :, None, None] * s["freqs"]      # far positions: an angle of 32 bits is off by whole degrees
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turned(y, cos, sin, c):
    r = c["rotary"]
    if c["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., r:]], dim=-1)
    a, b = y[..., 0:r:2], y[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), y[..., r:]], dim=-1)


def _plain_norm(s, c):
    turn = _sines(s) if c["rotary"] else None

    def one(x, w):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + 1e-6) * w.float()
        return (_turned(y, *turn, c) if turn else y).to(x.dtype)
    return one(s["x"][0], s["w"][0]), one(s["x"][1], s["w"][1])


def _plain_gradient(s, c):
    turn = _sines(s) if c["rotary"] else None

    def one(x, w, g):
        y, h = x.float(), g.float()
        h = _turned(h, turn[0], -turn[1], c) if turn else h
        r = torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + 1e-6)
        n, d = y * r, h * w.float()
        over = (h * n).double()      # many thousand terms
        return (r * (d - n * (d * n).mean(dim=-1, keepdim=True))).to(x.dtype), over.sum(dim=(0, 1) if c["each"] else (0, 1, 2)).to(w.dtype)
    (q, wq), (k, wk) = one(s["x"][0], s["w"][0], s["grads"][0]), one(s["x"][1], s["w"][1], s["grads"][1])
    return (q, k), (wq, wk)


def _slots(s, first, n):
    """Page and place of tokens first ... + n - 1 of every sequence."""
    page, each = s["k"].shape[2], s["table"].shape[1]
    at = first.long()[:, None] + torch.arange(n, device="cuda")
    return s["table"].long().gather(1, (at // page).clamp(max=each - 1)), at % page


def _back(s, c, which, where, dtype):
    codes, scales = s[which][:, where[0], where[1]], s[which + "_scales"][:, where[0], where[1]]
    return _values(codes, scales, c["form"]).to(dtype)


def _plain_append(s, c):
    where = _slots(s, s["lens"], c["tokens"])
    dtype = _TYPES[c["dtype"]]
    s["k"][:, where[0], where[1]], s["k_scales"][:, where[0], where[1]] = _quantize(s["k_new"].float(), c["form"])
    s["v"][:, where[0], where[1]], s["v_scales"][:, where[0], where[1]] = _quantize(s["v_new"].float(), c["form"])
    return _back(s, c, "k", where, dtype), _back(s, c, "v", where, dtype)


def _plain_read(s, c):
    where = _slots(s, s["first"], c["longest"])
    there = (torch.arange(c["longest"], device="cuda") < s["lens"][:, None])[None, :, :, None, None]
    dtype = _TYPES[c["dtype"]]
    return torch.where(there, _back(s, c, "k", where, dtype), 0.0), torch.where(there, _back(s, c, "v", where, dtype), 0.0)


def _plain_attend(s, c):
    b, t, kv, d, n = c["batch"], c["tokens"], c["kv"], c["dim"], c["longest"]
    group = c["heads"] // kv
    where = _slots(s, torch.zeros_like(s["lens"]), n)
    old = torch.arange(n, device="cuda") < s["lens"][:, None]                               # [b][n]
    tree = ((s["mask"] >> torch.arange(t, device="cuda")) & 1).bool().expand(b, t, t)
    seen = torch.cat([old[:, None, :].expand(b, t, n), tree], dim=2)                        # [b][t][n + t]
    k = torch.cat([_back(s, c, "k", where, torch.float32)[0], s["k_new"].float()], dim=1)
    v = torch.cat([_back(s, c, "v", where, torch.float32)[0], s["v_new"].float()], dim=1)
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


def _plain_sample(s, c):
    # 64 bits throughout: the answers are whole numbers, and sums of many small probabilities decide them
    n, v = c["rows"], c["words"]
    best = s["temperature"] <= 0
    x, order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)         # equal ones by their numbers
    e = torch.exp((x.double() - x[:, :1].double()) / torch.where(best, 1.0, s["temperature"].double())[:, None])
    place = torch.arange(v, device="cuda")
    k = torch.where(s["top_k"] > 0, s["top_k"].long(), v)[:, None]
    keep = (place < k) & (e >= 2.0 ** -64)
    upto = torch.cumsum(torch.where(keep, e, 0.0), dim=1)
    p = s["top_p"].double()[:, None]
    keep &= (p >= 1) | (upto - e < p * upto[:, -1:]) | (place == 0)
    keep &= e >= s["min_p"].double()[:, None]
    keep &= ~best[:, None] | (place == 0)
    weight = torch.zeros(n, v, dtype=torch.float64, device="cuda").scatter_(1, order, torch.where(keep, e, 0.0))
    over = torch.cumsum(weight, dim=1)
    over = over > s["uniforms"].double()[:, None] * over[:, -1:]
    return over.to(torch.uint8).argmax(dim=1).to(torch.int32), keep.sum(dim=1).to(torch.int32)


# ---- the same from the definitions in 64 bits --------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] == "sample":
        return None      # whole numbers
    s = prepare(c, seed)
    if c["kind"] == "norm":
        xs = [x.double().requires_grad_() for x in s["x"]]
        ws = [w.double().requires_grad_() for w in s["w"]]
        r, outs = c["rotary"], []
        for x, w in zip(xs, ws):
            y = w * x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + 1e-6)
            if r:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[..., None, None] * s["freqs"])
                z = y[..., :r].reshape(*x.shape[:3], 2, r // 2).transpose(3, 4) if c["layout"] == "half" else y[..., :r].reshape(*x.shape[:3], r // 2, 2)
                z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
                y = torch.cat([(z.transpose(3, 4) if c["layout"] == "half" else z).reshape(*x.shape[:3], r), y[..., r:]], dim=-1)
            outs.append(y)
        if not c["backward"]:
            return tuple(y.detach() for y in outs)
        made = torch.autograd.grad(outs, xs + ws, [g.double() for g in s["grads"]])
        return tuple(made[:2]), tuple(made[2:])
    if c["kind"] == "append":
        return tuple(_exact_held(x, c["form"]) for x in (s["k_new"], s["v_new"]))
    lens, table = s["lens"].tolist(), s["table"].long()
    if c["kind"] == "read":
        outs = []
        for which in ("k", "v"):
            out = torch.zeros(c["layers"], c["batch"], c["longest"], c["kv"], c["dim"], dtype=torch.float64, device="cuda")
            for b in range(c["batch"]):
                pages = [s[w][:, table[b]].flatten(1, 2)[:, :lens[b]] for w in (which, which + "_scales")]
                out[:, b, :lens[b]] = _values(*pages, c["form"], torch.float64)
            outs.append(out)
        return tuple(outs)
    rows = _ancestors(_parents(c))
    group = c["heads"] // c["kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        sees = torch.zeros(c["tokens"], c["tokens"], dtype=torch.bool)
        for i, r in enumerate(rows):
            sees[i, r] = True
        sees = torch.cat([torch.ones(c["tokens"], lens[b], dtype=torch.bool), sees], dim=1).cuda()
        for h in range(c["kv"]):
            k, v = (torch.cat([_values(s[w][0, table[b], :, h].flatten(0, 1)[:lens[b]], s[w + "_scales"][0, table[b], :, h].flatten(0, 1)[:lens[b]], c["form"], torch.float64),
                               s[w + "_new"][b, :, h].double()]) for w in ("k", "v"))
            for j in range(h * group, (h + 1) * group):
                x = (s["q"][b, :, j].double() @ k.t().contiguous() / math.sqrt(c["dim"])).masked_fill(~sees, float("-inf"))
                out[b, :, j] = torch.softmax(x, dim=1) @ v
                lse[b, :, j] = torch.logsumexp(x, dim=1)
    return out, lse


def _exact_held(x, form):
    """What the cache is to hold of heads x, 64 bits; scales are held in 32 bits, those of int4 in 16."""
    x = x.double()
    size = x.abs().amax(dim=-1, keepdim=True).clamp(min=_LEAST)
    if form == "e4m3":
        scale = torch.exp2(torch.ceil(torch.log2(size / 448)))
        y = x / scale
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # four bits, from 2^-6 downwards whole 2^-9
        return torch.round(y / step) * step * scale
    if form == "int8":
        return torch.round(x * 127 / size) * (size / 127).float().double()
    lo, hi = x.amin(dim=-1, keepdim=True), x.amax(dim=-1, keepdim=True)
    offset = ((lo + hi) / 2).to(torch.bfloat16).double()
    reach = torch.maximum(hi - offset, offset - lo)
    unit = torch.exp2(torch.floor(torch.log2(reach.clamp(min=_LEAST) / 8)) - 7)
    scale = torch.ceil(reach.clamp(min=_LEAST) / 8 / unit) * unit
    n = torch.floor((x - offset) / scale).clamp(-8, 7)
    return torch.where(reach > 0, offset + scale * (n + 0.5), offset)
