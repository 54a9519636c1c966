"""Verification of drafted tokens against a loop in 64 bits; the answers are whole numbers and have to be equal."""
import math

import numpy as np
import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def softmax(x, t):
    x = np.where(np.isnan(x), -np.inf, x)
    if x.max() == -np.inf:
        return np.zeros_like(x)
    if x.max() == np.inf:
        w = (x == np.inf).astype(float)
    else:
        w = np.zeros_like(x)
        w[x > -np.inf] = np.exp((x[x > -np.inf] - x.max()) / t)
    return w / w.sum()


def plain(logits, tokens, parents, uniforms, temperature, draft):
    """One sequence, numpy in 64 bits: (path, words)."""
    n, v = logits.shape
    node, path, words = 0, [0], []
    while True:
        if not temperature > 0:
            x = np.where(np.isnan(logits[node]), -np.inf, logits[node])
            best = int(x.argmax()) if x.max() > -np.inf else -1
            stands = [c for c in range(node + 1, n) if parents[c] == node and best >= 0 and tokens[c] == best]
            answer = best
        else:
            r, q = softmax(logits[node], temperature), None if draft is None else softmax(draft[node], temperature)
            stands = []
            for c in range(node + 1, n):
                if parents[c] != node:
                    continue
                w = tokens[c]
                have, by = (r[w], 1.0 if q is None else q[w]) if 0 <= w < v else (0.0, 0.0)
                if uniforms[c] * by < have:
                    stands = [c]
                    break
                if q is None:
                    less = r.copy()
                    if 0 <= w < v:
                        less[w] = 0.0
                else:
                    less = np.maximum(r - q, 0.0)
                if less.sum() > 0:
                    r = less / less.sum()
            run = np.cumsum(r)
            over = np.flatnonzero(run > uniforms[0] * run[-1])
            answer = int(over[0]) if over.size else -1
        if not stands:
            return path, words + [answer]
        node = stands[0]
        path.append(node)
        words.append(int(tokens[node]))


def compare(logits, tokens, parents, uniforms, temperature, draft, siblings=None, **kw):
    b, n, _ = logits.shape
    count, path, words = dp.dpllm_verify(logits, tokens, uniforms, temperature, parents=parents, draft=draft, siblings=siblings, **kw)
    par = [list(range(-1, n - 1))] * b if parents is None else parents.tolist()
    lengths = []
    for i in range(b):
        want_path, want_words = plain(logits[i].double().cpu().numpy(), tokens[i].tolist(), par[i], uniforms[i].double().cpu().numpy(), temperature[i].item(),
                                      None if draft is None else draft[i].double().cpu().numpy())
        m = len(want_path)
        got = (count[i].item(), path[i].tolist(), words[i].tolist())
        assert got == (m, want_path + [-1] * (n - m), want_words + [-1] * (n - m)), (i, got, want_path, want_words)
        lengths.append(m)
    return lengths


def tree(n, branch, g):
    parents, room = [-1], [0] * branch
    for i in range(1, n):
        parents.append(room.pop(int(torch.randint(0, len(room), (1,), generator=g))))
        room += [i] * branch
    return parents


def inputs(dtype, b, n, v, branch, drafted, seed, noise=0.4, size=2.5, greedy=0):
    g = torch.Generator().manual_seed(seed)
    parents = tree(n, branch, g) if branch else list(range(-1, n - 1))
    target = torch.randn(b, n, v, generator=g) * size
    draft = target + noise * torch.randn(b, n, v, generator=g)
    temperature = torch.rand(b, generator=g) + 0.5
    if greedy:
        temperature[::greedy] = 0.0
    tokens = torch.zeros(b, n, dtype=torch.int32)
    target, draft = target.to(TYPES[dtype]), draft.to(TYPES[dtype])
    for i in range(n):
        mine = [c for c in range(n) if parents[c] == i]
        if mine and drafted:
            p = torch.softmax(draft[:, i].double() / temperature.clamp(min=0.05)[:, None].double(), 1)
            tokens[:, mine] = torch.multinomial(p, len(mine), replacement=True, generator=g).int()
        elif mine:
            tokens[:, mine] = draft[:, i].float().topk(min(len(mine), v), 1).indices.int().repeat(1, len(mine))[:, :len(mine)]
    uniforms = torch.rand(b, n, generator=g)
    siblings = max([1] + [parents.count(p) for p in range(n)])
    return dict(logits=target.cuda(), tokens=tokens.cuda(), parents=torch.tensor([parents] * b, dtype=torch.int32).cuda() if branch else None, uniforms=uniforms.cuda(),
                temperature=temperature.cuda(), draft=draft.cuda() if drafted else None, siblings=siblings)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("drafted", [False, True])
@pytest.mark.parametrize("b,n,v,branch", [(1, 1, 1, 0), (3, 2, 2, 0), (4, 6, 1000, 0), (2, 9, 4097, 0), (3, 13, 517, 3), (2, 33, 8200, 4), (2, 70, 131, 2), (1, 256, 64, 5),
                                          (2, 5, 50001, 2)])
def test_against_a_loop(dtype, drafted, b, n, v, branch):
    compare(**inputs(dtype, b, n, v, branch, drafted, seed=n * 7 + v))


@pytest.mark.parametrize("drafted", [False, True])
@pytest.mark.parametrize("noise", [0.0, 0.1, 1.0, 5.0])
def test_drafts_near_and_far(drafted, noise):
    """From drafts that are the target (all stand) to such that have little to do with it."""
    lengths = compare(**inputs("f32", 24, 8, 300, 0, drafted, seed=int(noise * 10), noise=noise))
    if drafted and noise == 0.0:
        assert lengths == [8] * 24
    if noise == 5.0:
        assert sum(lengths) < 24 * 4


@pytest.mark.parametrize("drafted", [False, True])
def test_the_best_token(drafted):
    """Temperature 0 takes the largest logit, the first of several; tokens of either kind in one batch."""
    x = inputs("bf16", 12, 10, 333, 3, drafted, seed=5, noise=0.02, size=4.0, greedy=2)
    x["logits"][0, :, 40] = x["logits"][0, :, 7] = 100.0      # ties: the lower word
    x["tokens"][0] = 7
    lengths = compare(**x)
    assert lengths[0] > 1
    x["tokens"][0] = 40
    assert compare(**x)[0] == 1
    x["temperature"][1], x["temperature"][3] = -1.0, math.nan
    compare(**x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("drafted", [False, True])
def test_masked_infinite_and_missing_logits(dtype, drafted):
    x = inputs(dtype, 10, 5, 900, 0, drafted, seed=11)
    for rows in (x["logits"], x["draft"]) if drafted else (x["logits"],):
        rows[0, :, ::2] = -math.inf
        rows[1, :, 5:] = -math.inf
        rows[2] = -math.inf                       # a row without a number: nothing stands, no token
        rows[3, :, 17] = math.inf                 # all of the probability
        rows[3, :, 19] = math.inf
        rows[4, :, ::3] = math.nan
        rows[5, 2:] = math.nan
        rows[6] = torch.finfo(rows.dtype).min     # the lowest value is a number as any other
        rows[7, :, :] = torch.finfo(rows.dtype).min
        rows[7, :, 3] = torch.finfo(rows.dtype).max
    x["tokens"][3] = 19
    x["tokens"][4] = 6
    x["tokens"][7] = 3
    compare(**x)
    x["temperature"][:] = 0.0
    compare(**x)
    x["temperature"][:] = 1e-30
    x["temperature"][::2] = 1e30
    compare(**x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("drafted", [False, True])
def test_signaling_nan(dtype, drafted):
    x = inputs(dtype, 6, 4, 700, 0, drafted, seed=12, greedy=3)
    for rows in (x["logits"], x["draft"]) if drafted else (x["logits"],):
        bits, nan = {2: (torch.int16, {"f16": 0x7c01, "bf16": 0x7f81}.get(dtype)), 4: (torch.int32, 0x7f800001)}[rows.element_size()]
        rows.view(bits)[:, :, 1::3] = nan
    x["tokens"][:2] = 3
    compare(**x)


@pytest.mark.parametrize("dtype,drafted", [("f32", False), ("f16", True), ("bf16", True)])
def test_many_long_rows(dtype, drafted):
    compare(**inputs(dtype, 32, 8, 70001, 0, drafted, seed=13, greedy=5))


@pytest.mark.parametrize("drafted", [False, True])
def test_an_infinite_temperature(drafted):
    """Every word that is not masked is as likely as any other."""
    x = inputs("f32", 5, 6, 700, 2, drafted, seed=20)
    x["logits"][:, :, 100:300] = -math.inf
    x["temperature"][:] = math.inf
    compare(**x)


def test_tokens_and_parents_of_nobody():
    x = inputs("f32", 6, 20, 100, 3, False, seed=12)
    x["tokens"][0] = 100
    x["tokens"][1] = -1
    x["tokens"][2] = 2 ** 31 - 1
    x["parents"][3, 4:] = -1
    x["parents"][4, 7] = 7
    x["parents"][4, 8] = 15
    x["parents"][5] = 2 ** 31 - 1
    compare(**x)
    x["temperature"][:] = 0.0
    compare(**x)


@pytest.mark.parametrize("drafted", [False, True])
def test_uniforms_at_the_ends(drafted):
    x = inputs("f32", 4, 4, 50, 0, drafted, seed=13)
    for rows in (x["logits"], x["draft"]) if drafted else (x["logits"],):
        rows[:, :, :3] = -math.inf                # so that the first word with a probability is not word 0
        rows[:, :, 47:] = -math.inf
    x["uniforms"][0] = 0.0
    x["uniforms"][1] = 1.0 - 2.0 ** -24
    x["uniforms"][2, 0], x["uniforms"][2, 1:] = 0.0, 1.0 - 2.0 ** -24
    compare(**x)


def test_siblings_that_share_a_word():
    """The same word twice: named, the second can not stand any more; drawn, each is asked by itself."""
    for drafted in (False, True):
        x = inputs("f32", 16, 9, 40, 8, drafted, seed=14, noise=1.0)
        x["parents"][:] = 0
        x["parents"][:, 0] = -1
        x["tokens"][:, 1:] = torch.tensor([3, 3, 5, 3, 5, 39, 0, 0], dtype=torch.int32, device="cuda")
        x["siblings"] = 8
        compare(**x)


def test_views_and_unaligned_rows():
    """Rows of an odd number of words, at odd addresses, every second row of a larger tensor, target and draft unlike."""
    for dtype in TYPES:
        x = inputs(dtype, 3, 6, 4099, 2, True, seed=15)
        big = torch.full((3, 13, 4111), math.nan, dtype=TYPES[dtype], device="cuda")
        big[:, 1::2, 5:4104] = x["logits"]
        flat = torch.full((3 * 6 * 4099 + 3,), math.nan, dtype=TYPES[dtype], device="cuda")
        flat[3:] = x["draft"].flatten()
        x["logits"], x["draft"] = big[:, 1::2, 5:4104], flat[3:].view(3, 6, 4099)
        compare(**x)


def test_chosen_tokens_follow_the_target():
    """The first token of 60000 sequences, and the second where there is one, against the target's probabilities: within five standard deviations."""
    b, v = 60000, 12
    g = torch.Generator().manual_seed(16)
    target, draft = torch.randn(1, 7, v, generator=g) * 1.5, torch.randn(1, 7, v, generator=g) * 1.5
    parents = torch.tensor([[-1, 0, 0, 0, 1, 1, 3]], dtype=torch.int32)
    temperature = torch.full((b,), 0.8)
    p, q = (torch.softmax(x[0].double() / 0.8, 1) for x in (target, draft))
    for drafted in (True, False):
        tokens = torch.zeros(b, 7, dtype=torch.int32)
        for c in range(1, 7):
            at = parents[0, c].item()
            tokens[:, c] = torch.multinomial(q[at].expand(b, v), 1, generator=g)[:, 0] if drafted else (3 * c) % v
        _, path, words = dp.dpllm_verify(target.expand(b, 7, v).contiguous().cuda(), tokens.cuda(), torch.rand(b, 7, generator=g).cuda(), temperature.cuda(),
                                         parents=parents.expand(b, 7).contiguous().cuda(), draft=draft.expand(b, 7, v).contiguous().cuda() if drafted else None, siblings=3)
        path, words = path.cpu(), words.cpu()
        for rows, dist in ((words[:, 0], p[0]), (words[path[:, 1] == 1][:, 1], p[1]), (words[path[:, 1] == 3][:, 1], p[3])):
            m = rows.numel()
            assert m > 200
            freq = torch.bincount(rows.long(), minlength=v).double() / m
            assert ((freq - dist).abs() <= 5 * (dist * (1 - dist) / m).sqrt() + 1e-9).all(), (freq, dist)


def test_a_graph_follows_its_inputs():
    x = inputs("bf16", 5, 7, 3000, 2, True, seed=17)
    y = inputs("bf16", 5, 7, 3000, 2, True, seed=18, greedy=2)
    y["parents"] = x["parents"]
    n = max(x["siblings"], y["siblings"])
    names = ("logits", "tokens", "uniforms", "temperature", "draft")
    held = {k: x[k].clone() for k in names}
    outs = [torch.zeros(5, dtype=torch.int32, device="cuda")] + [torch.zeros(5, 7, dtype=torch.int32, device="cuda") for _ in range(2)]
    space = torch.empty(dp.dpllm_verify_workspace_bytes(5, 7, 3000, dp.DPLLM_BF16, True, n), dtype=torch.uint8, device="cuda")

    def go():
        dp.dpllm_verify(parents=x["parents"], siblings=n, count=outs[0], path=outs[1], words=outs[2], workspace=space, **held)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for z in (y, x, y):
        for k in names:
            held[k].copy_(z[k])
        space.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = dp.dpllm_verify(parents=x["parents"], siblings=n, **{k: z[k] for k in names})
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals_of_the_binding():
    x = inputs("f16", 2, 4, 30, 0, True, seed=19)
    base = {k: x[k] for k in ("logits", "tokens", "uniforms", "temperature", "draft")}
    for change, word in [({"logits": x["logits"].double()}, "float16"), ({"logits": x["logits"].transpose(1, 2)}, "logits"), ({"draft": x["draft"].float()}, "draft"),
                         ({"tokens": x["tokens"].long()}, "tokens"), ({"uniforms": x["uniforms"].double()}, "uniforms"), ({"temperature": x["temperature"][:1]}, "temperature"),
                         ({"parents": x["tokens"][:, :2]}, "parents"), ({"siblings": 0}, "siblings"), ({"count": torch.zeros(3, dtype=torch.int32, device="cuda")}, "count"),
                         ({"workspace": torch.zeros(16, dtype=torch.uint8, device="cuda")}, "workspace")]:
        with pytest.raises(dp.DpllmError, match=word):
            dp.dpllm_verify(**dict(base, **change))
    none = dp.dpllm_verify(**{k: v[:0] for k, v in base.items()})
    assert [tuple(t.shape) for t in none] == [(0,), (0, 4), (0, 4)]
