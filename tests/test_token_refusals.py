"""CPU: what the calls around the linears refuse, before anything is launched, and the text they give."""
import ctypes as C
import math

import pytest

from paper_2508_06041_amd import binding as b

lib = b.lib
SOME = 4096   # an address nothing reads: every call here is refused


def views(n, data=SOME, strides=(1024, 512, 128)):
    return (b._Heads * n)(*[b._Heads(data, *strides) for _ in range(n)])


def cache(**change):
    c = dict(k=SOME, v=SOME, layer_stride=1 << 20, page_stride=16 * 512, token_stride=512, head_stride=128, table=SOME, table_stride=4, dtype=b.DPLLM_F16,
             layers=2, pages=8, page=16, pages_per_seq=4, heads=4, head_dim=128)
    c.update(change)
    return b._Cache(*[c[name] for name, _ in b._Cache._fields_])


def refused(rc, code, word):
    text = lib.dpllm_call_error().decode()
    assert rc == code and word in text, (rc, text)


ROPE = dict(x=views(2), out=views(2), heads=(C.c_int * 2)(4, 2), tensors=2, batch=2, tokens=3, head_dim=128, dtype=0, rotary_dim=128, layout=0,
            freqs=SOME, scale=1.0, positions=SOME, stride=3, inverse=0, stream=None)


@pytest.mark.parametrize("change,code,word", [
    ({"x": None}, -1, "NULL"), ({"out": None}, -1, "NULL"), ({"heads": None}, -1, "NULL"), ({"freqs": None}, -1, "NULL"), ({"positions": None}, -1, "NULL"),
    ({"tensors": 0}, -2, "tensors"), ({"tensors": 5}, -2, "tensors"), ({"dtype": 3}, -1, "dtype"), ({"dtype": -1}, -1, "dtype"), ({"layout": 2}, -1, "layout"),
    ({"batch": -1}, -2, "sequences"), ({"tokens": -1}, -2, "sequences"), ({"batch": 1 << 20, "tokens": 1 << 20}, -2, "sequences"),
    ({"head_dim": 1}, -2, "rotary_dim"), ({"head_dim": 2048}, -2, "rotary_dim"), ({"rotary_dim": 0}, -2, "rotary_dim"), ({"rotary_dim": 31}, -2, "rotary_dim"),
    ({"rotary_dim": 130}, -2, "rotary_dim"), ({"heads": (C.c_int * 2)(4, 0)}, -2, "heads"), ({"heads": (C.c_int * 2)(1 << 30, 1 << 30)}, -2, "heads"),
    ({"x": views(2, data=SOME + 1)}, -1, "aligned"), ({"out": views(2, data=SOME + 2), "dtype": 2}, -1, "aligned"), ({"x": views(2, data=None)}, -1, "NULL"),
])
def test_rope(change, code, word):
    refused(lib.dpllm_rope(*dict(ROPE, **change).values()), code, word)


def test_rope_of_nothing():
    assert lib.dpllm_rope(*dict(ROPE, tokens=0).values()) == 0
    assert lib.dpllm_rope(*dict(ROPE, batch=0, x=views(2, data=None), out=views(2, data=None)).values()) == 0


@pytest.mark.parametrize("args,code,word", [
    ((0, 1e4, 0, 1, 0, 1, 2), -2, "rotary_dim"), ((7, 1e4, 0, 1, 0, 1, 2), -2, "rotary_dim"), ((2048, 1e4, 0, 1, 0, 1, 2), -2, "rotary_dim"),
    ((8, 1.0, 0, 1, 0, 1, 2), -1, "base"), ((8, math.nan, 0, 1, 0, 1, 2), -1, "base"), ((8, math.inf, 0, 1, 0, 1, 2), -1, "base"),
    ((8, 1e4, 5, 1, 0, 1, 2), -1, "scaling"), ((8, 1e4, -1, 1, 0, 1, 2), -1, "scaling"), ((8, 1e4, 1, 0.5, 0, 1, 2), -1, "factor"),
    ((8, 1e4, 1, math.nan, 0, 1, 2), -1, "factor"), ((2, 1e4, 2, 2, 0, 1, 2), -2, "NTK"), ((8, 1e4, 3, 2, 0, 1, 2), -1, "trained"),
    ((8, 1e4, 4, 2, 4096, 2, 2), -1, "trained"), ((8, 1e4, 4, 2, 4096, 0, 2), -1, "trained"), ((8, 1e4, 3, 2, math.inf, 1, 2), -1, "trained"),
])
def test_frequencies(args, code, word):
    f, s = (C.c_double * 2048)(), C.c_float()
    refused(lib.dpllm_rope_frequencies(*args, f, C.byref(s)), code, word)
    assert lib.dpllm_rope_frequencies(8, 1e4, 0, 1, 0, 1, 2, None, C.byref(s)) == -1


@pytest.mark.parametrize("rotary,base,scaling,factor,trained,low,high", [
    (2, 10000.0, 0, 1.0, 0, 1, 2), (128, 10000.0, 0, 1.0, 0, 1, 2), (96, 10000.0, 1, 4.0, 0, 1, 2), (64, 10000.0, 2, 8.0, 0, 1, 2),
    (128, 1e6, 3, 16.0, 8192, 1, 32), (64, 1e4, 3, 1.0, 2048, 1, 32), (128, 5e5, 4, 8.0, 8192, 1, 4), (4, 1e4, 3, 2.0, 16, 1, 32), (4, 1e4, 4, 2.0, 16, 1, 32),
])
def test_frequencies_follow_their_formulas(rotary, base, scaling, factor, trained, low, high):
    n = rotary // 2
    f, s = (C.c_double * n)(), C.c_float()
    assert lib.dpllm_rope_frequencies(rotary, base, scaling, factor, trained, low, high, f, C.byref(s)) == 0
    plain = [base ** (-2 * i / rotary) for i in range(n)]
    want = {0: plain, 1: [v / factor for v in plain]}.get(scaling)
    if scaling == 2:
        want = [(base * factor ** (rotary / (rotary - 2))) ** (-2 * i / rotary) for i in range(n)]
    if scaling == 3:
        def pair(turns):
            return rotary * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        a, z = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotary - 1)
        z = z if z > a else a + 0.001
        ramp = [min(max((i - a) / (z - a), 0), 1) for i in range(n)]
        want = [v * (1 - r) + v / factor * r for v, r in zip(plain, ramp)]
    if scaling == 4:
        ramp = [min(max((trained * v / (2 * math.pi) - low) / (high - low), 0), 1) for v in plain]
        want = [v * r + v / factor * (1 - r) for v, r in zip(plain, ramp)]
    assert list(f) == pytest.approx(want, rel=1e-13)
    assert s.value == pytest.approx(0.1 * math.log(factor) + 1 if scaling == 3 else 1.0, rel=2.0 ** -24)


APPEND = dict(cache=cache(), first=0, layers=2, batch=2, nodes=3, lens=SOME, k=views(1), k_layer=1 << 16, v=views(1), v_layer=1 << 16, path=SOME, stride=3,
              count=SOME, stream=None)
BAD_CACHES = [({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"dtype": 9}, -1, "dtype"), ({"layers": 0}, -2, "cache"), ({"pages": 0}, -2, "cache"),
              ({"page": 0}, -2, "cache"), ({"pages_per_seq": 0}, -2, "cache"), ({"heads": 0}, -2, "cache"), ({"head_dim": 0}, -2, "cache"),
              ({"head_dim": 2048}, -2, "cache"), ({"k": SOME + 1}, -1, "aligned"), ({"table": None}, -2, "table"),
              ({"table": None, "pages_per_seq": 1, "pages": 1}, -2, "table"), ({"table_stride": -1}, -2, "table_stride")]


@pytest.mark.parametrize("change,code,word", BAD_CACHES)
def test_append_of_a_bad_cache(change, code, word):
    refused(lib.dpllm_cache_append(*dict(APPEND, cache=cache(**change)).values()), code, word)


@pytest.mark.parametrize("change,code,word", [
    ({"cache": None}, -1, "NULL"), ({"lens": None}, -1, "NULL"), ({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"k": views(1, data=None)}, -1, "NULL"),
    ({"v": views(1, data=SOME + 1)}, -1, "aligned"), ({"first": -1}, -3, "layers"), ({"first": 1}, -3, "layers"), ({"layers": -1}, -3, "layers"),
    ({"first": 2 ** 31 - 1}, -3, "layers"), ({"batch": -1}, -2, "sequences"), ({"nodes": -1}, -2, "sequences"), ({"nodes": 1 << 30}, -2, "nodes"),
])
def test_append(change, code, word):
    refused(lib.dpllm_cache_append(*dict(APPEND, **change).values()), code, word)


def test_append_of_nothing():
    for change in ({"batch": 0}, {"nodes": 0}, {"layers": 0, "first": 2}):
        assert lib.dpllm_cache_append(*dict(APPEND, **change).values()) == 0


ATTEND = dict(cache=cache(), layer=0, batch=2, nodes=3, heads=8, lens=SOME, max_len=64, q=views(1), k=views(1), v=views(1), mask=SOME, mask_stride=3, scale=0.1,
              out=views(1), lse=SOME, ws=SOME, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code,word", BAD_CACHES)
def test_attention_over_a_bad_cache(change, code, word):
    refused(lib.dpllm_tree_attention(*dict(ATTEND, cache=cache(**change)).values()), code, word)


@pytest.mark.parametrize("change,code,word", [
    ({"cache": None}, -1, "NULL"), ({"cache": cache(dtype=2)}, -1, "float16"), ({"cache": cache(head_dim=80)}, -2, "head_dim"), ({"layer": -1}, -3, "layer"),
    ({"layer": 2}, -3, "layer"), ({"batch": -1}, -2, "sequences"), ({"batch": 65537}, -2, "sequences"), ({"nodes": -1}, -2, "nodes"), ({"nodes": 257}, -2, "nodes"),
    ({"heads": 6}, -2, "heads"), ({"heads": 0}, -2, "heads"), ({"heads": 2048}, -2, "heads"), ({"max_len": -1}, -2, "max_len"), ({"scale": math.inf}, -1, "scale"),
    ({"scale": math.nan}, -1, "scale"), ({"lens": None}, -1, "NULL"), ({"q": None}, -1, "NULL"), ({"q": views(1, data=None)}, -1, "NULL"), ({"out": None}, -1, "NULL"),
    ({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"k": views(1, data=None)}, -1, "NULL"), ({"q": views(1, data=SOME + 2)}, -1, "aligned"),
    ({"out": views(1, strides=(1024, 512, 129))}, -1, "aligned"), ({"k": views(1, strides=(1024, 510, 128))}, -1, "aligned"),
    ({"cache": cache(k=SOME + 8)}, -1, "aligned"), ({"cache": cache(page_stride=16 * 512 + 4)}, -1, "aligned"),
    ({"cache": cache(page=1 << 30, pages_per_seq=8)}, -2, "tokens"), ({"ws": None}, -4, "workspace"), ({"ws_bytes": 100}, -4, "workspace"), ({"ws": SOME + 8}, -4, "workspace"),
])
def test_attention(change, code, word):
    # a cache that is long enough for the work to be split, so that a workspace is needed
    refused(lib.dpllm_tree_attention(*dict(ATTEND, cache=change.get("cache", cache(page=1024)), max_len=change.get("max_len", 10000),
                                           **{k: v for k, v in change.items() if k not in ("cache", "max_len")}).values()), code, word)


def test_workspace_of_the_attention():
    n = C.c_size_t(1)
    f = lib.dpllm_tree_attention_workspace_bytes
    assert f(0, 4, 8, 2, 128, 1000, C.byref(n)) == 0 and n.value == 0
    assert f(1, 4, 8, 2, 128, 100000, C.byref(n)) == 0 and n.value > 0
    refused(f(1, 4, 8, 2, 128, 1000, None), -1, "NULL")
    refused(f(1, 4, 8, 3, 128, 1000, C.byref(n)), -2, "heads")
    refused(f(1, 4, 8, 2, 100, 1000, C.byref(n)), -2, "head_dim")
    refused(f(1, 4, 8, 2, 128, -1, C.byref(n)), -2, "max_len")


VERIFY = dict(batch=2, nodes=4, vocabulary=1000, dtype=1, logits=SOME, logits_batch=4000, logits_node=1000, draft=SOME, draft_batch=4000, draft_node=1000,
              tokens=SOME, parents=SOME, uniforms=SOME, temperature=SOME, siblings=2, count=SOME, path=SOME, words=SOME, ws=SOME, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("change,code,word", [
    ({"batch": -1}, -2, "sequences"), ({"batch": 70000}, -2, "sequences"), ({"nodes": 0}, -2, "nodes"), ({"nodes": 257}, -2, "nodes"), ({"vocabulary": 0}, -2, "vocabulary"),
    ({"vocabulary": 1 << 25}, -2, "vocabulary"), ({"dtype": 3}, -1, "dtype"), ({"siblings": 0}, -2, "siblings"), ({"siblings": 257}, -2, "siblings"),
    ({"batch": 65536, "nodes": 256}, -2, "too many"), ({"logits": None}, -1, "NULL"), ({"tokens": None}, -1, "NULL"), ({"uniforms": None}, -1, "NULL"),
    ({"temperature": None}, -1, "NULL"), ({"count": None}, -1, "NULL"), ({"path": None}, -1, "NULL"), ({"words": None}, -1, "NULL"),
    ({"logits": SOME + 1}, -1, "aligned"), ({"draft": SOME + 2, "dtype": 2}, -1, "aligned"), ({"ws": None}, -4, "workspace"), ({"ws": SOME + 8}, -4, "workspace"),
    ({"ws_bytes": 16}, -4, "workspace"),
])
def test_verify(change, code, word):
    refused(lib.dpllm_verify(*dict(VERIFY, **change).values()), code, word)


def test_verify_of_nothing_and_its_workspace():
    assert lib.dpllm_verify(*dict(VERIFY, batch=0).values()) == 0
    n, f = C.c_size_t(0), lib.dpllm_verify_workspace_bytes
    assert f(2, 4, 1000, 0, 1, 2, C.byref(n)) == 0 and n.value >= 2 * 4 * (2 * 16 + 2 * 8)
    small = n.value
    assert f(2, 4, 1000, 0, 0, 0, C.byref(n)) == 0 and 2 * 4 * 16 <= n.value < small
    refused(f(2, 4, 1000, 0, 1, 2, None), -1, "NULL")
    refused(f(2, 4, 0, 0, 1, 2, C.byref(n)), -2, "vocabulary")
