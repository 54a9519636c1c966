"""CPU: what the calls of a step over a quantised cache refuse, before anything is launched, and the text they give."""
import ctypes as C
import math

import pytest

from paper_2508_06041_amd import binding as b
from test_token_refusals import SOME, refused, views

lib = b.lib


def cache(**change):
    c = dict(k=SOME, v=SOME, k_scales=SOME, v_scales=SOME, layer_stride=1 << 20, page_stride=16 * 512, token_stride=512, head_stride=128, scale_layer_stride=1 << 12,
             scale_page_stride=64, scale_token_stride=4, scale_head_stride=1, table=SOME, table_stride=4, format=b.DPLLM_CACHE_INT8, layers=2, pages=8, page=16,
             pages_per_seq=4, heads=4, head_dim=128)
    c.update(change)
    return b._QuantizedCache(*[c[name] for name, _ in b._QuantizedCache._fields_])


def pointers(*p):
    return (C.c_void_p * len(p))(*p)


def longs(*v):
    return (C.c_int64 * len(v))(*v)


NORM = dict(x=views(2), out=views(2), heads=(C.c_int * 2)(4, 2), weights=pointers(SOME, SOME), strides=longs(0, 128), weight_dtype=0, eps=1e-6, tensors=2, batch=2, tokens=3,
            head_dim=128, dtype=0, rotary_dim=128, layout=0, freqs=SOME, scale=1.0, positions=SOME, stride=3, stream=None)
BACK = dict(x=views(2), grads=views(2), out=views(2), heads=(C.c_int * 2)(4, 2), weights=pointers(SOME, SOME), grad_weights=pointers(SOME, SOME), strides=longs(0, 128),
            weight_dtype=0, eps=1e-6, tensors=2, batch=2, tokens=3, head_dim=128, dtype=0, rotary_dim=128, layout=0, freqs=SOME, scale=1.0, positions=SOME, stride=3, ws=SOME,
            ws_bytes=1 << 30, stream=None)
BOTH = [
    ({"x": None}, -1, "NULL"), ({"out": None}, -1, "NULL"), ({"heads": None}, -1, "NULL"), ({"strides": None}, -1, "NULL"), ({"freqs": None}, -1, "NULL"), ({"positions": None}, -1, "NULL"),
    ({"tensors": 0}, -2, "tensors"), ({"tensors": 5}, -2, "tensors"), ({"dtype": 3}, -1, "dtype"), ({"dtype": -1}, -1, "dtype"), ({"weight_dtype": 3}, -1, "weight_dtype"),
    ({"layout": 2}, -1, "layout"), ({"eps": -1e-6}, -1, "eps"), ({"eps": math.nan}, -1, "eps"), ({"eps": math.inf}, -1, "eps"), ({"batch": -1}, -2, "sequences"),
    ({"tokens": -1}, -2, "sequences"), ({"batch": 1 << 20, "tokens": 1 << 20}, -2, "sequences"), ({"head_dim": 0}, -2, "head_dim"), ({"head_dim": 2048}, -2, "head_dim"),
    ({"rotary_dim": -2}, -2, "rotary_dim"), ({"rotary_dim": 31}, -2, "rotary_dim"), ({"rotary_dim": 130}, -2, "rotary_dim"), ({"heads": (C.c_int * 2)(4, 0)}, -2, "heads"),
    ({"heads": (C.c_int * 2)(1 << 30, 1 << 30)}, -2, "heads"), ({"x": views(2, data=SOME + 1)}, -1, "aligned"), ({"out": views(2, data=SOME + 2), "dtype": 2}, -1, "aligned"),
    ({"x": views(2, data=None)}, -1, "NULL"), ({"out": views(2, data=None)}, -1, "NULL"), ({"weights": pointers(SOME, SOME + 1)}, -1, "weight 1"),
    ({"weights": pointers(SOME + 2, None), "weight_dtype": 2}, -1, "weight 0"),
]


@pytest.mark.parametrize("change,code,word", BOTH)
@pytest.mark.parametrize("call", ["dpllm_norm_rope", "dpllm_norm_rope_backward"])
def test_norms(call, change, code, word):
    refused(getattr(lib, call)(*dict(NORM if call == "dpllm_norm_rope" else BACK, **change).values()), code, word)


@pytest.mark.parametrize("change,code,word", [
    ({"grads": None}, -1, "NULL"), ({"grads": views(2, data=None)}, -1, "NULL"), ({"grads": views(2, data=SOME + 1)}, -1, "aligned"), ({"weights": pointers(SOME, None)}, -1, "weight 1"),
    ({"weights": None}, -1, "weight 0"), ({"grad_weights": pointers(SOME + 1, SOME)}, -1, "weight 0"), ({"ws": None}, -4, "workspace"), ({"ws": SOME + 8}, -4, "workspace"),
    ({"ws_bytes": 64}, -4, "workspace"),
])
def test_gradients_of_norms(change, code, word):
    refused(lib.dpllm_norm_rope_backward(*dict(BACK, **change).values()), code, word)


def test_norms_of_nothing():
    nothing = views(2, data=None)
    assert lib.dpllm_norm_rope(*dict(NORM, tokens=0).values()) == 0
    assert lib.dpllm_norm_rope(*dict(NORM, batch=0, x=nothing, out=nothing, freqs=None, positions=None).values()) == 0
    assert lib.dpllm_norm_rope_backward(*dict(BACK, batch=0, x=nothing, grads=nothing, out=nothing, grad_weights=None, ws=None, ws_bytes=0).values()) == 0


def need(heads, strides, batch, tokens, head_dim):
    n = C.c_size_t(77)
    rc = lib.dpllm_norm_rope_backward_workspace_bytes((C.c_int * len(heads))(*heads), longs(*strides), len(heads), batch, tokens, head_dim, C.byref(n))
    return rc if rc else n.value


def test_workspaces_of_gradients():
    assert need((4, 2), (0, 0), 0, 5, 128) == 0
    assert 0 < need((4, 2), (0, 0), 1, 1, 128) <= need((4, 2), (0, 0), 4, 2049, 128) <= 4 << 20
    assert need((4, 2), (128, 128), 4, 2049, 128) > 0
    for args, code in (((), -2), (((4, 0), (0, 0), 1, 1, 128), -2), (((4,), (0,), 1, 1, 2048), -2), (((4,), (0,), -1, 1, 128), -2), (((1 << 30,), (0,), 1, 1, 128), -2)):
        assert need(*(args or ((), (), 1, 1, 128))) == code
    assert lib.dpllm_norm_rope_backward_workspace_bytes((C.c_int * 1)(4), longs(0), 1, 1, 1, 128, None) == -1


APPEND = dict(cache=cache(), first=0, layers=2, batch=2, nodes=3, lens=SOME, dtype=0, k=views(1), k_layer=1 << 16, v=views(1), v_layer=1 << 16, path=SOME, stride=3, count=SOME, stream=None)
READ = dict(cache=cache(), first=0, layers=2, batch=2, tokens=3, firsts=SOME, count=SOME, dtype=0, k=views(1), k_layer=1 << 16, v=views(1), v_layer=1 << 16, stream=None)
BAD_CACHES = [({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"k_scales": None}, -1, "NULL"), ({"v_scales": None}, -1, "NULL"), ({"format": 0}, -1, "format"), ({"format": 4}, -1, "format"),
              ({"layers": 0}, -2, "cache"), ({"pages": 0}, -2, "cache"), ({"page": 0}, -2, "cache"), ({"pages_per_seq": 0}, -2, "cache"), ({"heads": 0}, -2, "cache"),
              ({"head_dim": 0}, -2, "cache"), ({"head_dim": 2048}, -2, "cache"), ({"format": 3, "head_dim": 127}, -2, "odd"), ({"k_scales": SOME + 2}, -1, "aligned"),
              ({"v_scales": SOME + 1}, -1, "aligned"), ({"table": None}, -2, "table"), ({"table": None, "pages_per_seq": 1, "pages": 1}, -2, "table"),
              ({"table_stride": -1}, -2, "table_stride")]


@pytest.mark.parametrize("change,code,word", BAD_CACHES)
@pytest.mark.parametrize("call,args", [("dpllm_quantized_append", APPEND), ("dpllm_quantized_read", READ)])
def test_a_bad_cache(call, args, change, code, word):
    refused(getattr(lib, call)(*dict(args, cache=cache(**change)).values()), code, word)


@pytest.mark.parametrize("change,code,word", [
    ({"cache": None}, -1, "NULL"), ({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"k": views(1, data=None)}, -1, "NULL"), ({"v": views(1, data=SOME + 1)}, -1, "aligned"),
    ({"k": views(1, data=SOME + 2), "dtype": 2}, -1, "aligned"), ({"dtype": 3}, -1, "dtype"), ({"dtype": -1}, -1, "dtype"), ({"first": -1}, -3, "layers"), ({"first": 1}, -3, "layers"),
    ({"layers": -1}, -3, "layers"), ({"first": 2 ** 31 - 1}, -3, "layers"), ({"batch": -1}, -2, "sequences"), ({"batch": 65536}, -2, "sequences"), ({"tokens": -1}, -2, "sequences"),
    ({"tokens": 1 << 25}, -2, "sequences"),
])
@pytest.mark.parametrize("call,args", [("dpllm_quantized_append", APPEND), ("dpllm_quantized_read", READ)])
def test_append_and_read(call, args, change, code, word):
    if "tokens" in change and "nodes" in args:
        change = {"nodes": change["tokens"]}
    refused(getattr(lib, call)(*dict(args, **change).values()), code, word)


def test_append_without_lengths():
    refused(lib.dpllm_quantized_append(*dict(APPEND, lens=None).values()), -1, "NULL")


def test_append_and_read_of_nothing():
    for change in ({"batch": 0}, {"nodes": 0}, {"layers": 0, "first": 2}):
        assert lib.dpllm_quantized_append(*dict(APPEND, **change).values()) == 0
    for change in ({"batch": 0}, {"tokens": 0}, {"layers": 0, "first": 2}):
        assert lib.dpllm_quantized_read(*dict(READ, **change).values()) == 0


ATTEND = dict(cache=None, layer=0, batch=2, nodes=3, heads=8, dtype=0, lens=SOME, max_len=10000, q=views(1), k=views(1), v=views(1), mask=SOME, mask_stride=3, scale=0.1, out=views(1),
              lse=SOME, ws=SOME, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code,word", BAD_CACHES)
def test_attention_over_a_bad_cache(change, code, word):
    refused(lib.dpllm_quantized_attention(*dict(ATTEND, cache=cache(**change)).values()), code, word)


@pytest.mark.parametrize("change,code,word", [
    ({"cache": None}, -1, "NULL"), ({"dtype": 2}, -1, "float16"), ({"cache": cache(head_dim=80)}, -2, "head_dim"), ({"layer": -1}, -3, "layer"), ({"layer": 2}, -3, "layer"),
    ({"batch": -1}, -2, "sequences"), ({"batch": 65537}, -2, "sequences"), ({"nodes": -1}, -2, "nodes"), ({"nodes": 257}, -2, "nodes"), ({"heads": 6}, -2, "heads"), ({"heads": 0}, -2, "heads"),
    ({"heads": 2048}, -2, "heads"), ({"max_len": -1}, -2, "max_len"), ({"scale": math.inf}, -1, "scale"), ({"scale": math.nan}, -1, "scale"), ({"lens": None}, -1, "NULL"), ({"q": None}, -1, "NULL"),
    ({"q": views(1, data=None)}, -1, "NULL"), ({"out": None}, -1, "NULL"), ({"k": None}, -1, "NULL"), ({"v": None}, -1, "NULL"), ({"k": views(1, data=None)}, -1, "NULL"),
    ({"q": views(1, data=SOME + 2)}, -1, "aligned"), ({"out": views(1, strides=(1024, 512, 129))}, -1, "aligned"), ({"k": views(1, strides=(1024, 510, 128))}, -1, "aligned"),
    ({"cache": cache(k=SOME + 8)}, -1, "aligned"), ({"cache": cache(page_stride=16 * 512 + 4)}, -1, "aligned"), ({"cache": cache(page=1 << 30, pages_per_seq=8)}, -2, "tokens"),
    ({"ws": None}, -4, "workspace"), ({"ws_bytes": 100}, -4, "workspace"), ({"ws": SOME + 8}, -4, "workspace"),
])
def test_attention(change, code, word):
    # a cache that is long enough for the work to be split, so that a workspace is needed
    refused(lib.dpllm_quantized_attention(*dict(dict(ATTEND, cache=cache(page=4096)), **change).values()), code, word)


def test_attention_of_nothing():
    for change in ({"batch": 0}, {"nodes": 0}):
        assert lib.dpllm_quantized_attention(*dict(ATTEND, cache=cache(), **change).values()) == 0


def attention_need(*args):
    n = C.c_size_t(77)
    rc = lib.dpllm_quantized_attention_workspace_bytes(*args, C.byref(n))
    return rc if rc else n.value


def test_workspaces_of_attention():
    assert attention_need(0, 1, 32, 8, 128, 1000) == 0 and attention_need(1, 0, 32, 8, 128, 1000) == 0
    assert attention_need(1, 1, 32, 8, 128, 100000) > 0
    for args in ((1, 1, 32, 7, 128, 1), (1, 1, 32, 8, 80, 1), (1, 257, 32, 8, 128, 1), (65537, 1, 32, 8, 128, 1), (1, 1, 32, 8, 128, -1), (1, 1, 0, 1, 128, 1)):
        assert attention_need(*args) == -2
    assert lib.dpllm_quantized_attention_workspace_bytes(1, 1, 32, 8, 128, 1, None) == -1


SAMPLE = dict(rows=2, vocabulary=100, dtype=0, logits=SOME, stride=100, uniforms=SOME, temperature=SOME, top_k=SOME, top_p=SOME, min_p=SOME, words=SOME, kept=SOME, ws=SOME, ws_bytes=1 << 30,
              stream=None)


@pytest.mark.parametrize("change,code,word", [
    ({"rows": -1}, -2, "rows"), ({"rows": 65537}, -2, "rows"), ({"vocabulary": 0}, -2, "vocabulary"), ({"vocabulary": -5}, -2, "vocabulary"), ({"vocabulary": (1 << 22) + 1}, -2, "vocabulary"),
    ({"rows": 65536, "vocabulary": 1 << 22}, -2, "too many"), ({"dtype": 3}, -1, "dtype"), ({"dtype": -1}, -1, "dtype"), ({"logits": None}, -1, "NULL"), ({"uniforms": None}, -1, "NULL"),
    ({"temperature": None}, -1, "NULL"), ({"words": None}, -1, "NULL"), ({"logits": SOME + 1}, -1, "aligned"), ({"logits": SOME + 2, "dtype": 2}, -1, "aligned"), ({"ws": None}, -4, "workspace"),
    ({"ws_bytes": 64}, -4, "workspace"), ({"ws": SOME + 8}, -4, "workspace"),
])
def test_sample(change, code, word):
    refused(lib.dpllm_sample(*dict(SAMPLE, **change).values()), code, word)


def test_sample_of_nothing():
    assert lib.dpllm_sample(*dict(SAMPLE, rows=0, logits=None, words=None, ws=None, ws_bytes=0).values()) == 0
    n = C.c_size_t(77)
    assert lib.dpllm_sample_workspace_bytes(0, 5, 0, C.byref(n)) == 0 and n.value == 0
    assert lib.dpllm_sample_workspace_bytes(1, 5, 0, None) == -1
    assert lib.dpllm_sample_workspace_bytes(1, 0, 0, C.byref(n)) == -2 and lib.dpllm_sample_workspace_bytes(1, 5, 7, C.byref(n)) == -1
