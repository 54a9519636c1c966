"""CPU: tensors that are not where a call of a step over a quantised cache runs, and workspaces that are not what it writes to, are refused before anything is launched; both ways of a call
pass on the same."""
import ctypes as C

import pytest
import torch

import paper_2508_06041_amd as dp
from paper_2508_06041_amd import binding
from test_token_devices import OnAnother, OnDevice, calls, heads_first, on

NATIVE = ("dpllm_norm_rope", "dpllm_norm_rope_backward_workspace_bytes", "dpllm_norm_rope_backward", "dpllm_quantized_append", "dpllm_quantized_read", "dpllm_quantized_attention_workspace_bytes", "dpllm_quantized_attention", "dpllm_sample_workspace_bytes", "dpllm_sample")
DTYPES = (torch.float16, torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.float64)
KINDS = {"e4m3": dp.DPLLM_CACHE_E4M3, "int8": dp.DPLLM_CACHE_INT8, "int4": dp.DPLLM_CACHE_INT4}


def tokens():
    lib = binding.lib
    return tuple(C.cast(f, C.c_void_p).value for f in (lib.dpllm_rope, lib.dpllm_tree_attention_workspace_bytes, lib.dpllm_tree_attention, lib.dpllm_verify_workspace_bytes, lib.dpllm_verify,
                                                       lib.dpllm_cache_append))


def plain(v):
    """An argument of a C call as numbers that can be compared; of an array its first element."""
    if isinstance(v, C.Structure):
        return tuple(plain(getattr(v, n)) for n, _ in v._fields_)
    if isinstance(v, C._Pointer):
        return plain(v[0]) if v else None
    return v


@pytest.fixture
def made(monkeypatch):
    """The library functions that were called and with what, either way; device 0 is the current one."""
    got = []
    vp = C.c_void_p
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=None, device=None: on(empty(*shape, dtype=dtype)))
    stubs = {}

    def need(name):
        def f(*a):
            if name.endswith("bytes"):
                a[-1][0] = 64
            else:
                got.append((name, [plain(v) for v in a]))
            return 0
        return f
    for name in NATIVE:
        stubs[name] = C.CFUNCTYPE(C.c_int, *getattr(binding.lib, name).argtypes)(need(name))
        monkeypatch.setattr(binding.lib, name, stubs[name])
    calls.bind(1, 1, lambda: 0, lambda device: 0)
    calls.bind_tokens(tokens(), DTYPES, torch.empty_like)
    calls.bind_step(tuple(C.cast(stubs[n], vp).value for n in NATIVE))
    yield got
    monkeypatch.undo()
    lib = binding.lib
    calls.bind(C.cast(lib.dpllm_gemv, vp).value, C.cast(lib.dpllm_estimate, vp).value, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
    calls.bind_tokens(tokens(), DTYPES, torch.empty_like)
    calls.bind_step(tuple(C.cast(getattr(lib, n), vp).value for n in NATIVE))


def names(made):
    return [n for n, _ in made]


def zeros(*shape, dtype=torch.float16):
    return on(torch.zeros(*shape, dtype=dtype))


def norm_args():
    return dict(x=zeros(2, 3, 4, 64), weights=zeros(64, dtype=torch.float32), positions=zeros(2, 3, dtype=torch.int32), freqs=zeros(32, dtype=torch.float64), out=zeros(2, 3, 4, 64))


def back_args():
    return dict(x=zeros(2, 3, 4, 64), grads=zeros(2, 3, 4, 64), weights=zeros(4, 64, dtype=torch.float32), positions=zeros(3, dtype=torch.int32), freqs=zeros(32, dtype=torch.float64),
                out=zeros(2, 3, 4, 64), workspace=zeros(64, dtype=torch.uint8))


def cache(kind="int8", cls=OnDevice, **other):
    pair = kind == "int4"
    t = dict(k=torch.zeros(2, 8, 16, 2, 32 if pair else 64, dtype=torch.uint8), v=torch.zeros(2, 8, 16, 2, 32 if pair else 64, dtype=torch.uint8))
    for n in ("k_scales", "v_scales"):
        t[n] = torch.zeros(2, 8, 16, 2, 2, dtype=torch.bfloat16) if pair else torch.zeros(2, 8, 16, 2)
    t["table"] = torch.zeros(2, 4, dtype=torch.int32)
    t = {n: other[n](v) if n in other else on(v, cls) for n, v in t.items()}
    return dp.QuantizedCache(t["k"], t["v"], t["k_scales"], t["v_scales"], KINDS[kind], t["table"])


def append_args():
    return dict(cache=cache(), lens=zeros(2, dtype=torch.int32), k_new=zeros(2, 2, 3, 2, 64), v_new=zeros(2, 2, 3, 2, 64), path=zeros(2, 3, dtype=torch.int32), count=zeros(2, dtype=torch.int32))


def read_args():
    return dict(cache=cache("int4"), first=zeros(2, dtype=torch.int32), tokens=5, dtype=torch.float16, count=zeros(2, dtype=torch.int32), layer=1, out=(zeros(2, 5, 2, 64), zeros(2, 5, 2, 64)))


def attention_args():
    return dict(cache=cache("e4m3"), layer=0, lens=zeros(2, dtype=torch.int32), q=zeros(2, 3, 4, 64), k_new=zeros(2, 3, 2, 64), v_new=zeros(2, 3, 2, 64),
                mask=zeros(2, 3, 1, dtype=torch.int64), out=zeros(2, 3, 4, 64), lse=zeros(2, 3, 4, dtype=torch.float32), workspace=zeros(64, dtype=torch.uint8))


def sample_args():
    def floats():
        return zeros(2, dtype=torch.float32)
    return dict(logits=zeros(2, 10), uniforms=floats(), temperature=floats(), top_k=zeros(2, dtype=torch.int32), top_p=floats(), min_p=floats(), words=zeros(2, dtype=torch.int32),
                kept=zeros(2, dtype=torch.int32), workspace=zeros(64, dtype=torch.uint8))


CALLS = {"dpllm_norm_rope": norm_args, "dpllm_norm_rope_backward": back_args, "dpllm_quantized_append": append_args, "dpllm_quantized_read": read_args,
         "dpllm_quantized_attention": attention_args, "dpllm_sample": sample_args}
TENSORS = [(f, name) for f, args in CALLS.items() for name, value in args().items() if isinstance(value, torch.Tensor)]
OWN = {"dpllm_norm_rope": ("out",), "dpllm_quantized_read": ("out",), "dpllm_quantized_attention": ("workspace", "out", "lse"), "dpllm_sample": ("workspace", "words", "kept"),
       "dpllm_norm_rope_backward": ("workspace", "out")}


def ways(f, args):
    """The call as it is, and without a workspace and results of the caller's."""
    yield args
    yield {k: v for k, v in args.items() if k not in OWN.get(f, ())}


@pytest.mark.parametrize("f", CALLS)
def test_ordinary_calls_are_made(made, f):
    for n, args in enumerate(ways(f, CALLS[f]())):
        getattr(dp, f)(**args)
        assert names(made) == [f] * (n + 1)


@pytest.mark.parametrize("f,name", TENSORS)
@pytest.mark.parametrize("where", ["host", "another device"])
def test_a_tensor_that_is_elsewhere(made, f, name, where):
    def move(t):
        return t.as_subclass(torch.Tensor) if where == "host" else on(t.as_subclass(torch.Tensor), OnAnother)
    for args in ways(f, CALLS[f]()):
        if name in args:
            with pytest.raises(dp.DpllmError, match="device"):
                getattr(dp, f)(**dict(args, **{name: move(args[name])}))
    assert made == []


@pytest.mark.parametrize("which", [0, 1])
def test_results_of_a_read_that_are_elsewhere(made, which):
    a = read_args()
    out = list(a["out"])
    out[which] = on(out[which].as_subclass(torch.Tensor), OnAnother)
    with pytest.raises(dp.DpllmError, match="device"):
        dp.dpllm_quantized_read(**dict(a, out=tuple(out)))
    assert made == []


@pytest.mark.parametrize("f", ["dpllm_quantized_append", "dpllm_quantized_read", "dpllm_quantized_attention"])
def test_a_cache_that_is_elsewhere(made, f):
    for args in ways(f, CALLS[f]()):
        with pytest.raises(dp.DpllmError, match="device"):
            getattr(dp, f)(**dict(args, cache=cache("e4m3", OnAnother)))
    assert made == []


@pytest.mark.parametrize("name", ["k", "v", "k_scales", "v_scales", "table"])
@pytest.mark.parametrize("kind", KINDS)
def test_the_tensors_of_a_cache_share_a_device(kind, name):
    cache(kind)
    for move in (lambda t: t, lambda t: on(t, OnAnother)):
        with pytest.raises(dp.DpllmError, match="device"):
            cache(kind, **{name: move})


@pytest.mark.parametrize("f", ["dpllm_norm_rope_backward", "dpllm_quantized_attention", "dpllm_sample"])
def test_a_workspace_with_gaps(made, f):
    with pytest.raises(dp.DpllmError, match="workspace"):
        getattr(dp, f)(**dict(CALLS[f](), workspace=on(torch.zeros(256, dtype=torch.uint8)[::4])))
    assert made == []


@pytest.mark.parametrize("f", [f for f in CALLS if f in NATIVE])
def test_the_interpreter_is_free_while_the_library_works(made, f):
    """The function that is called says whether its thread holds the interpreter's lock: 0 is no, and OK."""
    holds = C.cast(C.pythonapi.PyGILState_Check, C.c_void_p).value
    nothing = C.CFUNCTYPE(C.c_int, *[C.c_int] * 6, C.POINTER(C.c_size_t))(lambda *a: 0)      # no workspace is needed
    small = C.CFUNCTYPE(C.c_int, *[C.c_int] * 3, C.POINTER(C.c_size_t))(lambda *a: 0)
    norms = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, *[C.c_int] * 4, C.POINTER(C.c_size_t))(lambda *a: 0)
    none = [C.cast(p, C.c_void_p).value for p in (nothing, small, norms)]
    calls.bind_step((holds, none[2], holds, holds, holds, none[0], holds, none[1], holds))
    args = list(ways(f, CALLS[f]()))[1]      # (without results of the caller's, which goes the native way)
    if f == "dpllm_sample":
        args["logits"] = zeros(2, 10)
    getattr(dp, f)(**args)
    assert made == []


def same(f, args, change):
    """The arguments that the library gets natively and the long way; `change` makes the call out of the ordinary and nothing else."""
    getattr(dp, f)(**args)
    getattr(dp, f)(**dict(args, **change))


def test_both_ways_pass_on_the_same(made):
    a = norm_args()
    xs, outs = (a["x"], zeros(2, 3, 2, 64)), (a["out"], zeros(2, 3, 2, 64))
    for weights in (None, (zeros(64), None), (None, zeros(2, 64)), (zeros(4, 64)[:, :], zeros(64))):
        for positions in (a["positions"], zeros(3, dtype=torch.int32)):
            same("dpllm_norm_rope", dict(x=xs, weights=weights, positions=positions, freqs=a["freqs"], out=outs, eps=1e-5, scale=0.5, layout=1), {"x": list(xs)})
    same("dpllm_norm_rope", dict(x=xs[0], weights=a["weights"], out=outs[0]), {"out": [outs[0]]})
    a = back_args()
    del a["workspace"], a["out"]
    xs, outs = (a["x"], zeros(2, 3, 2, 64)), (zeros(2, 3, 4, 64), zeros(2, 3, 2, 64))
    for weights, wanted in (((a["weights"], zeros(64, dtype=torch.float32)), None), ((a["weights"], None), [False, True]), (None, None)):
        args = dict(a, x=xs, grads=(a["grads"], zeros(2, 3, 2, 64)), weights=weights, wanted=wanted, out=outs, layout=1, scale=2.0)
        got = [dp.dpllm_norm_rope_backward(**dict(args, **change)) for change in ({}, {"workspace": zeros(64, dtype=torch.uint8)})]
        for o, w in got:
            assert o[0] is outs[0] and o[1] is outs[1]
            assert [None if t is None else t.shape for t in w] == [None if t is None or (wanted and not wanted[i]) else t.shape for i, t in enumerate(weights or (None, None))]
    a = append_args()
    calls_made = len(made)
    same("dpllm_quantized_append", dict(a, layer=0), {"count": on(torch.zeros(2, 2, dtype=torch.int32)[:, 0].contiguous())})
    assert len(made) == calls_made + 2
    a = attention_args()
    for change in ({}, {"k_new": None, "v_new": None}, {"mask": None}, {"scale": 2.0}, {"max_len": 17}, {"mask": zeros(1, 3, 1, dtype=torch.int64)}):
        args = dict(a, **change)
        del args["workspace"]
        same("dpllm_quantized_attention", args, {"workspace": a["workspace"]})
    a = sample_args()
    for change in ({}, {"top_k": None}, {"top_p": None, "min_p": None}, {"kept": None}):
        args = dict(a, **change)
        del args["workspace"]
        same("dpllm_sample", args, {"workspace": a["workspace"]})
    native, long = made[::2], made[1::2]
    kept = {"dpllm_quantized_attention": (-3,), "dpllm_sample": (-3,), "dpllm_norm_rope_backward": (-3, -2, 5)}      # (the workspace, its bytes and new gradients are others)
    assert len(native) == len(long) > 10
    for (f, x), (g, y) in zip(native, long):
        assert f == g
        if f in kept:
            for i in kept[f]:
                del x[i], y[i]
        if f == "dpllm_quantized_append":
            del x[-2], y[-2]      # count, which is a copy
        assert x == y, f


def test_a_read_passes_on_the_same(made):
    a = read_args()
    del a["out"]
    for layers in (None, 1):
        for change in ({}, {"first": None}, {"count": None}, {"first": None, "count": None}, {"dtype": torch.float32}):
            args = dict(a, layers=layers, **change)
            got = dp.dpllm_quantized_read(**args)
            again = dp.dpllm_quantized_read(**dict(args, out=got))
            assert [t.shape for t in got] == [t.shape for t in again] and got[0].dtype == args["dtype"] and got[0].dim() == (4 if layers is None else 5)
            assert made[-1] == made[-2]


def test_results_are_laid_out_alike_either_way(made):
    """Results that a call makes follow the order of the inputs' dimensions, natively and the long way."""
    a = norm_args()
    x = heads_first(a["x"])
    got = [dp.dpllm_norm_rope(y, a["weights"], a["positions"], a["freqs"]) for y in ((x,), [x])]      # (a list is out of the ordinary)
    assert names(made) == ["dpllm_norm_rope"] * 2 and [g[0].stride() for g in got] == [x.stride()] * 2
    a = attention_args()
    del a["out"]
    a["q"] = q = heads_first(a["q"])
    got = [dp.dpllm_quantized_attention(**dict(a, workspace=w)) for w in (None, a["workspace"])]
    assert [g.stride() for g in got] == [q.stride()] * 2


def test_a_gradient_that_results_in_out_would_not_have(made):
    a = norm_args()
    for change in ({"x": zeros(2, 3, 4, 64).requires_grad_()}, {"weights": zeros(64, dtype=torch.float32).requires_grad_()}, {"out": zeros(2, 3, 4, 64).requires_grad_()}):
        with pytest.raises(dp.DpllmError, match="gradient"):
            dp.dpllm_norm_rope(**dict(a, **change))
    assert made == []
    with torch.no_grad():
        dp.dpllm_norm_rope(**a)
    assert names(made) == ["dpllm_norm_rope"]


def test_what_records_nothing_goes_the_native_way(made, monkeypatch):
    """Weights and inputs that require a gradient, where none is recorded; and the gradient itself, whose inputs do."""
    def never(*a, **k):
        raise AssertionError("the long way")
    monkeypatch.setattr(binding, "_norm_weights", never)
    a = norm_args()
    graded = zeros(64, dtype=torch.float32).requires_grad_()
    with torch.no_grad():
        dp.dpllm_norm_rope(a["x"], graded, a["positions"], a["freqs"])
    b = back_args()
    del b["workspace"]
    dp.dpllm_norm_rope_backward(**dict(b, x=b["x"].requires_grad_(), weights=b["weights"].requires_grad_()))
    assert names(made) == ["dpllm_norm_rope", "dpllm_norm_rope_backward"]
    assert dp.dpllm_norm_rope(a["x"], graded, a["positions"], a["freqs"]).requires_grad


BAD = [
    ("dpllm_norm_rope", {"weights": (zeros(64), zeros(64))}, "weight"), ("dpllm_norm_rope", {"weights": zeros(63, dtype=torch.float32)}, "weight"), ("dpllm_norm_rope", {"weights": zeros(3, 64)}, "weight"),
    ("dpllm_norm_rope", {"positions": None}, "positions"), ("dpllm_norm_rope", {"positions": zeros(2, 4, dtype=torch.int32)}, "positions"), ("dpllm_norm_rope", {"x": zeros(3, 4, 64)}, "out"),
    ("dpllm_norm_rope", {"freqs": zeros(32, dtype=torch.float32)}, "freqs"), ("dpllm_norm_rope", {"out": zeros(2, 3, 5, 64)}, "out"), ("dpllm_norm_rope", {"x": zeros(2, 3, 4, 64, dtype=torch.int32)}, "float16"),
    ("dpllm_norm_rope_backward", {"grads": zeros(2, 3, 4, 64, dtype=torch.bfloat16)}, "grads"), ("dpllm_norm_rope_backward", {"out": zeros(2, 3, 4, 32)}, "out"),
    ("dpllm_quantized_append", {"k_new": zeros(2, 2, 3, 2, 32), "v_new": zeros(2, 2, 3, 2, 32)}, "head_dim"), ("dpllm_quantized_append", {"v_new": zeros(2, 2, 3, 2, 64, dtype=torch.bfloat16)}, "one type"),
    ("dpllm_quantized_append", {"lens": zeros(3, dtype=torch.int32)}, "lens"), ("dpllm_quantized_append", {"path": zeros(2, 4, dtype=torch.int32)}, "path"),
    ("dpllm_quantized_read", {"dtype": torch.int32, "out": None}, "dtype"), ("dpllm_quantized_read", {"first": zeros(3, dtype=torch.int32), "count": None, "out": None}, "sequences"),
    ("dpllm_quantized_read", {"count": zeros(1, dtype=torch.int32)}, "count"), ("dpllm_quantized_read", {"out": (zeros(2, 5, 2, 64), zeros(2, 4, 2, 64))}, "out"),
    ("dpllm_quantized_attention", {"q": zeros(2, 3, 4, 32)}, "head_dim"), ("dpllm_quantized_attention", {"q": zeros(2, 3, 4, 64, dtype=torch.float32)}, "k_new"),
    ("dpllm_quantized_attention", {"v_new": None}, "together"), ("dpllm_quantized_attention", {"k_new": zeros(2, 3, 4, 64)}, "k_new"),
    ("dpllm_quantized_attention", {"mask": zeros(2, 3, 2, dtype=torch.int64)}, "mask"), ("dpllm_quantized_attention", {"lse": zeros(2, 3, 5, dtype=torch.float32)}, "lse"),
    ("dpllm_quantized_attention", {"q": zeros(3, 3, 4, 64)}, "sequences"), ("dpllm_sample", {"logits": zeros(2, 3, 4)}, "rows"), ("dpllm_sample", {"uniforms": zeros(3, dtype=torch.float32)}, "uniforms"),
    ("dpllm_sample", {"top_p": zeros(2, dtype=torch.float64)}, "top_p"), ("dpllm_sample", {"top_k": zeros(2, dtype=torch.int64)}, "top_k"), ("dpllm_sample", {"words": zeros(3, dtype=torch.int32)}, "words"),
]


@pytest.mark.parametrize("f,change,word", BAD)
def test_shapes_and_types_that_do_not_fit(made, f, change, word):
    for args in ways(f, CALLS[f]()):
        if all(k in args for k in change):
            with pytest.raises(dp.DpllmError, match=word):
                getattr(dp, f)(**dict(args, **change))
    assert made == []
