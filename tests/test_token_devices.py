"""CPU: tensors that are not where a call around the linears runs, and workspaces that are not what it writes to, are refused before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2508_06041_amd as dp
from paper_2508_06041_amd import binding

calls = binding._calls


class OnDevice(torch.Tensor):
    """A tensor that says it is on a device; what is made of it is on the same one."""
    index = 0

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.index


class OnAnother(OnDevice):
    index = 1


def on(t, cls=OnDevice):
    return t.as_subclass(cls)


@pytest.fixture
def made(monkeypatch):
    """The names of the library functions that were called, either way; device 0 is the current one."""
    got = []
    vp = C.c_void_p
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=None, device=None: on(empty(*shape, dtype=dtype)))
    stubs, addresses = [], []

    def need(name):
        def f(*a):
            if name.endswith("bytes"):
                a[-1][0] = 64
            else:
                got.append(name)
            return 0
        return f
    for name in ("dpllm_rope", "dpllm_tree_attention_workspace_bytes", "dpllm_tree_attention", "dpllm_verify_workspace_bytes", "dpllm_verify", "dpllm_cache_append"):
        stubs.append(C.CFUNCTYPE(C.c_int, *getattr(binding.lib, name).argtypes)(need(name)))
        addresses.append(C.cast(stubs[-1], vp).value)
        monkeypatch.setattr(binding.lib, name, stubs[-1])
    dtypes = (torch.float16, torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.float64)
    calls.bind(1, 1, lambda: 0, lambda device: 0)
    calls.bind_tokens(tuple(addresses), dtypes, torch.empty_like)
    yield got
    monkeypatch.undo()
    lib = binding.lib
    calls.bind(C.cast(lib.dpllm_gemv, vp).value, C.cast(lib.dpllm_estimate, vp).value, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
    calls.bind_tokens(tuple(C.cast(f, vp).value for f in (lib.dpllm_rope, lib.dpllm_tree_attention_workspace_bytes, lib.dpllm_tree_attention,
                                                          lib.dpllm_verify_workspace_bytes, lib.dpllm_verify, lib.dpllm_cache_append)), dtypes, torch.empty_like)


def rope_args():
    x = on(torch.zeros(2, 3, 4, 64, dtype=torch.float16))
    return dict(x=x, positions=on(torch.zeros(2, 3, dtype=torch.int32)), freqs=on(torch.zeros(32, dtype=torch.float64)), out=on(torch.zeros_like(x)))


def cache(cls=OnDevice):
    return dp.Cache(*(on(torch.zeros(2, 8, 16, 2, 64, dtype=torch.float16), cls) for _ in range(2)), on(torch.zeros(2, 4, dtype=torch.int32), cls))


def attention_args():
    def new(heads):
        return on(torch.zeros(2, 3, heads, 64, dtype=torch.float16))
    return dict(cache=cache(), layer=0, lens=on(torch.zeros(2, dtype=torch.int32)), q=new(4), k_new=new(2), v_new=new(2), mask=on(torch.zeros(2, 3, 1, dtype=torch.int64)),
                out=new(4), lse=on(torch.zeros(2, 3, 4)), workspace=on(torch.zeros(64, dtype=torch.uint8)))


def verify_args():
    def ints(*shape):
        return on(torch.zeros(*shape, dtype=torch.int32))
    return dict(logits=on(torch.zeros(2, 3, 10)), tokens=ints(2, 3), uniforms=on(torch.zeros(2, 3)), temperature=on(torch.zeros(2)), parents=ints(2, 3),
                draft=on(torch.zeros(2, 3, 10)), siblings=2, count=ints(2), path=ints(2, 3), words=ints(2, 3), workspace=on(torch.zeros(64, dtype=torch.uint8)))


def append_args():
    def new():
        return on(torch.zeros(2, 2, 3, 2, 64, dtype=torch.float16))
    return dict(cache=cache(), lens=on(torch.zeros(2, dtype=torch.int32)), k_new=new(), v_new=new(), path=on(torch.zeros(2, 3, dtype=torch.int32)),
                count=on(torch.zeros(2, dtype=torch.int32)))


CALLS = {"dpllm_rope": rope_args, "dpllm_tree_attention": attention_args, "dpllm_verify": verify_args, "dpllm_cache_append": append_args}
TENSORS = [(f, name) for f, args in CALLS.items() for name, value in args().items() if isinstance(value, torch.Tensor)]


def ways(f, args):
    """The call as it is, and without a workspace and results of the caller's, which goes the native way."""
    yield args
    if "workspace" in args:
        yield {k: v for k, v in args.items() if k not in ("workspace", "out", "lse", "count" if f == "dpllm_verify" else "", "words", "path" if f == "dpllm_verify" else "")}


@pytest.mark.parametrize("f", CALLS)
def test_ordinary_calls_are_made(made, f):
    for n, args in enumerate(ways(f, CALLS[f]())):
        getattr(dp, f)(**args)
        assert made == [f] * (n + 1)


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


@pytest.mark.parametrize("f", ["dpllm_tree_attention", "dpllm_cache_append"])
def test_a_cache_that_is_elsewhere(made, f):
    for args in ways(f, CALLS[f]()):
        with pytest.raises(dp.DpllmError, match="device"):
            getattr(dp, f)(**dict(args, cache=cache(OnAnother)))
    assert made == []


def test_the_tensors_of_a_cache_share_a_device():
    k, v, table = torch.zeros(2, 8, 16, 2, 64, dtype=torch.float16), torch.zeros(2, 8, 16, 2, 64, dtype=torch.float16), torch.zeros(2, 4, dtype=torch.int32)
    for a in ((on(k), on(v, OnAnother), None), (on(k), on(v), on(table, OnAnother)), (on(k), v, None), (on(k), on(v), table)):
        with pytest.raises(dp.DpllmError, match="device"):
            dp.Cache(*a)


@pytest.mark.parametrize("f", ["dpllm_tree_attention", "dpllm_verify"])
def test_a_workspace_with_gaps(made, f):
    with pytest.raises(dp.DpllmError, match="workspace"):
        getattr(dp, f)(**dict(CALLS[f](), workspace=on(torch.zeros(256, dtype=torch.uint8)[::4])))
    assert made == []


@pytest.mark.parametrize("f", CALLS)
def test_the_interpreter_is_free_while_the_library_works(made, f):
    """The function that is called says whether its thread holds the interpreter's lock: 0 is no, and OK.  (ctypes gives it back on the long way.)"""
    holds = C.cast(C.pythonapi.PyGILState_Check, C.c_void_p).value
    nothing = C.CFUNCTYPE(C.c_int, *[C.c_int] * 6, C.POINTER(C.c_size_t))(lambda *a: 0)      # no workspace is needed
    none = C.cast(nothing, C.c_void_p).value
    calls.bind_tokens((holds, none, holds, none, holds, holds), (torch.float16, torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.float64),
                      torch.empty_like)
    for args in ways(f, CALLS[f]()):
        getattr(dp, f)(**args)
    # only what brings a workspace was called the long way: natively the lock was free
    assert made == ([f] if "workspace" in CALLS[f]() else [])


def heads_first(x):
    """The same tensor, laid out head after head."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def test_results_are_laid_out_alike_either_way(made):
    """Results that a call makes follow the order of the inputs' dimensions, natively and the long way."""
    a = rope_args()
    x = heads_first(a["x"])
    got = [dp.dpllm_rope(y, a["positions"], a["freqs"]) for y in ((x,), [x])]      # (a list is out of the ordinary)
    assert made == ["dpllm_rope"] * 2 and [g[0].stride() for g in got] == [x.stride()] * 2
    a = attention_args()
    del a["out"]
    a["q"] = q = heads_first(a["q"])
    got = [dp.dpllm_tree_attention(**dict(a, workspace=w)) for w in (None, a["workspace"])]
    assert [g.stride() for g in got] == [q.stride()] * 2


def test_a_gradient_that_results_in_out_would_not_have(made):
    a = rope_args()
    for change in ({"x": a["x"].requires_grad_()}, {"out": a["out"].requires_grad_()}):
        with pytest.raises(dp.DpllmError, match="gradient"):
            dp.dpllm_rope(**dict(a, **change))
    assert made == []
    with torch.no_grad():
        dp.dpllm_rope(**a)
    assert made == ["dpllm_rope"]
