"""ctypes binding with the same names as include/dpllm.h.  Argument marshalling only.

Tensors are torch tensors used purely as device memory: the binding passes data_ptr() and the
current HIP stream to the C functions.  Functions raise DpllmError on a negative return code.
"""
import ctypes as C
import os

import torch
from torch.autograd import forward_ad

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libdpllm.so")

DPLLM_OK, DPLLM_EINVAL, DPLLM_ESHAPE, DPLLM_ERANGE, DPLLM_ESTATE, DPLLM_EHIP = 0, -1, -2, -3, -4, -5
DPLLM_SEL_NONE, DPLLM_SEL_PROJ, DPLLM_SEL_LINREG = 0, 1, 2
DPLLM_MAX_BATCH = 8
DPLLM_MAX_PAIRS = 8
DPLLM_MAX_TARGETS = 8
DPLLM_STEP_SELECT, DPLLM_STEP_GEMV = 1, 2
DPLLM_F16, DPLLM_BF16, DPLLM_F32 = 0, 1, 2
DPLLM_MAX_NODES = 256
DPLLM_ROPE_PLAIN, DPLLM_ROPE_LINEAR, DPLLM_ROPE_NTK, DPLLM_ROPE_YARN, DPLLM_ROPE_BANDS = 0, 1, 2, 3, 4
DPLLM_ROPE_HALF, DPLLM_ROPE_INTERLEAVED = 0, 1
DPLLM_CACHE_E4M3, DPLLM_CACHE_INT8, DPLLM_CACHE_INT4 = 1, 2, 3

SYMBOLS = ["dpllm_model_create", "dpllm_model_destroy", "dpllm_last_error", "dpllm_linear_device_bytes",
           "dpllm_workspace_bytes", "dpllm_set_workspace",
           "dpllm_load_linear", "dpllm_set_selector", "dpllm_set_threshold", "dpllm_set_active_pair",
           "dpllm_set_target_entry", "dpllm_set_target", "dpllm_set_selector_input",
           "dpllm_estimate", "dpllm_estimate_noalloc", "dpllm_gemv", "dpllm_decode_step", "dpllm_decode_step_parts", "dpllm_debug_unpack", "dpllm_debug_locate",
           "dpllm_debug_set_polls", "dpllm_debug_set_one_launch", "dpllm_debug_step_launches", "dpllm_debug_copy", "dpllm_debug_read",
           "dpllm_call_error", "dpllm_rope_frequencies", "dpllm_rope",
           "dpllm_tree_attention_workspace_bytes", "dpllm_tree_attention", "dpllm_verify_workspace_bytes",
           "dpllm_verify", "dpllm_cache_append",
           "dpllm_norm_rope", "dpllm_norm_rope_backward_workspace_bytes", "dpllm_norm_rope_backward", "dpllm_quantized_append", "dpllm_quantized_read",
           "dpllm_quantized_attention_workspace_bytes", "dpllm_quantized_attention", "dpllm_sample_workspace_bytes", "dpllm_sample"]


class DpllmError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("dpllm error %d: %s" % (code, msg))
        self.code = code


class _Heads(C.Structure):
    """dpllm_heads: a tensor [batch][tokens][heads][head_dim]."""
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Cache(C.Structure):
    """dpllm_cache."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64), ("table", C.c_void_p), ("table_stride", C.c_int64), ("dtype", C.c_int32), ("layers", C.c_int32),
                ("pages", C.c_int32), ("page", C.c_int32), ("pages_per_seq", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32)]


class _QuantizedCache(C.Structure):
    """dpllm_quantized_cache."""
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_scales", "v_scales")] + \
               [(p + n + "_stride", C.c_int64) for p in ("", "scale_") for n in ("layer", "page", "token", "head")] + \
               [("table", C.c_void_p), ("table_stride", C.c_int64)] + \
               [(n, C.c_int32) for n in ("format", "layers", "pages", "page", "pages_per_seq", "heads", "head_dim")]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libdpllm.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(there is no fallback path)")
    L = C.CDLL(_LIB_PATH)
    vp, i32, f32, sz, i64, f64, heads, cache = C.c_void_p, C.c_int, C.c_float, C.c_size_t, C.c_int64, C.c_double, C.POINTER(_Heads), C.POINTER(_Cache)
    L.dpllm_model_create.argtypes = [C.POINTER(vp), i32]
    L.dpllm_model_destroy.argtypes = [vp]
    L.dpllm_model_destroy.restype = None
    L.dpllm_last_error.argtypes = [vp]
    L.dpllm_last_error.restype = C.c_char_p
    L.dpllm_linear_device_bytes.argtypes = [i32, i32, i32, i32, C.POINTER(sz)]
    L.dpllm_debug_locate.argtypes = [i32, i32, i32, i32, i32, i32, i32, C.POINTER(sz), C.POINTER(i32)]
    L.dpllm_load_linear.argtypes = [vp, i32, i32, i32, i32, i32, vp, C.POINTER(vp), i32, vp, sz, vp]
    L.dpllm_set_selector.argtypes = [vp, i32, i32, i32, i32, vp, i32, f32, f32, f32]
    L.dpllm_set_threshold.argtypes = [vp, i32, i32, i32, f32]
    L.dpllm_set_active_pair.argtypes = [vp, i32, i32, i32]
    L.dpllm_set_selector_input.argtypes = [vp, i32, vp]
    L.dpllm_workspace_bytes.argtypes = [vp, C.POINTER(sz)]
    L.dpllm_set_workspace.argtypes = [vp, vp, sz, vp]
    L.dpllm_set_target_entry.argtypes = [vp, i32, i32, i32, i32, f32]
    L.dpllm_set_target.argtypes = [vp, i32, vp]
    L.dpllm_estimate.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp]
    L.dpllm_estimate_noalloc.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp]
    L.dpllm_gemv.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp]
    L.dpllm_decode_step.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, vp, vp]
    L.dpllm_decode_step_parts.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, vp, i32, vp]
    L.dpllm_debug_unpack.argtypes = [vp, i32, i32, vp, vp]
    L.dpllm_debug_set_polls.argtypes = [vp, i32]
    L.dpllm_debug_set_one_launch.argtypes = [vp, i32, i32]
    L.dpllm_debug_step_launches.argtypes = [vp, C.POINTER(i32)]
    L.dpllm_debug_copy.argtypes = [vp, vp, sz, vp]
    L.dpllm_debug_read.argtypes = [vp, sz, vp, vp]
    L.dpllm_call_error.argtypes = []
    L.dpllm_call_error.restype = C.c_char_p
    L.dpllm_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, C.POINTER(f64), C.POINTER(f32)]
    L.dpllm_rope.argtypes = [heads, heads, C.POINTER(i32), i32, i32, i32, i32, i32, i32, i32, vp, f32, vp, i64, i32, vp]
    L.dpllm_tree_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, C.POINTER(sz)]
    L.dpllm_tree_attention.argtypes = [cache, i32, i32, i32, i32, vp, i32, heads, heads, heads, vp, i64, f32, heads, vp, vp, sz, vp]
    L.dpllm_verify_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, C.POINTER(sz)]
    L.dpllm_verify.argtypes = [i32, i32, i32, i32, vp, i64, i64, vp, i64, i64, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    L.dpllm_cache_append.argtypes = [cache, i32, i32, i32, i32, vp, heads, i64, heads, i64, vp, i64, vp, vp]
    quantized = C.POINTER(_QuantizedCache)
    L.dpllm_norm_rope.argtypes = [heads, heads, C.POINTER(i32), C.POINTER(vp), C.POINTER(i64), i32, f32, i32, i32, i32, i32, i32, i32, i32, vp, f32, vp, i64, vp]
    L.dpllm_norm_rope_backward_workspace_bytes.argtypes = [C.POINTER(i32), C.POINTER(i64), i32, i32, i32, i32, C.POINTER(sz)]
    L.dpllm_norm_rope_backward.argtypes = [heads, heads, heads, C.POINTER(i32), C.POINTER(vp), C.POINTER(vp), C.POINTER(i64), i32, f32, i32, i32, i32, i32, i32, i32, i32,
                                           vp, f32, vp, i64, vp, sz, vp]
    L.dpllm_quantized_append.argtypes = [quantized, i32, i32, i32, i32, vp, i32, heads, i64, heads, i64, vp, i64, vp, vp]
    L.dpllm_quantized_read.argtypes = [quantized, i32, i32, i32, i32, vp, vp, i32, heads, i64, heads, i64, vp]
    L.dpllm_quantized_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, C.POINTER(sz)]
    L.dpllm_quantized_attention.argtypes = [quantized, i32, i32, i32, i32, i32, vp, i32, heads, heads, heads, vp, i64, f32, heads, vp, vp, sz, vp]
    L.dpllm_sample_workspace_bytes.argtypes = [i32, i32, i32, C.POINTER(sz)]
    L.dpllm_sample.argtypes = [i32, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    return L


lib = _load()

try:
    from . import _calls
except ImportError as e:
    raise ImportError("_calls.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(there is no fallback path)") from e
_calls.bind(C.cast(lib.dpllm_gemv, C.c_void_p).value, C.cast(lib.dpllm_estimate, C.c_void_p).value,
            torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)

_calls.bind_tokens(tuple(C.cast(f, C.c_void_p).value for f in (lib.dpllm_rope, lib.dpllm_tree_attention_workspace_bytes, lib.dpllm_tree_attention,
                                                               lib.dpllm_verify_workspace_bytes, lib.dpllm_verify, lib.dpllm_cache_append)),
                   (torch.float16, torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.float64), torch.empty_like)
_calls.bind_step(tuple(C.cast(f, C.c_void_p).value for f in (lib.dpllm_norm_rope, lib.dpllm_norm_rope_backward_workspace_bytes, lib.dpllm_norm_rope_backward,
                                                             lib.dpllm_quantized_append, lib.dpllm_quantized_read,
                                                             lib.dpllm_quantized_attention_workspace_bytes, lib.dpllm_quantized_attention, lib.dpllm_sample_workspace_bytes,
                                                             lib.dpllm_sample)))


def _stream():
    """The current stream's handle.  torch.cuda.current_stream() builds a Stream object for it (2.9 us of a call of
    7.1 us, of which the library takes 3.3); the raw lookup takes 0.2 us but wants an initialised device."""
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check(model, rc):
    if rc != 0:
        msg = lib.dpllm_last_error(model).decode() if model else ""
        raise DpllmError(rc, msg)


def dpllm_linear_device_bytes(out, in_, p, kmin):
    n = C.c_size_t(0)
    rc = lib.dpllm_linear_device_bytes(out, in_, p, kmin, C.byref(n))
    if rc != 0:
        raise DpllmError(rc, "dpllm_linear_device_bytes(%d,%d,%d,%d)" % (out, in_, p, kmin))
    return n.value


def dpllm_debug_copy(dst, src):
    nbytes = src.numel() * src.element_size()
    rc = lib.dpllm_debug_copy(_ptr(dst), _ptr(src), nbytes, _stream())
    if rc != 0:
        raise DpllmError(rc, "dpllm_debug_copy")


def dpllm_debug_read(src, sink):
    nbytes = src.numel() * src.element_size()
    rc = lib.dpllm_debug_read(_ptr(src), nbytes, _ptr(sink), _stream())
    if rc != 0:
        raise DpllmError(rc, "dpllm_debug_read")


def _call(rc):
    """Raises what a call without a model was refused for."""
    if rc != 0:
        raise DpllmError(rc, lib.dpllm_call_error().decode())


_DTYPES = {torch.float16: DPLLM_F16, torch.bfloat16: DPLLM_BF16, torch.float32: DPLLM_F32}


def _need(ok, what):
    """Refuses what the library cannot see: types, shapes and devices of tensors."""
    if not ok:
        raise DpllmError(DPLLM_EINVAL, what)


def _on(t, what):
    """Whether t is on the device.  On another one than the current it is refused: the call would run on the current device's stream."""
    if not t.is_cuda:
        return False
    _need(t.get_device() == torch._C._cuda_getDevice(), "%s is on device %d, which is not the current one" % (what, t.get_device()))
    return True


def _dtype(t, what):
    _need(t.dtype in _DTYPES and _on(t, what), what + " has to be a device tensor of float16, bfloat16 or float32")
    return _DTYPES[t.dtype]


def _space(t):
    """The pointer and bytes of a caller's workspace (or of none)."""
    if t is None:
        return None, 0
    _need(_on(t, "the workspace") and t.is_contiguous(), "the workspace has to be a contiguous device tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def _index(t, shape, what):
    """The pointer of a contiguous int32 device tensor of this shape (None: not given)."""
    if t is None:
        return None
    _need(t.dtype == torch.int32 and _on(t, what) and tuple(t.shape) == tuple(shape) and t.is_contiguous(),
          "%s has to be a contiguous int32 device tensor %s" % (what, list(shape)))
    return t.data_ptr()


def _view(t, what):
    """dpllm_heads of a tensor [batch][tokens][heads][head_dim] (or of one layer of such)."""
    _need(t.dim() == 4 and _on(t, what), what + " has to be a device tensor [batch][tokens][heads][head_dim]")
    b, n, h, d = t.stride()
    _need(d == 1 or t.shape[3] == 1 or t.numel() == 0, "the last dimension of %s has to be contiguous" % what)
    return _Heads(t.data_ptr(), b, n, h)


def _no_tangents(*given):
    """Tensors (or tuples of them, or None) of a call that has a gradient; in forward mode it has none, and would lose what they carry."""
    for g in given:
        for t in (g,) if isinstance(g, torch.Tensor) else g or ():
            _need(t is None or forward_ad.unpack_dual(t).tangent is None, "this call has no derivative in forward mode, but one of the tensors has a tangent")


def dpllm_rope_frequencies(rotary_dim, base=10000.0, scaling=DPLLM_ROPE_PLAIN, factor=1.0, trained=0, low=1.0, high=32.0):
    """(angles per position: device, float64 [rotary_dim / 2]; what the rotated part is multiplied by): made once, for dpllm_rope."""
    f, scale = (C.c_double * max(1, rotary_dim // 2))(), C.c_float(0.0)
    _call(lib.dpllm_rope_frequencies(rotary_dim, base, scaling, factor, trained, low, high, f, C.byref(scale)))
    return torch.tensor(list(f), dtype=torch.float64, device="cuda"), scale.value


def dpllm_rope(x, positions, freqs, out=None, scale=1.0, layout=DPLLM_ROPE_HALF, inverse=False):
    """x: a tensor [batch][tokens][heads][head_dim], or a tuple of such that share everything but their heads (queries, keys).  positions: int32
    [batch][tokens], or [tokens] for all sequences.  out: where the results go (x itself: in place); new tensors unless given, with x's order of dimensions.
    New results of tensors that require a gradient have one (in reverse mode; a tensor with a tangent is refused)."""
    if forward_ad._current_level >= 0:
        _no_tangents(x)
    made = _calls.rope(x, positions, freqs, out, scale, layout, inverse)
    if type(made) is not int:
        return made
    if made != _calls.ELSEWHERE:
        _call(made)
    # out of the ordinary: the long way, with the errors that has
    xs = (x,) if isinstance(x, torch.Tensor) else tuple(x)
    _need(0 < len(xs) <= 4, "dpllm_rope takes 1 to 4 tensors")
    first = xs[0]
    if torch.is_grad_enabled() and any(t.requires_grad for t in (*xs, *(() if out is None else (out,) if isinstance(out, torch.Tensor) else out))):
        _need(out is None, "results that go into out have no gradient, but one of the tensors requires one")
        outs = _Rope.apply(positions, freqs, scale, layout, bool(inverse), *xs)
        return outs[0] if isinstance(x, torch.Tensor) else outs
    dtype = _dtype(first, "x")
    outs = tuple(torch.empty_like(t) for t in xs) if out is None else (out,) if isinstance(out, torch.Tensor) else tuple(out)
    _need(len(outs) == len(xs), "out has to hold a tensor for each of x")
    views = [_view(t, "x") for t in xs]
    into = [_view(t, "out") for t in outs]
    b, n, _, d = first.shape
    for t, o in zip(xs, outs):
        _need(t.dtype == o.dtype == first.dtype and t.shape == o.shape and t.shape[:2] == (b, n) and t.shape[3] == d,
              "the tensors of dpllm_rope share type, sequences, tokens and head_dim, and out the shapes of x")
    _need(freqs.dtype == torch.float64 and _on(freqs, "freqs") and freqs.is_contiguous() and freqs.dim() == 1, "freqs has to be a contiguous float64 device vector")
    pos = _index(positions, (n,) if positions.dim() == 1 else (b, n), "positions")
    m = len(xs)
    _call(lib.dpllm_rope((_Heads * m)(*views), (_Heads * m)(*into), (C.c_int * m)(*[t.shape[2] for t in xs]), m, b, n, d, dtype, 2 * freqs.shape[0],
                         layout, freqs.data_ptr(), scale, pos, 0 if positions.dim() == 1 else n, 1 if inverse else 0, _stream()))
    return outs[0] if isinstance(x, torch.Tensor) else outs


class _Rope(torch.autograd.Function):
    """dpllm_rope of tensors that require a gradient: a rotation's transpose is the inverse one, with the same scale."""

    @staticmethod
    def forward(ctx, positions, freqs, scale, layout, inverse, *xs):
        ctx.save_for_backward(positions, freqs)
        ctx.how = scale, layout, inverse
        return dpllm_rope(xs, positions, freqs, scale=scale, layout=layout, inverse=inverse)

    @staticmethod
    def backward(ctx, *grads):
        positions, freqs = ctx.saved_tensors
        scale, layout, inverse = ctx.how
        wanted = ctx.needs_input_grad[5:]
        # (the gradient of a sum is one number for all elements: the last dimension has no stride)
        given = tuple(g if g.stride(3) == 1 else g.contiguous() for g, w in zip(grads, wanted) if w)
        made = iter(dpllm_rope(given, positions, freqs, scale=scale, layout=layout, inverse=not inverse))
        return (None,) * 5 + tuple(next(made) if w else None for w in wanted)


class Cache:
    """A paged cache of keys and values: views of the caller's tensors k and v, [layers][pages][page][heads][head_dim] with the same strides (a pool
    whose pages hold head after head is passed transposed), and the page table, int32 [batch][pages per sequence] on the device.  Without a
    table sequence b has page b.  The table may change on the device at any time; the object holds the tensors alive."""

    def __init__(self, k, v, table=None):
        _need(k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.is_cuda and v.is_cuda and
              k.get_device() == v.get_device(),
              "k and v have to be device tensors [layers][pages][page][heads][head_dim] of one type, shape, strides and device")
        _need(k.dtype in _DTYPES, "k and v have to be float16, bfloat16 or float32")
        _need(k.stride(4) == 1 or k.shape[4] == 1, "the last dimension of k and v has to be contiguous")
        if table is not None:
            _need(table.dtype == torch.int32 and table.is_cuda and table.get_device() == k.get_device() and table.dim() == 2 and
                  (table.stride(1) == 1 or table.shape[1] == 1), "table has to be an int32 tensor [batch][pages per sequence] on the device of k and v")
        self.k, self.v, self.table, self.device = k, v, table, k.get_device()
        self.layers, self.pages, self.page, self.heads, self.head_dim = k.shape
        self.pages_per_seq = 1 if table is None else table.shape[1]
        self.batch = self.pages if table is None else table.shape[0]
        self.capacity = self.pages_per_seq * self.page
        self.c = _Cache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), k.stride(3), _ptr(table), 0 if table is None else table.stride(0),
                        _DTYPES[k.dtype], self.layers, self.pages, self.page, self.pages_per_seq, self.heads, self.head_dim)
        self.address, self.size = C.addressof(self.c), C.sizeof(self.c)      # (its size tells the native part which kind it is)


def dpllm_tree_attention_workspace_bytes(batch, nodes, heads, kv_heads, head_dim, max_len):
    n = C.c_size_t(0)
    _call(lib.dpllm_tree_attention_workspace_bytes(batch, nodes, heads, kv_heads, head_dim, max_len, C.byref(n)))
    return n.value


def dpllm_tree_attention(cache, layer, lens, q, k_new=None, v_new=None, mask=None, scale=None, out=None, lse=None, max_len=None, workspace=None):
    """q: [batch][nodes][heads][head_dim]; k_new, v_new: [batch][nodes][cache.heads][head_dim].  mask: int64 [batch or 1][nodes][ceil(nodes / 64)], bit j of
    row i: node i sees node j; None: a chain.  scale: 1 / sqrt(head_dim) unless given.  out: a new tensor with q's order of dimensions unless given.  lse:
    float32 [batch][nodes][heads] to be filled.  max_len: how long the longest context is expected to be (the cache's capacity unless given).  workspace:
    uint8, allocated for the call unless given.  The result has no gradient."""
    made = _calls.attention(cache, layer, lens, q, k_new, v_new, mask, scale, out, lse, max_len, workspace)
    if type(made) is not int:
        return made
    if made != _calls.ELSEWHERE:
        _call(made)
    _need(isinstance(cache, Cache), "cache has to be a Cache")
    _on(cache.k, "the cache")
    _need(q.dim() == 4 and q.dtype == cache.k.dtype and q.shape[3] == cache.head_dim, "q has to be [batch][nodes][heads][head_dim] of the cache's type and head_dim")
    b, n, h, d = q.shape
    _need(b <= cache.batch, "q has more sequences than the cache")
    new = (b, n, cache.heads, d)
    _need((k_new is None) == (v_new is None), "k_new and v_new are given together or not at all")
    if k_new is not None:
        _need(k_new.shape == new and v_new.shape == new and k_new.dtype == v_new.dtype == q.dtype,
              "k_new and v_new have to be [batch][nodes][kv heads][head_dim] of the cache's type")
    if out is None:
        out = torch.empty_like(q)
    _need(out.shape == q.shape and out.dtype == q.dtype, "out has to have the shape and type of q")
    if mask is not None:
        _need(mask.dtype == torch.int64 and _on(mask, "mask") and mask.is_contiguous() and mask.dim() == 3 and mask.shape[0] in (1, b) and
              mask.shape[1:] == (n, (n + 63) // 64), "mask has to be a contiguous int64 device tensor [batch or 1][nodes][ceil(nodes / 64)]")
    _need(lse is None or (lse.dtype == torch.float32 and _on(lse, "lse") and lse.shape == (b, n, h) and lse.is_contiguous()),
          "lse has to be a contiguous float32 device tensor [batch][nodes][heads]")
    max_len = cache.capacity if max_len is None else min(max_len, cache.capacity)
    if workspace is None:
        need = dpllm_tree_attention_workspace_bytes(b, n, h, cache.heads, d, max_len)
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    _call(lib.dpllm_tree_attention(C.byref(cache.c), layer, b, n, h, _index(lens, (b,), "lens"), max_len, C.byref(_view(q, "q")),
                                   None if k_new is None else C.byref(_view(k_new, "k_new")), None if v_new is None else C.byref(_view(v_new, "v_new")),
                                   _ptr(mask), 0 if mask is None or mask.shape[0] == 1 else mask.stride(0), d ** -0.5 if scale is None else scale,
                                   C.byref(_view(out, "out")), _ptr(lse), *_space(workspace), _stream()))
    return out


def dpllm_verify_workspace_bytes(batch, nodes, vocabulary, dtype, draft, siblings):
    n = C.c_size_t(0)
    _call(lib.dpllm_verify_workspace_bytes(batch, nodes, vocabulary, dtype, 1 if draft else 0, siblings, C.byref(n)))
    return n.value


def dpllm_verify(logits, tokens, uniforms, temperature, parents=None, draft=None, siblings=None, count=None, path=None, words=None, workspace=None):
    """logits, draft: [batch][nodes][vocabulary] of one type; tokens, parents: int32 [batch][nodes]; uniforms: float32 [batch][nodes]; temperature: float32
    [batch].  siblings: the most children that a node has (1 for a chain; every node but the root unless given, and with draft rows each is two launches).  Returns (count [batch], path, words
    [batch][nodes]), int32, new tensors unless given.  workspace: uint8, allocated for the call unless given."""
    if count is None and path is None and words is None and workspace is None:
        made = _calls.verify(logits, tokens, uniforms, temperature, parents, draft,
                             siblings if siblings is not None else 1 if parents is None else max(1, tokens.shape[-1] - 1))
        if type(made) is not int:
            return made
        if made != _calls.ELSEWHERE:
            _call(made)
    dtype = _dtype(logits, "logits")
    _need(logits.dim() == 3 and (logits.stride(2) == 1 or logits.shape[2] == 1 or logits.numel() == 0), "logits has to be [batch][nodes][vocabulary], the words contiguous")
    b, n, v = logits.shape
    if draft is not None:
        _need(draft.shape == logits.shape and draft.dtype == logits.dtype and _on(draft, "draft") and (draft.stride(2) == 1 or v == 1 or draft.numel() == 0),
              "draft has to be a device tensor of the shape and type of logits, the words contiguous")
    for t, shape, what in ((uniforms, (b, n), "uniforms"), (temperature, (b,), "temperature")):
        _need(t.dtype == torch.float32 and _on(t, what) and tuple(t.shape) == shape and t.is_contiguous(), "%s has to be a contiguous float32 device tensor %s" % (what, list(shape)))
    if siblings is None:
        siblings = 1 if parents is None else max(1, n - 1)
    count = torch.empty(b, dtype=torch.int32, device="cuda") if count is None else count
    path = torch.empty((b, n), dtype=torch.int32, device="cuda") if path is None else path
    words = torch.empty((b, n), dtype=torch.int32, device="cuda") if words is None else words
    if workspace is None:
        workspace = torch.empty(dpllm_verify_workspace_bytes(b, n, v, dtype, draft is not None, siblings), dtype=torch.uint8, device="cuda")
    _call(lib.dpllm_verify(b, n, v, dtype, _ptr(logits), logits.stride(0), logits.stride(1), _ptr(draft), 0 if draft is None else draft.stride(0),
                           0 if draft is None else draft.stride(1), _index(tokens, (b, n), "tokens"), _index(parents, (b, n), "parents"), _ptr(uniforms), _ptr(temperature),
                           siblings, _index(count, (b,), "count"), _index(path, (b, n), "path"), _index(words, (b, n), "words"), *_space(workspace), _stream()))
    return count, path, words


def dpllm_cache_append(cache, lens, k_new, v_new, path=None, count=None, layer=0):
    """k_new, v_new: [batch][nodes][heads][head_dim] for one layer, or [layers][batch]... for as many from `layer` on.  path: int32 [batch][nodes],
    count: int32 [batch]."""
    made = _calls.append(cache, lens, k_new, v_new, path, count, layer)
    if made != _calls.ELSEWHERE:
        return _call(made)
    _need(isinstance(cache, Cache), "cache has to be a Cache")
    _on(cache.k, "the cache")
    if k_new.dim() == 4:
        k_new, v_new = k_new.unsqueeze(0), v_new.unsqueeze(0)
    _need(k_new.dim() == 5 and k_new.shape == v_new.shape and k_new.dtype == v_new.dtype == cache.k.dtype,
          "k_new and v_new have to be [layers][batch][nodes][heads][head_dim] of the cache's type")
    layers, b, n, h, d = k_new.shape
    _need((h, d) == (cache.heads, cache.head_dim) and b <= cache.batch, "k_new and v_new have to fit the cache's heads, head_dim and sequences")
    _need(layers == 0 or (_on(k_new, "k_new") and _on(v_new, "v_new")), "k_new and v_new have to be device tensors")
    if layers == 0:
        return
    _call(lib.dpllm_cache_append(C.byref(cache.c), layer, layers, b, n, _index(lens, (b,), "lens"), C.byref(_view(k_new[0], "k_new")), k_new.stride(0),
                                 C.byref(_view(v_new[0], "v_new")), v_new.stride(0), _index(path, (b, n), "path"), n,
                                 _index(count, (b,), "count"), _stream()))


def _norm_weights(xs, weights, contiguous=False):
    """The weights of the tensors xs as tensors (or None) of one type, and what the library takes of them: pointers, strides, that type."""
    ws = (None,) * len(xs) if weights is None else (weights,) if isinstance(weights, torch.Tensor) else tuple(weights)
    _need(len(ws) == len(xs), "there has to be a weight (or None) for each tensor")
    made, dtype = [], None
    for t, w in zip(xs, ws):
        if w is not None:
            h, d = t.shape[2], t.shape[3]
            _need(w.dtype in _DTYPES and _on(w, "a weight") and w.shape in ((d,), (h, d)), "a weight has to be a device tensor [head_dim] or [heads][head_dim]")
            _need(dtype in (None, w.dtype), "the weights have to be of one type")
            dtype = w.dtype
            if (w.dim() == 2 and w.stride(0) == 0 and h > 1) or (d > 1 and w.stride(-1) != 1) or (contiguous and not w.is_contiguous()):
                w = w.contiguous()
        made.append(w)
    n = len(xs)
    return made, (C.c_void_p * n)(*[_ptr(w) for w in made]), (C.c_int64 * n)(*[w.stride(0) if w is not None and w.dim() == 2 and w.shape[0] > 1 else 0 for w in made]), \
        DPLLM_F32 if dtype is None else _DTYPES[dtype]


def _norm_plan(first, positions, freqs):
    """Pointers and sizes of a rotation: rotary_dim, freqs, positions, their stride."""
    if freqs is None:
        return 0, None, None, 0
    b, n = first.shape[:2]
    _need(freqs.dtype == torch.float64 and _on(freqs, "freqs") and freqs.is_contiguous() and freqs.dim() == 1, "freqs has to be a contiguous float64 device vector")
    _need(positions is not None, "a rotation needs positions")
    return 2 * freqs.shape[0], freqs.data_ptr(), _index(positions, (n,) if positions.dim() == 1 else (b, n), "positions"), 0 if positions.dim() == 1 else n


def _same_tokens(xs, others, what):
    first = xs[0]
    _need(first.dim() == 4 and len(xs) == len(others), what + " has to hold a tensor [batch][tokens][heads][head_dim] for each of x")
    for t, o in zip(xs, others):
        _need(t.dtype == o.dtype == first.dtype and t.dim() == 4 and t.shape == o.shape and t.shape[:2] == first.shape[:2] and t.shape[3] == first.shape[3],
              "the tensors share type, sequences, tokens and head_dim, and %s the shapes of x" % what)


def dpllm_norm_rope(x, weights, positions=None, freqs=None, eps=1e-6, out=None, scale=1.0, layout=DPLLM_ROPE_HALF):
    """x: a tensor [batch][tokens][heads][head_dim], or a tuple of such that share everything but their heads (queries, keys).  weights: a tensor [head_dim] or [heads][head_dim]
    for each (None: 1), all of one type.  positions, freqs, scale, layout: as for dpllm_rope; freqs None: the norm alone.  out: where the results go (x itself: in place); new tensors
    unless given.  New results have a gradient with respect to x and the weights (in reverse mode; a tensor with a tangent is refused)."""
    if forward_ad._current_level >= 0:
        _no_tangents(x, weights)
    made = _calls.norm_rope(x, weights, positions, freqs, eps, out, scale, layout, torch.is_grad_enabled())
    if type(made) is not int:
        return made
    if made != _calls.ELSEWHERE:
        _call(made)
    xs = (x,) if isinstance(x, torch.Tensor) else tuple(x)
    _need(0 < len(xs) <= 4, "dpllm_norm_rope takes 1 to 4 tensors")
    outs = None if out is None else (out,) if isinstance(out, torch.Tensor) else tuple(out)
    given = () if weights is None else (weights,) if isinstance(weights, torch.Tensor) else tuple(w for w in weights if w is not None)
    if torch.is_grad_enabled() and any(t.requires_grad for t in (*xs, *given, *(outs or ()))):
        _need(outs is None, "results that go into out have no gradient, but one of the tensors requires one")
        ws = (None,) * len(xs) if weights is None else (weights,) if isinstance(weights, torch.Tensor) else tuple(weights)
        made = _NormRope.apply(positions, freqs, eps, scale, layout, len(xs), *xs, *ws)
        return made[0] if isinstance(x, torch.Tensor) else made
    dtype = _dtype(xs[0], "x")
    outs = tuple(torch.empty_like(t) for t in xs) if outs is None else outs
    _same_tokens(xs, outs, "out")
    views, into = [_view(t, "x") for t in xs], [_view(t, "out") for t in outs]
    held, ws, strides, w_dtype = _norm_weights(xs, weights)
    rotary, f, pos, pos_stride = _norm_plan(xs[0], positions, freqs)
    b, n, _, d = xs[0].shape
    m = len(xs)
    _call(lib.dpllm_norm_rope((_Heads * m)(*views), (_Heads * m)(*into), (C.c_int * m)(*[t.shape[2] for t in xs]), ws, strides, w_dtype, eps, m, b, n, d, dtype, rotary, layout,
                              f, scale, pos, pos_stride, _stream()))
    return outs[0] if isinstance(x, torch.Tensor) else outs


def dpllm_norm_rope_backward_workspace_bytes(heads, weight_strides, batch, tokens, head_dim):
    m, n = len(heads), C.c_size_t(0)
    _call(lib.dpllm_norm_rope_backward_workspace_bytes((C.c_int * m)(*heads), (C.c_int64 * m)(*weight_strides), m, batch, tokens, head_dim, C.byref(n)))
    return n.value


def dpllm_norm_rope_backward(x, grads, weights, positions=None, freqs=None, eps=1e-6, out=None, scale=1.0, layout=DPLLM_ROPE_HALF, wanted=None, workspace=None):
    """The gradients of the inputs and of the weights of dpllm_norm_rope from those of its results, grads, as (like x, like weights).  out: where those of the inputs go (grads or x
    themselves, say).  wanted: a truth value for each weight whether its gradient is (all are unless given; the others give None).  workspace: uint8, allocated for the call unless given."""
    if forward_ad._current_level >= 0:
        _no_tangents(x, grads, weights)
    if workspace is None:
        made = _calls.norm_rope_backward(x, grads, weights, positions, freqs, eps, out, scale, layout, wanted)
        if type(made) is not int:
            return made
        if made != _calls.ELSEWHERE:
            _call(made)
    lone = isinstance(x, torch.Tensor)
    xs, gs = (x,) if lone else tuple(x), (grads,) if isinstance(grads, torch.Tensor) else tuple(grads)
    _need(0 < len(xs) <= 4, "dpllm_norm_rope_backward takes 1 to 4 tensors")
    dtype = _dtype(xs[0], "x")
    outs = tuple(torch.empty_like(t) for t in xs) if out is None else (out,) if isinstance(out, torch.Tensor) else tuple(out)
    _same_tokens(xs, gs, "grads")
    _same_tokens(xs, outs, "out")
    views, grad_views, into = [_view(t, "x") for t in xs], [_view(t, "grads") for t in gs], [_view(t, "out") for t in outs]
    held, ws, strides, w_dtype = _norm_weights(xs, weights, contiguous=True)
    wanted = [w is not None and (wanted is None or bool(wanted[i])) for i, w in enumerate(held)]
    made = tuple(torch.empty_like(w) if g else None for w, g in zip(held, wanted))
    rotary, f, pos, pos_stride = _norm_plan(xs[0], positions, freqs)
    b, n, _, d = xs[0].shape
    m = len(xs)
    heads = [t.shape[2] for t in xs]
    if workspace is None and any(wanted):
        need = dpllm_norm_rope_backward_workspace_bytes(heads, list(strides), b, n, d)
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    _call(lib.dpllm_norm_rope_backward((_Heads * m)(*views), (_Heads * m)(*grad_views), (_Heads * m)(*into), (C.c_int * m)(*heads), ws,
                                       (C.c_void_p * m)(*[_ptr(g) for g in made]), strides, w_dtype, eps, m, b, n, d, dtype, rotary, layout, f, scale, pos, pos_stride,
                                       *_space(workspace), _stream()))
    return (outs[0], made[0]) if lone else (outs, made)


class _NormRope(torch.autograd.Function):
    """dpllm_norm_rope of tensors (or weights) that require a gradient."""

    @staticmethod
    def forward(ctx, positions, freqs, eps, scale, layout, n, *tensors):
        xs, ws = tensors[:n], tensors[n:]
        ctx.save_for_backward(positions, freqs, *tensors)
        ctx.how = eps, scale, layout, n
        return dpllm_norm_rope(xs, ws, positions, freqs, eps=eps, scale=scale, layout=layout)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        positions, freqs, *tensors = ctx.saved_tensors
        eps, scale, layout, n = ctx.how
        needs = ctx.needs_input_grad[6:]
        # (the gradient of a sum is one number for all elements: the last dimension has no stride)
        grads = tuple(g if g.stride(3) == 1 or g.shape[3] == 1 else g.contiguous() for g in grads)
        some = [i for i in range(n) if needs[i] or needs[n + i]]
        made = [None] * (2 * n)
        outs, weights = dpllm_norm_rope_backward(tuple(tensors[i] for i in some), tuple(grads[i] for i in some), tuple(tensors[n + i] for i in some), positions, freqs, eps=eps,
                                                 scale=scale, layout=layout, wanted=[needs[n + i] for i in some])
        for i, o, w in zip(some, outs, weights):
            made[i], made[n + i] = o if needs[i] else None, w
        return (None,) * 6 + tuple(made)


class QuantizedCache:
    """A paged cache of keys and values in 8 or 4 bits: views of the caller's tensors.  k, v: codes, uint8 [layers][pages][page][heads][bytes of a head] with the same strides; k_scales, v_scales:
    float32 [layers][pages][page][heads], of DPLLM_CACHE_INT4 bfloat16 [layers][pages][page][heads][2] (scale, offset).  table: as of Cache.  The object holds the tensors alive."""

    def __init__(self, k, v, k_scales, v_scales, format, table=None):
        _need(format in (DPLLM_CACHE_E4M3, DPLLM_CACHE_INT8, DPLLM_CACHE_INT4), "unknown format %s" % (format,))
        pair = format == DPLLM_CACHE_INT4
        _need(k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype == torch.uint8,
              "k and v have to be uint8 tensors [layers][pages][page][heads][bytes] of one shape and strides")
        _need(k.stride(4) == 1 or k.shape[4] == 1, "the last dimension of k and v has to be contiguous")
        of = (*k.shape[:4], 2) if pair else tuple(k.shape[:4])
        _need(k_scales.shape == of and v_scales.shape == of and k_scales.stride() == v_scales.stride() and
              k_scales.dtype == v_scales.dtype == (torch.bfloat16 if pair else torch.float32),
              "k_scales and v_scales have to be %s tensors %s with the same strides" % ("bfloat16" if pair else "float32", list(of)))
        _need(all(t.is_cuda and t.get_device() == k.get_device() for t in (k, v, k_scales, v_scales)), "codes and scales have to be on one device")
        by = 2 if pair else 1
        strides = [s if n > 1 else 0 for s, n in zip(k_scales.stride()[:4], of)]
        _need(not pair or (k_scales.stride(4) == 1 and all(s % 2 == 0 for s in strides)), "scale and offset of a head have to lie side by side, and whole such pairs apart")
        if table is not None:
            _need(table.dtype == torch.int32 and table.is_cuda and table.get_device() == k.get_device() and table.dim() == 2 and
                  (table.stride(1) == 1 or table.shape[1] == 1), "table has to be an int32 tensor [batch][pages per sequence] on the device of k and v")
        self.k, self.v, self.k_scales, self.v_scales, self.format, self.table, self.device = k, v, k_scales, v_scales, format, table, k.get_device()
        self.layers, self.pages, self.page, self.heads, size = k.shape
        self.head_dim = 2 * size if pair else size
        self.pages_per_seq = 1 if table is None else table.shape[1]
        self.batch = self.pages if table is None else table.shape[0]
        self.capacity = self.pages_per_seq * self.page
        self.c = _QuantizedCache(_ptr(k), _ptr(v), _ptr(k_scales), _ptr(v_scales), *k.stride()[:4], *[s // by for s in strides], _ptr(table),
                                 0 if table is None else table.stride(0), format, self.layers, self.pages, self.page, self.pages_per_seq, self.heads, self.head_dim)
        self.address, self.size = C.addressof(self.c), C.sizeof(self.c)      # (its size tells the native part which kind it is)

    @classmethod
    def zeros(cls, format, layers, pages, page, heads, head_dim, table=None):
        """A new one on the current device."""
        pair = format == DPLLM_CACHE_INT4
        _need(not pair or head_dim % 2 == 0, "head_dim has to be even for DPLLM_CACHE_INT4")
        codes = [torch.zeros(layers, pages, page, heads, head_dim // 2 if pair else head_dim, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.zeros(layers, pages, page, heads, *((2,) if pair else ()), dtype=torch.bfloat16 if pair else torch.float32, device="cuda") for _ in range(2)]
        return cls(*codes, *scales, format, table)


def dpllm_quantized_append(cache, lens, k_new, v_new, path=None, count=None, layer=0):
    """dpllm_cache_append into a QuantizedCache; k_new and v_new are float16, bfloat16 or float32."""
    made = _calls.quantized_append(cache, lens, k_new, v_new, path, count, layer)
    if made != _calls.ELSEWHERE:
        return _call(made)
    _need(isinstance(cache, QuantizedCache), "cache has to be a QuantizedCache")
    _on(cache.k, "the cache")
    if k_new.dim() == 4:
        k_new, v_new = k_new.unsqueeze(0), v_new.unsqueeze(0)
    _need(k_new.dim() == 5 and k_new.shape == v_new.shape and k_new.dtype == v_new.dtype and k_new.dtype in _DTYPES,
          "k_new and v_new have to be [layers][batch][nodes][heads][head_dim] of one type")
    layers, b, n, h, d = k_new.shape
    _need((h, d) == (cache.heads, cache.head_dim) and b <= cache.batch, "k_new and v_new have to fit the cache's heads, head_dim and sequences")
    _need(layers == 0 or (_on(k_new, "k_new") and _on(v_new, "v_new")), "k_new and v_new have to be device tensors")
    if layers == 0:
        return
    _call(lib.dpllm_quantized_append(C.byref(cache.c), layer, layers, b, n, _index(lens, (b,), "lens"), _DTYPES[k_new.dtype], C.byref(_view(k_new[0], "k_new")),
                                     k_new.stride(0), C.byref(_view(v_new[0], "v_new")), v_new.stride(0), _index(path, (b, n), "path"), n, _index(count, (b,), "count"), _stream()))


def dpllm_quantized_read(cache, first, tokens, dtype=torch.bfloat16, count=None, layer=0, layers=None, out=None):
    """What a QuantizedCache holds of `tokens` tokens from first[b] on (int32 [batch]; None: 0), as (keys, values) [batch][tokens][heads][head_dim], of `layers` layers from `layer` on
    with a dimension more if that is given.  count: int32 [batch]; from there on, and where the cache holds nothing, are zeros.  out: a pair of tensors to be filled."""
    if out is None:
        made = _calls.quantized_read(cache, getattr(cache, "k", None), first, tokens, dtype, count, layer, layers)
        if type(made) is not int:
            return made
        if made != _calls.ELSEWHERE:
            _call(made)
    _need(isinstance(cache, QuantizedCache), "cache has to be a QuantizedCache")
    _on(cache.k, "the cache")
    b = cache.batch if first is None and count is None else (count if first is None else first).shape[0]
    shape = (1 if layers is None else layers, b, tokens, cache.heads, cache.head_dim)
    _need(dtype in _DTYPES, "dtype has to be float16, bfloat16 or float32")
    if out is None:
        k, v = (torch.empty(shape, dtype=dtype, device="cuda") for _ in range(2))
    else:
        k, v = (t.unsqueeze(0) if layers is None else t for t in out)
        _need(k.shape == shape and v.shape == shape and k.dtype == v.dtype == dtype and _on(k, "out") and _on(v, "out"), "out has to be two device tensors %s of dtype" % (list(shape),))
    _need(b <= cache.batch, "there are more sequences than the cache has")
    if shape[0] > 0:
        _call(lib.dpllm_quantized_read(C.byref(cache.c), layer, shape[0], b, tokens, _index(first, (b,), "first"), _index(count, (b,), "count"), _DTYPES[dtype],
                                       C.byref(_view(k[0], "out")), k.stride(0), C.byref(_view(v[0], "out")), v.stride(0), _stream()))
    return tuple(out) if out is not None else (k, v) if layers is not None else (k[0], v[0])


def dpllm_quantized_attention_workspace_bytes(batch, nodes, heads, kv_heads, head_dim, max_len):
    n = C.c_size_t(0)
    _call(lib.dpllm_quantized_attention_workspace_bytes(batch, nodes, heads, kv_heads, head_dim, max_len, C.byref(n)))
    return n.value


def dpllm_quantized_attention(cache, layer, lens, q, k_new=None, v_new=None, mask=None, scale=None, out=None, lse=None, max_len=None, workspace=None):
    """dpllm_tree_attention over a QuantizedCache; q, k_new, v_new and out are float16 or bfloat16.  The result has no gradient."""
    made = _calls.quantized_attention(cache, layer, lens, q, k_new, v_new, mask, scale, out, lse, max_len, workspace)
    if type(made) is not int:
        return made
    if made != _calls.ELSEWHERE:
        _call(made)
    _need(isinstance(cache, QuantizedCache), "cache has to be a QuantizedCache")
    _on(cache.k, "the cache")
    dtype = _dtype(q, "q")
    _need(q.dim() == 4 and q.shape[3] == cache.head_dim, "q has to be [batch][nodes][heads][head_dim] of the cache's head_dim")
    b, n, h, d = q.shape
    _need(b <= cache.batch, "q has more sequences than the cache")
    new = (b, n, cache.heads, d)
    _need((k_new is None) == (v_new is None), "k_new and v_new are given together or not at all")
    if k_new is not None:
        _need(k_new.shape == new and v_new.shape == new and k_new.dtype == v_new.dtype == q.dtype,
              "k_new and v_new have to be [batch][nodes][kv heads][head_dim] of q's type")
    if out is None:
        out = torch.empty_like(q)
    _need(out.shape == q.shape and out.dtype == q.dtype, "out has to have the shape and type of q")
    if mask is not None:
        _need(mask.dtype == torch.int64 and _on(mask, "mask") and mask.is_contiguous() and mask.dim() == 3 and mask.shape[0] in (1, b) and
              mask.shape[1:] == (n, (n + 63) // 64), "mask has to be a contiguous int64 device tensor [batch or 1][nodes][ceil(nodes / 64)]")
    _need(lse is None or (lse.dtype == torch.float32 and _on(lse, "lse") and lse.shape == (b, n, h) and lse.is_contiguous()),
          "lse has to be a contiguous float32 device tensor [batch][nodes][heads]")
    max_len = cache.capacity if max_len is None else min(max_len, cache.capacity)
    if workspace is None:
        need = dpllm_quantized_attention_workspace_bytes(b, n, h, cache.heads, d, max_len)
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    _call(lib.dpllm_quantized_attention(C.byref(cache.c), layer, b, n, h, dtype, _index(lens, (b,), "lens"), max_len, C.byref(_view(q, "q")),
                                        None if k_new is None else C.byref(_view(k_new, "k_new")), None if v_new is None else C.byref(_view(v_new, "v_new")),
                                        _ptr(mask), 0 if mask is None or mask.shape[0] == 1 else mask.stride(0), d ** -0.5 if scale is None else scale,
                                        C.byref(_view(out, "out")), _ptr(lse), *_space(workspace), _stream()))
    return out


def dpllm_sample_workspace_bytes(rows, vocabulary, dtype):
    n = C.c_size_t(0)
    _call(lib.dpllm_sample_workspace_bytes(rows, vocabulary, dtype, C.byref(n)))
    return n.value


def dpllm_sample(logits, uniforms, temperature, top_k=None, top_p=None, min_p=None, words=None, kept=None, workspace=None):
    """A word for every row of logits [rows][vocabulary], int32 [rows].  uniforms, temperature, top_p, min_p: float32 [rows]; top_k: int32 [rows]; the last three None: no such
    filter.  words: a new tensor unless given.  kept: int32 [rows], to be filled with how many words could have been drawn.  workspace: uint8, allocated for the call unless given."""
    if workspace is None:
        made = _calls.sample(logits, uniforms, temperature, top_k, top_p, min_p, words, kept)
        if type(made) is not int:
            return made
        if made != _calls.ELSEWHERE:
            _call(made)
    dtype = _dtype(logits, "logits")
    _need(logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1 or logits.numel() == 0), "logits has to be [rows][vocabulary], the words contiguous")
    n, v = logits.shape
    for t, what in ((uniforms, "uniforms"), (temperature, "temperature"), (top_p, "top_p"), (min_p, "min_p")):
        _need((t is None and what in ("top_p", "min_p")) or (t is not None and t.dtype == torch.float32 and _on(t, what) and tuple(t.shape) == (n,) and t.is_contiguous()),
              "%s has to be a contiguous float32 device tensor [%d]" % (what, n))
    words = torch.empty(n, dtype=torch.int32, device="cuda") if words is None else words
    if workspace is None:
        workspace = torch.empty(dpllm_sample_workspace_bytes(n, v, dtype), dtype=torch.uint8, device="cuda")
    _call(lib.dpllm_sample(n, v, dtype, _ptr(logits), logits.stride(0), _ptr(uniforms), _ptr(temperature), _index(top_k, (n,), "top_k"), _ptr(top_p), _ptr(min_p),
                           _index(words, (n,), "words"), _index(kept, (n,), "kept"), *_space(workspace), _stream()))
    return words


class Model:
    """Owns the C handle and the torch tensors used as device memory (arenas, workspace)."""

    def __init__(self, n_linears):
        h = C.c_void_p()
        rc = lib.dpllm_model_create(C.byref(h), n_linears)
        if rc != 0:
            raise DpllmError(rc, "dpllm_model_create")
        self.h = h
        self._address = h.value
        self.n = n_linears
        self.arenas = {}
        self.keep = {}
        self.shapes = {}
        self._sel_inputs = {}
        self.workspace = None
        self._ws_stale = True      # the model changed in a way that may ask for a larger workspace

    def dpllm_workspace_bytes(self):
        n = C.c_size_t(0)
        _check(self.h, lib.dpllm_workspace_bytes(self.h, C.byref(n)))
        return n.value

    def dpllm_set_workspace(self, tensor=None):
        """Hands the model a workspace: `tensor` (device, uint8) or a fresh allocation of the size the model asks
        for.  The calls that need one allocate it on first use; call this yourself to choose the moment."""
        need = self.dpllm_workspace_bytes()
        if tensor is None:
            tensor = torch.empty(need, dtype=torch.uint8, device="cuda")
        _check(self.h, lib.dpllm_set_workspace(self.h, _ptr(tensor), tensor.numel() * tensor.element_size(), _stream()))
        old, self.workspace = self.workspace, tensor
        self._ws_stale = False
        return old   # the caller decides when the previous one may go (work enqueued earlier may still use it)

    def _need_workspace(self):
        if self._ws_stale and (self.workspace is None or self.workspace.numel() < self.dpllm_workspace_bytes()):
            old = self.dpllm_set_workspace()
            if old is not None:
                torch.cuda.current_stream().synchronize()
        self._ws_stale = False

    def close(self):
        if self.h:
            lib.dpllm_model_destroy(self.h)
            self.h = None
            self._address = 0

    def __del__(self):
        self.close()

    def dpllm_load_linear(self, id, planes, luts, kmin):
        """planes: int32/uint32 [p][out][in/32] (numpy or torch, host or device);
        luts: dict or list of fp16/uint16 [out][2^k] for k = kmin..p."""
        import numpy as np
        if isinstance(planes, np.ndarray):
            planes = torch.from_numpy(planes.view(np.int32))
        p, out, nw = planes.shape
        if isinstance(luts, dict):
            luts = [luts[k] for k in range(kmin, p + 1)]
        luts = [torch.from_numpy(t.view(np.int16)) if isinstance(t, np.ndarray) else t for t in luts]
        on_dev = planes.is_cuda
        luts = [(t.cuda() if on_dev else t.cpu()).contiguous() for t in luts]
        planes = planes.contiguous()
        nbytes = dpllm_linear_device_bytes(out, nw * 32, p, kmin)
        arena = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        arr = (C.c_void_p * len(luts))(*[t.data_ptr() for t in luts])
        rc = lib.dpllm_load_linear(self.h, id, out, nw * 32, p, kmin, _ptr(planes), arr, 1 if on_dev else 0,
                                   _ptr(arena), nbytes, _stream())
        _check(self.h, rc)
        self.arenas[id] = arena
        self.shapes[id] = (out, nw * 32, p, kmin)
        self._ws_stale = True

    def dpllm_set_selector(self, id, l, h, kind, G=None, alpha=0.0, beta=0.0, T=float("inf")):
        r = 0
        if G is not None:
            G = G.contiguous()
            assert G.is_cuda and G.dtype == torch.float16
            r = G.shape[0]
            self.keep[(id, l, h)] = G
        _check(self.h, lib.dpllm_set_selector(self.h, id, l, h, kind, _ptr(G), r, alpha, beta, T))
        self._ws_stale = True

    def dpllm_set_threshold(self, id, l, h, T):
        _check(self.h, lib.dpllm_set_threshold(self.h, id, l, h, T))

    def dpllm_set_active_pair(self, id, l, h):
        _check(self.h, lib.dpllm_set_active_pair(self.h, id, l, h))

    def dpllm_set_target_entry(self, target, id, l, h, T):
        _check(self.h, lib.dpllm_set_target_entry(self.h, target, id, l, h, T))

    def dpllm_set_target(self, target):
        self._need_workspace()
        _check(self.h, lib.dpllm_set_target(self.h, target, _stream()))

    def dpllm_set_selector_input(self, id, x_sel):
        """x_sel: device fp16 [in] the selector of linear id reads in the step calls (None: its immediate input).
        The model keeps a reference to the tensor."""
        self._sel_inputs[id] = x_sel
        _check(self.h, lib.dpllm_set_selector_input(self.h, id, _ptr(x_sel)))

    def dpllm_estimate(self, id, l, h, x, e_out=None, k_out=None):
        if e_out is not None and k_out is not None and not self._ws_stale:
            rc = _calls.estimate(self._address, id, l, h, x, e_out, k_out)
            if rc != _calls.ELSEWHERE:
                _check(self.h, rc)
                return e_out, k_out
        e_out = torch.empty(1, dtype=torch.float32, device="cuda") if e_out is None else e_out
        k_out = torch.empty(1, dtype=torch.int32, device="cuda") if k_out is None else k_out
        self._need_workspace()
        _check(self.h, lib.dpllm_estimate(self.h, id, l, h, _ptr(x), _ptr(e_out), _ptr(k_out), _stream()))
        return e_out, k_out

    def dpllm_estimate_noalloc(self, id, l, h, x, e_out, k_out):
        """The variant that allocates nothing: the caller passes every buffer, no workspace is touched."""
        _check(self.h, lib.dpllm_estimate_noalloc(self.h, id, l, h, _ptr(x), _ptr(e_out), _ptr(k_out), _stream()))
        return e_out, k_out

    def dpllm_gemv(self, id, k, x, y=None, k_dev=None):
        """k >= 0: fixed bitwidth.  k < 0: read the bitwidth from k_dev on the device."""
        if y is not None and not self._ws_stale:
            rc = _calls.gemv(self._address, id, k, x, y, k_dev)
            if rc != _calls.ELSEWHERE:
                _check(self.h, rc)
                return y
        out = self.shapes.get(id, (1,))[0]   # an unknown id is reported by the library
        B = 1 if x.dim() == 1 else x.shape[0]
        if y is None:
            y = torch.empty((out,) if x.dim() == 1 else (B, out), dtype=torch.float16, device="cuda")
        self._need_workspace()
        _check(self.h, lib.dpllm_gemv(self.h, id, k, _ptr(k_dev), _ptr(x), _ptr(y), B, _stream()))
        return y

    def pointers(self, tensors):
        """The host array of n_linears device pointers the step calls take; build it once for tensors that stay
        where they are and pass it instead of the list (the caller keeps the tensors alive)."""
        if isinstance(tensors, C.Array):
            return tensors
        assert len(tensors) == self.n
        return (C.c_void_p * self.n)(*[t.data_ptr() for t in tensors])

    def dpllm_decode_step(self, xs, ys, k_out, e_out):
        self._need_workspace()
        _check(self.h, lib.dpllm_decode_step(self.h, self.pointers(xs), self.pointers(ys), _ptr(k_out), _ptr(e_out),
                                             _stream()))

    def dpllm_decode_step_parts(self, xs, ys, k_out, e_out, parts):
        self._need_workspace()
        _check(self.h, lib.dpllm_decode_step_parts(self.h, self.pointers(xs), self.pointers(ys), _ptr(k_out),
                                                   _ptr(e_out), parts, _stream()))

    def dpllm_debug_unpack(self, id, k):
        out, in_, _, _ = self.shapes.get(id, (1, 32, 0, 0))
        idx = torch.empty((out, in_), dtype=torch.uint8, device="cuda")
        _check(self.h, lib.dpllm_debug_unpack(self.h, id, k, _ptr(idx), _stream()))
        return idx

    def dpllm_debug_set_polls(self, polls):
        _check(self.h, lib.dpllm_debug_set_polls(self.h, polls))

    def dpllm_debug_set_one_launch(self, mode, seats=0):
        _check(self.h, lib.dpllm_debug_set_one_launch(self.h, mode, seats))

    def dpllm_debug_step_launches(self):
        n = C.c_int(0)
        _check(self.h, lib.dpllm_debug_step_launches(self.h, C.byref(n)))
        return n.value
