"""ctypes binding over ``libprunepath.so`` -- argument marshalling only.

Each function has the name and argument order of its C entry point in
``include/prunepath.h``; torch tensors are passed as raw device pointers and
streams as ``cudaStream_t`` handles (default: torch's current stream).  Every
step of the computation runs in the CUDA library; there is no Python or CPU
fallback: if the library is not built, ``load()`` raises.
"""
import ctypes
import os

from . import build as _build

PP_OK, PP_ERR_INVALID_ARG, PP_ERR_SHAPE, PP_ERR_DTYPE, PP_ERR_ALIGN = 0, 1, 2, 3, 4
PP_ERR_WORKSPACE, PP_ERR_CUDA, PP_ERR_TIMEOUT, PP_ERR_CAPACITY, PP_ERR_NONFINITE = 5, 6, 7, 8, 9
PP_ERR_UNSUPPORTED, PP_ERR_HOST = 10, 11
PP_F32, PP_BF16 = 0, 1
PP_ACT_RELU, PP_ACT_GELU_TANH, PP_ACT_SWIGLU = 0, 1, 2
PP_GATE_SIGMOID, PP_GATE_NONE = 0, 1
PP_SEL_MIN_PREFIX, PP_SEL_PAPER, PP_SEL_TOPK, PP_SEL_LTE = 0, 1, 2, 3

ACTS = {"relu": PP_ACT_RELU, "gelu_tanh": PP_ACT_GELU_TANH, "gelu": PP_ACT_GELU_TANH,
        "swiglu": PP_ACT_SWIGLU}
GATES = {"sigmoid": PP_GATE_SIGMOID, "none": PP_GATE_NONE}
RULES = {"min_prefix": PP_SEL_MIN_PREFIX, "paper": PP_SEL_PAPER, "topk": PP_SEL_TOPK, "lte": PP_SEL_LTE}
DTYPES = {"f32": PP_F32, "bf16": PP_BF16}
PP_ROPE_HALF, PP_ROPE_INTERLEAVED = 0, 1
PP_ROPE_NONE, PP_ROPE_LINEAR, PP_ROPE_NTK, PP_ROPE_BANDED, PP_ROPE_YARN = 0, 1, 2, 3, 4
ROPE_LAYOUTS = {"half": PP_ROPE_HALF, "interleaved": PP_ROPE_INTERLEAVED}
ROPE_SCALINGS = {"none": PP_ROPE_NONE, "linear": PP_ROPE_LINEAR, "ntk": PP_ROPE_NTK, "banded": PP_ROPE_BANDED,
                 "yarn": PP_ROPE_YARN}


class pp_desc(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int), ("d_ff", ctypes.c_int), ("n_experts", ctypes.c_int),
                ("d_expert", ctypes.c_int), ("dtype", ctypes.c_int), ("act", ctypes.c_int),
                ("gate", ctypes.c_int), ("rule", ctypes.c_int)]


class pp_selection(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("gates", ctypes.c_void_p),
                ("logits", ctypes.c_void_p)]


class pp_cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("n_heads", ctypes.c_int), ("n_kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("page_size", ctypes.c_int), ("n_pages", ctypes.c_int),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class pp_batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int), ("n_tokens", ctypes.c_int), ("max_pages", ctypes.c_int),
                ("q_start", ctypes.c_void_p), ("ctx_len", ctypes.c_void_p), ("pages", ctypes.c_void_p)]


class pp_rotation(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int), ("layout", ctypes.c_int), ("scale", ctypes.c_float),
                ("inv_freq", ctypes.c_void_p)]


class PPError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s failed: %s" % (what, status_name(status)))
        self.status = status


_lib = None
_P, _I, _F, _Z, _LL = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_longlong
_PD = ctypes.POINTER(pp_desc)
_PS = ctypes.POINTER(pp_selection)
_D = ctypes.c_double
_PC, _PB, _PR = ctypes.POINTER(pp_cache), ctypes.POINTER(pp_batch), ctypes.POINTER(pp_rotation)

EXPORTS = {
    "pp_workspace_size": (_Z, [_PD, _I]),
    "pp_workspace_init": (_I, [_P, _Z, _P]),
    "pp_route": (_I, [_PD, _P, _I, _P, _F, _PS, _P, _Z, _P]),
    "pp_select": (_I, [_PD, _P, _I, _F, _PS, _P, _Z, _P]),
    "pp_sparse_ffn": (_I, [_PD, _P, _I, _P, _P, _P, _PS, _P, _P, _Z, _P]),
    "pp_layer": (_I, [_PD, _P, _I, _P, _P, _P, _P, _F, _PS, _P, _P, _Z, _P]),
    "pp_layer_chained": (_I, [_PD, _P, _P, _P, _F, _I, _P, _P, _P, _P, _F, _PS, _P, _P, _P, _Z, _P]),
    "pp_layer_noalloc": (_I, [_PD, _P, _I, _P, _P, _P, _P, _F, _PS, _P, _P, _P]),
    "pp_sparsity_stats": (_I, [_P, _I, _I, _P, _P]),
    "pp_router_stats": (_I, [_PD, _P, _I, _F, _P, _P, _Z, _P]),
    "pp_moefy_cluster": (_I, [_PD, _P, _P, _P, _I, _P, _P, _P, _P]),
    "pp_moefy_permute": (_I, [_PD, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "pp_rope_frequencies": (_I, [_I, _I, _D, _D, _D, _D, _I, _P, _P]),
    "pp_rope": (_I, [_I, _PR, _P, _I, _I, _I, _P, _LL, _P, _LL, _I, _P]),
    "pp_attn_workspace_size": (_Z, [_PC]),
    "pp_kv_append": (_I, [_PC, _PB, _PR, _P, _P, _LL, _P, _LL, _P, _LL, _P, _LL, _P, _Z, _P]),
    "pp_tree_attention": (_I, [_PC, _PB, _P, _LL, _P, _I, _F, _P, _LL, _P, _Z, _P]),
    "pp_kv_commit": (_I, [_PC, _PB, _I, _LL, _P, _I, _P, _P, _P, _Z, _P]),
    "pp_get_device_status": (_I, [_P, _P]),
    "pp_debug_wait_timeout": (_I, [_P, _Z, _LL, _P]),
    "pp_debug_decode_timeline": (_I, [_PD, _P, _P, _P, _P, _P, _F, _P, _P, _Z, _P, _Z, _P]),
    "pp_status_string": (ctypes.c_char_p, [_I]),
    "pp_version": (ctypes.c_char_p, []),
}


def library_path() -> str:
    return _build.LIB


def load(path: str = None):
    """Load libprunepath.so (raises if it has not been built)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or library_path()
    if not os.path.exists(path):
        raise RuntimeError("libprunepath.so is not built (%s); run __graft_entry__.build()" % path)
    lib = ctypes.CDLL(path)
    for name, (res, args) in EXPORTS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_name(s: int) -> str:
    try:
        return load().pp_status_string(int(s)).decode()
    except RuntimeError:
        return "status %d" % s


def _check(s, what):
    if s != PP_OK:
        raise PPError(s, what)


def _ptr(t):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


_raw_stream = None


def _current_stream() -> int:
    """Handle of torch's current stream on the current device.  torch.cuda.current_stream() builds a Stream object in
    about 3 us, half of a small call; the raw handle takes a tenth of a microsecond."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        if get is not None and dev is not None:
            _raw_stream = lambda: get(dev())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream()


def _stream(stream):
    if stream is None:
        return ctypes.c_void_p(_current_stream())
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def make_desc(d_model, n_experts, dtype="bf16", act="swiglu", gate="sigmoid", rule="min_prefix",
              d_expert=64) -> pp_desc:
    return pp_desc(int(d_model), int(n_experts) * int(d_expert), int(n_experts), int(d_expert),
                   DTYPES.get(dtype, dtype), ACTS.get(act, act), GATES.get(gate, gate),
                   RULES.get(rule, rule))


class Selection:
    """Device tensors of a selection: ids/gates [T, E], counts [T], logits [T, E] or None."""

    def __init__(self, ids, counts, gates, logits=None):
        self.ids, self.counts, self.gates, self.logits = ids, counts, gates, logits

    @classmethod
    def empty(cls, T, E, device, with_logits=True):
        import torch
        return cls(torch.empty((T, E), dtype=torch.int32, device=device),
                   torch.empty((T,), dtype=torch.int32, device=device),
                   torch.empty((T, E), dtype=torch.float32, device=device),
                   torch.empty((T, E), dtype=torch.float32, device=device) if with_logits else None)

    def c(self) -> pp_selection:
        return pp_selection(self.ids.data_ptr(), self.counts.data_ptr(), self.gates.data_ptr(),
                            None if self.logits is None else self.logits.data_ptr())


def pp_workspace_size(desc, T) -> int:
    return int(load().pp_workspace_size(ctypes.byref(desc), int(T)))


def pp_workspace_init(ws, stream=None):
    _check(load().pp_workspace_init(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "pp_workspace_init")


def alloc_workspace(desc, T, device="cuda", stream=None):
    """A zero-initialised workspace tensor for calls with up to T tokens."""
    import torch
    ws = torch.empty(max(256, pp_workspace_size(desc, T)), dtype=torch.uint8, device=device)
    pp_workspace_init(ws, stream)
    return ws


def _wsargs(ws):
    return _ptr(ws), ws.numel() * ws.element_size()


def pp_route(desc, x, T, W_r, p, out, ws, stream=None):
    sel = out.c()
    _check(load().pp_route(ctypes.byref(desc), _ptr(x), int(T), _ptr(W_r), float(p), ctypes.byref(sel),
                           *_wsargs(ws), _stream(stream)), "pp_route")


def pp_select(desc, logits, T, p, out, ws, stream=None):
    sel = out.c()
    _check(load().pp_select(ctypes.byref(desc), _ptr(logits), int(T), float(p), ctypes.byref(sel),
                            *_wsargs(ws), _stream(stream)), "pp_select")


def pp_sparse_ffn(desc, x, T, W_gate, W_up, W_down, sel, y, ws, stream=None):
    s = sel.c()
    _check(load().pp_sparse_ffn(ctypes.byref(desc), _ptr(x), int(T), _ptr(W_gate), _ptr(W_up),
                                _ptr(W_down), ctypes.byref(s), _ptr(y), *_wsargs(ws), _stream(stream)),
           "pp_sparse_ffn")


def pp_layer(desc, x, T, W_r, W_gate, W_up, W_down, p, sel_out, y, ws, stream=None):
    s = None if sel_out is None else sel_out.c()
    _check(load().pp_layer(ctypes.byref(desc), _ptr(x), int(T), _ptr(W_r), _ptr(W_gate), _ptr(W_up),
                           _ptr(W_down), float(p), None if s is None else ctypes.byref(s), _ptr(y),
                           *_wsargs(ws), _stream(stream)), "pp_layer")


def pp_layer_chained(desc, x_prev, y_prev, gamma, eps, T, W_r, W_gate, W_up, W_down, p, sel_out, x, y, ws,
                     stream=None):
    """x = RMSNorm(x_prev + y_prev) * gamma, then y = pp_layer(x) (y_prev, gamma may be None)."""
    s = None if sel_out is None else sel_out.c()
    _check(load().pp_layer_chained(ctypes.byref(desc), _ptr(x_prev), _ptr(y_prev), _ptr(gamma), float(eps), int(T),
                                   _ptr(W_r), _ptr(W_gate), _ptr(W_up), _ptr(W_down), float(p),
                                   None if s is None else ctypes.byref(s), _ptr(x), _ptr(y), *_wsargs(ws),
                                   _stream(stream)), "pp_layer_chained")


def pp_layer_noalloc(desc, x, T, W_r, W_gate, W_up, W_down, p, sel_out, y, status_out=None, stream=None):
    """pp_layer without a workspace (library-owned static scratch, T <= 4)."""
    s = None if sel_out is None else sel_out.c()
    _check(load().pp_layer_noalloc(ctypes.byref(desc), _ptr(x), int(T), _ptr(W_r), _ptr(W_gate), _ptr(W_up),
                                   _ptr(W_down), float(p), None if s is None else ctypes.byref(s), _ptr(y),
                                   _ptr(status_out), _stream(stream)), "pp_layer_noalloc")


def pp_sparsity_stats(counts, T, n_experts, acc, stream=None):
    _check(load().pp_sparsity_stats(_ptr(counts), int(T), int(n_experts), _ptr(acc), _stream(stream)),
           "pp_sparsity_stats")


def pp_router_stats(desc, logits, T, eps, out, ws, stream=None):
    """L_ent, L_bal, L_gate of the logits [T][E] into out (3 float64, device)."""
    _check(load().pp_router_stats(ctypes.byref(desc), _ptr(logits), int(T), float(eps), _ptr(out),
                                  *_wsargs(ws), _stream(stream)), "pp_router_stats")


def _host(a):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def pp_moefy_cluster(desc, W_gate, W_up, init, max_iter=100):
    """Balanced k-means of the neurons (host numpy arrays: float32, or uint16
    bf16 bit patterns; init int32 [E]).  Returns (perm, labels, iters,
    objective)."""
    import numpy as np
    W_up = np.ascontiguousarray(W_up)
    W_gate = None if W_gate is None else np.ascontiguousarray(W_gate)
    init = np.ascontiguousarray(init, dtype=np.int32)
    perm = np.empty(desc.d_ff, np.int32)
    labels = np.empty(desc.d_ff, np.int32)
    iters = ctypes.c_int(0)
    obj = ctypes.c_double(0.0)
    _check(load().pp_moefy_cluster(ctypes.byref(desc), _host(W_gate), _host(W_up), _host(init), int(max_iter),
                                   _host(perm), _host(labels), ctypes.byref(iters), ctypes.byref(obj)),
           "pp_moefy_cluster")
    return perm, labels, iters.value, obj.value


def pp_moefy_permute(desc, perm, W_gate, W_up, W_down, W_gate_out, W_up_out, W_down_out, ws, stream=None):
    """Eq. (permuted_weights) on the device: *_out = the weights with neuron j = old neuron perm[j]."""
    _check(load().pp_moefy_permute(ctypes.byref(desc), _ptr(perm), _ptr(W_gate), _ptr(W_up), _ptr(W_down),
                                   _ptr(W_gate_out), _ptr(W_up_out), _ptr(W_down_out), *_wsargs(ws),
                                   _stream(stream)), "pp_moefy_permute")


_INT32 = None
_TORCH_DTYPES = {}


def _torch_types():
    """torch's types, once (importing this module does not import torch)."""
    global _INT32
    if _INT32 is None:
        import torch
        _TORCH_DTYPES.update({torch.bfloat16: PP_BF16, torch.float32: PP_F32})
        _INT32 = torch.int32


def _torch_dtype(dtype) -> int:
    """pp_dtype of a torch dtype (PP_ERR_DTYPE for any other)."""
    d = _TORCH_DTYPES.get(dtype)
    if d is None:
        raise PPError(PP_ERR_DTYPE, "dtype %s" % dtype)
    return d


def _rows(t, n_tokens, n_heads, head_dim, dtype, what):
    """Pointer and token stride of a token tensor [n_tokens, heads, head_dim] (or [n_tokens, heads * head_dim])
    whose tokens are each contiguous."""
    shape, stride = t.shape, t.stride()
    if t.dtype == dtype and shape == (n_tokens, n_heads, head_dim) and stride[1:] == (head_dim, 1):
        return t.data_ptr(), (stride[0] if n_tokens > 1 else n_heads * head_dim)
    if t.dtype != dtype:
        raise PPError(PP_ERR_DTYPE, what)
    if shape != (n_tokens, n_heads, head_dim) and shape != (n_tokens, n_heads * head_dim):
        raise PPError(PP_ERR_SHAPE, what)
    if (head_dim > 1 and stride[-1] != 1) or (len(shape) == 3 and n_heads > 1 and stride[1] != head_dim):
        raise PPError(PP_ERR_INVALID_ARG, what + ": the heads of a token must be contiguous")
    return t.data_ptr(), (stride[0] if n_tokens > 1 else n_heads * head_dim)


def _int32(t, what):
    if t.dtype is not _INT32:
        raise PPError(PP_ERR_DTYPE, what + " must be int32")
    if not t.is_contiguous():
        raise PPError(PP_ERR_INVALID_ARG, what + " must be contiguous")
    return t.data_ptr()


def _stream_handle(stream) -> int:
    if stream is None:
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


class Rotation:
    """Rotary positions: inv_freq (device, float32, one entry a rotated pair), layout, attention factor."""

    def __init__(self, inv_freq, layout="half", scale=1.0):
        import torch
        _torch_types()
        if inv_freq.dtype != torch.float32 or not inv_freq.is_contiguous():
            raise PPError(PP_ERR_DTYPE, "inv_freq must be contiguous float32")
        self.inv_freq = inv_freq
        self.c = pp_rotation(2 * inv_freq.numel(), ROPE_LAYOUTS.get(layout, layout), float(scale),
                             inv_freq.data_ptr())
        self.ref = ctypes.byref(self.c)

    @classmethod
    def make(cls, rot_dim, base=10000.0, layout="half", scaling="none", factor=1.0, low=1.0, high=32.0,
             trained_len=0, device="cuda"):
        """Frequencies from pp_rope_frequencies, on the device, with the scaling's attention factor."""
        import torch
        freq, scale = pp_rope_frequencies(scaling, rot_dim, base, factor, low, high, trained_len)
        return cls(torch.from_numpy(freq).to(device), layout, scale)


class KVCache:
    """A layer's key and value pages: k, v [n_pages, page_size, n_kv_heads, head_dim] of any strides (the same for
    both) with contiguous head_dim.  Pages stored head by head are passed as their transposed view."""

    def __init__(self, k, v, n_heads):
        _torch_types()
        if k.dim() != 4 or k.shape != v.shape:
            raise PPError(PP_ERR_SHAPE, "KVCache")
        if k.dtype != v.dtype:
            raise PPError(PP_ERR_DTYPE, "KVCache")
        if k.stride() != v.stride() or k.stride(3) != 1:
            raise PPError(PP_ERR_INVALID_ARG, "KVCache: strides")
        self.k, self.v = k, v
        self.c = pp_cache(_torch_dtype(k.dtype), int(n_heads), k.shape[2], k.shape[3], k.shape[1], k.shape[0], k.stride(0),
                          k.stride(1), k.stride(2), k.data_ptr(), v.data_ptr())
        self.ref = ctypes.byref(self.c)
        # what the calls compare their tensors with
        self.dtype, self.n_heads, self.n_kv_heads, self.head_dim = k.dtype, int(n_heads), k.shape[2], k.shape[3]


class Batch:
    """The sequences of a step: q_start [n_seqs + 1], ctx_len [n_seqs], pages [n_seqs, max_pages] (device, int32)."""

    def __init__(self, q_start, ctx_len, pages, n_tokens):
        _torch_types()
        n = ctx_len.numel()
        if q_start.numel() != n + 1 or pages.dim() != 2 or pages.shape[0] != n:
            raise PPError(PP_ERR_SHAPE, "Batch")
        self.q_start, self.ctx_len, self.pages = q_start, ctx_len, pages
        self.c = pp_batch(n, int(n_tokens), pages.shape[1], _int32(q_start, "q_start"), _int32(ctx_len, "ctx_len"),
                          _int32(pages, "pages"))
        self.ref, self.n_tokens, self.n_seqs = ctypes.byref(self.c), int(n_tokens), n


def pp_rope_frequencies(scaling, rot_dim, base=10000.0, factor=1.0, low=1.0, high=32.0, trained_len=0):
    """(inv_freq, a numpy float32 array of rot_dim / 2; attention factor)."""
    import numpy as np
    freq = np.empty(max(0, int(rot_dim)) // 2, np.float32)
    scale = ctypes.c_float(0.0)
    _check(load().pp_rope_frequencies(ROPE_SCALINGS.get(scaling, scaling), int(rot_dim), float(base), float(factor),
                                      float(low), float(high), int(trained_len), _host(freq), ctypes.byref(scale)),
           "pp_rope_frequencies")
    return freq, scale.value


def pp_rope(rot, positions, x, y, inverse=False, stream=None):
    """y = x [T, heads, head_dim] rotated by positions [T] (back, with inverse: the gradient); y may be x."""
    shape = x.shape
    if len(shape) != 3:
        raise PPError(PP_ERR_SHAPE, "pp_rope: x")
    T, H, D = shape
    if positions.numel() != T:
        raise PPError(PP_ERR_SHAPE, "pp_rope: positions")
    dt = x.dtype
    px, sx = _rows(x, T, H, D, dt, "pp_rope: x")
    py, sy = _rows(y, T, H, D, dt, "pp_rope: y")
    _check(load().pp_rope(_torch_dtype(dt), rot.ref, _int32(positions, "positions"), T, H, D, px, sx, py, sy,
                          1 if inverse else 0, _stream_handle(stream)), "pp_rope")


def pp_attn_workspace_size(cache) -> int:
    return int(load().pp_attn_workspace_size(cache.ref))


def alloc_attn_workspace(cache, device=None, stream=None):
    """A zero-initialised workspace tensor for the calls on caches of this shape."""
    import torch
    ws = torch.empty(max(256, pp_attn_workspace_size(cache)), dtype=torch.uint8, device=device or cache.k.device)
    pp_workspace_init(ws, stream)
    return ws


def pp_kv_append(cache, batch, rot, positions, q, k, v, q_out, ws, stream=None):
    """Append k, v [T, n_kv_heads, head_dim] to their pages, keys rotated; q_out = q rotated (both may be None)."""
    T, D, dt = batch.n_tokens, cache.head_dim, cache.dtype
    pq, sq, po, so = None, 0, None, 0
    if q is not None:
        pq, sq = _rows(q, T, cache.n_heads, D, dt, "pp_kv_append: q")
    if q_out is not None:
        po, so = _rows(q_out, T, cache.n_heads, D, dt, "pp_kv_append: q_out")
    pk, sk = _rows(k, T, cache.n_kv_heads, D, dt, "pp_kv_append: k")
    pv, sv = _rows(v, T, cache.n_kv_heads, D, dt, "pp_kv_append: v")
    pos = None
    if positions is not None:
        if positions.numel() != T:
            raise PPError(PP_ERR_SHAPE, "pp_kv_append: positions")
        pos = _int32(positions, "positions")
    _check(load().pp_kv_append(cache.ref, batch.ref, None if rot is None else rot.ref, pos, pq, sq, pk, sk, pv, sv, po,
                               so, ws.data_ptr(), ws.nbytes, _stream_handle(stream)), "pp_kv_append")


def pp_tree_attention(cache, batch, q, mask, scale, out, ws, stream=None):
    """out = attention of q [T, n_heads, head_dim] over the cache; mask [T, words] int32 bits, or None (chains)."""
    T, D, dt = batch.n_tokens, cache.head_dim, cache.dtype
    pq, sq = _rows(q, T, cache.n_heads, D, dt, "pp_tree_attention: q")
    po, so = _rows(out, T, cache.n_heads, D, dt, "pp_tree_attention: out")
    pm, words = None, 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[0] != T:
            raise PPError(PP_ERR_SHAPE, "pp_tree_attention: mask")
        pm, words = _int32(mask, "mask"), mask.shape[1]
    _check(load().pp_tree_attention(cache.ref, batch.ref, pq, sq, pm, words, scale, po, so, ws.data_ptr(), ws.nbytes,
                                    _stream_handle(stream)), "pp_tree_attention")


def pp_kv_commit(cache, batch, path, n_accept, ws, new_len=None, n_layers=1, layer_stride=0, stream=None):
    """Move the accepted path [n_seqs, max_path] of each tree behind its context, in every layer's cache (layer_stride:
    elements from one layer's pages to the next one's, for more than one layer)."""
    n = batch.n_seqs
    if path.dim() != 2 or path.shape[0] != n or n_accept.numel() != n or \
            (new_len is not None and new_len.numel() != n):
        raise PPError(PP_ERR_SHAPE, "pp_kv_commit")
    _check(load().pp_kv_commit(cache.ref, batch.ref, n_layers, layer_stride, _int32(path, "path"), path.shape[1],
                               _int32(n_accept, "n_accept"), None if new_len is None else _int32(new_len, "new_len"),
                               ws.data_ptr(), ws.nbytes, _stream_handle(stream)), "pp_kv_commit")


def pp_get_device_status(ws, stream=None) -> int:
    return int(load().pp_get_device_status(_ptr(ws), _stream(stream)))


def pp_debug_decode_timeline(desc, x, W_r, W_gate, W_up, W_down, p, y, ws, stamps, stream=None):
    """stamps: a device uint64 tensor of at least 256 * 16 entries."""
    _check(load().pp_debug_decode_timeline(ctypes.byref(desc), _ptr(x), _ptr(W_r), _ptr(W_gate), _ptr(W_up),
                                           _ptr(W_down), float(p), _ptr(y), *_wsargs(ws), _ptr(stamps),
                                           stamps.numel() * stamps.element_size(), _stream(stream)),
           "pp_debug_decode_timeline")


def pp_debug_wait_timeout(ws, timeout_ns, stream=None):
    _check(load().pp_debug_wait_timeout(*_wsargs(ws), int(timeout_ns), _stream(stream)),
           "pp_debug_wait_timeout")


def pp_status_string(s) -> str:
    return load().pp_status_string(int(s)).decode()


def pp_version() -> str:
    return load().pp_version().decode()
