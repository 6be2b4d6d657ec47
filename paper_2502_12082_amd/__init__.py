"""alpha-entmax flash attention for MI355X (gfx950): Python binding.

Argument marshalling over the C ABI declared in include/entmax_attn.h; every
step of the computation runs in the HIP kernels of libentmax_attn.so.  torch
is used only to own device memory and to name the stream.  There is no CPU
fallback: importing this module without the built library raises.

    import paper_2502_12082_amd as ea
    o, res = ea.forward(q, k, v, alpha=1.5, scale=d ** -0.5, causal=False)
    dq, dk, dv = ea.backward(q, k, v, do, res)

A transformer's layer on tokens packed from several sequences, with grouped
heads ([tokens, heads, d] tensors, such as parts of a fused projection's rows):

    plan = ea.packed_plan(cu_seqlens, tokens)                  # once a batch
    q, k = ea.norm_rotary(q, k, positions, freqs, q_weight, k_weight)
    o, res = ea.packed_forward(q, k, v, plan, alpha=1.5)
    dq, dk, dv = ea.packed_backward(q, k, v, do, res)
    dq, dk, dwq, dwk = ea.norm_rotary_backward(dq, dk, q_in, k_in, positions, freqs, q_weight, k_weight)

and one decoding step, for requests that share a prefix:

    o = ea.prefix_decode(q, k_cache, v_cache, lengths, k_prefix, v_prefix)

or with keys and values in pages and in 4 bits, for all layers of a step:

    cache = ea.paged_cache(pages, page_size, kv_heads, head_dim, layers)
    table, lengths, missing = ea.cache_update(cache, table, lengths, parents, counts)
    ea.cache_append(cache[layer], k, v, rows, positions, table)
    o = ea.paged_decode(q, cache[layer], table, lengths)
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libentmax_attn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError("libentmax_attn.so is not built; run `python paper_2502_12082_amd/build.py` "
                      "(or __graft_entry__.build()) first")

# torch ships its own HIP and HSA runtimes.  Importing it first lets the
# library's libamdhip64.so.7 dependency resolve to the copy torch already
# loaded; loaded the other way round the process holds two runtimes, and
# launches through the second one find no device.
import torch  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)

EA_OK, EA_ERR_INVALID_ARG, EA_ERR_UNSUPPORTED, EA_ERR_WORKSPACE, EA_ERR_HIP = range(5)
EA_BF16, EA_F32 = 0, 1
SYMBOLS = ("entmax_attn_default_params", "entmax_attn_sizes", "entmax_attn_fwd",
           "entmax_attn_bwd", "entmax_attn_fwd_stage", "entmax_attn_bwd_stage",
           "entmax_attn_status_string", "entmax_attn_last_hip_error", "entmax_rows_fwd",
           "entmax_rows_bwd", "entmax_attn_fwd_dense", "entmax_attn_bwd_dense",
           "entmax_attn_bwd_noalloc", "entmax_attn_lists_bytes", "entmax_attn_fwd_lists",
           "entmax_attn_bwd_lists", "entmax_attn_fwd_dense_lists", "entmax_attn_bwd_dense_lists",
           "entmax_attn_bwd_lists_workspace", "entmax_norm_rotary", "entmax_norm_rotary_workspace",
           "entmax_norm_rotary_bwd", "entmax_packed_plan_bytes", "entmax_packed_plan",
           "entmax_packed_sizes", "entmax_packed_fwd", "entmax_packed_bwd",
           "entmax_prefix_decode_workspace", "entmax_prefix_decode", "entmax_cache_page_bytes",
           "entmax_cache_append", "entmax_cache_read", "entmax_cache_workspace", "entmax_cache_update",
           "entmax_cache_compact", "entmax_paged_decode_workspace", "entmax_paged_decode")
EA_ALL_STAGES = -1
MAX_SEQLEN = 131072  # the longest sequence of every attention call
NOALLOC_MAX_ROWS = 1048576  # EA_NOALLOC_MAX_ROWS of include/entmax_attn.h


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("seqlen", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class Params(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("scale", ctypes.c_float),
                ("causal", ctypes.c_int32), ("max_iter", ctypes.c_int32),
                ("tol", ctypes.c_float), ("need_bwd", ctypes.c_int32)]


class ResidualPtrs(ctypes.Structure):
    """The ABI's ea_residuals.  `lists` and `lists_bytes`, set by
    Residuals.ptrs(), name the element lists that belong to them, and `owner`
    the Residuals itself; the calls below then pass those on."""
    lists, lists_bytes, lists_shape, owner = None, 0, None, None
    _fields_ = [(f, ctypes.c_void_p) for f in
                ("tau", "o2", "block_mask", "q_count", "q_index", "k_count", "k_index", "stats",
                 "tau_lo")]


class Sizes(ctypes.Structure):
    _fields_ = [(f, ctypes.c_size_t) for f in
                ("tau", "o2", "block_mask", "q_count", "q_index", "k_count", "k_index", "stats",
                 "ws_fwd", "ws_bwd", "tau_lo")]


_P = ctypes.POINTER
_v = ctypes.c_void_p
_lib.entmax_attn_default_params.argtypes = [_P(Params)]
_lib.entmax_attn_default_params.restype = None
_lib.entmax_attn_sizes.argtypes = [_P(Shape), _P(Params), _P(Sizes)]
_lib.entmax_attn_sizes.restype = ctypes.c_int
_lib.entmax_attn_fwd.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _P(ResidualPtrs), _v,
                                 ctypes.c_size_t, _v]
_lib.entmax_attn_fwd.restype = ctypes.c_int
_lib.entmax_attn_bwd.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _P(ResidualPtrs), _v, _v,
                                 _v, _v, ctypes.c_size_t, _v]
_lib.entmax_attn_bwd.restype = ctypes.c_int
_lib.entmax_attn_fwd_stage.argtypes = [ctypes.c_int, _P(Shape), _P(Params), _v, _v, _v, _v,
                                       _P(ResidualPtrs), _v, ctypes.c_size_t, _v]
_lib.entmax_attn_fwd_stage.restype = ctypes.c_int
_lib.entmax_attn_bwd_stage.argtypes = [ctypes.c_int, _P(Shape), _P(Params), _v, _v, _v, _v,
                                       _P(ResidualPtrs), _v, _v, _v, _v, ctypes.c_size_t, _v]
_lib.entmax_attn_bwd_stage.restype = ctypes.c_int
_lib.entmax_attn_status_string.argtypes = [ctypes.c_int]
_lib.entmax_attn_status_string.restype = ctypes.c_char_p
_lib.entmax_attn_fwd_dense.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _v, _v, _v, _v,
                                       ctypes.c_size_t, _v]
_lib.entmax_attn_fwd_dense.restype = ctypes.c_int
_lib.entmax_attn_bwd_dense.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _v, _v, _v, _v, _v,
                                       _v, _v, ctypes.c_size_t, _v]
_lib.entmax_attn_bwd_dense.restype = ctypes.c_int
_lib.entmax_rows_fwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int, _P(Params), _v, _v,
                                 _v, _v]
_lib.entmax_rows_fwd.restype = ctypes.c_int
_lib.entmax_rows_bwd.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int, _P(Params), _v, _v,
                                 _v, _v, _v]
_lib.entmax_rows_bwd.restype = ctypes.c_int
_lib.entmax_attn_bwd_noalloc.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _P(ResidualPtrs),
                                         _v, _v, _v, _v]
_lib.entmax_attn_bwd_noalloc.restype = ctypes.c_int
_lib.entmax_attn_fwd_dense_lists.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _v, _v, _v, _v,
                                             ctypes.c_size_t, _v, ctypes.c_size_t, _v]
_lib.entmax_attn_fwd_dense_lists.restype = ctypes.c_int
_lib.entmax_attn_bwd_dense_lists.argtypes = [_P(Shape), _P(Params), _v, _v, _v, _v, _v, _v, _v, _v,
                                             ctypes.c_size_t, _v, _v, _v, _v, ctypes.c_size_t, _v]
_lib.entmax_attn_bwd_dense_lists.restype = ctypes.c_int
_lib.entmax_attn_lists_bytes.argtypes = [_P(Shape), _P(Params), _P(ctypes.c_size_t)]
_lib.entmax_attn_lists_bytes.restype = ctypes.c_int
_lib.entmax_attn_bwd_lists_workspace.argtypes = [_P(Shape), _P(Params), _P(ctypes.c_size_t)]
_lib.entmax_attn_bwd_lists_workspace.restype = ctypes.c_int
_lib.entmax_attn_fwd_lists.argtypes = [ctypes.c_int, _P(Shape), _P(Params), _v, _v, _v, _v,
                                       _P(ResidualPtrs), _v, ctypes.c_size_t, _v, ctypes.c_size_t,
                                       _v]
_lib.entmax_attn_fwd_lists.restype = ctypes.c_int
_lib.entmax_attn_bwd_lists.argtypes = [ctypes.c_int, _P(Shape), _P(Params), _v, _v, _v, _v,
                                       _P(ResidualPtrs), _v, ctypes.c_size_t, _v, _v, _v, _v,
                                       ctypes.c_size_t, _v]
_lib.entmax_attn_bwd_lists.restype = ctypes.c_int
_lib.entmax_attn_last_hip_error.argtypes = []
_lib.entmax_attn_last_hip_error.restype = ctypes.c_char_p


class EntmaxAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = "%s: %s (status %d)" % (
            where, _lib.entmax_attn_status_string(status).decode(), status)
        if status == EA_ERR_HIP:
            msg += ": " + _lib.entmax_attn_last_hip_error().decode()
        super().__init__(msg)


def _check(status: int, where: str):
    if status != EA_OK:
        raise EntmaxAttnError(status, where)


# --------------------------------------------------------- raw C ABI calls

def default_params() -> Params:
    p = Params()
    _lib.entmax_attn_default_params(ctypes.byref(p))
    return p


def entmax_attn_sizes(shape: Shape, params: Params) -> Sizes:
    z = Sizes()
    _check(_lib.entmax_attn_sizes(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(z)),
           "entmax_attn_sizes")
    return z


def entmax_attn_lists_bytes(shape: Shape, params: Params) -> int:
    n = ctypes.c_size_t()
    _check(_lib.entmax_attn_lists_bytes(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(n)),
           "entmax_attn_lists_bytes")
    return n.value


def entmax_attn_bwd_lists_workspace(shape: Shape, params: Params) -> int:
    n = ctypes.c_size_t()
    _check(_lib.entmax_attn_bwd_lists_workspace(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(n)),
           "entmax_attn_bwd_lists_workspace")
    return n.value


def _dims(shape):
    return shape.batch, shape.heads, shape.seqlen, shape.head_dim


def _lists_of(res: ResidualPtrs, shape, params):
    """The lists of res, as (pointer, bytes), if they serve this shape."""
    if res.lists is None:
        return None, 0
    if res.lists_shape == _dims(shape):
        return res.lists, res.lists_bytes
    n = ctypes.c_size_t()
    st = _lib.entmax_attn_lists_bytes(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(n))
    return (res.lists, res.lists_bytes) if st == EA_OK and 0 < n.value <= res.lists_bytes else (None, 0)


def entmax_attn_fwd_lists(stage, shape, params, q, k, v, o, res: ResidualPtrs, lists, lists_bytes,
                          workspace, ws_bytes, stream):
    """Raw call; pointers are ints (device addresses), stream an int handle."""
    return _lib.entmax_attn_fwd_lists(stage, ctypes.byref(shape), ctypes.byref(params), q, k, v, o,
                                      ctypes.byref(res), lists, lists_bytes, workspace, ws_bytes,
                                      stream)


def entmax_attn_bwd_lists(stage, shape, params, q, k, v, dout, res: ResidualPtrs, lists,
                          lists_bytes, dq, dk, dv, workspace, ws_bytes, stream):
    return _lib.entmax_attn_bwd_lists(stage, ctypes.byref(shape), ctypes.byref(params), q, k, v,
                                      dout, ctypes.byref(res), lists, lists_bytes, dq, dk, dv,
                                      workspace, ws_bytes, stream)


def entmax_attn_fwd(shape, params, q, k, v, o, res: ResidualPtrs, workspace, ws_bytes, stream):
    lists = _lists_of(res, shape, params)
    if lists[0]:
        return entmax_attn_fwd_lists(EA_ALL_STAGES, shape, params, q, k, v, o, res, *lists, workspace,
                                     ws_bytes, stream)
    return _lib.entmax_attn_fwd(ctypes.byref(shape), ctypes.byref(params), q, k, v, o,
                                ctypes.byref(res), workspace, ws_bytes, stream)


def entmax_attn_bwd(shape, params, q, k, v, dout, res: ResidualPtrs, dq, dk, dv, workspace,
                    ws_bytes, stream):
    lists = _lists_of(res, shape, params)
    if lists[0] and workspace:
        return entmax_attn_bwd_lists(EA_ALL_STAGES, shape, params, q, k, v, dout, res, *lists, dq, dk,
                                     dv, workspace, ws_bytes, stream)
    return _lib.entmax_attn_bwd(ctypes.byref(shape), ctypes.byref(params), q, k, v, dout,
                                ctypes.byref(res), dq, dk, dv, workspace, ws_bytes, stream)


def entmax_attn_bwd_noalloc(shape, params, q, k, v, dout, res: ResidualPtrs, dq, dk, dv, stream):
    """As the C function.  The lists of a Residuals are sorted in a buffer that
    it holds (Residuals.keep_workspace; the first call makes it unless the
    stream is being captured, and without it the lists are not used)."""
    lists = _lists_of(res, shape, params)
    rows = shape.batch * shape.heads * shape.seqlen
    if lists[0] and res.owner is not None and rows <= NOALLOC_MAX_ROWS:
        ws = res.owner.keep_workspace(make=not torch.cuda.is_current_stream_capturing())
        if ws is not None and ws.numel() >= entmax_attn_bwd_lists_workspace(shape, params):
            return entmax_attn_bwd_lists(EA_ALL_STAGES, shape, params, q, k, v, dout, res, *lists, dq,
                                         dk, dv, ws.data_ptr(), ws.numel(), stream)
    return _lib.entmax_attn_bwd_noalloc(ctypes.byref(shape), ctypes.byref(params), q, k, v, dout,
                                        ctypes.byref(res), dq, dk, dv, stream)


def entmax_attn_fwd_stage(stage, shape, params, q, k, v, o, res: ResidualPtrs, workspace,
                          ws_bytes, stream):
    lists = _lists_of(res, shape, params)
    if lists[0] and stage >= 0:
        return entmax_attn_fwd_lists(stage, shape, params, q, k, v, o, res, *lists, workspace,
                                     ws_bytes, stream)
    return _lib.entmax_attn_fwd_stage(stage, ctypes.byref(shape), ctypes.byref(params), q, k, v,
                                      o, ctypes.byref(res), workspace, ws_bytes, stream)


def entmax_attn_bwd_stage(stage, shape, params, q, k, v, dout, res: ResidualPtrs, dq, dk, dv,
                          workspace, ws_bytes, stream):
    lists = _lists_of(res, shape, params)
    if lists[0] and stage >= 0:
        return entmax_attn_bwd_lists(stage, shape, params, q, k, v, dout, res, *lists, dq, dk, dv,
                                     workspace, ws_bytes, stream)
    return _lib.entmax_attn_bwd_stage(stage, ctypes.byref(shape), ctypes.byref(params), q, k, v,
                                      dout, ctypes.byref(res), dq, dk, dv, workspace, ws_bytes,
                                      stream)


# ------------------------------------------------------ torch conveniences

def make_shape(q) -> Shape:
    if q.dim() != 4:
        raise ValueError("expected [batch, heads, seqlen, head_dim]")
    if q.dtype == torch.bfloat16:
        dt = EA_BF16
    elif q.dtype == torch.float32:
        dt = EA_F32
    else:
        raise ValueError("dtype must be bfloat16 or float32")
    B, H, n, d = q.shape
    return Shape(B, H, n, d, dt)


def make_params(alpha=1.5, scale=None, causal=False, need_bwd=True, max_iter=None, tol=None,
                head_dim=64) -> Params:
    p = default_params()
    p.alpha = float(alpha)
    p.scale = float(scale if scale is not None else head_dim ** -0.5)
    p.causal = int(bool(causal))
    p.need_bwd = int(bool(need_bwd))
    if max_iter is not None:
        p.max_iter = int(max_iter)
    if tol is not None:
        p.tol = float(tol)
    return p


_memory = {}  # total memory of each device, a constant of the device
_held = {}    # bytes of the element lists that live Residuals hold on each device
_held_lock = threading.RLock()


def _lists_limit(device) -> int:
    """The most that the element lists of all Residuals of a device take
    together: a sixteenth of its memory."""
    if device.type != "cuda":
        return 1 << 30
    if device.index not in _memory:
        _memory[device.index] = torch.cuda.get_device_properties(device).total_memory
    return _memory[device.index] // 16


class _Claim:
    """`nbytes` of a device's share for element lists, given back when this
    object goes.  Saved and copied objects hold none."""

    def __init__(self, index, nbytes):
        self.index, self.nbytes = index, nbytes

    def __del__(self, lock=_held_lock, held=_held):  # (module globals may be gone at exit)
        with lock:
            held[self.index] -= self.nbytes

    def __reduce__(self):
        return type(None), ()


def _claim(device, nbytes):
    """A _Claim, or None where the limit would be passed."""
    limit = _lists_limit(device)
    with _held_lock:
        if _held.get(device.index, 0) + nbytes > limit:
            return None
        _held[device.index] = _held.get(device.index, 0) + nbytes
    return _Claim(device.index, nbytes)


def _lists_size(shape, params, least) -> int:
    """Bytes of the element lists, or 0: from `least` keys on (a quarter of
    that for fp32, whose products take longer), since the sort and the list
    kernel of the backward are launches of their own, and few blocks of a short
    sequence are listed."""
    if shape.seqlen <= (least if shape.dtype == EA_BF16 else least // 4):
        return 0
    return entmax_attn_lists_bytes(shape, params)


def _bytes_or_none(nbytes, device):
    try:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    except torch.OutOfMemoryError:
        return None


# Measured, in us, with lists against without: B64 H16 n128 d64 alpha 1.5
# c = 1 150 against 140 (no block listed), B1 H1 n256 fp32 inference 26 against
# 38; the no-mask mode collects its lists in a K pass more: B1 H2 n128 56
# against 44, B1 H16 n4096 d128 670 against 1040.
LISTS_FROM, DENSE_LISTS_FROM = 256, 1024


class Residuals:
    """Device buffers (torch tensors) that the forward fills and the backward
    reads, sized by entmax_attn_sizes: tau, o2, tau_lo (fp32 inputs: the low
    part of tau), lists (the element lists, see entmax_attn_fwd_lists; 582 bytes
    a row, which the backward reads; None with lists=False, where they would
    pass a sixteenth of the device's memory together with those of every other
    live Residuals, or where there is no memory for them: forward and backward
    then run without them), and
    block_mask, q_count, q_index, k_count, k_index and stats ([0]: K passes the
    solver streamed, [1]: its evaluations, per query block).

    The last six are parts of one allocation, made into tensors where they are
    asked for: ten allocations and views per forward took longer on the host
    than the kernels of a short sequence on the GPU (a training step at B1 H2
    n128: 79 us of host time with them, most of them never looked at)."""

    lists, _tables, _parts, _kept = None, None, {}, None  # objects that were saved with a tensor per table

    def __init__(self, shape: Shape, params: Params, device, with_stats: bool = True, lists: bool = True):
        z = entmax_attn_sizes(shape, params)
        BH, n, d = shape.batch * shape.heads, shape.seqlen, shape.head_dim
        T = (n + 63) // 64
        self.shape, self.params, self.sizes = shape, params, z
        self.tau = torch.empty((BH, n), dtype=torch.float32, device=device)
        self.o2 = (torch.empty((BH, n, d), dtype=torch.float32, device=device)
                   if params.need_bwd else None)
        self.tau_lo = (torch.empty((BH, n), dtype=torch.float32, device=device)
                       if z.tau_lo else None)
        nbytes = _lists_size(shape, params, LISTS_FROM) if lists else 0
        self._share = _claim(self.tau.device, nbytes) if nbytes else None
        self.lists = _bytes_or_none(nbytes, device) if self._share else None
        at, parts = 0, {}
        for name, nbytes, dims in (
                ("q_index", z.q_index, (BH, T, T)), ("k_index", z.k_index, (BH, T, T)),
                ("q_count", z.q_count, (BH, T)), ("k_count", z.k_count, (BH, T)),
                ("stats", z.stats, (2, BH, T)), ("block_mask", z.block_mask, (BH, T, T))):
            parts[name] = (at, nbytes, dims)
            at += (nbytes + 255) // 256 * 256
        self._parts = parts
        self._tables = torch.empty(at, dtype=torch.uint8, device=device)
        if not with_stats:
            self.stats = None

    def __getattr__(self, name):  # a part that is not a tensor yet
        part = self._parts.get(name)
        if part is None:
            raise AttributeError("Residuals has no attribute %r" % name)
        at, nbytes, dims = part
        t = self._tables[at:at + nbytes]
        if name != "block_mask":
            t = t.view(torch.int32)
        t = t.view(dims)
        self.__dict__[name] = t
        return t

    def ptrs(self) -> ResidualPtrs:
        own = self.__dict__
        base = self._tables.data_ptr() if self._parts else 0

        def f(name):
            if name in own:
                return None if own[name] is None else own[name].data_ptr()
            return base + self._parts[name][0]

        p = ResidualPtrs(*map(f, ("tau", "o2", "block_mask", "q_count", "q_index", "k_count",
                                  "k_index", "stats", "tau_lo")))
        if self.lists is not None:
            p.lists, p.lists_bytes = self.lists.data_ptr(), self.lists.numel()
            p.lists_shape = _dims(self.shape)
            p.owner = self
        return p

    def keep_workspace(self, make=True):
        """The buffer that entmax_attn_bwd_noalloc sorts the lists in, held from
        the first call on; None where there is none and `make` is false, or no
        memory for it."""
        if self._kept is None and make and self.lists is not None:
            self._kept = _bytes_or_none(entmax_attn_bwd_lists_workspace(self.shape, self.params),
                                        self.lists.device)
        return self._kept


def _stream_handle(device):
    return torch._C._cuda_getCurrentRawStream(device.index)  # current_stream without its object


# ------------------------------------------------------ argument checks
#
# The C ABI takes bare device pointers and no sizes for the residual buffers,
# so a tensor of the wrong shape, dtype or device would make the kernels read
# or write past its end.  Every tensor is checked here before any call.

def _need(t, name, shape, dtype, device=None):
    """Raises ValueError unless t is a contiguous tensor of this shape and
    dtype (and, given device, on that device).  Whether that device is a GPU
    is checked once per call by _on_gpu, after every tensor's shape."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))


def _on_gpu(device):
    if device is None or device.type != "cuda":
        raise ValueError("tensors must be on a GPU device, not %s" % device)


def _torch_dtype(shape: Shape):
    return torch.bfloat16 if shape.dtype == EA_BF16 else torch.float32


def _check_qkv(names_tensors, shape: Shape):
    """q, k, v (and dO) against one shape: [B, H, n, d] in the shape's dtype,
    all on the device of the first."""
    dims = (shape.batch, shape.heads, shape.seqlen, shape.head_dim)
    dev = names_tensors[0][1].device if isinstance(names_tensors[0][1], torch.Tensor) else None
    for name, t in names_tensors:
        _need(t, name, dims, _torch_dtype(shape), dev)
    return dev


def _same_shape(a: Shape, b: Shape) -> bool:
    return all(getattr(a, f) == getattr(b, f) for f, _ in Shape._fields_)


def _check_residuals(res, shape: Shape, device, need_o2: bool):
    if not isinstance(res, Residuals):
        raise ValueError("res must be the Residuals of a forward call")
    if not _same_shape(res.shape, shape):
        raise ValueError("res was sized for a different shape or dtype")
    BH, n, d = shape.batch * shape.heads, shape.seqlen, shape.head_dim
    T = (n + 63) // 64
    _need(res.tau, "res.tau", (BH, n), torch.float32, device)
    if need_o2:
        if res.o2 is None:
            raise ValueError("res has no o2 (forward ran with need_bwd=False)")
        _need(res.o2, "res.o2", (BH, n, d), torch.float32, device)
    # the tables that are still parts of one buffer have their sizes from it
    if res._parts:
        _need(res._tables, "res", res._tables.shape, torch.uint8, device)
    own = res.__dict__
    for name, dims, dtype in (("block_mask", (BH, T, T), torch.uint8), ("q_count", (BH, T), torch.int32),
                              ("q_index", (BH, T, T), torch.int32), ("k_count", (BH, T), torch.int32),
                              ("k_index", (BH, T, T), torch.int32), ("stats", (2, BH, T), torch.int32)):
        if name in own and not (name == "stats" and own[name] is None):
            _need(own[name], "res." + name, dims, dtype, device)
    if shape.dtype == EA_F32:
        _need(res.tau_lo, "res.tau_lo", (BH, n), torch.float32, device)
    if res.lists is not None:
        _check_bytes(res.lists, "res.lists", entmax_attn_lists_bytes(shape, res.params), device)


def _check_bytes(ws, name, need_bytes, device):
    if not isinstance(ws, torch.Tensor) or not ws.is_contiguous():
        raise ValueError("%s must be a contiguous tensor" % name)
    if ws.numel() * ws.element_size() < need_bytes:
        raise ValueError("%s holds %d bytes, needs %d" % (
            name, ws.numel() * ws.element_size(), need_bytes))
    if ws.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def backward_workspace(res: Residuals, device):
    """A device buffer for the workspace of backward: delta, and room to sort
    the element lists where res has them (without that room, as in a buffer of
    sizes.ws_bwd bytes, the backward does not use them)."""
    if res.lists is not None:
        ws = _bytes_or_none(entmax_attn_bwd_lists_workspace(res.shape, res.params), device)
        if ws is not None:
            return ws
    return torch.empty(max(res.sizes.ws_bwd, 16), dtype=torch.uint8, device=device)


def forward_workspace(res: Residuals, device):
    """A device buffer of sizes.ws_fwd bytes for the solver's candidate cache."""
    return torch.empty(max(res.sizes.ws_fwd, 16), dtype=torch.uint8, device=device)


def forward(q, k, v, alpha=1.5, scale=None, causal=False, need_bwd=True, max_iter=None,
            tol=None, out=None, res: Residuals | None = None, workspace=None, lists=True):
    """O and the residuals for Q, K, V ([B, H, n, d] bf16/fp32 CUDA tensors).

    workspace: a uint8 device tensor for the solver's candidate cache (None
    allocates sizes.ws_fwd bytes; False runs the solver without the cache).
    lists: whether new residuals hold element lists (see Residuals)."""
    shape = make_shape(q)
    dev = _check_qkv([("q", q), ("k", k), ("v", v)], shape)
    params = make_params(alpha, scale, causal, need_bwd, max_iter, tol, head_dim=q.shape[-1])
    if res is None:
        res = Residuals(shape, params, q.device, lists=lists)
    else:
        _check_residuals(res, shape, dev, bool(need_bwd))
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", q.shape, q.dtype, dev)
    if workspace is not None and workspace is not False:
        _check_bytes(workspace, "workspace", 0, dev)
    _on_gpu(dev)
    rp = res.ptrs()
    if workspace is None:
        workspace = forward_workspace(res, q.device)
    ws_ptr, ws_bytes = (None, 0) if workspace is False else (workspace.data_ptr(),
                                                            workspace.numel() * workspace.element_size())
    _check(entmax_attn_fwd(shape, params, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                           out.data_ptr(), rp, ws_ptr, ws_bytes, _stream_handle(q.device)),
           "entmax_attn_fwd")
    res.params = params
    return out, res


def backward(q, k, v, dout, res: Residuals, dq=None, dk=None, dv=None, workspace=None):
    """(dQ, dK, dV) in fp32 for the loss sum(dO * O) of the forward that filled res.

    workspace: a device tensor of at least sizes.ws_bwd bytes; to keep one from
    call to call, take it from backward_workspace."""
    shape = make_shape(q)
    dev = _check_qkv([("q", q), ("k", k), ("v", v), ("dout", dout)], shape)
    _check_residuals(res, shape, dev, True)
    if not res.params.need_bwd:
        raise ValueError("res comes from a forward with need_bwd=False")
    mk = lambda t: t if t is not None else torch.empty(q.shape, dtype=torch.float32, device=q.device)
    dq, dk, dv = mk(dq), mk(dk), mk(dv)
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        _need(t, name, q.shape, torch.float32, dev)
    if workspace is None:
        workspace = backward_workspace(res, q.device)
    else:
        _check_bytes(workspace, "workspace", res.sizes.ws_bwd, dev)
    _on_gpu(dev)
    rp = res.ptrs()
    _check(entmax_attn_bwd(shape, res.params, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                           dout.data_ptr(), rp, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                           workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                           _stream_handle(q.device)),
           "entmax_attn_bwd")
    return dq, dk, dv


# ------------------------------------------------------- row-wise entmax

def entmax_rows_fwd(rows, n, dtype, params, s, p, tau, stream):
    return _lib.entmax_rows_fwd(rows, n, dtype, ctypes.byref(params), s, p, tau, stream)


def entmax_rows_bwd(rows, n, dtype, params, s, tau, dp, ds, stream):
    return _lib.entmax_rows_bwd(rows, n, dtype, ctypes.byref(params), s, tau, dp, ds, stream)


def _row_params(alpha, scale, max_iter, tol):
    p = default_params()
    p.alpha, p.scale, p.causal, p.need_bwd = float(alpha), float(scale), 0, 0
    if max_iter is not None:
        p.max_iter = int(max_iter)
    if tol is not None:
        p.tol = float(tol)
    return p


def rows_forward(s, alpha=1.5, scale=1.0, max_iter=None, tol=None):
    """(p, tau): alpha-entmax of each row of s ([..., n] bf16/fp32 device tensor)."""
    if not s.is_cuda or not s.is_contiguous() or s.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("s must be a contiguous bf16 or fp32 device tensor")
    n = s.shape[-1]
    rows = s.numel() // n
    p = torch.empty(s.shape, dtype=torch.float32, device=s.device)
    tau = torch.empty(s.shape[:-1], dtype=torch.float32, device=s.device)
    params = _row_params(alpha, scale, max_iter, tol)
    _check(entmax_rows_fwd(rows, n, EA_BF16 if s.dtype == torch.bfloat16 else EA_F32, params,
                           s.data_ptr(), p.data_ptr(), tau.data_ptr(), _stream_handle(s.device)),
           "entmax_rows_fwd")
    return p, tau


def rows_backward(s, tau, dp, alpha=1.5, scale=1.0):
    """Gradient of sum(dp * p) with respect to s, for (p, tau) = rows_forward(s)."""
    if not isinstance(s, torch.Tensor) or s.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("s must be a bf16 or fp32 tensor")
    _need(s, "s", s.shape, s.dtype)
    n = s.shape[-1]
    rows = s.numel() // n
    _need(dp, "dp", s.shape, torch.float32, s.device)
    _need(tau, "tau", s.shape[:-1], torch.float32, s.device)
    _on_gpu(s.device)
    ds = torch.empty(s.shape, dtype=torch.float32, device=s.device)
    params = _row_params(alpha, scale, None, None)
    _check(entmax_rows_bwd(rows, n, EA_BF16 if s.dtype == torch.bfloat16 else EA_F32, params,
                           s.data_ptr(), tau.data_ptr(), dp.data_ptr(), ds.data_ptr(),
                           _stream_handle(s.device)), "entmax_rows_bwd")
    return ds


# ---------------------------------------------------------- no-mask mode

def _dense_backward_pays(shape, params) -> bool:
    """Whether the no-mask backward takes long enough by products (120 us and
    more; about 3.5 us per block of keys that a workgroup walks, or 215 blocks
    of 64 x 64 x 64 a microsecond, 1.6 times that with a general alpha) for the launches that look for sparse heads
    (15 us) and what those may gain: B4 H2 n1920 d64 causal, 88 us by products
    and 75 with lists at c = 12, is left out, B1 H8 n2431 d128 (181 us, 100 with
    lists) is not.  fp32 products take 16 times as long."""
    T = (shape.seqlen + 63) // 64
    blocks = shape.batch * shape.heads * T * (T + 1 if params.causal else 2 * T) // 2 * shape.head_dim // 64
    us = max(3.5 * T, blocks / 215) * (1.0 if params.alpha in (1.25, 1.5, 2.0) else 1.6)
    return shape.dtype == EA_F32 or us >= 120


def _scratch_lists(shape, params, device, lists):
    """Element lists for one call of the no-mask mode: (tensor or None, pointer, bytes)."""
    nbytes = _lists_size(shape, params, DENSE_LISTS_FROM) if lists else 0
    t = _bytes_or_none(nbytes, device) if 0 < nbytes <= _lists_limit(device) else None
    return (None, None, 0) if t is None else (t, t.data_ptr(), nbytes)


def forward_dense(q, k, v, alpha=1.5, scale=None, causal=False, need_bwd=True, max_iter=None,
                  tol=None, workspace=None, lists=True):
    """(O, tau, O2 or None, tau_lo or None) without block mask or tables
    (Algorithm 2 as written); tau_lo, the threshold's low part, exists for fp32
    inputs and goes back into backward_dense.  lists: whether the call may take
    scratch for element lists (582 bytes a row; backward_dense 1.2 KB)."""
    shape = make_shape(q)
    dev = _check_qkv([("q", q), ("k", k), ("v", v)], shape)
    _on_gpu(dev)
    params = make_params(alpha, scale, causal, need_bwd, max_iter, tol, head_dim=q.shape[-1])
    B, H, n, d = q.shape
    o = torch.empty_like(q)
    tau = torch.empty((B * H, n), dtype=torch.float32, device=q.device)
    tau_lo = torch.empty_like(tau) if q.dtype == torch.float32 else None
    o2 = torch.empty(q.shape, dtype=torch.float32, device=q.device) if need_bwd else None
    z = entmax_attn_sizes(shape, params)
    if workspace is None:
        workspace = torch.empty(max(z.ws_fwd, 16), dtype=torch.uint8, device=q.device)
    elif workspace is not False:
        _check_bytes(workspace, "workspace", 0, dev)
    _on_gpu(dev)
    ws_ptr, ws_bytes = (None, 0) if workspace is False else (workspace.data_ptr(),
                                                            workspace.numel() * workspace.element_size())
    _lists, lists_ptr, lists_bytes = _scratch_lists(shape, params, q.device, lists)
    _check(_lib.entmax_attn_fwd_dense_lists(
        ctypes.byref(shape), ctypes.byref(params), q.data_ptr(), k.data_ptr(), v.data_ptr(),
        o.data_ptr(), tau.data_ptr(), tau_lo.data_ptr() if tau_lo is not None else None,
        o2.data_ptr() if o2 is not None else None, lists_ptr, lists_bytes, ws_ptr, ws_bytes,
        _stream_handle(q.device)), "entmax_attn_fwd_dense")
    return o, tau, o2, tau_lo


def backward_dense(q, k, v, dout, tau, o2, alpha=1.5, scale=None, causal=False, tau_lo=None,
                   lists=True):
    """(dQ, dK, dV) in fp32 for the no-mask forward that produced tau, o2 and
    (fp32 inputs) tau_lo.  lists: as for forward_dense."""
    shape = make_shape(q)
    dev = _check_qkv([("q", q), ("k", k), ("v", v), ("dout", dout)], shape)
    B, H, n, d = q.shape
    _need(tau, "tau", (B * H, n), torch.float32, dev)
    _need(o2, "o2", q.shape, torch.float32, dev)
    if q.dtype == torch.float32:
        if tau_lo is None:
            raise ValueError("backward_dense: fp32 inputs need the forward's tau_lo")
        _need(tau_lo, "tau_lo", (B * H, n), torch.float32, dev)
    _on_gpu(dev)
    params = make_params(alpha, scale, causal, True, None, None, head_dim=q.shape[-1])
    mk = lambda: torch.empty(q.shape, dtype=torch.float32, device=q.device)
    dq, dk, dv = mk(), mk(), mk()
    _lists, lists_ptr, lists_bytes = _scratch_lists(shape, params, q.device,
                                                    lists and _dense_backward_pays(shape, params))
    ws = _bytes_or_none(entmax_attn_bwd_lists_workspace(shape, params), q.device) if lists_ptr else None
    if ws is None:
        ws = torch.empty(max(entmax_attn_sizes(shape, params).ws_bwd, 16), dtype=torch.uint8, device=q.device)
    _check(_lib.entmax_attn_bwd_dense_lists(
        ctypes.byref(shape), ctypes.byref(params), q.data_ptr(), k.data_ptr(), v.data_ptr(),
        dout.data_ptr(), tau.data_ptr(), tau_lo.data_ptr() if q.dtype == torch.float32 else None,
        o2.data_ptr(), lists_ptr, lists_bytes, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
        ws.data_ptr(), ws.numel(), _stream_handle(q.device)), "entmax_attn_bwd_dense")
    return dq, dk, dv


# ------------------------------------------- layouts of a transformer's layer
#
# The calls below take [tokens, heads, d] tensors, in the strides that the
# caller has them in.  They run on the tensors' device, whichever is current.

class Strides(ctypes.Structure):
    _fields_ = [("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class Rotary(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("weight_dtype", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("sections", ctypes.c_int32 * 4), ("eps", ctypes.c_float)]


class PackedShape(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in
                ("tokens", "seqs", "max_seqlen", "heads", "kv_heads", "head_dim", "dtype")]


class PackedSizes(ctypes.Structure):
    _fields_ = [(f, ctypes.c_size_t) for f in ("residuals", "ws_fwd", "ws_bwd", "lists", "ws_bwd_lists")]


class PackedStrides(ctypes.Structure):
    _fields_ = [(f, Strides) for f in ("q", "k", "v", "o")]


class DecodeShape(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in
                ("requests", "heads", "kv_heads", "head_dim", "dtype", "prefix", "capacity")]


class DecodeStrides(ctypes.Structure):
    _fields_ = ([(f, Strides) for f in ("q", "o", "k", "v", "k_prefix", "v_prefix")] +
                [("k_request", ctypes.c_int64), ("v_request", ctypes.c_int64)])


_i32, _i64, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
for _name, _args in (
        ("entmax_norm_rotary", [_P(Rotary), _v, _P(Strides), _v, _P(Strides), _v, _i64, _v, _v, _v, _v,
                                _P(Strides), _v, _P(Strides), _v]),
        ("entmax_norm_rotary_workspace", [_P(Rotary), _P(_sz)]),
        ("entmax_norm_rotary_bwd", [_P(Rotary), _v, _P(Strides), _v, _P(Strides), _v, _P(Strides), _v,
                                    _P(Strides), _v, _i64, _v, _v, _v, _v, _v, _v, _v, _v, _sz, _v]),
        ("entmax_packed_plan_bytes", [_i32, _i32, _P(_sz)]),
        ("entmax_packed_plan", [_i32, _i32, _i32, _i32, _v, _v, _sz, _v]),
        ("entmax_packed_sizes", [_P(PackedShape), _P(Params), _P(PackedSizes)]),
        ("entmax_packed_fwd", [_P(PackedShape), _P(Params), _v, _v, _v, _v, _v, _P(PackedStrides), _i32,
                               _v, _sz, _v, _sz, _v, _sz, _v]),
        ("entmax_packed_bwd", [_P(PackedShape), _P(Params), _v, _v, _v, _v, _v, _P(PackedStrides), _i32,
                               _v, _sz, _v, _sz, _v, _v, _v, _v, _sz, _v]),
        ("entmax_prefix_decode_workspace", [_P(DecodeShape), _P(_sz)]),
        ("entmax_prefix_decode", [_P(DecodeShape), _P(Params), _P(DecodeStrides), _v, _v, _v, _v, _v, _v,
                                  _v, _v, _sz, _v])):
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = ctypes.c_int


def _ea_dtype(t, name):
    if t.dtype == torch.bfloat16:
        return EA_BF16
    if t.dtype == torch.float32:
        return EA_F32
    raise ValueError("%s must be bfloat16 or float32, not %s" % (name, t.dtype))


def _strided(t, name, shape, dtype, device, written=False):
    """Raises ValueError unless t is a tensor of this shape, dtype and device
    whose last dimension is contiguous and whose rows start at multiples of 16
    bytes; a tensor to be written must not hold an element twice."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    if t.numel() == 0:
        return
    vec = 16 // t.element_size()
    if t.is_contiguous() and shape[-1] % vec == 0 and t.data_ptr() % 16 == 0:
        return
    if t.stride(-1) != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    bad = t.data_ptr() % 16
    for n, step in zip(t.shape, t.stride()[:-1]):  # (the stride of a dimension of one element is never used)
        if n > 1 and step % vec:
            bad = 1
    if bad:
        raise ValueError("%s: rows must start at multiples of 16 bytes" % name)
    if written:
        # each dimension steps over all of the smaller ones
        end = t.shape[-1]
        for n, s in sorted(((n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n > 1), key=lambda x: x[1]):
            if s < end:
                raise ValueError("%s has elements that share memory" % name)
            end = s * (n - 1) + end


def _stride(t, dim):
    return t.stride(dim) if t.shape[dim] > 1 else 0


# Argument structures are built once for each set of sizes that a program uses:
# a call at the sizes of a decoding step is a few microseconds of host time,
# and each structure one or two.  They are never written to afterwards, and
# no object that a caller gets holds one.
@functools.lru_cache(maxsize=1024)
def _strides_of(row, head):
    return Strides(row, head)


def _numbers(alpha, scale, max_iter, tol):
    """A call's parameters as plain numbers, whatever holds them."""
    return (float(alpha), None if scale is None else float(scale), None if max_iter is None else int(max_iter),
            None if tol is None else float(tol))


def _near(rows):
    """Raises ValueError where rows are further apart than a tile's offsets reach."""
    if max(rows) > 1 << 24:
        raise ValueError("rows are %d elements apart, at most 2^24 are possible" % max(rows))


def _row_head(t, row=0, head=1):
    return _strides_of(_stride(t, row), _stride(t, head))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _overlap(a, b):
    """Whether two tensors' memory ranges meet."""
    def span(t):
        lo = t.data_ptr()
        return lo, lo + t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))
    if a.numel() == 0 or b.numel() == 0:
        return False
    (a0, a1), (b0, b1) = span(a), span(b)
    return a0 < b1 and b0 < a1


class _SameDevice:
    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_same_device = _SameDevice()


def _on_device(device):
    """Makes a device current for a call where it is not (a launch goes to a
    stream of the current device)."""
    return _same_device if device.index == torch._C._cuda_getDevice() else torch.cuda.device(device)


# ------------------------------------------------------ norm and rotation

def _check_rotary(q, k, positions, freqs, q_weight, k_weight, sections, eps, interleaved):
    """(Rotary, positions' row stride) of a call's arguments."""
    for name, t in (("q", q), ("k", k)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError("%s must be a [tokens, heads, head_dim] tensor" % name)
    dt = _ea_dtype(q, "q")
    tokens, hq, d = q.shape
    hk, dev = k.shape[1], q.device
    _strided(q, "q", q.shape, q.dtype, dev)
    _strided(k, "k", (tokens, hk, d), q.dtype, dev)
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError("freqs must be a contiguous [rot_dim / 2] tensor")
    if freqs.dtype != torch.float32 or freqs.device != dev:
        raise ValueError("freqs has dtype %s on %s, expected float32 on %s" % (freqs.dtype, freqs.device, dev))
    pairs = freqs.shape[0]
    sections = (pairs,) if sections is None else tuple(int(s) for s in sections)
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or sum(sections) != pairs:
        raise ValueError("sections must be 1 to 4 numbers of pairs that add up to len(freqs) = %d" % pairs)
    if 2 * pairs > d or pairs % 8:
        raise ValueError("freqs must hold a multiple of 8 pairs, at most half of head_dim")
    axes = len(sections)
    if not isinstance(positions, torch.Tensor) or not (
            positions.shape == (axes, tokens) or (axes == 1 and positions.shape == (tokens,))):
        raise ValueError("positions must be a %s tensor" % ([axes, tokens],))
    if positions.dtype != torch.int32 or positions.device != dev:
        raise ValueError("positions must be int32 and on %s" % dev)
    if tokens > 1 and positions.stride(-1) != 1:
        raise ValueError("positions must be contiguous in its last dimension")
    wt = q.dtype
    given = [(n, w) for n, w in (("q_weight", q_weight), ("k_weight", k_weight)) if w is not None]
    if given:
        wt = given[0][1].dtype if isinstance(given[0][1], torch.Tensor) else None
        if wt not in (q.dtype, torch.float32):
            raise ValueError("weights must have the dtype of q, or be float32")
        for name, w in given:
            _need(w, name, (d,), wt, dev)
            if w.data_ptr() % 16:
                raise ValueError("%s must start at a multiple of 16 bytes" % name)
    r = _rotary_of(tokens, hq, hk, d, dt, EA_F32 if wt == torch.float32 else EA_BF16, 2 * pairs, bool(interleaved),
                   sections, float(eps))
    return r, positions.stride(0) if positions.dim() == 2 else 0


@functools.lru_cache(maxsize=256)
def _rotary_of(tokens, hq, hk, d, dt, weight_dt, rot, interleaved, sections, eps):
    return Rotary(tokens, hq, hk, d, dt, weight_dt, rot, int(interleaved), len(sections),
                  (ctypes.c_int32 * 4)(*sections), eps)


def norm_rotary(q, k, positions, freqs, q_weight=None, k_weight=None, sections=None, eps=1e-6,
                interleaved=False, q_out=None, k_out=None):
    """(q_out, k_out): every head of q [tokens, heads, d] and k [tokens, kv_heads, d]
    (bf16 or fp32, any strides with a contiguous last dimension) divided by
    sqrt(mean(x^2) + eps), times its weights ([d], of q's dtype or fp32; None:
    1), and rotated: pair i by positions * freqs[i] radians.

    freqs: fp32 [rot_dim / 2]; the pairs are (i, i + rot_dim / 2), or (2 i, 2 i + 1)
    with interleaved=True, and dimensions behind rot_dim are not rotated.
    positions: int32 [tokens]; with several axes [axes, tokens], and sections
    gives the number of consecutive pairs that each axis rotates.
    q_out, k_out: tensors to write, which may be q and k themselves."""
    r, pos_stride = _check_rotary(q, k, positions, freqs, q_weight, k_weight, sections, eps, interleaved)
    for name, out, like in (("q_out", q_out, q), ("k_out", k_out, k)):
        if out is None:
            continue
        _strided(out, name, like.shape, like.dtype, like.device, written=True)
        for other_name, t in (("q", q), ("k", k)):
            if _overlap(out, t) and not (t is like and out.data_ptr() == t.data_ptr() and out.stride() == t.stride()):
                if not _apart(out, t):
                    raise ValueError("%s overlaps %s" % (name, other_name))
    if q_out is not None and k_out is not None and _overlap(q_out, k_out) and not _apart(q_out, k_out):
        raise ValueError("q_out overlaps k_out")
    _on_gpu(q.device)
    with _on_device(q.device):
        q_out = q.new_empty(q.shape) if q_out is None else q_out
        k_out = k.new_empty(k.shape) if k_out is None else k_out
        _check(_lib.entmax_norm_rotary(
            r, q.data_ptr(), _row_head(q), k.data_ptr(), _row_head(k), positions.data_ptr(),
            pos_stride, freqs.data_ptr(), _ptr(q_weight), _ptr(k_weight), q_out.data_ptr(), _row_head(q_out),
            k_out.data_ptr(), _row_head(k_out), _stream_handle(q.device)), "entmax_norm_rotary")
    return q_out, k_out


def _apart(a, b):
    """Whether two tensors whose ranges meet are different columns of the same
    rows (parts of one fused projection)."""
    row = a.stride(0)
    if a.dim() != b.dim() or a.shape[0] != b.shape[0] or a.shape[0] < 2 or row != b.stride(0):
        return False
    width = lambda t: 1 + sum((n - 1) * s for n, s in zip(t.shape[1:], t.stride()[1:]))
    first, second = sorted((a, b), key=lambda t: t.data_ptr())
    gap = (second.data_ptr() - first.data_ptr()) // a.element_size()
    return gap >= width(first) and gap + width(second) <= row


def norm_rotary_backward(dq_out, dk_out, q, k, positions, freqs, q_weight=None, k_weight=None, sections=None,
                         eps=1e-6, interleaved=False):
    """(dq, dk, dq_weight, dk_weight) of sum(dq_out * q_out) + sum(dk_out * k_out)
    for (q_out, k_out) = norm_rotary(q, k, ...): dq, dk in q's dtype, the
    weights' gradients in fp32 (None for a weight that is None).  dq_out and
    dk_out have q's dtype."""
    r, pos_stride = _check_rotary(q, k, positions, freqs, q_weight, k_weight, sections, eps, interleaved)
    _strided(dq_out, "dq_out", q.shape, q.dtype, q.device)
    _strided(dk_out, "dk_out", k.shape, q.dtype, q.device)
    _on_gpu(q.device)
    with _on_device(q.device):
        dq, dk = q.new_empty(q.shape), k.new_empty(k.shape)
        dwq, dwk = (None if w is None else torch.empty(q.shape[-1], dtype=torch.float32, device=q.device)
                    for w in (q_weight, k_weight))
        n = ctypes.c_size_t()
        _check(_lib.entmax_norm_rotary_workspace(r, ctypes.byref(n)), "entmax_norm_rotary_workspace")
        ws = torch.empty(max(n.value, 16), dtype=torch.uint8, device=q.device)
        _check(_lib.entmax_norm_rotary_bwd(
            r, dq_out.data_ptr(), _row_head(dq_out), dk_out.data_ptr(), _row_head(dk_out),
            q.data_ptr(), _row_head(q), k.data_ptr(), _row_head(k), positions.data_ptr(), pos_stride,
            freqs.data_ptr(), _ptr(q_weight), _ptr(k_weight), dq.data_ptr(), dk.data_ptr(), _ptr(dwq),
            _ptr(dwk), ws.data_ptr(), ws.numel(), _stream_handle(q.device)), "entmax_norm_rotary_bwd")
    return dq, dk, dwq, dwk


# ------------------------------------------------------ packed sequences

class PackedPlan:
    """The tiles of a batch's sequences, listed on the device by packed_plan:
    for every packed_forward and packed_backward on these sequences, of any
    layer and head counts.  It lives on the stream that made it, as a tensor does."""

    def __init__(self, buffer, tokens, seqs, max_seqlen, causal):
        self.buffer, self.tokens, self.seqs = buffer, tokens, seqs
        self.max_seqlen, self.causal = max_seqlen, causal

    @property
    def device(self):
        return self.buffer.device


def packed_plan(cu_seqlens, tokens, max_seqlen=None, causal=True) -> PackedPlan:
    """Lists the tiles of the sequences cu_seqlens[s] .. cu_seqlens[s + 1] (int32
    [seqs + 1] on the device, ascending; up to 65536 sequences) of tensors with `tokens` rows.  One
    launch; the host does not wait for cu_seqlens.  max_seqlen: no sequence is
    longer (default: tokens); the residuals' tables grow with it.  A sequence
    that is longer, reaches outside the tensors or overlaps an earlier one is
    left out: its rows are NaN in outputs that a call makes, and in given ones
    stay (O) or are unspecified (gradients)."""
    if not isinstance(cu_seqlens, torch.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 2:
        raise ValueError("cu_seqlens must be a [seqs + 1] tensor of at least one sequence")
    _need(cu_seqlens, "cu_seqlens", cu_seqlens.shape, torch.int32)
    tokens, seqs = int(tokens), cu_seqlens.shape[0] - 1
    if tokens < 1:
        raise ValueError("tokens must be at least 1")
    # (no sequence is longer than its tensors, or than the kernels take)
    max_seqlen = min(tokens, MAX_SEQLEN) if max_seqlen is None else int(max_seqlen)
    if max_seqlen < 1:
        raise ValueError("max_seqlen must be at least 1")
    max_seqlen = min(max_seqlen, tokens)
    _on_gpu(cu_seqlens.device)
    n = ctypes.c_size_t()
    _check(_lib.entmax_packed_plan_bytes(tokens, seqs, ctypes.byref(n)), "entmax_packed_plan_bytes")
    with _on_device(cu_seqlens.device):
        buffer = torch.empty(n.value, dtype=torch.uint8, device=cu_seqlens.device)
        _check(_lib.entmax_packed_plan(tokens, seqs, max_seqlen, int(bool(causal)), cu_seqlens.data_ptr(),
                                       buffer.data_ptr(), n.value, _stream_handle(cu_seqlens.device)),
               "entmax_packed_plan")
    return PackedPlan(buffer, tokens, seqs, max_seqlen, bool(causal))


# Training steps of 8192 packed tokens, in us, without lists against with them:
# 16/4 heads, d = 128, c = 1, sequences of 256 291 against 307, of 512 361
# against 375, of 1024 497 against 485, of 2048 753 against 647; 8 heads, d =
# 64, c = 2, of 512 115 against 130, of 1024 161 against 157, of 2048 250 against
# 188; fp32 (2048 tokens), d = 64, of 256 152 against 121.
PACKED_LISTS_FROM = 512
# Forward alone (LISTS_FROM), 8192 tokens, us, without against with: 16/4 heads, d
# = 128, c = 1, sequences of 192 86 against 87, of 320 124 against 125, of 512 135
# against 137, of 1024 180 against 174, at c = 4 83 against 83, 100 against 98, 104
# against 94, 137 against 108; fp32 (4096 tokens) of 64, c = 1, 124 against 108, of 128
# 143 against 115.


class PackedResiduals:
    """What packed_forward leaves for packed_backward: thresholds, O^(2) and the
    block tables in one device buffer, the element lists (see Residuals) or
    None, and the plan."""

    def __init__(self, shape: PackedShape, params: Params, plan: PackedPlan, sizes: PackedSizes, device,
                 lists: bool = True):
        # (copies: the calls' structures are kept for later calls, see above)
        self.shape, self.params, self.sizes = (type(x).from_buffer_copy(x) for x in (shape, params, sizes))
        self.plan = plan
        self.buffer = torch.empty(sizes.residuals, dtype=torch.uint8, device=device)
        # (as for Residuals, short sequences are not listed; fp32 products take longer)
        least = PACKED_LISTS_FROM if params.need_bwd else LISTS_FROM
        short = shape.max_seqlen <= (least if shape.dtype == EA_BF16 else least // 4)
        nbytes = 0 if short or not lists else sizes.lists
        self._share = _claim(self.buffer.device, nbytes) if nbytes else None
        self.lists = _bytes_or_none(nbytes, device) if self._share else None

    def lists_ptr(self):
        return (None, 0) if self.lists is None else (self.lists.data_ptr(), self.lists.numel())


def _packed_shape(q, k, v, plan):
    for name, t in (("q", q), ("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError("%s must be a [tokens, heads, head_dim] tensor" % name)
    if not isinstance(plan, PackedPlan):
        raise ValueError("plan must come from packed_plan")
    dt = _ea_dtype(q, "q")
    tokens, hq, d = q.shape
    hk = k.shape[1]
    if tokens != plan.tokens:
        raise ValueError("q has %d rows, the plan is for %d" % (tokens, plan.tokens))
    if plan.device != q.device:
        raise ValueError("the plan is on %s, q on %s" % (plan.device, q.device))
    if hk < 1 or hq % hk:
        raise ValueError("q's %d heads must be a multiple of k's %d" % (hq, hk))
    _strided(q, "q", q.shape, q.dtype, q.device)
    _strided(k, "k", (tokens, hk, d), q.dtype, q.device)
    _strided(v, "v", (tokens, hk, d), q.dtype, q.device)
    return _packed_shape_of(tokens, plan.seqs, plan.max_seqlen, hq, hk, d, dt)


@functools.lru_cache(maxsize=256)
def _packed_shape_of(*sizes):
    return PackedShape(*sizes)


def _packed_strides(*tensors):
    return _packed_strides_of(*[s for t in tensors for s in (_stride(t, 0), _stride(t, 1))])


@functools.lru_cache(maxsize=1024)
def _packed_strides_of(*s):
    _near(s[::2])
    return PackedStrides(*[Strides(s[i], s[i + 1]) for i in range(0, 8, 2)])


@functools.lru_cache(maxsize=256)
def _packed_params(alpha, scale, max_iter, tol, causal, need_bwd, head_dim, *shape):
    """(Params, PackedSizes) of a call."""
    params = make_params(alpha, scale, causal, need_bwd, max_iter, tol, head_dim=head_dim)
    sizes = PackedSizes()
    _check(_lib.entmax_packed_sizes(_packed_shape_of(*shape), ctypes.byref(params), ctypes.byref(sizes)),
           "entmax_packed_sizes")
    return params, sizes


def packed_forward(q, k, v, plan: PackedPlan, alpha=1.5, scale=None, need_bwd=True, max_iter=None, tol=None,
                   out=None, workspace=None, lists=True):
    """(O, residuals) of alpha-entmax attention within each sequence of the plan
    (causal if the plan is): q [tokens, heads, d], k and v [tokens, kv_heads, d],
    bf16 or fp32, any strides with a contiguous last dimension; query head h
    attends to key head h // (heads // kv_heads).

    Rows of no sequence (before cu_seqlens[0], behind the last) are 0 in an O
    that the call makes and left as they are in `out`.  need_bwd=False gives
    residuals that packed_backward does not take.  tol: default 1e-5, for fp32
    1e-6.  max_iter: 12 updates by default; alpha > 2 wants 40 or more.  workspace: as for forward (sizes.ws_fwd bytes of the residuals).
    lists: whether the residuals hold element lists (see Residuals)."""
    shape = _packed_shape(q, k, v, plan)
    if tol is None and shape.dtype == EA_F32:
        tol = 1e-6  # (Sum p is off by up to tol, which the fp32 outputs show)
    params, sizes = _packed_params(*_numbers(alpha, scale, max_iter, tol), plan.causal, bool(need_bwd), q.shape[-1],
                                   shape.tokens, shape.seqs, shape.max_seqlen, shape.heads, shape.kv_heads,
                                   shape.head_dim, shape.dtype)
    made = out is None
    if not made:
        _strided(out, "out", q.shape, q.dtype, q.device, written=True)
        for name, t in (("q", q), ("k", k), ("v", v)):
            if _overlap(out, t):
                raise ValueError("out overlaps %s" % name)
    if workspace is not None and workspace is not False:
        _check_bytes(workspace, "workspace", 0, q.device)
    _on_gpu(q.device)
    with _on_device(q.device):
        if made:
            out = q.new_empty(q.shape)
        res = PackedResiduals(shape, params, plan, sizes, q.device, lists)
        if workspace is None:
            workspace = torch.empty(max(sizes.ws_fwd, 16), dtype=torch.uint8, device=q.device)
        ws, ws_bytes = (None, 0) if workspace is False else (workspace.data_ptr(),
                                                            workspace.numel() * workspace.element_size())
        _check(_lib.entmax_packed_fwd(
            shape, params, plan.buffer.data_ptr(), q.data_ptr(), k.data_ptr(),
            v.data_ptr(), out.data_ptr(), _packed_strides(q, k, v, out), int(made), res.buffer.data_ptr(),
            res.buffer.numel(), *res.lists_ptr(), ws, ws_bytes, _stream_handle(q.device)), "entmax_packed_fwd")
    return out, res


def packed_backward(q, k, v, dout, res: PackedResiduals, dq=None, dk=None, dv=None, workspace=None):
    """(dQ, dK, dV) of sum(dout * O) for the packed_forward that made res, in the
    inputs' dtype: [tokens, heads, d] and [tokens, kv_heads, d], contiguous.
    dout has any strides with a contiguous last dimension.  Rows of no sequence
    are 0 in gradients that the call makes; they are left as they are if dq, dk
    and dv are given (all three or none).  workspace: a device buffer of at least
    res.sizes.ws_bwd bytes (ws_bwd_lists, to use the element lists of res)."""
    if not isinstance(res, PackedResiduals):
        raise ValueError("res must be the residuals of a packed_forward call")
    shape = _packed_shape(q, k, v, res.plan)
    if any(getattr(shape, f) != getattr(res.shape, f) for f, _ in PackedShape._fields_):
        raise ValueError("res was made for another shape or dtype")
    if not res.params.need_bwd:
        raise ValueError("res comes from a forward with need_bwd=False")
    if res.buffer.device != q.device:
        raise ValueError("res is on %s, q on %s" % (res.buffer.device, q.device))
    _strided(dout, "dout", q.shape, q.dtype, q.device)
    given = [t is not None for t in (dq, dk, dv)]
    if any(given) != all(given):
        raise ValueError("dq, dk and dv must be given together")
    made = not given[0]
    if not made:
        for name, t, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
            _need(t, name, like.shape, q.dtype, q.device)
            if t.data_ptr() % 16:
                raise ValueError("%s must start at a multiple of 16 bytes" % name)
            for other_name, other in (("q", q), ("k", k), ("v", v), ("dout", dout)):
                if _overlap(t, other):
                    raise ValueError("%s overlaps %s" % (name, other_name))
        if _overlap(dq, dk) or _overlap(dq, dv) or _overlap(dk, dv):
            raise ValueError("dq, dk and dv overlap")
    if workspace is not None:
        _check_bytes(workspace, "workspace", res.sizes.ws_bwd, q.device)
    _on_gpu(q.device)
    with _on_device(q.device):
        if made:
            dq, dk, dv = (t.new_empty(t.shape) for t in (q, k, v))
        if workspace is None and res.lists is not None:
            workspace = _bytes_or_none(res.sizes.ws_bwd_lists, q.device)
        if workspace is None:
            workspace = torch.empty(res.sizes.ws_bwd, dtype=torch.uint8, device=q.device)
        _check(_lib.entmax_packed_bwd(
            shape, res.params, res.plan.buffer.data_ptr(), q.data_ptr(),
            k.data_ptr(), v.data_ptr(), dout.data_ptr(), _packed_strides(q, k, v, dout), int(made),
            res.buffer.data_ptr(), res.buffer.numel(), *res.lists_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_handle(q.device)),
            "entmax_packed_bwd")
    return dq, dk, dv


# ------------------------------------------------------ single tokens

def prefix_decode_workspace(q, k_cache, prefix=0):
    """Bytes of the workspace of prefix_decode for these tensors and a prefix of
    that many keys (about 4.4 bytes for every query head and key)."""
    return _decode_of(1.5, None, None, None, q.shape[0], q.shape[1], k_cache.shape[2], q.shape[2],
                      _ea_dtype(q, "q"), int(prefix), k_cache.shape[1])[2]


@functools.lru_cache(maxsize=256)
def _decode_of(alpha, scale, max_iter, tol, *sizes):
    """(DecodeShape, Params, bytes of the workspace) of a call."""
    shape, n = DecodeShape(*sizes), ctypes.c_size_t()
    params = make_params(alpha, scale, False, False, max_iter, tol, head_dim=shape.head_dim)
    _check(_lib.entmax_prefix_decode_workspace(shape, ctypes.byref(n)), "entmax_prefix_decode_workspace")
    return shape, params, n.value


@functools.lru_cache(maxsize=1024)
def _decode_strides_of(*s):
    _near((s[4], s[8]))  # (of the keys)
    return DecodeStrides(*[Strides(s[i], s[i + 1]) for i in range(0, 12, 2)], s[12], s[13])


def prefix_decode(q, k_cache, v_cache, lengths, k_prefix=None, v_prefix=None, alpha=1.5, scale=None,
                  max_iter=None, tol=None, out=None, workspace=None):
    """O [requests, heads, d] of one new token per request: q [requests, heads, d]
    attends to the keys of k_prefix, v_prefix [prefix, kv_heads, d] (None: no
    prefix), which all requests share, and to the first lengths[b] keys (int32
    on the device, taken as 0 .. capacity) of its own k_cache, v_cache
    [requests, capacity, kv_heads, d].  bf16 or fp32, any strides with a
    contiguous last dimension.  A request without any key has O = 0, and so has
    a query whose largest score is not finite.

    tol: default 1e-6.  max_iter: 12 updates by default; alpha > 2 wants 40 or
    more.  workspace: a device buffer of prefix_decode_workspace
    bytes, to keep from call to call (one call at a time)."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [requests, heads, head_dim] tensor")
    dt = _ea_dtype(q, "q")
    B, hq, d = q.shape
    dev = q.device
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a [requests, capacity, kv_heads, head_dim] tensor")
    cap, hk = k_cache.shape[1:3]
    if hk < 1 or hq % hk:
        raise ValueError("q's %d heads must be a multiple of k_cache's %d" % (hq, hk))
    _strided(q, "q", q.shape, q.dtype, dev)
    _strided(k_cache, "k_cache", (B, cap, hk, d), q.dtype, dev)
    _strided(v_cache, "v_cache", (B, cap, hk, d), q.dtype, dev)
    _need(lengths, "lengths", (B,), torch.int32, dev)
    if (k_prefix is None) != (v_prefix is None):
        raise ValueError("k_prefix and v_prefix must be given together")
    P = 0
    if k_prefix is not None:
        if not isinstance(k_prefix, torch.Tensor) or k_prefix.dim() != 3:
            raise ValueError("k_prefix must be a [prefix, kv_heads, head_dim] tensor")
        P = k_prefix.shape[0]
        _strided(k_prefix, "k_prefix", (P, hk, d), q.dtype, dev)
        _strided(v_prefix, "v_prefix", (P, hk, d), q.dtype, dev)
    if out is not None:
        _strided(out, "out", q.shape, q.dtype, dev, written=True)
        for name, t in (("q", q), ("k_cache", k_cache), ("v_cache", v_cache), ("k_prefix", k_prefix),
                        ("v_prefix", v_prefix)):
            if t is not None and _overlap(out, t):
                raise ValueError("out overlaps %s" % name)
    shape, params, nbytes = _decode_of(*_numbers(alpha, scale, max_iter, 1e-6 if tol is None else tol), B, hq, hk, d,
                                       dt, P, cap)
    if workspace is not None:
        _check_bytes(workspace, "workspace", nbytes, dev)
    _on_gpu(dev)
    with _on_device(dev):
        if out is None:
            out = q.new_empty(q.shape)
        if workspace is None:
            workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=dev)
        strides = _decode_strides_of(
            _stride(q, 0), _stride(q, 1), _stride(out, 0), _stride(out, 1), _stride(k_cache, 1), _stride(k_cache, 2),
            _stride(v_cache, 1), _stride(v_cache, 2),
            *((0, 0, 0, 0) if P == 0 else (_stride(k_prefix, 0), _stride(k_prefix, 1), _stride(v_prefix, 0),
                                           _stride(v_prefix, 1))),
            _stride(k_cache, 0), _stride(v_cache, 0))
        _check(_lib.entmax_prefix_decode(
            shape, params, strides, q.data_ptr(), k_cache.data_ptr(),
            v_cache.data_ptr(), lengths.data_ptr(), _ptr(k_prefix), _ptr(v_prefix), out.data_ptr(),
            workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_handle(dev)),
            "entmax_prefix_decode")
    return out


# ------------------------------------------- a cache in pages and in 4 bits
#
# A layer's cache is a uint8 tensor [pages, kv_heads, 2, page_size / 16, 17 head_dim / 2]
# (the layout of its bytes: include/entmax_attn.h), a model's one [layers, ...] of
# those; a table of pages is an int32 tensor [rows, width].

class Cache(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("pages", "page_size", "kv_heads", "head_dim")]


class PageTable(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("width", ctypes.c_int32), ("stride", ctypes.c_int64)]


class PagedShape(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("queries", "heads", "dtype", "longest")]


for _name, _args in (
        ("entmax_cache_page_bytes", [_P(Cache), _P(_sz)]),
        ("entmax_cache_append", [_P(Cache), _v, _P(PageTable), _v, _i32, _i32, _v, _v, _v, _P(Strides), _v, _P(Strides),
                                 _v]),
        ("entmax_cache_read", [_P(Cache), _v, _P(PageTable), _v, _i32, _i32, _v, _v, _v, _P(Strides), _v, _P(Strides),
                               _v]),
        ("entmax_cache_workspace", [_P(Cache), _i32, _P(_sz)]),
        ("entmax_cache_update", [_P(Cache), _i32, _v, _P(PageTable), _v, _v, _i32, _v, _v, _v, _i64, _v, _v, _v, _sz,
                                 _v]),
        ("entmax_cache_compact", [_P(Cache), _i32, _v, _P(PageTable), _v, _v, _v, _i64, _v, _v, _sz, _v]),
        ("entmax_paged_decode_workspace", [_P(PagedShape), _P(Cache), _P(_sz)]),
        ("entmax_paged_decode", [_P(PagedShape), _P(Params), _P(Cache), _v, _P(PageTable), _v, _v, _P(Strides), _v, _v,
                                 _v, _P(Strides), _v, _sz, _v])):
    getattr(_lib, _name).argtypes = _args
    getattr(_lib, _name).restype = ctypes.c_int

# What a call's checks gave for tensors of these shapes, strides, types and devices: at
# the sizes of a decoding step the checks take longer than the kernels (an append of 64
# tokens 13 us of host time with them, 8 without).  Nothing here depends on
# what a tensor holds or where it lies; addresses are checked at each call.
_checked = {}


def _launch(dev, name, call, *args):
    """Calls an entry point on the device's current stream, with that device current."""
    if dev.index == torch._C._cuda_getDevice():
        status = call(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    else:
        with torch.cuda.device(dev):
            status = call(*args, torch._C._cuda_getCurrentRawStream(dev.index))
    if status:
        _check(status, name)


def _remember(key, value):
    if key is not None:
        if len(_checked) >= 1024:
            _checked.clear()
        _checked[key] = value
    return value


@functools.lru_cache(maxsize=256)
def _cache_of(shape):
    """The Cache of a layer's tensor of this shape."""
    if len(shape) != 5 or shape[2] != 2 or shape[4] not in (544, 1088):
        raise ValueError("a layer's cache is a [pages, kv_heads, 2, page_size / 16, 17 head_dim / 2] tensor, not %s" %
                         (shape,))
    c, n = Cache(shape[0], 16 * shape[3], shape[1], shape[4] * 2 // 17), ctypes.c_size_t()
    _check(_lib.entmax_cache_page_bytes(c, ctypes.byref(n)), "entmax_cache_page_bytes")
    return c


def paged_cache(pages, page_size, kv_heads, head_dim, layers=None, device="cuda"):
    """A cache of `pages` pages of page_size tokens (a power of two, 16 to 1024), each
    of kv_heads heads of 64 or 128 dimensions: a uint8 tensor of one layer, or with
    layers=n [n, ...] of as many, filled with zeros.  A token takes 17 head_dim / 16
    bytes of every key head."""
    if page_size % 16 or head_dim not in (64, 128):
        raise ValueError("page_size must be a multiple of 16, and head_dim 64 or 128")
    shape = (pages, kv_heads, 2, page_size // 16, 17 * head_dim // 2)
    _cache_of(shape)
    return torch.zeros(shape if layers is None else (layers,) + shape, dtype=torch.uint8, device=device)


def _layer(cache):
    if not isinstance(cache, torch.Tensor) or cache.dtype != torch.uint8:
        raise ValueError("cache must be a uint8 tensor")
    c = _cache_of(cache.shape)
    if not cache.is_contiguous():
        raise ValueError("cache must be contiguous")
    if cache.data_ptr() % 16:
        raise ValueError("cache must start at a multiple of 16 bytes")
    return c


def _layers(cache):
    """(Cache, layers) of a model's or one layer's cache."""
    if isinstance(cache, torch.Tensor) and cache.dim() == 6:
        if cache.shape[0] < 1:
            raise ValueError("cache has no layers")
        if not cache.is_contiguous():
            raise ValueError("cache must be contiguous")
        return _layer(cache[0]), cache.shape[0]
    return _layer(cache), 1


def _table(table, c, device, name="table"):
    if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.dtype != torch.int32:
        raise ValueError("%s must be an int32 [rows, width] tensor" % name)
    rows, width = table.shape
    if rows < 1 or width < 1:
        raise ValueError("%s has no entries" % name)
    if table.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, table.device, device))
    if width > 1 and table.stride(1) != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    if width * c.page_size > MAX_SEQLEN:
        raise ValueError("%s holds %d tokens a row, at most %d are possible" % (name, width * c.page_size, MAX_SEQLEN))
    return _page_table_of(rows, width, _stride(table, 0))


@functools.lru_cache(maxsize=256)
def _page_table_of(rows, width, stride):
    return PageTable(rows, width, stride)


def _check_places(cache, rows, positions, table):
    c = _layer(cache)
    t = _table(table, c, cache.device)
    if not isinstance(rows, torch.Tensor) or rows.dim() != 1:
        raise ValueError("rows must be a [tokens] tensor")
    _need(rows, "rows", rows.shape, torch.int32, cache.device)
    _need(positions, "positions", rows.shape, torch.int32, cache.device)
    return c, t


def _check_append(cache, k, v, rows, positions, table):
    c, t = _check_places(cache, rows, positions, table)
    shape = (rows.shape[0], c.kv_heads, c.head_dim)
    if not isinstance(k, torch.Tensor):
        raise ValueError("k must be a torch tensor")
    dt = _ea_dtype(k, "k")
    _strided(k, "k", shape, k.dtype, cache.device)
    _strided(v, "v", shape, k.dtype, cache.device)
    _on_gpu(cache.device)
    return c, t, shape[0], dt, _row_head(k), _row_head(v)


def cache_append(cache, k, v, rows, positions, table):
    """Writes keys and values k, v [tokens, kv_heads, head_dim] (bf16 or fp32, any strides
    with a contiguous last dimension) into a layer's cache, rounded to 4 bits: token
    i becomes token positions[i] of the table's row rows[i] (int32 on the device).
    Tokens without a place (a negative position, no such row, no page) are left
    out.  Two tokens of one call must not have the same place, and rows that share
    a page must not write to it (cache_update gives them pages of their own)."""
    try:
        dev = cache.device
        key = ("append", dev, cache.shape, cache.stride(), cache.dtype, k.shape, k.stride(), k.dtype, k.device, v.shape,
               v.stride(), v.dtype, v.device, rows.shape, rows.stride(), rows.dtype, rows.device, positions.shape,
               positions.stride(), positions.dtype, positions.device, table.shape, table.stride(), table.dtype,
               table.device)
        at, k_at, v_at = cache.data_ptr(), k.data_ptr(), v.data_ptr()
        args = None if (at | k_at | v_at) & 15 else _checked.get(key)
    except (AttributeError, TypeError):
        key = args = None
    c, t, tokens, dt, ks, vs = args or _remember(key, _check_append(cache, k, v, rows, positions, table))
    _launch(dev, "entmax_cache_append", _lib.entmax_cache_append, c, at, t, table.data_ptr(), tokens, dt,
            rows.data_ptr(), positions.data_ptr(), k_at, ks, v_at, vs)


def _check_read(cache, rows, positions, table, dtype, k_out, v_out):
    c, t = _check_places(cache, rows, positions, table)
    shape, dev = (rows.shape[0], c.kv_heads, c.head_dim), cache.device
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dtype must be bfloat16 or float32, not %s" % dtype)
    for name, out in (("k_out", k_out), ("v_out", v_out)):
        if out is not None:
            _strided(out, name, shape, dtype, dev, written=True)
            for other_name, other in (("cache", cache), ("table", table), ("rows", rows), ("positions", positions)):
                if _overlap(out, other):
                    raise ValueError("%s overlaps %s" % (name, other_name))
    if k_out is not None and v_out is not None and _overlap(k_out, v_out) and not _apart(k_out, v_out):
        raise ValueError("k_out overlaps v_out")
    _on_gpu(dev)
    return c, t, shape, EA_BF16 if dtype == torch.bfloat16 else EA_F32, _strides_of(c.kv_heads * c.head_dim, c.head_dim)


def cache_read(cache, rows, positions, table, dtype=torch.bfloat16, k_out=None, v_out=None):
    """(k, v) [tokens, kv_heads, head_dim]: the values that a layer's cache holds for the
    tokens positions[i] of the table's rows rows[i], 0 where there is no page.
    dtype: bfloat16 or float32, exact in both.  k_out, v_out: tensors to write."""
    try:
        dev = cache.device
        key = ("read", dev, dtype, cache.shape, cache.stride(), cache.dtype, rows.shape, rows.stride(), rows.dtype,
               rows.device, positions.shape, positions.stride(), positions.dtype, positions.device, table.shape,
               table.stride(), table.dtype, table.device)
        # (tensors to write are checked each time: whether they overlap is where they lie)
        at = cache.data_ptr()
        args = None if k_out is not None or v_out is not None or at & 15 else _checked.get(key)
    except (AttributeError, TypeError):
        key = args = None
    c, t, shape, dt, strides = args or _remember(key, _check_read(cache, rows, positions, table, dtype, k_out, v_out))
    ks = vs = strides
    if k_out is None:
        k_out = torch.empty(shape, dtype=dtype, device=dev)
    else:
        ks = _row_head(k_out)
    if v_out is None:
        v_out = torch.empty_like(k_out) if ks is strides else torch.empty(shape, dtype=dtype, device=dev)
    else:
        vs = _row_head(v_out)
    _launch(dev, "entmax_cache_read", _lib.entmax_cache_read, c, at, t, table.data_ptr(), shape[0], dt,
            rows.data_ptr(), positions.data_ptr(), k_out.data_ptr(), ks, v_out.data_ptr(), vs)
    return k_out, v_out


@functools.lru_cache(maxsize=256)
def _cache_workspace(c_shape, rows):
    n = ctypes.c_size_t()
    _check(_lib.entmax_cache_workspace(_cache_of(c_shape), rows, ctypes.byref(n)), "entmax_cache_workspace")
    return n.value


def cache_workspace(cache, rows):
    """Bytes of the workspace of cache_update for that many new rows, or of
    cache_compact for a table of as many."""
    _layers(cache)
    return _cache_workspace(cache.shape[-5:], int(rows))


def _written(outs, inputs):
    """Raises ValueError where one of outs (name, tensor) overlaps another or an input."""
    for n, (name, out) in enumerate(outs):
        for other_name, other in outs[n + 1:] + inputs:
            if _overlap(out, other):
                raise ValueError("%s overlaps %s" % (name, other_name))


def _check_table_out(table_out, rows, c, t, dev):
    if not isinstance(table_out, torch.Tensor) or table_out.shape != (rows, t.width):
        raise ValueError("table_out must be a %s tensor" % ([rows, t.width],))
    if rows:
        _table(table_out, c, dev, "table_out")
    if rows > 1 and table_out.stride(0) < t.width:
        raise ValueError("table_out has elements that share memory")


def _check_update(cache, table, lengths, parents, counts, table_out, lengths_out, missing_out, workspace):
    c, layers = _layers(cache)
    dev = cache.device
    t = _table(table, c, dev)
    _need(lengths, "lengths", (t.rows,), torch.int32, dev)
    if not isinstance(parents, torch.Tensor) or parents.dim() != 1:
        raise ValueError("parents must be a [rows] tensor")
    rows = parents.shape[0]
    _need(parents, "parents", (rows,), torch.int32, dev)
    _need(counts, "counts", (rows,), torch.int32, dev)
    if table_out is not None or lengths_out is not None or missing_out is not None:
        if table_out is None or lengths_out is None or missing_out is None:
            raise ValueError("table_out, lengths_out and missing_out must be given together")
        _check_table_out(table_out, rows, c, t, dev)
        _need(lengths_out, "lengths_out", (rows,), torch.int32, dev)
        _need(missing_out, "missing_out", (rows,), torch.int32, dev)
        _written([("table_out", table_out), ("lengths_out", lengths_out), ("missing_out", missing_out)],
                 [("table", table), ("lengths", lengths), ("parents", parents), ("counts", counts), ("cache", cache)])
    nbytes = _cache_workspace(cache.shape[-5:], rows)
    if workspace is not None:
        _check_bytes(workspace, "workspace", nbytes, dev)
    _on_gpu(dev)
    return c, layers, t, rows, nbytes


def cache_update(cache, table, lengths, parents, counts, table_out=None, lengths_out=None, missing_out=None,
                 workspace=None):
    """(table_out, lengths_out, missing_out): the table of the next step.  Its row r
    goes on from row parents[r] of the table, of lengths[parents[r]] tokens (from none,
    where that is no row), and gains counts[r] tokens (loses its last ones, where
    negative), for which it gets pages; all are int32 tensors on the device.

    Rows may go on from the same row: they share its pages, and where a row is
    about to write to a page that others hold as well, it gets a copy in every
    layer (cache: a model's, or one layer's).  Where all rows that hold a page are
    about to write to it, one keeps it: the lowest, or, with fewer free pages than all
    rows need, the one whose tokens end furthest into it.  Pages that no new row
    holds are free; they are given out lowest first, row by row.  Entries behind a
    row's pages are -1.

    A row gets all of its pages or none: missing_out[r] is 0, or the pages that it
    needed where the rows up to it needed more than are free (one that gets none counts
    for those behind it all the same), or -1 where its tokens do not fit the table.
    Such a row keeps its tokens and gains none: leave it out of the step's
    cache_append (negative positions), which would write over its last tokens.

    table_out [rows, width], lengths_out, missing_out [rows]: tensors to write, whose
    ranges of memory do not meet those of the tensors that the call reads.
    workspace: cache_workspace bytes, to keep from call to call (one call at a time)."""
    given = table_out is not None or lengths_out is not None or missing_out is not None or workspace is not None
    try:
        dev = cache.device
        key = ("update", dev, cache.shape, cache.stride(), cache.dtype, table.shape, table.stride(), table.dtype,
               table.device, lengths.shape, lengths.stride(), lengths.dtype, lengths.device, parents.shape,
               parents.stride(), parents.dtype, parents.device, counts.shape, counts.stride(), counts.dtype,
               counts.device)
        at = cache.data_ptr()
        args = None if given or at & 15 else _checked.get(key)
    except (AttributeError, TypeError):
        key = args = None
    c, layers, t, rows, nbytes = args or _remember(key, _check_update(
        cache, table, lengths, parents, counts, table_out, lengths_out, missing_out, workspace))
    out_stride = t.width
    if table_out is None:
        table_out = parents.new_empty((rows, t.width))
        lengths_out, missing_out = torch.empty_like(parents), torch.empty_like(parents)
    else:
        out_stride = max(_stride(table_out, 0), out_stride)
    if workspace is None:
        workspace = cache.new_empty(nbytes)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _launch(dev, "entmax_cache_update", _lib.entmax_cache_update, c, layers, at, t, table.data_ptr(),
            lengths.data_ptr(), rows, parents.data_ptr(), counts.data_ptr(), table_out.data_ptr(), out_stride,
            lengths_out.data_ptr(), missing_out.data_ptr(), workspace.data_ptr(), nbytes)
    return table_out, lengths_out, missing_out


def _check_compact(cache, table, lengths, table_out, used_out, workspace):
    c, layers = _layers(cache)
    dev = cache.device
    t = _table(table, c, dev)
    _need(lengths, "lengths", (t.rows,), torch.int32, dev)
    if (table_out is None) != (used_out is None):
        raise ValueError("table_out and used_out must be given together")
    if table_out is not None:
        _check_table_out(table_out, t.rows, c, t, dev)
        _need(used_out, "used_out", (1,), torch.int32, dev)
        _written([("table_out", table_out), ("used_out", used_out)],
                 [("table", table), ("lengths", lengths), ("cache", cache)])
    nbytes = _cache_workspace(cache.shape[-5:], t.rows)
    if workspace is not None:
        _check_bytes(workspace, "workspace", nbytes, dev)
    _on_gpu(dev)
    return c, layers, t, nbytes


def cache_compact(cache, table, lengths, table_out=None, used_out=None, workspace=None):
    """(table_out, used_out): the table, its rows of lengths[r] tokens, after all pages in
    use have moved to the lowest numbers, in every layer; used_out (int32 [1]) is their
    count, so that pages from there on are free.  Pages that are below it already
    stay.  table_out, used_out: tensors to write, which are not the call's inputs."""
    given = table_out is not None or used_out is not None or workspace is not None
    try:
        dev = cache.device
        key = ("compact", dev, cache.shape, cache.stride(), cache.dtype, table.shape, table.stride(), table.dtype,
               table.device, lengths.shape, lengths.stride(), lengths.dtype, lengths.device)
        at = cache.data_ptr()
        args = None if given or at & 15 else _checked.get(key)
    except (AttributeError, TypeError):
        key = args = None
    c, layers, t, nbytes = args or _remember(key, _check_compact(cache, table, lengths, table_out, used_out, workspace))
    out_stride = t.width
    if table_out is None:
        table_out, used_out = lengths.new_empty((t.rows, t.width)), lengths.new_empty(1)
    else:
        out_stride = max(_stride(table_out, 0), out_stride)
    if workspace is None:
        workspace = cache.new_empty(nbytes)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _launch(dev, "entmax_cache_compact", _lib.entmax_cache_compact, c, layers, at, t, table.data_ptr(),
            lengths.data_ptr(), table_out.data_ptr(), out_stride, used_out.data_ptr(), workspace.data_ptr(), nbytes)
    return table_out, used_out


@functools.lru_cache(maxsize=256)
def _paged_of(alpha, scale, max_iter, tol, c_shape, *sizes):
    """(PagedShape, Params, bytes of the workspace) of a call."""
    c, shape, n = _cache_of(c_shape), PagedShape(*sizes), ctypes.c_size_t()
    params = make_params(alpha, scale, False, False, max_iter, tol, head_dim=c.head_dim)
    _check(_lib.entmax_paged_decode_workspace(shape, c, ctypes.byref(n)), "entmax_paged_decode_workspace")
    return shape, params, n.value


def _longest(table, c, max_length):
    most = table.shape[1] * c.page_size
    return most if max_length is None else min(most, max(0, int(max_length)))


def paged_decode_workspace(q, cache, table, max_length=None):
    """Bytes of the workspace of paged_decode for these tensors (8 bytes for every query
    head and key that the table, or max_length, allows; few of them are written)."""
    c = _layer(cache)
    return _paged_of(1.5, None, None, None, cache.shape, q.shape[0], q.shape[1], _ea_dtype(q, "q"),
                     _longest(table, c, max_length))[2]


def _check_paged(q, cache, table, lengths, rows, numbers, max_length, out, workspace):
    c = _layer(cache)
    dev = cache.device
    t = _table(table, c, dev)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [queries, heads, head_dim] tensor")
    dt = _ea_dtype(q, "q")
    n, heads, d = q.shape
    if d != c.head_dim:
        raise ValueError("q has head_dim %d, the cache %d" % (d, c.head_dim))
    if heads < 1 or heads % c.kv_heads:
        raise ValueError("q's %d heads must be a multiple of the cache's %d" % (heads, c.kv_heads))
    _strided(q, "q", q.shape, q.dtype, dev)
    _need(lengths, "lengths", (n,), torch.int32, dev)
    if rows is not None:
        _need(rows, "rows", (n,), torch.int32, dev)
    elif n > t.rows:
        raise ValueError("q has %d queries, the table %d rows: give rows" % (n, t.rows))
    if out is not None:
        _strided(out, "out", q.shape, q.dtype, dev, written=True)
        _written([("out", out)], [("q", q), ("cache", cache), ("table", table), ("lengths", lengths)] +
                 ([] if rows is None else [("rows", rows)]))
    shape, params, nbytes = _paged_of(*numbers, cache.shape, n, heads, dt, _longest(table, c, max_length))
    if workspace is not None:
        _check_bytes(workspace, "workspace", nbytes, dev)
    _on_gpu(dev)
    return shape, params, c, t, _row_head(q), _strides_of(heads * d, d), max(nbytes, 16)


def paged_decode(q, cache, table, lengths, rows=None, alpha=1.5, scale=None, max_iter=None, tol=None, out=None,
                 workspace=None, max_length=None):
    """O [queries, heads, head_dim] of q [queries, heads, head_dim] (bf16 or fp32, any strides
    with a contiguous last dimension): query i attends to the first lengths[i] tokens
    (int32 on the device) of the table's row rows[i] (None: row i) in a layer's
    cache.  Several queries may have the same row, with lengths of their own (the
    last tokens of a draft).  A query without any key has O = 0, and so has one
    whose largest score is not finite.  1 < alpha <= 2.

    max_length: no query has more keys (default: what the table holds; grids and
    workspace, 8 bytes for every query head and key, grow with it, and only up to 2048 is
    a short row's call one launch).  tol: default 1e-6.  workspace: a device buffer of
    paged_decode_workspace bytes, to keep from call to call (one call at a time)."""
    numbers = _numbers(alpha, scale, max_iter, 1e-6 if tol is None else tol)
    max_length = None if max_length is None else int(max_length)
    try:
        dev = cache.device
        key = ("paged", dev, numbers, max_length, cache.shape, cache.stride(), cache.dtype, q.shape, q.stride(), q.dtype,
               q.device, table.shape, table.stride(), table.dtype, table.device, lengths.shape, lengths.stride(),
               lengths.dtype, lengths.device, rows is not None and (rows.shape, rows.stride(), rows.dtype, rows.device))
        at, q_at = cache.data_ptr(), q.data_ptr()
        args = None if out is not None or workspace is not None or (at | q_at) & 15 else _checked.get(key)
    except (AttributeError, TypeError):
        key = args = None
    shape, params, c, t, qs, os_, nbytes = args or _remember(key, _check_paged(
        q, cache, table, lengths, rows, numbers, max_length, out, workspace))
    if out is None:
        out = q.new_empty(q.shape)
    else:
        os_ = _row_head(out)
    if workspace is None:
        workspace = cache.new_empty(nbytes)
    else:
        nbytes = workspace.numel() * workspace.element_size()
    _launch(dev, "entmax_paged_decode", _lib.entmax_paged_decode, shape, params, c, at, t, table.data_ptr(), q_at, qs,
            lengths.data_ptr(), None if rows is None else rows.data_ptr(), out.data_ptr(), os_, workspace.data_ptr(),
            nbytes)
    return out
