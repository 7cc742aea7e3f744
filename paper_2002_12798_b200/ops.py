"""Operators on the heads that a composed map has split: rotary positions, a paged key/value cache, and the attention
of one new token per request (include/amap_serve.h has the definitions; this module marshals arguments).

One decoding step, for every layer the last two lines:

    step = ops.pages_extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens)
    q = rope.append(q, k, v, step.positions, step.slots, cache)
    out = attention.attend(q, cache, block_table, step.seq_lens)

Calls enqueue one kernel on the current CUDA stream (or `stream`) and neither synchronise nor copy to the host, so a
step can be captured in a CUDA graph.  Tensors a call is given must stay alive and unchanged until that stream has run
it; tensors it makes belong to that stream.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from collections import namedtuple
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_void_p

import torch

from .binding import AmapError, LIBRARY_PATH

EXPORTS = [
    "amap_pages_extend", "amap_pages_release", "amap_rope_plan", "amap_rope_destroy", "amap_rope_rotate",
    "amap_rope_append", "amap_cache_encode", "amap_attend", "amap_attend_workspace",
    "amap_serve_error",
]
_BF16, _FP16, _FP32, _E4M3 = 1, 2, 3, 4
_DTYPES = {torch.bfloat16: _BF16, torch.float16: _FP16, torch.float32: _FP32, torch.float8_e4m3fn: _E4M3}
_PAIRS = {"half": 0, "adjacent": 1}

# The argument structs are packed with struct's native alignment, which is C's, and passed by address: a fifth of what
# filling a ctypes.Structure costs, which is felt in a step of small kernels.  Names as in amap_serve.h.
_EXTEND = struct.Struct("6iq12P")  # amap_pages_extend_args
_RELEASE = struct.Struct("4iq7P")  # amap_pages_release_args
_ROTATE = struct.Struct("2iqP2q2i")  # amap_rope_args up to part[]
_PART = struct.Struct("2P4q2i")  # amap_rope_part
_APPEND = struct.Struct("q2i4P8qP2q2iP")  # amap_append_args up to cache
_ATTEND = struct.Struct("4i3P5qPqP2f2iPqP")  # amap_attend_args up to cache
_CACHE = struct.Struct("2P6q4ii2f4x")  # amap_cache
_MAPS = struct.Struct("32Q2i")  # amap_cache_maps


def _load():
    lib = ctypes.PyDLL(LIBRARY_PATH)  # calls enqueue and return: not worth giving up the interpreter lock
    lib.amap_serve_error.restype = c_char_p
    lib.amap_serve_error.argtypes = []
    for name in ("amap_pages_extend", "amap_pages_release"):
        getattr(lib, name).argtypes = [c_char_p, c_void_p]
    for name in ("amap_rope_rotate", "amap_rope_append"):
        getattr(lib, name).argtypes = [c_void_p, c_char_p, c_void_p]
    lib.amap_attend.argtypes = [c_char_p, c_void_p]
    lib.amap_cache_encode.argtypes = [c_char_p, c_void_p]
    lib.amap_attend_workspace.argtypes = [c_int32, c_int32, c_int32, c_int32, POINTER(c_int64), POINTER(c_int64)]
    lib.amap_rope_plan.argtypes = [c_int32, c_int32, POINTER(c_double), POINTER(c_int32), c_int32, c_int32, c_float, POINTER(c_void_p)]
    lib.amap_rope_destroy.argtypes = [c_void_p]
    lib.amap_rope_destroy.restype = None
    for name in EXPORTS:
        getattr(lib, name)
    return lib


_lib = _load()


def _check(rc, where):
    if rc != 0:
        why = _lib.amap_serve_error().decode()
        raise AmapError(rc, "%s (%s)" % (where, why) if why else where)


def _require(ok, why):
    if not ok:
        raise ValueError(why)


_raw_stream = torch._C._cuda_getCurrentRawStream  # by device number: a fortieth of what a Stream object costs
_current_device = torch._C._cuda_getDevice


def _enqueues(call):
    """Adds `stream=None` to a call that works on the current stream: it is made the current one for the call, so that
    what the call allocates belongs to it, too."""

    @functools.wraps(call)
    def wrapped(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            return call(*args, **kw)

    return wrapped


def _stream_of(device):
    """The current stream of device number `device`, which has to be the current device: kernels are launched there."""
    if device != _current_device():
        raise ValueError("the tensors are on %s, the current device is another (torch.cuda.device)"
                         % ("cuda:%d" % device if device >= 0 else "the CPU"))
    return _raw_stream(device)


_INT32 = torch.int32


def _ints(name, t, n, device):
    """Address of n int32 numbers that lie side by side on device number `device`."""
    if t.dtype is not _INT32 or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: %d contiguous int32 numbers on the device of the other tensors" % (name, n))
    return t.data_ptr()


def _table(t):
    """(address, rows, entries of a row, stride of a row) of a block table."""
    if t.dtype is not _INT32 or not t.is_cuda or t.dim() != 2:
        raise ValueError("block_table: an int32 CUDA tensor [requests, pages]")
    (rows, entries), (stride, one) = t.shape, t.stride()
    if one != 1 and entries > 1:
        raise ValueError("block_table: rows are contiguous")
    return t.data_ptr(), rows, entries, stride if rows > 1 else max(stride, entries)


# ----------------------------------------------------------------------------------------------------------------------
# pages
# ----------------------------------------------------------------------------------------------------------------------
PagesStep = namedtuple("PagesStep", "query_start slots positions requests seq_lens free_count status")


@_enqueues
def pages_extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens, *, n_pages=None, out=None):
    """Gives every request room for new_lens[r] more tokens (amap_pages_extend).

    new_lens, seq_lens: int32 [R]; block_table: int32 [R, pages], extended in place; free_pages: int32 stack of free
    page numbers, of which the first free_count[0] count; n_pages: page numbers lie below it (default: the length of
    free_pages).  Returns a PagesStep of int32 tensors: query_start [R+1]; slots, positions, requests [max_tokens]
    (-1, 0, -1 behind the last token); seq_lens [R] and free_count [1], to be used from now on in place of the inputs
    (which are unchanged); status [R] (0 granted, 1 too long, 2 no pages, 3 no room in the step).  `out`: a PagesStep
    to write to."""
    table, n, row, stride = _table(block_table)
    device = block_table.get_device()
    raw = _stream_of(device)
    sizes = (n + 1, max_tokens, max_tokens, max_tokens, n, 1, n)
    if out is None:
        whole = torch.empty(3 * n + 2 + 3 * max_tokens, dtype=_INT32, device=block_table.device)
        out = PagesStep._make(whole.split_with_sizes(sizes))
        start = whole.data_ptr()
        slots = start + 4 * (n + 1)
        positions = slots + 4 * max_tokens
        requests = positions + 4 * max_tokens
        seq_out = requests + 4 * max_tokens
        to = (start, slots, positions, requests, seq_out, seq_out + 4 * n, seq_out + 4 * n + 4)
    else:
        to = tuple(_ints(name, t, m, device) for name, t, m in zip(PagesStep._fields, out, sizes))
    capacity = free_pages.numel()
    args = _EXTEND.pack(
        n, row, page_size, capacity if n_pages is None else n_pages, capacity, max_tokens, stride, _ints("new_lens", new_lens, n, device),
        _ints("seq_lens", seq_lens, n, device), table, _ints("free_pages", free_pages, capacity, device),
        _ints("free_count", free_count, 1, device), *to)
    rc = _lib.amap_pages_extend(args, raw)
    if rc:
        _check(rc, "amap_pages_extend")
    return out


@_enqueues
def pages_release(done, seq_lens, block_table, free_pages, free_count, page_size):
    """Puts the pages of the requests with done[r] (bool or uint8 [R]) back on the stack free_pages, in place
    (amap_pages_release).  Returns (seq_lens, free_count) to be used from now on in place of the inputs."""
    table, n, row, stride = _table(block_table)
    device = block_table.get_device()
    raw = _stream_of(device)
    if done.dtype not in (torch.bool, torch.uint8) or done.get_device() != device or done.numel() != n or not done.is_contiguous():
        raise ValueError("done: %d contiguous bool or uint8 values on the device of the other tensors" % n)
    whole = torch.empty(n + 1, dtype=_INT32, device=block_table.device)
    to = whole.data_ptr()
    capacity = free_pages.numel()
    args = _RELEASE.pack(n, row, page_size, capacity, stride, done.data_ptr(), _ints("seq_lens", seq_lens, n, device), table,
                         _ints("free_pages", free_pages, capacity, device), _ints("free_count", free_count, 1, device), to, to + 4 * n)
    rc = _lib.amap_pages_release(args, raw)
    if rc:
        _check(rc, "amap_pages_release")
    return tuple(whole.split_with_sizes((n, 1)))


# ----------------------------------------------------------------------------------------------------------------------
# the paged cache
# ----------------------------------------------------------------------------------------------------------------------
class PagedCache:
    """K and V as CUDA tensors [pages, page_size, heads, head_dim] of bf16, fp16 or float8_e4m3fn; any strides with the
    head's elements contiguous, so memory may also be ordered [pages, heads, page_size, head_dim] (pass the transposed
    view).  An element of an e4m3 cache stands for its value times k_scale / v_scale.  Keeps the tensors alive."""

    def __init__(self, k, v, *, k_scale=1.0, v_scale=1.0):
        _require(k.is_cuda and k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device,
                 "k and v: CUDA tensors [pages, page_size, heads, head_dim] of one shape and type")
        _require(_DTYPES.get(k.dtype) in (_BF16, _FP16, _E4M3), "cache: bfloat16, float16 or float8_e4m3fn")
        _require(k.stride(3) == 1 and v.stride(3) == 1, "cache: the elements of a head are contiguous")
        self.k, self.v, self.k_scale, self.v_scale = k, v, float(k_scale), float(v_scale)
        self.pages, self.page_size, self.heads, self.head_dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        self._args = _CACHE.pack(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], *k.shape, _DTYPES[k.dtype],
                                 self.k_scale, self.v_scale)
        self._maps = ctypes.create_string_buffer(_MAPS.size)  # for attention; a cache that it refuses is refused there
        readable = _lib.amap_cache_encode(self._args, self._maps) == 0
        self._maps_at = ctypes.addressof(self._maps) if readable else 0


# ----------------------------------------------------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------------------------------------------------
def _heads(name, x, dim):
    """((tokens, heads, dim), (stride of a token, stride of a head, 1)) of a tensor of heads."""
    shape, stride = x.shape, x.stride()
    if not x.is_cuda or len(shape) != 3 or shape[2] != dim or (stride[2] != 1 and dim > 1):
        raise ValueError("%s: a CUDA tensor [tokens, heads, %d] whose heads are contiguous" % (name, dim))
    return shape, stride


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, positions, inverse, *xs):
        ctx.save_for_backward(positions)
        ctx.plan, ctx.inverse = plan, inverse
        return tuple(plan._rotate(xs, positions, inverse, None))

    @staticmethod
    def backward(ctx, *grads):
        (positions,) = ctx.saved_tensors
        grads = [g if g.stride(2) == 1 else g.contiguous() for g in grads]
        return (None, None, None) + tuple(ctx.plan._rotate(grads, positions, not ctx.inverse, None))


class RopePlan:
    """Rotary positions of heads of `head_dim` elements, the first `rotary_dim` of which turn (amap_rope_plan).

    base / inv_freq: angle per position of pair i: base**(-2i/rotary_dim), or the given rotary_dim/2 values.
    axes: which row of `positions` each pair goes by (rotary_dim/2 numbers); sections=[a, b, c] is short for the first a
    pairs by row 0, the next b by row 1 and so on.  pairs: "half" couples elements i and i + rotary_dim/2, "adjacent"
    elements 2i and 2i+1.  scale multiplies the result's rotated part."""

    def __init__(self, head_dim, rotary_dim=None, *, base=10000.0, inv_freq=None, axes=None, sections=None, pairs="half", scale=1.0):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        half = rotary_dim // 2
        if inv_freq is None:
            inv_freq = [float(base) ** (-2.0 * i / rotary_dim) for i in range(half)]
        if sections is not None:
            _require(axes is None, "axes or sections, not both")
            axes = [a for a, n in enumerate(sections) for _ in range(n)]
        axes = [0] * half if axes is None else [int(a) for a in axes]
        inv_freq = [float(f) for f in inv_freq]
        _require(len(inv_freq) == half and len(axes) == half, "inv_freq, axes: rotary_dim/2 values")
        _require(pairs in _PAIRS, 'pairs: "half" or "adjacent"')
        self.head_dim, self.rotary_dim, self.n_axes = head_dim, rotary_dim, 1 + max(axes, default=0)
        self._h = None
        h = c_void_p()
        _check(_lib.amap_rope_plan(head_dim, rotary_dim, (c_double * max(half, 1))(*inv_freq), (c_int32 * max(half, 1))(*axes), self.n_axes,
                                   _PAIRS[pairs], scale, byref(h)), "amap_rope_plan")
        self._h = h.value

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:  # module globals are gone at interpreter shutdown
            _lib.amap_rope_destroy(self._h)
            self._h = None

    def _positions(self, positions, tokens, device):
        """(pointer, stride of an axis, stride of a token, bits) of int32 / int64 positions [tokens] or [axes, tokens]."""
        shape, stride = positions.shape, positions.stride()
        d = len(shape)
        if d not in (1, 2) or shape[-1] != tokens or (shape[0] if d == 2 else 1) < self.n_axes or positions.get_device() != device:
            raise ValueError("positions: [%stokens] with one position per token, on the device of the other tensors"
                             % ("axes, " if self.n_axes > 1 else ""))
        bits = 32 if positions.dtype is _INT32 else 64 if positions.dtype is torch.int64 else 0
        if not bits:
            raise ValueError("positions: int32 or int64")
        return positions.data_ptr(), stride[0] if d == 2 else 0, stride[-1], bits

    def _rotate(self, xs, positions, inverse, outs):
        n, dim = len(xs), self.head_dim
        _require(1 <= n <= 4, "rotate takes 1 to 4 tensors")
        first = xs[0]
        dtype, device, tokens = first.dtype, first.get_device(), first.shape[0]
        raw = _stream_of(device)
        if outs is None:
            outs = [torch.empty_like(x) for x in xs]
        _require(len(outs) == n, "outs: one per tensor")
        parts = b""
        for x, y in zip(xs, outs):
            shape, xs_ = _heads("x", x, dim)
            y_shape, ys_ = _heads("out", y, dim)
            if x.dtype is not dtype or y.dtype is not dtype or shape[0] != tokens or y_shape != shape or x.get_device() != device or y.get_device() != device:
                raise ValueError("rotate: tensors of one type, token count and device, each with an output like itself")
            parts += _PART.pack(x.data_ptr(), y.data_ptr(), xs_[0], xs_[1], ys_[0], ys_[1], shape[1], 0)
        at = self._positions(positions, tokens, device)
        if tokens == 0:
            return outs
        rc = _lib.amap_rope_rotate(self._h, _ROTATE.pack(n, _DTYPES.get(dtype, 0), tokens, *at, inverse) + parts + bytes((4 - n) * _PART.size), raw)
        if rc:
            _check(rc, "amap_rope_rotate")
        return outs

    @_enqueues
    def rotate(self, xs, positions, *, inverse=False, outs=None):
        """Turns up to four tensors [tokens, heads, head_dim] (q and k) by the same positions in one launch; returns
        the results in a list.  inverse=True turns back, which is the gradient; tensors that require one are
        differentiated through.  outs: tensors to write to (an x itself for in place)."""
        if torch.is_grad_enabled():
            for x in xs:
                if x.requires_grad:
                    _require(outs is None, "rotate: no outs where a gradient is required")
                    return list(_Rotate.apply(self, positions, bool(inverse), *xs))
        return self._rotate(xs, positions, bool(inverse), outs)

    @_enqueues
    def append(self, q, k, v, positions, slots, cache, *, out=None):
        """One step of a decoder layer before its attention (amap_rope_append): returns the rotated q [tokens, heads,
        head_dim] and writes the rotated k and the v [tokens, cache.heads, head_dim] to the slots (int32 [tokens], -1
        for none) of the cache.  Views of a fused projection are taken as they are.  Not differentiable."""
        dim, dtype, device = self.head_dim, q.dtype, q.get_device()
        raw = _stream_of(device)
        (tokens, heads, _), qs = _heads("q", q, dim)
        k_shape, ks = _heads("k", k, dim)
        v_shape, vs = _heads("v", v, dim)
        if k_shape != v_shape or k_shape[0] != tokens or k_shape[1] != cache.heads or k.dtype is not dtype or v.dtype is not dtype:
            raise ValueError("append: q, k and v of one type and token count, k and v with the cache's heads")
        if not device == k.get_device() == v.get_device() == cache.device.index:
            raise ValueError("append: q, k, v and the cache on one device")
        if out is None:
            out = torch.empty_like(q)
        out_shape, outs = _heads("out", out, dim)
        if out.dtype is not dtype or out_shape != q.shape or out.get_device() != device:
            raise ValueError("out: like q")
        at = self._positions(positions, tokens, device)
        where = _ints("slots", slots, tokens, device)
        if tokens == 0:
            return out
        args = _APPEND.pack(tokens, _DTYPES.get(dtype, 0), heads, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), qs[0], qs[1], ks[0],
                            ks[1], vs[0], vs[1], outs[0], outs[1], *at, 0, where) + cache._args
        rc = _lib.amap_rope_append(self._h, args, raw)
        if rc:
            _check(rc, "amap_rope_append")
        return out


# ----------------------------------------------------------------------------------------------------------------------
# attention of one new token per request
# ----------------------------------------------------------------------------------------------------------------------
class AttendPlan:
    """Decode attention for up to `max_requests` requests (amap_attend): owns the workspace in which the parts of a
    split cache are joined, so one plan serves all layers.  scale: of the scores (default 1/sqrt(head_dim)); window:
    each token sees the last `window` tokens (0: all); softcap: scores are softcap * tanh(score / softcap) (0: none).

    Calls of one plan run one after another, also when they come from different streams (the later stream is made to
    wait).  Inside a graph capture that order is the caller's: a plan captured in a graph should serve that graph."""

    def __init__(self, max_requests, q_heads, kv_heads, head_dim, *, scale=None, window=0, softcap=0.0, device=None):
        self.max_requests, self.q_heads, self.kv_heads, self.head_dim = max_requests, q_heads, kv_heads, head_dim
        self.scale = float(scale) if scale is not None else 1.0 / math.sqrt(head_dim)
        self.window, self.softcap = int(window), float(softcap)
        device = torch.device("cuda" if device is None else device)
        self.device = device if device.index is not None else torch.device("cuda", torch.cuda.current_device())
        n, failed = c_int64(), c_int64()
        with torch.cuda.device(self.device):
            _check(_lib.amap_attend_workspace(max_requests, q_heads, kv_heads, head_dim, byref(n), byref(failed)), "amap_attend_workspace")
            self._bytes, self._failed = n.value, failed.value
            self._stream = torch.cuda.current_stream()
            self._workspace = torch.zeros(self._bytes, dtype=torch.uint8, device=self.device)
            self._workspace_at = self._workspace.data_ptr()
        self._raw = self._stream.cuda_stream

    def failed(self):
        """Whether a wait inside a kernel of this plan has ever run out (after two seconds: its outputs are worth
        nothing).  Waits for the device."""
        torch.cuda.synchronize(self.device)
        return bool(self._workspace[self._failed : self._failed + 4].any())

    def _order(self):
        if torch.cuda.is_current_stream_capturing():
            return
        s = torch.cuda.current_stream(self.device)
        s.wait_stream(self._stream)
        self._workspace.record_stream(s)
        self._stream, self._raw = s, s.cuda_stream

    @_enqueues
    def attend(self, q, cache, block_table, seq_lens, *, out=None, return_lse=False):
        """q: [requests, q_heads, head_dim]; row r is the newest token of the request in row r of block_table (int32
        [requests, pages]), which holds seq_lens[r] tokens (int32), the newest included.  Returns the output, shaped
        like q; with return_lse=True also the fp32 logarithm of the softmax's sum [requests, q_heads].  A request
        without tokens gets zeros and -inf."""
        dim, device = self.head_dim, self.device.index
        raw = _stream_of(device)
        (n, heads, _), qs = _heads("q", q, dim)
        table, rows, entries, stride = _table(block_table)
        if n > self.max_requests or heads != self.q_heads or cache.heads != self.kv_heads or cache.head_dim != dim or rows != n:
            raise ValueError("attend: at most %d requests of %d heads of %d, %d heads in the cache, a table row per request"
                             % (self.max_requests, self.q_heads, dim, self.kv_heads))
        if not device == q.get_device() == cache.device.index == block_table.get_device():
            raise ValueError("attend: plan, q, block_table and cache on one device")
        if out is None:
            out = torch.empty_like(q)
        out_shape, outs = _heads("out", out, dim)
        if out.dtype is not q.dtype or out_shape != q.shape or out.get_device() != device:
            raise ValueError("out: like q")
        lse = torch.empty((n, heads), dtype=torch.float32, device=self.device) if return_lse else None
        if n:
            if raw != self._raw:
                self._order()
            args = _ATTEND.pack(n, heads, _DTYPES.get(q.dtype, 0), entries, q.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else 0, qs[0],
                                qs[1], outs[0], outs[1], heads, table, stride, _ints("seq_lens", seq_lens, n, device), self.scale, self.softcap,
                                self.window, 0, self._workspace_at, self._bytes, cache._maps_at) + cache._args
            rc = _lib.amap_attend(args, raw)
            if rc:
                _check(rc, "amap_attend")
        return (out, lse) if return_lse else out
