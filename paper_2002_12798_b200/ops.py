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

import contextlib
import ctypes
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


def _current(stream, device):
    """(stream object, context in which tensors are made for it)."""
    if stream is None:
        return torch.cuda.current_stream(device), contextlib.nullcontext()
    return stream, torch.cuda.stream(stream)


def _ints(name, t, shape):
    if t.dtype is not torch.int32 or not t.is_cuda or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: a contiguous int32 CUDA tensor of shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def _table(t):
    if t.dtype is not torch.int32 or not t.is_cuda or t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("block_table: an int32 CUDA tensor [requests, pages] with contiguous rows")


# ----------------------------------------------------------------------------------------------------------------------
# pages
# ----------------------------------------------------------------------------------------------------------------------
PagesStep = namedtuple("PagesStep", "query_start slots positions requests seq_lens free_count status")


def pages_extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens, *, n_pages=None, out=None, stream=None):
    """Gives every request room for new_lens[r] more tokens (amap_pages_extend).

    new_lens, seq_lens: int32 [R]; block_table: int32 [R, pages], extended in place; free_pages: int32 stack of free
    page numbers, of which the first free_count[0] count; n_pages: page numbers lie below it (default: the length of
    free_pages).  Returns a PagesStep of int32 tensors: query_start [R+1]; slots, positions, requests [max_tokens]
    (-1, 0, -1 behind the last token); seq_lens [R] and free_count [1], to be used from now on in place of the inputs
    (which are unchanged); status [R] (0 granted, 1 too long, 2 no pages, 3 no room in the step).  `out`: a PagesStep
    to write to."""
    _table(block_table)
    n, row = block_table.shape
    device = block_table.device
    s, made = _current(stream, device)
    if out is None:
        with made:
            whole = torch.empty(3 * n + 2 + 3 * max_tokens, dtype=torch.int32, device=device)
        out = PagesStep(*whole.split([n + 1, max_tokens, max_tokens, max_tokens, n, 1, n]))
    capacity = free_pages.numel()
    one = (1,)
    per_request, per_token = (n,), (max_tokens,)
    args = _EXTEND.pack(
        n, row, page_size, capacity if n_pages is None else n_pages, capacity, max_tokens, block_table.stride(0),
        _ints("new_lens", new_lens, per_request), _ints("seq_lens", seq_lens, per_request), block_table.data_ptr(),
        _ints("free_pages", free_pages, (capacity,)), _ints("free_count", free_count, one),
        _ints("query_start", out.query_start, (n + 1,)), _ints("slots", out.slots, per_token),
        _ints("positions", out.positions, per_token), _ints("requests", out.requests, per_token),
        _ints("seq_lens", out.seq_lens, per_request), _ints("free_count", out.free_count, one), _ints("status", out.status, per_request))
    _check(_lib.amap_pages_extend(args, s.cuda_stream), "amap_pages_extend")
    return out


def pages_release(done, seq_lens, block_table, free_pages, free_count, page_size, *, stream=None):
    """Puts the pages of the requests with done[r] (bool or uint8 [R]) back on the stack free_pages, in place
    (amap_pages_release).  Returns (seq_lens, free_count) to be used from now on in place of the inputs."""
    _table(block_table)
    n, row = block_table.shape
    device = block_table.device
    _require(done.dtype in (torch.bool, torch.uint8) and done.is_cuda and done.shape == (n,) and done.is_contiguous(),
             "done: a contiguous bool or uint8 CUDA tensor [requests]")
    s, made = _current(stream, device)
    with made:
        whole = torch.empty(n + 1, dtype=torch.int32, device=device)
    seq_out, count_out = whole.split([n, 1])
    capacity = free_pages.numel()
    args = _RELEASE.pack(n, row, page_size, capacity, block_table.stride(0), done.data_ptr(), _ints("seq_lens", seq_lens, (n,)),
                         block_table.data_ptr(), _ints("free_pages", free_pages, (capacity,)), _ints("free_count", free_count, (1,)),
                         seq_out.data_ptr(), count_out.data_ptr())
    _check(_lib.amap_pages_release(args, s.cuda_stream), "amap_pages_release")
    return seq_out, count_out


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
    if not x.is_cuda or x.dim() != 3 or x.shape[2] != dim or x.stride(2) != 1:
        raise ValueError("%s: a CUDA tensor [tokens, heads, %d] whose heads are contiguous" % (name, dim))


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, positions, inverse, stream, *xs):
        ctx.save_for_backward(positions)
        ctx.plan, ctx.inverse = plan, inverse
        return tuple(plan._rotate(xs, positions, inverse, None, stream))

    @staticmethod
    def backward(ctx, *grads):
        (positions,) = ctx.saved_tensors
        grads = [g if g.stride(2) == 1 else g.contiguous() for g in grads]
        return (None, None, None, None) + tuple(ctx.plan._rotate(grads, positions, not ctx.inverse, None, None))


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

    def _positions(self, positions, tokens):
        """(pointer, stride of an axis, stride of a token, bits) of int32 / int64 positions [tokens] or [axes, tokens]."""
        d = positions.dim()
        if not positions.is_cuda or d not in (1, 2) or positions.shape[-1] != tokens or (d == 2 and positions.shape[0] < self.n_axes) \
                or (d == 1 and self.n_axes > 1):
            raise ValueError("positions: a CUDA tensor [%stokens] with one position per token" % ("axes, " if self.n_axes > 1 else ""))
        bits = 32 if positions.dtype is torch.int32 else 64 if positions.dtype is torch.int64 else 0
        _require(bits, "positions: int32 or int64")
        return positions.data_ptr(), positions.stride(0) if d == 2 else 0, positions.stride(-1), bits

    def _rotate(self, xs, positions, inverse, outs, stream):
        _require(1 <= len(xs) <= 4, "rotate takes 1 to 4 tensors")
        first = xs[0]
        dtype = _DTYPES.get(first.dtype, 0)
        s, made = _current(stream, first.device)
        if outs is None:
            with made:
                outs = [torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in xs]
        _require(len(outs) == len(xs), "outs: one per tensor")
        parts = []
        for x, y in zip(xs, outs):
            _heads("x", x, self.head_dim)
            _heads("out", y, self.head_dim)
            _require(x.dtype is first.dtype and y.dtype is x.dtype and x.shape[0] == first.shape[0] and y.shape == x.shape
                     and x.device == first.device, "rotate: tensors of one type and token count, each with an output like itself")
            parts.append(_PART.pack(x.data_ptr(), y.data_ptr(), x.stride(0), x.stride(1), y.stride(0), y.stride(1), x.shape[1], 0))
        tokens = first.shape[0]
        p, axis, row, bits = self._positions(positions, tokens)
        if tokens == 0:
            return outs
        args = _ROTATE.pack(len(parts), dtype, tokens, p, axis, row, bits, 1 if inverse else 0) + b"".join(parts)
        args += bytes((4 - len(parts)) * _PART.size)
        _check(_lib.amap_rope_rotate(self._h, args, s.cuda_stream), "amap_rope_rotate")
        return outs

    def rotate(self, xs, positions, *, inverse=False, outs=None, stream=None):
        """Turns up to four tensors [tokens, heads, head_dim] (q and k) by the same positions in one launch; returns
        the results in a list.  inverse=True turns back, which is the gradient; tensors that require one are
        differentiated through.  outs: tensors to write to (an x itself for in place)."""
        if torch.is_grad_enabled() and any(x.requires_grad for x in xs):
            _require(outs is None, "rotate: no outs where a gradient is required")
            return list(_Rotate.apply(self, positions, inverse, stream, *xs))
        return self._rotate(xs, positions, inverse, outs, stream)

    def append(self, q, k, v, positions, slots, cache, *, out=None, stream=None):
        """One step of a decoder layer before its attention (amap_rope_append): returns the rotated q [tokens, heads,
        head_dim] and writes the rotated k and the v [tokens, cache.heads, head_dim] to the slots (int32 [tokens], -1
        for none) of the cache.  Views of a fused projection are taken as they are.  Not differentiable."""
        dim = self.head_dim
        _heads("q", q, dim)
        _heads("k", k, dim)
        _heads("v", v, dim)
        tokens = q.shape[0]
        _require(k.shape == v.shape and k.shape[0] == tokens and k.shape[1] == cache.heads and k.dtype is q.dtype and v.dtype is q.dtype,
                 "append: q, k and v of one type and token count, k and v with the cache's heads")
        _require(q.device == cache.device, "append: the cache is on another device")
        s, made = _current(stream, q.device)
        if out is None:
            with made:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            _heads("out", out, dim)
            _require(out.shape == q.shape and out.dtype is q.dtype, "out: like q")
        p, axis, row, bits = self._positions(positions, tokens)
        at = _ints("slots", slots, (tokens,))
        if tokens == 0:
            return out
        args = _APPEND.pack(tokens, _DTYPES.get(q.dtype, 0), q.shape[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                            q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1), out.stride(0), out.stride(1),
                            p, axis, row, bits, 0, at) + cache._args
        _check(_lib.amap_rope_append(self._h, args, s.cuda_stream), "amap_rope_append")
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
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        n, failed = c_int64(), c_int64()
        with torch.cuda.device(self.device):
            _check(_lib.amap_attend_workspace(max_requests, q_heads, kv_heads, head_dim, byref(n), byref(failed)), "amap_attend_workspace")
            self._bytes, self._failed = n.value, failed.value
            self._stream = torch.cuda.current_stream()
            self._workspace = torch.zeros(self._bytes, dtype=torch.uint8, device=self.device)
        self._raw = self._stream.cuda_stream

    def failed(self):
        """Whether a wait inside a kernel of this plan has ever run out (after two seconds: its outputs are worth
        nothing).  Waits for the device."""
        torch.cuda.synchronize(self.device)
        return bool(self._workspace[self._failed : self._failed + 4].any())

    def _order(self, s):
        if torch.cuda.is_current_stream_capturing():
            return
        s.wait_stream(self._stream)
        self._workspace.record_stream(s)
        self._stream, self._raw = s, s.cuda_stream

    def attend(self, q, cache, block_table, seq_lens, *, out=None, return_lse=False, stream=None):
        """q: [requests, q_heads, head_dim]; row r is the newest token of the request in row r of block_table (int32
        [requests, pages]), which holds seq_lens[r] tokens (int32), the newest included.  Returns the output, shaped
        like q; with return_lse=True also the fp32 logarithm of the softmax's sum [requests, q_heads].  A request
        without tokens gets zeros and -inf."""
        _heads("q", q, self.head_dim)
        _table(block_table)
        n = q.shape[0]
        if n > self.max_requests or q.shape[1] != self.q_heads or cache.heads != self.kv_heads or cache.head_dim != self.head_dim:
            raise ValueError("attend: at most %d requests of %d heads of %d, %d heads in the cache"
                             % (self.max_requests, self.q_heads, self.head_dim, self.kv_heads))
        _require(block_table.shape[0] == n, "block_table: a row per request")
        _require(q.device == self.device and cache.device == self.device, "attend: plan, q and cache on one device")
        s, made = _current(stream, self.device)
        with made:
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            else:
                _heads("out", out, self.head_dim)
                _require(out.shape == q.shape and out.dtype is q.dtype, "out: like q")
            lse = torch.empty((n, self.q_heads), dtype=torch.float32, device=q.device) if return_lse else None
            if n:
                if s.cuda_stream != self._raw:
                    self._order(s)
                args = _ATTEND.pack(n, self.q_heads, _DTYPES.get(q.dtype, 0), block_table.shape[1], q.data_ptr(), out.data_ptr(),
                                    lse.data_ptr() if return_lse else 0, q.stride(0), q.stride(1), out.stride(0), out.stride(1), self.q_heads,
                                    block_table.data_ptr(), block_table.stride(0), _ints("seq_lens", seq_lens, (n,)), self.scale, self.softcap,
                                    self.window, 0, self._workspace.data_ptr(), self._bytes, cache._maps_at) + cache._args
                _check(_lib.amap_attend(args, s.cuda_stream), "amap_attend")
        return (out, lse) if return_lse else out
