"""Operators on the heads that a composed map has split: rotary positions, a paged key/value cache, the attention of one
new token per request, and the choice of the next (include/amap_serve.h has the definitions; this module marshals arguments).

One decoding step, for every layer the lines from `append` on:

    step = ops.pages_extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens)
    q = rope.append(q, k, v, step.positions, step.slots, cache)
    rows = q.new_zeros(max_requests + 1, q_heads, 128)
    rows[step.requests.long()] = q
    out = attention.attend(rows[:-1], cache, block_table, step.seq_lens)

append takes the step's tokens, one behind the other; attend a row per request, of which some may have no token in the
step (idle, or refused).  Where every request has one, `rows` is q.  cache is a PagedCache (16 bits, or 8 with a scale) or a
PackedCache (4 bits, quantised as they are written).  Behind the last layer `sample` draws a token for every row of logits.

Calls enqueue one kernel on the current CUDA stream (or `stream`) and neither synchronise nor copy to the host, so a
step can be captured in a CUDA graph.  Tensors a call is given must stay alive and unchanged until that stream has run
it; tensors it makes belong to that stream.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.machinery
import importlib.util
import math
import threading
from collections import namedtuple
from ctypes import POINTER, Structure, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_uint64, c_void_p

import torch
from torch.autograd import forward_ad

from . import build as _build
from .binding import AmapError, LIBRARY_PATH

EXPORTS = [
    "amap_pages_extend", "amap_pages_release", "amap_pages_release_within", "amap_rope_plan", "amap_rope_destroy", "amap_rope_rotate",
    "amap_rope_append", "amap_cache_encode", "amap_attend", "amap_attend_workspace", "amap_serve_error", "amap_packed_bytes",
    "amap_packed_append", "amap_packed_read", "amap_packed_attend", "amap_sample",
]
_BF16, _FP16, _FP32, _E4M3 = 1, 2, 3, 4
_DTYPES = {torch.bfloat16: _BF16, torch.float16: _FP16, torch.float32: _FP32, torch.float8_e4m3fn: _E4M3}
_PAIRS = {"half": 0, "adjacent": 1}


# Plans and caches are described once, in C's structs (amap_serve.h has the fields); the calls themselves go through
# _serve_torch (csrc/serve_torch.cpp), which is given the structs' addresses.
class _Cache(Structure):  # amap_cache
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("strides", c_int64 * 6), ("n_pages", c_int32), ("page_size", c_int32), ("heads", c_int32),
                ("head_dim", c_int32), ("dtype", c_int32), ("k_scale", c_float), ("v_scale", c_float)]


class _Packed(Structure):  # amap_packed
    _fields_ = [("data", c_void_p), ("page", c_int64), ("head", c_int64), ("n_pages", c_int32), ("page_size", c_int32), ("heads", c_int32),
                ("head_dim", c_int32), ("group", c_int32), ("reserved", c_int32)]


class _Maps(Structure):  # amap_cache_maps
    _fields_ = [("maps", c_uint64 * 32), ("box_shift", c_int32), ("usable", c_int32)]


class _Attend(Structure):  # amap_attend_args
    _fields_ = [("n_requests", c_int32), ("q_heads", c_int32), ("dtype", c_int32), ("max_pages", c_int32), ("q", c_void_p), ("out", c_void_p),
                ("lse", c_void_p), ("strides", c_int64 * 5), ("block_table", c_void_p), ("table_stride", c_int64), ("seq_lens", c_void_p),
                ("scale", c_float), ("softcap", c_float), ("window", c_int32), ("reserved", c_int32), ("workspace", c_void_p),
                ("workspace_bytes", c_int64), ("maps", c_void_p), ("cache", _Cache)]


def _load():
    lib = ctypes.CDLL(LIBRARY_PATH)
    lib.amap_serve_error.restype = c_char_p
    lib.amap_serve_error.argtypes = []
    lib.amap_cache_encode.argtypes = [POINTER(_Cache), POINTER(_Maps)]
    lib.amap_attend_workspace.argtypes = [c_int32, c_int32, c_int32, c_int32, POINTER(c_int64), POINTER(c_int64)]
    lib.amap_packed_bytes.argtypes = [c_int32, c_int32, c_int32]
    lib.amap_packed_bytes.restype = c_int64
    lib.amap_rope_plan.argtypes = [c_int32, c_int32, POINTER(c_double), POINTER(c_int32), c_int32, c_int32, c_float, POINTER(c_void_p)]
    lib.amap_rope_destroy.argtypes = [c_void_p]
    lib.amap_rope_destroy.restype = None
    path = _build.build_torch_entry()
    loader = importlib.machinery.ExtensionFileLoader("_serve_torch", path)
    entry = importlib.util.module_from_spec(importlib.util.spec_from_file_location("_serve_torch", path, loader=loader))
    loader.exec_module(entry)
    entry.refuse_with(AmapError)
    return lib, entry


_lib, _entry = _load()
_raw_stream = torch._C._cuda_getCurrentRawStream  # by device number: a fortieth of what a Stream object costs


def _check(rc, where):
    if rc != 0:
        why = _lib.amap_serve_error().decode()
        raise AmapError(rc, "%s (%s)" % (where, why) if why else where)


def _require(ok, why):
    if not ok:
        raise ValueError(why)


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
    if stream is not None:
        with torch.cuda.stream(stream):  # current for the call, so that what the call makes belongs to it, too
            return pages_extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens, n_pages=n_pages, out=out)
    got = _entry.extend(new_lens, seq_lens, block_table, free_pages, free_count, page_size, max_tokens, n_pages, out)
    return out if out is not None else PagesStep._make(got)


def pages_release(done, seq_lens, block_table, free_pages, free_count, page_size, *, n_pages=None, stream=None):
    """Puts the pages of the requests with done[r] (bool or uint8 [R]) back on the stack free_pages, in place
    (amap_pages_release).  Negative table entries are holes and are passed over; with n_pages, so is every entry beyond
    its pages.  Returns (seq_lens, free_count) to be used from now on in place of the inputs."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return pages_release(done, seq_lens, block_table, free_pages, free_count, page_size, n_pages=n_pages)
    return _entry.release(done, seq_lens, block_table, free_pages, free_count, page_size, n_pages)


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
        self._args = _Cache(k.data_ptr(), v.data_ptr(), (c_int64 * 6)(*k.stride()[:3], *v.stride()[:3]), *k.shape, _DTYPES[k.dtype], self.k_scale,
                            self.v_scale)
        self._maps = _Maps()  # for attention, which refuses a cache that this refuses
        readable = _lib.amap_cache_encode(byref(self._args), byref(self._maps)) == 0
        self._at, self._maps_at, self._device = ctypes.addressof(self._args), ctypes.addressof(self._maps) if readable else 0, k.get_device()


class PackedCache:
    """K and V in 4 bits (amap_packed): a group of `group` (32 or 64) elements of a head is held as codes 0 .. 15 that stand for
    low + step * code, with low (the smallest element, rounded down) and step in bf16.  RopePlan.append quantises into it,
    AttendPlan.attend reads it as it is, `read` gives tokens back.

    data: uint8 CUDA tensor [pages, heads, page_bytes(page_size, head_dim, group)], of any strides that are multiples of 16
    with a page of a head contiguous; `zeros` makes one.  page_size is a multiple of 16, head_dim 64, 96, 128 or 256.
    Keeps the tensor alive."""

    def __init__(self, data, page_size, head_dim, *, group=64):
        size = self.page_bytes(page_size, head_dim, group)
        _require(data.is_cuda and data.dim() == 3 and data.dtype == torch.uint8 and data.shape[2] == size and data.stride(2) == 1,
                 "data: a uint8 CUDA tensor [pages, heads, %d] with contiguous pages of a head" % size)
        _require(data.data_ptr() % 16 == 0 and data.stride(0) % 16 == 0 and data.stride(1) % 16 == 0, "data: aligned to 16 bytes, as are its strides")
        self.data, self.page_size, self.head_dim, self.group = data, page_size, head_dim, group
        self.pages, self.heads, self.device = data.shape[0], data.shape[1], data.device
        self._args = _Packed(data.data_ptr(), data.stride(0), data.stride(1), self.pages, page_size, self.heads, head_dim, group, 0)
        self._at, self._maps_at, self._device = ctypes.addressof(self._args), 0, data.get_device()

    @classmethod
    def zeros(cls, pages, page_size, heads, head_dim, *, group=64, device="cuda"):
        """A cache of its own memory, all zeros."""
        return cls(torch.zeros(pages, heads, cls.page_bytes(page_size, head_dim, group), dtype=torch.uint8, device=device), page_size, head_dim, group=group)

    @staticmethod
    def page_bytes(page_size, head_dim, group=64):
        """Bytes that a page of one head takes (K and V)."""
        size = _lib.amap_packed_bytes(page_size, head_dim, group)
        _require(size > 0, _lib.amap_serve_error().decode())
        return size

    def write(self, k, v, slots, *, stream=None):
        """Quantises k and v (bf16 or fp16 [tokens, heads, head_dim]) as they are into the slots (int32 [tokens], -1 for none)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.write(k, v, slots)
        _entry.packed_write(k, v, slots, self._at, self._device)

    def read(self, slots, *, dtype=torch.bfloat16, out=None, stream=None):
        """What the cache holds at the slots (int32 [tokens]) as (k, v), each [tokens, heads, head_dim] of dtype (bf16, fp16 or
        fp32); zeros for a slot that there is not.  out: a pair to write to."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.read(slots, dtype=dtype, out=out)
        code = _DTYPES.get(dtype)
        _require(code in (_BF16, _FP16, _FP32), "read: bfloat16, float16 or float32")
        return _entry.packed_read(slots, self._at, self._device, code, None if out is None else tuple(out))


# ----------------------------------------------------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------------------------------------------------
def _tracked(tensors):
    """Whether autograd, backward or forward, follows one of the tensors."""
    if torch.is_grad_enabled():
        for x in tensors:
            if getattr(x, "requires_grad", False):  # what is no tensor is refused later
                return True
    if forward_ad._current_level >= 0 and torch._C._is_fwd_grad_enabled():
        return any(isinstance(x, torch.Tensor) and forward_ad.unpack_dual(x).tangent is not None for x in tensors)
    return False


class _NoDerivative(torch.autograd.Function):
    """A call that has none: its results are as without autograd, and asking for their derivative says so."""

    @staticmethod
    def forward(ctx, name, call, args, *inputs):
        ctx.name = name
        return call(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("%s is not differentiable" % ctx.name)

    @staticmethod
    def jvp(ctx, *tangents):
        raise RuntimeError("%s is not differentiable" % ctx.name)


def _without_derivative(name, call, args, out, *inputs):  # where the entry has launched nothing, as autograd follows an input
    _require(out is None, "%s: no out where a gradient is required" % name)
    return _NoDerivative.apply(name, call, args, *inputs)


class _Rotate(torch.autograd.Function):
    """The turn is linear and its own transpose with the angle negated: derivatives are turns again, of every order."""

    @staticmethod
    def forward(ctx, plan, positions, inverse, *xs):
        ctx.save_for_backward(positions)
        ctx.save_for_forward(positions)
        ctx.plan, ctx.inverse, ctx.like = plan, inverse, [(x.shape, x.dtype, x.device) for x in xs]
        return tuple(_entry.rotate(plan._h, plan.head_dim, plan.n_axes, xs, positions, inverse, None))

    @staticmethod
    def backward(ctx, *grads):
        (positions,) = ctx.saved_tensors
        grads = [g if g.stride(2) == 1 else g.contiguous() for g in grads]
        return (None, None, None, *_Rotate.apply(ctx.plan, positions, not ctx.inverse, *grads))

    @staticmethod
    def jvp(ctx, _plan, _positions, _inverse, *tangents):
        (positions,) = ctx.saved_tensors
        tangents = [torch.zeros(shape, dtype=dtype, device=device) if t is None else t if t.stride(2) == 1 else t.contiguous()
                    for t, (shape, dtype, device) in zip(tangents, ctx.like)]
        return tuple(_Rotate.apply(ctx.plan, positions, ctx.inverse, *tangents))


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
        self._made_of = inv_freq, axes, _PAIRS[pairs], scale
        self._make()

    def _make(self):
        self._h = None
        inv_freq, axes, pairs, scale = self._made_of
        n, h = max(len(axes), 1), c_void_p()
        _check(_lib.amap_rope_plan(self.head_dim, self.rotary_dim, (c_double * n)(*inv_freq), (c_int32 * n)(*axes), self.n_axes, pairs, scale, byref(h)),
               "amap_rope_plan")
        self._h = h.value

    # a copy (copy, deepcopy, pickle) makes a plan of its own: the handle has one owner
    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_h"}

    def __setstate__(self, state):
        self.__dict__.update(state)
        self._make()

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:  # module globals are gone at interpreter shutdown
            _lib.amap_rope_destroy(self._h)
            self._h = None

    def rotate(self, xs, positions, *, inverse=False, outs=None, stream=None):
        """Turns up to four tensors [tokens, heads, head_dim] (q and k) by the same positions in one launch; returns
        the results in a list.  inverse=True turns back, which is the gradient; tensors that require one are
        differentiated through, to any order and in either mode.  outs: tensors to write to (an x itself for in place)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.rotate(xs, positions, inverse=inverse, outs=outs)
        if _tracked(xs):
            _require(outs is None, "rotate: no outs where a gradient is required")
            return list(_Rotate.apply(self, positions, bool(inverse), *xs))
        return _entry.rotate(self._h, self.head_dim, self.n_axes, xs, positions, inverse, outs)

    def append(self, q, k, v, positions, slots, cache, *, out=None, stream=None):
        """One step of a decoder layer before its attention (amap_rope_append): returns the rotated q [tokens, heads,
        head_dim] and writes the rotated k and the v [tokens, cache.heads, head_dim] to the slots (int32 [tokens], -1
        for none) of the cache (a PackedCache: quantised as the exact rotation gives it).  Views of a fused projection are taken as they are.  Not differentiable: a result that
        autograd follows raises when its derivative is asked for."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.append(q, k, v, positions, slots, cache, out=out)
        entry = _entry.packed_append if isinstance(cache, PackedCache) else _entry.append
        got = entry(self._h, self.head_dim, self.n_axes, q, k, v, positions, slots, cache._at, cache._device, out)
        if got is NotImplemented:
            return _without_derivative("append", self.append, (q, k, v, positions, slots, cache), out, q, k, v)
        return got


# ----------------------------------------------------------------------------------------------------------------------
# attention of one new token per request
# ----------------------------------------------------------------------------------------------------------------------
class AttendPlan:
    """Decode attention for up to `max_requests` requests (amap_attend): owns the workspace in which the parts of a
    split cache are joined, so one plan serves all layers.  scale: of the scores (default 1/sqrt(head_dim)); window:
    each token sees the last `window` tokens (0: all); softcap: scores are softcap * tanh(score / softcap) (0: none).

    Calls of one plan run one after another, also when they come from different streams (the later stream is made to
    wait) or threads.  Inside a graph capture that order is the caller's: a plan captured in a graph should serve that graph."""

    def __init__(self, max_requests, q_heads, kv_heads, head_dim, *, scale=None, window=0, softcap=0.0, device=None):
        self.max_requests, self.q_heads, self.kv_heads, self.head_dim = max_requests, q_heads, kv_heads, head_dim
        self.scale = float(scale) if scale is not None else 1.0 / math.sqrt(head_dim)
        self.window, self.softcap = int(window), float(softcap)
        device = torch.device("cuda" if device is None else device)
        self.device = device if device.index is not None else torch.device("cuda", torch.cuda.current_device())
        self._make()

    def _make(self):
        n, failed = c_int64(), c_int64()
        with torch.cuda.device(self.device):
            _check(_lib.amap_attend_workspace(self.max_requests, self.q_heads, self.kv_heads, self.head_dim, byref(n), byref(failed)), "amap_attend_workspace")
            self._bytes, self._failed = n.value, failed.value
            self._stream = torch.cuda.current_stream()
            self._workspace = torch.zeros(self._bytes, dtype=torch.uint8, device=self.device)
        self._raw, self._lock = self._stream.cuda_stream, threading.Lock()
        self._args = _Attend(q_heads=self.q_heads, scale=self.scale, softcap=self.softcap, window=self.window, workspace=self._workspace.data_ptr(),
                             workspace_bytes=self._bytes, cache=_Cache(heads=self.kv_heads, head_dim=self.head_dim))
        self._at, self._device = ctypes.addressof(self._args), self.device.index

    # a copy (copy, deepcopy, pickle) is a plan with a workspace of its own
    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k not in ("_bytes", "_failed", "_stream", "_workspace", "_raw", "_lock", "_args", "_at")}

    def __setstate__(self, state):
        self.__dict__.update(state)
        self._make()

    def failed(self):
        """Whether a wait inside a kernel of this plan has run out (after two seconds: its outputs, and those of the calls
        after it, are worth nothing until reset()).  Waits for the device."""
        torch.cuda.synchronize(self.device)
        return bool(self._workspace[self._failed : self._failed + 4].any())

    def reset(self):
        """Zeroes the workspace, after the plan's calls so far: what failed() calls for.  Kernels leave the workspace ready
        for the next call by themselves, but not one that has given up."""
        with torch.cuda.device(self.device), self._lock:
            if _raw_stream(self._device) != self._raw:
                self._order()
            self._workspace.zero_()

    def _order(self):
        if torch.cuda.is_current_stream_capturing():
            return
        s = torch.cuda.current_stream(self.device)
        s.wait_stream(self._stream)
        self._workspace.record_stream(s)
        self._stream, self._raw = s, s.cuda_stream

    def attend(self, q, cache, block_table, seq_lens, *, out=None, return_lse=False, stream=None):
        """q: [requests, q_heads, head_dim]; row r is the newest token of the request in row r of block_table (int32
        [requests, pages]), which holds seq_lens[r] tokens (int32), the newest included.  Returns the output, shaped
        like q; with return_lse=True also the fp32 logarithm of the softmax's sum [requests, q_heads].  A request
        without tokens gets zeros and -inf.  Not differentiable, as append."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.attend(q, cache, block_table, seq_lens, out=out, return_lse=return_lse)
        with self._lock:  # from a call's place in the order to its launch
            if _raw_stream(self._device) != self._raw:
                self._order()
            entry = _entry.packed_attend if isinstance(cache, PackedCache) else _entry.attend
            got = entry(self._at, self._device, self.max_requests, self.head_dim, q, cache._at, cache._maps_at, cache._device, block_table,
                                seq_lens, out, return_lse)
        if got is NotImplemented:
            return _without_derivative("attend", functools.partial(self.attend, return_lse=return_lse), (q, cache, block_table, seq_lens), out, q)
        return got


# ----------------------------------------------------------------------------------------------------------------------
# the next token
# ----------------------------------------------------------------------------------------------------------------------
def sample(logits, uniforms, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, return_logprob=False, stream=None):
    """A token for every row of logits (bf16, fp16 or fp32 [rows, vocab]) from uniforms (fp32 [rows], in [0, 1)), as int32 [rows]
    (amap_sample).  Weights are exp(logit / temperature); top_k (0: all) keeps that many of the largest logits, min_p those
    with at least this part of the largest one's weight, top_p the fewest of what these leave whose weights are that part of
    their sum; the token is where the sum over the kept tokens, by index, passes its uniform.  temperature 0 takes the
    largest logit.  Ties go to the lowest index, NaN is never drawn, a row with no logit above
    -infinity gives -1.  Every setting is a number, or a tensor with one per row (fp32; top_k int32).  With
    return_logprob=True also the log of the probability that the token was drawn with, fp32 [rows].  Not differentiable, as
    append."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return sample(logits, uniforms, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, out=out, return_logprob=return_logprob)
    got = _entry.sample(logits, uniforms, temperature, top_k, top_p, min_p, out, return_logprob)
    if got is NotImplemented:
        call = functools.partial(sample, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, return_logprob=return_logprob)
        return _without_derivative("sample", call, (logits, uniforms), out, logits)
    return got
