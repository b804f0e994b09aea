"""Paged key-value cache: exact attention of views that arrive one after another.

Binding of the vp_rotary*, vp_norm_rotary*, vp_cache_* and vp_cache8_* calls of include/vggt_prime.h, in the manner of vp.py
(argument checks and marshalling; the operators run in the library's kernels, on the current torch
stream, without synchronising), and StreamLayer, which runs them together.

Handles: a PagedCache names the pool, a Batch the sequences of a call.  Both hold
the tensors they name; what the tensors contain may change between calls.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional, Sequence

import torch
from torch.autograd import forward_ad

from . import vp
from .vp import HEAD_DIM, VPError, _check, _dt, _need, _ptr, _wrote, load_library

ROT_INTERLEAVED, ROT_HALF = 0, 1
ROT_SCALE_NONE, ROT_SCALE_LINEAR, ROT_SCALE_PARTS = 0, 1, 2
_LAYOUTS = {"interleaved": ROT_INTERLEAVED, "half": ROT_HALF}
_NORMS = {"layer": vp.NORM_LAYER, "rms": vp.NORM_RMS}
_CODES = {torch.float8_e4m3fn: vp.VP_E4M3, torch.int8: vp.VP_INT8}
_SCALINGS = {"none": ROT_SCALE_NONE, "linear": ROT_SCALE_LINEAR, "parts": ROT_SCALE_PARTS}


# A single token's attention takes the GPU some 10 us, so the calls below keep the host's part short:
# addresses go to the library as plain integers, a tensor's properties are compared in one
# pass, and only a tensor that fails is looked at again for the message.

def _stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _done(code: int, where: str):
    if code:
        raise VPError(code, where)


_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_grad_enabled = torch.is_grad_enabled


def _here(*tensors) -> int:
    """The current device's current stream; refuses tensors that are elsewhere."""
    dev = _device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("a tensor is on %s, the current device is %d" % (t.device, dev))
    return _raw_stream(dev)


def _no_tangents(*tensors):
    """Refuses dual tensors (forward-mode derivatives), whose tangents a call through addresses would lose."""
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError("forward-mode derivatives are not available (unpack_dual gives a tensor without)")


def _no_gradients(*tensors):
    """Refuses tensors that require gradients, in calls that have none to give."""
    if _grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("the cache's operators have no gradients: call them under torch.no_grad (norm_rotary alone has some)")
    if forward_ad._current_level >= 0:
        _no_tangents(*tensors)


def _rows(t: torch.Tensor, name: str, T: int, H: int, dtype) -> int:
    """Checks a [T, H, 64] tensor whose tokens may lie apart; returns their distance."""
    try:
        st = t.stride()
        if t.shape == (T, H, HEAD_DIM) and t.dtype is dtype and t.is_cuda and \
                (T == 0 or (st[2] == 1 and (H == 1 or st[1] == HEAD_DIM))):
            return st[0] if T > 1 else H * HEAD_DIM
    except AttributeError:
        raise TypeError("%s must be a tensor" % name) from None
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.dtype != dtype:
        raise ValueError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    if tuple(t.shape) != (T, H, HEAD_DIM):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), (T, H, HEAD_DIM)))
    raise ValueError("%s must have contiguous [H, %d] rows" % (name, HEAD_DIM))


def _whole(t: torch.Tensor, name: str, shape, dtype) -> int:
    """Checks a contiguous tensor; returns its address."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.is_cuda and \
            t.is_contiguous():
        return t.data_ptr()
    _need(t, name, shape, dtype)
    raise ValueError("%s is not as expected" % name)


def _work(ws: torch.Tensor):
    """Address and size in bytes of a workspace."""
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.is_contiguous()):
        _need(ws, "ws")
    return ws.data_ptr(), ws.numel() * ws.element_size()


class Rotary:
    """Rotary positions: per-pair frequencies (int64 [dim / 2], fractions of a revolution per
    position times 2^64), pair layout ("half" or "interleaved"), number of position axes and the
    factor on the rotated features."""

    def __init__(self, freq: torch.Tensor, layout: str = "half", axes: int = 1, mag: float = 1.0):
        _need(freq, "freq", None, torch.int64)
        if freq.dim() != 1:
            raise ValueError("freq must be [dim / 2]")
        self.freq, self.layout, self.axes, self.mag = freq, layout, int(axes), float(mag)
        self.dim = 2 * freq.numel()
        self._fields = (freq.data_ptr(), self.dim, self.axes, _LAYOUTS[layout], self.mag)

    @staticmethod
    def make(dim: int = HEAD_DIM, base: float = 10000.0, axes: int = 1, layout: str = "half",
             scaling: str = "none", factor: float = 1.0, original: float = 0.0, low: float = 1.0,
             high: float = 32.0, device="cuda") -> "Rotary":
        """Frequencies base^(-2j / section) with the scaling named (vp_rotary_frequencies)."""
        out = torch.zeros(max(1, dim // 2), dtype=torch.int64)
        mag = ctypes.c_float(0.0)
        _check(load_library().vp_rotary_frequencies(int(dim), int(axes), float(base),
                                                    _SCALINGS[scaling], float(factor),
                                                    float(original), float(low), float(high),
                                                    _ptr(out), ctypes.byref(mag)),
               "vp_rotary_frequencies")
        return Rotary(out.to(device), layout, axes, mag.value)

    def at(self, pos: torch.Tensor, T: int):
        """The C argument for positions pos int32 [T, axes]."""
        return ctypes.byref(vp.vp_rotary_spec(_whole(pos, "pos", (T, self.axes), torch.int32),
                                              *self._fields))


def rotary(x, pos, rot: Rotary, out: Optional[torch.Tensor] = None, transpose: bool = False):
    """x [T, H, 64] with the features turned by their positions; with `transpose` the gradient's
    map.  `out` may be x.  An x that requires gradients gets them (no `out` then); the cache's
    operators below have none."""
    if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
        if out is not None:
            raise ValueError("out would not be part of the gradient's graph")
        return _Rotation.apply(x, pos, rot, transpose)
    if forward_ad._current_level >= 0:
        _no_tangents(x, out)
    T, H = x.shape[0], x.shape[1]
    xs = _rows(x, "x", T, H, x.dtype)
    given = out is not None
    if not given:
        out = torch.empty(T, H, HEAD_DIM, dtype=x.dtype, device=x.device)
    ys = _rows(out, "out", T, H, x.dtype)
    _done(load_library().vp_rotary(rot.at(pos, T), _dt(x), T, H, x.data_ptr(), xs, out.data_ptr(), ys,
                                   transpose, _stream()), "vp_rotary")
    if given:
        _wrote(out)
    return out


class _Rotation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, rot, transpose):
        ctx.save_for_backward(pos, rot.freq)
        ctx.rot, ctx.transpose = rot, bool(transpose)
        return rotary(x, pos, rot, None, transpose)

    @staticmethod
    def backward(ctx, g):
        pos, _ = ctx.saved_tensors
        if not g.is_contiguous() or g.data_ptr() % 16:     # (broadcast, or a part of something)
            g = g.clone(memory_format=torch.contiguous_format)
        return rotary(g, pos, ctx.rot, None, not ctx.transpose), None, None, None


def _memory(gain, bias):
    """Where gain and bias lie, and how: what the kernels read changes with any of these."""
    return (gain is not None and (gain.data_ptr(), gain.numel(), gain.stride(), gain.dtype),
            bias is not None and (bias.data_ptr(), bias.numel(), bias.stride(), bias.dtype))


class HeadNorm:
    """The norm of a head's row over its 64 features: kind "layer" (mean and variance) or "rms" (mean
    square), with gain and bias fp32 [64], or [H, 64] for a norm per head, or None (see vp_head_norm).  Gain and bias
    may be exchanged later; kind and eps may not."""

    def __init__(self, kind: str = "layer", gain: Optional[torch.Tensor] = None,
                 bias: Optional[torch.Tensor] = None, eps: float = 1e-6):
        if not 0 < ctypes.c_float(eps).value < float("inf"):
            raise ValueError("eps must be positive")
        self._kind, self.gain, self.bias, self._eps = kind, gain, bias, float(eps)
        self._bind()

    kind, eps = property(lambda self: self._kind), property(lambda self: self._eps)

    def __reduce__(self):               # (copied and pickled as what it is made of, parameters with their module's)
        return HeadNorm, (self._kind, self.gain, self.bias, self._eps)

    def _bind(self):
        shape = None
        for t, name in ((self.gain, "gain"), (self.bias, "bias")):
            if t is None:
                continue
            _need(t, name, shape, torch.float32)
            shape = tuple(t.shape)
            if shape[-1:] != (HEAD_DIM,) or t.dim() > 2:
                raise ValueError("%s must be [%d] or [heads, %d]" % (name, HEAD_DIM, HEAD_DIM))
            if t.data_ptr() % 16:
                raise ValueError("%s must start at a multiple of 16 bytes" % name)
        if self.gain is not None and self.bias is not None and self.gain.device != self.bias.device:
            raise ValueError("gain and bias are on different devices")
        self.tensor = self.bias if self.gain is None else self.gain       # (for its device)
        self.heads = shape[0] if shape is not None and len(shape) == 2 else None
        self._at = _memory(self.gain, self.bias)
        ptr = lambda t: None if t is None else t.data_ptr()
        self._ref = ctypes.byref(vp.vp_head_norm(_NORMS[self._kind], ptr(self.gain), ptr(self.bias), self.heads is not None,
                                                 self._eps))

    def at(self, H: int):
        """The C argument for rows of H heads."""
        if self._at != _memory(self.gain, self.bias):
            self._bind()                # (a parameter whose storage was exchanged)
        if self.heads is not None and self.heads != H:
            raise ValueError("a norm of %d heads for %d" % (self.heads, H))
        return self._ref


def norm_rotary(x, norm: HeadNorm, pos=None, rot: Optional[Rotary] = None, out: Optional[torch.Tensor] = None):
    """x [T, H, 64], every head's row normalised and turned by its token's position, in one pass (without
    `rot` only normalised).  `out` may be x.  Where x, gain or bias require gradients they get them (no `out`
    then).  As with every operator of torch's: while a training step is captured into a graph, no eager graph of
    the same leaves may be alive."""
    if (rot is None) != (pos is None):
        raise ValueError("a rotation needs positions" if pos is None else "positions need a rotation (rot)")
    if torch.is_grad_enabled() and (x.requires_grad or (norm.gain is not None and norm.gain.requires_grad) or
                                    (norm.bias is not None and norm.bias.requires_grad) or
                                    (out is not None and out.requires_grad)):
        if out is not None:
            raise ValueError("out would not be part of the gradient's graph")
        return _NormRotation.apply(x, norm.gain, norm.bias, pos, norm, rot)
    if forward_ad._current_level >= 0:
        _no_tangents(x, norm.gain, norm.bias, out)
    T, H = x.shape[0], x.shape[1]
    xs = _rows(x, "x", T, H, x.dtype)
    given = out is not None
    if not given:
        out = torch.empty(T, H, HEAD_DIM, dtype=x.dtype, device=x.device)
    ys = _rows(out, "out", T, H, x.dtype)
    _done(load_library().vp_norm_rotary(norm.at(H), None if rot is None else rot.at(pos, T), _dt(x), T, H, x.data_ptr(), xs,
                                        out.data_ptr(), ys, _here(x, out, norm.tensor, pos, rot and rot.freq)),
          "vp_norm_rotary")
    if given:
        _wrote(out)
    return out


class _NormRotation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, bias, pos, norm, rot):
        ctx.save_for_backward(x, gain, bias, pos, None if rot is None else rot.freq)
        ctx.norm, ctx.rot = norm, rot
        return norm_rotary(x, norm, pos, rot)

    @staticmethod
    def backward(ctx, g):
        # (once_differentiable's bookkeeping takes a third of a small call's time: only where it has something to do)
        return (_second if torch.is_grad_enabled() else _norm_gradients)(ctx, g)


def _norm_gradients(ctx, g):
    x, gain, bias, pos, _ = ctx.saved_tensors          # (refuses values that were changed in place)
    if forward_ad._current_level >= 0:
        _no_tangents(g)
    norm, rot = ctx.norm, ctx.rot
    if norm._at != _memory(gain, bias):                # (it got others, or the graph kept copies)
        norm = HeadNorm(norm.kind, gain, bias, norm.eps)
    T, H, _ = x.shape
    if not g.is_contiguous() or g.data_ptr() % 16:     # (broadcast, or a part of something)
        g = g.clone(memory_format=torch.contiguous_format)
    need = ctx.needs_input_grad
    dx = dgain = dbias = None
    at_x = at_gain = at_bias = at_ws = n = 0
    if need[0]:
        dx = torch.empty(T, H, HEAD_DIM, dtype=x.dtype, device=x.device)
        at_x = dx.data_ptr()
    if need[1]:
        dgain = torch.empty_like(gain)
        at_gain = dgain.data_ptr()
    if need[2]:
        dbias = torch.empty_like(bias)
        at_bias = dbias.data_ptr()
    if need[1] or need[2]:
        n = _norm_workspace(T, H, norm.heads is not None)
        ws = torch.empty(n, dtype=torch.uint8, device=x.device)
        at_ws = ws.data_ptr()
    _done(load_library().vp_norm_rotary_grad(norm._ref, None if rot is None else rot.at(pos, T), _dt(x), T, H, x.data_ptr(),
                                             x.stride(0) if T > 1 else H * HEAD_DIM, g.data_ptr(), H * HEAD_DIM, at_x,
                                             at_gain, at_bias, at_ws, n, _stream()), "vp_norm_rotary_grad")
    return dx, dgain, dbias, None, None, None


_second = torch.autograd.function.once_differentiable(_norm_gradients)


@functools.lru_cache(maxsize=256)
def _norm_workspace(T: int, H: int, per_head: bool) -> int:
    return load_library().vp_norm_rotary_grad_workspace_bytes(T, H, per_head)


class PagedCache:
    """The pool: K, V [npages, Hkv, page, 64], and per slot weight fp32 and stamp int32 [npages,
    Hkv, page] (needed by the eviction, optional otherwise).

    K and V may be 8-bit codes (torch.float8_e4m3fn or torch.int8) with `scale` bf16 [npages, Hkv, page, 2],
    a key's and a value's (see vp_cache8); `rows` is then the type of the calls' Q, K, V and O."""

    def __init__(self, K, V, weight: Optional[torch.Tensor] = None,
                 stamp: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                 rows: Optional[torch.dtype] = None):
        _need(K, "K")
        if K.dim() != 4 or K.shape[3] != HEAD_DIM:
            raise ValueError("K must be [pages, heads, page, %d]" % HEAD_DIM)
        _need(V, "V", K.shape, K.dtype)
        self.npages, self.Hkv, self.page = K.shape[:3]
        if weight is not None:
            _need(weight, "weight", K.shape[:3], torch.float32)
        if stamp is not None:
            _need(stamp, "stamp", K.shape[:3], torch.int32)
        self.codes = K.dtype in _CODES
        if self.codes and any(t is not None and t.device != K.device for t in (V, weight, stamp, scale)):
            raise ValueError("the cache's tensors are on different devices")
        if self.codes:
            if scale is None:
                raise ValueError("a cache of codes needs scales")
            _need(scale, "scale", tuple(K.shape[:3]) + (2,), torch.bfloat16)
            rows = torch.bfloat16 if rows is None else rows
            if rows not in (torch.bfloat16, torch.float32):
                raise ValueError("rows are bf16 or fp32")
        elif scale is not None or rows not in (None, K.dtype):
            raise ValueError("scales, and rows of another type, are for codes")
        self.K, self.V, self.weight, self.stamp, self.scale = K, V, weight, stamp, scale
        self.dtype = rows if self.codes else K.dtype       # of the calls' rows
        ptr = lambda t: None if t is None else t.data_ptr()
        self._c = vp.vp_cache(K.data_ptr(), V.data_ptr(), ptr(weight), ptr(stamp), self.npages,
                              self.page, self.Hkv, HEAD_DIM, _CODES[K.dtype] if self.codes else _dt(K))
        self._c8 = vp.vp_cache8(self._c, ptr(scale), vp.VP_BF16 if self.dtype is torch.bfloat16 else vp.VP_F32)
        self._ref8 = ctypes.byref(self._c8)
        self._ref = self._ref8 if self.codes else ctypes.byref(self._c)
        self._pool = [t for t in (K, V, weight, stamp, scale) if t is not None]
        self._where = [K] + [t for t in self._pool if t.get_device() != K.get_device()]   # (as Batch's)

    def _call(self, name: str):
        """The library's call for this cache."""
        return getattr(load_library(), ("vp_cache8_" if self.codes else "vp_cache_") + name)

    @staticmethod
    def empty(npages: int, Hkv: int, page: int = 64, dtype=torch.bfloat16, device="cuda",
              rows: Optional[torch.dtype] = None) -> "PagedCache":
        kv = lambda: torch.empty(npages, Hkv, page, HEAD_DIM, dtype=dtype, device=device)
        scale = None
        if dtype in _CODES:
            scale = torch.empty(npages, Hkv, page, 2, dtype=torch.bfloat16, device=device)
        return PagedCache(kv(), kv(),
                          torch.zeros(npages, Hkv, page, dtype=torch.float32, device=device),
                          torch.zeros(npages, Hkv, page, dtype=torch.int32, device=device), scale, rows)


class Batch:
    """The sequences of a call: page table int32 [B, max_pages], slots in use int32 [B] (the new
    tokens included), first rows int32 [B + 1] of the new tokens, bounds of the largest chunk and
    sequence, and the tokens seen so far int32 [B] (new ones included)."""

    def __init__(self, table, length, q_start, max_q: int, max_len: int,
                 seen: Optional[torch.Tensor] = None):
        _need(table, "table", None, torch.int32)
        if table.dim() != 2:
            raise ValueError("table must be [B, pages]")
        self.B, self.max_pages = table.shape
        _need(length, "length", (self.B,), torch.int32)
        _need(q_start, "q_start", (self.B + 1,), torch.int32)
        if seen is not None:
            _need(seen, "seen", (self.B,), torch.int32)
        self.table, self.length, self.q_start, self.seen = table, length, q_start, seen
        self.max_q, self.max_len = int(max_q), int(max_len)
        # (to check their device by: the table, and what is not with it)
        self._where = [table] + [t for t in (length, q_start, seen) if t is not None and t.get_device() != table.get_device()]
        self._first = (table.data_ptr(), length.data_ptr(), None if seen is None else seen.data_ptr(),
                       q_start.data_ptr(), self.B, self.max_pages)
        self._last = (None, None)

    def _for(self, T: int):
        """The C argument for calls of T rows."""
        sizes, last = (T, self.max_q, self.max_len), self._last
        if last[0] != sizes:            # (made once for the calls of a step: a microsecond each)
            self._last = last = (sizes, ctypes.byref(vp.vp_cache_batch(*self._first, *sizes)))
        return last[1]


def append(pc: PagedCache, batch: Batch, Q, K, V, pos=None, rot: Optional[Rotary] = None,
           Q_out: Optional[torch.Tensor] = None, q_norm: Optional[HeadNorm] = None,
           k_norm: Optional[HeadNorm] = None):
    """New tokens into the cache: K [T, Hkv, 64] rotated, V as it is; returns the rotated Q [T, Hq,
    64] (None without Q).  With q_norm or k_norm Q's or K's heads are normalised before the rotation.  A cache
    of codes gets them quantised.  There are no gradients: with norms or codes, rows, gains and biases that require them are
    refused, but under torch.no_grad."""
    T, Hkv, dt = K.shape[0], pc.Hkv, pc.dtype
    ks, vs = _rows(K, "K", T, Hkv, dt), _rows(V, "V", T, Hkv, dt)
    Hq = qs = q = qo = 0
    given = ()
    if Q is not None:
        Hq = Q.shape[1]
        qs, q = _rows(Q, "Q", T, Hq, dt), Q.data_ptr()
        if Q_out is None:
            Q_out = torch.empty(T, Hq, HEAD_DIM, dtype=dt, device=Q.device)
        else:
            given = (Q_out,)
        qo = _whole(Q_out, "Q_out", (T, Hq, HEAD_DIM), dt)
    if (rot is None) != (pos is None):
        raise ValueError("a rotation needs positions" if pos is None else "positions need a rotation (rot)")
    turn = None if rot is None else rot.at(pos, T)
    if pc.codes or q_norm is not None or k_norm is not None:
        qn = qg = qb = kn = kg = kb = None
        if q_norm is not None and Q is not None:
            qn, qg, qb = q_norm.at(Hq), q_norm.gain, q_norm.bias       # (as they are after `at`)
        if k_norm is not None:
            kn, kg, kb = k_norm.at(Hkv), k_norm.gain, k_norm.bias
        _no_gradients(K, V, Q, Q_out, qg, qb, kg, kb)
        st = _here(*pc._where, K, V, Q, Q_out, pos, rot and rot.freq, q_norm and q_norm.tensor, k_norm and k_norm.tensor,
                   *batch._where)
        _done(load_library().vp_cache8_append(pc._ref8, batch._for(T), Hq, q, qs, K.data_ptr(), ks, V.data_ptr(), vs,
                                              qn, kn, turn, qo, st), "vp_cache8_append")
    else:
        _done(load_library().vp_cache_append(pc._ref, batch._for(T), Hq, q, qs, K.data_ptr(), ks, V.data_ptr(), vs,
                                             turn, qo, _stream()), "vp_cache_append")
    _wrote(*pc._pool, *given)
    return Q_out if Q is not None else None


def read(pc: PagedCache, batch: Batch, T: int, dtype: Optional[torch.dtype] = None,
         K_out: Optional[torch.Tensor] = None, V_out: Optional[torch.Tensor] = None):
    """The last slots of every sequence, as many as the batch gives it rows, as (K, V) [T, Hkv, 64]: what an
    append of those rows left in the cache.  `dtype`: bf16 or fp32 (that of K_out, or of the cache's rows)."""
    if dtype is None:
        dtype = pc.dtype if K_out is None else K_out.dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("rows are read in bf16 or fp32")
    # (zeros: rows past the last sequence's are left as they are)
    new = lambda: torch.zeros(T, pc.Hkv, HEAD_DIM, dtype=dtype, device=pc.K.device)
    K_given, V_given = K_out is not None, V_out is not None
    K_out, V_out = new() if K_out is None else K_out, new() if V_out is None else V_out
    shape = (T, pc.Hkv, HEAD_DIM)
    if K_given or V_given:
        _no_gradients(K_out, V_out)
    st = _here(*pc._where, K_out, V_out, *batch._where)
    _done(load_library().vp_cache8_read(pc._ref8, batch._for(T), vp.VP_BF16 if dtype is torch.bfloat16 else vp.VP_F32,
                                        _whole(K_out, "K_out", shape, dtype), _whole(V_out, "V_out", shape, dtype),
                                        st), "vp_cache8_read")
    if K_given or V_given:
        _wrote(K_out, V_out)
    return K_out, V_out


def attend_workspace(pc: PagedCache, batch: Batch, Hq: int, T: int) -> torch.Tensor:
    n = pc._call("attend_workspace_bytes")(pc._ref, batch._for(T), int(Hq))
    if n == 0:
        raise ValueError("invalid cache or batch")
    return torch.empty(n, dtype=torch.uint8, device=pc.K.device)


def attend_plan(pc: PagedCache, batch: Batch, Hq: int, T: int) -> vp.vp_cache_plan:
    """How a call with these bounds is computed (see vp_cache_plan)."""
    plan = vp.vp_cache_plan()
    _done(pc._call("attend_plan")(pc._ref, batch._for(T), int(Hq), ctypes.byref(plan)), "vp_cache_attend_plan")
    return plan


def attend(pc: PagedCache, batch: Batch, Q, causal: bool = True, scale: float = 0.0,
           O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
           weight_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Attention of the new tokens' queries Q [T, Hq, 64] over their sequences' slots: (O [T, Hq,
    64], lse [T, Hq] fp32).  With `weight_out` (it may be pc.weight) the attention weights of
    the call are added to the slots they fall on.  There are no gradients: over codes, a Q that requires them is refused, but
    under torch.no_grad."""
    T, Hq, _ = Q.shape
    dt = pc.dtype
    qs = _rows(Q, "Q", T, Hq, dt)
    given = O is not None or lse is not None
    if O is None:
        O = torch.empty(T, Hq, HEAD_DIM, dtype=dt, device=Q.device)
    if lse is None:
        lse = torch.empty(T, Hq, dtype=torch.float32, device=Q.device)
    o, ls, wo = _whole(O, "O", (T, Hq, HEAD_DIM), dt), _whole(lse, "lse", (T, Hq), torch.float32), None
    if pc.codes:
        _no_gradients(Q, O, lse, weight_out)
        st = _here(pc.K, Q, O, lse, weight_out, ws, *batch._where)
    else:
        st = _stream()
    if weight_out is not None:
        if pc.weight is None:
            raise ValueError("the cache has no weights")
        wo = _whole(weight_out, "weight_out", pc.weight.shape, torch.float32)
    if ws is None:
        ws = attend_workspace(pc, batch, Hq, T)
    w, n = _work(ws)
    _done(pc._call("attend")(pc._ref, batch._for(T), Hq, Q.data_ptr(), qs, causal, scale, o, ls, wo, w, n, st),
          "vp_cache_attend")
    if weight_out is not None:
        _wrote(O, lse, weight_out)
    elif given:
        _wrote(O, lse)
    return O, lse


def evict_workspace(pc: PagedCache, B: int, max_len: int) -> torch.Tensor:
    n = load_library().vp_cache_evict_workspace_bytes(int(B), pc.Hkv, int(max_len))
    if n == 0:
        raise ValueError("invalid batch")
    return torch.empty(n, dtype=torch.uint8, device=pc.K.device)


def evict(pc: PagedCache, table, length, seen, keep: int, max_len: int, sink: int = 0,
          recent: int = 0, weight_out: Optional[torch.Tensor] = None,
          stamp_out: Optional[torch.Tensor] = None, length_out: Optional[torch.Tensor] = None,
          ws: Optional[torch.Tensor] = None):
    """Brings every sequence down to `keep` slots (see vp_cache_evict); without the *_out
    tensors in place.  Returns the new lengths."""
    if pc.weight is None or pc.stamp is None:
        raise ValueError("the eviction needs the cache's weights and stamps")
    _need(table, "table", None, torch.int32)
    B, pages = table.shape
    _need(length, "length", (B,), torch.int32)
    _need(seen, "seen", (B,), torch.int32)
    weight_out = pc.weight if weight_out is None else weight_out
    stamp_out = pc.stamp if stamp_out is None else stamp_out
    length_out = length if length_out is None else length_out
    wo = _whole(weight_out, "weight_out", pc.weight.shape, torch.float32)
    so = _whole(stamp_out, "stamp_out", pc.stamp.shape, torch.int32)
    lo = _whole(length_out, "length_out", (B,), torch.int32)
    if ws is None:
        ws = evict_workspace(pc, B, max_len)
    w, n = _work(ws)
    if pc.codes:
        _here(pc.K, table, length, seen, weight_out, stamp_out, length_out, ws)
    c = vp.vp_cache_batch(table.data_ptr(), length.data_ptr(), seen.data_ptr(), None, B, pages, 0, 0,
                          int(max_len))
    _done(pc._call("evict")(pc._ref, ctypes.byref(c), int(keep), int(sink), int(recent), wo, so, lo, w, n, _stream()),
          "vp_cache_evict")
    _wrote(weight_out, stamp_out, length_out, *pc._pool)
    return length_out


class StreamLayer:
    """Exact attention of one layer over sequences whose views arrive chunk by chunk, in a cache of
    at most `keep` slots per sequence and head between the chunks: step() appends a chunk, attends
    it over the cache and itself, gathers the attention weights, and evicts down to `keep`.

    B sequences of chunks up to `max_chunk` tokens.  `sink` first tokens (the first view, which the
    scene's frame of reference hangs on) and the `recent` latest ones are kept whatever
    weight they have.  `causal`: a token sees its own chunk up to itself, not all of
    it.  `rot`: positions given to step() are applied to Q and K; `q_norm`, `k_norm`: norms of their heads
    before.  `dtype`: of the cache; torch.float8_e4m3fn or torch.int8 for 8-bit codes, `rows` (bf16 when not
    given) then of Q, K, V and O.

    There are no gradients; with norms or codes, rows and parameters that require them are refused, but under torch.no_grad.

    A step is enqueued on the current stream without waiting for it.  Its chunks' starts and bounds
    are the host's, so a captured step would repeat those of the capture."""

    def __init__(self, B: int, keep: int, max_chunk: int, Hq: int = vp.MAX_HEADS,
                 Hkv: Optional[int] = None, page: int = 64, dtype=torch.bfloat16, sink: int = 0,
                 recent: int = 0, causal: bool = False, rot: Optional[Rotary] = None,
                 device="cuda", q_norm: Optional[HeadNorm] = None, k_norm: Optional[HeadNorm] = None,
                 rows: Optional[torch.dtype] = None):
        Hkv = Hq if Hkv is None else Hkv
        if Hkv < 1 or Hq < Hkv or Hq % Hkv:
            raise ValueError("%d query heads for %d key heads" % (Hq, Hkv))
        if min(B, keep, max_chunk) < 1 or min(sink, recent) < 0:
            raise ValueError("B, keep and max_chunk must be at least 1, sink and recent at least 0")
        pages = -(-(keep + max_chunk) // page)
        self.B, self.Hq, self.keep, self.max_chunk = B, Hq, keep, max_chunk
        self.sink, self.recent, self.causal, self.rot = sink, recent, causal, rot
        self.q_norm, self.k_norm = q_norm, k_norm
        self.pc = PagedCache.empty(B * pages, Hkv, page, dtype, device, rows)
        self.table = torch.arange(B * pages, dtype=torch.int32, device=device).view(B, pages)
        self.length = torch.zeros(B, dtype=torch.int32, device=device)
        self.seen = torch.zeros(B, dtype=torch.int32, device=device)
        self.lens = [0] * B            # the lengths, known on the host as well
        self.ws = evict_workspace(self.pc, B, keep + max_chunk)
        self.attend_ws: Optional[torch.Tensor] = None

    def step(self, Q, K, V, pos=None, counts: Optional[Sequence[int]] = None):
        """Q [T, Hq, 64], K, V [T, Hkv, 64]: the chunks of the sequences, one after the other,
        counts[b] tokens each (equal parts when not given).  Returns O [T, Hq, 64]."""
        T = Q.shape[0]
        if Q.dim() != 3 or Q.shape[1] != self.Hq:
            raise ValueError("Q has shape %s, the layer %d heads" % (tuple(Q.shape), self.Hq))
        if counts is None:
            if T % self.B:
                raise ValueError("%d tokens for %d sequences: give counts" % (T, self.B))
            counts = [T // self.B] * self.B
        counts = [int(c) for c in counts]
        if len(counts) != self.B or min(counts) < 0 or sum(counts) != T or max(counts) > self.max_chunk:
            raise ValueError("counts must be %d numbers of 0 to %d that sum to %d"
                             % (self.B, self.max_chunk, T))
        start = [0]
        for c in counts:
            start.append(start[-1] + c)
        # (from pinned memory, which torch holds until the copy is done: the host does not wait)
        q_start = torch.tensor(start, dtype=torch.int32, pin_memory=True).to(Q.device, non_blocking=True)
        new = q_start[1:] - q_start[:-1]
        # (the layer's own counts change once the chunk is in: a refused one leaves it as it was)
        length, seen = self.length + new, self.seen + new
        lens = [n + c for n, c in zip(self.lens, counts)]
        batch = Batch(self.table, length, q_start, max(counts), max(lens), seen)
        Q = append(self.pc, batch, Q, K, V, pos, self.rot, None, self.q_norm, self.k_norm)
        n = self.pc._call("attend_workspace_bytes")(self.pc._ref, batch._for(T), self.Hq)
        if self.attend_ws is None or self.attend_ws.numel() < n:
            self.attend_ws = torch.empty(n, dtype=torch.uint8, device=Q.device)
        O, _ = attend(self.pc, batch, Q, self.causal, weight_out=self.pc.weight, ws=self.attend_ws)
        self.length, self.seen, self.lens = length, seen, lens
        if max(self.lens) > self.keep:
            evict(self.pc, self.table, self.length, self.seen, self.keep, max(self.lens), self.sink,
                  self.recent, ws=self.ws)
            self.lens = [min(n, self.keep) for n in self.lens]
        return O
