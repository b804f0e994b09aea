"""Paged key-value cache: exact attention of views that arrive one after another.

Binding of the vp_rotary* and vp_cache_* calls of include/vggt_prime.h, in the manner of vp.py
(argument checks and marshalling; the operators run in the library's kernels, on the current torch
stream, without synchronising), and StreamLayer, which runs them together.

Handles: a PagedCache names the pool, a Batch the sequences of a call.  Both hold
the tensors they name; what the tensors contain may change between calls.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import vp
from .vp import HEAD_DIM, VPError, _check, _dt, _need, _ptr, load_library

ROT_INTERLEAVED, ROT_HALF = 0, 1
ROT_SCALE_NONE, ROT_SCALE_LINEAR, ROT_SCALE_PARTS = 0, 1, 2
_LAYOUTS = {"interleaved": ROT_INTERLEAVED, "half": ROT_HALF}
_SCALINGS = {"none": ROT_SCALE_NONE, "linear": ROT_SCALE_LINEAR, "parts": ROT_SCALE_PARTS}


# A single token's attention takes the GPU some 10 us, so the calls below keep the host's part short:
# addresses go to the library as plain integers, a tensor's properties are compared in one
# pass, and only a tensor that fails is looked at again for the message.

def _stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _done(code: int, where: str):
    if code:
        raise VPError(code, where)


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
    T, H = x.shape[0], x.shape[1]
    xs = _rows(x, "x", T, H, x.dtype)
    if out is None:
        out = torch.empty(T, H, HEAD_DIM, dtype=x.dtype, device=x.device)
    ys = _rows(out, "out", T, H, x.dtype)
    _done(load_library().vp_rotary(rot.at(pos, T), _dt(x), T, H, x.data_ptr(), xs, out.data_ptr(), ys,
                                   transpose, _stream()), "vp_rotary")
    return out


class _Rotation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, rot, transpose):
        ctx.save_for_backward(pos)
        ctx.rot, ctx.transpose = rot, bool(transpose)
        return rotary(x, pos, rot, None, transpose)

    @staticmethod
    def backward(ctx, g):
        pos, = ctx.saved_tensors
        if not g.is_contiguous() or g.data_ptr() % 16:     # (broadcast, or a part of something)
            g = g.clone(memory_format=torch.contiguous_format)
        return rotary(g, pos, ctx.rot, None, not ctx.transpose), None, None, None


class PagedCache:
    """The pool: K, V [npages, Hkv, page, 64], and per slot weight fp32 and stamp int32 [npages,
    Hkv, page] (needed by the eviction, optional otherwise)."""

    def __init__(self, K, V, weight: Optional[torch.Tensor] = None,
                 stamp: Optional[torch.Tensor] = None):
        _need(K, "K")
        if K.dim() != 4 or K.shape[3] != HEAD_DIM:
            raise ValueError("K must be [pages, heads, page, %d]" % HEAD_DIM)
        _need(V, "V", K.shape, K.dtype)
        self.npages, self.Hkv, self.page = K.shape[:3]
        if weight is not None:
            _need(weight, "weight", K.shape[:3], torch.float32)
        if stamp is not None:
            _need(stamp, "stamp", K.shape[:3], torch.int32)
        self.K, self.V, self.weight, self.stamp, self.dtype = K, V, weight, stamp, K.dtype
        ptr = lambda t: None if t is None else t.data_ptr()
        self._c = vp.vp_cache(K.data_ptr(), V.data_ptr(), ptr(weight), ptr(stamp), self.npages,
                              self.page, self.Hkv, HEAD_DIM, _dt(K))
        self._ref = ctypes.byref(self._c)

    @staticmethod
    def empty(npages: int, Hkv: int, page: int = 64, dtype=torch.bfloat16, device="cuda") -> "PagedCache":
        kv = lambda: torch.empty(npages, Hkv, page, HEAD_DIM, dtype=dtype, device=device)
        return PagedCache(kv(), kv(),
                          torch.zeros(npages, Hkv, page, dtype=torch.float32, device=device),
                          torch.zeros(npages, Hkv, page, dtype=torch.int32, device=device))


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
        self._first = (table.data_ptr(), length.data_ptr(), None if seen is None else seen.data_ptr(),
                       q_start.data_ptr(), self.B, self.max_pages)

    def _for(self, T: int):
        return ctypes.byref(vp.vp_cache_batch(*self._first, T, self.max_q, self.max_len))


def append(pc: PagedCache, batch: Batch, Q, K, V, pos=None, rot: Optional[Rotary] = None,
           Q_out: Optional[torch.Tensor] = None):
    """New tokens into the cache: K [T, Hkv, 64] rotated, V as it is; returns the rotated Q [T, Hq,
    64] (None without Q)."""
    T, Hkv, dt = K.shape[0], pc.Hkv, pc.dtype
    ks, vs = _rows(K, "K", T, Hkv, dt), _rows(V, "V", T, Hkv, dt)
    Hq = qs = q = qo = 0
    if Q is not None:
        Hq = Q.shape[1]
        qs, q = _rows(Q, "Q", T, Hq, dt), Q.data_ptr()
        if Q_out is None:
            Q_out = torch.empty(T, Hq, HEAD_DIM, dtype=dt, device=Q.device)
        qo = _whole(Q_out, "Q_out", (T, Hq, HEAD_DIM), dt)
    if (rot is None) != (pos is None):
        raise ValueError("a rotation needs positions" if pos is None else "positions need a rotation (rot)")
    _done(load_library().vp_cache_append(pc._ref, batch._for(T), Hq, q, qs, K.data_ptr(), ks, V.data_ptr(), vs,
                                         None if rot is None else rot.at(pos, T), qo, _stream()),
          "vp_cache_append")
    return Q_out if Q is not None else None


def attend_workspace(pc: PagedCache, batch: Batch, Hq: int, T: int) -> torch.Tensor:
    n = load_library().vp_cache_attend_workspace_bytes(pc._ref, batch._for(T), int(Hq))
    if n == 0:
        raise ValueError("invalid cache or batch")
    return torch.empty(n, dtype=torch.uint8, device=pc.K.device)


def attend_plan(pc: PagedCache, batch: Batch, Hq: int, T: int) -> vp.vp_cache_plan:
    """How a call with these bounds is computed (see vp_cache_plan)."""
    plan = vp.vp_cache_plan()
    _done(load_library().vp_cache_attend_plan(pc._ref, batch._for(T), int(Hq), ctypes.byref(plan)),
          "vp_cache_attend_plan")
    return plan


def attend(pc: PagedCache, batch: Batch, Q, causal: bool = True, scale: float = 0.0,
           O: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
           weight_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Attention of the new tokens' queries Q [T, Hq, 64] over their sequences' slots: (O [T, Hq,
    64], lse [T, Hq] fp32).  With `weight_out` (it may be pc.weight) the attention weights of
    the call are added to the slots they fall on."""
    T, Hq, _ = Q.shape
    dt = pc.dtype
    qs = _rows(Q, "Q", T, Hq, dt)
    if O is None:
        O = torch.empty(T, Hq, HEAD_DIM, dtype=dt, device=Q.device)
    if lse is None:
        lse = torch.empty(T, Hq, dtype=torch.float32, device=Q.device)
    o, ls, wo = _whole(O, "O", (T, Hq, HEAD_DIM), dt), _whole(lse, "lse", (T, Hq), torch.float32), None
    if weight_out is not None:
        if pc.weight is None:
            raise ValueError("the cache has no weights")
        wo = _whole(weight_out, "weight_out", pc.weight.shape, torch.float32)
    if ws is None:
        ws = attend_workspace(pc, batch, Hq, T)
    w, n = _work(ws)
    _done(load_library().vp_cache_attend(pc._ref, batch._for(T), Hq, Q.data_ptr(), qs, causal, scale, o, ls, wo, w,
                                         n, _stream()), "vp_cache_attend")
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
    c = vp.vp_cache_batch(table.data_ptr(), length.data_ptr(), seen.data_ptr(), None, B, pages, 0, 0,
                          int(max_len))
    _done(load_library().vp_cache_evict(pc._ref, ctypes.byref(c), int(keep), int(sink), int(recent), wo, so, lo, w, n,
                                        _stream()), "vp_cache_evict")
    return length_out


class StreamLayer:
    """Exact attention of one layer over sequences whose views arrive chunk by chunk, in a cache of
    at most `keep` slots per sequence and head between the chunks: step() appends a chunk, attends
    it over the cache and itself, gathers the attention weights, and evicts down to `keep`.

    B sequences of chunks up to `max_chunk` tokens.  `sink` first tokens (the first view, which the
    scene's frame of reference hangs on) and the `recent` latest ones are kept whatever
    weight they have.  `causal`: a token sees its own chunk up to itself, not all of
    it.  `rot`: positions given to step() are applied to Q and K.

    A step is enqueued on the current stream without waiting for it.  Its chunks' starts and bounds
    are the host's, so a captured step would repeat those of the capture."""

    def __init__(self, B: int, keep: int, max_chunk: int, Hq: int = vp.MAX_HEADS,
                 Hkv: Optional[int] = None, page: int = 64, dtype=torch.bfloat16, sink: int = 0,
                 recent: int = 0, causal: bool = False, rot: Optional[Rotary] = None,
                 device="cuda"):
        Hkv = Hq if Hkv is None else Hkv
        if Hkv < 1 or Hq < Hkv or Hq % Hkv:
            raise ValueError("%d query heads for %d key heads" % (Hq, Hkv))
        if min(B, keep, max_chunk) < 1 or min(sink, recent) < 0:
            raise ValueError("B, keep and max_chunk must be at least 1, sink and recent at least 0")
        pages = -(-(keep + max_chunk) // page)
        self.B, self.Hq, self.keep, self.max_chunk = B, Hq, keep, max_chunk
        self.sink, self.recent, self.causal, self.rot = sink, recent, causal, rot
        self.pc = PagedCache.empty(B * pages, Hkv, page, dtype, device)
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
        Q = append(self.pc, batch, Q, K, V, pos, self.rot)
        n = load_library().vp_cache_attend_workspace_bytes(self.pc._ref, batch._for(T), self.Hq)
        if self.attend_ws is None or self.attend_ws.numel() < n:
            self.attend_ws = torch.empty(n, dtype=torch.uint8, device=Q.device)
        O, _ = attend(self.pc, batch, Q, self.causal, weight_out=self.pc.weight, ws=self.attend_ws)
        self.length, self.seen, self.lens = length, seen, lens
        if max(self.lens) > self.keep:
            evict(self.pc, self.table, self.length, self.seen, self.keep, max(self.lens), self.sink,
                  self.recent, ws=self.ws)
            self.lens = [min(n, self.keep) for n in self.lens]
        return O
