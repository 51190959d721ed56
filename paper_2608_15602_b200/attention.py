"""The attention side of a decode step on torch tensors: rotary positions, the 8-bit block-paged key/value cache, attention
over it and the block tables both go by.  torch owns the memory and the stream, the C-ABI library does the work
(include/fluxbin.h states every rule); the checks here are those of types and shapes that the C side cannot see.

    rope = Rotary(128)
    cache = KVCache(num_blocks, 16, kv_heads=8, head_dim=128, fmt="int8")
    tables = BlockTables.empty(batch, max_blocks, num_blocks, 16)
    step = tables.advance(lengths, new_tokens, num_free, tokens)          # blocks, positions and slots of the new tokens
    q = cache.append(k, v, step.slots, rotary=rope, positions=step.positions, q=q)
    out = cache.attend(q, tables.table, step.lengths, ws, query_start=step.query_start)

`stream` (a torch stream, else the current one): what a call allocates comes from that stream's memory, so nothing queued
elsewhere still uses it, and is recorded on the current stream too, so it may be dropped there.  The tensors given to the call
have to be ready on `stream` and are the caller's to keep until it is through, as with any torch call on another stream.

Where query and key heads are normed first, NormedRotary(rope, q_weight, k_weight) takes rope's place; the cache then gets keys
that are turned already, and rounded to their type once more than those that append() turns on the way, in fp32.  A step that
checks a tree of drafted tokens at once:

    tree = DraftTree(parents, step.query_start, step.lengths, nodes=64)   # masks and positions, once for all layers
    q, k = normed.apply(q, k, tree.positions)
    cache.append(k, v, step.slots)
    out = cache.attend(q, tables.table, step.lengths, ws, query_start=step.query_start, tree=tree.mask)
    kept = tree.accept(drafted, answers)                                  # the path that the model itself would have answered
    cache.keep(step.slots, step.query_start, kept.path)                   # its entries move to the step's first slots, in every layer
    step = tables.advance(step.lengths, kept.surplus * step.granted, step.num_free, 0)    # and the others are dropped

Rotary.apply and NormedRotary.apply carry gradients.  The other calls are those of answering: their results have none.
"""
from __future__ import annotations

import ctypes
import math
from types import SimpleNamespace

import torch

from . import fluxbin
from .layer import Workspace, _stream_ptr

_TYPES = {torch.float16: fluxbin.TYPE_FP16, torch.float32: fluxbin.TYPE_FP32, torch.bfloat16: fluxbin.TYPE_BF16}
_STORED = {torch.int8: fluxbin.CACHE_INT8, torch.float8_e4m3fn: fluxbin.CACHE_E4M3}
_FORMATS = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_KINDS = {"none": fluxbin.ROPE_NONE, "linear": fluxbin.ROPE_LINEAR, "base": fluxbin.ROPE_BASE, "ramp": fluxbin.ROPE_RAMP,
          "bands": fluxbin.ROPE_BANDS}


_device = torch._C._cuda_getDevice               # the current device: every tensor of a call has to lie on it


def _stream(stream) -> int:
    """The raw stream of a call: `stream`, or the current one."""
    return torch._C._cuda_getCurrentRawStream(_device()) if stream is None else _stream_ptr(stream)


def _capturing(stream) -> bool:
    """Whether a call on `stream` becomes part of a graph."""
    if stream is None:
        return torch._C._cuda_isCurrentStreamCapturing()
    with torch.cuda.stream(stream):
        return torch._C._cuda_isCurrentStreamCapturing()


def _made(stream, make):
    """The new tensor make() for a call on `stream`."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        y = make()
    y.record_stream(torch.cuda.current_stream())
    return y


def _heads(x: torch.Tensor, tokens: int, dim: int, dtype: torch.dtype, what: str):
    """(pointer, heads, token stride, head stride) of a [tokens][heads][dim] tensor with contiguous heads."""
    if x.dtype is not dtype or x.dim() != 3 or x.get_device() != _device():
        raise TypeError(f"{what}: a tensor [tokens][heads][dim] of {dtype} on the current CUDA device is wanted")
    t, h, d = x.shape
    if t != tokens or d != dim:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, wanted [{tokens}][heads][{dim}]")
    st, sh, se = x.stride()
    if se != 1:
        raise ValueError(f"{what}: the elements of a head have to be contiguous")
    return x.data_ptr(), h, st, sh


def _int32(x: torch.Tensor, n: int, what: str) -> int:
    if x.dtype is not torch.int32 or x.get_device() != _device() or x.shape != (n,) or (n > 1 and x.stride(0) != 1):
        raise ValueError(f"{what}: a contiguous int32 tensor of {n} elements on the current CUDA device is wanted")
    return x.data_ptr()


def _row_stride(table: torch.Tensor) -> int:
    """The stride between a block table's rows; that of a single row says nothing, and is not used."""
    return table.stride(0) if table.shape[0] > 1 else table.shape[1]


def _output(given: torch.Tensor | None, like: torch.Tensor, heads: int, what: str, stream):
    """An output like a [tokens][heads][dim] input: (tensor, pointer, token stride, head stride)."""
    if given is None:
        y = _made(stream, lambda: torch.empty_like(like))
        st, sh, _ = y.stride()
        return y, y.data_ptr(), st, sh
    y = given
    p, h, st, sh = _heads(y, like.shape[0], like.shape[2], like.dtype, what)
    if h != heads:
        raise ValueError(f"{what}: {heads} heads are wanted")
    return y, p, st, sh


class _Turned(torch.autograd.Function):
    """Rotary.apply for heads that want a gradient: that of a turn is the turn back."""

    @staticmethod
    def forward(ctx, rotary, q, k, positions, inverse, stream):
        ctx.rotary, ctx.inverse = rotary, inverse
        ctx.save_for_backward(positions)
        return rotary._turn(q, k, positions, inverse, None, None, stream)

    @staticmethod
    def backward(ctx, *grads):
        # (a gradient may come expanded, and one of the two may not be there)
        heads = [None if g is None or not wanted else g if g.stride(2) == 1 else g.contiguous() for g, wanted in zip(grads, ctx.needs_input_grad[1:3])]
        there = [g for g in heads if g is not None]
        back = iter(ctx.rotary.apply(*there, *[None] * (2 - len(there)), *ctx.saved_tensors, inverse=not ctx.inverse) if there else ())
        return (None, *(None if g is None else next(back) for g in heads), None, None, None)


class Rotary:
    """Rotary positions (fluxbin_rotary): the frequencies live on the device, angles are formed in the kernels.

    `scaling`: "none", "linear" (factor), "base" (factor), "ramp" (factor, original, fast, slow) or "bands" (factor, original,
    low, high), see fluxbin_rotary_frequencies."""

    def __init__(self, head_dim: int, rotary_dim: int | None = None, base: float = 10000.0, interleaved: bool = False,
                 scaling: str = "none", factor: float = 1.0, original: float = 1.0, fast: float = 32.0, slow: float = 1.0,
                 low: float = 1.0, high: float = 4.0, device="cuda"):
        if scaling not in _KINDS:
            raise ValueError(f"scaling: one of {sorted(_KINDS)} is wanted")
        self.head_dim, self.rotary_dim, self.interleaved = head_dim, head_dim if rotary_dim is None else rotary_dim, bool(interleaved)
        if self.rotary_dim > head_dim:
            raise fluxbin.FluxBinError(3, "Rotary: rotary_dim past head_dim")
        a, b = (fast, slow) if scaling == "ramp" else (low, high)
        turns, self.magnitude = fluxbin.rotary_frequencies(self.rotary_dim, base, _KINDS[scaling], factor, original, a, b)
        self.turns = torch.from_numpy(turns.view("int64")).to(device)
        self.desc = fluxbin.RotaryDesc(head_dim, self.rotary_dim, int(self.interleaved), self.magnitude, self.turns.data_ptr())
        self._ref = ctypes.addressof(self.desc)

    def apply(self, q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor, inverse: bool = False,
              q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, stream=None):
        """q, k [tokens][heads][head_dim] turned to positions [tokens] (int32); outputs may be the inputs.  `inverse` turns
        back: the gradient of the turned heads with respect to q and k.  Returns (q_out, k_out), k_out None without k.  New
        outputs of heads that require a gradient carry it; outputs that were given are written without one."""
        if k is None:
            k_out = None
        wanted = q_out is None and q.requires_grad, k is not None and k_out is None and k.requires_grad
        if (wanted[0] or wanted[1]) and torch.is_grad_enabled():
            if q_out is None and k_out is None:
                return _Turned.apply(self, q, k, positions, inverse, stream)
            if wanted[0]:                                # (each by itself)
                return _Turned.apply(self, q, None, positions, inverse, stream)[0], self._turn(k, None, positions, inverse, k_out, None, stream)[0]
            return self._turn(q, None, positions, inverse, q_out, None, stream)[0], _Turned.apply(self, k, None, positions, inverse, stream)[0]
        return self._turn(q, k, positions, inverse, q_out, k_out, stream)

    def _turn(self, q, k, positions, inverse, q_out, k_out, stream):
        n, dt = q.shape[0], q.dtype
        if dt not in _TYPES:
            raise TypeError("q: fp16, bf16 or fp32 is wanted")
        if self.turns.get_device() != _device():
            raise ValueError("the frequencies have to lie on the current CUDA device")
        qp, qh, qt, qs = _heads(q, n, self.head_dim, dt, "q")
        q_out, op, ot, os_ = _output(q_out, q, qh, "q_out", stream)
        kp = kh = kt = ks = kop = kot = kos = 0
        if k is None:
            k_out = None
        else:
            kp, kh, kt, ks = _heads(k, n, self.head_dim, dt, "k")
            k_out, kop, kot, kos = _output(k_out, k, kh, "k_out", stream)
        fluxbin.rotary_call(self._ref, _TYPES[dt], inverse, n, _int32(positions, n, "positions"), qp, qh, qt, qs, op, ot, os_,
                            kp, kh, kt, ks, kop, kot, kos, _stream(stream))
        return q_out, k_out


class _NormedAndTurned(torch.autograd.Function):
    """NormedRotary.apply for heads or gains that want a gradient."""

    @staticmethod
    def forward(ctx, normed, q, k, q_weight, k_weight, positions, stream):
        ctx.normed, ctx.stream = normed, stream
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        ctx.set_materialize_grads(False)
        return normed._apply(q, k, q_weight, k_weight, positions, None, None, stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, q_grad, k_grad=None):
        return (None, *ctx.normed._backward(*ctx.saved_tensors, q_grad, k_grad, *ctx.needs_input_grad[1:5]), None, None)


class NormedRotary:
    """Norms of query and key heads and rotary positions in one pass (fluxbin_norm_rotary): the root mean square of a head's
    elements is taken out of them, a gain for each element comes in, then the head is turned by `rotary`.

    `q_weight`, `k_weight`: [head_dim] gains of one type (fp16, bf16 or fp32), None for 1; parameters may require a gradient."""

    def __init__(self, rotary: Rotary, q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6):
        if not 0.0 < eps < 3e38:
            raise ValueError("eps: a positive number is wanted")
        self.rotary, self.q_weight, self.k_weight, self.eps = rotary, q_weight, k_weight, float(eps)
        self._gains(q_weight, k_weight)

    def apply(self, q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor, q_out: torch.Tensor | None = None,
              k_out: torch.Tensor | None = None, stream=None):
        """q, k [tokens][heads][head_dim] normed and turned to positions [tokens] (int32); outputs may be the inputs.  Returns
        (q_out, k_out), k_out None without k.  New outputs carry gradients (of the heads and of the gains, the first ones; they are
        formed on the stream that the gradients come on); outputs that were given are written without."""
        qw, kw = self.q_weight, self.k_weight
        if k is None:
            k_out = None
        if torch.is_grad_enabled():
            wanted = (q_out is None and (q.requires_grad or (qw is not None and qw.requires_grad)),
                      k is not None and k_out is None and (k.requires_grad or (kw is not None and kw.requires_grad)))
            if wanted[0] or wanted[1]:
                if q_out is None and k_out is None:
                    return _NormedAndTurned.apply(self, q, k, qw, kw, positions, stream)
                if wanted[0]:                            # (each by itself)
                    return _NormedAndTurned.apply(self, q, None, qw, None, positions, stream)[0], self._apply(k, None, kw, None, positions, k_out, None, stream)[0]
                return self._apply(q, None, qw, None, positions, q_out, None, stream)[0], _NormedAndTurned.apply(self, k, None, kw, None, positions, stream)[0]
        return self._apply(q, k, qw, kw, positions, q_out, k_out, stream)

    def _gains(self, q_weight, k_weight):
        """What gains have to be."""
        for w, what in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if w is not None and (w.dtype not in _TYPES or w.shape != (self.rotary.head_dim,) or not w.is_contiguous()):
                raise ValueError(f"{what}: a contiguous tensor of {self.rotary.head_dim} gains in fp16, bf16 or fp32 is wanted")
        if q_weight is not None and k_weight is not None and q_weight.dtype is not k_weight.dtype:
            raise TypeError("q_weight, k_weight: one type is wanted")

    def _weights(self, q_weight, k_weight):
        """(type, addresses); parameters may have been given another type or size since the last call"""
        here, D, kind, qp, kp = _device(), self.rotary.head_dim, torch.float32, 0, 0
        if q_weight is not None:
            kind, qp = q_weight.dtype, q_weight.data_ptr()
            if q_weight.numel() != D or not q_weight.is_contiguous():
                self._gains(q_weight, k_weight)
            if q_weight.get_device() != here:
                raise ValueError("the gains have to lie on the current CUDA device")
        if k_weight is not None:
            if k_weight.numel() != D or not k_weight.is_contiguous() or (qp and k_weight.dtype is not kind):
                self._gains(q_weight, k_weight)
            if k_weight.get_device() != here:
                raise ValueError("the gains have to lie on the current CUDA device")
            kind, kp = k_weight.dtype, k_weight.data_ptr()
        if kind not in _TYPES:
            self._gains(q_weight, k_weight)
        return _TYPES[kind], qp, kp

    def _check(self, q):
        if q.dtype not in _TYPES:
            raise TypeError("q: fp16, bf16 or fp32 is wanted")
        if self.rotary.turns.get_device() != _device():
            raise ValueError("the frequencies have to lie on the current CUDA device")

    def _apply(self, q, k, q_weight, k_weight, positions, q_out, k_out, stream):
        self._check(q)
        n, dt, D = q.shape[0], q.dtype, self.rotary.head_dim
        wt, qw, kw = self._weights(q_weight, k_weight)
        qp, qh, qt, qs = _heads(q, n, D, dt, "q")
        q_out, op, ot, os_ = _output(q_out, q, qh, "q_out", stream)
        kp = kh = kt = ks = kop = kot = kos = 0
        if k is None:
            k_out = None
        else:
            kp, kh, kt, ks = _heads(k, n, D, dt, "k")
            k_out, kop, kot, kos = _output(k_out, k, kh, "k_out", stream)
        fluxbin.norm_rotary_call(self.rotary._ref, self.eps, _TYPES[dt], wt, n, _int32(positions, n, "positions"), qp, qh, qt, qs, qw, op, ot, os_,
                                 kp, kh, kt, ks, kw, kop, kot, kos, _stream(stream))
        return q_out, k_out

    def _backward(self, q, k, q_weight, k_weight, positions, q_grad, k_grad, *wanted):
        """The gradients of q, k and the gains, None where none is wanted or comes."""
        self._check(q)
        n, dt, D = q.shape[0], q.dtype, self.rotary.head_dim
        wt, *wp = self._weights(q_weight, k_weight)
        words, results, ws, held = [], [], None, []       # (what the call reads is held until it is queued)
        for x, g, w, weight, want, want_w, what in ((q, q_grad, wp[0], q_weight, wanted[0], wanted[2], "q"), (k, k_grad, wp[1], k_weight, wanted[1], wanted[3], "k")):
            if x is None or g is None or n == 0 or not (want or want_w):       # (tensors of no elements have no address)
                results += [torch.empty_like(x) if want and n == 0 else None, torch.zeros_like(weight) if want_w and x is not None else None]
                words += [0] * 12
                continue
            if g.stride(2) != 1 and D > 1:
                g = g.contiguous()
            held.append(g)
            xp, xh, xt, xs = _heads(x, n, D, dt, what)
            gp, gh, gt, gs = _heads(g, n, D, dt, what + "'s gradient")
            if gh != xh:
                raise ValueError(f"{what}'s gradient: {xh} heads are wanted")
            dx = torch.empty_like(x, memory_format=torch.contiguous_format) if want else None
            dw = torch.empty_like(weight) if want_w else None
            if want_w and ws is None:
                ws = torch.empty(fluxbin.norm_rotary_backward_workspace_size(D), dtype=torch.uint8, device=x.device)
            results += [dx, dw]
            words += [xp, xh, xt, xs, w, gp, gt, gs, 0 if dx is None else dx.data_ptr(), xh * D, D, 0 if dw is None else dw.data_ptr()]
        if held:
            fluxbin.norm_rotary_backward_call(self.rotary._ref, self.eps, _TYPES[dt], wt, n, _int32(positions, n, "positions"), *words,
                                              0 if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream(None))
        return results[0], results[2], results[1], results[3]


class KVCache:
    """Keys and values in 8 bits, in blocks of tokens, one scale for each block and key head (fluxbin_kv_cache_t).

    `k`, `v`: [num_blocks][kv_heads][block_tokens][head_dim] int8 or float8_e4m3fn tensors (any strides with contiguous
    elements, the same for both); `k_scale`, `v_scale`: fp32 [num_blocks][kv_heads].  `token_major` lays a block out as
    [block_tokens][kv_heads][head_dim] in memory."""

    def __init__(self, num_blocks: int, block_tokens: int, kv_heads: int, head_dim: int, fmt: str = "int8", token_major: bool = False,
                 device="cuda"):
        if fmt not in _FORMATS:
            raise ValueError(f"fmt: one of {sorted(_FORMATS)} is wanted")
        shape = (num_blocks, block_tokens, kv_heads, head_dim) if token_major else (num_blocks, kv_heads, block_tokens, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.int8, device=device).view(_FORMATS[fmt]) for _ in range(2))
        if token_major:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        scales = (torch.zeros((num_blocks, kv_heads), dtype=torch.float32, device=device) for _ in range(2))
        self._set(k, v, *scales)

    @classmethod
    def wrap(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor) -> "KVCache":
        """A cache over tensors that are there already."""
        c = object.__new__(cls)
        c._set(k, v, k_scale, v_scale)
        return c

    def _set(self, k, v, k_scale, v_scale):
        if k.dtype not in _STORED or v.dtype is not k.dtype:
            raise TypeError("k, v: int8 or float8_e4m3fn is wanted")
        if k.dim() != 4 or v.shape != k.shape or any(a != b for a, b, n in zip(k.stride(), v.stride(), k.shape) if n > 1) or k.stride(3) != 1:
            raise ValueError("k, v: [num_blocks][kv_heads][block_tokens][head_dim] with the same strides and contiguous elements are wanted")
        nb, H, bs, D = k.shape
        for s in (k_scale, v_scale):
            if s.dtype is not torch.float32 or s.shape != (nb, H) or not s.is_contiguous():
                raise ValueError("scales: contiguous fp32 [num_blocks][kv_heads] is wanted")
        if len({t.device for t in (k, v, k_scale, v_scale)}) != 1:
            raise ValueError("k, v and the scales have to be on one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_blocks, self.kv_heads, self.block_tokens, self.head_dim, self.device = nb, H, bs, D, k.device
        self.desc = fluxbin.CacheDesc(nb, bs, H, D, _STORED[k.dtype], k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2),
                                      k_scale.data_ptr(), v_scale.data_ptr())
        self._ref, self._scale, self._last = ctypes.addressof(self.desc), 1.0 / math.sqrt(D), {}
        status = fluxbin.kv_validate_status(self.desc)
        if status:
            raise fluxbin.FluxBinError(status, "fluxbin_kv_validate")

    def _new(self, shape: tuple, dtype: torch.dtype, stream) -> torch.Tensor:
        """torch.empty(shape, dtype) on the cache's device, made like the last one of that type (one element seen as many): half
        the time."""
        last = self._last.get(dtype)
        if last is None or last.shape != shape:
            last = self._last[dtype] = torch.empty((1,) * len(shape), dtype=dtype, device=self.device).expand(shape)
        return _made(stream, lambda: torch.empty_like(last, memory_format=torch.contiguous_format))

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, rotary: Rotary | None = None,
               positions: torch.Tensor | None = None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, stream=None):
        """fluxbin_kv_append: quantise and store k, v [tokens][kv_heads][head_dim] at `slots` [tokens] (int32).  With `rotary` the
        keys, and the q heads if given, are turned to `positions` on the way; returns the turned q (else None)."""
        n, dt = k.shape[0], k.dtype
        if self.k.get_device() != _device():
            raise ValueError("the cache has to lie on the current CUDA device")
        if dt not in _TYPES:
            raise TypeError("k: fp16, bf16 or fp32 is wanted")
        kp, kh, kt, ks = _heads(k, n, self.head_dim, dt, "k")
        vp, vh, vt, vs = _heads(v, n, self.head_dim, dt, "v")
        if kh != self.kv_heads or vh != self.kv_heads:
            raise ValueError(f"k, v: {self.kv_heads} heads are wanted")
        rp = pp = qp = qh = qt = qs = op = ot = os_ = 0
        if rotary is not None:
            if positions is None:
                raise ValueError("positions are wanted with rotary")
            if rotary.turns.get_device() != _device():
                raise ValueError("rotary: the frequencies have to lie on the current CUDA device")
            rp, pp = rotary._ref, _int32(positions, n, "positions")
            if q is not None:
                qp, qh, qt, qs = _heads(q, n, self.head_dim, dt, "q")
                q_out, op, ot, os_ = _output(q_out, q, qh, "q_out", stream)
        elif q is not None:
            raise ValueError("q is only turned with rotary")
        fluxbin.kv_append_call(self._ref, _TYPES[dt], n, _int32(slots, n, "slots"), kp, kt, ks, vp, vt, vs, rp, pp, qp, qh, qt, qs,
                               op, ot, os_, _stream(stream))
        return None if q is None else q_out

    def read(self, slots: torch.Tensor, dtype: torch.dtype = torch.float16, stream=None):
        """fluxbin_kv_read: the keys and values that the entries at `slots` stand for, two [tokens][kv_heads][head_dim] tensors."""
        if dtype not in _TYPES:
            raise TypeError("dtype: fp16, bf16 or fp32 is wanted")
        if self.k.get_device() != _device():
            raise ValueError("the cache has to lie on the current CUDA device")
        n = slots.shape[0]
        k, v = self._new((2, n, self.kv_heads, self.head_dim), dtype, stream).unbind()
        fluxbin.kv_read_call(self._ref, _TYPES[dtype], n, _int32(slots, n, "slots"), k.data_ptr(), v.data_ptr(), _stream(stream))
        return k, v

    def keep(self, slots: torch.Tensor, query_start: torch.Tensor, path: torch.Tensor, stream=None) -> None:
        """fluxbin_kv_keep: the entries of each request's `path` (int32 [tokens], DraftTree.accept) move to the first slots of its
        new tokens.  `slots` int32 [tokens] and `query_start` int32 [batch + 1] are those the tokens were appended with."""
        if self.k.get_device() != _device():
            raise ValueError("the cache has to lie on the current CUDA device")
        n, B = slots.shape[0], query_start.shape[0] - 1
        fluxbin.kv_keep_call(self._ref, B, n, _int32(query_start, B + 1, "query_start"), _int32(slots, n, "slots"), _int32(path, n, "path"), _stream(stream))

    def workspace(self, batch: int, tokens: int, q_heads: int, tree: bool = False) -> Workspace:
        """The workspace of attend() for up to `batch` requests with `tokens` new tokens in all, with `tree` also of trees of them."""
        size = fluxbin.kv_attend_tree_workspace_size if tree else fluxbin.kv_attend_workspace_size
        n = size(batch, tokens, q_heads, self.kv_heads, self.head_dim)
        if n == 0:
            raise ValueError("workspace: batch >= 1, tokens >= 0 and a multiple of kv_heads for q_heads are wanted")
        return Workspace(n, self.device)

    def attend(self, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, ws: Workspace, query_start: torch.Tensor | None = None,
               scale: float | None = None, out: torch.Tensor | None = None, with_lse: bool = False, stream=None,
               tree: torch.Tensor | None = None):
        """fluxbin_kv_attend: q [tokens][q_heads][head_dim] (fp16 or bf16) over the cached tokens of its requests.

        `table` int32 [batch][max_blocks] (its rows may be one row expanded over the batch), `lengths` int32 [batch] (the new tokens included), `query_start` int32
        [batch + 1] or None for one token a request, `scale` head_dim ** -0.5 if not given.  `tree` int32 [tokens][words]: which
        of its request's new tokens each one sees (fluxbin_kv_attend_tree; DraftTree.mask), those up to itself if not given; the
        workspace is then one for trees.  Returns out [tokens][q_heads]
        [head_dim], with `with_lse` also the natural log of each row's sum, fp32 [tokens][q_heads]."""
        n, dt = q.shape[0], q.dtype
        if dt is not torch.float16 and dt is not torch.bfloat16:
            raise TypeError("q: fp16 or bf16 is wanted")
        qp, qh, qt, qs = _heads(q, n, self.head_dim, dt, "q")
        if table.dtype is not torch.int32 or table.dim() != 2 or table.get_device() != _device() or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table: an int32 tensor [batch][max_blocks] with contiguous rows on the current CUDA device is wanted")
        if self.k.get_device() != _device():
            raise ValueError("the cache has to lie on the current CUDA device")
        if ws.tensor.get_device() != _device():
            raise ValueError("the workspace has to lie on the current CUDA device")
        B, width = table.shape
        call, masks = fluxbin.kv_attend_call, ()
        if tree is not None:
            if tree.dtype is not torch.int32 or tree.dim() != 2 or tree.shape[0] != n or tree.get_device() != _device() or (tree.shape[1] > 1 and tree.stride(1) != 1):
                raise ValueError("tree: an int32 tensor [tokens][words] with contiguous rows on the current CUDA device is wanted")
            call, masks = fluxbin.kv_attend_tree_call, (tree.data_ptr(), tree.stride(0), tree.shape[1])
        out, op, ot, os_ = _output(out, q, qh, "out", stream)
        lse = self._new((n, qh), torch.float32, stream) if with_lse else None
        call(self._ref, _TYPES[dt], B, n, qp, qh, qt, qs, 0 if query_start is None else _int32(query_start, B + 1, "query_start"),
             _int32(lengths, B, "lengths"), *masks, table.data_ptr(), _row_stride(table), width, self._scale if scale is None else scale,
             op, ot, os_, 0 if lse is None else lse.data_ptr(), ws.tensor.data_ptr(), ws.nbytes, _stream(stream))
        return (out, lse) if with_lse else out


class BlockTables:
    """The blocks of a batch of requests and the free list they come from (fluxbin_kv_advance).

    `table` int32 [batch][max_blocks] and `free` int32 [capacity] are changed in place by advance(); the lengths and the
    number of free blocks go in and come out."""

    def __init__(self, table: torch.Tensor, free: torch.Tensor, block_tokens: int):
        if table.dtype is not torch.int32 or table.dim() != 2 or table.get_device() != _device() or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table: an int32 tensor [batch][max_blocks] with contiguous rows on the current CUDA device is wanted")
        if _row_stride(table) < table.shape[1]:
            raise ValueError("table: rows that do not overlap are wanted (they are written)")
        self.table, self.free, self.block_tokens = table, free, block_tokens
        self._tokens, self._sets = None, {}              # the size of the last step; two sets of outputs of each of the last two sizes
        self._captured = []                              # sets that graphs write: as long as this object, whatever else it is asked
        self._free = _int32(free, free.shape[0], "free")
        self.batch, self.max_blocks = table.shape
        self._args = (table.data_ptr(), _row_stride(table), table.shape[1], self._free, free.shape[0])

    @classmethod
    def empty(cls, batch: int, max_blocks: int, num_blocks: int, block_tokens: int, device="cuda") -> "BlockTables":
        """No request holds a block yet: all num_blocks are free (the number of free blocks starts as num_blocks)."""
        return cls(torch.full((batch, max_blocks), -1, dtype=torch.int32, device=device),
                   torch.arange(num_blocks - 1, -1, -1, dtype=torch.int32, device=device), block_tokens)

    def advance(self, lengths: torch.Tensor, new_tokens: torch.Tensor, num_free: torch.Tensor, tokens: int, stream=None) -> SimpleNamespace:
        """One step: `new_tokens` int32 [batch] tokens to add (> 0) or drop (< 0), `tokens` the sum of those to add.  Returns
        lengths, num_free, granted, query_start, positions, slots, requests: int32 tensors that belong to this object, two
        sets in turn for each size, so that a step's outputs can be the next step's inputs; keep a copy of what has to live longer.  A step
        captured into a graph has a set of its own, which lives as long as this object."""
        B = self.batch
        lp, np_, fp = _int32(lengths, B, "lengths"), _int32(new_tokens, B, "new_tokens"), _int32(num_free, 1, "num_free")
        if self.table.get_device() != _device():
            raise ValueError("the tables have to lie on the current CUDA device")
        if _capturing(stream):
            step = self._outputs(tokens, stream)
            self._captured.append(step)
        else:
            sets = self._sets.get(tokens)                # (a decode loop has one size, one that drops drafted tokens has 0 besides)
            if sets is None:
                if len(self._sets) == 2:
                    self._sets = {self._tokens: self._sets[self._tokens]}
                sets = self._sets[tokens] = [self._outputs(tokens, stream), self._outputs(tokens, stream)]
            self._tokens = tokens
            step = sets[0]
            if step.first <= lp < step.last or step.first <= np_ < step.last or step.first <= fp < step.last:
                step = self._outputs(tokens, stream)     # an input of this step is an output of the last but one: keep that
            sets[0], sets[1] = sets[1], step
        on = _stream(stream)
        if on != step.made_on:                           # a set may be dropped while another stream still writes it
            step.num_free.record_stream(torch.cuda.current_stream() if stream is None else stream)
        fluxbin.kv_advance_call(B, tokens, self.block_tokens, lp, np_, *self._args, fp, *step.pointers, on)
        return step

    def _outputs(self, tokens: int, stream) -> SimpleNamespace:
        B = self.batch
        sizes = (1, B, B, B + 1, tokens, tokens, tokens)
        parts = _made(stream, lambda: torch.empty(sum(sizes), dtype=torch.int32, device=self.table.device)).split(sizes)
        step = SimpleNamespace(**dict(zip(("num_free", "lengths", "granted", "query_start", "positions", "slots", "requests"), parts)))
        first = parts[0].data_ptr()
        step.pointers = tuple(first + 4 * sum(sizes[:i]) for i in range(7))
        step.first, step.last, step.made_on = first, first + 4 * sum(sizes), _stream(stream)
        return step


class DraftTree:
    """The drafted tokens of a step, each behind another one of its request's (its parent) or behind the request's cached tokens
    (fluxbin_draft_tree).

    `parents` int32 [tokens]: the place of a token's parent among its request's new tokens, -1 for none; `query_start` int32
    [batch + 1] and `lengths` int32 [batch] (the new tokens included) as for KVCache.attend; `nodes` the most new tokens of a
    request that count, up to 1024.  Then `mask` int32 [tokens][ceil(nodes / 32)] says which of its request's new tokens each one sees,
    and `positions` int32 [tokens] where it stands."""

    def __init__(self, parents: torch.Tensor, query_start: torch.Tensor, lengths: torch.Tensor, nodes: int, stream=None):
        n, B = parents.shape[0], lengths.shape[0]
        if not 1 <= nodes <= 1024:
            raise ValueError("nodes: 1 to 1024 are wanted")
        pointers = _int32(query_start, B + 1, "query_start"), _int32(lengths, B, "lengths"), _int32(parents, n, "parents")
        self.parents, self.query_start, self.nodes = parents, query_start, nodes
        self.mask = _made(stream, lambda: torch.empty((n, -(-nodes // 32)), dtype=torch.int32, device=parents.device))
        self.positions = _made(stream, lambda: torch.empty_like(parents))
        fluxbin.draft_tree_call(B, n, nodes, *pointers, self.mask.data_ptr(), self.positions.data_ptr(), _stream(stream))

    def accept(self, drafted: torch.Tensor, answers: torch.Tensor, stream=None) -> SimpleNamespace:
        """fluxbin_draft_accept: the path of each request's tree that the model itself would have answered.  `drafted` int32
        [tokens]: the new tokens; `answers` int32 [tokens]: what the model answered at each.  Returns `path` int32 [tokens] (places
        among the request's new tokens, then -1: for KVCache.keep), and int32 [batch] `count`, tokens of the path, `answer`, what
        comes after it, `surplus`, what is to be dropped (as BlockTables.advance takes it; nothing of requests that were not granted
        their blocks, whose tokens were not added: times the step's `granted`)."""
        n, B = self.parents.shape[0], self.query_start.shape[0] - 1
        inputs = (_int32(self.query_start, B + 1, "query_start"), _int32(self.parents, n, "parents"), _int32(drafted, n, "drafted"), _int32(answers, n, "answers"))
        path = _made(stream, lambda: torch.empty_like(self.parents))
        three = _made(stream, lambda: torch.empty((3, B), dtype=torch.int32, device=self.parents.device))
        at = three.data_ptr()
        fluxbin.draft_accept_call(B, n, self.nodes, *inputs, path.data_ptr(), at, at + 4 * B, at + 8 * B, _stream(stream))
        count, answer, surplus = three.unbind()
        return SimpleNamespace(path=path, count=count, answer=answer, surplus=surplus)


class AttentionBlock:
    """The attention block of a decoder layer on packed linears: q/k/v projections, positions, cache, attention, output
    projection.  `q`, `k`, `v`, `o` are FluxBinLinear layers; the cache and the block tables may serve a whole batch of requests.
    A NormedRotary in the place of `rotary` norms the heads too."""

    def __init__(self, q, k, v, o, cache: KVCache, rotary: Rotary | NormedRotary):
        D = cache.head_dim
        if k.M != cache.kv_heads * D or v.M != k.M or q.M % k.M or o.N != q.M or not q.N == k.N == v.N == o.M:
            raise ValueError("the layers do not fit the cache's heads and each other")
        self.q, self.k, self.v, self.o, self.cache, self.rotary, self.q_heads = q, k, v, o, cache, rotary, q.M // D

    def buffers(self, batch: int, tokens: int, tree: bool = False) -> SimpleNamespace:
        """What forward() works in for up to `tokens` new tokens of `batch` requests (`tree`: also for trees of them), and its input x
        [tokens][hidden] and output y: q, k and v run as one plan, so the buffers are theirs."""
        from .layer import FluxBinPlan
        new = lambda n: torch.empty((tokens, n), dtype=torch.float16, device=self.cache.device)  # noqa: E731
        b = SimpleNamespace(x=new(self.q.N), q=new(self.q.M), k=new(self.k.M), v=new(self.v.M), a=new(self.q.M), y=new(self.o.M))
        b.plan = FluxBinPlan([(self.q, b.x, b.q), (self.k, b.x, b.k), (self.v, b.x, b.v)], device=self.cache.device)
        b.linear_ws, b.ws = self.o.workspace(tokens), self.cache.workspace(batch, tokens, self.q_heads, tree)
        return b

    def forward(self, b: SimpleNamespace, tables: BlockTables, step: SimpleNamespace, stream=None, tree: DraftTree | None = None) -> torch.Tensor:
        """y = o(attention(x)) for the new tokens of `step` (BlockTables.advance) in b.x; the result is b.y (of tokens past the
        step's own: o(0)).  With `tree` they stand and see as it says, and follow each other without.  A decode step is three
        launches besides the output projection (the append of a prompt turns its queries in one of its own, normed heads take one
        more, and projections of many tokens take several); nothing is allocated, so a step can be captured into a graph."""
        n, D = b.x.shape[0], self.cache.head_dim
        b.plan.run(stream)
        q, a = b.q.view(n, self.q_heads, D), b.a.view(n, self.q_heads, D)
        k, v = b.k.view(n, -1, D), b.v.view(n, -1, D)
        positions = step.positions if tree is None else tree.positions
        if isinstance(self.rotary, NormedRotary):
            self.rotary.apply(q, k, positions, q_out=q, k_out=k, stream=stream)
            self.cache.append(k, v, step.slots, stream=stream)
        else:
            self.cache.append(k, v, step.slots, rotary=self.rotary, positions=positions, q=q, q_out=q, stream=stream)
        self.cache.attend(q, tables.table, step.lengths, b.ws, query_start=step.query_start, out=a, stream=stream,
                          tree=None if tree is None else tree.mask)
        return self.o.forward(b.a, b.linear_ws, out=b.y, stream=stream)
