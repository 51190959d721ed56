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

Rotary.apply carries gradients.  The other calls are those of answering: their results have none.
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
        if q_out is None and k_out is None and (q.requires_grad or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
            return _Turned.apply(self, q, k, positions, inverse, stream)
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

    def workspace(self, batch: int, tokens: int, q_heads: int) -> Workspace:
        """The workspace of attend() for up to `batch` requests with `tokens` new tokens in all."""
        n = fluxbin.kv_attend_workspace_size(batch, tokens, q_heads, self.kv_heads, self.head_dim)
        if n == 0:
            raise ValueError("workspace: batch >= 1, tokens >= 0 and a multiple of kv_heads for q_heads are wanted")
        return Workspace(n, self.device)

    def attend(self, q: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, ws: Workspace, query_start: torch.Tensor | None = None,
               scale: float | None = None, out: torch.Tensor | None = None, with_lse: bool = False, stream=None):
        """fluxbin_kv_attend: q [tokens][q_heads][head_dim] (fp16 or bf16) over the cached tokens of its requests.

        `table` int32 [batch][max_blocks] (its rows may be one row expanded over the batch), `lengths` int32 [batch] (the new tokens included), `query_start` int32
        [batch + 1] or None for one token a request, `scale` head_dim ** -0.5 if not given.  Returns out [tokens][q_heads]
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
        out, op, ot, os_ = _output(out, q, qh, "out", stream)
        lse = self._new((n, qh), torch.float32, stream) if with_lse else None
        fluxbin.kv_attend_call(self._ref, _TYPES[dt], B, n, qp, qh, qt, qs, 0 if query_start is None else _int32(query_start, B + 1, "query_start"),
                               _int32(lengths, B, "lengths"), table.data_ptr(), _row_stride(table), width,
                               self._scale if scale is None else scale, op, ot, os_, 0 if lse is None else lse.data_ptr(), ws.tensor.data_ptr(),
                               ws.nbytes, _stream(stream))
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
        self._tokens = self._sets = None
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
        sets in turn, so that a step's outputs can be the next step's inputs; keep a copy of what has to live longer.  A step
        captured into a graph has a set of its own, which lives as long as this object."""
        B = self.batch
        lp, np_, fp = _int32(lengths, B, "lengths"), _int32(new_tokens, B, "new_tokens"), _int32(num_free, 1, "num_free")
        if self.table.get_device() != _device():
            raise ValueError("the tables have to lie on the current CUDA device")
        if _capturing(stream):
            step = self._outputs(tokens, stream)
            self._captured.append(step)
        else:
            if tokens != self._tokens:                   # (a decode loop keeps one size)
                self._tokens, self._sets = tokens, [self._outputs(tokens, stream), self._outputs(tokens, stream)]
            step, other = self._sets
            self._sets = [other, step]
            if step.first <= lp < step.last or step.first <= np_ < step.last or step.first <= fp < step.last:
                step = self._sets[1] = self._outputs(tokens, stream)  # an input of this step is an output of the last but one: keep that
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


class AttentionBlock:
    """The attention block of a decoder layer on packed linears: q/k/v projections, positions, cache, attention, output
    projection.  `q`, `k`, `v`, `o` are FluxBinLinear layers; the cache and the block tables may serve a whole batch of requests."""

    def __init__(self, q, k, v, o, cache: KVCache, rotary: Rotary):
        D = cache.head_dim
        if k.M != cache.kv_heads * D or v.M != k.M or q.M % k.M or o.N != q.M or not q.N == k.N == v.N == o.M:
            raise ValueError("the layers do not fit the cache's heads and each other")
        self.q, self.k, self.v, self.o, self.cache, self.rotary, self.q_heads = q, k, v, o, cache, rotary, q.M // D

    def buffers(self, batch: int, tokens: int) -> SimpleNamespace:
        """What forward() works in for up to `tokens` new tokens of `batch` requests, and its input x [tokens][hidden]
        and output y: q, k and v run as one plan, so the buffers are theirs."""
        from .layer import FluxBinPlan
        new = lambda n: torch.empty((tokens, n), dtype=torch.float16, device=self.cache.device)  # noqa: E731
        b = SimpleNamespace(x=new(self.q.N), q=new(self.q.M), k=new(self.k.M), v=new(self.v.M), a=new(self.q.M), y=new(self.o.M))
        b.plan = FluxBinPlan([(self.q, b.x, b.q), (self.k, b.x, b.k), (self.v, b.x, b.v)], device=self.cache.device)
        b.linear_ws, b.ws = self.o.workspace(tokens), self.cache.workspace(batch, tokens, self.q_heads)
        return b

    def forward(self, b: SimpleNamespace, tables: BlockTables, step: SimpleNamespace, stream=None) -> torch.Tensor:
        """y = o(attention(x)) for the new tokens of `step` (BlockTables.advance) in b.x; the result is b.y (of tokens past the
        step's own: o(0)).  A decode step is three launches besides the output projection (the append of a prompt turns its
        queries in one of its own, and projections of many tokens take several); nothing is allocated, so a step can be captured
        into a graph."""
        n, D = b.x.shape[0], self.cache.head_dim
        b.plan.run(stream)
        q, a = b.q.view(n, self.q_heads, D), b.a.view(n, self.q_heads, D)
        k, v = b.k.view(n, -1, D), b.v.view(n, -1, D)
        self.cache.append(k, v, step.slots, rotary=self.rotary, positions=step.positions, q=q, q_out=q, stream=stream)
        self.cache.attend(q, tables.table, step.lengths, b.ws, query_start=step.query_start, out=a, stream=stream)
        return self.o.forward(b.a, b.linear_ws, out=b.y, stream=stream)
