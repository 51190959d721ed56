"""The attention block of a decoder layer -- packed linears, positions, cache, attention, output projection -- over prompts
and decode steps, against the 64-bit oracles of its parts.

Between the parts everything is rounded to fp16 (2^-11 of a value) five times, and keys and values to 8 bits, where the
oracle rounds the same way but may fall on the other side of a tie for the few entries that lie within fp32 rounding of one.
Rounding errors of 2^-11 in x, q, k, v, a and the 8-bit ones' ties add up to well below 1e-2 of a row's norm."""
import os
import sys

import numpy as np
import pytest

import oracle
from oracle import attention as oa
from paper_2608_15602_b200 import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt,hq,hk,dim,bs", [("int8", 8, 2, 64, 16), ("e4m3", 4, 4, 128, 32)])
def test_prompts_and_decode_steps(fmt, hq, hk, dim, bs):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_15602_b200 import build
    build.build()
    from paper_2608_15602_b200 import attention, layer
    hidden, B, width = 256, 3, 4
    L = [synth.make_linear(5, i, M, N, 2, 1, 128, synth.salient_random(5, i, N, 0.05))
         for i, (M, N) in enumerate([(hq * dim, hidden), (hk * dim, hidden), (hk * dim, hidden), (hidden, hq * dim)])]
    block = attention.AttentionBlock(*[layer.FluxBinLinear(x) for x in L], attention.KVCache(B * width, bs, hk, dim, fmt), attention.Rotary(dim))
    tables = attention.BlockTables.empty(B, width, B * width, bs)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    f, m = oa.frequencies(dim)
    zero = np.zeros((B * width, hk, bs, dim))
    ck, cv = oa.Cache(zero, np.zeros((B * width, hk)), fmt), oa.Cache(zero, np.zeros((B * width, hk)), fmt)
    half = lambda a: np.asarray(a, np.float64).astype(np.float16)  # noqa: E731
    lengths, free = i32([0] * B), i32([B * width])
    for new in ([7, 20, 1], [1, 1, 1], [1, 3, 1], [1, 1, 1]):
        T = sum(new)
        buf = block.buffers(B, T)
        x = synth.make_activations(9, T, T, hidden)
        buf.x.copy_(torch.from_numpy(x.view(np.float16)))
        step = tables.advance(lengths, i32(new), free, T)
        y = block.forward(buf, tables, step).cpu().numpy().astype(np.float64)
        slots, pos = step.slots.cpu().numpy(), step.positions.cpu().numpy()
        q, k, v = (half(oracle.linear_direct(l, x)).reshape(T, -1, dim) for l in L[:3])
        q = half(oa.rotary(q, pos, f, m, dim, False))
        ck.append(oa.rotary(k, pos, f, m, dim, False), slots)
        cv.append(v, slots)
        a = oa.attend(q, ck.values(), cv.values(), tables.table.cpu().numpy(), step.lengths.tolist(), step.query_start.tolist(), dim ** -0.5)[0]
        want = oracle.linear_direct(L[3], half(a).reshape(T, hq * dim).view(np.uint16))
        for t in range(T):
            assert np.linalg.norm(y[t] - want[t]) <= 1e-2 * np.linalg.norm(want[t]), (new, t)
        lengths, free = step.lengths.clone(), step.num_free.clone()


def test_block_refuses_layers_that_do_not_fit():
    from paper_2608_15602_b200 import attention, layer
    lins = [layer.FluxBinLinear(synth.make_linear(5, i, M, N)) for i, (M, N) in enumerate([(256, 128), (128, 128), (128, 128), (128, 256)])]
    cache, rope = attention.KVCache(4, 16, 2, 64), attention.Rotary(64)
    attention.AttentionBlock(*lins, cache, rope)
    for bad in [(lins[0], lins[1], lins[0], lins[3]), (lins[1], lins[0], lins[0], lins[3]), (lins[0], lins[1], lins[2], lins[0])]:
        with pytest.raises(ValueError):
            attention.AttentionBlock(*bad, cache, rope)


def test_example_runs():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import decode_attention
        argv, sys.argv = sys.argv, ["decode_attention.py", "--batch", "3", "--prompt", "20", "--steps", "5", "--heads", "4", "--kv-heads", "2", "--head-dim", "64"]
        try:
            decode_attention.main()
        finally:
            sys.argv = argv
    finally:
        sys.path.pop(0)
