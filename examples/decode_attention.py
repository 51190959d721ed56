"""One decoder layer's attention block as a server would run it: prompts go into the 8-bit cache, then decode steps are
replayed from a CUDA graph -- block tables, q/k/v projections, positions, cache, attention, output projection, with no word
from the host between steps.

    python examples/decode_attention.py [--batch 16] [--prompt 500] [--steps 64] [--heads 64] [--kv-heads 8] [--format int8]

Random weights and activations of the 70B-shaped decode stack's attention layers by default."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_15602_b200 import attention, layer, synth  # noqa: E402


def make_block(hidden, q_heads, kv_heads, dim, fmt, num_blocks, block_tokens, seed=1):
    sizes = [(q_heads * dim, hidden), (kv_heads * dim, hidden), (kv_heads * dim, hidden), (hidden, q_heads * dim)]
    lins = [layer.FluxBinLinear(synth.make_linear(seed, i, M, N, 2, 0, 128)) for i, (M, N) in enumerate(sizes)]
    return attention.AttentionBlock(*lins, attention.KVCache(num_blocks, block_tokens, kv_heads, dim, fmt), attention.Rotary(dim))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=500)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--format", choices=["int8", "e4m3"], default="int8")
    ap.add_argument("--block-tokens", type=int, default=16)
    args = ap.parse_args()
    B, hidden = args.batch, args.heads * args.head_dim
    rng = np.random.default_rng(0)
    prompts = rng.integers(max(1, args.prompt // 2), args.prompt + 1, B).astype(np.int32)
    width = -(-(args.prompt + args.steps) // args.block_tokens)
    block = make_block(hidden, args.heads, args.kv_heads, args.head_dim, args.format, B * width, args.block_tokens)
    tables = attention.BlockTables.empty(B, width, B * width, args.block_tokens)

    # the prompts of all requests in one pass
    total = int(prompts.sum())
    buf = block.buffers(B, total)
    buf.x.normal_()
    step = tables.advance(torch.zeros(B, dtype=torch.int32, device="cuda"), torch.from_numpy(prompts).cuda(),
                          torch.tensor([B * width], dtype=torch.int32, device="cuda"), total)
    block.forward(buf, tables, step)
    lengths, num_free = step.lengths.clone(), step.num_free.clone()

    # a decode step, captured once: lengths and the free list go on from where the last step left them
    buf = block.buffers(B, B)
    buf.x.normal_()
    ones = torch.ones(B, dtype=torch.int32, device="cuda")

    def decode():
        step = tables.advance(lengths, ones, num_free, B)
        block.forward(buf, tables, step)
        lengths.copy_(step.lengths)
        num_free.copy_(step.num_free)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    steps = max(1, args.steps - 1)
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    assert lengths.tolist() == (prompts + args.steps).tolist() if args.steps > 1 else True
    assert torch.isfinite(buf.y).all()
    held = int(lengths.sum()) * args.kv_heads * args.head_dim * 2
    print(f"{B} requests of {int(prompts.min())} to {int(prompts.max())} prompt tokens, {steps} decode steps: "
          f"{begin.elapsed_time(end) / steps * 1e3:.1f} us a step ({args.heads}/{args.kv_heads} heads of {args.head_dim}, {args.format} cache, "
          f"{held / 1e6:.1f} MB of it read by the last step)")


if __name__ == "__main__":
    main()
