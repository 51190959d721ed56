"""Calls of the attention side with tensors of unusual strides, against the same calls with plain ones."""
import numpy as np
import pytest

from test_gpu_attention import at, check_attend, dev, normal, setup  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_one_row_of_blocks_for_all_requests(at):  # noqa: F811
    """Samples of one prompt: the table's row expanded over the batch."""
    Hq, H, D, B, L = 8, 2, 64, 5, 90
    c, table = setup(at, "int8", 16, H, D, [L], 3)
    q = normal(61, (B, Hq, D), "fp16")
    lengths = [90, 80, 16, 1, 33]
    ws = c.workspace(B, B, Hq)
    row = dev(table)
    out, lse = c.attend(q, row.expand(B, -1), dev(lengths), ws, with_lse=True)
    check_attend(c, q, np.repeat(table, B, 0), lengths, np.arange(B + 1), D ** -0.5, out, lse, "fp16")
    assert torch.equal(out, c.attend(q, row.repeat(B, 1), dev(lengths), ws))


def test_a_captured_step_and_steps_of_other_sizes(at):  # noqa: F811
    """Warm-up, capture, then a prompt of another size through the same tables and new tensors in whatever memory is free: the
    graph goes on with what is its own."""
    B, bs = 3, 16
    t = at.BlockTables.empty(B, 8, 24, bs)
    lengths, nf, ones = dev([0] * B), dev([24]), dev([1] * B)
    kept = {}

    def step():
        s = t.advance(lengths, ones, nf, B)
        lengths.copy_(s.lengths)
        nf.copy_(s.num_free)
        kept["slots"] = s.slots.data_ptr()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
        step()
    g.replay()
    s = t.advance(lengths, dev([20, 0, 7]), nf, 27)
    lengths.copy_(s.lengths)
    nf.copy_(s.num_free)
    others = [torch.full((n,), 7, dtype=torch.int32, device="cuda") for n in (1, B, 3 * B, 7 * B, 64) for _ in range(200)]
    for _ in range(4):
        g.replay()
    s = t.advance(lengths, ones, nf, B)
    assert lengths.tolist() == [31, 11, 18] and s.lengths.tolist() == [32, 12, 19] and s.positions.tolist() == [31, 11, 18]
    assert all((o == 7).all() for o in others)
    used = t.table.cpu().numpy()
    held = [b for r, n in enumerate(s.lengths.tolist()) for b in used[r, :-(-n // bs)]]
    assert len(set(held)) == len(held) == 24 - int(s.num_free[0])
