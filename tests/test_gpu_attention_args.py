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


def test_calls_on_a_stream_of_their_own_while_the_current_one_is_busy(at):  # noqa: F811
    """The current stream still has to read tensors that were dropped: what a call on another stream allocates is not theirs."""
    B, Hq, H, D, bs = 6, 8, 2, 64, 16
    c, plain = at.KVCache(40, bs, H, D), at.KVCache(40, bs, H, D)
    r = at.Rotary(D)
    tables, other = at.BlockTables.empty(B, 4, 40, bs), at.BlockTables.empty(B, 4, 40, bs)
    ws, ws2 = c.workspace(B, B, Hq), plain.workspace(B, B, Hq)
    q, k, v = normal(1, (B, Hq, D), "fp16"), normal(2, (B, H, D), "fp16"), normal(3, (B, H, D), "fp16")
    lengths, ones, nf = dev([0] * B), dev([1] * B), dev([40])
    s = torch.cuda.Stream()

    def step(c, tables, ws, **kw):
        st = tables.advance(lengths, ones, nf, B, **kw)
        qr = c.append(k, v, st.slots, rotary=r, positions=st.positions, q=q, **kw)
        qk = r.apply(q, k, st.positions, **kw)
        out = c.attend(qr, tables.table, st.lengths, ws, query_start=st.query_start, with_lse=True, **kw)
        return [st.lengths, st.slots, qr, *qk, *out, *c.read(st.slots, **kw)]

    want = step(plain, other, ws2)
    sizes = [w.numel() * w.element_size() for w in want] + [4 * (2 + 3 * B + 3 * B)]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                        # about a tenth of a second
    dropped = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    copies = [d.clone() for d in dropped]
    del dropped
    got = step(c, tables, ws, stream=s)
    torch.cuda.synchronize()
    assert all((x == 9).all() for x in copies)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
