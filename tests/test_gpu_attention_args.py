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


@pytest.mark.parametrize("Hq,H,D,dtype", [(8, 2, 64, "fp16"), (16, 1, 128, "bf16"), (4, 4, 256, "fp16"), (40, 1, 128, "fp16")])
@pytest.mark.parametrize("before,after", [(0, 3), (2, 0), (1, 700), (0, 0)])
def test_tokens_of_no_request_get_empty_rows(at, Hq, H, D, dtype, before, after):  # noqa: F811
    lengths, new = [40, 3, 90], [1, 2, 0]
    c, table = setup(at, "int8", 16, H, D, lengths, 4)
    starts = before + np.concatenate([[0], np.cumsum(new)])
    n = before + 3 + after
    q = normal(71, (n, Hq, D), dtype)
    out = torch.full((Hq, n, D), float("nan"), dtype=q.dtype, device="cuda").transpose(0, 1)
    ws = c.workspace(3, n, Hq)
    _, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), out=out, with_lse=True)
    check_attend(c, q, table, lengths, starts, D ** -0.5, out, lse, dtype)        # (the definition's rows of no request: 0 and -inf)
    nobody = torch.ones(n, dtype=torch.bool)
    nobody[before:before + 3] = False
    assert (out[nobody] == 0).all() and (lse[nobody] == float("-inf")).all()
    # no request asks at all
    out.fill_(float("nan"))
    _, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev([n] * 4 if before else [0] * 4), out=out, with_lse=True)
    assert (out == 0).all() and (lse == float("-inf")).all()


def test_a_block_with_room_for_more_tokens_than_there_are(at):  # noqa: F811
    """A graph's fixed number of tokens: rows past the last request's come out as the output projection of 0."""
    from paper_2608_15602_b200 import layer, synth
    hq, hk, dim, hidden, B, T, room = 4, 2, 64, 128, 2, 5, 9
    L = [synth.make_linear(5, i, M, N) for i, (M, N) in enumerate([(hq * dim, hidden), (hk * dim, hidden), (hk * dim, hidden), (hidden, hq * dim)])]
    rows = []
    for n in (T, room):
        block = at.AttentionBlock(*[layer.FluxBinLinear(x) for x in L], at.KVCache(8, 16, hk, dim), at.Rotary(dim))
        tables = at.BlockTables.empty(B, 4, 8, 16)
        buf = block.buffers(B, n)
        buf.x.copy_(normal(81, (room, hidden), "fp16")[:n])
        buf.a.fill_(float("nan"))
        rows.append(block.forward(buf, tables, tables.advance(dev([0] * B), dev([3, 2]), dev([8]), n)).clone())
    assert torch.equal(rows[0], rows[1][:T]) and (rows[1][T:] == 0).all()


def test_strides_of_axes_of_one(at):  # noqa: F811
    D, L = 64, 40
    c, table = setup(at, "int8", 16, 1, D, [L], 9)
    for Hq in (1, 4):
        q = normal(91, (1, Hq, D), "fp16")
        odd = torch.as_strided(q, (1, Hq, D), (3, D if Hq > 1 else 5, 1))
        out = torch.empty(Hq * D, dtype=q.dtype, device="cuda")
        ws = c.workspace(1, 1, Hq)
        want = c.attend(q, dev(table), dev([L]), ws)
        c.attend(odd, dev(table), dev([L]), ws, out=torch.as_strided(out, (1, Hq, D), (1, D if Hq > 1 else 7, 1)))
        assert torch.equal(out.view(1, Hq, D), want)
    one = at.KVCache.wrap(torch.as_strided(torch.zeros(1024, dtype=torch.int8, device="cuda"), (1, 1, 16, D), (1, 7, D, 1)),
                          torch.as_strided(torch.zeros(1024, dtype=torch.int8, device="cuda"), (1, 1, 16, D), (2, 9, D, 1)),
                          *(torch.zeros(1, 1, device="cuda") for _ in range(2)))
    plain = at.KVCache(1, 16, 1, D)
    k, v = normal(92, (5, 1, D), "fp16"), normal(93, (5, 1, D), "fp16")
    for x in (one, plain):
        x.append(k, v, dev(np.arange(5)))
    for a, b in zip(one.read(dev(np.arange(5))), plain.read(dev(np.arange(5)))):
        assert torch.equal(a, b)
    q = normal(94, (1, 2, D), "fp16")
    assert torch.equal(*(x.attend(q, dev([[0]]), dev([5]), x.workspace(1, 1, 2)) for x in (one, plain)))
