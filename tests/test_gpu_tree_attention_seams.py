"""Attention under masks where jobs are cut between CTAs, seen from the values' side, and scales that are no number.

Values are 0 but for one token of every 16, which is positive and has an element of its own among its neighbours: a group of tokens that
is lost, or counted twice, changes an element by a good part of itself.  The mean of |v| is then the result, so the bound of the attention tests is
one of the result's own size:
    |error| <= u |out| + (2^-15 + 2^-19 + (2 D + 8) 2^-24 S + L 2^-23) |out|, and 1e-7 for what fp16 holds to steps"""
import numpy as np
import pytest

from oracle import drafts as od
from test_gpu_attention import U, at, dev, entries_of, f64, normal, setup  # noqa: F401
from test_gpu_drafts import batch_of
from test_gpu_tree_attention import check_tree, clean

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def sees_of(mask, a, n):
    return torch.tensor([[(int(mask[a + i, j // 32]) >> (j % 32)) & 1 for j in range(n)] for i in range(n)], dtype=torch.bool, device="cuda")


@pytest.mark.parametrize("fmt,dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("Hq,H,D,nodes,length", [(8, 1, 128, 16, 20001), (16, 2, 64, 40, 9999), (4, 4, 128, 5, 5003), (6, 2, 256, 24, 4097), (64, 1, 128, 9, 6000),
                                                 (4, 1, 256, 3, 7777), (2, 1, 64, 11, 12345), (12, 1, 256, 40, 3333), (8, 1, 64, 63, 30000)])
def test_no_group_of_tokens_is_lost_or_counted_twice(at, Hq, H, D, nodes, length, fmt, dtype):  # noqa: F811
    lengths, new = [length, length // 7, nodes, length // 3], [nodes, 1, nodes, nodes]
    c, table = setup(at, fmt, 16, H, D, lengths, 5)
    clean(c)
    parents, starts = batch_of(np.random.default_rng(length), new, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
    mask, T = tree.mask.cpu().numpy(), sum(new)
    ws = c.workspace(4, T, Hq, tree=True)
    for turn, spread in ((0, 0.0), (7, 0.0), (15, 1.0)):
        c.v.view(torch.uint8).zero_()
        for r, L in enumerate(lengths):
            blocks = dev(table[r, :-(-L // 16)]).long()
            i = torch.arange(len(blocks), device="cuda")
            one = torch.zeros(len(blocks), D, device="cuda")
            one[i, i % D] = 120.0
            c.v[blocks, :, turn] = one[:, None].to(c.v.dtype)
        q = normal(9, (T, Hq, D), dtype, spread)
        nothing = torch.full_like(q, float("nan"))
        out = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), tree=tree.mask, out=nothing)
        for r, L in enumerate(lengths):
            a, n = starts[r], new[r]
            ids = dev(table[r, :-(-L // 16)]).long()
            k, v = (x[ids].double() * s[ids].double()[..., None, None] for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
            k, v = (x.transpose(0, 1).reshape(H, -1, D)[:, :L] for x in (k, v))
            qq = q[a:a + n].double().view(n, H, Hq // H, D)
            x = torch.einsum("nhgd,hld->nhgl", qq, k) * D ** -0.5
            x[..., L - n:] = x[..., L - n:].masked_fill(~sees_of(mask, a, n)[:, None, None, :], float("-inf"))
            want = torch.einsum("nhgl,hld->nhgd", torch.softmax(x, -1), v)
            S = torch.einsum("nhgd,hld->nhgl", qq.abs(), k.abs()).amax(-1)[..., None] * D ** -0.5
            bound = (U[dtype] + 2.0 ** -15 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * want + 1e-7
            got = out[a:a + n].double().view(n, H, Hq // H, D)
            assert ((got - want).abs() <= bound).all(), (r, turn, ((got - want).abs() / bound).max())


def check_rows(c, q, table, lengths, starts, mask, scale, out, lse, dtype, rows):
    """check_tree for some of the tokens."""
    k, v = (e * f64(s)[:, :, None, None] for e, s in zip(entries_of(c), (c.k_scale, c.v_scale)))
    want, wl, mean, size = (x[rows] for x in od.attend(f64(q), k, v, table, lengths, starts, mask, scale))
    D, L, S = q.shape[2], max(lengths), size[:, :, None]
    bound = U[dtype] * np.abs(want) + (2.0 ** -15 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * mean
    assert (np.abs(f64(out)[rows] - want) <= bound).all()
    assert (np.abs(f64(lse)[rows] - wl) <= (D + 4) * 2.0 ** -24 * size + 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -23 * np.abs(wl)).all()


# few rows (the kernel of chains, with masks) and many, at every head dimension: new tokens 0 to 7 lie in one block, the others in the next ones
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,nodes", [(4, 4, 128, 16), (2, 2, 128, 12), (2, 2, 64, 30), (2, 2, 256, 24), (8, 1, 128, 24), (32, 2, 128, 17), (16, 2, 64, 40), (6, 1, 256, 30)])
@pytest.mark.parametrize("side,bad", [("v", "nan"), ("v", "inf"), ("k", "nan")])
def test_a_scale_that_is_no_number_of_new_tokens(at, side, bad, Hq, H, D, nodes, fmt):  # noqa: F811
    """Rows that see a token of the block show it, the others are those of a cache in which the block's scale is 0: within the bound
    above (value scales meet the probabilities over the largest one that was met, so the last bits go by the others of the tile too)."""
    lengths, base = [72 + nodes, 40], 72
    c, table = setup(at, fmt, 16, H, D, lengths, 3)
    clean(c)
    parents, starts = batch_of(np.random.default_rng(nodes), [nodes, nodes], "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
    mask = tree.mask.cpu().numpy()
    q = normal(5, (2 * nodes, Hq, D), "bf16")
    ws = c.workspace(2, 2 * nodes, Hq, tree=True)
    call = lambda: c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)  # noqa: E731
    out, lse = call()
    check_tree(c, q, table, lengths, starts, mask, D ** -0.5, out, lse, "bf16")
    scales, G, head = getattr(c, side + "_scale"), Hq // H, H - 1
    mine = slice(head * G, Hq)
    for block in range(base // 16 + 1, (lengths[0] - 1) // 16 + 1):
        first, past = max(block * 16 - base, 0), min(block * 16 + 16 - base, nodes)
        see = torch.zeros(2 * nodes, dtype=torch.bool, device="cuda")
        see[:nodes] = sees_of(mask, 0, nodes)[:, first:past].any(1)
        assert first > 0 and see.any() and not see.all()
        old = scales[table[0, block], head].item()
        scales[table[0, block], head] = float(bad)
        got, glse = call()
        assert torch.isnan(got[see][:, mine]).all()
        assert torch.equal(got[:, :head * G], out[:, :head * G]) and torch.equal(glse[:, :head * G], lse[:, :head * G])
        assert torch.isnan(glse[see][:, mine]).all() if side == "k" else torch.equal(glse, lse)
        scales[table[0, block], head] = 0.0
        got[see], glse[see] = out[see], lse[see]
        check_rows(c, q, table, lengths, starts, mask, D ** -0.5, got, glse, "bf16", (~see).cpu().numpy())
        scales[table[0, block], head] = old
