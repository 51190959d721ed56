"""Attention of drafted tokens under masks against its 64-bit definition.

Bounds as in the attention tests, with a probability times its value's scale entering its product as two bf16 numbers (2^-16 of it):
    |error| <= u |out| + (2^-15 + 2^-19 + (2 D + 8) 2^-24 S + L 2^-23) A,   A the mean of |v| under the probabilities"""
import numpy as np
import pytest

from oracle import drafts as od
from test_gpu_attention import U, at, dev, entries_of, f64, normal, setup  # noqa: F401
from test_gpu_drafts import batch_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def check_tree(c, q, table, lengths, starts, mask, scale, out, lse, dtype):
    k, v = (e * f64(s)[:, :, None, None] for e, s in zip(entries_of(c), (c.k_scale, c.v_scale)))
    want, wl, mean, size = od.attend(f64(q), np.nan_to_num(k), np.nan_to_num(v), table, lengths, starts, mask, scale)
    D, L = q.shape[2], max(max(lengths), 1)
    S = size[:, :, None]
    bound = U[dtype] * np.abs(want) + (2.0 ** -15 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * mean + 1e-7 * (dtype == "fp16")
    err = np.abs(f64(out) - want)
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-30)).max()
    if lse is not None:
        got = f64(lse)
        assert np.array_equal(np.isinf(got), np.isinf(wl))
        ok = np.isfinite(wl)
        assert (np.abs(got[ok] - wl[ok]) <= (D + 4) * 2.0 ** -24 * size[ok] + 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -23 * np.abs(wl[ok])).all()
    return want


def clean(c):
    """No NaN patterns anywhere (what a cache that was only appended to holds)."""
    if c.k.dtype is not torch.int8:
        for x in (c.k, c.v):
            raw = x.view(torch.uint8)
            raw.copy_(torch.where((raw & 127) == 127, torch.zeros_like(raw), raw))


SHAPES = [(4, 4, 128), (8, 1, 128), (16, 2, 64), (6, 2, 256), (14, 2, 64), (40, 1, 128), (3, 3, 64), (12, 1, 256), (64, 2, 128)]


@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "fp16"), ("int8", "fp16")])
@pytest.mark.parametrize("bs", [16, 48, 128])
@pytest.mark.parametrize("Hq,H,D", SHAPES)
def test_trees(at, Hq, H, D, bs, fmt, dtype):  # noqa: F811
    # one token, several, none, more new tokens than cached ones, prompts that end with a block, many words of masks
    new, lengths = [1, 5, 0, 33, 3, 70, 16], [40, 5, 77, 200, 2, 70, 144]
    rng = np.random.default_rng(Hq + bs)
    c, table = setup(at, fmt, bs, H, D, lengths, 3 * Hq)
    parents, starts = batch_of(rng, new, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), 70)
    q = normal(8, (sum(new), Hq, D), dtype)
    ws = c.workspace(len(lengths), sum(new), Hq, tree=True)
    out, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)
    check_tree(c, q, table, lengths, starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, dtype)
    again = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), tree=tree.mask)
    assert torch.equal(out, again)
    for nodes in (20, 33):                                # fewer words than tokens: what is past them is not seen
        short = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
        out = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), tree=short.mask)
        check_tree(c, q, table, lengths, starts, short.mask.cpu().numpy(), D ** -0.5, out, None, dtype)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,nodes", [(8, 1, 128, 16), (64, 2, 128, 9), (16, 2, 64, 37), (6, 2, 256, 40), (4, 4, 128, 7)])
def test_any_masks(at, Hq, H, D, nodes, fmt):  # noqa: F811
    """Masks that no tree makes, in any strides: rows that see nothing of the new tokens, not even themselves, or all of them; bits
    past a request's count; requests of nothing but new tokens, whose rows may be empty."""
    new, lengths = [nodes, nodes - 3, nodes], [nodes, 129, 61 + nodes]
    rng = np.random.default_rng(nodes)
    c, table = setup(at, fmt, 16, H, D, lengths, 7)
    clean(c)
    T, starts = sum(new), np.concatenate([[0], np.cumsum(new)])
    words = 3
    wide = dev(rng.integers(-2 ** 31, 2 ** 31, (T, words + 2)))
    mask = wide[:, 1:1 + words]
    mask[0] = 0
    mask[1] = -1
    mask[2, 0] = -2 ** 31
    mask[nodes] = 0
    q = normal(9, (T, Hq, D), "fp16")
    ws = c.workspace(3, T, Hq, tree=True)
    out, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=mask)
    check_tree(c, q, table, lengths, starts, mask.cpu().numpy(), D ** -0.5, out, lse, "fp16")
    assert (out[0] == 0).all() and torch.isinf(lse[0]).all() and torch.isfinite(lse[nodes]).all()
    same = mask[1:2].expand(T, words)                     # one mask for all
    out = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), tree=same)
    check_tree(c, q, table, lengths, starts, same.cpu().numpy(), D ** -0.5, out, None, "fp16")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,nodes,length", [(8, 1, 128, 16, 20001), (16, 2, 64, 40, 9999), (4, 4, 128, 5, 5003), (6, 2, 256, 24, 4097), (64, 1, 128, 9, 6000)])
def test_long_context_split_over_the_device(at, Hq, H, D, nodes, length, fmt):  # noqa: F811
    lengths, new = [length, nodes, length // 7], [nodes, nodes, 1]
    c, table = setup(at, fmt, 16, H, D, lengths, 5)
    rng = np.random.default_rng(length)
    parents, starts = batch_of(rng, new, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
    T = sum(new)
    q = normal(9, (T, Hq, D), "fp16")
    ws = c.workspace(3, T, Hq, tree=True)
    outs = [c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask) for _ in range(3)]
    for o in outs[1:]:
        assert torch.equal(o[0], outs[0][0]) and torch.equal(o[1], outs[0][1])
    # against 64 bits on the GPU
    mask = tree.mask.cpu().numpy()
    for r, L in enumerate(lengths):
        a, n = starts[r], new[r]
        ids = dev(table[r, :-(-L // 16)]).long()
        k, v = (x[ids].double() * s[ids].double()[..., None, None] for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        k, v = (x.transpose(0, 1).reshape(H, -1, D)[:, :L] for x in (k, v))
        qq = q[a:a + n].double().view(n, H, Hq // H, D)
        x = torch.einsum("nhgd,hld->nhgl", qq, k) * D ** -0.5
        sees = np.array([[(int(mask[a + i, j // 32]) >> (j % 32)) & 1 for j in range(n)] for i in range(n)], bool)
        x[..., L - n:] = x[..., L - n:].masked_fill(~torch.from_numpy(sees).cuda()[:, None, None, :], float("-inf"))
        p = torch.softmax(x, -1)
        want, mean = torch.einsum("nhgl,hld->nhgd", p, v), torch.einsum("nhgl,hld->nhgd", p, v.abs())
        S = torch.einsum("nhgd,hld->nhgl", qq.abs(), k.abs()).amax(-1)[..., None] * D ** -0.5
        bound = U["fp16"] * want.abs() + (2.0 ** -15 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * mean + 1e-7
        assert ((outs[0][0][a:a + n].double().view(n, H, Hq // H, D) - want).abs() <= bound).all()
        lse = torch.logsumexp(x, -1)
        assert ((outs[0][1][a:a + n].double().view(n, H, Hq // H) - lse).abs() <= (D + 4) * 2.0 ** -24 * S[..., 0] + 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -23 * lse.abs()).all()
    # a workspace serves calls without trees, and smaller ones, after larger ones
    out = c.attend(q[:1], dev(table[2:]), dev(lengths[2:]), ws)
    assert torch.isfinite(out).all()
    out, _ = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)
    assert torch.equal(out, outs[0][0])


@pytest.mark.parametrize("Hq,H,D,nodes", [(8, 1, 128, 16), (4, 4, 128, 5), (40, 1, 128, 9), (16, 2, 64, 40), (6, 1, 256, 30)])
def test_what_a_row_does_not_see_has_no_influence(at, Hq, H, D, nodes):  # noqa: F811
    """NaN entries and NaN scales past the length, in blocks that are none, and among new tokens: rows that do not see them equal
    those of a clean cache, rows that see one show it."""
    L, bs = 16 * 5 + nodes, 16
    rng = np.random.default_rng(nodes)
    c, table = setup(at, "e4m3", bs, H, D, [L], 3)
    clean(c)
    table = np.concatenate([table, [[c.num_blocks + 5, -1]]], 1)
    parents, starts = batch_of(rng, [nodes], "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev([L]), nodes)
    mask = tree.mask.cpu().numpy()
    q = normal(5, (nodes, Hq, D), "bf16")
    ws = c.workspace(1, nodes, Hq, tree=True)
    call = lambda table=table: c.attend(q, dev(table), dev([L]), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)  # noqa: E731
    out, lse = call()
    check_tree(c, q, table, [L], starts, mask, D ** -0.5, out, lse, "bf16")
    sees = np.array([[(int(mask[i, j // 32]) >> (j % 32)) & 1 for j in range(nodes)] for i in range(nodes)], bool)
    hit = 3                                               # a new token, element 5 of head 0
    p = L - nodes + hit
    raw = c.v.view(torch.uint8)
    old = raw[table[0, p // bs], 0, p % bs, 5].item()
    raw[table[0, p // bs], 0, p % bs, 5] = 0x7f
    if L % bs:
        raw[table[0, L // bs], :, L % bs:] = 0xff          # past the end
        c.k.view(torch.uint8)[table[0, L // bs], :, L % bs:] = 0x7f
    got, glse = call()
    see = torch.from_numpy(sees[:, hit]).cuda()
    G = Hq // H
    assert torch.equal(got[~see], out[~see]) and torch.equal(glse, lse) and torch.equal(got[:, G:], out[:, G:])
    assert torch.isnan(got[see][:, :G, 5]).all()
    keep = torch.arange(D, device="cuda") != 5
    assert torch.equal(got[..., keep], out[..., keep])
    raw[table[0, p // bs], 0, p % bs, 5] = old
    # a scale that is no number, of the last block: rows that see a token of it
    last = (L - 1) // bs
    first = max(0, last * bs - (L - nodes))
    if first > 0:
        c.v_scale[table[0, last], 0] = float("nan")
        got, _ = call()
        see = torch.from_numpy(sees[:, first:].any(1)).cuda()
        assert torch.equal(got[~see], out[~see]) and torch.isnan(got[see][:, :G]).all()
        c.v_scale[table[0, last], 0] = 0.01
    # blocks that are none: their tokens are masked out
    out, lse = call()
    holes = table.copy()
    holes[0, 1], holes[0, 3] = -1, c.num_blocks
    got, glse = call(holes)
    check_tree(c, q, holes, [L], starts, mask, D ** -0.5, got, glse, "bf16")


def test_strides_streams_and_tokens_of_no_request(at):  # noqa: F811
    Hq, H, D, new, lengths = 16, 2, 128, [9, 20], [60, 300]
    c, table = setup(at, "int8", 32, H, D, lengths, 13, major=True)
    T = 33
    rows = normal(14, (T, (Hq + 2 * H) * D), "bf16")
    q = rows[:, :Hq * D].unflatten(1, (Hq, D))
    starts = np.array([2, 11, 31])
    parents = np.full(T, -1, np.int32)
    p, _ = batch_of(np.random.default_rng(1), new, "tree")
    parents[2:31] = p
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), 20)
    wide = torch.full((T, Hq, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[..., :D]
    ws = c.workspace(2, T, Hq, tree=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), out=out, with_lse=True, tree=tree.mask, stream=side)
    side.synchronize()
    assert got is out and (wide[..., D:] == 7).all()
    check_tree(c, q, table, lengths, starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, "bf16")
    assert (out[:2] == 0).all() and (out[31:] == 0).all() and torch.isinf(lse[:2]).all() and torch.isinf(lse[31:]).all()


@pytest.mark.parametrize("Hq,H,D,nodes", [(8, 1, 128, 16), (16, 2, 64, 24), (4, 1, 256, 40), (4, 2, 128, 3)])
@pytest.mark.parametrize("order", [1, -1])
def test_scores_that_grow_and_scales_that_differ(at, Hq, H, D, nodes, order):  # noqa: F811
    L = 700
    c, table = setup(at, "int8", 16, H, D, [L], 11)
    n = -(-L // 16)
    ramp = sorted(torch.linspace(0.001, 0.08, n).tolist(), reverse=order < 0)
    for i in range(n):
        c.k_scale[table[0, i]] = float(ramp[i])
        c.v_scale[table[0, i]] = 2.0 ** float((i * 7 % 40) - 30)
    c.v_scale[table[0, n // 2]] = 0.0
    parents, starts = batch_of(np.random.default_rng(3), [nodes], "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev([L]), nodes)
    for spread in (0.1, 1.0):
        q = normal(12, (nodes, Hq, D), "fp16", spread)
        out, lse = c.attend(q, dev(table), dev([L]), c.workspace(1, nodes, Hq, tree=True), query_start=dev(starts), with_lse=True, tree=tree.mask)
        check_tree(c, q, table, [L], starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, "fp16")
    # values and scales at the ends of fp32's range
    for top in (1e30, 1e-30):
        c.v_scale[:] = top
        q = normal(13, (nodes, Hq, D), "bf16", 0.3)
        out, lse = c.attend(q, dev(table), dev([L]), c.workspace(1, nodes, Hq, tree=True), query_start=dev(starts), with_lse=True, tree=tree.mask)
        check_tree(c, q, table, [L], starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, "bf16")


def test_one_token_each_without_starts(at):  # noqa: F811
    lengths, Hq, H, D = [1, 0, 17, 300, -3], 16, 2, 128
    c, table = setup(at, "e4m3", 16, H, D, lengths, 2)
    q = normal(7, (5, Hq, D), "fp16")
    ws = c.workspace(5, 5, Hq, tree=True)
    ones = torch.ones(5, 1, dtype=torch.int32, device="cuda")
    out, lse = c.attend(q, dev(table), dev(lengths), ws, with_lse=True, tree=ones)
    check_tree(c, q, table, lengths, np.arange(6), ones.cpu().numpy(), D ** -0.5, out, lse, "fp16")
    assert (out[1] == 0).all() and torch.isinf(lse[4]).all()
    out, lse = c.attend(q, dev(table), dev(lengths), ws, with_lse=True, tree=ones * 2)                    # not even itself
    check_tree(c, q, table, lengths, np.arange(6), 2 * ones.cpu().numpy(), D ** -0.5, out, lse, "fp16")
    assert (out[0] == 0).all()
