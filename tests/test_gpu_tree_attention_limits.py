"""Attention under masks and keeping at the ends of their ranges: caches whose entries lie past 32 bits, many requests, long trees, scales
below 0, workspaces and streams that calls share."""
import numpy as np
import pytest

from oracle import drafts as od
from test_gpu_attention import U, at, dev, f64, normal, setup  # noqa: F401
from test_gpu_drafts import batch_of, grow
from test_gpu_tree_attention import check_tree, clean

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,H,D,nodes", [(8, 2, 128, 3), (32, 2, 128, 20)])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.5])
def test_any_scale(at, Hq, H, D, nodes, scale):  # noqa: F811
    lengths = [75, nodes, 300]
    c, table = setup(at, "int8", 16, H, D, lengths, 3)
    parents, starts = batch_of(np.random.default_rng(1), [nodes] * 3, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
    q = normal(8, (3 * nodes, Hq, D), "bf16", 0.5)
    out, lse = c.attend(q, dev(table), dev(lengths), c.workspace(3, 3 * nodes, Hq, tree=True), query_start=dev(starts), scale=scale, with_lse=True, tree=tree.mask)
    check_tree(c, q, table, lengths, starts, tree.mask.cpu().numpy(), scale, out, lse, "bf16")


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("Hq,H,D,nodes", [(4, 4, 128, 2), (64, 4, 128, 9), (32, 4, 64, 12)])
def test_a_cache_past_32_bits(at, Hq, H, D, nodes, order):  # noqa: F811
    """Blocks that begin past 2^31 and 2^32 bytes; the others are never touched."""
    bs = 128
    nb = (1 << 32) // (bs * H * D) + 40
    k, v = (torch.empty(nb, H, bs, D, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(nb, H, device="cuda") for _ in range(2))
    big = at.KVCache.wrap(k, v, ks, vs)
    ids = np.array([[nb - 1, nb // 2 + 1, 3], [nb - 7, nb - 30, nb // 2 + 5]])[:, ::order]
    lengths = [2 * bs + 77, 3 * bs]
    small, table = setup(at, "int8", bs, H, D, lengths, 7)
    for r in range(2):
        for i in range(3):
            for x, y in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
                x[ids[r, i]] = y[table[r, i]]
    parents, starts = batch_of(np.random.default_rng(1), [nodes] * 2, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), nodes)
    q = normal(8, (2 * nodes, Hq, D), "fp16")
    ws = big.workspace(2, 2 * nodes, Hq, tree=True)
    a = big.attend(q, dev(ids.copy()), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)
    b = small.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True, tree=tree.mask)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_tree(small, q, table, lengths, starts, tree.mask.cpu().numpy(), D ** -0.5, *b, "fp16")
    slots = lambda t: np.concatenate([t[r, (n - nodes + np.arange(nodes)) // bs] * bs + (n - nodes + np.arange(nodes)) % bs for r, n in enumerate(lengths)])  # noqa: E731
    path = np.tile(np.r_[np.arange(0, nodes, 2), [-1] * (nodes // 2)], 2)
    assert slots(ids).max() * H * D > 2 ** (31 if order == 1 else 32)   # the new tokens are in the last blocks
    big.keep(dev(slots(ids)), dev(starts), dev(path))
    small.keep(dev(slots(table)), dev(starts), dev(path))
    for r in range(2):
        for i in range(3):
            for x, y in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
                assert torch.equal(x[ids[r, i]], y[table[r, i]])


@pytest.mark.parametrize("Hq,H,D,fmt", [(6, 2, 64, "int8"), (48, 2, 64, "e4m3"), (24, 1, 128, "int8")])
def test_many_requests(at, Hq, H, D, fmt):  # noqa: F811
    """More requests than a CTA has threads, some without new tokens, over blocks that they share."""
    B, rng = 900, np.random.default_rng(5)
    lengths = rng.integers(0, 60, B)
    new = np.minimum(rng.integers(0, 5, B), lengths)
    c, small = setup(at, fmt, 16, H, D, [64] * 8, 5)
    clean(c)
    table = small[rng.integers(0, 8, B)]
    parents, starts = batch_of(rng, list(new), "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), 4)
    q = normal(9, (int(new.sum()), Hq, D), "fp16")
    out, lse = c.attend(q, dev(table), dev(lengths), c.workspace(B, len(q), Hq, tree=True), query_start=dev(starts), with_lse=True, tree=tree.mask)
    check_tree(c, q, table, list(lengths), starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, "fp16")


def test_a_row_of_blocks_for_all_requests_and_long_trees(at):  # noqa: F811
    """Several trees behind one prompt whose block row is expanded; trees of several tiles of rows and many words."""
    Hq, H, D, n, L, B = 16, 1, 64, 130, 200, 3
    c, table = setup(at, "int8", 16, H, D, [L], 2)
    parents, starts = batch_of(np.random.default_rng(2), [n] * B, "tree")
    tree = at.DraftTree(dev(parents), dev(starts), dev([L] * B), n)
    q = normal(3, (n * B, Hq, D), "bf16")
    row = dev(table).expand(B, -1)
    out, lse = c.attend(q, row, dev([L] * B), c.workspace(B, n * B, Hq, tree=True), query_start=dev(starts), with_lse=True, tree=tree.mask)
    check_tree(c, q, np.repeat(table, B, 0), [L] * B, starts, tree.mask.cpu().numpy(), D ** -0.5, out, lse, "bf16")


def test_graphs_that_share_a_workspace_and_calls_at_once(at):  # noqa: F811
    """Two captured calls and eager ones of both kernels on one workspace, one after the other; two streams with one each."""
    H, D, lengths = 2, 128, [3000, 40, 777]
    c, table = setup(at, "int8", 16, H, D, lengths, 6)
    table, ln = dev(table), dev(lengths)
    calls = []
    for Hq, n in ((32, 6), (4, 3)):
        parents, starts = batch_of(np.random.default_rng(n), [n] * 3, "tree")
        starts = dev(starts)
        tree = at.DraftTree(dev(parents), starts, ln, n)
        q = normal(n, (3 * n, Hq, D), "fp16")
        calls.append(lambda ws, q=q, starts=starts, tree=tree, **kw: c.attend(q, table, ln, ws, query_start=starts, tree=tree.mask, with_lse=True, **kw))
    ws, other = c.workspace(3, 18, 32, tree=True), c.workspace(3, 18, 32, tree=True)
    want = [f(ws) for f in calls]
    chain = c.attend(normal(1, (3, 32, D), "fp16"), table, ln, ws)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(f(ws))
        graphs.append(g)
    for _ in range(3):
        for g, o, w in zip(graphs, outs, want):
            o[0].zero_()
            g.replay()
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
        for f, w in zip(calls, want):
            assert torch.equal(f(ws)[0], w[0])
        assert torch.equal(c.attend(normal(1, (3, 32, D), "fp16"), table, ln, ws), chain)
    torch.cuda.synchronize()
    for _ in range(5):                                     # at once, each stream with its own workspace
        a, b = calls[0](ws), calls[0](other, stream=side)
        d = calls[0](ws)
        side.synchronize()
        assert all(torch.equal(x[0], want[0][0]) for x in (a, b, d))


def test_chains_and_stars(at):  # noqa: F811
    """A chain sees what attend() without a mask sees; children of one token see it and themselves."""
    Hq, H, D, n, L = 16, 1, 128, 40, 333
    c, table = setup(at, "e4m3", 32, H, D, [L], 4)
    q = normal(4, (n, Hq, D), "bf16")
    ws = c.workspace(1, n, Hq, tree=True)
    plain, plain_lse = c.attend(q, dev(table), dev([L]), ws, query_start=dev([0, n]), with_lse=True)
    for kind in ("chain", "star"):
        tree = at.DraftTree(dev(grow(None, n, kind)), dev([0, n]), dev([L]), n)
        out, lse = c.attend(q, dev(table), dev([L]), ws, query_start=dev([0, n]), with_lse=True, tree=tree.mask)
        check_tree(c, q, table, [L], [0, n], tree.mask.cpu().numpy(), D ** -0.5, out, lse, "bf16")
        if kind == "chain":
            # both within the bound above of the same numbers: one step of bf16 and the sums' errors
            assert (np.abs(f64(out) - f64(plain)) <= 3 * U["bf16"] * np.abs(f64(plain)) + 2.0 ** -13 * np.abs(f64(plain)).max()).all()
            assert torch.allclose(lse, plain_lse, rtol=0, atol=1e-4)
        else:
            mask, _ = od.tree(grow(None, n, kind), [0, n], [L], n)
            assert (mask[5] == np.array([1 | 32, 0], np.int32)).all()


@pytest.mark.parametrize("Hq,H,D", [(32, 2, 128), (8, 2, 128), (64, 2, 64)])
def test_a_captured_call_follows_its_inputs(at, Hq, H, D):  # noqa: F811
    """One capture of tree and attention; lengths, starts, parents, blocks and queries change in place between replays."""
    B, T, nodes, rng = 4, 40, 12, np.random.default_rng(6)
    c, table = setup(at, "int8", 16, H, D, [900] * B, 6)
    t, ln, starts, parents, q = dev(table), dev([900] * B), dev([0, 10, 20, 30, 40]), dev(np.full(T, -1)), normal(1, (T, Hq, D), "fp16")
    ws = c.workspace(B, T, Hq, tree=True)

    def step():
        tree = at.DraftTree(parents, starts, ln, nodes)
        return tree, *c.attend(q, t, ln, ws, query_start=starts, with_lse=True, tree=tree.mask)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tree, out, lse = step()
    for lengths, new in (([900, 12, 7, 333], [10, 12, 7, 11]), ([0, 64, 1, 5], [0, 12, 1, 5]), ([9] * 4, [0, 0, 9, 0]), ([880, 891, 1, 900], [12, 12, 1, 12])):
        p, s = batch_of(rng, new, "tree")
        parents.fill_(-1)
        parents[:len(p)] = dev(p)
        starts.copy_(dev(s))
        ln.copy_(dev(lengths))
        t.copy_(dev(rng.permutation(table.reshape(-1)).reshape(table.shape)))
        q.copy_(normal(int(s[-1]), (T, Hq, D), "fp16"))
        out.fill_(7.0)
        graph.replay()
        check_tree(c, q[:s[-1]], t.cpu().numpy(), lengths, s, tree.mask.cpu().numpy(), D ** -0.5, out[:s[-1]], lse[:s[-1]], "fp16")
        assert (out[int(s[-1]):] == 0).all()               # rows of no request


def test_thousands_of_trees(at):  # noqa: F811
    B, rng = 5000, np.random.default_rng(8)
    new = rng.integers(0, 9, B)
    parents, starts = batch_of(rng, list(new), "tree")
    lengths = rng.integers(8, 100, B)
    drafted, answers = rng.integers(0, 2, (2, len(parents))).astype(np.int32)
    tree = at.DraftTree(dev(parents), dev(starts), dev(lengths), 8)
    kept = tree.accept(dev(drafted), dev(answers))
    mask, positions = od.tree(parents, starts, lengths, 8)
    assert np.array_equal(tree.mask.cpu().numpy(), mask) and np.array_equal(tree.positions.cpu().numpy(), positions)
    want = od.accept(parents, drafted, answers, starts, B, 8)
    for got, w in zip((kept.path, kept.count, kept.answer, kept.surplus), want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_a_request_without_blocks_keeps_what_it_has(at):  # noqa: F811
    """A step in which one request is refused: its cached tokens, its length and its blocks stay, the others go on."""
    B, n, nb = 3, 20, 8
    ints = lambda v: dev(np.asarray(v))  # noqa: E731
    cache, tables = at.KVCache(nb, 16, 2, 64), at.BlockTables.empty(B, 4, nb, 16)
    step = tables.advance(ints([0] * B), ints([30, 33, 16]), ints([nb]), 79)          # 2 + 3 + 1 blocks
    k, v = normal(1, (79, 2, 64), "fp16"), normal(2, (79, 2, 64), "fp16")
    cache.append(k, v, step.slots)
    old = [t.clone() for t in cache.read(step.slots)]
    slots = step.slots.clone()
    step = tables.advance(step.lengths, ints([n] * B), step.num_free, B * n)           # 2 + 1 + 2 wanted, 2 there
    granted = step.granted.cpu().numpy()
    assert granted.tolist().count(0) >= 1 and granted.tolist().count(1) >= 1
    parents = np.tile(np.r_[-1, np.arange(n - 1) // 2], B)
    tree = at.DraftTree(ints(parents), step.query_start, step.lengths, n)
    cache.append(normal(3, (B * n, 2, 64), "fp16"), normal(4, (B * n, 2, 64), "fp16"), step.slots)
    cache.attend(normal(5, (B * n, 8, 64), "fp16"), tables.table, step.lengths, cache.workspace(B, B * n, 8, tree=True), query_start=step.query_start, tree=tree.mask)
    kept = tree.accept(ints([0] * B * n), ints([0] * B * n))
    cache.keep(step.slots, step.query_start, kept.path)
    before = [30, 33, 16]
    after = tables.advance(step.lengths, kept.surplus * step.granted, step.num_free, 0)
    count = kept.count.cpu().numpy()
    assert after.lengths.tolist() == [b + c * g for b, c, g in zip(before, count, granted)]
    refused = torch.from_numpy(np.repeat(granted == 0, before)).cuda()
    for x, y in zip(old, cache.read(slots)):
        assert torch.equal(x[refused], y[refused])
