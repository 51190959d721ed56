"""Trees of drafted tokens: masks and positions, the accepted path, keeping it, and a whole step, against the 64-bit definitions."""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od
from test_gpu_attention import CACHES, at, check_cache, dev, entries_of, f64, fill, normal  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def grow(rng, n, kind):
    """Parents of n tokens."""
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1) if n else []
    if kind == "wild":                                    # none, later ones, themselves, far away
        return [int(rng.choice([-1, i - 1, i, i + 1, rng.integers(-5, n + 5), 2 ** 31 - 1, -2 ** 31])) for i in range(n)]
    return [-1 if i == 0 or rng.random() < 0.05 else int(rng.integers(max(0, i - 6), i)) for i in range(n)]


def batch_of(rng, counts, kind):
    return np.array(sum((grow(rng, n, kind) for n in counts), []), np.int64).astype(np.int32), np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


TREES = [([1], 1), ([5], 8), ([0, 3, 1, 0, 9], 9), ([16] * 16, 16), ([63, 1, 40], 63), ([33, 32, 31, 64, 65], 65), ([300, 2, 1000], 1000), ([1024], 1024), ([20, 7], 5), ([70, 3], 33)]


@pytest.mark.parametrize("kind", ["tree", "chain", "star", "wild"])
@pytest.mark.parametrize("counts,nodes", TREES)
def test_masks_and_paths(at, counts, nodes, kind):  # noqa: F811
    rng = np.random.default_rng(sum(counts) + nodes)
    parents, start = batch_of(rng, counts, kind)
    lengths = np.array([n + int(rng.integers(0, 5000)) for n in counts])
    lengths[-1] = max(0, counts[-1] - 2)                  # fewer than there are new ones
    t = at.DraftTree(dev(parents), dev(start), dev(lengths), nodes)
    mask, pos = od.tree(parents, start, lengths, nodes)
    assert np.array_equal(t.mask.cpu().numpy(), mask) and np.array_equal(t.positions.cpu().numpy(), pos)
    drafted = rng.integers(0, 4, len(parents))            # few tokens, so that siblings are alike
    answers = rng.integers(0, 4, len(parents))
    for r, n in enumerate(counts):                        # long paths
        for i in range(1, n):
            p = parents[start[r] + i]
            if 0 <= p < i and rng.random() < 0.7:
                answers[start[r] + p] = drafted[start[r] + i]
    kept = t.accept(dev(drafted), dev(answers))
    want = od.accept(parents, drafted, answers, start, len(counts), nodes)
    for got, w in zip((kept.path, kept.count, kept.answer, kept.surplus), want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_tokens_of_no_request(at):  # noqa: F811
    """Ahead of the first request and behind the last; starts past the tokens."""
    for start, T in (([3, 5, 5, 9], 12), ([0, 4, 6, 40], 8), ([-2, 3, 3, 4], 6), ([2, 2, 2, 2], 3)):
        parents = np.tile([-1, 0, 1, 0], 3)[:T].astype(np.int32)
        t = at.DraftTree(dev(parents), dev(start), dev([50, 60, 70]), 8)
        mask, pos = od.tree(parents, start, [50, 60, 70], 8)
        assert np.array_equal(t.mask.cpu().numpy(), mask) and np.array_equal(t.positions.cpu().numpy(), pos)
        kept = t.accept(dev(np.zeros(T)), dev(np.zeros(T)))
        for got, w in zip((kept.path, kept.count, kept.answer, kept.surplus), od.accept(parents, np.zeros(T), np.zeros(T), start, 3, 8)):
            assert np.array_equal(got.cpu().numpy(), w)
    t = at.DraftTree(dev(np.zeros(0)), dev([0, 0]), dev([7]), 8)
    kept = t.accept(dev(np.zeros(0)), dev(np.zeros(0)))
    assert t.mask.shape == (0, 1) and kept.count.tolist() == [0] and kept.answer.tolist() == [-1] and kept.surplus.tolist() == [0]


@pytest.mark.parametrize("fmt,bs,H,D,major", CACHES)
@pytest.mark.parametrize("base", [0, 5, -2])
def test_keep(at, fmt, bs, H, D, major, base):  # noqa: F811
    """Paths that stay, that move within a block and into the next, that fill whole blocks."""
    rng = np.random.default_rng(bs + H)
    paths = [[0, 1, 2], [0, 2, 3, 7], [0, 1, 4, 5, 6, 9, 11], [1], [], [0, 3], list(range(1, 2 * bs + 3, 1))]
    counts = [3, 9, 14, 4, 2, 5, 2 * bs + 4]
    at_ = [base % bs, 3, bs - 3, bs - 1, 0, bs - 1, (base + 7) % bs]     # place of a request's first new token in its block
    width = 4
    nb = width * len(counts) + 1
    c = at.KVCache(nb, bs, H, D, fmt, token_major=major)
    fill(c, 3 + base)
    if base == 5:
        c.v_scale[::3] = 0.0
        c.k_scale[1::4] = float("nan")
    order = rng.permutation(nb)
    slots, path = [], []
    for r, n in enumerate(counts):
        slots += [int(order[r * width + (at_[r] + i) // bs]) * bs + (at_[r] + i) % bs for i in range(n)]
        path += paths[r] + [-1] * (n - len(paths[r]))
    start = np.concatenate([[0], np.cumsum(counts)])
    want = [oa.Cache(e, f64(s), fmt) for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
    before = [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)]
    for w in want:
        od.keep(w, start, slots, path)
    c.keep(dev(slots), dev(start), dev(path))
    check_cache(c, want, fmt, False)
    # nothing but the blocks of moved tokens was touched
    moved = {slots[start[r] + j] // bs for r, p in enumerate(paths) for j, i in enumerate(p) if i != j}
    rest = torch.tensor([b for b in range(nb) if b not in moved], device="cuda")
    for a, b in zip(before, (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)):
        assert torch.equal(a[rest].nan_to_num() if a.is_floating_point() else a[rest], b[rest].nan_to_num() if b.is_floating_point() else b[rest])


def test_keep_with_bad_slots_and_paths(at):  # noqa: F811
    """Slots outside the cache are not written, read as 0; a path that does not ascend ends there."""
    bs, H, D = 16, 2, 64
    for path, slots in (([0, 2, 4, -1, -1], [3, -1, 5, 6, 7]), ([0, 2, 4, -1, -1], [3, 4, -7, 6, 7]), ([0, 3, 2, 4, -1], [3, 4, 5, 6, 7]), ([0, 2, 9, 10, 11], [3, 4, 5, 6, 7]),
                        ([1, 2, 3, 4, 4], [14, 15, 16 * 4, 6, 7]), ([2, 1, 0, -1, -1], [3, 4, 5, 6, 7]), ([-1] * 5, [3, 4, 5, 6, 7]), ([1, 3, 4, -1, 2], [3, 9, 10, 11, 60])):
        c = at.KVCache(4, bs, H, D, "int8")
        fill(c, 9)
        want = [oa.Cache(e, f64(s), "int8") for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
        for w in want:
            od.keep(w, [0, 5], slots, path)
        c.keep(dev(slots), dev([0, 5]), dev(path))
        check_cache(c, want, "int8", False)


def test_what_is_kept_is_what_an_append_would_have_written(at):  # noqa: F811
    """Entries of one block's own scale move as they are: keeping a path equals appending its tokens alone, bit for bit in int8."""
    bs, H, D = 32, 2, 128
    x, y = normal(1, (8, H, D), "fp32"), normal(2, (8, H, D), "fp32")
    x[0], y[0] = 9.0, 9.0                                  # the first new token sets the block's scale
    path = [0, 2, 3, 6]
    a, b = (at.KVCache(2, bs, H, D) for _ in range(2))
    a.append(x, y, dev(np.arange(4, 12)))
    b.append(x[path], y[path], dev(np.arange(4, 8)))
    a.keep(dev(np.arange(4, 12)), dev([0, 8]), dev(path + [-1] * 4))
    assert torch.equal(a.k[0, :, :8], b.k[0, :, :8]) and torch.equal(a.v[0, :, :8], b.v[0, :, :8]) and torch.equal(a.k_scale, b.k_scale)


@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("fmt,hq,hk,dim", [("int8", 8, 2, 64), ("e4m3", 32, 1, 128)])
def test_a_step_with_trees_goes_where_single_steps_go(at, fmt, hq, hk, dim, normed):  # noqa: F811
    """A step of an attention block over drafted trees, replayed from a graph: each token's row is that of the step that appends its
    ancestors and itself alone (the same roundings up to the 8-bit scales of its blocks, so to 3 % of a row's norm), and after
    keeping and dropping the cache goes on as if only the accepted path had been there."""
    from paper_2608_15602_b200 import layer, synth
    hidden, B, bs, width = 256, 3, 16, 4
    L = [synth.make_linear(5, i, M, N, 2, 1, 128, synth.salient_random(5, i, N, 0.05)) for i, (M, N) in enumerate([(hq * dim, hidden), (hk * dim, hidden), (hk * dim, hidden), (hidden, hq * dim)])]
    lins = [layer.FluxBinLinear(x) for x in L]
    rope = at.Rotary(dim)
    if normed:
        g = torch.Generator().manual_seed(1)
        rope = at.NormedRotary(rope, *(torch.rand(dim, generator=g).add(0.5).half().cuda() for _ in range(2)))

    def fresh():
        block = at.AttentionBlock(*lins, at.KVCache(B * width, bs, hk, dim, fmt), rope)
        return block, at.BlockTables.empty(B, width, B * width, bs)

    def feed(block, tables, x, lengths, new, free):
        buf = block.buffers(B, len(x))
        buf.x.copy_(x)
        step = tables.advance(dev(lengths), dev(new), dev([free]), len(x))
        return block.forward(buf, tables, step).clone(), step

    prompts, counts = [13, 7, 21], [6, 1, 9]
    parents = [-1, 0, 0, 1, 3, 2] + [-1] + [-1, 0, 1, 1, 2, 0, 4, 6, 7]
    start = np.concatenate([[0], np.cumsum(counts)])
    xp, xd = normal(7, (sum(prompts), hidden), "fp16"), normal(8, (sum(counts), hidden), "fp16")
    block, tables = fresh()
    _, step = feed(block, tables, xp, [0] * B, prompts, B * width)
    buf = block.buffers(B, sum(counts), tree=True)
    buf.x.copy_(xd)
    lengths, free = step.lengths.clone(), step.num_free.clone()
    new, par = dev(counts), dev(parents)
    state = [t.clone() for t in (block.cache.k.view(torch.uint8), block.cache.v.view(torch.uint8), block.cache.k_scale, block.cache.v_scale, tables.table, tables.free)]

    drafted = dev(np.arange(sum(counts)))
    answers = torch.full((sum(counts),), -5, dtype=torch.int32, device="cuda")
    for r, path in enumerate([[0, 2, 5], [0], [0, 1, 4, 7, 8][:4]]):
        for a, b in zip(path, path[1:]):
            if parents[start[r] + b] == a:
                answers[start[r] + a] = int(start[r] + b)

    def one():
        s = tables.advance(lengths, new, free, sum(counts))
        t = at.DraftTree(par, s.query_start, s.lengths, 16)
        y = block.forward(buf, tables, s, tree=t)
        kept = t.accept(drafted, answers)
        block.cache.keep(s.slots, s.query_start, kept.path)
        after = tables.advance(s.lengths, kept.surplus, s.num_free, 0)
        return y, kept, after

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, kept, after = one()
    for dst, src in zip((block.cache.k.view(torch.uint8), block.cache.v.view(torch.uint8), block.cache.k_scale, block.cache.v_scale, tables.table, tables.free), state):
        dst.copy_(src)
    graph.replay()
    torch.cuda.synchronize()
    want_path = od.accept(parents, np.arange(sum(counts)), answers.cpu().numpy(), start, B, 16)
    assert np.array_equal(kept.path.cpu().numpy(), want_path[0]) and kept.count.tolist() == want_path[1].tolist()
    assert after.lengths.tolist() == [p + int(c) for p, c in zip(prompts, want_path[1])]

    # every drafted token on its own: its ancestors and itself, one after the other
    rows = y.double().cpu().numpy()
    for r, n in enumerate(counts):
        for i in range(n):
            line, j = [], i
            while j >= 0:
                line.insert(0, j)
                j = parents[start[r] + j]
            b2, t2 = fresh()
            _, s2 = feed(b2, t2, xp, [0] * B, prompts, B * width)
            got, _ = feed(b2, t2, xd[[start[r] + j for j in line]], s2.lengths.tolist(), [len(line) if q == r else 0 for q in range(B)], int(s2.num_free))
            a, b = rows[start[r] + i], got[-1].double().cpu().numpy()
            assert np.linalg.norm(a - b) <= 0.03 * np.linalg.norm(b), (r, i)
    # and the next step from what was kept, next to one that never saw the others
    b2, t2 = fresh()
    _, s2 = feed(b2, t2, xp, [0] * B, prompts, B * width)
    order = [start[r] + p for r in range(B) for p in want_path[0][start[r]:start[r + 1]] if p >= 0]
    _, s2 = feed(b2, t2, xd[order], s2.lengths.tolist(), want_path[1].tolist(), int(s2.num_free))
    xn = normal(9, (B, hidden), "fp16")
    want, _ = feed(b2, t2, xn, s2.lengths.tolist(), [1] * B, int(s2.num_free))
    got, _ = feed(block, tables, xn, after.lengths.tolist(), [1] * B, int(after.num_free))
    for a, b in zip(got.double(), want.double()):
        assert (a - b).norm() <= 0.03 * b.norm()
