"""One workspace for caches of different head dimensions, with and without masks, few rows and many: what one call leaves there is not
what another one looks for."""
import numpy as np
import pytest

from test_gpu_attention import at, dev, normal, setup  # noqa: F401
from test_gpu_drafts import batch_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def calls_of(at, fmt):  # noqa: F811
    """(name, call(ws, out)) of long requests, whose jobs are cut over all CTAs."""
    found = []
    for D in (256, 128, 64):
        lengths = [9001, 5003]
        c, table = setup(at, fmt, 16, 1, D, lengths, D)
        table, ln = dev(table), dev(lengths)
        for Hq, n in ((4, 1), (8, 2), (8, 5), (8, 20)):        # 4, 16, 40 and 160 rows a key head
            parents, starts = batch_of(np.random.default_rng(n), [n, n], "tree")
            starts = dev(starts)
            mask = at.DraftTree(dev(parents), starts, ln, n).mask
            q = normal(n + D, (2 * n, Hq, D), "fp16")
            for tree in (None, mask):
                found.append((c, (D, Hq * n, tree is not None), lambda ws, out=None, c=c, q=q, table=table, ln=ln, starts=starts, tree=tree: c.attend(
                    q, table, ln, ws, query_start=starts, tree=tree, with_lse=True, out=out)))
    return found


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_every_call_after_every_other(at, fmt):  # noqa: F811
    calls = calls_of(at, fmt)
    want = [f(c.workspace(2, 40, 8, tree=True)) for c, _, f in calls]
    shared = calls[0][0].workspace(2, 40, 8, tree=True)        # of the largest head dimension
    for _, first, f in calls:
        for (_, name, g), (out, lse) in zip(calls, want):
            f(shared)
            nothing = torch.full_like(out, float("nan"))
            got = g(shared, nothing)
            assert torch.equal(nothing, out) and torch.equal(got[1], lse), (first, name)


def test_a_plain_call_on_a_plain_workspace_after_larger_ones(at):  # noqa: F811
    """A workspace without room for trees serves the smaller head dimensions too."""
    calls = [x for x in calls_of(at, "int8") if not x[1][2]]
    want = [f(c.workspace(2, 40, 8)) for c, _, f in calls]
    shared = calls[0][0].workspace(2, 40, 8)
    for _, first, f in calls:
        for (_, name, g), (out, lse) in zip(calls, want):
            f(shared)
            nothing = torch.full_like(out, float("nan"))
            got = g(shared, nothing)
            assert torch.equal(nothing, out) and torch.equal(got[1], lse), (first, name)
