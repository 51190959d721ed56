"""Waits of the kernel for many rows that run out: a stage of the ring that is never full.  The call ends, the rows that it could not
answer are NaN, and the next call on the same workspace answers as ever."""
import numpy as np
import pytest

from test_gpu_attention import at, dev, normal, setup  # noqa: F401
from test_gpu_drafts import batch_of
from test_gpu_tree_attention import clean

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,nodes,length", [(64, 8, 128, 16, 9600), (24, 6, 64, 20, 12000), (16, 4, 256, 40, 9600)])
def test_a_wait_that_runs_out_ends_the_call(at, Hq, H, D, nodes, length, fmt):  # noqa: F811
    lengths = [length, 300, length // 2]
    c, table = setup(at, fmt, 32, H, D, lengths, 5)
    clean(c)
    parents, starts = batch_of(np.random.default_rng(1), [nodes] * 3, "tree")
    table, ln, starts = dev(table), dev(lengths), dev(starts)
    tree = at.DraftTree(dev(parents), starts, ln, nodes)
    q = normal(3, (3 * nodes, Hq, D), "bf16")
    ws = c.workspace(3, 3 * nodes, Hq, tree=True)
    call = lambda **kw: c.attend(q, table, ln, ws, query_start=starts, tree=tree.mask, with_lse=True, **kw)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    for stage in (3, 0, 2):
        at.fluxbin.debug_tree_waits(1_000_000, stage)           # a millisecond
        try:
            out, lse = call(out=torch.full_like(q, 7.0))
            torch.cuda.synchronize()
        finally:
            at.fluxbin.debug_tree_waits()
        bad = torch.isnan(lse)
        assert bad.any() and (stage > 0 or bad.all())           # (no CTA has done anything without the first stage)
        assert torch.equal(lse[~bad], want[1][~bad]) and torch.equal(out[~bad], want[0][~bad]) and torch.isnan(out[bad]).all()
        for _ in range(2):
            got = call(out=torch.full_like(q, 7.0))
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
