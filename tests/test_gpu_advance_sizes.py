"""Block tables of every batch size at which the launch changes, in processes of their own: whether a kernel was allowed more
shared memory is a process's state."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

CODE = """
import sys, numpy as np, torch
sys.path.insert(0, {root!r})
from paper_2608_15602_b200 import attention
from oracle import attention as oa
for B in {sizes}:
    rng = np.random.default_rng(B)
    table, free = np.full((B, 3), -1, np.int32), rng.permutation(2 * B).astype(np.int32)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    t = attention.BlockTables(i32(table), i32(free), 16)
    new = rng.integers(0, 40, B)
    T = int(new.sum())
    got = t.advance(i32(np.zeros(B)), i32(new), i32([2 * B]), T)
    want = oa.advance(np.zeros(B, int), new, table, free, 2 * B, 16, T)
    for name in ("lengths", "granted", "query_start", "positions", "slots", "requests"):
        assert np.array_equal(getattr(got, name).cpu().numpy(), want[name]), (B, name)
    assert int(got.num_free[0]) == want["num_free"] and np.array_equal(t.table.cpu().numpy(), table)
print("ok")
"""


@pytest.mark.parametrize("sizes", [[4064], [4065], [4096], [4097], [2048, 2049, 4095, 8192, 4080]])
def test_batch_sizes(sizes):
    from paper_2608_15602_b200 import build
    build.build()
    p = subprocess.run([sys.executable, "-c", CODE.format(root=ROOT, sizes=sizes)], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip() == "ok", p.stderr[-2000:]
