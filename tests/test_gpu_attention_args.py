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
