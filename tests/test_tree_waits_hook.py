"""What the test hook for tree attention's waits takes (no GPU)."""
import pytest

from paper_2608_15602_b200 import build, fluxbin

build.build()


def test_what_it_takes_and_refuses():
    for limit, withheld in ((0, -1), (1, 0), (2_000_000_000, 3)):
        fluxbin.debug_tree_waits(limit, withheld)
    for limit, withheld in ((-1, -1), (2_000_000_001, -1), (0, -2)):
        with pytest.raises(fluxbin.FluxBinError) as e:
            fluxbin.debug_tree_waits(limit, withheld)
        assert e.value.status == 3
    fluxbin.debug_tree_waits()
