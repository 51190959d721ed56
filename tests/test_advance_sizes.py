"""The outputs of block tables whose steps have two sizes in turn, on CPU tensors: made once, and never those that a step reads."""
import pytest

torch = pytest.importorskip("torch")
from test_attention_arguments import calls, ints  # noqa: E402,F401
from test_draft_arguments import at  # noqa: E402


@pytest.fixture
def tables(calls, monkeypatch):  # noqa: F811
    t = at.BlockTables(ints(3, 5), ints(9), 16)
    t.made, make = [], t._outputs
    monkeypatch.setattr(t, "_outputs", lambda tokens, stream: t.made.append(tokens) or make(tokens, stream))
    t.calls = calls
    return t


def test_a_loop_of_two_sizes_makes_its_outputs_once(tables):
    step = tables.advance(ints(3), ints(3), ints(1), 12)
    for _ in range(5):
        dropped = tables.advance(step.lengths, ints(3), step.num_free, 0)
        read = tables.calls[-1][1]
        assert read[3] == step.lengths.data_ptr() and dropped.lengths.data_ptr() != step.lengths.data_ptr()
        held, step = step, tables.advance(dropped.lengths, ints(3), dropped.num_free, 12)
        assert step.lengths.data_ptr() not in (dropped.lengths.data_ptr(), held.lengths.data_ptr()) and len(step.slots) == 12
    assert sorted(tables.made) == [0, 0, 12, 12]


def test_two_steps_one_after_the_other_have_sets_of_their_own(tables):
    a = tables.advance(ints(3), ints(3), ints(1), 4)
    b = tables.advance(a.lengths, ints(3), a.num_free, 4)
    c = tables.advance(b.lengths, ints(3), b.num_free, 4)
    assert a.slots.data_ptr() == c.slots.data_ptr() != b.slots.data_ptr()
    d = tables.advance(b.lengths, ints(3), b.num_free, 4)      # what it would write it reads: a new set
    assert d.lengths.data_ptr() != b.lengths.data_ptr() and len(tables.made) == 3
    e = tables.advance(d.lengths, ints(3), d.num_free, 4)
    assert e.lengths.data_ptr() == c.lengths.data_ptr()


def test_no_more_than_two_sizes_are_kept(tables):
    for n in (4, 0, 5, 0, 6, 0, 7, 0):
        step = tables.advance(ints(3), ints(3), ints(1), n)
        assert len(step.slots) == len(step.positions) == n and step.query_start.shape == (4,)
    assert tables.made == [4, 4, 0, 0, 5, 5, 6, 6, 7, 7]
