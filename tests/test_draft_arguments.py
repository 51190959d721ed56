"""What the torch wrapper hands to the calls for trees of drafted tokens, on CPU tensors, and what it refuses itself."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_15602_b200 import build, fluxbin  # noqa: E402

build.build()
from paper_2608_15602_b200 import attention as at  # noqa: E402
from test_attention_arguments import FakeStream, Scratch, calls, ints, memory  # noqa: E402,F401

CALLS = ("norm_rotary_call", "norm_rotary_backward_call", "draft_tree_call", "draft_accept_call", "kv_attend_tree_call", "kv_keep_call")


@pytest.fixture
def draft_calls(calls, monkeypatch):  # noqa: F811
    for name in CALLS:
        monkeypatch.setattr(fluxbin, name, lambda *words, name=name: calls.append((name, words)))
    return calls


def half(*shape):
    return torch.zeros(shape, dtype=torch.float16)


def test_masks_are_read_where_they_lie(draft_calls):
    c, q = at.KVCache(8, 16, 2, 64, device="cpu"), half(6, 4, 64)
    wide = ints(6, 5)
    for tree in (ints(6, 1), ints(6, 2), wide[:, 1:3], ints(1, 2).expand(6, 2), ints(6)[:, None]):
        c.attend(q, ints(2, 3), ints(2), Scratch, query_start=ints(3), tree=tree)
        name, words = draft_calls[-1]
        assert name == "kv_attend_tree_call" and words[10:13] == (tree.data_ptr(), tree.stride(0), tree.shape[1])
    c.attend(q, ints(2, 3), ints(2), Scratch, query_start=ints(3))
    assert draft_calls[-1][0] == "kv_attend_call"
    for tree in (ints(5, 1), ints(6), ints(6, 1).long(), ints(2, 6).T, ints(6, 4)[:, ::2]):
        with pytest.raises(ValueError, match="tree"):
            c.attend(q, ints(2, 3), ints(2), Scratch, query_start=ints(3), tree=tree)


def test_a_tree_checks_its_arguments(draft_calls):
    t = at.DraftTree(ints(7), ints(4), ints(3), 40)
    assert t.mask.shape == (7, 2) and t.positions.shape == (7,) and draft_calls[-1][1][:3] == (3, 7, 40)
    kept = t.accept(ints(7), ints(7))
    assert kept.path.shape == (7,) and kept.count.shape == kept.answer.shape == kept.surplus.shape == (3,)
    for bad in (lambda: at.DraftTree(ints(7), ints(3), ints(3), 4), lambda: at.DraftTree(ints(7), ints(4), ints(3), 0), lambda: at.DraftTree(ints(7), ints(4), ints(3), 1025),
                lambda: at.DraftTree(ints(7).long(), ints(4), ints(3), 4), lambda: t.accept(ints(6), ints(7)), lambda: t.accept(ints(7), ints(7).float()),
                lambda: at.KVCache(8, 16, 2, 64, device="cpu").keep(ints(7), ints(4), ints(6))):
        with pytest.raises(ValueError):
            bad()
    at.KVCache(8, 16, 2, 64, device="cpu").keep(ints(7), ints(4), ints(7))
    assert draft_calls[-1][1][1:3] == (3, 7)


def test_norms_check_their_arguments(draft_calls):
    r = at.Rotary(64, device="cpu")
    for kw in (dict(eps=0.0), dict(eps=float("nan")), dict(q_weight=half(63)), dict(q_weight=half(128)[::2]), dict(k_weight=half(64).double())):
        with pytest.raises(ValueError):
            at.NormedRotary(r, **kw)
    with pytest.raises(TypeError):
        at.NormedRotary(r, half(64), half(64).float())
    n = at.NormedRotary(r, half(64).float())
    q, k = half(3, 4, 64), half(3, 2, 64)
    qo, ko = n.apply(q, k, ints(3))
    words = draft_calls[-1][1]
    assert words[3] == fluxbin.TYPE_FP32 and words[10] == n.q_weight.data_ptr() and words[18] == 0 and qo.shape == q.shape and ko.shape == k.shape
    assert n.apply(q, None, ints(3))[1] is None
    for bad in (lambda: n.apply(q.double(), None, ints(3)), lambda: n.apply(q, k.float(), ints(3))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: n.apply(q, half(2, 2, 64), ints(3)), lambda: n.apply(q, k, ints(2)), lambda: n.apply(half(3, 4, 32), None, ints(3)),
                lambda: n.apply(half(3, 4, 128)[..., ::2], None, ints(3)), lambda: n.apply(q, None, ints(3), q_out=half(3, 3, 64))):
        with pytest.raises(ValueError):
            bad()


def test_what_the_calls_on_another_stream_allocate_is_that_streams(draft_calls, memory):  # noqa: F811
    made, recorded = memory
    s = FakeStream()
    c, n = at.KVCache(8, 16, 2, 64, device="cpu"), at.NormedRotary(at.Rotary(64, device="cpu"))
    q, k = half(3, 4, 64), half(3, 2, 64)
    t = at.DraftTree(ints(3), ints(3), ints(2), 4)
    for what in (lambda: n.apply(q, k, ints(3), stream=s), lambda: c.attend(q, ints(2, 4), ints(2), Scratch, query_start=ints(3), tree=t.mask, with_lse=True, stream=s),
                 lambda: [at.DraftTree(ints(3), ints(3), ints(2), 4, stream=s).mask], lambda: [t.accept(ints(3), ints(3), stream=s).path]):
        made.clear()
        recorded.clear()
        results = what()
        storages = {y.untyped_storage().data_ptr(): stream for stream, y in made}
        for y in results:
            assert storages[y.untyped_storage().data_ptr()] is s
            assert (y.untyped_storage().data_ptr(), "the current one") in recorded
