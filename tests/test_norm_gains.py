"""Gains of normed heads that are changed after the norm was made: every call looks at them as they are then, on CPU tensors (the calls
are taken down in the place of being made)."""
import pytest

torch = pytest.importorskip("torch")
from test_attention_arguments import calls, ints  # noqa: E402,F401
from test_draft_arguments import at, draft_calls, half  # noqa: E402,F401


@pytest.mark.parametrize("change,error", [(lambda w: w.float(), TypeError), (lambda w: w.double(), ValueError), (lambda w: w[:32], ValueError), (lambda w: torch.zeros(128, dtype=w.dtype)[::2], ValueError)])
@pytest.mark.parametrize("which", ["q_weight", "k_weight"])
def test_changed_gains_are_refused(draft_calls, change, error, which):  # noqa: F811
    q, k = half(3, 4, 64), half(3, 2, 64)
    for assign in (lambda n, w: setattr(n, which, w), lambda n, w: setattr(getattr(n, which), "data", w)):
        n = at.NormedRotary(at.Rotary(64, device="cpu"), half(64), half(64))
        n.apply(q, k, ints(3))
        made = len(draft_calls)
        assign(n, change(half(64)))
        with pytest.raises(error, match="weight"):
            n.apply(q, k, ints(3))
        assert len(draft_calls) == made


def test_gains_changed_together_are_taken(draft_calls):  # noqa: F811
    n = at.NormedRotary(at.Rotary(64, device="cpu"), half(64), half(64))
    n.q_weight.data, n.k_weight.data = half(64).bfloat16(), half(64).bfloat16()
    n.apply(half(3, 4, 64), half(3, 2, 64), ints(3))
    assert draft_calls[-1][1][3] == at.fluxbin.TYPE_BF16
    n.k_weight = None                                          # one of two
    n.q_weight = half(64).float()
    n.apply(half(3, 4, 64), half(3, 2, 64), ints(3))
    assert draft_calls[-1][1][3] == at.fluxbin.TYPE_FP32 and draft_calls[-1][1][18] == 0


def test_changed_gains_are_refused_by_the_backward_pass(draft_calls):  # noqa: F811
    """(the tensors that were kept for it are the caller's own)"""
    n = at.NormedRotary(at.Rotary(64, device="cpu"), half(64).requires_grad_(), half(64).requires_grad_())
    q, k = n.apply(half(3, 4, 64), half(3, 2, 64), ints(3))
    made = len(draft_calls)
    n.k_weight.data = half(32)
    with pytest.raises(ValueError, match="weight"):
        torch.autograd.backward((q, k), (half(3, 4, 64), half(3, 2, 64)))
    assert len(draft_calls) == made
