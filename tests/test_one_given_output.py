"""Heads that are turned (and normed) where one output is given and the other is new: the new one carries its gradient, on CPU tensors."""
import pytest

torch = pytest.importorskip("torch")
from test_attention_arguments import calls, ints  # noqa: E402,F401
from test_draft_arguments import at, draft_calls, half  # noqa: E402,F401


def norm(weights=False):
    w = [half(64).requires_grad_() for _ in range(2)] if weights else [None, None]
    return at.NormedRotary(at.Rotary(64, device="cpu"), *w)


@pytest.mark.parametrize("make,call", [(lambda: at.Rotary(64, device="cpu"), "rotary_call"), (norm, "norm_rotary_call")])
def test_the_new_output_carries_a_gradient(draft_calls, make, call):  # noqa: F811
    r, pos = make(), ints(3)
    for which in ("q", "k"):
        q, k = half(3, 4, 64).requires_grad_(), half(3, 2, 64).requires_grad_()
        given = torch.empty_like((q, k)[which == "k"], requires_grad=False)
        draft_calls.clear()
        outs = r.apply(q, k, pos, **{which + "_out": given})
        old, new = outs if which == "q" else outs[::-1]
        assert old is given and not given.requires_grad and new.requires_grad
        heads = lambda w: ((w[6], w[11]), (w[14], w[19])) if call == "norm_rotary_call" else ((w[5], w[9]), (w[12], w[16]))  # noqa: E731
        assert all(name == call for name, _ in draft_calls)
        # each input goes to its output, and no more than once
        pairs = [p for _, w in draft_calls for p in heads(w) if p[0]]
        assert sorted(pairs) == sorted([(q.data_ptr(), outs[0].data_ptr()), (k.data_ptr(), outs[1].data_ptr())])
        x = k if which == "q" else q
        (got,) = torch.autograd.grad(new, x, torch.ones_like(new))
        assert got.shape == x.shape
    # an output for keys that are not there
    q = half(3, 4, 64).requires_grad_()
    assert r.apply(q, None, pos, k_out=half(3, 2, 64))[0].requires_grad


def test_gains_of_the_side_that_is_new(draft_calls):  # noqa: F811
    n, pos = norm(True), ints(3)
    q, k = half(3, 4, 64), half(3, 2, 64)
    qo, ko = n.apply(q, k, pos, q_out=torch.empty_like(q))
    assert not qo.requires_grad and ko.requires_grad
    got = torch.autograd.grad(ko, (n.k_weight, n.q_weight), torch.ones_like(ko), allow_unused=True)
    assert got[0].shape == (64,) and got[1] is None
    name, w = [c for c in draft_calls if c[0] == "norm_rotary_call"][-1]
    assert w[6] == k.data_ptr() and w[10] == n.k_weight.data_ptr()         # its own gains


def test_both_given_and_none_wanted(draft_calls):  # noqa: F811
    for r in (at.Rotary(64, device="cpu"), norm()):
        q, k = half(3, 4, 64).requires_grad_(), half(3, 2, 64)
        a, b = torch.empty_like(q, requires_grad=False), torch.empty_like(k)
        draft_calls.clear()
        outs = r.apply(q, k, ints(3), q_out=a, k_out=b)
        assert outs[0] is a and outs[1] is b and not a.requires_grad and len(draft_calls) == 1
        outs = r.apply(q, k, ints(3), q_out=a)               # the new one's input wants none
        assert not outs[1].requires_grad and len(draft_calls) == 2
        with torch.no_grad():
            assert not r.apply(k, q, ints(3), q_out=b)[1].requires_grad and len(draft_calls) == 3
