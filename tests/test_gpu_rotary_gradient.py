"""The gradient of rotary positions through autograd: against the formula in 64 bits, against differences, and what it may come with.

The turn is linear, so a difference over any step is its derivative up to the rounding of its two ends: with values of size 1,
fp32 and a step of 1, (|f(x + e)| + |f(x - e)|) 2^-23 < 2^-19."""
import numpy as np
import pytest

from oracle import attention as oa
from test_gpu_attention import KW, U, at, check_turn, dev, f64, normal, rope  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype,kind", [(5, 3, 1, 64, 64, False, "fp32", "none"), (7, 4, 2, 128, 64, True, "bf16", "ramp"), (3, 2, 0, 80, 20, True, "fp16", "linear"),
                                                        (300, 4, 2, 64, 64, False, "fp16", "none")])
@pytest.mark.parametrize("inverse", [False, True])
def test_gradient_is_the_turn_back(at, T, hq, hk, D, d, inter, dtype, kind, inverse):  # noqa: F811
    r = rope(at, D, d, inter, kind)
    pos = np.random.default_rng(T).integers(0, 5000, T)
    q, k = normal(1, (T, hq, D), dtype).requires_grad_(), normal(2, (T, hk, D), dtype).requires_grad_() if hk else None
    qo, ko = r.apply(q, k, dev(pos), inverse=inverse)
    plain = r.apply(q.detach(), None if k is None else k.detach(), dev(pos), inverse=inverse)
    assert torch.equal(qo, plain[0]) and (k is None or torch.equal(ko, plain[1])) and not plain[0].requires_grad
    gq, gk = normal(3, (T, hq, D), dtype), normal(4, (T, hk, D), dtype) if hk else None
    torch.autograd.backward([qo] + ([ko] if hk else []), [gq] + ([gk] if hk else []))
    check_turn(q.grad, gq, pos, r, dtype, not inverse)
    if hk:
        check_turn(k.grad, gk, pos, r, dtype, not inverse)


@pytest.mark.parametrize("inter", [False, True])
def test_gradient_against_differences(at, inter):  # noqa: F811
    r = rope(at, 64, 32, inter, "ramp")
    x, w, pos = normal(1, (2, 1, 64), "fp32").requires_grad_(), normal(2, (2, 1, 64), "fp32"), dev([3, 700])
    (r.apply(x, None, pos)[0] * w).sum().backward()
    with torch.no_grad():
        for e in (0, 5, 16, 31, 40, 63):
            step = torch.zeros_like(x)
            step[:, :, e] = 1.0
            change = (r.apply(x + step, None, pos)[0] - r.apply(x - step, None, pos)[0]) / 2
            want = (f64(change) * f64(w)).sum(-1)
            # five elements at most differ; those that do carry the bound above, the sum of the gradient its own roundings
            assert (np.abs(f64(x.grad)[..., e] - want) <= 2.0 ** -17 * np.abs(f64(w)).max()).all()


def test_gradients_that_come_expanded_alone_or_not_at_all(at):  # noqa: F811
    r, pos = rope(at, 64, 64, False, "none"), dev([1, 2, 3])
    q, k = (normal(i, (3, 2, 64), "fp32").requires_grad_() for i in (1, 2))
    ones = torch.ones(3, 2, 64, device="cuda")
    r.apply(q, k, pos)[0].sum().backward()                # expanded, and none for k
    check_turn(q.grad, ones, [1, 2, 3], r, "fp32", True)
    assert k.grad is None or (k.grad == 0).all()
    q.grad = None
    frozen = q.detach()
    r.apply(frozen, k, pos)[1].sum().backward()           # k alone
    check_turn(k.grad if k.grad is not None else ones, ones, [1, 2, 3], r, "fp32", True)
    assert frozen.grad is None
    shared = normal(5, (3, 1, 64), "fp32").requires_grad_()
    r.apply(shared.expand(3, 4, 64), None, pos)[0].sum().backward()                # one head seen as four: their gradients add up
    check_turn(shared.grad / 4, ones[:, :1], [1, 2, 3], r, "fp32", True)
    again = torch.autograd.grad(r.apply(q, None, pos)[0].square().sum(), q, create_graph=True)[0]
    again.sum().backward()                                # q -> |turn q|^2 -> its gradient 2 q: the second derivative is 2
    assert (q.grad - 2).abs().max() < 2.0 ** -18


def test_without_gradient_nothing_changes(at):  # noqa: F811
    r, pos = rope(at, 64, 64, False, "none"), dev([1, 2])
    q = normal(1, (2, 2, 64), "fp16").requires_grad_()
    with torch.no_grad():
        assert not r.apply(q, None, pos)[0].requires_grad
    out = torch.empty_like(q)
    got = r.apply(q, None, pos, q_out=out)[0]
    assert got is out and not out.requires_grad and torch.equal(out, r.apply(q, None, pos)[0])
