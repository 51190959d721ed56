"""Norms of query and key heads with their turn, and its gradients, against the 64-bit definitions and against differences.

Bounds.  u is the unit roundoff of the result's type, e24 = 2^-24.
  norms      a sum of D squares of one sign is off by at most D e24 of itself, its root by half of that; with the division, eps,
             root and two products: r w x is off by (D / 2 + 8) e24 of itself, the turn adds 2^-20 of |a| + |b| (the rotary tests')
  gradient   e (what is turned back) is off by E = 2^-20 (|ga| + |gb|).  With n = x r and m = mean(w e n):
             m is off by mean(|w n| E) + (D + 8) e24 mean|w e n|, so r (w e - n m) by u |dx| + r (|w| E + |n| (that) + (D + 16) e24 (|w e| + |n m|));
             a gain's gradient, a sum of N terms e n, by u |dw| + sum(|n| E) + (N + D / 2 + 16) e24 sum|e n|
"""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od
from test_gpu_attention import DT, KW, U, at, dev, f64, normal, rope  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
EPS = 1e-5
E24 = 2.0 ** -24


def gains(seed, D, dtype):
    return None if dtype is None else (normal(seed, (D,), "fp32", 0.4) + 1.0).to(DT[dtype])


def frequencies(r):
    return oa.frequencies(r.rotary_dim, scaling=r.kind, **KW[r.kind])


def check_normed(got, x, w, pos, r, dtype, eps=EPS):
    f, m = frequencies(r)
    w64 = None if w is None else f64(w)
    want = od.norm_rotary(f64(x), w64, eps, pos, f, m, r.rotary_dim, r.interleaved)
    size = od.pair_size(od.norm(f64(x), eps)[0] * (1.0 if w is None else w64), r.rotary_dim, r.interleaved) * max(m, 1.0)
    bound = U[dtype] * np.abs(want) + (2.0 ** -20 + (x.shape[2] / 2 + 8) * E24) * size + 1e-7 * (dtype == "fp16")
    err = np.abs(f64(got) - want)
    assert (err <= bound).all(), (err / bound).max()


def check_gradients(dx, dw, x, w, g, pos, r, dtype, w_dtype, eps=EPS):
    f, m = frequencies(r)
    D, N = x.shape[2], x.shape[0] * x.shape[1]
    w64 = np.ones(D) if w is None else f64(w)
    want, want_w, e = od.norm_rotary_backward(f64(x), w64, eps, f64(g), pos, f, m, r.rotary_dim, r.interleaved)
    n, size = od.norm(f64(x), eps)
    E = 2.0 ** -20 * od.pair_size(f64(g), r.rotary_dim, r.interleaved) * max(m, 1.0)
    mean = np.abs((w64 * e * n).mean(-1, keepdims=True))
    off = (np.abs(w64 * n) * E).mean(-1, keepdims=True) + (D + 8) * E24 * np.abs(w64 * e * n).mean(-1, keepdims=True)
    if dx is not None:
        bound = U[dtype] * np.abs(want) + (np.abs(w64) * E + np.abs(n) * off + (D + 16) * E24 * (np.abs(w64 * e) + np.abs(n) * mean)) / size + 1e-7 * (dtype == "fp16")
        err = np.abs(f64(dx) - want)
        assert (err <= bound).all(), (err / bound).max()
    if dw is not None:
        bound = U[w_dtype] * np.abs(want_w) + (np.abs(n) * E).sum((0, 1)) + (N + D / 2 + 16) * E24 * np.abs(e * n).sum((0, 1)) + 1e-7 * (w_dtype == "fp16")
        err = np.abs(f64(dw) - want_w)
        assert (err <= bound).all(), (err / bound).max()


CASES = [  # tokens, q heads, k heads, head dim, rotary dim, interleaved, dtype, gains' type, scaling
    (1, 1, 1, 64, 64, False, "fp16", "fp16", "none"), (3, 5, 0, 128, 128, True, "bf16", None, "none"), (7, 4, 2, 128, 64, False, "fp32", "fp32", "linear"),
    (5, 3, 1, 80, 20, True, "fp16", "fp32", "base"), (2, 2, 2, 96, 34, False, "bf16", "bf16", "ramp"), (33, 8, 2, 256, 256, False, "fp16", "fp32", "bands"),
    (4, 1, 1, 6, 2, True, "fp32", "fp16", "none"), (9, 12, 12, 64, 32, True, "fp16", "fp16", "ramp"), (130, 72, 8, 128, 128, False, "bf16", "bf16", "none"),
    (3, 3, 3, 512, 512, False, "fp32", "fp32", "none"), (2, 33, 1, 512, 256, True, "bf16", "fp32", "none"), (5, 40, 2, 96, 96, True, "bf16", "bf16", "none"),
    (6, 1, 9, 16, 16, False, "fp16", "fp32", "none"), (4, 2, 2, 272, 48, False, "fp32", None, "none"), (3, 2, 1, 511, 64, False, "fp32", "fp32", "none")]


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype,wt,kind", CASES)
def test_normed_heads(at, T, hq, hk, D, d, inter, dtype, wt, kind):  # noqa: F811
    r = rope(at, D, d, inter, kind)
    wq, wk = gains(1, D, wt), gains(2, D, wt)
    pos = np.random.default_rng(T).integers(0, 131072, T)
    pos[0] = 0
    if T > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -5
    q, k = normal(1, (T, hq, D), dtype, 3.0), normal(2, (T, hk, D), dtype, 0.01) if hk else None
    q[0, 0] = 0                                           # a head of zeros stays one
    n = at.NormedRotary(r, wq, wk, eps=EPS)
    qo, ko = n.apply(q, k, dev(pos))
    check_normed(qo, q, wq, pos, r, dtype)
    assert (qo[0, 0] == 0).all()
    if hk:
        check_normed(ko, k, wk, pos, r, dtype)
    mixed = at.NormedRotary(r, None, wk, eps=0.5).apply(q, k, dev(pos))
    check_normed(mixed[0], q, None, pos, r, dtype, 0.5)
    # in place
    qc, kc = q.clone(), None if k is None else k.clone()
    assert n.apply(qc, kc, dev(pos), q_out=qc, k_out=kc)[0] is qc and torch.equal(qc, qo) and (k is None or torch.equal(kc, ko))


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype,wt,kind", CASES)
def test_gradients(at, T, hq, hk, D, d, inter, dtype, wt, kind):  # noqa: F811
    r = rope(at, D, d, inter, kind)
    wq, wk = gains(1, D, wt), gains(2, D, wt)
    pos = np.random.default_rng(T).integers(0, 131072, T)
    q, k = normal(1, (T, hq, D), dtype, 3.0), normal(2, (T, hk, D), dtype, 0.3) if hk else None
    gq, gk = normal(3, (T, hq, D), dtype), normal(4, (T, hk, D), dtype, 20.0) if hk else None
    leaves = [x for x in (q, k, wq, wk if hk else None) if x is not None]
    for x in leaves:
        x.requires_grad_()
    n = at.NormedRotary(r, wq, wk, eps=EPS)
    outs = [y for y in n.apply(q, k, dev(pos)) if y is not None]
    plain = at.NormedRotary(r, None if wq is None else wq.detach(), None if wk is None else wk.detach(), eps=EPS).apply(q.detach(), None if k is None else k.detach(), dev(pos))
    assert all(torch.equal(a, b) and not b.requires_grad for a, b in zip(outs, plain))
    got = dict(zip(map(id, leaves), torch.autograd.grad(outs, leaves, [g for g in (gq, gk) if g is not None], retain_graph=True)))
    check_gradients(got[id(q)], got.get(id(wq)), q, wq, gq, pos, r, dtype, wt)
    if hk:
        check_gradients(got[id(k)], got.get(id(wk)), k, wk, gk, pos, r, dtype, wt)
    again = torch.autograd.grad(outs, leaves, [g for g in (gq, gk) if g is not None])
    assert all(torch.equal(got[id(x)], y) for x, y in zip(leaves, again))               # the same sums each time


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype", [(700, 3, 0, 128, 64, True, "bf16"), (333, 40, 2, 64, 32, False, "fp32"), (601, 1, 1, 256, 256, True, "fp16"),
                                                      (1500, 33, 1, 128, 128, False, "fp16"), (650, 2, 2, 80, 40, False, "bf16"), (97, 70, 65, 64, 64, False, "bf16")])
def test_prompts(at, T, hq, hk, D, d, inter, dtype):  # noqa: F811
    """More tokens than there are CTAs at once, heads that fill no round."""
    r = rope(at, D, d, inter, "none")
    pos = np.random.default_rng(T).integers(0, 131072, T)
    q, k = normal(1, (T, hq, D), dtype).requires_grad_(), normal(2, (T, hk, D), dtype).requires_grad_() if hk else None
    wq, wk = gains(1, D, "fp32").requires_grad_(), gains(2, D, "fp32").requires_grad_()
    n = at.NormedRotary(r, wq, wk, eps=EPS)
    qo, ko = n.apply(q, k, dev(pos))
    gq = normal(3, (T, hq, D), dtype)
    check_normed(qo, q, wq, pos, r, dtype)
    if hk:
        check_normed(ko, k, wk, pos, r, dtype)
        gk = normal(4, (T, hk, D), dtype)
        dq, dk, dwq, dwk = torch.autograd.grad([qo, ko], [q, k, wq, wk], [gq, gk])
        check_gradients(dk, dwk, k, wk, gk, pos, r, dtype, "fp32")
    else:
        dq, dwq = torch.autograd.grad([qo], [q, wq], [gq])
    check_gradients(dq, dwq, q, wq, gq, pos, r, dtype, "fp32")


@pytest.mark.parametrize("shift", [0, 1, 8])
def test_slices_of_a_projection(at, shift):  # noqa: F811
    """q and k in one projection's rows, results in another's; a shift of one element leaves no wide access aligned."""
    T, hq, hk, D = 11, 6, 2, 64
    r, pos = rope(at, D, D, False, "none"), np.arange(T) * 1000
    wide = normal(3, (T, (hq + hk) * D + 24), "bf16")
    rows = wide[:, shift:shift + (hq + hk) * D]
    q, k = rows[:, :hq * D].unflatten(1, (hq, D)), rows[:, hq * D:].unflatten(1, (hk, D))
    w = gains(1, D, "bf16")
    n = at.NormedRotary(r, w, None, eps=EPS)
    qo, ko = n.apply(q, k, dev(pos))
    check_normed(qo, q, w, pos, r, "bf16")
    check_normed(ko, k, None, pos, r, "bf16")
    before = wide.clone()
    n.apply(q, k, dev(pos), q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(wide[:, :shift], before[:, :shift]) and torch.equal(wide[:, shift + (hq + hk) * D:], before[:, shift + (hq + hk) * D:])
    # heads outside, tokens inside; gradients of slices
    x = normal(5, (hq, T, D), "bf16").requires_grad_()
    y, _ = at.NormedRotary(r, eps=EPS).apply(x.transpose(0, 1), None, dev(pos))
    check_normed(y, x.transpose(0, 1), None, pos, r, "bf16")
    leaf = wide.clone().requires_grad_()
    part = leaf[:, shift:shift + hq * D].unflatten(1, (hq, D))
    y, _ = at.NormedRotary(r, eps=EPS).apply(part, None, dev(pos))
    g = normal(6, (T, hq, D), "bf16")
    (dx,) = torch.autograd.grad(y, leaf, g)
    check_gradients(dx[:, shift:shift + hq * D].unflatten(1, (hq, D)), None, part, None, g, pos, r, "bf16", None)
    assert (dx[:, :shift] == 0).all() and (dx[:, shift + hq * D:] == 0).all()


def test_gradients_alone_expanded_or_not_at_all(at):  # noqa: F811
    r, pos = rope(at, 64, 64, False, "none"), dev([1, 2, 3])
    q, k = (normal(i, (3, 2, 64), "fp32").requires_grad_() for i in (1, 2))
    wq, wk = gains(1, 64, "fp32").requires_grad_(), gains(2, 64, "fp32").requires_grad_()
    n = at.NormedRotary(r, wq, wk, eps=EPS)
    ones = torch.ones(3, 2, 64, device="cuda")
    got = torch.autograd.grad(n.apply(q, k, pos)[0].sum(), [q, wq, k, wk], allow_unused=True)       # expanded, and none for k
    check_gradients(got[0], got[1], q, wq, ones, [1, 2, 3], r, "fp32", "fp32")
    assert all(g is None or (g == 0).all() for g in got[2:])
    got = torch.autograd.grad(n.apply(q.detach(), k, pos)[1].sum(), [k, wk, wq], allow_unused=True)
    check_gradients(got[0], got[1], k, wk, ones, [1, 2, 3], r, "fp32", "fp32")
    assert got[2] is None or (got[2] == 0).all()
    (dw,) = torch.autograd.grad(n.apply(q.detach(), None, pos)[0].sum(), [wq])                      # a gain alone
    check_gradients(None, dw, q, wq, ones, [1, 2, 3], r, "fp32", "fp32")
    shared = normal(5, (3, 1, 64), "fp32").requires_grad_()
    (dx,) = torch.autograd.grad(at.NormedRotary(r, eps=EPS).apply(shared.expand(3, 4, 64), None, pos)[0].sum(), shared)    # one head seen as four
    check_gradients(dx / 4, None, shared, None, ones[:, :1], [1, 2, 3], r, "fp32", None)
    empty = torch.zeros(0, 2, 64, device="cuda", requires_grad=True)
    y, _ = n.apply(empty, None, dev(np.zeros(0)))
    dx, dw = torch.autograd.grad(y.sum(), [empty, wq])
    assert dx.shape == empty.shape and (dw == 0).all()
    with torch.no_grad():
        assert not n.apply(q, k, pos)[0].requires_grad
    with pytest.raises(RuntimeError):                     # one derivative
        g = torch.autograd.grad(n.apply(q, k, pos)[0].square().sum(), q, create_graph=True)[0]
        g.sum().backward()


@pytest.mark.parametrize("inter", [False, True])
def test_gradients_against_differences(at, inter):  # noqa: F811
    """Central differences in fp32.  With heads of size 1 and a step h = 2^-6 a function of the norm's smoothness is off by h^2 (third
    derivatives below 16 times the sizes involved, over 6) and its values of size |y| <= 3 by 2^-20 each, over h: below 2^-9."""
    D = 64
    r, pos = rope(at, D, 32, inter, "ramp"), dev([3, 700])
    x, g = normal(1, (2, 1, D), "fp32").requires_grad_(), normal(2, (2, 1, D), "fp32")
    w = gains(3, D, "fp32").requires_grad_()
    n = at.NormedRotary(r, w, eps=EPS)
    dx, dw = torch.autograd.grad(n.apply(x, None, pos)[0], [x, w], g)
    h = 2.0 ** -6
    loss = lambda x, w: f64(at.NormedRotary(r, w.detach(), eps=EPS).apply(x.detach(), None, pos)[0] * 1.0) * f64(g)  # noqa: E731
    size = np.abs(f64(g)).sum(-1).max()
    for e in (0, 5, 16, 31, 40, 63):
        step = torch.zeros(D, device="cuda")
        step[e] = h
        change = (loss(x + step, w) - loss(x - step, w)) / (2 * h)
        assert (np.abs(f64(dx)[:, 0, e] - change.sum(-1)[:, 0]) <= 2.0 ** -9 * size).all()
        assert abs(f64(dw)[e] - (loss(x, w + step) - loss(x, w - step)).sum() / (2 * h)) <= 2.0 ** -9 * size


def test_a_captured_pass_and_a_stream_of_its_own(at):  # noqa: F811
    r, pos = rope(at, 128, 128, False, "none"), dev(np.arange(40))
    q, k, g = normal(1, (40, 8, 128), "bf16"), normal(2, (40, 2, 128), "bf16"), normal(3, (40, 8, 128), "bf16")
    w = gains(1, 128, "fp32")
    n = at.NormedRotary(r, w, w, eps=EPS)
    want = n.apply(q, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = n.apply(q, k, pos, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # forward and backward in one graph, replayed over new inputs
    static = [x.clone() for x in (q, g)]
    with torch.cuda.stream(side):
        leaf, lw = static[0].detach().requires_grad_(), w.clone().requires_grad_()
        m = at.NormedRotary(r, lw, eps=EPS)
        torch.autograd.grad(m.apply(leaf, None, pos)[0], [leaf, lw], static[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = m.apply(leaf, None, pos)[0]
        dx, dw = torch.autograd.grad(y, [leaf, lw], static[1])
    del y
    for seed in (11, 12):
        static[0].copy_(normal(seed, q.shape, "bf16"))
        static[1].copy_(normal(seed + 5, q.shape, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        check_gradients(dx, dw, static[0], w, static[1], np.arange(40), r, "bf16", "fp32")
