"""The 64-bit definitions of checking trees of drafted tokens, pinned by hand-made cases, and the calls' refusals (no GPU)."""
import ctypes

import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od
from paper_2608_15602_b200 import build, fluxbin

build.build()


def test_a_normed_head_has_mean_square_one_and_its_gradient_is_that_of_differences():
    rng = np.random.default_rng(1)
    f, m = oa.frequencies(4)
    x, w, g = rng.normal(size=(2, 3, 6)), rng.normal(size=6), rng.normal(size=(2, 3, 6))
    y = od.norm_rotary(x, None, 1e-12, [5, 9], f, m, 4, False)
    assert np.allclose((y * y).mean(-1), 1.0)
    dx, dw, _ = od.norm_rotary_backward(x, w, 0.1, g, [5, 9], f, m, 4, False)
    loss = lambda x, w: (od.norm_rotary(x, w, 0.1, [5, 9], f, m, 4, False) * g).sum()  # noqa: E731
    h = 1e-6
    for i in np.ndindex(2, 3, 6):
        d = np.zeros_like(x)
        d[i] = h
        assert abs((loss(x + d, w) - loss(x - d, w)) / (2 * h) - dx[i]) < 1e-7
    for i in range(6):
        d = np.zeros(6)
        d[i] = h
        assert abs((loss(x, w + d) - loss(x, w - d)) / (2 * h) - dw[i]) < 1e-7


def test_a_tree_by_hand():
    #      0        the last known token
    #     / \
    #    1   2     3 stands beside 0
    #    |
    #    4
    parents, start = [-1, 0, 0, -1, 1, 9, 0], [0, 5, 5, 7]
    mask, pos = od.tree(parents, start, [15, 4, 2], 33)
    assert mask.tolist() == [[1, 0], [3, 0], [5, 0], [8, 0], [19, 0], [1, 0], [3, 0]] and pos.tolist() == [10, 11, 11, 10, 12, 0, 1]
    mask, pos = od.tree(parents, start, [15, 4, 2], 3)                   # only three count
    assert mask[:, 0].tolist() == [1, 3, 5, 0, 0, 1, 3] and pos.tolist() == [10, 11, 11, 10, 10, 0, 1]
    drafted, answers = [50, 51, 52, 50, 53, 60, 61], [52, 53, 54, 0, 55, 61, 62]
    path, count, answer, surplus = od.accept(parents, drafted, answers, start, 3, 33)
    assert path.tolist() == [0, 2, -1, -1, -1, 0, 1] and count.tolist() == [2, 0, 2] and answer.tolist() == [54, -1, 62] and surplus.tolist() == [-3, 0, 0]
    answers[0] = 51
    assert od.accept(parents, drafted, answers, start, 3, 33)[0][:5].tolist() == [0, 1, 4, -1, -1]


def test_masks_of_a_chain_are_attention_up_to_itself():
    rng = np.random.default_rng(2)
    k, v, q = rng.normal(size=(4, 2, 16, 8)), rng.normal(size=(4, 2, 16, 8)), rng.normal(size=(5, 4, 8))
    table, lengths, start = np.array([[2, 0], [3, 1]]), [20, 7], [0, 3, 5]
    mask, _ = od.tree([-1, 0, 1, -1, 0], start, lengths, 3)
    for a, b in zip(od.attend(q, k, v, table, lengths, start, mask, 0.3), oa.attend(q, k, v, table, lengths, start, 0.3)):
        assert np.allclose(a, b)


def test_keeping_moves_what_entries_stand_for():
    rng = np.random.default_rng(3)
    c = oa.Cache(rng.integers(-127, 128, (3, 1, 16, 4)).astype(float), [[1.0], [4.0], [1.0]], "int8")
    before = c.values()
    slots = [13, 14, 15, 16, 17, 18]                                     # a request across two blocks
    od.keep(c, [0, 6], slots, [0, 2, 4, 5, -1, -1])
    after = c.values().reshape(48, 4)
    old = before.reshape(48, 4)
    assert np.array_equal(after[13], old[13]) or c.scale[0, 0] > 1
    assert np.abs(after[14] - old[15]).max() <= c.scale[0, 0] / 2 and np.abs(after[15] - old[17]).max() <= c.scale[0, 0] / 2
    assert np.abs(after[16] - old[18]).max() <= c.scale[1, 0] / 2 and c.scale[1, 0] <= 4.0


# ---- refusals --------------------------------------------------------------------------------------------------------

P = 1 << 25


def a_cache(**kw):
    d = dict(num_blocks=8, block_tokens=16, kv_heads=2, head_dim=64, format=0, d_k=1 << 20, d_v=1 << 21, block_stride=2048, head_stride=1024,
             token_stride=64, d_k_scale=1 << 22, d_v_scale=1 << 23)
    d.update(kw)
    return fluxbin.CacheDesc(**d)


def test_refused_norms():
    r = fluxbin.RotaryDesc(64, 64, 0, 1.0, 1 << 24)
    R = ctypes.addressof(r)
    good = dict(desc=R, eps=1e-6, dt=0, wt=1, n=2, pos=P, q=P, qh=2, qt=128, qs=64, qw=P, qo=P, qot=128, qos=64, k=None, kh=0, kt=0, ks=0, kw=None, ko=None, kot=0, kos=0)
    call = lambda **kw: fluxbin.norm_rotary_status(*{**good, **kw}.values(), None)  # noqa: E731
    for kw, status in [(dict(n=0), 0), (dict(desc=None), 1), (dict(dt=3), 7), (dict(wt=-1), 7), (dict(eps=0.0), 3), (dict(eps=-1.0), 3), (dict(eps=float("nan")), 3),
                       (dict(eps=float("inf")), 3), (dict(n=-1), 3), (dict(pos=None), 1), (dict(q=None), 1), (dict(qo=None), 1), (dict(qh=0), 3), (dict(k=P), 3),
                       (dict(k=P, kh=1), 1), (dict(q=P + 1), 6), (dict(qo=P + 1), 6), (dict(qw=P + 2), 6), (dict(pos=P + 2), 6), (dict(qot=64), 3), (dict(qos=0), 3)]:
        assert call(**kw) == status, kw
    for bad in [fluxbin.RotaryDesc(64, 66, 0, 1.0, P), fluxbin.RotaryDesc(64, 3, 0, 1.0, P), fluxbin.RotaryDesc(1024, 64, 0, 1.0, P)]:
        assert call(desc=ctypes.addressof(bad)) == 3


def test_refused_norm_gradients():
    r = fluxbin.RotaryDesc(64, 64, 0, 1.0, 1 << 24)
    ws = fluxbin.norm_rotary_backward_workspace_size(64)
    assert ws > 0 and fluxbin.norm_rotary_backward_workspace_size(1) == 0 and fluxbin.norm_rotary_backward_workspace_size(513) == 0
    good = dict(desc=ctypes.addressof(r), eps=1e-6, dt=0, wt=1, n=2, pos=P, q=P, qh=2, qt=128, qs=64, qw=P, g=P, gt=0, gs=0, dx=P, dt_=128, ds=64, dw=P,
                k=None, kh=0, kt=0, ks=0, kw=None, kg=None, kgt=0, kgs=0, kdx=None, kdt=0, kds=0, kdw=None, w=P, wb=ws)
    call = lambda **kw: fluxbin.norm_rotary_backward_status(*{**good, **kw}.values(), None)  # noqa: E731
    for kw, status in [(dict(desc=None), 1), (dict(dt=3), 7), (dict(wt=3), 7), (dict(eps=0.0), 3), (dict(n=-1), 3), (dict(pos=None), 1), (dict(g=None), 1), (dict(qh=0), 3),
                       (dict(dx=P + 1), 6), (dict(g=P + 1), 6), (dict(dw=P + 2), 6), (dict(w=None), 1), (dict(w=P + 8), 6), (dict(wb=ws - 1), 5), (dict(dt_=64), 3),
                       (dict(q=None), 0), (dict(dx=None, dw=None), 0), (dict(k=P), 3), (dict(k=P, kh=1), 1)]:
        assert call(**kw) == status, kw


def test_refused_trees():
    tree = lambda b=2, n=3, nodes=8, s=P, ln=P, p=P, m=P, pos=P: fluxbin.draft_tree_status(b, n, nodes, s, ln, p, m, pos, None)  # noqa: E731
    assert tree(n=0) == 0 and tree(b=0) == 3 and tree(n=-1) == 3 and tree(nodes=0) == 3 and tree(nodes=1025) == 3
    assert tree(s=None) == 1 and tree(ln=None) == 1 and tree(p=None) == 1 and tree(m=None) == 1 and tree(pos=None) == 1 and tree(m=P + 2) == 6 and tree(p=P + 1) == 6
    acc = lambda b=2, n=3, nodes=8, s=P, p=P, d=P, a=P, path=P, c=P, x=P, y=P: fluxbin.draft_accept_status(b, n, nodes, s, p, d, a, path, c, x, y, None)  # noqa: E731
    assert acc(b=0) == 3 and acc(n=-1) == 3 and acc(nodes=0) == 3 and acc(nodes=2000) == 3
    assert acc(s=None) == 1 and acc(p=None) == 1 and acc(d=None) == 1 and acc(a=None) == 1 and acc(path=None) == 1 and acc(c=None) == 1 and acc(y=None) == 1 and acc(x=P + 2) == 6
    c = a_cache()
    C = ctypes.addressof(c)
    keep = lambda desc=C, b=2, n=3, s=P, sl=P, p=P: fluxbin.kv_keep_status(desc, b, n, s, sl, p, None)  # noqa: E731
    assert keep(n=0) == 0 and keep(desc=None) == 1 and keep(b=0) == 3 and keep(n=-1) == 3 and keep(s=None) == 1 and keep(sl=None) == 1 and keep(p=None) == 1 and keep(sl=P + 1) == 6
    bad = a_cache(head_dim=96)
    assert keep(desc=ctypes.addressof(bad)) == 7


def test_refused_tree_attention():
    c = a_cache()
    ws = fluxbin.kv_attend_tree_workspace_size(2, 2, 4, 2, 64)
    assert ws >= fluxbin.kv_attend_workspace_size(2, 2, 4, 2, 64) and fluxbin.kv_attend_tree_workspace_size(2, 2, 3, 2, 64) == 0
    good = dict(desc=ctypes.addressof(c), dt=0, b=2, n=2, q=P, qh=4, qt=256, qs=64, start=None, ln=P, tree=P, ts=1, tw=1, tb=P, st=8, w=8, scale=0.125, o=P, ot=256, os=64,
                lse=None, wsp=P, wb=ws)
    call = lambda **kw: fluxbin.kv_attend_tree_status(*{**good, **kw}.values(), None)  # noqa: E731
    for kw, status in [(dict(start=P, n=0), 0), (dict(desc=None), 1), (dict(dt=1), 7), (dict(b=0), 3), (dict(n=3), 3), (dict(qh=3), 3), (dict(w=0), 3), (dict(st=7), 3), (dict(q=None), 1),
                       (dict(ln=None), 1), (dict(tb=None), 1), (dict(tree=None), 1), (dict(wsp=None), 1), (dict(q=P + 8), 6), (dict(tree=P + 2), 6), (dict(qt=260), 6), (dict(wb=ws - 1), 5),
                       (dict(tw=0), 3), (dict(tw=1 << 27), 3), (dict(ts=-1), 3), (dict(os=0), 3), (dict(ts=0, wb=0), 5), (dict(st=0, wb=0), 5)]:
        assert call(**kw) == status, kw
    # by words, in the same order
    with pytest.raises(fluxbin.FluxBinError) as e:
        fluxbin.kv_attend_tree_call(*(0 if v is None else v for v in {**good, "wb": ws - 1}.values()), 0)
    assert e.value.status == 5
    lib = fluxbin.library()
    for which in (15, 22):
        assert lib.fluxbin_call_words(which, bytes(400)) == 7
    for which, status in ((16, 1), (17, 1), (18, 3), (19, 3), (20, 1), (21, 1)):
        assert lib.fluxbin_call_words(which, bytes(400)) == status
