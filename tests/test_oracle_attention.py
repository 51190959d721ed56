"""The 64-bit definitions of the attention side, pinned on the CPU against what they should be by other routes, and the
refusals of the C entry points (which come before anything touches a GPU)."""
import ctypes
import math

import numpy as np
import pytest

from oracle import attention as oa
from paper_2608_15602_b200 import build, fluxbin

build.build()


def test_a_turn_keeps_lengths_and_depends_on_the_difference_of_positions():
    rng = np.random.default_rng(1)
    f, m = oa.frequencies(32)
    assert m == 1.0 and f[0] == 1.0 and abs(f[-1] - 10000.0 ** (-30 / 32)) < 1e-15
    q, k = rng.standard_normal((2, 1, 1, 40))
    for inter in (False, True):
        at = lambda x, p: oa.rotary(x, [p], f, m, 32, inter)[0, 0]  # noqa: E731
        assert abs(np.linalg.norm(at(q, 91)) - np.linalg.norm(q)) < 1e-12
        assert abs(at(q, 107) @ at(k, 100) - at(q, 7) @ at(k, 0)) < 1e-10
        assert np.array_equal(at(q, 91)[32:], q[0, 0, 32:])
        assert np.abs(oa.rotary(at(q, 91)[None, None], [91], f, m, 32, inter, inverse=True) - q).max() < 1e-12


def test_the_gradient_of_a_turn_is_the_turn_back():
    rng = np.random.default_rng(2)
    f, m = oa.frequencies(8, scaling="ramp", factor=4.0, original=64)
    x, g = rng.standard_normal((2, 3, 2, 12))
    pos = [0, 5, 77]
    for inter in (False, True):
        grad = oa.rotary(g, pos, f, m, 8, inter, inverse=True)
        for at in [(0, 0, 0), (1, 1, 3), (2, 0, 7), (2, 1, 11)]:
            d = np.zeros_like(x)
            d[at] = 1e-3                     # the map is linear: a difference is exact up to rounding
            slope = ((oa.rotary(x + d, pos, f, m, 8, inter) - oa.rotary(x - d, pos, f, m, 8, inter)) * g).sum() / 2e-3
            assert abs(slope - grad[at]) < 1e-9


@pytest.mark.parametrize("kind,kw", [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                     ("ramp", dict(factor=16.0, original=4096, fast=32.0, slow=1.0)),
                                     ("bands", dict(factor=8.0, original=8192, low=1.0, high=4.0))])
@pytest.mark.parametrize("d", [4, 64, 128])
def test_frequencies_are_the_fractions_of_a_turn(kind, kw, d):
    f, m = oa.frequencies(d, scaling=kind, **kw)
    a, b = (kw.get("fast", 0), kw.get("slow", 0)) if kind == "ramp" else (kw.get("low", 0), kw.get("high", 0))
    code = ["none", "linear", "base", "ramp", "bands"].index(kind)
    turns, mag = fluxbin.rotary_frequencies(d, 10000.0, code, kw.get("factor", 1.0), kw.get("original", 1.0), a, b)
    got = turns.astype(np.float64) / 2.0 ** 64 * 2 * math.pi
    assert np.abs(got / f - 1).max() < 1e-12 and abs(mag - m) < 1e-6


def test_refused_frequencies():
    lib, out, mag = fluxbin.library(), (ctypes.c_uint64 * 256)(), ctypes.c_float()
    call = lambda *a: lib.fluxbin_rotary_frequencies(*a, ctypes.addressof(out), ctypes.byref(mag))  # noqa: E731
    assert call(128, 1e4, 0, 1.0, 1.0, 0.0, 0.0) == 0
    for bad in [(127, 1e4, 0, 1.0, 1.0, 0.0, 0.0), (0, 1e4, 0, 1.0, 1.0, 0.0, 0.0), (514, 1e4, 0, 1.0, 1.0, 0.0, 0.0), (128, 1.0, 0, 1.0, 1.0, 0.0, 0.0),
                (128, float("nan"), 0, 1.0, 1.0, 0.0, 0.0), (128, 1e4, 1, 0.5, 1.0, 0.0, 0.0), (2, 1e4, 2, 2.0, 1.0, 0.0, 0.0),
                (128, 1e4, 3, 2.0, 4096.0, 1.0, 32.0), (128, 1e4, 4, 2.0, 4096.0, 4.0, 1.0), (128, 1e4, 3, 2.0, 0.0, 32.0, 1.0)]:
        assert call(*bad) == 3, bad
    assert call(128, 1e4, 9, 1.0, 1.0, 0.0, 0.0) == 7
    assert lib.fluxbin_rotary_frequencies(128, 1e4, 0, 1.0, 1.0, 0.0, 0.0, None, ctypes.byref(mag)) == 1


def test_entries_are_the_nearest_ones():
    v = oa.e4m3_values()
    assert v[0x7e] == 448.0 and v[1] == 2.0 ** -9 and np.isnan(v[0x7f])
    fine = v[np.isfinite(v)]
    assert np.array_equal(oa.to_entry(fine, "e4m3"), fine)
    x = np.random.default_rng(3).uniform(-448, 448, 4000)
    near = np.abs(x[:, None] - fine[None, :]).min(1)
    assert np.array_equal(np.abs(oa.to_entry(x, "e4m3") - x), near)
    assert oa.to_entry(np.array([17.0]), "e4m3")[0] == 16.0 and oa.to_entry(np.array([19.0]), "e4m3")[0] == 20.0      # ties to even
    assert np.array_equal(oa.to_entry(np.array([0.5, 1.5, -200.0]), "int8"), [0.0, 2.0, -127.0])


@pytest.mark.parametrize("fmt,step", [("int8", 0.5 / 127), ("e4m3", 2.0 ** -4)])
def test_appending_keeps_values_within_half_a_step(fmt, step):
    rng = np.random.default_rng(4)
    c = oa.Cache(np.full((3, 2, 16, 8), 99.0), np.full((3, 2), 7.0), fmt)
    x = rng.standard_normal((21, 2, 8)) * np.linspace(0.1, 3, 21)[:, None, None]
    for a, b in [(0, 5), (5, 6), (6, 21)]:
        c.append(x[a:b], [16 + t if t < 16 else t - 16 for t in range(a, b)])
    got = np.concatenate([c.values()[1], c.values()[0][:, :5]], 1).transpose(1, 0, 2)
    # each requantisation adds at most half a step of the final scale; at most one growth per append call
    top = np.concatenate([np.repeat(np.abs(x[:16]).max((0, 2))[None], 16, 0), np.repeat(np.abs(x[16:]).max((0, 2))[None], 5, 0)])[:, :, None]
    bound = top * step if fmt == "int8" else np.maximum(np.abs(x) * step, top / 448 * 2.0 ** -10)
    assert (np.abs(got - x) <= 3.2 * bound).all()
    assert (c.values()[2] == 99.0 * 7.0).all() and (c.values()[0][:, 5:] == 99.0 * c.scale[0][:, None, None]).all()


def test_attention_of_one_head_is_softmax():
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((2, 2, 1, 16, 4))
    q = rng.standard_normal((2, 1, 4))
    table = np.array([[1, 0]])
    out, lse, _, _ = oa.attend(q, k, v, table, [19], [0, 2], 0.5)
    K, V = np.concatenate([k[1, 0], k[0, 0, :3]]), np.concatenate([v[1, 0], v[0, 0, :3]])
    for t, n in ((0, 18), (1, 19)):
        e = np.exp(0.5 * (K[:n] @ q[t, 0]))
        assert np.abs(out[t, 0] - (e[:, None] * V[:n]).sum(0) / e.sum()).max() < 1e-13
        assert abs(lse[t, 0] - np.log(e.sum())) < 1e-13
    out, lse, _, _ = oa.attend(q, k, v, table, [1], [0, 2], 0.5)             # two queries, one cached token: the first sees nothing
    assert (out[0] == 0).all() and np.isinf(lse[0, 0]) and np.abs(out[1, 0] - v[1, 0, 0]).max() < 1e-15


def test_blocks_are_neither_lost_nor_shared():
    rng = np.random.default_rng(6)
    B, width, bs, nb = 9, 6, 16, 40
    table, free = np.full((B, width), -1, np.int32), rng.permutation(nb).astype(np.int32)
    lengths, nf = np.zeros(B, np.int64), nb
    for _ in range(60):
        new = rng.integers(-40, 45, B)
        T = int(new.clip(0).sum())
        r = oa.advance(lengths, new, table, free, nf, bs, T)
        lengths, nf = r["lengths"], r["num_free"]
        held = [b for i in range(B) for b in table[i, :-(-lengths[i] // bs)]]
        assert sorted(held + list(free[:nf])) == list(range(nb))
        live = r["slots"][r["slots"] >= 0]
        assert len(set(live)) == len(live)


# ---- refusals -----------------------------------------------------------------------------------------------------

def cache(**kw):
    d = dict(num_blocks=4, block_tokens=16, kv_heads=2, head_dim=64, format=0, d_k=1 << 20, d_v=1 << 21, block_stride=2048, head_stride=1024,
             token_stride=64, d_k_scale=1 << 22, d_v_scale=1 << 23)
    d.update(kw)
    return fluxbin.CacheDesc(**d)


@pytest.mark.parametrize("kw,status", [
    ({}, 0), (dict(d_k=None), 1), (dict(d_v_scale=None), 1), (dict(num_blocks=0), 3), (dict(kv_heads=0), 3), (dict(format=2), 7),
    (dict(head_dim=96), 7), (dict(block_tokens=24), 7), (dict(block_tokens=2048), 7), (dict(d_k=(1 << 20) + 8), 6), (dict(d_k_scale=(1 << 22) + 2), 6),
    (dict(token_stride=72), 6), (dict(token_stride=48), 3), (dict(head_stride=512), 3), (dict(block_stride=1024), 3), (dict(num_blocks=1 << 28), 3),
    (dict(token_stride=128, head_stride=64), 0),                       # the other order of the middle axes
    (dict(num_blocks=1, block_stride=0), 0), (dict(token_stride=-64), 3)])
def test_refused_caches(kw, status):
    assert fluxbin.kv_validate_status(cache(**kw)) == status


def test_refused_calls():
    c, r = cache(), fluxbin.RotaryDesc(64, 64, 0, 1.0, 1 << 24)
    C, R, P = ctypes.addressof(c), ctypes.addressof(r), 1 << 25
    rot = lambda desc=R, dt=0, n=2, pos=P, q=P, qh=2, qo=P, k=None, kh=0, ko=None: fluxbin.rotary_status(  # noqa: E731
        desc, dt, 0, n, pos, q, qh, 128, 64, qo, 128, 64, k, kh, 128, 64, ko, 128, 64, None)
    assert rot(n=0) == 0 and rot(desc=None) == 1 and rot(dt=3) == 7 and rot(n=-1) == 3 and rot(pos=None) == 1 and rot(q=None) == 1
    assert rot(qh=0) == 3 and rot(k=P) == 3 and rot(k=P, kh=1) == 1 and rot(q=P + 1) == 6 and rot(qo=P + 1) == 6
    for bad in [fluxbin.RotaryDesc(64, 66, 0, 1.0, P), fluxbin.RotaryDesc(64, 3, 0, 1.0, P), fluxbin.RotaryDesc(1024, 64, 0, 1.0, P)]:
        assert rot(desc=ctypes.addressof(bad)) == 3
    app = lambda desc=C, dt=0, n=2, slots=P, k=P, v=P, rt=None, pos=None, q=None, qh=0, qo=None: fluxbin.kv_append_status(  # noqa: E731
        desc, dt, n, slots, k, 128, 64, v, 128, 64, rt, pos, q, qh, 128, 64, qo, 128, 64, None)
    assert app(n=0) == 0 and app(desc=None) == 1 and app(dt=5) == 7 and app(n=-1) == 3 and app(slots=None) == 1 and app(v=None) == 1
    assert app(rt=R) == 1 and app(rt=R, pos=P, q=P, qh=0) == 3 and app(rt=R, pos=P, q=P, qh=2) == 1 and app(k=P + 1) == 6
    other = fluxbin.RotaryDesc(128, 64, 0, 1.0, P)
    assert app(rt=ctypes.addressof(other), pos=P) == 7
    read = lambda desc=C, dt=0, n=2, slots=P, ko=P, vo=P: fluxbin.kv_read_status(desc, dt, n, slots, ko, vo, None)  # noqa: E731
    assert read(n=0) == 0 and read(dt=9) == 7 and read(slots=None) == 1 and read(ko=P + 4) == 6 and read(ko=None, vo=None) == 0
    ws = fluxbin.kv_attend_workspace_size(2, 2, 4, 2, 64)
    assert ws > 0 and fluxbin.kv_attend_workspace_size(2, 2, 3, 2, 64) == 0
    att = lambda desc=C, dt=0, b=2, n=2, q=P, qh=4, qt=256, qs=None, ln=P, tb=P, st=8, w=8, o=P, wsp=P, wb=ws: fluxbin.kv_attend_status(  # noqa: E731
        desc, dt, b, n, q, qh, qt, 64, qs, ln, tb, st, w, 0.125, o, 256, 64, None, wsp, wb, None)
    assert att(qs=P, n=0) == 0 and att(desc=None) == 1 and att(dt=1) == 7 and att(b=0) == 3 and att(n=3) == 3 and att(qh=3) == 3 and att(w=0) == 3
    assert att(st=7) == 3 and att(q=None) == 1 and att(ln=None) == 1 and att(tb=None) == 1 and att(wsp=None) == 1 and att(q=P + 8) == 6
    assert att(qt=260) == 6 and att(wb=ws - 1) == 5
    adv = lambda b=2, t=2, bs=16, ln=P, tb=P, st=4, w=4, fr=P, cap=4, nf=P, lo=2 * P, nfo=2 * P, po=P: fluxbin.kv_advance_status(  # noqa: E731
        b, t, bs, ln, P, tb, st, w, fr, cap, nf, nfo, lo, P, P, po, P, P, None)
    assert adv(b=0) == 3 and adv(b=8193) == 3 and adv(t=-1) == 3 and adv(bs=0) == 3 and adv(w=0) == 3 and adv(st=3) == 3 and adv(cap=0) == 3
    assert adv(ln=None) == 1 and adv(po=None) == 1 and adv(lo=P) == 3 and adv(nfo=P) == 3 and adv(ln=P + 2) == 6


def test_calls_by_words_refuse_what_the_calls_refuse():
    lib = fluxbin.library()
    assert lib.fluxbin_call_words(0, None) == 1 and lib.fluxbin_call_words(5, bytes(200)) == 7 and lib.fluxbin_call_words(-1, bytes(200)) == 7
    assert lib.fluxbin_call_words(0, bytes(200)) == 1 and lib.fluxbin_call_words(1, bytes(200)) == 1        # no descriptor
    assert lib.fluxbin_call_words(3, bytes(200)) == 1 and lib.fluxbin_call_words(4, bytes(200)) == 3        # no cache; no request
    c = cache()
    P = 1 << 25
    ws = fluxbin.kv_attend_workspace_size(2, 2, 4, 2, 64)
    good = dict(desc=ctypes.addressof(c), dtype=0, batch=2, tokens=0, q=P, heads=4, qt=256, qh=64, start=P, lengths=P, table=P, stride=8, width=8, scale=0.5,
                out=P, ot=256, oh=64, lse=0, ws=P, bytes=ws, stream=0)
    fluxbin.kv_attend_call(*good.values())                                                                   # no tokens: nothing to do
    for name, value, status in [("dtype", 1, 7), ("batch", 0, 3), ("heads", 3, 3), ("width", 9, 3), ("desc", 0, 1)]:
        with pytest.raises(fluxbin.FluxBinError) as e:
            fluxbin.kv_attend_call(*{**good, name: value}.values())
        assert e.value.status == status, name
