"""GPU parity of the attention side (rotary positions, 8-bit cache, attention, block tables) against its 64-bit definitions.

Bounds.  u is the unit roundoff of the result's type (2^-11 fp16, 2^-8 bf16, 2^-24 fp32).
  turns      the angle is off by 2^-24 half turns (one fp32 rounding, sincospif within 2 ulp) and there are three fp32
             roundings: |error| <= u |y| + 2^-20 (|a| + |b|)
  attention  with A the mean of |v| under the probabilities, S the largest scale * sum |q k| of the row and L its length:
             a score is off by at most (D + 4) 2^-24 S, a probability enters its product rounded to fp16 (2^-11) after two
             fp32 factors, its exponential is good to 2^-21, sums add L 2^-24:
             |error| <= u |out| + (2^-11 + 2^-19 + (2 D + 8) 2^-24 S + L 2^-23) A
             |lse error| <= (D + 4) 2^-24 S + 2^-20 + L 2^-24 + 2^-23 |lse|
  cache      entries equal those of the same rule in fp32 except where a quotient lies within fp32 rounding of a tie:
             then they are neighbours; scales within 2^-22
"""
import numpy as np
import pytest

from oracle import attention as oa

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
DT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def at():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2608_15602_b200 import build
    build.build()
    from paper_2608_15602_b200 import attention
    return attention


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def normal(seed, shape, dtype, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * spread).to(DT[dtype]).cuda()


def entries_of(c):
    return f64(c.k.to(torch.float32)), f64(c.v.to(torch.float32))


# ---- rotary -------------------------------------------------------------------------------------------------------

ROPE = [  # tokens, q heads, k heads, head dim, rotary dim, interleaved, dtype, scaling
    (1, 1, 1, 64, 64, False, "fp16", "none"), (3, 5, 0, 128, 128, True, "bf16", "none"), (7, 4, 2, 128, 64, False, "fp32", "linear"),
    (5, 3, 1, 80, 20, True, "fp16", "base"), (2, 2, 2, 96, 34, False, "bf16", "ramp"), (33, 8, 2, 256, 256, False, "fp16", "bands"),
    (4, 1, 1, 6, 2, True, "fp32", "none"), (9, 12, 12, 64, 32, True, "fp16", "ramp"), (130, 72, 8, 128, 128, False, "bf16", "none")]
KW = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "ramp": dict(factor=16.0, original=4096, fast=32.0, slow=1.0),
      "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0)}


def check_turn(got, x, pos, r, dtype, inverse=False):
    f, m = oa.frequencies(r.rotary_dim, scaling=r.kind, **KW[r.kind])
    want = oa.rotary(f64(x), pos, f, m, r.rotary_dim, r.interleaved, inverse)
    size = oa.rotary(np.abs(f64(x)), [0] * len(pos), f * 0, 1.0, r.rotary_dim, r.interleaved)
    half = r.rotary_dim // 2
    both = np.zeros_like(size)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if r.interleaved else (i, i + half)
        both[..., a] = both[..., b] = size[..., a] + size[..., b]
    err = np.abs(f64(got) - want)
    assert (err <= U[dtype] * np.abs(want) + 2.0 ** -20 * both + 1e-7 * (dtype == "fp16")).all(), err.max()
    assert np.array_equal(f64(got)[..., r.rotary_dim:], f64(x)[..., r.rotary_dim:])


def rope(at, D, d, inter, kind):
    r = at.Rotary(D, d, interleaved=inter, scaling=kind, **KW[kind])
    r.kind = kind
    return r


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype,kind", ROPE)
def test_rotary(at, T, hq, hk, D, d, inter, dtype, kind):
    r = rope(at, D, d, inter, kind)
    pos = np.random.default_rng(T).integers(0, 131072, T)
    pos[0] = 0
    if T > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -5
    q, k = normal(1, (T, hq, D), dtype), normal(2, (T, hk, D), dtype) if hk else None
    for inverse in (False, True):
        qo, ko = r.apply(q, k, dev(pos), inverse=inverse)
        check_turn(qo, q, pos, r, dtype, inverse)
        if hk:
            check_turn(ko, k, pos, r, dtype, inverse)


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype,kind", ROPE[:4])
def test_rotary_in_place_strided_and_unaligned(at, T, hq, hk, D, d, inter, dtype, kind):
    r = rope(at, D, d, inter, kind)
    pos = dev(np.arange(T) * 1000)
    for shift in (0, 1, 2, 8):
        # q and k are slices of one projection's rows; a shift of one element leaves no wide access aligned
        rows = normal(3, (T, (hq + hk) * D + 24), dtype)
        q = rows[:, shift:shift + hq * D].unflatten(1, (hq, D))
        k = rows[:, shift + hq * D:shift + (hq + hk) * D].unflatten(1, (hk, D)) if hk else None
        before, qc, kc = rows.clone(), q.clone(), k.clone() if hk else None
        qo, ko = r.apply(q, k, pos)
        check_turn(qo, qc, np.arange(T) * 1000, r, dtype)
        assert torch.equal(rows, before)
        r.apply(q, k, pos, q_out=q, k_out=k)
        assert torch.equal(q, qo) and (not hk or torch.equal(k, ko))
        assert torch.equal(rows[:, :shift], before[:, :shift]) and torch.equal(rows[:, shift + (hq + hk) * D:], before[:, shift + (hq + hk) * D:])


def test_rotary_no_tokens_and_head_major_input(at):
    r = rope(at, 128, 128, False, "none")
    q = normal(1, (0, 4, 128), "fp16")
    assert r.apply(q, None, dev(np.zeros(0)))[0].shape == q.shape
    q = normal(2, (6, 5, 128), "fp16").transpose(0, 1)             # [token 5][head 6]: the head stride is the larger one
    check_turn(r.apply(q, None, dev([3, 1, 4, 1, 5]))[0], q, [3, 1, 4, 1, 5], r, "fp16")


@pytest.mark.parametrize("T,hq,hk,D,d,inter,dtype", [(148, 5, 3, 128, 128, False, "fp16"), (700, 3, 0, 128, 64, True, "bf16"), (333, 40, 2, 64, 32, False, "fp32"),
                                                       (601, 1, 1, 256, 256, True, "fp16"), (149, 70, 1, 96, 96, True, "fp32"), (650, 2, 2, 80, 40, False, "bf16")])
def test_rotary_prompts(at, T, hq, hk, D, d, inter, dtype):
    """Enough tokens for the kernels that go over them (and, with the last, heads that allow no wide access to both halves)."""
    r = rope(at, D, d, inter, "none")
    pos = np.random.default_rng(T).integers(0, 131072, T)
    q, k = normal(1, (T, hq, D), dtype), normal(2, (T, hk, D), dtype) if hk else None
    qo, ko = r.apply(q, k, dev(pos))
    check_turn(qo, q, pos, r, dtype)
    if hk:
        check_turn(ko, k, pos, r, dtype)
    back, _ = r.apply(qo, None, dev(pos), inverse=True, q_out=qo)
    assert back is qo and (np.abs(f64(qo) - f64(q)) <= 4 * U[dtype] * np.abs(f64(q)).max()).all()


# ---- append and read ----------------------------------------------------------------------------------------------

def run_starts(slots, bs, t):
    return slots[t] >= 0 and (t == 0 or slots[t] % bs == 0 or slots[t - 1] != slots[t] - 1)


CACHES = [("int8", 16, 2, 64, False), ("int8", 32, 3, 128, True), ("e4m3", 16, 1, 256, False), ("e4m3", 64, 2, 128, True), ("int8", 128, 5, 64, False),
          ("e4m3", 48, 2, 64, False)]


def fill(c, seed):
    """Old contents: random entries (NaN patterns of e4m3 among them) and scales."""
    g = torch.Generator().manual_seed(seed)
    for x in (c.k, c.v):
        raw = torch.randint(0, 256, x.shape, generator=g, dtype=torch.uint8)
        if x.dtype is torch.int8:
            raw[raw == 128] = 0
        x.view(torch.uint8).copy_(raw)
    for s in (c.k_scale, c.v_scale):
        s.copy_(torch.rand(s.shape, generator=g) * 0.02 + 0.001)


def neighbours(got, want, fmt):
    """Whether entries are equal or next to each other."""
    if fmt == "int8":
        return np.abs(got - want) <= 1
    order = np.unique(oa.e4m3_values()[np.isfinite(oa.e4m3_values())])
    return np.abs(np.searchsorted(order, got) - np.searchsorted(order, want)) <= 1


def check_cache(c, want, fmt, turned):
    for name, w in zip("kv", want):
        scale = f64(getattr(c, name + "_scale"))
        assert np.array_equal(np.isnan(scale), np.isnan(w.scale))
        ok = ~np.isnan(w.scale)
        assert (np.abs(scale - w.scale)[ok] <= 2.0 ** (-18 if turned and name == "k" else -22) * np.abs(w.scale)[ok]).all()
        got = f64(getattr(c, name).to(torch.float32))
        live = ok[:, :, None, None] & ~np.isnan(w.entries)
        assert np.array_equal(np.isnan(got) & ok[:, :, None, None], np.isnan(w.entries) & ok[:, :, None, None])
        off = (got != w.entries) & live
        assert neighbours(got[off], w.entries[off], fmt).all()
        # a quotient in fp32 carries at most five roundings, 2^-21 of itself; a turned key is off by 2^-20 of its pair and
        # so is its scale, together less than 2^-17 of the largest entry.  Only a quotient that near to the midpoint of two
        # entries may have gone to the other one.
        middle = (got[off] + w.entries[off]) / 2
        near = 2.0 ** -17 * oa.TOP[fmt] if turned and name == "k" else 2.0 ** -21 * np.abs(middle)
        assert (np.abs(w.quotients[off] - middle) <= near).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("fmt,bs,H,D,major", CACHES)
def test_append_without_positions(at, fmt, bs, H, D, major, dtype):
    c = at.KVCache(7, bs, H, D, fmt, token_major=major)
    fill(c, 1)
    want = [oa.Cache(e, f64(s), fmt) for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
    order = [5, 2, 0, 6]
    length = 0
    for step, n in enumerate([1, 1, bs - 3, 1, 2 * bs + 5, 1, 3]):
        pos = np.arange(length, length + n)
        slots = np.array([order[p // bs] * bs + p % bs for p in pos], np.int32)
        k, v = normal(10 + step, (n, H, D), dtype, 0.3 + step), normal(50 + step, (n, H, D), dtype, 3.0 - 0.4 * step)
        c.append(k, v, dev(slots))
        for w, x in zip(want, (k, v)):
            w.append(f64(x), slots)
        check_cache(c, want, fmt, False)
        # carry on from what the kernel holds, so that a tie is not counted again
        for w, e, s in zip(want, entries_of(c), (c.k_scale, c.v_scale)):
            w.entries, w.quotients, w.scale = e, e.copy(), f64(s)
        length += n
    for name, kv in zip("kv", c.read(dev(np.arange(7 * bs)), dtype=DT[dtype])):
        w = want["kv".index(name)].values().transpose(0, 2, 1, 3).reshape(7 * bs, H, D)
        got, live = f64(kv), np.isfinite(w)
        assert (np.abs(got - w)[live] <= (U[dtype] + 2.0 ** -23) * np.abs(w)[live] + 1e-7 * (dtype == "fp16")).all()
        assert np.isnan(got[~live]).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("fmt,bs,H,D,major", CACHES)
@pytest.mark.parametrize("part,inter", [(1, False), (2, True)])
def test_append_with_positions(at, fmt, bs, H, D, major, dtype, part, inter):
    c = at.KVCache(6, bs, H, D, fmt, token_major=major)
    fill(c, 2)
    want = [oa.Cache(e, f64(s), fmt) for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
    r = rope(at, D, D // part, inter, "none")
    f, m = oa.frequencies(r.rotary_dim)
    # three requests at once: one starts, one goes on inside a block, one crosses a block; one token has no slot
    slots = np.concatenate([np.arange(3), 2 * bs + np.arange(5, 9), [-1], 3 * bs + np.arange(bs - 2, bs), 5 * bs + np.arange(4)]).astype(np.int32)
    pos = np.concatenate([np.arange(3), np.arange(5, 9), [77], bs - 2 + np.arange(6)]) + 3000
    n = len(slots)
    k, v, q = normal(1, (n, H, D), dtype, 1.0), normal(2, (n, H, D), dtype), normal(3, (n, 2 * H, D), dtype)
    qc = q.clone()
    qo = c.append(k, v, dev(slots), rotary=r, positions=dev(pos), q=q)
    check_turn(qo, qc, pos, r, dtype)
    assert torch.equal(q, qc)
    want[0].append(oa.rotary(f64(k), pos, f, m, r.rotary_dim, inter), slots)
    want[1].append(f64(v), slots)
    check_cache(c, want, fmt, True)
    # in place, and the same cache without any q
    before = [t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)]
    assert c.append(k, v, dev(slots), rotary=r, positions=dev(pos), q=q, q_out=q) is q and torch.equal(q, qo)
    assert c.append(k, v, dev(slots), rotary=r, positions=dev(pos)) is None
    for a, b in zip(before, (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)):
        assert torch.equal(a, b)                          # the same tokens again change nothing


@pytest.mark.parametrize("fmt,bs,H,D,T,dtype", [("int8", 128, 2, 128, 300, "fp16"), ("e4m3", 256, 1, 256, 601, "bf16"), ("int8", 48, 3, 256, 130, "fp32"), ("e4m3", 16, 1, 64, 4100, "fp16"),
                                                 ("int8", 1024, 1, 64, 1500, "fp16")])
@pytest.mark.parametrize("turn", [False, True])
def test_append_prompts_in_wide_blocks(at, fmt, bs, H, D, T, dtype, turn):
    """Runs of more tokens than a pass holds, and enough tokens for every way a launch is cut; then one token more."""
    nb = -(-(T + 1) // bs) + 1
    c = at.KVCache(nb, bs, H, D, fmt)
    fill(c, 5)
    want = [oa.Cache(e, f64(s), fmt) for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
    r = rope(at, D, D, False, "none") if turn else None
    f, m = oa.frequencies(D)
    order = np.random.default_rng(T).permutation(nb)
    q = normal(7, (T, 2, D), dtype) if turn else None
    for lo, hi in ((0, T), (T, T + 1)):
        pos = np.arange(lo, hi)
        slots = (order[pos // bs] * bs + pos % bs).astype(np.int32)
        k, v = normal(3 + lo, (hi - lo, H, D), dtype), normal(4 + lo, (hi - lo, H, D), dtype, 5.0)
        out = c.append(k, v, dev(slots), rotary=r, positions=dev(pos) if turn else None, q=q[:hi - lo] if turn else None)
        if turn:
            check_turn(out, q[:hi - lo], pos, r, dtype)
        want[0].append(oa.rotary(f64(k), pos, f, m, D, False) if turn else f64(k), slots)
        want[1].append(f64(v), slots)
        check_cache(c, want, fmt, turn)
        for w, e, s in zip(want, entries_of(c), (c.k_scale, c.v_scale)):
            w.entries, w.quotients, w.scale = e, e.copy(), f64(s)


def test_append_equals_turning_first_in_fp32(at):
    a, b = (at.KVCache(5, 16, 2, 128, "int8") for _ in range(2))
    r = rope(at, 128, 128, False, "none")
    k, v, pos = normal(1, (40, 2, 128), "fp32"), normal(2, (40, 2, 128), "fp32"), dev(np.arange(40) + 100)
    a.append(k, v, dev(np.arange(40)), rotary=r, positions=pos)
    b.append(r.apply(k, None, pos)[0], v, dev(np.arange(40)))
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.k_scale, b.k_scale)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_special_values(at, fmt):
    bs, H, D = 16, 4, 64
    c = at.KVCache(4, bs, H, D, fmt)
    fill(c, 3)
    keep = [t.clone() for t in (c.k.view(torch.uint8), c.k_scale)]
    k, v = normal(1, (6, H, D), "fp32"), normal(2, (6, H, D), "fp32")
    k[:, 0] = 0.0                                         # a block of zeros
    k[:, 1] *= 1e-33                                      # a scale below 2^-100
    k[2, 2, 5] = float("inf")
    k[3, 3, 7] = float("nan")
    slots = dev([-1, 4 * bs, 16, 17, 18, 2 ** 31 - 1])    # two outside the cache, three stored, one outside
    c.append(k, v, slots)
    got, _ = c.read(dev([16, 17, 18, -1, 4 * bs]), dtype=torch.float32)
    assert (got[:3, :2] == 0).all() and torch.isnan(got[:3, 2:]).all() and (got[3:] == 0).all()
    assert (c.k_scale[1, :2] == 0).all() and torch.isnan(c.k_scale[1, 2:]).all()
    for i in (0, 2, 3):
        assert torch.equal(c.k.view(torch.uint8)[i], keep[0][i]) and torch.equal(c.k_scale[i], keep[1][i])
    # NaN stays until the block starts anew
    c.append(normal(3, (1, H, D), "fp32"), v[:1], dev([19]))
    assert torch.isnan(c.k_scale[1, 2:]).all() and (c.k_scale[1, :2] > 0).all()
    got, _ = c.read(dev([16, 17, 18]), dtype=torch.float32)
    assert (got[:, :2] == 0).all()
    c.append(normal(3, (1, H, D), "fp32"), v[:1], dev([16]))
    assert torch.isfinite(c.k_scale[1]).all()


def test_append_strided_unaligned_and_empty(at):
    for shift in (0, 1, 4):
        rows = normal(1, (20, 3 * 2 * 64 + 9), "fp16")
        k = rows[:, shift:shift + 128].unflatten(1, (2, 64))
        v = rows[:, shift + 128:shift + 256].unflatten(1, (2, 64))
        a, b = at.KVCache(3, 16, 2, 64), at.KVCache(3, 16, 2, 64, token_major=True)
        a.append(k, v, dev(np.arange(20)))
        b.append(k.contiguous(), v.contiguous(), dev(np.arange(20)))
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.v_scale, b.v_scale)
        a.append(k[:0], v[:0], dev(np.zeros(0)))
        assert a.read(dev(np.zeros(0)))[0].shape == (0, 2, 64)


# ---- attention ----------------------------------------------------------------------------------------------------

def setup(at, fmt, bs, H, D, lengths, seed, major=False, spread=1.0):
    need = [-(-max(0, n) // bs) for n in lengths]
    width = max(max(need), 1) + 1
    rng = np.random.default_rng(seed)
    nb = sum(need) + 3
    ids = rng.permutation(nb)
    table = rng.integers(-5, nb + 5, (len(lengths), width)).astype(np.int32)      # entries past a length are not read
    i = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[i:i + n]
        i += n
    c = at.KVCache(nb, bs, H, D, fmt, token_major=major)
    fill(c, seed)
    bad = torch.isnan(c.k.to(torch.float32)) if fmt == "e4m3" else None
    if fmt == "e4m3":                                     # NaN patterns stay only past the lengths
        mask = torch.ones((nb, bs), dtype=torch.bool)
        for r, n in enumerate(lengths):
            for j in range(max(0, n)):
                mask[table[r, j // bs], j % bs] = False
        mask = mask[:, None, :, None].cuda()
        for x in (c.k, c.v):
            raw = x.view(torch.uint8)
            raw.copy_(torch.where(((raw & 127) == 127) & ~mask, torch.zeros_like(raw), raw))
        c.k_scale *= 127 / 448 * 4
        c.v_scale *= 127 / 448 * 4
    c.k_scale *= spread
    return c, table


def check_attend(c, q, table, lengths, starts, scale, out, lse, dtype):
    k, v = (e * f64(s)[:, :, None, None] for e, s in zip(entries_of(c), (c.k_scale, c.v_scale)))
    want, wl, mean, size = oa.attend(f64(q), k, v, table, lengths, starts, scale)
    D, L = q.shape[2], max(max(lengths), 1)
    S = size[:, :, None]
    bound = U[dtype] * np.abs(want) + (2.0 ** -11 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * mean + 1e-7 * (dtype == "fp16")
    err = np.abs(f64(out) - want)
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-30)).max()
    if lse is not None:
        got = f64(lse)
        assert np.array_equal(np.isinf(got), np.isinf(wl))
        ok = np.isfinite(wl)
        assert (np.abs(got[ok] - wl[ok]) <= (D + 4) * 2.0 ** -24 * size[ok] + 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -23 * np.abs(wl[ok])).all()


SHAPES = [(4, 4, 128), (8, 1, 128), (16, 2, 64), (6, 2, 256), (14, 2, 64), (40, 1, 128), (3, 3, 64), (12, 1, 256)]


@pytest.mark.parametrize("fmt,dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("bs", [16, 48, 128])
@pytest.mark.parametrize("Hq,H,D", SHAPES)
def test_attend_one_token_each(at, Hq, H, D, bs, fmt, dtype):
    lengths = [1, 0, 17, 16, 300, 2, 129, 64, -3, 63]
    c, table = setup(at, fmt, bs, H, D, lengths, Hq + bs)
    q = normal(7, (len(lengths), Hq, D), dtype)
    ws = c.workspace(len(lengths), len(lengths), Hq)
    out, lse = c.attend(q, dev(table), dev(lengths), ws, with_lse=True)
    check_attend(c, q, table, lengths, np.arange(len(lengths) + 1), D ** -0.5, out, lse, dtype)
    assert (out[1] == 0).all() and torch.isinf(lse[8]).all()
    out2 = c.attend(q, dev(table), dev(lengths), ws)
    assert torch.equal(out, out2)


@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("Hq,H,D", SHAPES)
def test_attend_several_tokens_each(at, Hq, H, D, fmt, dtype):
    # drafted tokens, a prompt's first and later chunk, no new token, more new tokens than cached ones (rows that see nothing)
    new, lengths = [1, 5, 0, 33, 3, 70], [40, 5, 77, 200, 2, 70]
    c, table = setup(at, fmt, 16, H, D, lengths, 3 * Hq)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = normal(8, (sum(new), Hq, D), dtype)
    ws = c.workspace(len(lengths), sum(new), Hq)
    out, lse = c.attend(q, dev(table), dev(lengths), ws, query_start=dev(starts), with_lse=True)
    check_attend(c, q, table, lengths, starts, D ** -0.5, out, lse, dtype)
    assert (out[39] == 0).all() and torch.isinf(lse[39]).all()          # the first of three tokens of a request of two


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,length", [(8, 1, 128, 20001), (16, 2, 64, 9999), (4, 4, 128, 5003), (6, 2, 256, 4097)])
def test_attend_long_context_split_over_the_device(at, Hq, H, D, length, fmt):
    lengths = [length, 3, length // 7]
    c, table = setup(at, fmt, 16, H, D, lengths, 5)
    q = normal(9, (3, Hq, D), "fp16")
    ws = c.workspace(3, 3, Hq)
    outs = [c.attend(q, dev(table), dev(lengths), ws, with_lse=True) for _ in range(3)]
    check_attend(c, q, table, lengths, [0, 1, 2, 3], D ** -0.5, *outs[0], "fp16")
    for o in outs[1:]:
        assert torch.equal(o[0], outs[0][0]) and torch.equal(o[1], outs[0][1])
    # a workspace serves smaller calls after larger ones
    out = c.attend(q[1:2], dev(table[1:2]), dev(lengths[1:2]), ws)
    check_attend(c, q[1:2], table[1:2], lengths[1:2], [0, 1], D ** -0.5, out, None, "fp16")


@pytest.mark.parametrize("Hq,H,D,new", [(8, 1, 128, 5), (40, 1, 128, 1), (16, 2, 128, 2), (9, 1, 128, 4), (7, 1, 64, 5), (6, 2, 256, 4)])
def test_attend_row_tiles(at, Hq, H, D, new):
    """33 to 40, 9 to 16 and just above as many query rows of a key head."""
    lengths = [61, 300, 5]
    c, table = setup(at, "int8", 16, H, D, lengths, Hq + new)
    q = normal(31, (3 * new, Hq, D), "bf16")
    starts = np.arange(4) * new
    out, lse = c.attend(q, dev(table), dev(lengths), c.workspace(3, 3 * new, Hq), query_start=dev(starts), with_lse=True)
    check_attend(c, q, table, lengths, starts, D ** -0.5, out, lse, "bf16")


def test_attend_shares_that_are_drawn(at):
    """Long enough that the ends of the ranges are drawn: against 64 bits on the GPU, and twice the same."""
    B, Hq, H, D, bs, fmt = 7, 8, 8, 64, 128, "int8"
    lengths = [90001, 3, 89000, 90500, 1, 89999, 88000]        # 95 units for each of 296 CTAs: nine of them are drawn
    c, table = setup(at, fmt, bs, H, D, lengths, 41)
    q = normal(42, (B, Hq, D), "fp16")
    ws = c.workspace(B, B, Hq)
    first = c.attend(q, dev(table), dev(lengths), ws, with_lse=True)
    for _ in range(3):
        again = c.attend(q, dev(table), dev(lengths), ws, with_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    for r, L in enumerate(lengths):
        ids = dev(table[r, :-(-L // bs)]).long()
        k, v = (x[ids].double() * s[ids].double()[..., None, None] for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        k, v = (x.transpose(0, 1).reshape(H, -1, D)[:, :L] for x in (k, v))
        x = torch.einsum("hd,hld->hl", q[r].double(), k) * D ** -0.5
        p = torch.softmax(x, -1)
        want, mean = torch.einsum("hl,hld->hd", p, v), torch.einsum("hl,hld->hd", p, v.abs())
        S = (q[r].double().abs()[:, None, :] * k.abs()).sum(-1).amax(-1)[:, None] * D ** -0.5
        bound = U["fp16"] * want.abs() + (2.0 ** -11 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * S + L * 2.0 ** -23) * mean + 1e-7
        assert ((first[0][r].double() - want).abs() <= bound).all()
        lse = torch.logsumexp(x, -1)
        assert ((first[1][r].double() - lse).abs() <= (D + 4) * 2.0 ** -24 * S[:, 0] + 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -23 * lse.abs()).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("order", [1, -1])
def test_attend_scores_that_grow_and_scales_that_differ(at, fmt, order):
    """A running maximum that moves all the time, values whose scales span many powers of two, one block of zeros."""
    Hq, H, D, L = 8, 2, 128, 700
    c, table = setup(at, fmt, 16, H, D, [L], 11)
    n = -(-L // 16)
    ramp = sorted(torch.linspace(0.001, 0.08, n).tolist(), reverse=order < 0)
    for i in range(n):
        c.k_scale[table[0, i]] = float(ramp[i])
        c.v_scale[table[0, i]] = 2.0 ** float((i * 7 % 40) - 30)
    c.v_scale[table[0, n // 2]] = 0.0
    for spread in (0.1, 1.0):
        q = normal(12, (1, Hq, D), "fp16", spread)
        out, lse = c.attend(q, dev(table), dev([L]), c.workspace(1, 1, Hq), with_lse=True)
        check_attend(c, q, table, [L], [0, 1], D ** -0.5, out, lse, "fp16")


def test_attend_extreme_queries_scales_and_strides(at):
    Hq, H, D = 16, 2, 128
    lengths = [37, 300]
    c, table = setup(at, "int8", 32, H, D, lengths, 13, major=True)
    rows = normal(14, (2, (Hq + 2 * H) * D), "bf16")
    q = rows[:, :Hq * D].unflatten(1, (Hq, D))                # the q part of a fused projection's rows
    out = torch.full((Hq, 2, D), float("nan"), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    wide = dev(np.pad(table, ((0, 0), (0, 5)), constant_values=-9))[:, :table.shape[1]]
    ws = c.workspace(2, 2, Hq)
    assert c.attend(q, wide, dev(lengths), ws, out=out, scale=0.3) is out
    check_attend(c, q, table, lengths, [0, 1, 2], 0.3, out, None, "bf16")
    for size, scale in [(1e5, 1e-6), (1e-9, 1e8), (3e30, 1e-32), (1e-30, 1e29), (1.0, 0.0), (1.0, -0.1)]:       # beyond fp16's range
        big = (normal(15, (2, Hq, D), "fp32") * size).to(torch.bfloat16)
        out, lse = c.attend(big, wide, dev(lengths), ws, scale=scale, with_lse=True)
        check_attend(c, big, table, lengths, [0, 1, 2], scale, out, lse, "bf16")
    zero = torch.zeros_like(q)
    out, lse = c.attend(zero, wide, dev(lengths), ws, with_lse=True)
    check_attend(c, zero, table, lengths, [0, 1, 2], D ** -0.5, out, lse, "bf16")


def test_attend_bad_table_entries_and_lengths_are_masked(at):
    Hq, H, D, bs = 8, 2, 128, 16
    lengths = [100, 90, 40]
    c, table = setup(at, "e4m3", bs, H, D, lengths, 17)
    table = table[:, :7].copy()
    table[0, 2], table[0, 5], table[1, :6], table[2, 0] = -1, c.num_blocks, 2 ** 31 - 1, -2 ** 31
    given = [10 ** 9, 90, 40]                                 # cut to the table's width: 7 blocks
    table[0, 6] = table[0, 0]
    c.k.view(torch.uint8)[c.k.view(torch.uint8) % 128 == 127] = 0
    c.v.view(torch.uint8)[c.v.view(torch.uint8) % 128 == 127] = 0
    q = normal(18, (3, Hq, D), "fp16")
    out, lse = c.attend(q, dev(table), dev(given), c.workspace(3, 3, Hq), with_lse=True)
    check_attend(c, q, table, [112, 90, 40], [0, 1, 2, 3], D ** -0.5, out, lse, "fp16")
    assert (out[1] == 0).all() and torch.isinf(lse[1]).all()


def test_attend_nan_scale_shows_and_stays_in_its_head(at):
    c, table = setup(at, "int8", 16, 2, 64, [50], 19)
    q = normal(20, (1, 4, 64), "fp16")
    c.v_scale[table[0, 1], 0] = float("nan")
    out = c.attend(q, dev(table), dev([50]), c.workspace(1, 1, 4))
    assert torch.isnan(out[0, :2]).all() and torch.isfinite(out[0, 2:]).all()
    c.v_scale[table[0, 1], 0] = 0.01
    c.k_scale[table[0, 1], 1] = float("nan")
    out = c.attend(q, dev(table), dev([50]), c.workspace(1, 1, 4))
    assert torch.isfinite(out[0, :2]).all() and torch.isnan(out[0, 2:]).all()


def test_attend_cache_past_four_gigabytes(at):
    """Entries beyond 2^32 bytes: a pool whose blocks lie far apart."""
    H, D, bs, nb = 1, 64, 16, 70
    stride = 1 << 26
    free = torch.cuda.mem_get_info()[0]
    assert free > 12 << 30
    big = [torch.empty(stride * nb, dtype=torch.int8, device="cuda") for _ in range(2)]
    view = [b.as_strided((nb, H, bs, D), (stride, bs * D, D, 1)) for b in big]
    sc = [torch.zeros((nb, H), device="cuda") for _ in range(2)]
    c = at.KVCache.wrap(*view, *sc)
    fill(c, 21)
    L = nb * bs - 5
    table = np.random.default_rng(22).permutation(nb)[None].astype(np.int32)
    q = normal(23, (1, 4, D), "fp16")
    out, lse = c.attend(q, dev(table), dev([L]), c.workspace(1, 1, 4), with_lse=True)
    check_attend(c, q, table, [L], [0, 1], D ** -0.5, out, lse, "fp16")
    k = normal(24, (1, H, D), "fp16")
    c.append(k, k, dev([table[0].tolist().index(0) * 0 + (nb - 1) * bs]))
    got = c.read(dev([(nb - 1) * bs]))[0]
    assert (f64(got) - f64(k)).__abs__().max() <= np.abs(f64(k)).max() / 127
    del big, view, c
    torch.cuda.empty_cache()


# ---- block tables -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,width,nb,bs,most", [(1, 4, 5, 16, 20), (9, 6, 40, 16, 45), (70, 9, 300, 32, 300), (1500, 5, 3000, 16, 60), (8192, 3, 9000, 16, 30)])
def test_advance(at, B, width, nb, bs, most):
    rng = np.random.default_rng(B)
    table, free = np.full((B, width), -1, np.int32), rng.permutation(nb).astype(np.int32)
    free = np.concatenate([free, np.full(7, -1, np.int32)])
    t = at.BlockTables(dev(table), dev(free), bs)
    lengths, nf = dev(np.zeros(B)), dev([nb])
    for step in range(6):
        new = rng.integers(-most, most + 1, B) if step else rng.integers(0, most, B)
        new[rng.random(B) < 0.3] = 1
        if step == 4:
            new[:] = -10 ** 9                                 # everybody leaves
        T = int(new.clip(0).sum())
        cap = T + (5 if step % 2 else 0) - (T // 3 if step == 5 else 0)
        got = t.advance(lengths, dev(new), nf, cap)
        want = oa.advance(lengths.cpu().numpy(), new, table, free, int(nf[0]), bs, cap)
        for name in ("lengths", "granted", "query_start", "positions", "slots", "requests"):
            assert np.array_equal(getattr(got, name).cpu().numpy(), want[name]), (step, name)
        assert int(got.num_free[0]) == want["num_free"]
        assert np.array_equal(t.table.cpu().numpy(), table) and np.array_equal(t.free.cpu().numpy(), free)
        lengths, nf = got.lengths, got.num_free
    if B < 100:
        held = [b for i in range(B) for b in table[i, :-(-int(lengths[i]) // bs)]]
        assert sorted(held + list(free[:int(nf[0])])) == list(range(nb))


def test_advance_decode_steps_and_no_tokens(at):
    B, bs = 5, 16
    t = at.BlockTables.empty(B, 4, 12, bs)
    lengths, nf = dev([0] * B), dev([12])
    s = t.advance(lengths, dev([15, 16, 17, 0, 31]), nf, 79)
    assert s.lengths.tolist() == [15, 16, 17, 0, 31] and s.num_free.tolist() == [6] and s.query_start.tolist() == [0, 15, 31, 48, 48, 79]
    s = t.advance(s.lengths, dev([0] * B), s.num_free, 0)
    assert s.lengths.tolist() == [15, 16, 17, 0, 31] and s.slots.numel() == 0
    for _ in range(20):
        s = t.advance(s.lengths, dev([1] * B), s.num_free, B)
    # 12 blocks: some requests ran into the end of the pool and stayed where they were
    assert int(s.num_free[0]) == 0 and (s.slots[s.granted == 0] == -1).all() and (s.granted == 0).any()


# ---- streams, graphs, refusals ------------------------------------------------------------------------------------

def test_one_step_on_another_stream_and_in_a_graph(at):
    B, Hq, H, D, bs = 4, 8, 2, 128, 16
    c, tables, r = at.KVCache(64, bs, H, D), at.BlockTables.empty(B, 8, 64, bs), rope(at, D, D, False, "none")
    ws = c.workspace(B, B, Hq)
    q, k, v = normal(1, (B, Hq, D), "fp16"), normal(2, (B, H, D), "fp16"), normal(3, (B, H, D), "fp16")
    ones = dev([1] * B)
    lengths, nf = dev([0] * B), dev([64])
    out = torch.empty_like(q)

    def step():
        s = tables.advance(lengths, ones, nf, B)
        qr = c.append(k, v, s.slots, rotary=r, positions=s.positions, q=q)
        c.attend(qr, tables.table, s.lengths, ws, query_start=s.query_start, out=out)
        lengths.copy_(s.lengths)
        nf.copy_(s.num_free)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(17):
        g.replay()
    torch.cuda.synchronize()
    assert lengths.tolist() == [20] * B and int(nf[0]) == 64 - 2 * B
    check_attend(c, r.apply(q, None, dev([19] * B))[0], tables.table.cpu().numpy(), [20] * B, np.arange(B + 1), D ** -0.5, out, None, "fp16")


def test_refused_tensors(at):
    with pytest.raises(ValueError):
        at.Rotary(128, scaling="other")
    with pytest.raises(Exception, match="out of range"):
        at.Rotary(128, 130)
    with pytest.raises(Exception, match="unsupported"):
        at.KVCache(4, 16, 2, 96)
    with pytest.raises(ValueError):
        at.KVCache(4, 16, 2, 64, fmt="fp4")
    c, r = at.KVCache(4, 16, 2, 64), at.Rotary(64)
    x, s = normal(1, (3, 2, 64), "fp16"), dev([0, 1, 2])
    for bad in [lambda: c.append(x, x[:2], s), lambda: c.append(x, x, s[:2]), lambda: c.append(x, x, s.long()), lambda: c.append(x, x, s, rotary=r),
                lambda: c.append(x, x, s, q=x), lambda: c.append(x[:, :1], x, s), lambda: c.append(x[..., ::2], x, s), lambda: r.apply(x[..., :32], None, s),
                lambda: c.attend(x, s[None].long(), s[:1], c.workspace(1, 1, 2)), lambda: c.workspace(1, 1, 3),
                lambda: at.KVCache.wrap(c.k, c.v[:, :1], c.k_scale, c.v_scale), lambda: at.KVCache.wrap(c.k, c.v, c.k_scale[:, :1], c.v_scale),
                lambda: at.BlockTables(s[None].float(), s, 16)]:
        with pytest.raises((ValueError, TypeError)):
            bad()
    for bad in [lambda: c.append(x, x.float(), s), lambda: c.append(x.double(), x.double(), s), lambda: c.attend(x.float(), s[None], s[:1], None),
                lambda: c.read(s, dtype=torch.int8)]:
        with pytest.raises(TypeError):
            bad()
    from paper_2608_15602_b200.fluxbin import FluxBinError
    table = dev([[0], [1], [2]])
    with pytest.raises(FluxBinError, match="range"):
        c.attend(x, table[:2], s[:2], c.workspace(3, 3, 2))              # three tokens, two requests, no query_start
