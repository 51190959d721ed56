"""A NaN or infinity among a later token's values stays with the rows that see that token.

Rows that do not see it have to equal the same rows of a call over a cache without it, bit for bit (the same lengths, so the
same sums); rows that see it show it, in every element where the scale is NaN and in its own element where only an entry is."""
import numpy as np
import pytest

from test_gpu_attention import at, dev, f64, normal, setup  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROWS = [(8, 1, 128), (4, 4, 128), (3, 1, 128), (4, 1, 64), (16, 2, 64), (4, 2, 256), (2, 1, 256)]        # with 5 tokens: tiles of 8, 16 and 40 rows


B = 600                                                   # requests over the same blocks: most of a request is one CTA's work


def call(c, q, table, L, new, **kw):
    """The same five tokens asked by B requests."""
    n = q.shape[0]
    ws = c.workspace(B, B * n, q.shape[1])
    out, lse = c.attend(q.repeat(B, 1, 1), dev(np.repeat(table, B, 0)), dev([L] * B), ws, query_start=dev(np.arange(B + 1) * new), with_lse=True, **kw)
    return out.unflatten(0, (B, n)), lse.unflatten(0, (B, n))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D", ROWS)
@pytest.mark.parametrize("last", [0, 2])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_draft_that_opens_a_block_with_a_nan(at, Hq, H, D, last, value, fmt):  # noqa: F811
    bs, new = 16, 5
    L = 16 * bs + 1 + last                                # the last 1 or 3 of five tokens lie in a block of their own
    k, v = normal(1, (L, H, D), "fp16"), normal(2, (L, H, D), "fp16")
    bad = v.clone()
    bad[16 * bs, 0, 7] = value
    q = normal(3, (new, Hq, D), "fp16")
    outs = []
    for values in (v, bad):
        c = at.KVCache(17, bs, H, D, fmt)
        c.append(k, values, dev(np.arange(L)))
        assert torch.isnan(c.v_scale[16, 0]) == (values is bad)
        outs.append(call(c, q, np.arange(17)[None], L, new))
    (out, lse), (got, got_lse) = outs
    see = torch.arange(new) >= 4 - last                   # these see the first token of the last block
    G = Hq // H
    assert torch.equal(got[:, ~see], out[:, ~see]) and torch.equal(got[:, :, G:], out[:, :, G:]) and torch.equal(got_lse, lse)
    assert torch.isnan(got[:, see][:, :, :G]).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("Hq,H,D", ROWS)
def test_a_nan_entry_under_a_finite_scale(at, Hq, H, D):  # noqa: F811
    """A cache that others filled: single e4m3 NaN entries, among the new tokens and among those that all rows see."""
    new, L = 5, 70
    c, table = setup(at, "e4m3", 16, H, D, [L], 5)
    q = normal(4, (new, Hq, D), "bf16")
    for x in (c.k, c.v):                                  # no NaN to begin with
        raw = x.view(torch.uint8)
        raw.copy_(torch.where((raw & 127) == 127, torch.zeros_like(raw), raw))
    for where, sign in [((66, 5), 0x7f), ((68, D - 1), 0xff), ((69, 40), 0x7f), ((20, 33), 0xff)]:
        t, e = where
        raw = c.v.view(torch.uint8)[table[0, t // 16], 0, t % 16]
        keep = raw[e].clone()
        raw[e] = 0
        out = call(c, q, table, L, new)[0]
        raw[e] = sign
        got = call(c, q, table, L, new)[0]
        raw[e] = keep
        nan = torch.isnan(got)
        want = torch.zeros_like(nan)
        want[:, max(0, t - (L - new)):, :Hq // H, e] = True   # rows from the token itself on
        assert torch.equal(nan, want), where
        assert torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, out))


def test_a_nan_key_scale_of_a_later_draft(at):  # noqa: F811
    Hq, H, D, new, L = 8, 1, 128, 5, 65
    c, table = setup(at, "int8", 16, H, D, [L], 6)
    q = normal(5, (new, Hq, D), "fp16")
    out, lse = call(c, q, table, L, new)
    c.k_scale[table[0, 4]] = float("nan")
    got, got_lse = call(c, q, table, L, new)
    assert torch.equal(got[:, :4], out[:, :4]) and torch.equal(got_lse[:, :4], lse[:, :4]) and torch.isnan(got[:, 4]).all() and torch.isnan(got_lse[:, 4]).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_an_infinite_scale_stays_with_the_rows_that_see_it(at, fmt):  # noqa: F811
    Hq, H, D, new, L = 8, 1, 128, 2, 257
    c, table = setup(at, fmt, 16, H, D, [L], 8)
    q = normal(6, (new, Hq, D), "fp16")
    out = call(c, q, table, L, new)[0]
    c.v_scale[table[0, 16]] = float("inf")
    got = call(c, q, table, L, new)[0]
    assert torch.equal(got[:, 0], out[:, 0]) and not torch.isfinite(got[:, 1]).any()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_nan_is_seen_however_small_its_probability(at, fmt):  # noqa: F811
    """Also where the token's probability underflows in its warp, its CTA or its part of a cut request."""
    Hq, H, D, L = 8, 1, 128, 40
    c, table = setup(at, fmt, 16, H, D, [L], 7)
    c.k.copy_(torch.zeros(c.k.shape, device="cuda").to(c.k.dtype))
    c.k_scale.fill_(1.0)
    c.k[table[0, 2], :, :, 0] = torch.tensor(-100.0, device="cuda").to(c.k.dtype)
    c.k_scale[table[0, 2]] = 10.0
    c.v_scale[table[0, 2]] = float("nan")
    q = torch.zeros((1, Hq, D), dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    out = c.attend(q, dev(table), dev([L]), c.workspace(1, 1, Hq), scale=1.0)
    assert torch.isnan(out).all() and torch.isnan(call(c, q, table, L, 1, scale=1.0)[0]).all()
