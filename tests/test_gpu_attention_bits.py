"""What attention over the 8-bit cache holds in how many bits, and over what range, against 64 bits.

Bounds.  Notation of test_gpu_attention.py: u the unit roundoff of the result's type, A the mean of |v| under the probabilities,
S the largest scale * sum |q k| of the row, L its length.  A probability (times its block's value scale) enters the product as
two bf16 numbers: the second rounds what the first left, at most 2^-8 of it, to 2^-8 again, so it is off by 2^-16 of itself.
Everything else is as there, so
    |error| <= u |out| + (2^-16 + 2^-19 + (2 D + 8) 2^-24 S + L 2^-23) A
and this holds however far below the largest one the probabilities are that decide the result, and however far the value
scales of a request's blocks differ, within fp32's range (fp16 results: the type's smallest step, 2^-24, besides).
"""
import numpy as np
import pytest

from oracle import attention as oa
from test_gpu_attention import U, at, dev, entries_of, f64, normal, setup  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROWS = [(8, 1, 128, 1), (16, 1, 128, 1), (8, 1, 128, 5), (4, 4, 64, 1), (9, 1, 64, 1), (6, 2, 256, 1), (12, 1, 256, 1)]    # q heads, key heads, dim, tokens


def check(c, q, table, lengths, starts, scale, out, dtype):
    k, v = (e * f64(s)[:, :, None, None] for e, s in zip(entries_of(c), (c.k_scale, c.v_scale)))
    want, _, mean, size = oa.attend(f64(q), k, v, table, lengths, starts, scale)
    D, L = q.shape[2], max(lengths)
    bound = U[dtype] * np.abs(want) + (2.0 ** -16 + 2.0 ** -19 + (2 * D + 8) * 2.0 ** -24 * size[:, :, None] + L * 2.0 ** -23) * mean + 2.0 ** -24 * (dtype == "fp16")
    err = np.abs(f64(out) - want)
    assert (err <= bound).all(), (err / np.maximum(bound, 1e-300)).max()
    return want


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("Hq,H,D,new", ROWS)
def test_probabilities_carry_sixteen_bits(at, Hq, H, D, new, fmt):  # noqa: F811
    lengths = [40, 25, 300]
    c, table = setup(at, fmt, 16, H, D, lengths, 3)
    q = normal(51, (3 * new, Hq, D), "fp16", 0.3)
    starts = np.arange(4) * new
    out = c.attend(q, dev(table), dev(lengths), c.workspace(3, 3 * new, Hq), query_start=dev(starts))
    check(c, q, table, lengths, starts, D ** -0.5, out, "fp16")


def flat(at, fmt, H, D, bs, L, seed):  # noqa: F811
    """A request of L tokens: keys 0, values random at scale 2^-7 (so of size 1 with int8)."""
    nb = -(-L // bs)
    c = at.KVCache(nb, bs, H, D, fmt)
    rng = np.random.default_rng(seed)
    values = torch.from_numpy(rng.integers(-100, 101, c.v.shape).astype(np.float32)).cuda()
    c.v.copy_(values.to(c.v.dtype))
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(2.0 ** -7)
    return c, rng.permutation(nb)[None].astype(np.int32)


def score(c, block, token, value):
    """Makes the score of a cached token `value` for a query that is 1 in its first element and 0 else, with scale 1."""
    c.k_scale[block] = abs(value) / 64.0
    c.k[block, :, :, 0] = torch.zeros((), device="cuda").to(c.k.dtype)
    c.k[block, :, token, 0] = torch.tensor(64.0 if value > 0 else -64.0, device="cuda").to(c.k.dtype)


def unit_queries(n, Hq, D, dtype):
    q = torch.zeros((n, Hq, D), dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    return q


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("above", [21.0, 23.0, 30.0, 60.0])
@pytest.mark.parametrize("Hq,H,D,new", ROWS)
def test_one_probability_dominates_and_its_value_is_zero(at, Hq, H, D, new, above, fmt):  # noqa: F811
    L = 2000
    c, table = flat(at, fmt, H, D, 16, L, 7)
    first = int(table[0, 3])
    score(c, first, 5, above)
    c.v[first, :, 5] = torch.zeros((), device="cuda").to(c.v.dtype)
    q = unit_queries(new, Hq, D, torch.bfloat16)
    out = c.attend(q, dev(table), dev([L]), c.workspace(1, new, Hq), query_start=dev([0, new]), scale=1.0)
    want = check(c, q, table, [L], [0, new], 1.0, out, "bf16")
    assert (want != 0).mean() > 0.9


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("ratio", [2.0 ** 25, 2.0 ** 33, 2.0 ** 60])
@pytest.mark.parametrize("where", [0, 60])
@pytest.mark.parametrize("Hq,H,D,new", ROWS)
def test_a_block_of_large_values_and_small_probabilities(at, Hq, H, D, new, where, ratio, fmt):  # noqa: F811
    L = 1000
    c, table = flat(at, fmt, H, D, 16, L, 8)
    big = int(table[0, where])
    c.k_scale[big] = 1.5                                  # every token of the block 96 below the others
    c.k[big, :, :, 0] = torch.tensor(-64.0, device="cuda").to(c.k.dtype)
    c.v_scale[big] = 2.0 ** -7 * ratio
    for dtype in ("fp16", "bf16"):
        q = unit_queries(new, Hq, D, torch.float16 if dtype == "fp16" else torch.bfloat16)
        out = c.attend(q, dev(table), dev([L]), c.workspace(1, new, Hq), query_start=dev([0, new]), scale=1.0)
        check(c, q, table, [L], [0, new], 1.0, out, dtype)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_block_of_large_values_that_only_the_last_token_sees(at, fmt):  # noqa: F811
    Hq, H, D, L = 8, 1, 128, 33
    c, table = flat(at, fmt, H, D, 16, L, 9)
    c.v_scale[int(table[0, 2])] = 2.0 ** 40
    q = unit_queries(5, Hq, D, torch.bfloat16)
    out = c.attend(q, dev(table), dev([L]), c.workspace(1, 5, Hq), query_start=dev([0, 5]), scale=1.0)
    check(c, q, table, [L], [0, 5], 1.0, out, "bf16")


def test_the_smallest_e4m3_entries(at):  # noqa: F811
    """Entries below the format's normal range only, keys and values."""
    Hq, H, D, L = 8, 2, 128, 100
    c, table = flat(at, "e4m3", H, D, 16, L, 10)
    rng = np.random.default_rng(11)
    for x in (c.k, c.v):
        x.view(torch.uint8).copy_(torch.from_numpy((rng.integers(0, 8, x.shape) | rng.integers(0, 2, x.shape) << 7).astype(np.uint8)))
    c.k_scale.fill_(60.0)
    c.v_scale.fill_(80.0)
    q = normal(52, (1, Hq, D), "fp16")
    out = c.attend(q, dev(table), dev([L]), c.workspace(1, 1, Hq))
    check(c, q, table, [L], [0, 1], D ** -0.5, out, "fp16")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L", [20, 3000])
@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** 126, 2.0 ** -80])
@pytest.mark.parametrize("Hq,H,D,new", ROWS)
def test_values_near_the_ends_of_the_range(at, Hq, H, D, new, L, size, fmt):  # noqa: F811
    """A weighted mean is no larger than its values, so bf16 holds it whatever the sums on the way are."""
    c, table = flat(at, fmt, H, D, 16, L, 12)
    c.v_scale.fill_(size / 128)                           # entries up to 100
    c.k_scale.fill_(0.01)
    rng = np.random.default_rng(13)
    c.k.copy_(torch.from_numpy(rng.integers(-100, 101, c.k.shape).astype(np.float32)).cuda().to(c.k.dtype))
    q = normal(53, (new, Hq, D), "bf16")
    out = c.attend(q, dev(table), dev([L]), c.workspace(1, new, Hq), query_start=dev([0, new]))
    check(c, q, table, [L], [0, new], D ** -0.5, out, "bf16")
