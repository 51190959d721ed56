"""What the torch wrapper of the attention side hands to the C calls, on CPU tensors: the calls are taken down in the place of
being made (they go by addresses and sizes alone)."""
import ctypes

import pytest

from paper_2608_15602_b200 import build, fluxbin

torch = pytest.importorskip("torch")
build.build()
from paper_2608_15602_b200 import attention as at  # noqa: E402

CALLS = ("rotary_call", "kv_append_call", "kv_read_call", "kv_attend_call", "kv_advance_call")


@pytest.fixture
def calls(monkeypatch):
    """The words of every call that would have been made, by name; device -1 (the CPU's) counts as the current one."""
    got = []
    monkeypatch.setattr(at, "_device", lambda: -1)        # (get_device() of a CPU tensor)
    monkeypatch.setattr(at, "_stream", lambda stream: 0)
    monkeypatch.setattr(at, "_capturing", lambda stream: False, raising=False)
    for name in CALLS:
        monkeypatch.setattr(fluxbin, name, lambda *words, name=name: got.append((name, words)))
    return got


class Scratch:
    tensor, nbytes = torch.empty(1, dtype=torch.uint8), 1


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def attend(table, n=None):
    c = at.KVCache(8, 16, 2, 64, device="cpu")
    n = table.shape[0] if n is None else n
    return c.attend(torch.zeros(n, 4, 64, dtype=torch.float16), table, ints(table.shape[0]), Scratch)


def last_read(words):
    """The last element of the table that the call's kernel may read: (batch - 1) * stride + width - 1."""
    batch, stride, width = words[2], words[11], words[12]
    return (batch - 1) * stride + width - 1


def elements(t):
    return t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()


def test_the_rows_of_a_table_are_read_where_they_lie(calls):
    wide = ints(4, 9)
    for table in (ints(4, 5), wide[:, :5], wide[:, 3:8], ints(1, 5), wide[1:2, :5], ints(5)[None], wide[::2, :5]):
        attend(table)
        words = calls[-1][1]
        assert words[11] == table.stride(0) or table.shape[0] == 1
        assert words[11] >= words[12] and last_read(words) < elements(table)


def test_one_row_for_all_requests(calls):
    """Several samples of one prompt: a row expanded over the batch is read again for each, not past its end."""
    row = ints(1, 5)
    attend(row.expand(4, 5))
    words = calls[-1][1]
    assert words[11] == 0 and last_read(words) < elements(row)
    attend(torch.as_strided(ints(1), (4, 1), (0, 1)))
    assert calls[-1][1][11] == 0


def test_overlapping_rows_are_handed_over_as_they_are(calls):
    """(and refused by the call)"""
    table = torch.as_strided(ints(20), (4, 8), (4, 1))
    attend(table)
    words = calls[-1][1]
    assert words[11] == 4 and last_read(words) < 20


def test_tables_that_advance_writes_have_rows_of_their_own(calls):
    for table in (ints(1, 5).expand(4, 5), torch.as_strided(ints(20), (4, 8), (4, 1))):
        with pytest.raises(ValueError, match="rows"):
            at.BlockTables(table, ints(9), 16)
    for table in (ints(4, 5), ints(4, 9)[:, :5], ints(1, 5), torch.as_strided(ints(5), (1, 5), (0, 1))):
        b = table.shape[0]
        at.BlockTables(table, ints(9), 16).advance(ints(b), ints(b), ints(1), 0)
        batch, stride, width = calls[-1][1][0], *calls[-1][1][6:8]
        assert stride >= width and (batch - 1) * stride + width <= elements(table)


P = 1 << 25


def a_cache(**kw):
    d = dict(num_blocks=8, block_tokens=16, kv_heads=2, head_dim=64, format=0, d_k=1 << 20, d_v=1 << 21, block_stride=2048, head_stride=1024,
             token_stride=64, d_k_scale=1 << 22, d_v_scale=1 << 23)
    d.update(kw)
    return fluxbin.CacheDesc(**d)


def attend_status(cache=None, batch=2, tokens=2, heads=4, q=(256, 64), out=(256, 64), stride=8):
    """5 for what is taken as far as the workspace, which is too small."""
    cache = cache or a_cache()
    return fluxbin.kv_attend_status(ctypes.addressof(cache), 0, batch, tokens, P, heads, *q, None, P, P, stride, 8, 0.125, P, *out, None, P, 16, None)


def test_strides_that_the_call_takes_and_refuses():
    for stride, status in ((0, 5), (8, 5), (9, 5), (7, 3), (1, 3), (-8, 3)):                # 5: taken as far as the workspace, which is too small
        assert attend_status(stride=stride) == status


def test_the_stride_of_an_axis_of_one_is_not_looked_at():
    one = a_cache(kv_heads=1)
    for kw, status in ((dict(q=(260, 64)), 6), (dict(out=(260, 64)), 6), (dict(q=(256, 65)), 6), (dict(out=(256, 65)), 6),
                       (dict(batch=1, tokens=1, q=(261, 64)), 5), (dict(batch=1, tokens=1, out=(0, 64)), 5), (dict(cache=one, heads=1, q=(64, 3)), 5),
                       (dict(cache=one, heads=1, out=(64, 1)), 5), (dict(cache=one, batch=1, tokens=1, heads=1, q=(1, 1), out=(1, 1)), 5)):
        assert attend_status(**kw) == status, kw
    for kw in (dict(num_blocks=1, block_stride=1), dict(kv_heads=1, head_stride=7), dict(num_blocks=1, kv_heads=1, block_stride=3, head_stride=5)):
        assert fluxbin.kv_validate_status(a_cache(**kw)) == 0, kw
    k = torch.zeros(1, 2, 16, 64, dtype=torch.int8)
    v = torch.as_strided(torch.zeros(4096, dtype=torch.int8), (1, 2, 16, 64), (9, 1024, 64, 1))
    s = torch.zeros(1, 2)
    assert at.KVCache.wrap(k, v, s, s.clone()).num_blocks == 1
    with pytest.raises(ValueError):
        at.KVCache.wrap(torch.zeros(2, 2, 16, 64, dtype=torch.int8), torch.zeros(2, 16, 2, 64, dtype=torch.int8).transpose(1, 2), torch.zeros(2, 2), torch.zeros(2, 2))


def outputs(words):
    """The addresses that an advance writes besides its tables: num_free, lengths, granted, query_start, positions, slots, requests."""
    return words[11:18]


def test_a_captured_step_keeps_its_outputs(calls, monkeypatch):
    """A graph holds the addresses of a step's outputs, and nobody else may: neither another size of step nor the steps outside
    the graph may get that memory, and it may not go back to the allocator."""
    B, T = 3, 5
    t = at.BlockTables(ints(B, 4), ints(9), 16)
    inputs = ints(B), ints(B), ints(1)
    t.advance(*inputs, T)                                 # the warm-up before a capture
    monkeypatch.setattr(at, "_capturing", lambda stream: True)
    for _ in range(2):
        t.advance(*inputs, T)                             # (the captured function keeps nothing)
    monkeypatch.setattr(at, "_capturing", lambda stream: False)
    sizes = (1, B, B, B + 1, T, T, T)
    held = [(p, p + 4 * n) for _, words in calls[-2:] for p, n in zip(outputs(words), sizes)]
    for tokens in (T, T, 7, 7, T, T):
        t.advance(*inputs, tokens)
        assert not any(lo <= p < hi for p in outputs(calls[-1][1]) for lo, hi in held)
    others = [torch.full((sum(sizes),), 7, dtype=torch.int32) for _ in range(2000)]
    assert not any(lo <= o.data_ptr() < hi for o in others for lo, hi in held)
    assert len({lo for lo, _ in held}) == len(held)


class FakeStream:
    cuda_stream = 5


@pytest.fixture
def memory(calls, monkeypatch):
    """Allocations as (stream that was current, tensor), and (tensor's address, stream) of every record_stream."""
    current, made, recorded = ["the current one"], [], []

    class Under:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream)

        def __exit__(self, *_):
            current.pop()

    def taken_down(make):
        def f(*a, **k):
            y = make(*a, **k)
            made.append((current[-1], y))
            return y
        return f

    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: current[-1])
    monkeypatch.setattr(at, "_stream", lambda stream: 0 if stream is None and current[-1] == "the current one" else 5)
    monkeypatch.setattr(torch, "empty", taken_down(torch.empty))
    monkeypatch.setattr(torch, "empty_like", taken_down(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: recorded.append((self.untyped_storage().data_ptr(), s)), raising=False)
    return made, recorded


def test_what_a_call_on_another_stream_allocates_is_that_streams(memory):
    """Memory of the current stream may still be in use there when the other stream writes it."""
    made, recorded = memory
    s = FakeStream()
    c, r = at.KVCache(8, 16, 2, 64, device="cpu"), at.Rotary(64, device="cpu")
    t = at.BlockTables(ints(3, 4), ints(9), 16)
    q, k = torch.zeros(3, 4, 64, dtype=torch.float16), torch.zeros(3, 2, 64, dtype=torch.float16)
    for what in (lambda: r.apply(q, k, ints(3), stream=s), lambda: c.append(k, k, ints(3), rotary=r, positions=ints(3), q=q, stream=s)[None],
                 lambda: c.read(ints(3), stream=s), lambda: c.attend(q, t.table, ints(3), Scratch, with_lse=True, stream=s),
                 lambda: [t.advance(ints(3), ints(3), ints(1), 3, stream=s).slots], lambda: [t.advance(ints(3), ints(3), ints(1), 4, stream=s).slots]):
        made.clear()
        recorded.clear()
        results = what()
        storages = {y.untyped_storage().data_ptr(): stream for stream, y in made}
        for y in results:
            assert storages[y.untyped_storage().data_ptr()] is s
            assert (y.untyped_storage().data_ptr(), "the current one") in recorded
    for what in (lambda: r.apply(q, k, ints(3)), lambda: c.read(ints(3)), lambda: c.attend(q, t.table, ints(3), Scratch, with_lse=True)):
        made.clear()
        recorded.clear()
        what()
        assert all(stream == "the current one" for stream, _ in made) and not recorded


def test_a_set_of_outputs_written_on_another_stream_is_recorded_there(memory):
    made, recorded = memory
    s = FakeStream()
    t = at.BlockTables(ints(3, 4), ints(9), 16)
    t.advance(ints(3), ints(3), ints(1), 3)               # both sets are the current stream's
    assert not recorded
    step = t.advance(ints(3), ints(3), ints(1), 3, stream=s)
    assert recorded == [(step.slots.untyped_storage().data_ptr(), s)]
    with torch.cuda.stream(s):
        step = t.advance(ints(3), ints(3), ints(1), 3)
    assert recorded[1:] == [(step.slots.untyped_storage().data_ptr(), s)]


def test_outputs_whose_heads_overlap_are_refused():
    """They would be written by several threads at once: an expanded output, for instance."""
    r, c = fluxbin.RotaryDesc(64, 64, 0, 1.0, 1 << 24), a_cache()
    R, C = ctypes.addressof(r), ctypes.addressof(c)
    for strides, apart in (((256, 64), True), ((64, 192), True), ((0, 64), False), ((256, 0), False), ((64, 64), False), ((256, 32), False), ((192, 64), False)):
        if apart:
            assert attend_status(tokens=2, heads=4 if strides[0] > 64 else 2, out=strides) == 5
            continue
        assert attend_status(out=strides) == 3
        rot = lambda q, k: fluxbin.rotary_status(R, 0, 0, 2, P, P, 4, 256, 64, P, *q, P, 4, 256, 64, P, *k, None)  # noqa: E731
        assert rot(strides, (256, 64)) == 3 and rot((256, 64), strides) == 3
        assert fluxbin.kv_append_status(C, 0, 2, P, P, 128, 64, P, 128, 64, R, P, P, 4, 256, 64, P, *strides, None) == 3
    assert attend_status(batch=1, tokens=1, out=(0, 64)) == 5             # one token


def test_a_turned_part_of_no_elements_is_refused():
    """(and not taken for the whole head)"""
    for d in (0, -2, 1, 66):
        with pytest.raises(fluxbin.FluxBinError, match="range"):
            at.Rotary(64, d, device="cpu")
    assert at.Rotary(64, device="cpu").rotary_dim == 64 and at.Rotary(64, None, device="cpu").rotary_dim == 64 and at.Rotary(64, 2, device="cpu").rotary_dim == 2


def test_a_workspace_elsewhere_is_refused(calls):
    class OfAnother(torch.Tensor):
        def get_device(self):
            return 1

    class Elsewhere:
        tensor, nbytes = torch.empty(1, dtype=torch.uint8).as_subclass(OfAnother), 1

    c = at.KVCache(8, 16, 2, 64, device="cpu")
    with pytest.raises(ValueError, match="workspace"):
        c.attend(torch.zeros(1, 4, 64, dtype=torch.float16), ints(1, 2), ints(1), Elsewhere)
    assert not calls
