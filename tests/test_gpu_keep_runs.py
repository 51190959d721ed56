"""Keeping where a block's moved tokens are several runs: slots outside the cache between them, and offsets that leave some out.  What is
read for a later run stands for what it stood for before the call, whatever the earlier run made of the block's scale.

An entry that is requantised by a later run has been rounded twice, and the first rounding may have been of a tie (an e4m3 block whose
largest entry is 384 makes 3 steps 3.5 steps: 448 / 384 = 7 / 6), which fp32 may take either way.  So the bound follows both ends: each
step takes the lowest and the highest entry that there may be to those of their quotients less and more E.  E counts fp32 roundings: a
scale three (entry times scale, the reciprocal of the largest entry, their product), a quotient two scales, a reciprocal, their
product and that with the entry: nine of 2^-24, less than 2^-20."""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od
from test_gpu_attention import at, dev, entries_of, f64, fill  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
E = 2.0 ** -20


class Ends(oa.Cache):
    """The 64-bit cache with the lowest and the highest entry that fp32 may make of each."""

    def __init__(self, entries, scale, fmt):
        super().__init__(entries, scale, fmt)
        self.lo, self.hi = self.entries.copy(), self.entries.copy()

    def append(self, x, slots):
        bs, t = self.entries.shape[2], 0
        while t < len(slots):
            b, off, n = slots[t] // bs, slots[t] % bs, 1
            if not 0 <= b < len(self.entries):
                t += 1
                continue
            while t + n < len(slots) and off + n < bs and slots[t + n] == slots[t] + n:
                n += 1
            old = self.scale[b].copy()
            super().append(x[t:t + n], slots[t:t + n])
            for h, now in enumerate(self.scale[b]):
                inv = 1.0 / now if now > 0 else 0.0
                if off and now != old[h]:
                    self._ends(b, h, slice(0, off), self.lo[b, h, :off] * old[h] * inv, self.hi[b, h, :off] * old[h] * inv)
                new = np.asarray(x[t:t + n, h], np.float64) * inv
                self._ends(b, h, slice(off, off + n), new, new)
            t += n

    def _ends(self, b, h, where, lo, hi):
        all_of_them = [oa.to_entry(q * f, self.fmt) for q in (lo, hi) for f in (1 - E, 1 + E)]
        self.lo[b, h, where], self.hi[b, h, where] = np.min(all_of_them, 0), np.max(all_of_them, 0)


def check_ends(c, want):
    for name, w in zip("kv", want):
        assert (np.abs(f64(getattr(c, name + "_scale")) - w.scale) <= 2.0 ** -22 * w.scale).all()
        got = f64(getattr(c, name).to(torch.float32))
        assert ((w.lo <= got) & (got <= w.hi) | np.isnan(got) & np.isnan(w.entries)).all()
        assert (w.lo == w.hi).mean() > 0.9                 # (mostly there is one answer)


STEPS = [  # slots in a block of 16 (the next block's from 16 on, -1 outside the cache), path
    ([0, -1, 2, 3], [1, 2, 3, -1]),                       # a first run of zeros: the block's scale becomes 0
    ([0, 1, -1, 3, 4, 5], [1, 3, 4, 5, -1, -1]),          # ... of the block's own values
    ([0, 2, 3, 6, 7, 9, 10], [1, 2, 3, 4, 6, -1, -1]),    # offsets that are left out
    ([0, 1, 3, 4, -1, 7, 12, 13, 16, 17, -1, 19, 20, 21], [0, 2, 3, 5, 6, 7, 8, 9, 11, 13, -1, -1, -1, -1]),
    ([5, 6, 99 * 16, 8, 9, 10], [1, 3, 4, 5, -1, -1]),
    ([14, 15, 16, -1, 18, 20, 21], [1, 2, 4, 5, 6, -1, -1])]


@pytest.mark.parametrize("fmt,H,D,major", [("int8", 2, 64, False), ("e4m3", 1, 128, True), ("int8", 3, 256, False), ("e4m3", 2, 64, False)])
@pytest.mark.parametrize("slots,path", STEPS)
def test_runs_of_one_block(at, slots, path, fmt, H, D, major):  # noqa: F811
    c = at.KVCache(8, 16, H, D, fmt, token_major=major)
    fill(c, len(slots))
    blocks = [3, 6]
    slots = [blocks[s // 16] * 16 + s % 16 if 0 <= s < 32 else s for s in slots]
    start = [0, len(slots)]
    # (large entries and small ones in turn, so that a run's largest is not the block's)
    for x in (c.k, c.v):
        raw = x.view(torch.uint8)
        raw[:, :, 1::2] = torch.where((raw[:, :, 1::2] & 128) != 0, 3 if fmt == "e4m3" else 2, raw[:, :, 1::2] & 7)
        if fmt == "e4m3":
            raw.copy_(torch.where((raw & 127) == 127, torch.zeros_like(raw), raw))
    want = [Ends(e, f64(s), fmt) for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
    for w in want:
        od.keep(w, start, slots, path)
    c.keep(dev(slots), dev(start), dev(path))
    check_ends(c, want)


def test_long_runs_around_a_slot_outside(at):  # noqa: F811
    """Runs longer than what a warp holds at once, behind a first run that restarts the block's scale."""
    for D, bs, gap in ((64, 128, 3), (128, 64, 5), (256, 128, 1)):
        c = at.KVCache(4, bs, 2, D, "int8")
        fill(c, D)
        n = bs
        slots = np.arange(n) + 2 * bs
        slots[gap] = -1
        path = np.r_[np.arange(1, n), -1]
        want = [Ends(e, f64(s), "int8") for e, s in zip(entries_of(c), (c.k_scale, c.v_scale))]
        for w in want:
            od.keep(w, [0, n], slots, path)
        c.keep(dev(slots), dev([0, n]), dev(path))
        check_ends(c, want)
