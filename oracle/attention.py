"""Plain 64-bit definitions of the attention side of a decode step (test infrastructure): rotary positions, the 8-bit
block-paged cache, attention over it, block tables.  numpy, element by element or request by request, written from the
rules of include/fluxbin.h; shares no code with the kernels."""
from __future__ import annotations

import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


# ---- rotary positions ---------------------------------------------------------------------------------------------

def frequencies(d, base=10000.0, scaling="none", factor=1.0, original=1.0, fast=32.0, slow=1.0, low=1.0, high=4.0):
    """(radians per position [d / 2], magnitude)"""
    out, magnitude = [], 1.0
    if scaling == "base":
        base = base * factor ** (d / (d - 2))
    if scaling == "ramp":
        magnitude = 0.1 * math.log(factor) + 1.0
        first = max(0, math.floor(d * math.log(original / (fast * 2 * math.pi)) / (2 * math.log(base))))
        last = min(d - 1, math.ceil(d * math.log(original / (slow * 2 * math.pi)) / (2 * math.log(base))))
    for i in range(d // 2):
        f = base ** (-2 * i / d)
        if scaling == "linear":
            f = f / factor
        elif scaling == "ramp":
            w = min(1.0, max(0.0, (i - first) / max(last - first, 1e-3)))
            f = w * f / factor + (1 - w) * f
        elif scaling == "bands":
            turns = original * f / (2 * math.pi)
            w = min(1.0, max(0.0, (turns - low) / (high - low)))
            f = w * f + (1 - w) * f / factor
        out.append(f)
    return np.array(out), magnitude


def rotary(x, positions, f, magnitude, rotary_dim, interleaved, inverse=False):
    """x [T][H][D] in 64 bits."""
    y = np.array(x, np.float64)
    half = rotary_dim // 2
    for t, p in enumerate(positions):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = math.cos(int(p) * f[i]) * magnitude, math.sin(int(p) * f[i]) * magnitude * (-1 if inverse else 1)
            u, v = x[t, :, a].astype(np.float64), x[t, :, b].astype(np.float64)
            y[t, :, a], y[t, :, b] = u * c - v * s, v * c + u * s
    return y


# ---- the 8-bit cache ----------------------------------------------------------------------------------------------

def e4m3_values():
    """The value of each of the 256 patterns (NaN for 0x7f and 0xff)."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        a = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = np.nan if (b & 127) == 127 else -a if b & 128 else a
    return v


_E4M3 = e4m3_values()[:127]


def to_entry(x, fmt):
    """The value of the nearest 8-bit entry (ties to even) for x within the format's range."""
    x = np.clip(x, -TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return np.rint(x)
    a = np.abs(x)
    hi = np.searchsorted(_E4M3, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    dl, dh = a - _E4M3[lo], _E4M3[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(up, _E4M3[hi], _E4M3[lo]) * np.sign(x)


class Cache:
    """Entries as the numbers they hold (before the scale) and scales, one side (keys or values)."""

    def __init__(self, entries, scale, fmt):
        self.entries, self.scale, self.fmt = np.array(entries, np.float64), np.array(scale, np.float64), fmt   # [NB][H][bs][D], [NB][H]
        self.quotients = self.entries.copy()        # what each entry last written was rounded from

    def append(self, x, slots):
        """x [T][H][D] at slots [T]; a block's tokens are consecutive."""
        nb, H, bs, _ = self.entries.shape
        t = 0
        while t < len(slots):
            if slots[t] < 0 or slots[t] >= nb * bs:
                t += 1
                continue
            b, off, n = slots[t] // bs, slots[t] % bs, 1
            while t + n < len(slots) and off + n < bs and slots[t + n] == slots[t] + n:
                n += 1
            for h in range(H):
                new = np.asarray(x[t:t + n, h], np.float64)
                old = self.scale[b, h] if off else 0.0
                need = np.abs(new).max() / TOP[self.fmt]
                if not np.isfinite(need):
                    need = np.nan
                now = need if (need > old or np.isnan(need)) else old
                if now < 2.0 ** -100:
                    now = 0.0
                inv = 1.0 / now if now > 0 else 0.0
                if off and not now == old:
                    if now == now:
                        self._write(b, h, slice(0, off), self.entries[b, h, :off] * old * inv)
                if now == now:
                    self._write(b, h, slice(off, off + n), new * inv)
                self.scale[b, h] = now
            t += n

    def _write(self, b, h, where, quotients):
        self.quotients[b, h, where] = quotients
        self.entries[b, h, where] = to_entry(quotients, self.fmt)

    def values(self):
        return self.entries * self.scale[:, :, None, None]


def attend(q, k, v, table, lengths, query_start, scale):
    """q [T][Hq][D]; k, v [NB][H][bs][D] values; returns out, lse, and two magnitudes an error bound needs: the mean of |v|
    under the probabilities [T][Hq][D] and the largest scale * sum |q k| [T][Hq]."""
    T, Hq, D = q.shape
    nb, H, bs, _ = k.shape
    out, mean = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for r, length in enumerate(lengths):
        length = min(int(length), table.shape[1] * bs)
        a, b = int(query_start[r]), int(query_start[r + 1])
        for t in range(a, b):
            js = [j for j in range(length - (b - 1 - t)) if 0 <= table[r, j // bs] < nb]
            if not js:
                continue
            ids, off = table[r, np.array(js) // bs], np.array(js) % bs
            for h in range(Hq):
                K, V = k[ids, h // (Hq // H), off], v[ids, h // (Hq // H), off]
                s = scale * (K @ q[t, h].astype(np.float64))
                m = s.max()
                p = np.exp(s - m)
                out[t, h], mean[t, h] = p @ V / p.sum(), p @ np.abs(V) / p.sum()
                lse[t, h] = m + math.log(p.sum())
                size[t, h] = abs(scale) * (np.abs(K) @ np.abs(q[t, h].astype(np.float64))).max()
    return out, lse, mean, size


# ---- block tables -------------------------------------------------------------------------------------------------

def advance(lengths, new, table, free, num_free, bs, tokens):
    """One step, request after request; table and free are changed."""
    B, width = table.shape
    stack = list(free[:num_free])
    length = [max(0, int(x)) for x in lengths]
    need_blocks = lambda n: -(-n // bs)  # noqa: E731
    for r in range(B):
        if new[r] < 0 and need_blocks(length[r]) <= width:
            stack += list(table[r, need_blocks(max(0, length[r] + int(new[r]))):need_blocks(length[r])])
    stack = stack[:len(free)]
    free[num_free:len(stack)] = stack[num_free:]
    out, granted, asked, room = [], [], 0, len(stack)
    for r in range(B):
        n = int(new[r])
        after = max(0, length[r] + n)
        if n <= 0:
            out.append(after)
            granted.append(1)
            continue
        more = need_blocks(after) - need_blocks(length[r])
        if need_blocks(after) > width:
            out.append(length[r])
            granted.append(0)
            continue
        asked += more
        ok = more == 0 or asked <= room
        if ok:
            for i in range(more):
                table[r, need_blocks(length[r]) + i] = stack.pop()
        out.append(after if ok else length[r])
        granted.append(int(ok))
    start, pos, slot, req = [0], [], [], []
    for r in range(B):
        for i in range(max(0, int(new[r]))):
            p = length[r] + i
            pos.append(p)
            slot.append(int(table[r, p // bs]) * bs + p % bs if granted[r] else -1)
            req.append(r)
        start.append(len(pos))
    fill = max(0, tokens - len(pos))
    cut = lambda v, x: np.array((v + [x] * fill)[:tokens], np.int32)  # noqa: E731
    return dict(lengths=np.array(out), granted=np.array(granted), num_free=len(stack), query_start=np.array(start), positions=cut(pos, 0),
                slots=cut(slot, -1), requests=cut(req, -1))
