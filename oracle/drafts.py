"""Plain 64-bit definitions of checking trees of drafted tokens (test infrastructure): normed and turned heads with their
gradients, masks and positions of a tree, attention under masks, the accepted path, keeping it.  numpy, written from the rules of
include/fluxbin.h; shares no code with the kernels."""
from __future__ import annotations

import math

import numpy as np

from . import attention as oa


def norm(x, eps):
    """(x / size, size) of heads x [T][H][D]: size [T][H][1] the root of the mean square plus eps"""
    x = np.asarray(x, np.float64)
    size = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x / size, size


def norm_rotary(x, weight, eps, positions, f, magnitude, rotary_dim, interleaved):
    n, _ = norm(x, eps)
    return oa.rotary(n * (1.0 if weight is None else weight), positions, f, magnitude, rotary_dim, interleaved)


def norm_rotary_backward(x, weight, eps, grad, positions, f, magnitude, rotary_dim, interleaved):
    """(gradient of x, of the weight) and the magnitudes that an error bound needs: of what is turned back, [T][H][D]"""
    D = x.shape[-1]
    w = np.ones(D) if weight is None else np.asarray(weight, np.float64)
    n, size = norm(x, eps)
    e = oa.rotary(grad, positions, f, magnitude, rotary_dim, interleaved, inverse=True)
    dx = (w * e - n * (w * e * n).mean(-1, keepdims=True)) / size
    return dx, (e * n).sum((0, 1)), e


def pair_size(x, rotary_dim, interleaved):
    """|a| + |b| of each element's pair (the element itself where it is not turned)"""
    y, half = np.abs(np.asarray(x, np.float64)), rotary_dim // 2
    out = y.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[..., a] = out[..., b] = y[..., a] + y[..., b]
    return out


def spans(query_start, batch, tokens):
    clip = lambda v: min(max(int(v), 0), tokens)  # noqa: E731
    return [(clip(query_start[r]), max(clip(query_start[r + 1]) - clip(query_start[r]), 0)) for r in range(batch)]


def tree(parents, query_start, lengths, nodes):
    """(mask words [T][W], positions [T])"""
    T, W = len(parents), -(-nodes // 32)
    mask, positions = np.zeros((T, W), np.uint32), np.zeros(T, np.int64)
    for r, (first, count) in enumerate(spans(query_start, len(lengths), T)):
        base = max(max(int(lengths[r]), 0) - count, 0)
        for i in range(count):
            positions[first + i] = base
            if i >= nodes:
                continue
            p = int(parents[first + i])
            if 0 <= p < i:
                mask[first + i] = mask[first + p]
                positions[first + i] = positions[first + p] + 1
            mask[first + i, i // 32] |= np.uint32(1 << (i % 32))
    return mask.view(np.int32), positions


def accept(parents, drafted, answers, query_start, batch, nodes):
    T = len(parents)
    path, count, answer, surplus = np.full(T, -1), np.zeros(batch, int), np.full(batch, -1), np.zeros(batch, int)
    for r, (first, n) in enumerate(spans(query_start, batch, T)):
        at = 0 if n else -1
        while at >= 0:
            path[first + count[r]] = at
            count[r] += 1
            answer[r] = answers[first + at]
            at = next((i for i in range(at + 1, min(n, nodes)) if parents[first + i] == at and drafted[first + i] == answer[r]), -1)
        surplus[r] = count[r] - n
    return path, count, answer, surplus


def attend(q, k, v, table, lengths, query_start, mask, scale):
    """As oracle.attention.attend, for rows that see their request's tokens before the new ones and what their mask [T][W] says."""
    T, Hq, D = q.shape
    nb, H, bs, _ = k.shape
    mask = np.asarray(mask).astype(np.int64) & 0xffffffff
    out, mean = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for r, (first, count) in enumerate(spans(query_start, len(lengths), T)):
        length = min(int(lengths[r]), table.shape[1] * bs)
        base = length - count
        for t in range(first, first + count):
            sees = lambda j: j < base or (0 <= j - base < min(count, mask.shape[1] * 32) and (int(mask[t, (j - base) // 32]) >> ((j - base) % 32)) & 1)  # noqa: E731,B023
            js = np.array([j for j in range(max(length, 0)) if 0 <= table[r, j // bs] < nb and sees(j)], int)
            if not len(js):
                continue
            ids, off = table[r, js // bs], js % bs
            K, V = k[ids, :, off], v[ids, :, off]                                            # [J][H][D]
            for h in range(Hq):
                s = scale * (K[:, h // (Hq // H)] @ q[t, h].astype(np.float64))
                m = s.max()
                p = np.exp(s - m)
                Vh = V[:, h // (Hq // H)]
                out[t, h], mean[t, h] = p @ Vh / p.sum(), p @ np.abs(Vh) / p.sum()
                lse[t, h] = m + math.log(p.sum())
                size[t, h] = abs(scale) * (np.abs(K[:, h // (Hq // H)]) @ np.abs(q[t, h].astype(np.float64))).max()
    return out, lse, mean, size


def keep(cache, query_start, slots, path):
    """cache: oracle.attention.Cache of one side, changed in place"""
    nb, H, bs, D = cache.entries.shape
    before = cache.values()
    for first, n in spans(query_start, len(query_start) - 1, len(slots)):
        moved = []
        for j in range(n):
            p = int(path[first + j])
            if p < j or p >= n or (j and p <= path[first + j - 1]):
                break
            if p != j or moved:
                moved.append((j, p))
        to = [int(slots[first + j]) for j, _ in moved]
        x = np.zeros((len(moved), H, D))
        for i, (_, p) in enumerate(moved):
            s = int(slots[first + p])
            if 0 <= s < nb * bs:
                x[i] = before[s // bs, :, s % bs]
        cache.append(x, to)
