"""Measured cases of checking a tree of drafted tokens over the 8-bit cache: heads that are normed and turned to their
positions in one pass (with gradients), the masks and positions of the drafted tokens from their parents, attention in which
a token sees the cache and its own ancestors, and keeping the path that the model itself would have answered.

Every case exists twice: in a plain form of elementary torch operations in 32 bits (``own`` false) and through the
package's entry points (``own`` true).  The head counts are those of the decode stacks this repository is measured on
(32 heads of 128, 40 heads of 128, 64 query heads sharing 8 key heads of 128), drawn cases also take heads of 64 and 256.
"""
import math
import random

import torch

own = False

HEADS = [(32, 32, 128), (40, 40, 128), (64, 8, 128), (64, 8, 128), (16, 2, 256), (24, 6, 64), (14, 2, 64), (12, 1, 128)]
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}        # the largest value an 8-bit entry stands for, before its scale
STORED = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6


# ---- cases --------------------------------------------------------------------------------------------------------------

def _turn_case(name, op, tokens, longest, heads, dtype, rotary, interleaved):
    return dict(name=name, op=op, tokens=tokens, longest=longest, q_heads=heads[0], kv_heads=heads[1], dim=heads[2], dtype=dtype,
                rotary=rotary, interleaved=interleaved)


def _tree(name, batch, nodes, longest, heads, fmt, dtype, block, mix=0):
    return dict(name=name, op="tree", batch=batch, nodes=nodes, longest=longest, q_heads=heads[0], kv_heads=heads[1], dim=heads[2],
                fmt=fmt, dtype=dtype, block=block, mix=mix)


def _masks(name, batch, nodes, longest, mix=0):
    return dict(name=name, op="masks", batch=batch, nodes=nodes, longest=longest, mix=mix)


def _keep(name, batch, nodes, longest, heads, fmt, dtype, block, mix=0):
    return dict(_tree(name, batch, nodes, longest, heads, fmt, dtype, block, mix), op="keep")


def listed():
    return [
        # positions of a decode step's tokens, whose heads are normed: nothing but latency
        _turn_case("norm_b16", "turn", 16, 4095, (64, 8, 128), "fp16", 128, False),
        # a long prompt
        _turn_case("norm_prompt", "turn", 8191, 131071, (64, 8, 128), "bf16", 128, False),
        # learning on a short text, neighbouring pairs, half of each head
        _turn_case("norm_learn_short", "learn", 257, 257, (14, 2, 64), "fp32", 32, True),
        # learning on a batch of texts
        _turn_case("norm_learn", "learn", 8190, 4096, (40, 40, 128), "bf16", 128, False),
        # one conversation a few words in, a handful of drafted tokens
        _tree("tree_start", 1, 7, 61, (32, 32, 128), "int8", "fp16", 16),
        # 16 conversations, 16 drafted tokens each: 128 query rows a key head
        _tree("tree_b16", 16, 16, 8190, (64, 8, 128), "int8", "bf16", 16, 1),
        # 8 conversations with wide trees: 504 rows a key head, the most products
        _tree("tree_b8_wide", 8, 63, 4095, (64, 8, 128), "e4m3", "fp16", 32, 2),
        # one very long document: the longest axis
        _tree("tree_long", 1, 32, 131071, (64, 8, 128), "e4m3", "bf16", 64),
        # what a step of 16 conversations needs to know about its trees
        _masks("masks_b16", 16, 16, 4095),
        # a full server with wide trees
        _masks("masks_b1024", 1024, 63, 16384, 1),
        # keeping what was right, of 16 conversations
        _keep("keep_b16", 16, 16, 4095, (64, 8, 128), "int8", "fp16", 16, 1),
        # of a full server with a key head for every query head
        _keep("keep_b256", 256, 33, 600, (40, 40, 128), "e4m3", "bf16", 64, 2),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "turn", "learn", "masks", "keep"])
    heads = rng.choice(HEADS)
    fmt, dtype, block = rng.choice(["int8", "e4m3"]), rng.choice(["fp16", "bf16"]), rng.choice([16, 16, 32, 64, 128])
    mix = rng.randrange(1 << 20)
    if op in ("turn", "learn"):
        most = 8190 * 72 * 128 // ((heads[0] + heads[1]) * heads[2])
        c = _turn_case("", op, _log(rng, 1, most), _log(rng, 100, 131072), heads, rng.choice(["fp16", "bf16", "fp32"]) if op == "learn" else dtype,
                       rng.choice([heads[2], heads[2], heads[2] // 2, 32]), rng.random() < 0.4)
    elif op == "tree":
        batch, nodes = _log(rng, 1, 64), _log(rng, 2, 64)
        # no more cached values, and no more products, than the largest listed cases have
        most = min(16 * 8190 * 8 * 128 // (batch * heads[1] * heads[2]), 8 * 4095 * 63 * 64 * 128 // (batch * heads[0] * heads[2] * nodes), 131072)
        c = _tree("", batch, nodes, max(nodes, _log(rng, 17, max(most, 18))), heads, fmt, dtype, block, mix)
    elif op == "masks":
        c = _masks("", _log(rng, 1, 1024), _log(rng, 1, 63), _log(rng, 64, 16384), mix)
    else:
        batch, nodes = _log(rng, 1, 256), _log(rng, 2, 33)
        most = 256 * 600 * 40 * 128 // (batch * heads[1] * heads[2])
        c = _keep("", batch, nodes, max(nodes, _log(rng, 40, min(max(most, 41), 8192))), heads, fmt, dtype, block, mix)
    del c["name"]
    return c


def _lengths(case):
    """Tokens of each request with the drafted ones, and how many those are: part of the case, so that its work is known."""
    rng = random.Random(case["mix"] * 1000003 + case["batch"])
    total, fresh = [], []
    for r in range(case["batch"]):
        n = case["nodes"] if r == 0 else rng.randint(max(1, case["nodes"] // 2), case["nodes"])
        total.append(max(n, case["longest"] if r == 0 else rng.randint(max(n, case["longest"] // 4), max(n, case["longest"]))))
        fresh.append(n)
    return total, fresh


def _parents(case, fresh, seed):
    """Each drafted token's parent among its request's drafted ones: the first is the last known token, a few stand beside it."""
    rng = random.Random(seed * 7919 + case["mix"])
    out = []
    for n in fresh:
        for i in range(n):
            out.append(-1 if i == 0 or rng.random() < 0.03 else rng.randint(max(0, i - 5), i - 1) if rng.random() < 0.6 else rng.randint(0, i - 1))
    return out


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(fresh):
    s = [0]
    for n in fresh:
        s.append(s[-1] + n)
    return s


def _pool(case, g, total):
    """A pool of blocks a little larger than what is used, and the requests' blocks in it, in no order."""
    need = [-(-t // case["block"]) for t in total]
    blocks = sum(need) + 1 + len(need) // 8
    order = torch.randperm(blocks, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    width = max(need)
    table = torch.full((len(need), width), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(width, device="cuda")[None, :].expand(len(need), width)
    live = at < torch.tensor(need, device="cuda")[:, None]
    first = torch.tensor([0] + need[:-1], device="cuda").cumsum(0)
    table[live] = order[(first[:, None] + at)[live]]
    return blocks, table


def _cache(case, g, blocks):
    """Keys and values as a quantiser leaves them: blocks [block][head][token][dim], every block of a head at its own scale."""
    H, bs, D, fmt = case["kv_heads"], case["block"], case["dim"], case["fmt"]
    parts = []
    for spread in (1.5, 0.7):
        held = torch.empty((blocks, H, bs, D), dtype=STORED[fmt], device="cuda")
        scale = torch.empty((blocks, H), dtype=torch.float32, device="cuda")
        step = max(1, (1 << 27) // (H * bs * D))
        for a in range(0, blocks, step):
            x = torch.randn((min(step, blocks - a), H, bs, D), generator=g, device="cuda") * spread
            m = x.abs().amax((2, 3)) * torch.tensor(1.0 / TOP[fmt], dtype=torch.float32)
            x = x / m[..., None, None]
            held[a:a + step] = (x.round() if fmt == "int8" else x).clamp(-TOP[fmt], TOP[fmt]).to(STORED[fmt])
            scale[a:a + step] = m
        parts += [held, scale]
    return parts


def _frequencies(case):
    """Radians per position of each pair of a head's turned part, in 64 bits."""
    return 10000.0 ** (-2.0 * torch.arange(case["rotary"] // 2, dtype=torch.float64) / case["rotary"])


def _fixed(f):
    """A pair's frequency as a binary fraction of a turn in 64 bits: products with a position wrap around as angles do."""
    whole = [int(round(float(x) / (2 * math.pi) * 2.0 ** 64)) for x in f]
    return torch.tensor([w - (1 << 64) if w >= 1 << 63 else w for w in whole], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] in ("turn", "learn"):
        dt, T, D = TYPES[case["dtype"]], case["tokens"], case["dim"]
        s["q"], s["k"] = _normal(g, (T, case["q_heads"], D), dt) * 1.7, _normal(g, (T, case["kv_heads"], D), dt) * 0.6
        s["wq"], s["wk"] = (1 + 0.3 * _normal(g, (D,), torch.float32)).to(dt), (1 + 0.3 * _normal(g, (D,), torch.float32)).to(dt)
        s["pos"] = torch.randint(0, case["longest"], (T,), generator=g, device="cuda", dtype=torch.int32)
        s["turns"] = _fixed(_frequencies(case))
        if case["op"] == "learn":
            s["gq"], s["gk"] = _normal(g, s["q"].shape, dt), _normal(g, s["k"].shape, dt)
        if own:
            from paper_2608_15602_b200 import attention
            wants = case["op"] == "learn"
            for name in ("q", "k", "wq", "wk"):
                s[name].requires_grad_(wants)
            s["plan"] = attention.NormedRotary(attention.Rotary(D, case["rotary"], interleaved=case["interleaved"]), s["wq"], s["wk"], eps=EPS)
        return s
    total, fresh = _lengths(case)
    start, parents = _starts(fresh), _parents(case, fresh, seed)
    s["tokens"], s["words"] = start[-1], -(-case["nodes"] // 32)
    s["lengths"], s["fresh"], s["start"], s["parents"] = _ints(total), _ints(fresh), _ints(start), _ints(parents)
    s["request"] = torch.repeat_interleave(torch.arange(len(fresh)), torch.tensor(fresh)).cuda()
    if case["op"] == "masks":
        return s
    blocks, s["table"] = _pool(case, g, total)
    s["k"], s["k_scale"], s["v"], s["v_scale"] = _cache(case, g, blocks)
    if own:
        from paper_2608_15602_b200 import attention
        s["cache"] = attention.KVCache.wrap(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["plan"] = attention.DraftTree(s["parents"], s["start"], s["lengths"], case["nodes"])
    if case["op"] == "tree":
        s["q"] = _normal(g, (s["tokens"], case["q_heads"], case["dim"]), TYPES[case["dtype"]])
        s["sees"] = _ancestors(s)
        if own:
            s["ws"] = s["cache"].workspace(case["batch"], s["tokens"], case["q_heads"], tree=True)
        return s
    # keep: drafted tokens of a small vocabulary, and answers that agree with one of a token's children more often than not
    rng = random.Random(seed * 104729 + case["mix"])
    drafted = [rng.randrange(50000) for _ in parents]
    answers = [rng.randrange(50000) for _ in parents]
    slots = []
    host = s["table"].cpu().tolist()
    for r, (t, n) in enumerate(zip(total, fresh)):
        for i in range(n):
            if parents[start[r] + i] >= 0 and rng.random() < 0.75:
                answers[start[r] + parents[start[r] + i]] = drafted[start[r] + i]
            p = t - n + i
            slots.append(host[r][p // case["block"]] * case["block"] + p % case["block"])
    s["drafted"], s["answers"], s["slots"] = _ints(drafted), _ints(answers), _ints(slots)
    # the tokens of every block that takes part, earlier ones of it among them, so that what a new scale does to them is seen
    seen = []
    for r, (t, n) in enumerate(zip(total, fresh)):
        for p in range((t - n) // case["block"] * case["block"], t):
            seen.append(host[r][p // case["block"]] * case["block"] + p % case["block"])
    s["seen"] = _ints(seen)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _angles(s):
    turn = ((s["pos"].long()[:, None] * s["turns"][None, :]) >> 32).float() * (2 * math.pi / 2.0 ** 32)
    return torch.cos(turn)[:, None], torch.sin(turn)[:, None]


def _turn(x, c, d, s):
    """The turned heads of x [T][heads][D] in 32 bits."""
    r, half = s["rotary"], s["rotary"] // 2
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s["interleaved"] else (x[..., :half], x[..., half:r])
    u, v = a * c - b * d, b * c + a * d
    y = torch.stack((u, v), -1).flatten(-2) if s["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((y, x[..., r:]), -1)


def _turn_plain(s):
    out = {}
    c, d = _angles(s)
    for name in ("q", "k"):
        x, w = s[name].float(), s["w" + name].float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        out[name] = _turn(x * r * w, c, d, s).to(s[name].dtype)
        if s["op"] == "learn":
            g = _turn(s["g" + name].float(), c, -d, s)
            n = x * r
            out["d" + name] = (r * (g * w - n * (g * w * n).mean(-1, keepdim=True))).to(s[name].dtype)
            out["dw" + name] = (g * n).sum((0, 1), dtype=torch.float64).to(s["w" + name].dtype)
    return out


def _padded(s, x, fill):
    """x [tokens] as [batch][nodes], and which of those there are."""
    at = torch.arange(s["nodes"], device="cuda")[None, :]
    there = at < s["fresh"][:, None]
    idx = (s["start"][:-1, None] + at).clamp_max(s["tokens"] - 1).long()
    return torch.where(there, x[idx], fill), there, idx


def _ancestors(s):
    """Whether a drafted token [tokens] sees its request's drafted token [nodes]: itself and what it comes after."""
    T, N = s["tokens"], s["nodes"]
    sees = torch.zeros((T, N), dtype=torch.bool, device="cuda")
    tok, first = torch.arange(T, device="cuda"), s["start"].long()[s["request"]]
    at, live = tok - first, torch.ones(T, dtype=torch.bool, device="cuda")
    for _ in range(N):
        sees[tok, at] = sees[tok, at] | live
        up = s["parents"].long()[first + at]
        live = live & (up >= 0)
        at = torch.where(live, up, at)
    return sees


def _masks_plain(s):
    sees = _ancestors(s)
    bits = torch.zeros((s["tokens"], s["words"] * 32), dtype=torch.int64, device="cuda")
    bits[:, :s["nodes"]] = sees.long()
    words = (bits.view(s["tokens"], s["words"], 32) << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    depth = sees.sum(-1) - 1
    return {"mask": words, "positions": ((s["lengths"] - s["fresh"])[s["request"]] + depth).to(torch.int32)}


def _tree_plain(s):
    bs, D, H, G, N = s["block"], s["dim"], s["kv_heads"], s["q_heads"] // s["kv_heads"], s["nodes"]
    B, width = s["table"].shape
    idx, L = s["table"].long().clamp_min(0), s["table"].shape[1] * s["block"]
    pos = torch.arange(L, device="cuda")
    at = torch.arange(N, device="cuda")[None, :]
    there = at < s["fresh"][:, None]
    tok = (s["start"][:-1, None] + at).clamp_max(s["tokens"] - 1).long()                     # [B][N]
    q = s["q"].float()[tok].view(B, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, D)
    k = s["k"][idx].float() * s["k_scale"][idx][..., None, None]                        # [B][block][H][token][D]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)
    x = torch.matmul(q, k.transpose(2, 3)) * (D ** -0.5)
    del k
    base = s["lengths"] - s["fresh"]
    new = (pos[None, :] - base[:, None]).clamp(0, N - 1).long()                              # which drafted token a cached one is
    among = s["sees"][tok].gather(2, new[:, None, :].expand(B, N, L))
    seen = (pos[None, None, :] < base[:, None, None]) | (among & (pos[None, None, :] < s["lengths"][:, None, None]))
    x = x.view(B, H, G, N, L).masked_fill(~seen[:, None, None], float("-inf")).view(B, H, G * N, L)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m.masked_fill(m == float("-inf"), 0.0))
    del x
    l = p.sum(-1, keepdim=True)
    v = s["v"][idx].float() * s["v_scale"][idx][..., None, None]
    v = v.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)
    v = v.masked_fill((pos[None, :] >= s["lengths"][:, None])[:, None, :, None], 0.0)
    o = torch.matmul(p, v) / l.masked_fill(l == 0, 1.0)
    back = lambda t, d: t.reshape(B, H, G, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, H * G, d)[there]  # noqa: E731
    return {"out": back(o, D).to(s["q"].dtype), "lse": back(m + torch.log(l), 1)[..., 0]}


def _accept_plain(s):
    parents, there, _ = _padded(s, s["parents"], -2)
    drafted, answers = _padded(s, s["drafted"], -1)[0], _padded(s, s["answers"], -1)[0]
    B, N = parents.shape
    cur, live = torch.zeros(B, dtype=torch.int64, device="cuda"), s["fresh"] > 0
    path = torch.full((B, N), -1, dtype=torch.int64, device="cuda")
    count, answer = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.full((B,), -1, dtype=torch.int64, device="cuda")
    at = torch.arange(N, device="cuda")[None, :]
    for j in range(N):
        path[:, j] = torch.where(live, cur, -1)
        count = count + live
        said = answers.gather(1, cur[:, None])[:, 0].long()
        answer = torch.where(live, said, answer)
        child = there & (at > cur[:, None]) & (parents == cur[:, None]) & (drafted == said[:, None])
        first = torch.where(child, at, N).amin(1)
        live = live & (first < N)
        cur = torch.where(live, first, cur)
    return {"path": path[there].to(torch.int32), "count": count.to(torch.int32), "answer": answer.to(torch.int32),
            "surplus": (count - s["fresh"]).to(torch.int32)}


def _keep_plain(s):
    bs, top, fmt = s["block"], TOP[s["fmt"]], s["fmt"]
    out = _accept_plain(s)
    path = out["path"].long()
    own_at = torch.arange(s["tokens"], device="cuda") - s["start"].long()[s["request"]]
    moved = ((path >= 0) & (path != own_at)).nonzero()[:, 0]
    slots = s["slots"].long()
    to = slots[moved]
    source = slots[s["start"].long()[s["request"][moved]] + path[moved]]
    blk, off = to // bs, to % bs
    touched = torch.unique(blk)
    for name in ("k", "v"):
        held, scale = s[name], s[name + "_scale"]
        blocks, H = scale.shape
        x = held[source // bs, :, source % bs].float() * scale[source // bs][..., None]
        first = torch.full((blocks,), bs, dtype=torch.int64, device="cuda").scatter_reduce(0, blk, off, "amin")
        most = torch.zeros((blocks, H), device="cuda").scatter_reduce(0, blk[:, None].expand(-1, H), x.abs().amax(-1), "amax")
        old = torch.where(first[:, None] == 0, 0.0, scale)
        new = torch.maximum(old, most * torch.tensor(1.0 / top, dtype=torch.float32, device="cuda"))
        inv = torch.where(new > 0, torch.reciprocal(new), 0.0)
        rounded = lambda t: (t.round() if fmt == "int8" else t).clamp(-top, top).to(held.dtype)  # noqa: E731,B023
        h = held[touched]                                                                    # [touched][H][token][D]
        ratio = (old * inv)[touched][..., None, None]
        grown = (new > old)[touched][..., None, None] & (torch.arange(bs, device="cuda") < first[touched][:, None])[:, None, :, None]
        held[touched] = torch.where(grown, rounded(h.float() * ratio).float(), h.float()).to(held.dtype)
        held[blk, :, off] = rounded(x * inv[blk][..., None])
        scale[touched] = new[touched]
    blk, off = s["seen"].long() // bs, s["seen"].long() % bs
    for name in ("k", "v"):
        out[name] = (s[name][blk, :, off].float() * s[name + "_scale"][blk][..., None]).to(TYPES[s["dtype"]])
        out[name + "_scale"] = s[name + "_scale"]
    return out


def run(state):
    s = state
    if not own:
        return {"turn": _turn_plain, "learn": _turn_plain, "tree": _tree_plain, "masks": _masks_plain, "keep": _keep_plain}[s["op"]](s)
    if s["op"] == "turn":
        q, k = s["plan"].apply(s["q"], s["k"], s["pos"])
        return {"q": q, "k": k}
    if s["op"] == "learn":
        q, k = s["plan"].apply(s["q"], s["k"], s["pos"])
        dq, dk, dwq, dwk = torch.autograd.grad((q, k), (s["q"], s["k"], s["wq"], s["wk"]), (s["gq"], s["gk"]))
        return {"q": q.detach(), "dq": dq, "dwq": dwq, "k": k.detach(), "dk": dk, "dwk": dwk}
    if s["op"] == "tree":
        out, lse = s["cache"].attend(s["q"], s["table"], s["lengths"], s["ws"], query_start=s["start"], tree=s["plan"].mask, with_lse=True)
        return {"out": out, "lse": lse}
    if s["op"] == "masks":
        from paper_2608_15602_b200 import attention
        tree = attention.DraftTree(s["parents"], s["start"], s["lengths"], s["nodes"])
        return {"mask": tree.mask, "positions": tree.positions}
    kept = s["plan"].accept(s["drafted"], s["answers"])
    s["cache"].keep(s["slots"], s["start"], kept.path)
    k, v = s["cache"].read(s["seen"], dtype=TYPES[s["dtype"]])
    return {"path": kept.path, "count": kept.count, "answer": kept.answer, "surplus": kept.surplus,
            "k": k, "k_scale": s["k_scale"], "v": v, "v_scale": s["v_scale"]}


# ---- work ---------------------------------------------------------------------------------------------------------------

def work(case):
    size = {"fp16": 2, "bf16": 2, "fp32": 4}.get(case.get("dtype"), 0)
    if case["op"] in ("turn", "learn"):
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        turned = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["rotary"]
        if case["op"] == "turn":
            return {"bytes": 2 * values * size + 4 * case["tokens"] + 2 * case["dim"] * size, "flops": 4 * values + 3 * turned}
        # the result is written, then heads and gradients are read and the heads' gradients written
        return {"bytes": 5 * values * size + 8 * case["tokens"] + 6 * case["dim"] * size, "flops": 14 * values + 6 * turned}
    total, fresh = _lengths(case)
    T, B, words = sum(fresh), len(fresh), -(-case["nodes"] // 32)
    if case["op"] == "masks":
        return {"bytes": 4 * (2 * T + 2 * B + 1 + T * words), "flops": 4 * T * words}
    H, D, Hq, bs = case["kv_heads"], case["dim"], case["q_heads"], case["block"]
    if case["op"] == "tree":
        # (each drafted token sees the cache and, counted as half of them, its ancestors)
        pairs = sum(n * (t - n) + n * (n + 1) // 2 for t, n in zip(total, fresh))
        return {"bytes": sum(total) * H * D * 2 + sum(-(-t // bs) for t in total) * (8 * H + 4) + T * Hq * (2 * D * size + 4) + 4 * T * words,
                "flops": 4 * pairs * Hq * D}
    # the trees, a third of the drafted tokens moved, and every token of the blocks read back as values
    seen = sum(t - (t - n) // bs * bs for t, n in zip(total, fresh))
    return {"bytes": 4 * (5 * T + 4 * B) + T // 3 * 4 * H * D + 2 * seen * H * D * (1 + size) + 4 * seen, "flops": T // 3 * 6 * H * D}


# ---- from the definition, in 64 bits ------------------------------------------------------------------------------------

def _turn64(x, s, sign):
    r, x = s["rotary"], x.double()
    a = s["pos"].double()[:, None] * _frequencies(s).cuda()[None, :] * sign
    z, y = torch.polar(torch.ones_like(a), a)[:, None, :], x.clone()
    if s["interleaved"]:
        y[..., :r] = torch.view_as_real(torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * z
        y[..., :r // 2], y[..., r // 2:r] = w.real, w.imag
    return y


def exact(case, seed):
    global own
    if case["op"] == "masks":
        return None
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    D = case["dim"]
    if case["op"] in ("turn", "learn"):
        out = {}
        for name in ("q", "k"):
            x, w = s[name].double(), s["w" + name].double()
            size = torch.sqrt(torch.einsum("thd,thd->th", x, x) / D + EPS)[..., None]
            out[name] = _turn64(x / size * w, s, 1.0)
            if case["op"] == "learn":
                e = _turn64(s["g" + name], s, -1.0)
                out["d" + name] = w * e / size - x * torch.einsum("thd,thd,d->th", x, e, w)[..., None] / (D * size ** 3)
                out["dw" + name] = torch.einsum("thd,thd->d", x / size, e)
        return out
    bs, H = case["block"], case["kv_heads"]
    start, parents = s["start"].tolist(), s["parents"].tolist()
    if case["op"] == "tree":
        G = case["q_heads"] // H
        outs, lses = [], []
        for r, length in enumerate(s["lengths"].tolist()):
            a, n = start[r], start[r + 1] - start[r]
            ids = s["table"][r, :-(-length // bs)].long()
            q = s["q"][a:a + n].double().view(n, H, G, D)
            side = lambda x, c: (x[ids].double() * c[ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, D)[:, :length]  # noqa: E731,B023
            x = torch.einsum("nhgd,hld->nhgl", q, side(s["k"], s["k_scale"])) / math.sqrt(D)
            hidden = torch.ones((n, n), dtype=torch.bool)
            for i in range(n):
                if parents[a + i] >= 0:
                    hidden[i] = hidden[parents[a + i]]
                hidden[i, i] = False
            x[..., length - n:] = x[..., length - n:].masked_fill(hidden.cuda()[:, None, None, :], float("-inf"))
            lse = torch.logsumexp(x, -1)
            w = torch.exp(x - lse[..., None])
            outs.append(torch.einsum("nhgl,hld->nhgd", w, side(s["v"], s["v_scale"])).reshape(n, H * G, D))
            lses.append(lse.reshape(n, H * G))
        return {"out": torch.cat(outs), "lse": torch.cat(lses)}
    # keep: request by request, block by block, as the cache is defined
    top, fmt = TOP[case["fmt"]], case["fmt"]
    drafted, answers, slots = s["drafted"].tolist(), s["answers"].tolist(), s["slots"].tolist()
    moves = []                                       # (block, its first new place, sources) in order
    for r in range(case["batch"]):
        a, n = start[r], start[r + 1] - start[r]
        path, cur = [], 0 if n else -1
        while cur >= 0:
            path.append(cur)
            cur = next((i for i in range(cur + 1, n) if parents[a + i] == cur and drafted[a + i] == answers[a + cur]), -1)
        for j, i in enumerate(path):
            if i == j:
                continue
            to = slots[a + j]
            if moves and moves[-1][3] == r and moves[-1][0] == to // bs:
                moves[-1][2].append(slots[a + i])
            else:
                moves.append((to // bs, to % bs, [slots[a + i]], r))
    out = dict.fromkeys(("path", "count", "answer", "surplus"))
    seen_blk, seen_off = s["seen"].long() // bs, s["seen"].long() % bs
    blocks, place = torch.unique(seen_blk, return_inverse=True)
    to8 = (lambda t: t.round()) if fmt == "int8" else (lambda t: t.float().clamp(-top, top).to(torch.float8_e4m3fn).double())
    where = {b: i for i, b in enumerate(blocks.tolist())}
    for name in ("k", "v"):
        scale, started = s[name + "_scale"].double(), s[name + "_scale"].double()
        entries = s[name][blocks].double()
        unmoved = entries.clone()
        for b, off, source, _ in moves:
            i = where[b]
            sb, so = [where[x // bs] for x in source], [x % bs for x in source]
            x = unmoved[sb, :, so] * started[[x // bs for x in source]][..., None]              # [moved][H][D]
            old = started[b] if off else torch.zeros_like(started[b])
            now = torch.maximum(old, x.abs().amax((0, 2)) / top)
            safe = now.masked_fill(now == 0, 1.0)[:, None, None]
            again = to8(unmoved[i, :, :off] * old[:, None, None] / safe)
            entries[i, :, :off] = torch.where((now > old)[:, None, None], again, unmoved[i, :, :off])
            entries[i, :, off:off + len(source)] = to8(x.transpose(0, 1) / safe)
            scale[b] = now
        out[name], out[name + "_scale"] = entries[place, :, seen_off] * scale[seen_blk][..., None], scale
    return {x: out[x] for x in ("path", "count", "answer", "surplus", "k", "k_scale", "v", "v_scale")}
