"""Measured cases of the attention side of a decode step: rotary positions, appending keys and values to a block-paged
cache held in 8 bits, attention over that cache, and the block tables and slot maps both go by.

Every case exists twice: in a plain form of elementary torch operations in 32 bits (``own`` false) and through the
package's entry points (``own`` true).  The head counts are those of the decode stacks this repository is measured on
(32 heads of 128, 40 heads of 128, 64 query heads sharing 8 key heads of 128), drawn cases also take heads of 64 and 256.
"""
import math
import random

import torch

own = False

HEADS = [(32, 32, 128), (40, 40, 128), (64, 8, 128), (16, 2, 256), (24, 6, 64), (14, 2, 64), (12, 1, 128)]
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}        # the largest value an 8-bit entry stands for, before its scale
STORED = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ---- cases --------------------------------------------------------------------------------------------------------------

def _attend(name, batch, new, longest, heads, fmt, dtype, block, mix=0):
    return dict(name=name, op="attend", batch=batch, new=new, longest=longest, q_heads=heads[0], kv_heads=heads[1], dim=heads[2],
                fmt=fmt, dtype=dtype, block=block, mix=mix)


def _append(name, batch, new, longest, heads, fmt, dtype, block, rotary, interleaved, mix=0):
    return dict(name=name, op="append", batch=batch, new=new, longest=longest, q_heads=heads[0], kv_heads=heads[1], dim=heads[2],
                fmt=fmt, dtype=dtype, block=block, rotary=rotary, interleaved=interleaved, mix=mix)


def _rope(name, tokens, longest, heads, dtype, rotary, interleaved, scaling):
    return dict(name=name, op="rope", tokens=tokens, longest=longest, q_heads=heads[0], kv_heads=heads[1], dim=heads[2], dtype=dtype,
                rotary=rotary, interleaved=interleaved, scaling=scaling)


def _tables(name, batch, new, longest, block, mix=0):
    return dict(name=name, op="tables", batch=batch, new=new, longest=longest, block=block, mix=mix)


def listed():
    return [
        # one conversation a few words in: nothing but latency
        _attend("attend_start", 1, 1, 37, (32, 32, 128), "int8", "fp16", 16),
        # a decode step of 16 conversations, shared key heads, small blocks
        _attend("attend_b16", 16, 1, 4095, (64, 8, 128), "int8", "fp16", 16, 1),
        # a decode step with a key head for every query head at the batch of 8
        _attend("attend_b8_full_heads", 8, 1, 4096, (40, 40, 128), "e4m3", "fp16", 32, 2),
        # one very long document
        _attend("attend_long", 1, 1, 131071, (64, 8, 128), "e4m3", "bf16", 64),
        # five drafted tokens of each conversation checked at once
        _attend("attend_draft5", 16, 5, 8190, (64, 8, 128), "int8", "bf16", 32, 3),
        # a full server: the most bytes
        _attend("attend_b64", 64, 1, 16384, (64, 8, 128), "int8", "fp16", 64, 4),
        # a decode step's new token: turn queries and keys, quantise, store
        _append("append_b16", 16, 1, 4095, (64, 8, 128), "int8", "fp16", 16, 128, False, 1),
        # the prompts of three requests, uneven, one of them going on from an earlier turn
        _append("append_prompts", 3, 4099, 6001, (64, 8, 128), "e4m3", "bf16", 64, 128, False, 2),
        # positions of a decode step
        _rope("rope_b16", 16, 4095, (64, 8, 128), "fp16", 128, False, "none"),
        # positions of a long prompt: half of each head, neighbouring pairs, stretched frequencies
        _rope("rope_prompt", 8191, 131071, (40, 40, 128), "bf16", 64, True, "ramp"),
        # blocks for the next token of a small batch
        _tables("tables_b16", 16, 1, 4095, 16),
        # blocks for a full server that takes in prompts, drops drafted tokens and lets requests go
        _tables("tables_b1024", 1024, 257, 16384, 16, 1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "rope", "tables"])
    heads = rng.choice(HEADS)
    fmt, dtype, block = rng.choice(["int8", "e4m3"]), rng.choice(["fp16", "bf16"]), rng.choice([16, 16, 32, 64, 128])
    mix = rng.randrange(1 << 20)
    if op == "attend":
        new = rng.choice([1, 1, 1, 2, 4, 7])
        batch = _log(rng, 1, 64)
        # no more cached values, and no more products, than the largest listed case has
        held = sum(_lengths(listed()[5])[0]) * 128
        most = min(held * 8 // (batch * heads[1] * heads[2]), held * 64 // (batch * heads[0] * heads[2] * new), 131072)
        c = _attend("", batch, new, _log(rng, max(new, 9), max(most, 17)), heads, fmt, dtype, block, mix)
    elif op == "append":
        batch = _log(rng, 1, 64)
        new = rng.choice([1, 1, _log(rng, 2, max(3, 8192 // batch))])
        rotary = rng.choice([0, heads[2], heads[2], heads[2] // 2])
        c = _append("", batch, new, new + _log(rng, 1, max(2, 32768 // batch)), heads, fmt, dtype, block, rotary, rng.random() < 0.4, mix)
    elif op == "rope":
        most = 8191 * 80 * 128 // ((heads[0] + heads[1]) * heads[2])
        c = _rope("", _log(rng, 1, most), _log(rng, 100, 131072), heads, rng.choice(["fp16", "bf16", "fp32"]),
                  rng.choice([heads[2], heads[2] // 2, 32]), rng.random() < 0.5, rng.choice(["none", "linear", "base", "ramp", "bands"]))
    else:
        batch = _log(rng, 1, 1024)
        c = _tables("", batch, rng.choice([1, 1, 5, _log(rng, 2, 257)]), _log(rng, 300, 16384), rng.choice([16, 16, 32, 64]), mix)
    del c["name"]
    return c


def _lengths(case):
    """Tokens of each request after this step, and how many of them are new: part of the case, so that its work is known."""
    rng = random.Random(case["mix"] * 1000003 + case["batch"])
    longest, new = case["longest"], case["new"]
    total, fresh = [], []
    for r in range(case["batch"]):
        if case["op"] == "attend":
            n = new
        elif case["op"] == "append":
            n = new if r == 0 else rng.randint(max(1, new // 3), new)
        else:                                       # mostly the next token; some prompts, some rollbacks, some that end
            kind = rng.random()
            n = 1 if new == 1 or kind < 0.7 else rng.randint(2, new) if kind < 0.85 else -rng.randint(1, 7) if kind < 0.95 else -longest
        t = longest if r == 0 else rng.randint(max(1, n), longest)
        total.append(t)
        fresh.append(max(n, -t))
    return total, fresh


# ---- the frequencies of the pairs, in 64 bits ---------------------------------------------------------------------------

def _scaling(case):
    return {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
            "ramp": {"factor": 16.0, "original": 4096, "fast": 32.0, "slow": 1.0},
            "bands": {"factor": 8.0, "original": 8192, "low": 1.0, "high": 4.0}}[case.get("scaling", "none")]


def _frequencies(case):
    """Radians per position of each pair of a head's turned part, and the factor on the turned values."""
    kind, s, d, base = case.get("scaling", "none"), _scaling(case), case["rotary"], 10000.0
    i = torch.arange(d // 2, dtype=torch.float64)
    if kind == "base":
        base = base * s["factor"] ** (d / (d - 2))
    f, magnitude = base ** (-2.0 * i / d), 1.0
    if kind == "linear":
        f = f / s["factor"]
    elif kind == "ramp":
        pair = lambda turns: d * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0, math.floor(pair(s["fast"]))), min(d - 1, math.ceil(pair(s["slow"])))
        slow = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f / s["factor"] * slow + f * (1 - slow)
        magnitude = 0.1 * math.log(s["factor"]) + 1.0
    elif kind == "bands":
        turns = s["original"] * f / (2 * math.pi)
        keep = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        f = f * keep + f / s["factor"] * (1 - keep)
    return f, magnitude


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


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


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    dt = TYPES[case["dtype"]] if "dtype" in case else None
    if case["op"] in ("attend", "append", "tables"):
        total, fresh = _lengths(case)
    if case["op"] == "attend":
        blocks, s["table"] = _pool(case, g, total)
        s["k"], s["k_scale"], s["v"], s["v_scale"] = _cache(case, g, blocks)
        n, B = case["new"], case["batch"]
        s["q"] = _normal(g, (B * n, case["q_heads"], case["dim"]), dt)
        s["lengths"] = _ints(total)
        s["start"] = None if n == 1 else torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
        if own:
            from paper_2608_15602_b200 import attention
            s["cache"] = attention.KVCache.wrap(s["k"], s["v"], s["k_scale"], s["v_scale"])
            s["ws"] = s["cache"].workspace(B, B * n, case["q_heads"])
    elif case["op"] == "append":
        blocks, table = _pool(case, g, total)
        s["k"], s["k_scale"], s["v"], s["v_scale"] = _cache(case, g, blocks)
        pos = torch.cat([torch.arange(t - n, t) for t, n in zip(total, fresh)])
        req = torch.repeat_interleave(torch.arange(len(fresh)), torch.tensor(fresh))
        tb = table.cpu().long()
        slots = tb[req, pos // case["block"]] * case["block"] + pos % case["block"]
        s["slots"], s["pos"] = slots.to(torch.int32).cuda(), pos.to(torch.int32).cuda()
        s["k_new"], s["v_new"] = _normal(g, (len(pos), case["kv_heads"], case["dim"]), dt) * 1.5, _normal(g, (len(pos), case["kv_heads"], case["dim"]), dt)
        # the tokens of every block that takes part, earlier ones of it among them, so that what a new scale does to them is seen
        keep = []
        for r, (t, n) in enumerate(zip(total, fresh)):
            p = torch.arange((t - n) // case["block"] * case["block"], t)
            keep.append(tb[r, p // case["block"]] * case["block"] + p % case["block"])
        s["seen"] = torch.cat(keep).to(torch.int32).cuda()
        s["touched"] = torch.unique(slots // case["block"]).cuda()
        if case["rotary"]:
            s["q"] = _normal(g, (len(pos), case["q_heads"], case["dim"]), dt)
            f, s["magnitude"] = _frequencies(case)
            s["turns"] = _fixed(f)
        if own:
            from paper_2608_15602_b200 import attention
            s["cache"] = attention.KVCache.wrap(s["k"], s["v"], s["k_scale"], s["v_scale"])
            s["rotary_plan"] = attention.Rotary(case["dim"], case["rotary"], interleaved=case["interleaved"]) if case["rotary"] else None
    elif case["op"] == "rope":
        s["q"] = _normal(g, (case["tokens"], case["q_heads"], case["dim"]), dt)
        s["k"] = _normal(g, (case["tokens"], case["kv_heads"], case["dim"]), dt)
        s["pos"] = torch.randint(0, case["longest"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
        f, s["magnitude"] = _frequencies(case)
        s["turns"] = _fixed(f)
        if own:
            from paper_2608_15602_b200 import attention
            s["rotary_plan"] = attention.Rotary(case["dim"], case["rotary"], interleaved=case["interleaved"], scaling=case["scaling"], **_scaling(case))
    else:
        blocks, s["table"] = _pool(case, g, total)
        most = [t + max(n, 0) for t, n in zip(total, fresh)]
        wide = max(-(-m // case["block"]) for m in most)
        s["table"] = torch.nn.functional.pad(s["table"], (0, wide - s["table"].shape[1]), value=-1)
        spare = torch.ones(blocks, dtype=torch.bool, device="cuda")
        spare[s["table"][s["table"] >= 0].long()] = False
        room = sum(max(n, 0) // case["block"] + 1 for n in fresh) + 3
        extra = torch.arange(blocks, blocks + room, device="cuda")
        free = torch.cat([torch.nonzero(spare)[:, 0], extra])
        free = free[torch.randperm(free.numel(), generator=g, device="cuda")].to(torch.int32)
        s["num_free"] = _ints([free.numel()])
        s["free"] = torch.nn.functional.pad(free, (0, blocks), value=-1)
        s["lengths"], s["fresh"] = _ints(total), _ints(fresh)
        s["tokens"] = sum(max(n, 0) for n in fresh)
        if own:
            from paper_2608_15602_b200 import attention
            s["plan"] = attention.BlockTables(s["table"], s["free"], case["block"])
    return s


def _fixed(f):
    """A pair's frequency as a binary fraction of a turn in 64 bits: products with a position wrap around as angles do."""
    whole = [int(round(float(x) / (2 * math.pi) * 2.0 ** 64)) for x in f]
    return torch.tensor([w - (1 << 64) if w >= 1 << 63 else w for w in whole], dtype=torch.int64, device="cuda")


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _attend_plain(s):
    bs, D, H, G, n = s["block"], s["dim"], s["kv_heads"], s["q_heads"] // s["kv_heads"], s["new"]
    B, width = s["table"].shape
    idx = s["table"].long().clamp_min(0)
    L = width * bs
    at = torch.arange(L, device="cuda")
    q = s["q"].float().view(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    k = s["k"][idx].float() * s["k_scale"][idx][..., None, None]                        # [B][block][H][token][D]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)
    x = torch.matmul(q, k.transpose(2, 3)) * (D ** -0.5)
    del k
    own_pos = s["lengths"][:, None] - n + torch.arange(n, device="cuda")[None, :]       # the position of each query
    seen = at[None, None, :] <= own_pos[:, :, None]                                     # [B][n][L]
    seen = seen[:, None, None].expand(B, H, G, n, L).reshape(B, H, G * n, L)
    x = x.masked_fill(~seen, float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m.masked_fill(m == float("-inf"), 0.0))
    l = p.sum(-1, keepdim=True)
    v = s["v"][idx].float() * s["v_scale"][idx][..., None, None]
    v = v.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)
    v = v.masked_fill((at[None, :] >= s["lengths"][:, None])[:, None, :, None], 0.0)
    o = torch.matmul(p, v) / l.masked_fill(l == 0, 1.0)
    back = lambda t, d: t.reshape(B, H, G, n, d).permute(0, 3, 1, 2, 4).reshape(B * n, H * G, d)  # noqa: E731
    return {"out": back(o, D).to(s["q"].dtype), "lse": back(m + torch.log(l), 1)[..., 0]}


def _turn(x, pos, s):
    """The turned heads of x [T][heads][D] in 32 bits."""
    r, half = s["rotary"], s["rotary"] // 2
    turn = ((pos.long()[:, None] * s["turns"][None, :]) >> 32).float() * (2 * math.pi / 2.0 ** 32)
    c, d = torch.cos(turn)[:, None] * s["magnitude"], torch.sin(turn)[:, None] * s["magnitude"]
    x = x.float()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s["interleaved"] else (x[..., :half], x[..., half:r])
    u, v = a * c - b * d, b * c + a * d
    y = torch.stack((u, v), -1).flatten(-2) if s["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((y, x[..., r:]), -1)


def _store_plain(x, held, scale, s):
    bs, top, fmt = s["block"], TOP[s["fmt"]], s["fmt"]
    blocks, H = scale.shape
    slots, touched = s["slots"].long(), s["touched"]
    blk, off = slots // bs, slots % bs
    first = torch.full((blocks,), bs, dtype=torch.int64, device="cuda").scatter_reduce(0, blk, off, "amin")
    most = torch.zeros((blocks, H), device="cuda").scatter_reduce(0, blk[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    old = torch.where(first[:, None] == 0, 0.0, scale)
    new = torch.maximum(old, most * torch.tensor(1.0 / top, dtype=torch.float32, device="cuda"))
    inv = torch.where(new > 0, torch.reciprocal(new), 0.0)
    rounded = lambda t: (t.round() if fmt == "int8" else t).clamp(-top, top).to(held.dtype)  # noqa: E731
    h = held[touched]                                                                    # [touched][H][token][D]
    ratio = (old * inv)[touched][..., None, None]
    grown = (new > old)[touched][..., None, None] & (torch.arange(bs, device="cuda") < first[touched][:, None])[:, None, :, None]
    held[touched] = torch.where(grown, rounded(h.float() * ratio).float(), h.float()).to(held.dtype)
    held[blk, :, off] = rounded(x * inv[blk][..., None])
    scale[touched] = new[touched]


def _append_plain(s):
    out = {}
    k = s["k_new"].float()
    if s["rotary"]:
        out["q"] = _turn(s["q"], s["pos"], s).to(s["q"].dtype)
        k = _turn(k, s["pos"], s)
    _store_plain(k, s["k"], s["k_scale"], s)
    _store_plain(s["v_new"].float(), s["v"], s["v_scale"], s)
    blk, off = s["seen"].long() // s["block"], s["seen"].long() % s["block"]
    for name in ("k", "v"):
        out[name] = (s[name][blk, :, off].float() * s[name + "_scale"][blk][..., None]).to(s["k_new"].dtype)
        out[name + "_scale"] = s[name + "_scale"]
    return out


def _tables_plain(s):
    bs, T = s["block"], s["tokens"]
    table, free, length, fresh = s["table"], s["free"], s["lengths"].long(), s["fresh"].long()
    B, width = table.shape
    nf = s["num_free"].long()
    upto = (length + fresh).clamp_min(0)
    had, want = (length + bs - 1) // bs, (upto + bs - 1) // bs
    gone, need = (had - want).clamp_min(0), (want - had).clamp_min(0)
    fits = want <= width
    need = torch.where(fits, need, 0)
    given_back, asked = gone.cumsum(0), need.cumsum(0)
    granted = fits & ((need == 0) | (asked <= nf + given_back[-1]))
    need = torch.where(granted, need, 0)
    first = asked - torch.where(granted, need, 0)
    # what is given back lies on the free list, in order of the requests and of their blocks; what is asked for comes off its end
    at = torch.arange(width, device="cuda")[None, :]
    back = (at >= want[:, None]) & (at < had[:, None])
    place = torch.where(back, nf + (given_back - gone)[:, None] + at - want[:, None], free.numel())
    free_now = torch.nn.functional.pad(free, (0, 1)).scatter(0, place.reshape(-1), torch.where(back, table, 0).reshape(-1))[:-1]
    end = nf + given_back[-1]
    take = granted[:, None] & (at >= had[:, None]) & (at < want[:, None])
    which = (end - 1 - (first[:, None] + at - had[:, None])).clamp(0, free.numel() - 1)
    table_now = torch.where(take, free_now[which], table)
    table.copy_(table_now)
    free.copy_(free_now)
    lengths = torch.where(granted | (fresh <= 0), upto, length)
    count = fresh.clamp_min(0)
    starts = torch.nn.functional.pad(count.cumsum(0), (1, 0))
    tok = torch.arange(T, device="cuda")
    req = torch.searchsorted(starts[1:].contiguous(), tok, right=True)
    pos = length[req] + tok - starts[req]
    slot = table_now[req, (pos // bs).clamp_max(width - 1)].long() * bs + pos % bs
    slot = torch.where(granted[req], slot, -1)
    i32 = lambda t: t.to(torch.int32)  # noqa: E731
    return {"table": table, "free": free, "num_free": i32(end - need.sum()), "lengths": i32(lengths), "start": i32(starts), "positions": i32(pos),
            "slots": i32(slot), "requests": i32(req), "granted": i32(granted | (fresh <= 0))}


def run(state):
    s = state
    if not own:
        if s["op"] == "rope":
            return {"q": _turn(s["q"], s["pos"], s).to(s["q"].dtype), "k": _turn(s["k"], s["pos"], s).to(s["k"].dtype)}
        return {"attend": _attend_plain, "append": _append_plain, "tables": _tables_plain}[s["op"]](s)
    if s["op"] == "attend":
        out, lse = s["cache"].attend(s["q"], s["table"], s["lengths"], s["ws"], query_start=s["start"], with_lse=True)
        return {"out": out, "lse": lse}
    if s["op"] == "append":
        out = {}
        if s["rotary"]:
            out["q"] = s["cache"].append(s["k_new"], s["v_new"], s["slots"], rotary=s["rotary_plan"], positions=s["pos"], q=s["q"])
        else:
            s["cache"].append(s["k_new"], s["v_new"], s["slots"])
        out["k"], out["v"] = s["cache"].read(s["seen"], dtype=s["k_new"].dtype)
        out["k_scale"], out["v_scale"] = s["k_scale"], s["v_scale"]
        return out
    if s["op"] == "rope":
        q, k = s["rotary_plan"].apply(s["q"], s["k"], s["pos"])
        return {"q": q, "k": k}
    step = s["plan"].advance(s["lengths"], s["fresh"], s["num_free"], s["tokens"])
    return {"table": s["table"], "free": s["free"], "num_free": step.num_free, "lengths": step.lengths, "start": step.query_start,
            "positions": step.positions, "slots": step.slots, "requests": step.requests, "granted": step.granted}


# ---- work ---------------------------------------------------------------------------------------------------------------

def work(case):
    size = {"fp16": 2, "bf16": 2, "fp32": 4}.get(case.get("dtype"), 0)
    if case["op"] == "rope":
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        turned = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["rotary"]
        return {"bytes": 2 * values * size + 4 * case["tokens"], "flops": 3 * turned}
    total, fresh = _lengths(case)
    bs = case["block"]
    if case["op"] == "tables":
        T = sum(max(n, 0) for n in fresh)
        moved = sum(abs(-(-max(t + n, 0) // bs) - -(-t // bs)) for t, n in zip(total, fresh))
        return {"bytes": 4 * (5 * len(total) + 3 * T + 2 * moved) + 12, "flops": 4 * T + 10 * len(total)}
    H, D, Hq = case["kv_heads"], case["dim"], case["q_heads"]
    if case["op"] == "attend":
        n = case["new"]
        pairs = sum(sum(max(0, t - n + i + 1) for i in range(n)) for t in total)
        return {"bytes": sum(total) * H * D * 2 + sum(-(-t // bs) for t in total) * (8 * H + 4) + len(total) * n * Hq * (2 * D * size + 4),
                "flops": 4 * pairs * Hq * D}
    T = sum(fresh)
    seen = sum(t - (t - n) // bs * bs for t, n in zip(total, fresh))
    q = 2 * T * Hq * D * size if case["rotary"] else 0
    # new keys and values in, 8 bits out; then every token of the blocks is read back as values
    return {"bytes": 2 * T * H * D * (size + 1) + q + 8 * T + 2 * seen * H * D * (1 + size) + 4 * seen, "flops": 6 * T * H * D + 3 * T * (Hq + H) * case["rotary"]}


# ---- from the definition, in 64 bits ------------------------------------------------------------------------------------

def _angles64(pos, case):
    f, magnitude = _frequencies(case)
    a = pos.double()[:, None] * f.cuda()[None, :]
    return torch.polar(torch.full_like(a, magnitude), a)[:, None, :]


def _turn64(x, pos, case):
    r = case["rotary"]
    z, y = _angles64(pos, case), x.double().clone()
    if case["interleaved"]:
        y[..., :r] = torch.view_as_real(torch.view_as_complex(x.double()[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(x.double()[..., :r // 2], x.double()[..., r // 2:r]) * z
        y[..., :r // 2], y[..., r // 2:r] = w.real, w.imag
    return y


def exact(case, seed):
    global own
    if case["op"] == "tables":
        return None
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    if case["op"] == "rope":
        return {"q": _turn64(s["q"], s["pos"], case), "k": _turn64(s["k"], s["pos"], case)}
    bs, D, H = case["block"], case["dim"], case["kv_heads"]
    if case["op"] == "attend":
        n, G = case["new"], case["q_heads"] // H
        outs, lses = [], []
        for r, length in enumerate(s["lengths"].tolist()):
            ids = s["table"][r, :-(-length // bs)].long()
            q = s["q"][r * n:(r + 1) * n].double().view(n, H, G, D)
            side = lambda x, c: (x[ids].double() * c[ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, D)[:, :length]  # noqa: E731,B023
            x = torch.einsum("nhgd,hld->nhgl", q, side(s["k"], s["k_scale"])) / math.sqrt(D)
            for i in range(n):
                x[i, :, :, max(0, length - n + i + 1):] = float("-inf")
            lse = torch.logsumexp(x, -1)
            w = torch.where(torch.isinf(lse)[..., None], 0.0, torch.exp(x - lse[..., None]))
            outs.append(torch.einsum("nhgl,hld->nhgd", w, side(s["v"], s["v_scale"])).reshape(n, H * G, D))
            lses.append(lse.reshape(n, H * G))
        return {"out": torch.cat(outs), "lse": torch.cat(lses)}
    # append: block by block, as the cache is defined
    out, top = {}, TOP[case["fmt"]]
    new = {"k": _turn64(s["k_new"], s["pos"], case) if case["rotary"] else s["k_new"].double(), "v": s["v_new"].double()}
    if case["rotary"]:
        out["q"] = _turn64(s["q"], s["pos"], case)
    slots = s["slots"].long()
    by_block = torch.argsort(slots // bs, stable=True)
    ids, counts = torch.unique_consecutive((slots // bs)[by_block], return_counts=True)
    seen_blk, seen_off = s["seen"].long() // bs, s["seen"].long() % bs
    for name in ("k", "v"):
        scale, full = s[name + "_scale"].double(), {}
        values = torch.zeros((scale.shape[0], H, bs, D), dtype=torch.float64, device="cuda")
        values[s["touched"]] = s[name][s["touched"]].double() * scale[s["touched"]][..., None, None]
        a = 0
        for b, c in zip(ids.tolist(), counts.tolist()):
            tok = by_block[a:a + c]
            a += c
            off = slots[tok] % bs
            first = int(off.min())
            before_scale = scale[b] if first else torch.zeros_like(scale[b])
            now = torch.maximum(before_scale, new[name][tok].abs().amax((0, 2)) / top)
            step = now[:, None, None]
            to8 = (lambda t: t.round()) if case["fmt"] == "int8" else (lambda t: t.float().clamp(-top, top).to(torch.float8_e4m3fn).double())
            again = to8(values[b, :, :first] / step) * step
            values[b, :, :first] = torch.where((now > before_scale)[:, None, None], again, values[b, :, :first])
            values[b, :, off] = to8(new[name][tok].transpose(0, 1) / step) * step
            full[b] = now
        for b, now in full.items():
            scale[b] = now
        out[name], out[name + "_scale"] = values[seen_blk, :, seen_off], scale
    return out
