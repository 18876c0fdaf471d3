"""The calls around a decoder's paged 4-bit K/V cache whose speed is tracked, beside those of perf/operators.py: pages and
slots given to requests (`cache_reserve`), the ranges of a page's keys (`cache_bounds`), the pages that a query picks by
them (`cache_pick`), and attention over the picked pages alone (`cache_attend_picked`).

A page holds, for each key head, `page` rows of e2m1 codes (two to a byte, the even channel in the low four bits) and one
e4m3 scale for every 16 channels of a row. A request's pages stand in its row of a table. Free pages lie in a ring, from
state[0] on, state[1] of them. A page's range of keys is, for each key head and channel, the largest and the smallest
value as whole numbers of a power of two that the channels of the head share.

Sizes are those of this repository's workloads after token selection (1 to 128 requests, 460 to 1800 kept visual tokens
with the text behind them, 4/4 to 32/32 heads of 64 or 128) and of the decoding that follows: one token, a handful of
drafts, a chunk of a prompt, caches of up to 128 Ki tokens. Lengths are drawn from a case's own `sizes` number, so that a
case is a dict of plain values.
"""
import math
import random

import numpy as np
import torch

own = False  # False: the operators from elementary torch operations; True: the library's calls

# bytes and operations of a drawn case, the tokens x key heads of its pool, and the keys that its queries visit
_MOST = {"reserve": 1.3e7, "bounds": 3.4e8, "pick": 1.8e8, "attend": 6.0e8}
_MOST_FLOPS = {"reserve": 0.0, "bounds": 1.7e9, "pick": 9.7e9, "attend": 5.4e10}
_MOST_POOL, _MOST_VISITS = 1.7e7, 1.4e7


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decoding step of the largest batch: every request one token further, a few of them over a page's end. Latency
        dict(name="reserve_step", kind="reserve", batch=128, n_lo=1101, n_hi=1164, t_lo=1, t_hi=1, p_lo=0, p_hi=0,
             done=0.0, fresh=0.0, spare=1.5, page=64, sizes=1),
        # a busy server between two steps: requests that end, prompts of up to 8 Ki tokens that begin, drafts in between
        dict(name="reserve_churn", kind="reserve", batch=1024, n_lo=100, n_hi=16000, t_lo=1, t_hi=8, p_lo=400, p_hi=8191,
             done=0.3, fresh=0.35, spare=1.1, page=32, sizes=2),
        # the last page of every request of the largest batch, one token fuller
        dict(name="bounds_token", kind="bounds", batch=128, n_lo=1101, n_hi=1164, t_lo=1, t_hi=1, hq=32, hkv=32, d=128,
             page=64, sizes=3),
        # the prompts of the largest batch, just appended: 1036 kept visual and 64 text tokens for each of 128 requests
        dict(name="bounds_prompts", kind="bounds", batch=128, n_lo=1100, n_hi=1100, t_lo=1100, t_hi=1100, hq=32, hkv=32,
             d=128, page=64, sizes=4),
        # a decoded token over one long cache with grouped heads, odd length: latency
        dict(name="pick_token", kind="pick", batch=1, n_lo=40013, n_hi=40013, t_lo=1, t_hi=1, hq=28, hkv=4, d=128,
             dtype="bf16", page=64, budget=32, sink=1, recent=2, sizes=5),
        # a decoded token of many long caches, 8-bit queries, small pages
        dict(name="pick_batch_fp8", kind="pick", batch=32, n_lo=30001, n_hi=131071, t_lo=1, t_hi=1, hq=32, hkv=8, d=128,
             dtype="e4m3", page=32, budget=64, sink=1, recent=4, sizes=6),
        # a chunk of a long prompt, every query with pages of its own
        dict(name="pick_prompt", kind="pick", batch=2, n_lo=20000, n_hi=32767, t_lo=777, t_hi=1024, hq=28, hkv=4, d=128,
             dtype="bf16", page=64, budget=32, sink=1, recent=2, sizes=7),
        # a decoded token of one request, 16 heads: latency
        dict(name="attend_token", kind="attend", batch=1, n_lo=9001, n_hi=9001, t_lo=1, t_hi=1, hq=16, hkv=16, d=128,
             dtype="bf16", page=16, budget=64, sink=1, recent=4, sizes=8),
        # a decoded token of every request of the largest batch, a quarter of its keys
        dict(name="attend_token_sweep", kind="attend", batch=128, n_lo=4001, n_hi=4200, t_lo=1, t_hi=1, hq=32, hkv=32,
             d=128, dtype="bf16", page=64, budget=16, sink=1, recent=2, sizes=9),
        # a decoded token over long caches with grouped heads
        dict(name="attend_token_long", kind="attend", batch=32, n_lo=30001, n_hi=131071, t_lo=1, t_hi=1, hq=28, hkv=4,
             d=128, dtype="bf16", page=128, budget=32, sink=1, recent=2, sizes=10),
        # drafted tokens of a ragged 8-bit batch, one to eight a request
        dict(name="attend_drafts_fp8", kind="attend", batch=32, n_lo=3000, n_hi=16000, t_lo=1, t_hi=8, hq=32, hkv=8,
             d=128, dtype="e4m3", page=32, budget=48, sink=1, recent=4, sizes=11),
        # a chunk of a long prompt
        dict(name="attend_prompt", kind="attend", batch=2, n_lo=20000, n_hi=32767, t_lo=777, t_hi=1024, hq=28, hkv=4,
             d=128, dtype="bf16", page=64, budget=32, sink=1, recent=2, sizes=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["reserve", "bounds", "pick", "pick", "attend", "attend", "attend"])
    c = dict(kind=kind, batch=_log(rng, 1, 1024 if kind == "reserve" else 128), sizes=rng.randrange(1 << 30),
             page=rng.choice([16, 32, 64, 128, 256]))
    form = rng.choice(["token", "token", "drafts", "prompt"])
    c["t_hi"] = {"token": 1, "drafts": rng.randint(2, 12), "prompt": _log(rng, 13, 1024)}[form]
    c["t_lo"] = max(1, int(c["t_hi"] * rng.uniform(0.2, 1.0)))
    c["n_hi"] = c["t_hi"] + _log(rng, 1, 130000)
    c["n_lo"] = max(c["t_hi"], int(c["n_hi"] * rng.uniform(0.2, 1.0)))
    if kind == "reserve":
        c["p_hi"] = _log(rng, 1, 16000)
        c["p_lo"] = max(1, int(c["p_hi"] * rng.uniform(0.1, 1.0)))
        c["done"], c["fresh"] = round(rng.choice([0.0, rng.uniform(0.0, 0.4)]), 3), round(rng.uniform(0.0, 0.4), 3)
        c["spare"] = round(rng.choice([rng.uniform(1.0, 3.0), rng.uniform(0.2, 1.0)]), 3)  # (below 1: pages run out)
    else:
        c["hq"], c["hkv"], c["d"] = rng.choice([(4, 4, 64), (14, 2, 64), (16, 16, 128), (28, 4, 128), (32, 8, 128),
                                                (32, 2, 128), (32, 32, 128)])
        if kind != "bounds":
            c["dtype"] = "e4m3" if c["d"] == 128 and rng.random() < 0.4 else "bf16"
            c["budget"] = _log(rng, 2, 128)
            c["sink"] = rng.randint(0, 1)
            c["recent"] = rng.randint(1, max(1, min(4, c["budget"] - c["sink"])))
            c["budget"] = max(c["budget"], 3 if kind == "pick" else 2)
    least = c["t_hi"]
    if kind == "pick":
        least = max(least, 16 * c["page"])
        c["n_hi"] = max(c["n_hi"], least)
        c["n_lo"] = max(c["n_lo"], least)
    while c["batch"] > 1 and _costs_much(c):
        c["batch"] -= 1
    while c["n_hi"] > least and _costs_much(c):
        c["n_hi"] = max(least, c["n_hi"] // 2)
        c["n_lo"] = min(c["n_lo"], c["n_hi"])
    while c["t_hi"] > 1 and _costs_much(c):
        c["t_hi"] //= 2
        c["t_lo"] = min(c["t_lo"], c["t_hi"])
    if kind == "pick":  # the longest request has twice the pages that its queries pick, at least
        c["budget"] = min(c["budget"], _pages(max(_lens(c)[0]), c["page"]) // 2)
        c["recent"] = min(c["recent"], c["budget"] - c["sink"] - 1)
    return c


def _costs_much(case):
    w, kind = work(case), case["kind"]
    pool = 0 if kind in ("reserve", "pick") else sum(_lens(case)[0]) * case["hkv"]
    visits = w["flops"] / (case["hq"] // case["hkv"] * case["d"] * 4) if kind == "attend" else 0
    return w["bytes"] > _MOST[kind] or w["flops"] > _MOST_FLOPS[kind] or pool > _MOST_POOL or visits > _MOST_VISITS


def _lens(case):
    """The request lengths of a case, the last of them new tokens or queries (or both), and those new tokens."""
    r = random.Random(case["sizes"])
    n = [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["batch"])]
    t = [r.randint(case["t_lo"], case["t_hi"]) for _ in range(case["batch"])]
    return n, t


def _turnover(case):
    """Tokens that each request's pages hold, tokens that they are to hold, and the new ones among these."""
    r = random.Random(case["sizes"] + 1)
    held, want, new = [], [], []
    for n, t in zip(*_lens(case)):
        u = r.random()
        if u < case["done"]:
            w, t = 0, 0
        elif u < case["done"] + case["fresh"]:
            n, w = 0, r.randint(case["p_lo"], case["p_hi"])
            t = w
        else:
            w = n + t
        held.append(n)
        want.append(w)
        new.append(t)
    return held, want, new


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _pages(n, page):
    return -(-n // page)


def work(case):
    page = case["page"]
    if case["kind"] == "reserve":
        held, want, new = _turnover(case)
        moved = sum(abs(_pages(w, page) - _pages(h, page)) for h, w in zip(held, want))
        return {"bytes": 16 * case["batch"] + 8 * moved + 8 * sum(new), "flops": 0}
    n, t = _lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "bounds":
        pages = sum(_pages(x, page) - (x - y) // page for x, y in zip(n, t))
        rows = sum(x - (x - y) // page * page for x, y in zip(n, t))
        return {"bytes": hkv * (rows * (d // 2 + d // 16) + pages * (2 * d + 1)), "flops": rows * hkv * d * 3}
    esize, rows, budget = 2 if case["dtype"] == "bf16" else 1, sum(t), case["budget"]
    if case["kind"] == "pick":  # the pages' ranges once for a request whose pages are more than it may pick
        scored = [(_pages(x, page), y) for x, y in zip(n, t) if _pages(x, page) > budget]
        return {"bytes": sum(p for p, _ in scored) * hkv * (2 * d + 1) + rows * (hq * d * esize + 4 * hkv * budget),
                "flops": sum(p * y for p, y in scored) * hq * 2 * 2 * d}
    picked = [min(_pages(x, page), budget) for x in n]  # of a query; of all a request's queries at most all pages
    held = [min(_pages(x, page), y * p) for x, y, p in zip(n, t, picked)]
    return {"bytes": sum(held) * page * hkv * 2 * (d // 2 + d // 16) + rows * (hq * d * (esize + 2) + 4 * hkv * budget),
            "flops": sum(y * p for y, p in zip(t, picked)) * page * hq * d * 4}


# ----------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tables(case, lens, g, more=0):
    """Pages of the pool in random order, a table row for every request (-1 behind its last page), the pages of no
    request."""
    pages = [_pages(x, case["page"]) for x in lens]
    total, width = sum(pages) + more, max(1, max(pages))
    perm = torch.randperm(total, generator=g, device="cuda", dtype=torch.int64).to(torch.int32).cpu().numpy()
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, m in enumerate(pages):
        table[b, :m] = perm[at:at + m]
        at += m
    return table, perm[at:], total


def _rows(shape, g, sigma):
    """Key or value rows: N(0, 1) channels, lognormal norms over the tokens."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x * torch.exp(sigma * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))


def _quantise(y):
    """Rows [..., d] -> packed e2m1 codes and e4m3 scales: a block of 16 channels has its largest magnitude at 6."""
    y = y.unflatten(-1, (-1, 16))
    s = (y.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    a = (y / s.float()[..., None].clamp(min=1e-30)).abs()
    c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    c = (c | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s.view(torch.uint8)


def _pool(case, total, g, salient):
    """A cache's tensors. Every twentieth token or so is one that the queries look for."""
    hkv, d, ps = case["hkv"], case["d"], case["page"]
    c = dict(k_scale=0.25, v_scale=0.125)
    some = max(1, (1 << 26) // (hkv * ps * d))  # (some pages at a time)
    for name in "kv":
        codes = torch.empty((total, hkv, ps, d // 2), dtype=torch.uint8, device="cuda")
        scales = torch.empty((total, hkv, ps, d // 16), dtype=torch.uint8, device="cuda")
        for i in range(0, total, some):
            x = _rows((min(some, total - i), hkv, ps, d), g, 0.5 if name == "k" else 0.2)
            if name == "k":
                hit = torch.rand((x.shape[0], 1, ps, 1), generator=g, device="cuda") < 0.05
                x = x + hit * salient[:, None, :]
            codes[i:i + some], scales[i:i + some] = _quantise(x / c[name + "_scale"])
        c[name + "_codes"], c[name + "_scales"] = codes, scales
    return c


def _ranges(case, total, g, salient):
    """Ranges of pages of keys as _pool makes them: the largest and smallest of a page's normal values, wider where a
    token is one that the queries look for."""
    shape = (total, case["hkv"], case["d"])
    reach = math.sqrt(2.0 * math.log(case["page"]))  # of the largest of so many normal values
    size = torch.exp(0.2 * torch.randn(shape[:2] + (1,), generator=g, device="cuda")) * 4.0
    hit = (torch.rand((total, 1, 1), generator=g, device="cuda") < 0.3) * salient
    hi = size * ((reach + 0.4 * torch.randn(shape, generator=g, device="cuda")).clamp(min=0.1) + hit.clamp(min=0.0))
    lo = -size * ((reach + 0.4 * torch.randn(shape, generator=g, device="cuda")).clamp(min=0.1) - hit.clamp(max=0.0))
    return _whole(hi, lo)


def _positions(n, t):
    """Request and position of every query."""
    req = np.repeat(np.arange(len(n)), t)
    pos = np.concatenate([np.arange(x - y, x) for x, y in zip(n, t)])
    return torch.from_numpy(req).cuda(), torch.from_numpy(pos).cuda()


def _some_picks(case, n, t, g):
    """Pages as a score picks them: the first, the last, and others that neighbouring queries mostly agree on."""
    req, pos = _positions(n, t)
    last = pos // case["page"]
    most = _pages(max(n), case["page"])
    j = torch.arange(most, device="cuda")
    x = torch.rand((len(n), case["hkv"], most), generator=g, device="cuda")[req]
    x = 0.7 * x + 0.3 * torch.rand(x.shape, generator=g, device="cuda")
    x = torch.where((j < case["sink"]) | (j > last[:, None, None] - case["recent"]), 2.0, x)
    x = torch.where(j > last[:, None, None], -1.0, x)
    v, i = torch.topk(x, min(case["budget"], most), dim=-1)
    i = torch.where(v < 0.0, most, i).sort(-1)[0]
    out = torch.full(x.shape[:2] + (case["budget"],), -1, dtype=torch.int32, device="cuda")
    out[..., :i.shape[-1]] = torch.where(i == most, -1, i).to(torch.int32)
    return out


def _queries(case, rows, g, direction):
    q = torch.randn((rows, case["hkv"], case["hq"] // case["hkv"], case["d"]), generator=g, device="cuda")
    q = (q + 0.25 * direction[:, None, :]).reshape(rows, case["hq"], case["d"])
    if case["dtype"] == "bf16":
        return q.to(torch.bfloat16), 1.0
    scale = float(np.float32(float(q.abs().max()) / 448.0))
    return (q / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["kind"] == "reserve":
        held, want, t = _turnover(case)
        need = sum(max(0, _pages(w, case["page"]) - _pages(h, case["page"])) for h, w in zip(held, want))
        # (the pool has pages of requests that are no part of the call, too)
        table, spare, total = _tables(case, held, g, 1024 + max(1, int(need * case["spare"])))
        spare = spare[1024:]
        width = _pages(max(held + want), case["page"]) + 1
        s["table"] = torch.full((len(held), width), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :table.shape[1]] = torch.from_numpy(table[:, :width]).cuda()
        head = seed % total
        ring = np.full(total, -1, np.int32)
        ring[(head + np.arange(len(spare))) % total] = spare
        s["free"] = torch.from_numpy(ring).cuda()
        s["state"] = torch.tensor([head, len(spare)], dtype=torch.int32, device="cuda")
        s["held"], s["want"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (held, want))
    else:
        n, t = _lens(case)
        table, _, total = _tables(case, n, g)
        s["table"] = torch.from_numpy(table).cuda()
        s["lens"] = torch.tensor(n, dtype=torch.int32, device="cuda")
        s["most"] = max(n)
        direction = torch.randn((case["hkv"], case["d"]), generator=g, device="cuda")
    off = _offsets(t)
    s["off_h"], s["off"] = off, torch.from_numpy(off).cuda()
    if case["kind"] == "bounds":
        s.update(_pool(case, total, g, direction))
        s["codes"] = torch.zeros((total, case["hkv"], 2, case["d"]), dtype=torch.int8, device="cuda")
        s["exps"] = torch.zeros((total, case["hkv"]), dtype=torch.int8, device="cuda")
    elif case["kind"] == "pick":
        s["codes"], s["exps"] = _ranges(case, total, g, direction)
        s["q"], _ = _queries(case, int(off[-1]), g, direction)
    elif case["kind"] == "attend":
        s.update(_pool(case, total, g, direction))
        s["q"], s["q_scale"] = _queries(case, int(off[-1]), g, direction)
        s["picked"] = _some_picks(case, n, t, g)
    s["sel"], s["cache"], s["bounds"] = _handles(s)
    return s


def _handles(s):
    """What a user's program keeps: the handle, and the library's view of the cache's and the ranges' tensors."""
    if own:
        from paper_2506_07416_gb300 import select
        case = s["case"]
        most = max(1, int(s["off_h"][-1]))
        sel = select.Selector(case["batch"], most, most, case.get("hq", 4), case.get("hkv", 4), case.get("d", 128),
                              "e4m3" if case.get("dtype") == "e4m3" else "bf16")
        cache = bounds = None
        if "k_codes" in s:
            cache = select.KVCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["k_scale"], s["v_scale"])
        if "codes" in s:
            bounds = select.KeyBounds(s["codes"], s["exps"], case["page"])
        return sel, cache, bounds
    return None, None, None


# ------------------------------------------------------------------------------------------------------ plain forms
def _reserve(s):
    ps, table, free, off = s["case"]["page"], s["table"], s["free"], s["off"].long()
    held, want, new = s["held"].long(), s["want"].long(), off[1:] - off[:-1]
    head, count = s["state"][0].long(), s["state"][1].long()
    total = free.shape[0]
    has, needs = (held + ps - 1) // ps, (want + ps - 1) // ps
    take, give = (needs - has).clamp(min=0), (has - needs).clamp(min=0)
    taken = torch.cumsum(take, 0)
    served = (take == 0) | (taken <= count)
    o = torch.arange(table.shape[1], device=off.device)[None]
    # pages that go back follow the free ones, a request's in order
    back = count + (torch.cumsum(give, 0) - give)[:, None] + o - needs[:, None]
    goes = (o >= needs[:, None]) & (o < has[:, None])
    ring = torch.cat((free, free[:1]))  # (the place behind the last takes what stays)
    ring.scatter_(0, torch.where(goes & (back < total), (head + back) % total, total).flatten(), table.flatten())
    # pages that are taken
    comes = (o >= has[:, None]) & (o < needs[:, None]) & served[:, None]
    fresh = free[(head + (taken - take)[:, None] + o - has[:, None]) % total]
    table.copy_(torch.where(comes, fresh, table))
    free.copy_(ring[:total])
    granted = torch.where(served, want, held)
    used = torch.where(served, take, 0).sum()
    state = torch.stack(((head + used) % total, count - used + torch.minimum(give.sum(), total - count)))
    # slots of the new tokens, the last ones that a request is to hold
    r = torch.arange(int(s["off_h"][-1]), device=off.device)
    b = torch.searchsorted(off, r, right=True) - 1
    pos = want[b] - new[b] + r - off[b]
    page = table[b, (pos // ps).clamp(0, table.shape[1] - 1)].long()
    slots = torch.where(served[b] & (pos >= 0) & (page >= 0), page * ps + pos % ps, -1)
    return {"granted": granted.to(torch.int32), "state": state.to(torch.int32), "slots": slots, "table": table,
            "free": free}


def _values(codes, scales):
    """What packed codes stand for, without the tensor's scale."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                       device=codes.device)
    x = torch.stack((lut[(codes & 15).int()], lut[(codes >> 4).int()]), -1).flatten(-2)
    return (x.unflatten(-1, (-1, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _whole(hi, lo):
    """Ranges [..., d] as whole numbers, outwards, in units of a power of two at which the largest is 64 to 127."""
    m = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
    e = torch.where(m > 0, torch.frexp(m)[1] - 7, 0)
    e = torch.where(m > 127.0 * torch.exp2(e.float()), e + 1, e)
    unit = torch.exp2(-e.float())
    return torch.stack((torch.ceil(hi * unit), torch.floor(lo * unit)), -2).to(torch.int8), e[..., 0].to(torch.int8)


def _bounds(s):
    ps, off, lens = s["case"]["page"], s["off"], s["lens"].long()
    new = (off[1:] - off[:-1]).long()
    last = (lens - 1) // ps
    most = _pages(int((s["off_h"][1:] - s["off_h"][:-1]).max()), ps) + 1
    # pages behind the last one repeat it: the same bytes to the same place
    o = torch.minimum(((lens - new) // ps)[:, None] + torch.arange(most, device=off.device), last[:, None])
    page = torch.gather(s["table"], 1, o).long()
    k = _values(s["k_codes"][page], s["k_scales"][page])  # [B, pages, Hkv, ps, d]
    there = o[..., None] * ps + torch.arange(ps, device=off.device) < lens[:, None, None]
    there = there[:, :, None, :, None]
    hi, lo = torch.where(there, k, -math.inf).amax(-2), torch.where(there, k, math.inf).amin(-2)
    s["codes"][page], s["exps"][page] = _whole(hi, lo)
    return {"codes": s["codes"], "exps": s["exps"]}


def _pick(s):
    case, off, lens = s["case"], s["off"], s["lens"].long()
    hq, hkv, ps, budget = case["hq"], case["hkv"], case["page"], case["budget"]
    t_most = int((s["off_h"][1:] - s["off_h"][:-1]).max())
    i = torch.arange(t_most, device=off.device)
    t = (off[1:] - off[:-1])[:, None]
    row = (off[:-1, None] + i).clamp(max=s["q"].shape[0] - 1).long()  # [B, T]
    q = s["q"].float() if case["dtype"] == "bf16" else s["q"].view(torch.float8_e4m3fn).float()
    # the queries of a key head as whole numbers in units of a power of two
    q = q.unflatten(1, (hkv, hq // hkv))
    e = torch.frexp(q.abs().amax((-1, -2), keepdim=True))[1].clamp(min=-119)
    q = torch.round(q * torch.exp2((7 - e).float())).clamp(-127.0, 127.0)[row]  # [B, T, Hkv, G, d]
    q = torch.cat((q.clamp(min=0.0), q.clamp(max=0.0)), -1).permute(0, 2, 1, 3, 4).flatten(2, 3)
    pages = _pages(s["most"], ps)
    page = s["table"][:, :pages].clamp(min=0).long()
    k = s["codes"][page].float().flatten(-2).permute(0, 2, 3, 1)  # [B, Hkv, 2d, pages]
    x = (q @ k).unflatten(2, (t_most, hq // hkv)).amax(3)  # whole numbers below 2^24: exact in any order
    x = x * torch.exp2(s["exps"][page].float()).permute(0, 2, 1)[:, :, None]  # [B, Hkv, T, pages]
    last = ((lens[:, None] - t + i) // ps)[:, None, :, None]
    j = torch.arange(pages, device=off.device)
    x = torch.where((j < case["sink"]) | (j > last - case["recent"]), math.inf, x)
    x = torch.where(j > last, -math.inf, x)
    v, order = torch.sort(x, dim=-1, descending=True, stable=True)
    width = min(budget, pages)
    order = torch.where(v == -math.inf, pages, order)[..., :width].sort(-1)[0]
    out = torch.full(order.shape[:-1] + (budget,), -1, dtype=torch.int32, device=off.device)
    out[..., :width] = torch.where(order == pages, -1, order).to(torch.int32)
    r = torch.arange(s["q"].shape[0], device=off.device)
    b = torch.searchsorted(off, r.to(torch.int32), right=True) - 1
    return {"picked": out.transpose(1, 2)[b, r - off[b]].contiguous()}


def _attend(s):
    case, off, lens, picked = s["case"], s["off"], s["lens"].long(), s["picked"].long()
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["page"]
    r = torch.arange(s["q"].shape[0], device=off.device)
    b = torch.searchsorted(off, r.to(torch.int32), right=True) - 1
    pos = lens[b] - (off[b + 1] - r)  # the last queries stand at the last positions
    page = s["table"][b[:, None, None], picked.clamp(min=0)].long()  # [R, Hkv, budget]
    head = torch.arange(hkv, device=off.device)[:, None]
    k, v = (_values(s[x + "_codes"][page, head], s[x + "_scales"][page, head]).flatten(2, 3) for x in "kv")
    at = picked[..., None] * ps + torch.arange(ps, device=off.device)
    sees = ((at <= pos[:, None, None, None]) & (picked >= 0)[..., None]).flatten(2)[:, :, None]  # [R, Hkv, 1, keys]
    q = s["q"].float() if case["dtype"] == "bf16" else s["q"].view(torch.float8_e4m3fn).float() * s["q_scale"]
    x = q.unflatten(1, (hkv, hq // hkv)) @ k.transpose(-1, -2) * (s["k_scale"] / math.sqrt(d))
    x = torch.where(sees, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-38)
    return {"out": (p @ torch.where(sees.transpose(-1, -2), v, 0.0) * s["v_scale"]).flatten(1, 2).to(torch.bfloat16)}


_PLAIN = {"reserve": _reserve, "bounds": _bounds, "pick": _pick, "attend": _attend}


# -------------------------------------------------------------------------------------------------------------- run
def run(s):
    if own:
        return _OWN[s["case"]["kind"]](s)
    return _PLAIN[s["case"]["kind"]](s)


def _own_reserve(s):
    granted, state, slots = s["sel"].cache_reserve(s["table"], s["held"], s["want"], s["free"], s["state"],
                                                   s["case"]["page"], offsets=s["off"], offsets_h=s["off_h"])
    return {"granted": granted, "state": state, "slots": slots, "table": s["table"], "free": s["free"]}


def _own_bounds(s):
    s["sel"].cache_bounds(s["cache"], s["bounds"], s["table"], s["lens"], s["off"], offsets_h=s["off_h"])
    return {"codes": s["codes"], "exps": s["exps"]}


def _own_pick(s):
    case = s["case"]
    return {"picked": s["sel"].cache_pick(s["bounds"], s["table"], s["lens"], s["q"], s["off"], s["most"],
                                          case["budget"], case["sink"], case["recent"], offsets_h=s["off_h"])}


def _own_attend(s):
    return {"out": s["sel"].cache_attend_picked(s["cache"], s["table"], s["lens"], s["q"], s["off"], s["picked"],
                                                q_scale=s["q_scale"], offsets_h=s["off_h"])}


_OWN = {"reserve": _own_reserve, "bounds": _own_bounds, "pick": _own_pick, "attend": _own_attend}


# ------------------------------------------------------------------------------------------------------------ exact
def _e2m1(c):
    e, m = (c >> 1) & 3, (c & 1).double()
    x = torch.where(e == 0, 0.5 * m, torch.exp2(e.double() - 1.0) * (1.0 + 0.5 * m))
    return torch.where(c >= 8, -x, x)


def _e4m3(c):
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e == 0, m / 8 * 2.0 ** -6, torch.exp2(e.double() - 7.0) * (1.0 + m / 8))
    return torch.where(c >= 128, -x, x)


def exact(case, seed):
    if case["kind"] != "attend":  # whole numbers: the same in any precision
        return None
    s = prepare(case, seed)
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["page"]
    n, t = _lens(case)
    q = s["q"].double() if case["dtype"] == "bf16" else _e4m3(s["q"].long()) * s["q_scale"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    some = max(1, (1 << 26) // (case["budget"] * ps * d))  # (some queries at a time)
    for b in range(case["batch"]):
        for first in range(0, t[b], some):
            last = min(t[b], first + some)
            rows = slice(int(s["off_h"][b]) + first, int(s["off_h"][b]) + last)
            place = torch.arange(n[b] - t[b] + first, n[b] - t[b] + last, device="cuda")
            for h in range(hkv):
                o = s["picked"][rows, h].long()
                pos = (o[:, :, None] * ps + torch.arange(ps, device="cuda")).flatten(1)
                hidden = (pos > place[:, None]) | (o < 0).repeat_interleave(ps, 1)
                x = {}
                for name in "kv":
                    page = s["table"][b].long()[o.clamp(min=0)]
                    c, f = s[name + "_codes"][page, h].long(), _e4m3(s[name + "_scales"][page, h].long())
                    c = torch.stack((_e2m1(c % 16), _e2m1(c // 16)), -1).flatten(-2)
                    x[name] = (c * f.repeat_interleave(16, -1) * s[name + "_scale"]).flatten(1, 2)
                heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                y = torch.einsum("rgd,rkd->rgk", q[rows, heads], x["k"]) / math.sqrt(d)
                p = torch.softmax(y.masked_fill(hidden[:, None], -math.inf), -1)
                out[rows, heads] = torch.einsum("rgk,rkd->rgd", p, x["v"])
    return {"out": out}
