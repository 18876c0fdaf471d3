"""The calls of a decoder's 4-bit K/V cache whose speed is tracked: rows quantised into the cache (`cache_append`),
attention that reads it and adds up the weight every cached token receives (`cache_attend`), eviction by that weight
(`cache_evict`), and the verification of drafted tokens (`verify`).

The cache is paged. A page holds, for each key head, `page` rows of e2m1 codes (two to a byte, the even channel in the
low four bits) and one e4m3 scale for every 16 channels of a row; a tensor has one float scale over these. A request's
pages stand in its row of a table. Sizes are those of this repository's workloads after token selection (1 to 128
requests, 460 to 1800 kept visual tokens with the text behind them, 4/4 to 32/32 heads of 64 or 128), and the decoding
that follows: one token, a handful of drafts, a chunk of a prompt, caches of up to 128 Ki tokens.

A case's lengths are drawn from its own `sizes` number, so that a case is a dict of plain values.
"""
import math
import random

import numpy as np
import torch

own = False  # False: the operators from elementary torch operations; True: the library's calls

_MOST = {"append": 3.0e9, "attend": 6.6e8, "evict": 4.5e8, "verify": 7.0e7}  # bytes of a drawn case
_MOST_FLOPS = 1.4e11


# ------------------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of one request, 16 heads: nothing but latency
        dict(name="append_token", kind="append", batch=1, n_lo=523, n_hi=523, t_lo=1, t_hi=1, sizes=1, hq=16, hkv=16,
             d=128, dtype="bf16", page=16, picked=False),
        # the prompts of the largest batch after selection: 1036 kept visual and 64 text tokens for each of 128 requests
        dict(name="append_prompts", kind="append", batch=128, n_lo=0, n_hi=0, t_lo=1100, t_hi=1100, sizes=2, hq=32,
             hkv=32, d=128, dtype="bf16", page=64, picked=False),
        # the kept rows of a ragged 8-bit batch, picked by the top-k's indices out of all visual rows
        dict(name="append_kept_fp8", kind="append", batch=32, n_lo=19, n_hi=48, t_lo=115, t_hi=691, sizes=3, hq=32,
             hkv=32, d=128, dtype="e4m3", page=32, picked=True),
        # a decoded token of one request: latency
        dict(name="attend_token", kind="attend", batch=1, n_lo=524, n_hi=524, t_lo=1, t_hi=1, sizes=4, hq=16, hkv=16,
             d=128, dtype="bf16", page=16, weights=True),
        # a decoded token of every request of the largest batch
        dict(name="attend_token_sweep", kind="attend", batch=128, n_lo=1101, n_hi=1164, t_lo=1, t_hi=1, sizes=5, hq=32,
             hkv=32, d=128, dtype="bf16", page=64, weights=True),
        # a decoded token over few very long caches with grouped heads, odd lengths
        dict(name="attend_token_long", kind="attend", batch=4, n_lo=30001, n_hi=131071, t_lo=1, t_hi=1, sizes=6, hq=28,
             hkv=4, d=128, dtype="bf16", page=128, weights=True),
        # drafted tokens of a ragged 8-bit batch, one to eight a request
        dict(name="attend_drafts_fp8", kind="attend", batch=32, n_lo=700, n_hi=8200, t_lo=1, t_hi=8, sizes=7, hq=32,
             hkv=8, d=128, dtype="e4m3", page=32, weights=True),
        # a chunk of a long prompt over the part that is cached
        dict(name="attend_prompt", kind="attend", batch=2, n_lo=5000, n_hi=8191, t_lo=777, t_hi=1024, sizes=8, hq=28,
             hkv=4, d=128, dtype="bf16", page=64, weights=False),
        # one request that is a few tokens over its budget
        dict(name="evict_few", kind="evict", batch=1, n_lo=560, n_hi=560, budget=524, sink=4, recent=64, sizes=9, hq=16,
             hkv=16, d=128, page=16),
        # a batch cut back to a quarter, some requests already below
        dict(name="evict_batch", kind="evict", batch=64, n_lo=1500, n_hi=8191, budget=2048, sink=4, recent=256,
             sizes=10, hq=32, hkv=8, d=128, page=64),
        # four drafts of one request against a small vocabulary: latency
        dict(name="verify_one", kind="verify", batch=1, t_lo=4, t_hi=4, sizes=11, vocab=32000, dtype="f32", drafts=True),
        # up to eight drafts of every request of a batch, a large vocabulary of odd size
        dict(name="verify_batch", kind="verify", batch=64, t_lo=0, t_hi=8, sizes=12, vocab=128003, dtype="f32",
             drafts=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "evict", "evict", "verify"])
    if kind == "verify":
        c = dict(kind=kind, batch=_log(rng, 1, 64), t_lo=0, t_hi=rng.randint(1, 8), sizes=rng.randrange(1 << 30),
                 vocab=_log(rng, 1000, 160000), dtype=rng.choice(["f32", "f32", "bf16"]), drafts=rng.random() < 0.8)
        c["t_lo"] = rng.randint(0, c["t_hi"])
        while c["batch"] > 1 and work(c)["bytes"] > _MOST[kind]:
            c["batch"] -= 1
        return c
    hq, hkv, d = rng.choice([(4, 4, 64), (14, 2, 64), (16, 16, 128), (28, 4, 128), (32, 8, 128), (32, 32, 128)])
    c = dict(kind=kind, batch=_log(rng, 1, 128), sizes=rng.randrange(1 << 30), hq=hq, hkv=hkv, d=d,
             page=rng.choice([16, 32, 64, 128]))
    if kind == "evict":
        c["n_hi"] = _log(rng, 40, 40000)
        c["n_lo"] = max(1, int(c["n_hi"] * rng.uniform(0.1, 1.0)))
        c["budget"] = max(8, int(c["n_hi"] * rng.uniform(0.1, 0.95)))
        c["sink"] = rng.randint(0, 4)
        c["recent"] = rng.randint(0, c["budget"] // 2 - 2)
    else:
        c["dtype"] = "e4m3" if d == 128 and rng.random() < 0.4 else "bf16"
        if kind == "append":
            c["n_lo"], c["n_hi"], c["picked"] = 0, rng.choice([0, 700]), rng.random() < 0.4
            c["t_hi"] = _log(rng, 1, 3000)
            c["t_lo"] = max(1, int(c["t_hi"] * rng.uniform(0.2, 1.0)))
        else:
            c["weights"] = rng.random() < 0.7
            form = rng.choice(["token", "token", "drafts", "prompt"])
            c["t_hi"] = {"token": 1, "drafts": rng.randint(2, 12), "prompt": _log(rng, 13, 1024)}[form]
            c["t_lo"] = max(1, int(c["t_hi"] * rng.uniform(0.2, 1.0)))
            c["n_hi"] = c["t_hi"] + _log(rng, 1, 100000)
            c["n_lo"] = max(c["t_hi"], int(c["n_hi"] * rng.uniform(0.2, 1.0)))
    while c["batch"] > 1 and (work(c)["bytes"] > _MOST[kind] or work(c)["flops"] > _MOST_FLOPS):
        c["batch"] -= 1
    while kind == "attend" and work(c)["flops"] > _MOST_FLOPS:
        c["n_hi"] = max(c["t_hi"], c["n_hi"] // 2)
        c["n_lo"] = min(c["n_lo"], c["n_hi"])
    return c


def _lens(case):
    """The request lengths of a case: cached tokens (before an append, else with the queries' own) and new tokens."""
    r = random.Random(case["sizes"])
    n = [r.randint(case.get("n_lo", 0), case.get("n_hi", 0)) for _ in range(case["batch"])]
    t = [r.randint(case.get("t_lo", 0), case.get("t_hi", 0)) for _ in range(case["batch"])]
    return n, t


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def work(case):
    n, t = _lens(case)
    if case["kind"] == "verify":
        row = case["vocab"] * (4 if case["dtype"] == "f32" else 2)
        rows = sum(2 if case["drafts"] and x else 1 for x in t)  # the row that is sampled, of both models
        return {"bytes": rows * row + 12 * (sum(t) + len(t)), "flops": 3 * rows * case["vocab"]}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    held = hkv * 2 * (d // 2 + d // 16)  # bytes of a cached token
    if case["kind"] == "evict":
        kept = sum(min(x, case["budget"]) for x in n)
        return {"bytes": 4 * sum(n) + kept * (2 * held + 4 + 4), "flops": 0}
    esize = 2 if case["dtype"] == "bf16" else 1
    if case["kind"] == "append":  # rows in; codes, scales and the values that they stand for out
        rows = sum(t)
        return {"bytes": rows * (2 * hkv * d * (esize + 2) + held + 4), "flops": rows * 2 * hkv * d * 4}
    seen = sum(x * y - y * (y - 1) // 2 for x, y in zip(n, t))
    return {"bytes": sum(n) * (held + (8 if case["weights"] else 0)) + sum(t) * hq * d * (esize + 2),
            "flops": 4 * seen * hq * d}


# ----------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tables(case, lens, g):
    """Pages of the pool in random order, a table row for every request (-1 behind its last page)."""
    pages = [-(-x // case["page"]) for x in lens]
    total, width = sum(pages), max(1, max(pages))
    perm = torch.randperm(total, generator=g, device="cuda", dtype=torch.int64).to(torch.int32).cpu().numpy()
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, m in enumerate(pages):
        table[b, :m] = perm[at:at + m]
        at += m
    return table, total


def _rows(shape, g, sigma):
    """Key or value rows: N(0, 1) channels, lognormal norms over the tokens."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x * torch.exp(sigma * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))


def _encode(x, dtype):
    """bf16 values, or e4m3 codes under one scale (absmax / 448) -> (tensor, scale)."""
    if dtype == "bf16":
        return x.to(torch.bfloat16), 1.0
    scale = float(np.float32(float(x.abs().max()) / 448.0))
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _pool(case, total, g, salient=None):
    """A cache's tensors: filled pages for the calls that read it, untouched ones for the append."""
    hkv, d, ps = case["hkv"], case["d"], case["page"]
    c = dict(k_scale=0.25, v_scale=0.125)
    for name in "kv":
        if case["kind"] == "append":
            c[name + "_codes"] = torch.zeros((total, hkv, ps, d // 2), dtype=torch.uint8, device="cuda")
            c[name + "_scales"] = torch.zeros((total, hkv, ps, d // 16), dtype=torch.uint8, device="cuda")
            continue
        codes, scales, some = [], [], max(1, (1 << 26) // (hkv * ps * d))  # (some pages at a time)
        for i in range(0, total, some):
            x = _rows((min(some, total - i), hkv, ps, d), g, 0.5 if name == "k" else 0.2)
            if name == "k":  # every twentieth token or so is one that the queries look for
                hit = torch.rand((x.shape[0], 1, ps, 1), generator=g, device="cuda") < 0.05
                x = x + hit * salient[:, None, :]
            y, s = _quantise(x / c[name + "_scale"])
            codes.append(y)
            scales.append(s)
        c[name + "_codes"], c[name + "_scales"] = torch.cat(codes), torch.cat(scales)
    # what earlier calls have added up: heavy-tailed, most tokens next to nothing
    c["weights"] = torch.exp(2.0 * torch.randn((total, ps), generator=g, device="cuda") - 5.0)
    return c


def prepare(case, seed):
    g = _gen(seed)
    n, t = _lens(case)
    off = _offsets(t)
    s = dict(case=case, off_h=off, off=torch.from_numpy(off).cuda(), sel=_selector(case, n, t))
    if case["kind"] == "verify":
        rows, v = int(off[-1]), case["vocab"]
        kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        logits = 3.0 * torch.randn((rows + len(t), v), generator=g, device="cuda")
        req = torch.from_numpy(np.repeat(np.arange(len(t)), t).astype(np.int64)).cuda()
        near = logits[torch.arange(rows, device="cuda") + req]
        near = near + 0.7 * torch.randn(near.shape, generator=g, device="cuda")  # the draft model is a little off
        s["p"] = torch.softmax(logits, -1).to(kind)
        q = torch.softmax(near, -1).to(kind)
        x = torch.multinomial(q.float(), 1, generator=g)[:, 0] if rows else req
        s["tokens"] = x.to(torch.int32)
        s["q"] = q if case["drafts"] else None
        s["u"] = torch.rand(rows, generator=g, device="cuda")
        s["u_last"] = torch.rand(len(t), generator=g, device="cuda")
        return s
    after = [x + y for x, y in zip(n, t)] if case["kind"] == "append" else n
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "evict":  # the rows that stay move to pages of their own (the old ones may be shared)
        both, total = _tables(case, n + [min(x, case["budget"]) for x in n], g)
        table, to = both[:len(n)], both[len(n):, :max(1, -(-min(max(n), case["budget"]) // case["page"]))]
        s["to"] = torch.from_numpy(np.ascontiguousarray(to)).cuda()
        s["budget"], s["sink"], s["recent"] = case["budget"], case["sink"], case["recent"]
    else:
        table, total = _tables(case, after, g)
    s["table"] = torch.from_numpy(table).cuda()
    s["lens"] = torch.from_numpy(np.asarray(n, np.int32)).cuda()
    s["most"] = max(n)
    direction = torch.randn((hkv, d), generator=g, device="cuda")
    s.update(_pool(case, total, g, direction))
    if case["kind"] == "attend":
        q = torch.randn((int(off[-1]), hkv, hq // hkv, d), generator=g, device="cuda") + 0.25 * direction[:, None, :]
        s["q"], s["q_scale"] = _encode(q.reshape(-1, hq, d), case["dtype"])
        s["weights_next"] = s["weights"].clone() if case["weights"] else None
    if case["kind"] == "append":
        source = int(off[-1]) * (5 if case["picked"] else 1)
        s["k"], s["k_in"] = _encode(_rows((source, hkv, d), g, 0.5), case["dtype"])
        s["v"], s["v_in"] = _encode(_rows((source, hkv, d), g, 0.2), case["dtype"])
        s["rows"] = None
        if case["picked"]:  # ascending, as a top-k gives them
            s["rows"] = torch.randperm(source, generator=g, device="cuda")[:int(off[-1])].sort()[0].to(torch.int32)
    s["cache"] = _cache(s)
    return s


def _selector(case, n, t):
    """The handle that a user's program keeps."""
    if own:
        from paper_2506_07416_gb300 import select
        most = max(1, sum(n) + sum(t))
        return select.Selector(case["batch"], most, most, case.get("hq", 4), case.get("hkv", 4), case.get("d", 128),
                               "e4m3" if case.get("dtype") == "e4m3" else "bf16")
    return None


def _cache(s):
    """The library's view of the cache's tensors."""
    if own:
        from paper_2506_07416_gb300 import select
        return select.KVCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["k_scale"], s["v_scale"],
                              weights=s["weights"])
    return None


# ------------------------------------------------------------------------------------------------------ plain forms
def _quantise(y):
    """Rows [..., d] -> packed e2m1 codes and e4m3 scales: a block of 16 channels has its largest magnitude at 6."""
    y = y.unflatten(-1, (-1, 16))
    s = (y.abs().amax(-1) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    z = y / s.float()[..., None]
    a = z.abs()
    # round to nearest, a tie to the even code
    c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    c = torch.where(s.float()[..., None] == 0.0, torch.zeros_like(c), c) | (torch.signbit(y).to(torch.uint8) << 3)
    c = c.flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s.view(torch.uint8)


def _values(codes, scales):
    """What packed codes stand for, without the tensor's scale."""
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                       device=codes.device)
    x = torch.stack((lut[(codes & 15).int()], lut[(codes >> 4).int()]), -1).flatten(-2)
    return (x.unflatten(-1, (-1, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _places(table, page, pos):
    """Page and slot of the positions [B, L] (any place of the pool for those behind a request's pages)."""
    p = torch.gather(table, 1, (pos // page).clamp(max=table.shape[1] - 1).expand(table.shape[0], -1))
    return p.clamp(min=0).long(), (pos % page).expand(table.shape[0], -1).long()


def _append(s):
    case, off = s["case"], s["off"]
    r = torch.arange(int(s["off_h"][-1]), device=off.device)
    b = torch.searchsorted(off, r.to(torch.int32), right=True) - 1
    pos = s["lens"][b].long() + r - off[b]
    page, slot = s["table"][b, pos // case["page"]].long(), pos % case["page"]
    stored = []
    for name in "kv":
        x = s[name] if s["rows"] is None else s[name][s["rows"].long()]
        x = x.float() if case["dtype"] == "bf16" else x.view(torch.float8_e4m3fn).float() * s[name + "_in"]
        codes, scales = _quantise(x / s[name + "_scale"])
        s[name + "_codes"][page, :, slot] = codes
        s[name + "_scales"][page, :, slot] = scales
        stored.append((_values(codes, scales) * s[name + "_scale"]).to(torch.bfloat16))
    s["weights"][page, slot] = 0.0
    return {"lens": s["lens"] + (off[1:] - off[:-1]), "k": stored[0], "v": stored[1]}


def _attend(s):
    case, off, lens = s["case"], s["off"], s["lens"]
    hq, hkv, d, most = case["hq"], case["hkv"], case["d"], s["most"]
    t_most = int((s["off_h"][1:] - s["off_h"][:-1]).max())
    pos = torch.arange(most, device=off.device)[None]
    page, slot = _places(s["table"], case["page"], pos)
    k, v = (_values(s[x + "_codes"][page, :, slot], s[x + "_scales"][page, :, slot]) for x in "kv")  # [B, L, Hkv, d]
    there = pos < lens[:, None]
    v = torch.where(there[..., None, None], v, 0.0)
    i = torch.arange(t_most, device=off.device)
    t = (off[1:] - off[:-1])[:, None]
    row = (off[:-1, None] + i.clamp(max=t_most)).clamp(max=s["q"].shape[0] - 1).long()  # [B, T]
    q = s["q"][row]
    q = q.float() if case["dtype"] == "bf16" else q.view(torch.float8_e4m3fn).float() * s["q_scale"]
    q = q.unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [B, Hkv, G*T, d]
    x = q @ k.permute(0, 2, 3, 1) * (s["k_scale"] / math.sqrt(d))
    x = x.unflatten(2, (hq // hkv, t_most))
    sees = there[:, None] & (pos[:, None] <= (lens[:, None] - t + i)[..., None]) & (i < t)[..., None]  # [B, T, L]
    x = torch.where(sees[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-38)
    o = p.flatten(2, 3) @ v.permute(0, 2, 1, 3) * s["v_scale"]  # [B, Hkv, G*T, d]
    o = o.unflatten(2, (hq // hkv, t_most)).permute(0, 3, 1, 2, 4).flatten(2, 3)
    r = torch.arange(s["q"].shape[0], device=off.device)
    b = torch.searchsorted(off, r.to(torch.int32), right=True) - 1
    out = {"out": o[b, r - off[b]].to(torch.bfloat16)}
    if case["weights"]:
        w = torch.where(there, p.sum((1, 2, 3)) / hq, 0.0)
        flat = s["weights"].flatten().clone()
        flat.scatter_add_(0, (page * case["page"] + slot).flatten(), w.flatten())
        s["weights_next"].copy_(flat.view_as(s["weights"]))
        out["weights"] = s["weights_next"]
    return out


def _evict(s):
    case, lens, budget = s["case"], s["lens"].long(), s["budget"]
    pos = torch.arange(s["most"], device=lens.device)[None]
    page, slot = _places(s["table"], case["page"], pos)
    w = s["weights"][page, slot]
    there = pos < lens[:, None]
    kept = lens.clamp(max=budget)
    # the order in which tokens stay: protected ones, numbers from the largest on, NaN; equal ones by their place
    tier = torch.where(torch.isnan(w), 2, 1)
    tier = torch.where((pos < s["sink"]) | (pos >= lens[:, None] - s["recent"]) | (lens <= budget)[:, None], 0, tier)
    tier = torch.where(there, tier, 3)
    order = torch.sort(torch.where(torch.isnan(w), 0.0, w), dim=1, descending=True, stable=True)[1]
    order = order.gather(1, torch.sort(tier.gather(1, order), dim=1, stable=True)[1])
    stays = torch.zeros_like(there).scatter_(1, order, pos < kept[:, None])
    to = torch.where(stays, torch.cumsum(stays, 1) - 1, budget)
    idx = torch.full((lens.shape[0], budget + 1), -1, dtype=torch.int32, device=lens.device)
    idx.scatter_(1, to, pos.expand_as(to).to(torch.int32))
    idx = idx[:, :budget].contiguous()
    # rows behind the last kept one repeat it: the same bytes to the same place
    width = min(budget, s["most"])
    i = torch.minimum(torch.arange(width, device=lens.device)[None], kept[:, None] - 1)
    j = idx.gather(1, i).long()
    p_from, s_from = page.gather(1, j), slot.gather(1, j)
    p_to, s_to = s["to"].gather(1, i // case["page"]).long(), i % case["page"]
    for x in ("k_codes", "k_scales", "v_codes", "v_scales"):
        s[x][p_to, :, s_to] = s[x][p_from, :, s_from]
    s["weights"][p_to, s_to] = s["weights"][p_from, s_from]
    return {"kept": idx, "lens": kept.to(torch.int32), **_held(s)}


def _held(s):
    """The cache after rows have moved. They move byte for byte, so what is held is told by its bytes."""
    return {x: s[x] for x in ("k_codes", "k_scales", "v_codes", "v_scales", "weights")}


def _verify(s):
    off, x = s["off"].long(), s["tokens"].long()
    n_req = off.shape[0] - 1
    t = off[1:] - off[:-1]
    r = torch.arange(x.shape[0], device=off.device)
    b = torch.searchsorted(off, r, right=True) - 1
    p_x = s["p"][r + b, x].double()
    q_x = s["q"][r, x].double() if s["q"] is not None else torch.ones_like(p_x)
    refused = ~(s["u"].double() * q_x < p_x)
    accepted = t.scatter_reduce(0, b, torch.where(refused, r - off[b], t[b]), "amin")
    at = off[:-1] + torch.arange(n_req, device=off.device) + accepted
    p = s["p"][at].double()
    row = (off[:-1] + accepted).clamp(max=max(0, x.shape[0] - 1))
    less = (accepted < t)[:, None]
    if x.shape[0] == 0:
        w = p
    elif s["q"] is not None:
        w = torch.where(less, p - s["q"][row].double(), p)
    else:  # the draft model is certain of its token
        w = torch.where(less & (torch.arange(p.shape[1], device=p.device) == x[row][:, None]), 0.0, p)
    w = torch.where(w > 0, w, 0.0)
    p = torch.where(p > 0, p, 0.0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p)
    c = torch.cumsum(w, 1)
    hit = (c > s["u_last"].double()[:, None] * c[:, -1:]) & (w > 0)
    place = torch.arange(w.shape[1], device=w.device)
    first = torch.where(hit, place, w.shape[1]).amin(1)
    last = torch.where(w > 0, place, -1).amax(1)
    token = torch.where(first < w.shape[1], first, last).to(torch.int32)
    tokens = torch.full((x.shape[0] + n_req,), -1, dtype=torch.int32, device=x.device)
    tokens[r + b] = torch.where(r - off[b] < accepted[b], x, -1).to(torch.int32)
    tokens[at] = token
    return {"accepted": accepted.to(torch.int32), "tokens": tokens}


_PLAIN = {"append": _append, "attend": _attend, "evict": _evict, "verify": _verify}


# -------------------------------------------------------------------------------------------------------------- run
def run(s):
    if own:
        return _OWN[s["case"]["kind"]](s)
    return _PLAIN[s["case"]["kind"]](s)


def _own_append(s):
    lens, k, v = s["sel"].cache_append(s["cache"], s["table"], s["lens"], s["k"], s["v"], s["off"], rows=s["rows"],
                                       k_in_scale=s["k_in"], v_in_scale=s["v_in"], offsets_h=s["off_h"], stored=True)
    return {"lens": lens, "k": k, "v": v}


def _own_attend(s):
    out = {"out": s["sel"].cache_attend(s["cache"], s["table"], s["lens"], s["q"], s["off"], s["most"],
                                        q_scale=s["q_scale"], weights_out=s["weights_next"], offsets_h=s["off_h"])}
    if s["case"]["weights"]:
        out["weights"] = s["weights_next"]
    return out


def _own_evict(s):
    kept, lens = s["sel"].cache_evict(s["cache"], s["table"], s["lens"], s["most"], s["budget"], s["sink"], s["recent"],
                                      to_table=s["to"])
    return {"kept": kept, "lens": lens, **_held(s)}


def _own_verify(s):
    accepted, tokens = s["sel"].verify(s["tokens"], s["p"], s["u"], s["u_last"], s["off"], draft_probs=s["q"],
                                       offsets_h=s["off_h"])
    return {"accepted": accepted, "tokens": tokens}


_OWN = {"append": _own_append, "attend": _own_attend, "evict": _own_evict, "verify": _own_verify}


# ------------------------------------------------------------------------------------------------------------ exact
def _e2m1(c):
    e, m = (c >> 1) & 3, (c & 1).double()
    x = torch.where(e == 0, 0.5 * m, torch.exp2(e.double() - 1.0) * (1.0 + 0.5 * m))
    return torch.where(c >= 8, -x, x)


def _e4m3(c):
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e == 0, m / 8 * 2.0 ** -6, torch.exp2(e.double() - 7.0) * (1.0 + m / 8))
    return torch.where(c >= 128, -x, x)


def _nearest(x, grid):
    """Each x's nearest value of an ascending grid, a tie to the value of even place."""
    i = torch.searchsorted(grid, x).clamp(1, grid.shape[0] - 1)
    lo, hi = grid[i - 1], grid[i]
    up = (hi - x < x - lo) | ((hi - x == x - lo) & (i % 2 == 0))
    return torch.where(up, hi, lo)


def _exact_append(s, case):
    codes = torch.arange(127, device="cuda")
    fine, coarse = _e4m3(codes), _e2m1(torch.arange(8, device="cuda"))
    out = {"lens": None}
    for name in "kv":
        x = s[name] if s["rows"] is None else s[name][s["rows"].long()]
        got = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for i in range(0, x.shape[0], 4096):
            y = x[i:i + 4096]
            y = y.double() if case["dtype"] == "bf16" else _e4m3(y.long()) * s[name + "_in"]
            y = (y / s[name + "_scale"]).reshape(y.shape[0], -1, 16)
            block = _nearest(y.abs().amax(-1) / 6, fine)[..., None]
            z = torch.where(block > 0, _nearest((y.abs() / block).clamp(max=6.0), coarse) * block, 0.0)
            got[i:i + 4096] = (torch.sign(y) * z).reshape(got[i:i + 4096].shape) * s[name + "_scale"]
        out[name] = got
    return out


def _exact_rows(s, name, b, n, page):
    """Rows [n, Hkv, d] of a request in 64 bits."""
    pos = torch.arange(n, device="cuda")
    p, i = s["table"][b].long()[pos // page], pos % page
    c, f = s[name + "_codes"][p, :, i].long(), _e4m3(s[name + "_scales"][p, :, i].long())
    x = torch.stack((_e2m1(c % 16), _e2m1(c // 16)), -1).flatten(-2)
    return x * f.repeat_interleave(16, -1) * s[name + "_scale"]


def _exact_attend(s, case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    n, t = _lens(case)
    q = s["q"].double() if case["dtype"] == "bf16" else _e4m3(s["q"].long()) * s["q_scale"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    weights = s["weights"].double()
    for b in range(case["batch"]):
        k, v = (_exact_rows(s, x, b, n[b], case["page"]) for x in "kv")
        rows = slice(int(s["off_h"][b]), int(s["off_h"][b + 1]))
        last = torch.arange(t[b], device="cuda") + n[b] - t[b]
        pos = torch.arange(n[b], device="cuda")
        total = torch.zeros(n[b], dtype=torch.float64, device="cuda")
        for h in range(hq):
            x = q[rows, h] @ k[:, h // (hq // hkv)].T / math.sqrt(d)
            p = torch.softmax(x.masked_fill(pos[None] > last[:, None], -math.inf), -1)
            out[rows, h] = p @ v[:, h // (hq // hkv)]
            total += p.sum(0) / hq
        weights[s["table"][b].long()[pos // case["page"]], pos % case["page"]] += total
    return {"out": out, "weights": weights} if case["weights"] else {"out": out}


def exact(case, seed):
    if case["kind"] in ("evict", "verify"):  # whole numbers and moved bytes: the same in any precision
        return None
    s = prepare(case, seed)
    return _exact_append(s, case) if case["kind"] == "append" else _exact_attend(s, case)
