"""Plain restatement in 64 bits of the calls around a paged cache's pages (numpy, loops over requests): pages and slots
given to requests, the ranges of a page's keys, the pages that a query picks, attention over them. It shares no code with
the library."""
import math

import numpy as np

import cache_ref as ref


def reserve(table, held, want, free, state, page, new):
    """(granted, state, slots, table, free) of one call; the arrays given are left as they are. Valid states only."""
    table, free, total = table.copy(), free.copy(), len(free)
    old = free.copy()
    head, count = (int(x) for x in state)
    limit = table.shape[1] * page
    taken, back, full = 0, 0, False
    granted, slots, lost = [], [], 0
    for b in range(len(held)):
        n, w = (min(max(int(x[b]), 0), limit) for x in (held, want))
        hp, wp = -(-n // page), -(-w // page)
        ok = True
        if wp > hp:
            full = full or taken + wp - hp > count
            ok = not full
            if ok:
                for o in range(hp, wp):
                    table[b, o] = old[(head + taken) % total]
                    taken += 1
        for o in range(wp, hp):
            if count + back < total:
                free[(head + count + back) % total] = table[b, o]
            else:
                lost += 1
            back += 1
        granted.append(w if ok else n)
        for i in range(int(new[b])):
            p = w - int(new[b]) + i
            pg = int(table[b, p // page]) if ok and p >= 0 else -1
            slots.append(pg * page + p % page if 0 <= pg < total else -1)
    state = [(head + taken) % total, count - taken + min(back, total - count)]
    return np.array(granted, np.int32), np.array(state, np.int32), np.array(slots, np.int64), table, free


def key_values(codes, scales):
    """Values of packed rows without the tensor's scale, NaN as 0."""
    x = ref.values(codes, scales, 1.0)
    return np.where(np.isnan(x), 0.0, x)


def page_bounds(k):
    """Ranges of the rows [tokens, Hkv, d] of one page: (codes [Hkv, 2, d], exps [Hkv])."""
    hi, lo = k.max(0), k.min(0)
    m = np.maximum(np.abs(hi), np.abs(lo)).max(-1)
    e = np.where(m > 0, np.frexp(m)[1] - 7, 0)
    unit = 2.0 ** e[:, None]
    return np.stack((np.ceil(hi / unit), np.floor(lo / unit)), 1).astype(np.int8), e.astype(np.int8)


def bounds(cache, table, lens, new, codes, exps):
    """codes, exps after a call (the arrays given are left as they are)."""
    codes, exps = codes.copy(), exps.copy()
    ps = cache["k_codes"].shape[2]
    for b in range(len(lens)):
        n, t = int(lens[b]), min(int(new[b]), int(lens[b]))
        if t <= 0:
            continue
        for o in range((n - t) // ps, (n - 1) // ps + 1):
            p, rows = table[b, o], min(ps, n - o * ps)
            k = key_values(cache["k_codes"][p, :, :rows], cache["k_scales"][p, :, :rows]).transpose(1, 0, 2)
            codes[p], exps[p] = page_bounds(k)
    return codes, exps


def page_scores(q, codes, exps):
    """Scores [pages] (exact whole numbers times powers of two) of the heads q [G, d] of one key head, without q's unit;
    codes [pages, 2, d], exps [pages]."""
    top = np.abs(q).max()
    p = max(int(np.frexp(top)[1]) if top > 0 else -200, -119)
    r = np.clip(np.round(q * 2.0 ** (7 - p)), -127, 127)  # (numpy rounds ties to even)
    c = codes.astype(np.float64)
    s = np.maximum(r, 0) @ c[:, 0].T + np.minimum(r, 0) @ c[:, 1].T
    return s.max(0) * 2.0 ** exps.astype(np.float64)


def pick(q, off, lens, table, codes, exps, page, budget, sink, recent, hkv):
    """Picked pages int32 [rows, Hkv, budget]; q float64 [rows, Hq, d], finite."""
    rows, hq, _ = q.shape
    out = np.full((rows, hkv, budget), -1, np.int32)
    for b in range(len(lens)):
        n, t0, t1 = int(lens[b]), int(off[b]), int(off[b + 1])
        for i in range(t0, t1):
            pos = n - (t1 - i)
            if pos < 0:
                continue
            seen = pos // page + 1
            for h in range(hkv):
                if seen <= budget:
                    out[i, h, :seen] = np.arange(seen)
                    continue
                pg = table[b, :seen]
                there = (pg >= 0) & (pg < len(codes))
                s = page_scores(q[i, h * (hq // hkv):(h + 1) * (hq // hkv)], codes[np.where(there, pg, 0), h],
                                exps[np.where(there, pg, 0), h])
                s = np.where(there, s, -np.inf)
                j = np.arange(seen)
                s = np.where((j < sink) | (j >= seen - recent), np.inf, s)
                out[i, h] = np.sort(np.lexsort((j, -s))[:budget])
    return out


def attend(cache, table, lens, q, off, picked):
    """(out, slack): as cache_ref.attend, over the positions of the picked pages that a query sees. The slack counts the
    same steps: a score is a sum of d products in fp32, off by (d + 8) 2^-24 sum |q k| / sqrt(d) =: delta, which moves
    a probability and the row's sum by a factor 1 +- 2 delta, with 2^-20 for exp2, log2 and their arguments; f16
    probabilities (or their products with a scale) are off by 2^-11, those below f16's normal range by 2^-25 of the largest
    value; the output is rounded to bf16 (2^-8, a step's half counted twice)."""
    hkv, d = cache["k_codes"].shape[1], 2 * cache["k_codes"].shape[3]
    ps, hq = cache["k_codes"].shape[2], q.shape[1]
    out, slack = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(lens)):
        n, t0, t1 = int(lens[b]), int(off[b]), int(off[b + 1])
        for i in range(t0, t1):
            pos = n - (t1 - i)
            for h in range(hkv):
                k, v = [], []
                for o in map(int, picked[i, h]):
                    if o < 0 or o * ps > pos or o >= table.shape[1] or not 0 <= table[b, o] < len(cache["k_codes"]):
                        continue
                    rows = min(ps, pos - o * ps + 1)
                    for x, to in (("k", k), ("v", v)):
                        to.append(ref.values(cache[x + "_codes"][table[b, o], h, :rows],
                                             cache[x + "_scales"][table[b, o], h, :rows], cache[x + "_scale"]))
                if not k:
                    continue
                k, v = np.concatenate(k), np.concatenate(v)
                for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    with np.errstate(invalid="ignore"):
                        s = k @ q[i, g] / math.sqrt(d)
                        delta = (d + 8) * 2.0 ** -24 * (np.abs(k) @ np.abs(q[i, g])).max() / math.sqrt(d)
                        p = np.exp(s - s.max())
                        p /= p.sum()
                        out[i, g] = p @ v
                        slack[i, g] = (2.0 ** -8 * np.abs(out[i, g]) + (2.0 ** -11 + 2 * delta + 2.0 ** -20) *
                                       (p @ np.abs(v)) + len(k) * 2.0 ** -25 * np.abs(v).max())
    return out, slack
