"""Plain 64-bit restatement of the 4-bit cache's operators and of draft verification (numpy, loops over requests),
for the tests. It shares no code with the library."""
import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1 = np.concatenate([E2M1, -E2M1])


def e4m3_table():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, 2.0 ** (e - 7.0) * (1 + m / 8.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c >= 128, -v, v)


E4M3 = e4m3_table()


def bf16_bits(x):
    """Nearest bf16 of float64 values (through float32, whose rounding is not visible in bf16 for the values here),
    as float64."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16
    return r.astype(np.uint32).view(np.float32).astype(np.float64)


def _nearest_even(x, grid):
    """Index of the nearest value of an ascending grid; a tie to the even index."""
    i = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo, hi = grid[i - 1], grid[i]
    up = (hi - x < x - lo) | ((hi - x == x - lo) & (i % 2 == 0))
    return np.where(up, i, i - 1)


def quantise(x, scale, in_scale=1.0):
    """Rows [..., d] -> (codes [..., d/2], scales [..., d/16]) uint8, fp32 steps as the definition has them."""
    with np.errstate(all="ignore"):
        y = (x.astype(np.float32) * np.float32(in_scale)) / np.float32(scale)
        blk = y.reshape(*y.shape[:-1], -1, 16)
        top = np.max(np.abs(blk), -1)  # NaN stays NaN
        s = np.minimum(top / np.float32(6), np.float32(448)).astype(np.float64)
        code_s = np.where(np.isnan(s), 0x7F, _nearest_even(np.nan_to_num(s), E4M3[:127])).astype(np.uint8)
        sv = np.where(np.isnan(s), 0, E4M3[code_s])[..., None]
        z = np.where(sv > 0, np.abs(blk.astype(np.float64)) / np.where(sv > 0, sv, 1), 0)
        c = _nearest_even(np.minimum(np.nan_to_num(z, posinf=6.0), 6.0), E2M1[:8]) | (np.signbit(blk).astype(np.int64) << 3)
        c = np.where(np.isnan(s)[..., None], 0, c).reshape(y.shape).astype(np.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), code_s


def values(codes, scales, scale):
    x = np.stack((E2M1[codes & 15], E2M1[codes >> 4]), -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    with np.errstate(invalid="ignore"):
        return x * np.repeat(E4M3[scales], 16, -1) * float(np.float32(scale))


def cached_rows(cache, table, b, n, which):
    """Rows [n, Hkv, d] of request b in 64 bits (cache: dict of numpy arrays and scales)."""
    ps = cache["k_codes"].shape[2]
    pos = np.arange(n)
    page, slot = table[b][pos // ps], pos % ps
    return values(cache[which + "_codes"][page, :, slot], cache[which + "_scales"][page, :, slot],
                  cache[which + "_scale"])


def attend(cache, table, lens, q, off, hq, weights=None):
    """(out, weights, slack_out, slack_w): q float64 [rows, Hq, d] with its scale applied. The slacks bound what fp32
    scores, 11-bit probabilities and fp32 sums may change, from the rounding steps:
      a score in natural units is a sum of d products in fp32, off by (d + 8) 2^-24 sum |q k| / sqrt(d) =: delta, which
      moves a probability (and the row's sum) by a factor 1 +- 2 delta, with 2^-20 for exp2, log2 and their arguments;
      f16 probabilities are off by 2^-11, those below f16's normal range by 2^-25 of the reference;
      the output is rounded to bf16 (2^-8)."""
    hkv, d = cache["k_codes"].shape[1], 2 * cache["k_codes"].shape[3]
    ps = cache["k_codes"].shape[2]
    out, slack = np.zeros(q.shape), np.zeros(q.shape)
    w = None if weights is None else weights.astype(np.float64).copy()
    slack_w = None if weights is None else np.zeros(weights.shape)
    for b in range(len(lens)):
        n, t0, t1 = int(lens[b]), int(off[b]), int(off[b + 1])
        t = t1 - t0
        k, v = (cached_rows(cache, table, b, n, x) for x in "kv")
        add, add_s = np.zeros(n), np.zeros(n)
        for i in range(t):
            see = n - t + i + 1
            if see <= 0:
                continue
            for h in range(hq):
                kk, vv = k[:see, h // (hq // hkv)], v[:see, h // (hq // hkv)]
                with np.errstate(invalid="ignore"):
                    s = kk @ q[t0 + i, h] / math.sqrt(d)
                    delta = (d + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(q[t0 + i, h])).max() / math.sqrt(d)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[t0 + i, h] = p @ vv
                    rel = 2 * delta + 2.0 ** -20
                    slack[t0 + i, h] = (2.0 ** -8 * np.abs(out[t0 + i, h]) + (2.0 ** -11 + rel) * (p @ np.abs(vv)) +
                                        see * 2.0 ** -25 * np.abs(vv).max())
                    add[:see] += p / hq
                    add_s[:see] += p / hq * (rel + 2.0 ** -23 * (t * hq / hkv + hkv + 8))
        if w is not None:
            pos = np.arange(n)
            page, slot = table[b][pos // ps], pos % ps
            w[page, slot] += add
            slack_w[page, slot] = add_s + 2.0 ** -24 * np.abs(w[page, slot]) + 1e-30
    return out, w, slack, slack_w


def evict(weights_row, n, budget, sink, recent):
    """Kept positions of one request, ascending."""
    if n <= budget:
        return np.arange(n)

    def rank(j):  # the larger, the sooner it stays
        w = float(weights_row[j])
        if j < sink or j >= n - recent:
            return (2, 0.0, -j)
        return (0, 0.0, -j) if math.isnan(w) else (1, w, -j)
    return np.array(sorted(sorted(range(n), key=rank, reverse=True)[:budget]), np.int64)


def verify(tokens, p, q, u, u_last):
    """One request: (accepted, tokens [T + 1])."""
    t, vocab = len(tokens), p.shape[1]
    p = p.astype(np.float64)
    acc = 0
    while acc < t:
        x = int(tokens[acc])
        if not 0 <= x < vocab:
            break
        qx = 1.0 if q is None else float(q[acc, x])
        if not float(u[acc]) * qx < p[acc, x]:
            break
        acc += 1
    with np.errstate(invalid="ignore"):
        if acc < t and q is not None:
            w = p[acc] - q[acc].astype(np.float64)
        else:
            w = p[acc].copy()
            if acc < t and 0 <= tokens[acc] < vocab:
                w[tokens[acc]] = 0
        w = np.where(w > 0, w, 0)
        if not w.sum() > 0:
            w = np.where(p[acc] > 0, p[acc], 0)
        out = np.full(t + 1, -1, np.int64)
        out[:acc] = tokens[:acc]
        if (w > 0).any():
            c = np.cumsum(w)
            hit = np.nonzero((c > float(u_last) * c[-1]) & (w > 0))[0]
            out[acc] = hit[0] if len(hit) else np.nonzero(w > 0)[0][-1]
    return acc, out
