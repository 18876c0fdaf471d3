"""Attention over the 4-bit cache at the ends of its range: queries and scales whose product is below or beyond 32 bits,
block scales of every size, long flat tails behind one strong key, and prompts as long as a call takes."""
import math

import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import i32, make_q, offsets, random_pool, select, tables, to_cache  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# hq, hkv, d, lens, queries: a row, 8, 16, 128 and 256 rows a CTA; every tile has keys that some of its rows do not see
ROWS = [
    (2, 2, 128, [300, 40], [1, 1]),
    (8, 1, 128, [300, 129], [1, 1]),
    (4, 1, 64, [300, 40], [3, 7]),
    (8, 1, 128, [300, 129], [10, 3]),
    (8, 1, 64, [290, 40], [11, 40]),
    (8, 1, 128, [300, 45], [40, 45]),
]


def zero_rows(q):
    """Every third row is 0, every sixth all but one channel."""
    q[::3] = 0
    q[::6, :, 5] = 2.0 ** -130
    return q


@pytest.mark.parametrize("hq,hkv,d,lens,counts", ROWS)
@pytest.mark.parametrize("dtype,k_scale,q_scale", [("bf16", 2.0 ** -40, 1.0), ("bf16", 2.0 ** -60, 1.0),
                                                   ("e4m3", 2.0 ** -60, 1e-30)])
def test_zero_queries_and_scales_whose_product_is_below_32_bits(select, hq, hkv, d, lens, counts, dtype, k_scale, q_scale):  # noqa: F811
    if dtype == "e4m3" and d == 64:
        pytest.skip("e4m3 heads have 128 channels")
    rng = np.random.default_rng(hq + d + len(dtype))
    table, pool = tables(rng, lens, 16)
    c = random_pool(rng, pool, hkv, 16, d, k_scale=k_scale)
    off = offsets(counts)
    x = zero_rows(rng.standard_normal((int(off[-1]), hq, d)))
    if dtype == "bf16":
        q = torch.from_numpy(x).to(torch.bfloat16).cuda()
        qv = q.double().cpu().numpy()
    else:
        q = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        qv = ref.E4M3[q.cpu().numpy()] * float(np.float32(q_scale))
    w = np.exp(rng.standard_normal((pool, 16)) - 5).astype(np.float32)
    cache = to_cache(select, c, w)
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, dtype)
    out = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), max(lens), q_scale=q_scale, accumulate=True)
    s.check_device()
    o, wn, slack, slack_w = ref.attend(c, table, lens, qv, off, hq, w)
    assert (np.abs(out.double().cpu().numpy() - o) <= slack).all()
    g = cache.weights.double().cpu().numpy()
    assert (np.abs(g - wn) <= np.where(slack_w > 0, slack_w, 0)).all()
    s.close()


@pytest.mark.parametrize("hq,hkv,d,lens,counts", ROWS)
@pytest.mark.parametrize("dtype,k_scale,q_scale", [("bf16", 2.0 ** 14, 1.0), ("bf16", 2.0 ** 40, 1.0),
                                                   ("bf16", 2.0 ** 60, 1.0), ("e4m3", 2.0 ** 60, 1e30)])
def test_scores_beyond_24_bits(select, hq, hkv, d, lens, counts, dtype, k_scale, q_scale):  # noqa: F811
    """The largest score takes all of a row where it leads by more than fp32 sums can be off (by 60 in log2 units and by
    four times (d + 8) 2^-24 of the sum of the products' magnitudes); nowhere is anything but a number."""
    if dtype == "e4m3" and d == 64:
        pytest.skip("e4m3 heads have 128 channels")
    rng = np.random.default_rng(hq + d + 7)
    table, pool = tables(rng, lens, 16)
    c = random_pool(rng, pool, hkv, 16, d, k_scale=k_scale)
    off = offsets(counts)
    x = rng.standard_normal((int(off[-1]), hq, d))
    if dtype == "bf16":
        x[1::3] *= 2.0 ** 60
        x[2::3] *= 2.0 ** 120
        q = torch.from_numpy(x).to(torch.bfloat16).cuda()
        qv = q.double().cpu().numpy()
    else:
        q = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        qv = ref.E4M3[q.cpu().numpy()] * float(np.float32(q_scale))
    w = np.zeros((pool, 16), np.float32)
    cache = to_cache(select, c, w)
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, dtype)
    out = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), max(lens), q_scale=q_scale, accumulate=True)
    s.check_device()
    got, g = out.double().cpu().numpy(), cache.weights.double().cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(g).all()
    sure, most = np.zeros(w.shape), np.zeros(w.shape)
    led = rows = 0
    for b, n in enumerate(lens):
        k, v = (ref.cached_rows(c, table, b, n, y) for y in "kv")
        for i in range(counts[b]):
            see = n - counts[b] + i + 1
            place = table[b][np.arange(see) // 16], np.arange(see) % 16
            for h in range(hq if see > 0 else 0):
                kk, qq, rows = k[:see, h // (hq // hkv)], qv[off[b] + i, h], rows + 1
                z = kk @ qq / math.sqrt(d) * math.log2(math.e)
                top = int(z.argmax())
                gap = z[top] - np.max(np.delete(z, top), initial=-np.inf)
                room = 4 * (d + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(qq)).max() / math.sqrt(d) * math.log2(math.e)
                if gap <= max(60.0, room):
                    most[place] += 1 / hq
                    continue
                led += 1
                at = place[0][top], place[1][top]
                sure[at] += 1 / hq
                most[at] += 1 / hq
                want = v[top, h // (hq // hkv)]
                assert (np.abs(got[off[b] + i, h] - want) <= (2.0 ** -8 + 2.0 ** -18) * np.abs(want)).all()
    assert led > 0.9 * rows
    assert (g >= sure * (1 - 2.0 ** -18)).all() and (g <= most * (1 + 2.0 ** -18)).all()
    s.close()
