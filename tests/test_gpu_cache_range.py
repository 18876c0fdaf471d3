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


def strict(slack, n, v_abs):
    """cache_ref's slack without its term for probabilities below f16's normal range (n 2^-25 of the largest value)."""
    return slack - n * 2.0 ** -25 * v_abs


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 300])
def test_a_single_row_over_small_block_scales(select, d, at):  # noqa: F811
    """One strong key and a flat tail whose probabilities are 2^-20 of its, values with the smallest block scales, in a
    batch whose keys are not split: a probability's weight does not depend on the size of the scales it meets. What p
    times the scale may be off by: 2^-11 (its rounding to f16), and 2^-34 of the largest value for a product below
    f16's normal range. The request's tokens lie in two pages, of which the second is named again and again."""
    rng = np.random.default_rng(d + at)
    heads, batch, page, n = 32, 58, 256, 131072 + 300
    table = np.full((batch, -(-n // page)), 1, np.int32)
    table[0, at] = 0
    lens = np.ones(batch, np.int64)
    lens[0] = n
    c = random_pool(rng, 2, heads, page, d, k_scale=1.0, v_scale=1.0)
    c["k_codes"][:] = 0
    c["k_codes"][0, :, 7] = 0x22  # 1.0 in every channel of the strong key
    c["k_scales"][:] = 0x38
    c["v_codes"] &= 0x77          # no negative values: the tail adds up
    c["v_scales"][:] = 1 + np.arange(d // 16)
    c["v_codes"][0, :, 7] = 0
    q = torch.full((batch, heads, d), 20.4 * math.log(2) / math.sqrt(d)).to(torch.bfloat16).cuda()
    s = select.Selector(batch, 8, 8, heads, heads, d, "bf16")
    out = s.cache_attend(to_cache(select, c), i32(table), i32(lens), q, i32(np.arange(batch + 1)), n)
    s.check_device()
    v = ref.values(c["v_codes"], c["v_scales"], 1.0)  # [page, head, slot, d]
    strong = math.exp(float(q[0, 0, 0]) * math.sqrt(d))
    count = np.array([np.bincount(np.arange(n) % page, (table[0][np.arange(n) // page] == x)) for x in (0, 1)])
    want = np.einsum("ps,phsd->hd", count, v) / (strong + n - 1)
    delta = (d + 8) * 2.0 ** -24 * math.log(strong)
    slack = (2.0 ** -8 + 2.0 ** -11 + 2 * delta + 2.0 ** -20) * want + n * 2.0 ** -34 * v.max()
    assert (np.abs(out[0].double().cpu().numpy() - want) <= slack).all()
    s.close()


@pytest.mark.parametrize("d", [64, 128])
def test_a_single_row_over_block_scales_of_every_size(select, d):  # noqa: F811
    rng = np.random.default_rng(d)
    lens = [700, 33, 400]
    table, pool = tables(rng, lens, 32)
    c = random_pool(rng, pool, 3, 32, d)
    c["v_scales"] = rng.integers(0, 0x7F, c["v_scales"].shape, dtype=np.uint8)
    c["v_scales"][:, 1, :, 0] = 0x7E   # the largest throughout
    c["v_scales"][:, 1, :, 1] = rng.integers(0, 4, c["v_scales"].shape[0::2][:2], dtype=np.uint8)
    for b, at in ((0, 650), (1, 32), (2, 3)):  # a large one among the smallest
        c["v_scales"][table[b, at // 32], 1, at % 32, 1] = 0x78
    q, qv, _ = make_q(rng, 3, 3, d, "bf16")
    s = select.Selector(3, 8, 8, 3, 3, d, "bf16")
    out = s.cache_attend(to_cache(select, c), i32(table), i32(lens), q, i32([0, 1, 2, 3]), 700)
    s.check_device()
    o, _, slack, _ = ref.attend(c, table, lens, qv, offsets([1, 1, 1]), 3)
    for b, n in enumerate(lens):
        top = np.abs(ref.cached_rows(c, table, b, n, "v")).max((0, 2))[:, None]
        assert (np.abs(out[b].double().cpu().numpy() - o[b]) <= strict(slack[b], n, top) + n * 2.0 ** -34 * top).all()
    s.close()


@pytest.mark.parametrize("hq,hkv,d,batch,t", [
    (256, 32, 128, 58, 1),    # 8 rows a CTA
    (64, 32, 64, 43, 8),      # 16
    (256, 32, 128, 32, 8),    # 64
    (256, 32, 128, 16, 20),   # 160
])
def test_a_flat_tail_behind_one_strong_key(select, hq, hkv, d, batch, t):  # noqa: F811
    """One request of 2^20 tokens among short ones, in a batch whose keys are not split: a tail of probabilities of
    2^-25.3 of the largest. Its tokens lie in two pages, of which the second is named again and again. Probabilities
    are rounded to f16 (2^-11), those below its normal range by 2^-32 of the largest."""
    rng = np.random.default_rng(t)
    n, page = (1 << 20) + 77, 256
    table = np.full((batch, -(-n // page)), 1, np.int32)
    table[0, 0] = 0
    lens = np.full(batch, t)
    lens[0] = n
    c = random_pool(rng, 2, hkv, page, d, k_scale=1.0, v_scale=0.125)
    c["k_codes"][:] = 0
    c["k_scales"][:] = 0x38
    c["k_codes"][0, :, 0] = 0x22
    c["v_codes"] &= 0x77
    c["v_codes"][0, :, 0] = 0
    q = torch.full((batch * t, hq, d), 25.3 * math.log(2) / math.sqrt(d)).to(torch.bfloat16).cuda()
    s = select.Selector(batch, 8, 8, hq, hkv, d, "bf16")
    out = s.cache_attend(to_cache(select, c), i32(table), i32(lens), q, i32(offsets([t] * batch)), n)
    s.check_device()
    v = ref.values(c["v_codes"], c["v_scales"], c["v_scale"])  # [page, head, slot, d]
    strong = math.exp(float(q[0, 0, 0]) * math.sqrt(d))
    pos = np.arange(n)
    for i in (0, t - 1):
        see = n - t + i + 1
        first = min(see, page)
        slots = np.bincount(pos[page:see] % page, minlength=page)
        total = v[0, :, :first].sum(1) + np.einsum("s,hsd->hd", slots, v[1])
        want = np.repeat(total / (strong + see - 1), hq // hkv, 0)
        got = out[i].double().cpu().numpy()
        delta = (d + 8) * 2.0 ** -24 * math.log(strong)
        slack = (2.0 ** -8 + 2.0 ** -11 + 2 * delta + 2.0 ** -20) * want + see * 2.0 ** -32 * np.abs(v).max()
        assert (np.abs(got - want) <= slack).all(), float((np.abs(got - want) / slack).max())
    for b in range(1, batch):  # t tokens of the same score: the mean of those seen
        for i in (0, t - 1):
            want = np.repeat(v[1, :, :i + 1].mean(1), hq // hkv, 0)
            assert (np.abs(out[b * t + i].double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -10) * want + 1e-9).all()
    s.close()


@pytest.mark.parametrize("weights", [False, True])
def test_a_prompt_of_16384_queries(select, weights):  # noqa: F811
    """A call's limit is that of the tiles its kernels take, 256 rows a CTA (128 with weights)."""
    n, hq, d, page = 16384, 32, 64, 256
    rng = np.random.default_rng(16)
    c = random_pool(rng, n // page, hq, page, d)
    table = np.arange(n // page, dtype=np.int32)[None]
    cache = to_cache(select, c, np.zeros((n // page, page), np.float32))
    q, _, _ = make_q(rng, n, hq, d, "bf16")
    s = select.Selector(1, 8, 8, hq, hq, d, "bf16")
    out = s.cache_attend(cache, i32(table), i32([n]), q, i32([0, n]), n, accumulate=weights)
    s.check_device()
    total = 0.0
    for h in (0, 31):
        k, v = (torch.from_numpy(ref.values(c[x + "_codes"][:, h], c[x + "_scales"][:, h], c[x + "_scale"])
                                 .reshape(n, d)).cuda() for x in "kv")
        for i in (0, 1, 255, 256, 9000, n - 1):
            z = k[:i + 1] @ q[i, h].double() / math.sqrt(d)
            p = torch.softmax(z, 0)
            want = p @ v[:i + 1]
            delta = (d + 8) * 2.0 ** -24 * (k[:i + 1].abs() @ q[i, h].double().abs()).max() / math.sqrt(d)
            slack = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * delta + 2.0 ** -20) * (p @ v[:i + 1].abs()) + \
                (i + 1) * 2.0 ** -25 * v.abs().max()
            assert ((out[i, h].double() - want).abs() <= slack).all()
    if weights:  # every query gives away 1 in all
        total = float(cache.weights.double().sum())
        assert abs(total - n) <= n * 2.0 ** -12
    s.close()


def test_the_limits_of_a_call_s_rows(select):  # noqa: F811
    """65535 CTAs: 255 key heads by 257 tiles of 256 rows, or of 128 where weights are wanted."""
    s = select.Selector(1, 8, 8, 255, 255, 128, "bf16")
    space = lambda t, w: select.cache_attend_workspace(s.handle, 1, np.array([0, t], np.int32), 1000, w)  # noqa: E731
    assert space(257 * 256, False) == 0  # (whole keys: nothing to join)
    assert space(257 * 128, True) > 0
    for t, w in ((257 * 256 + 1, False), (257 * 128 + 1, True)):
        with pytest.raises(select.LitevlmError) as e:
            space(t, w)
        assert e.value.name == "UNSUPPORTED", str(e.value)
    s.close()
