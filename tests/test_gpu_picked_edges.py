"""The selection's edge inputs in each of the kernels that score pages (up to 8, up to 64 and more columns of query heads),
in both element types, and attention over picked pages at head layouts and types beside the usual ones."""
import numpy as np
import pytest

import cache_ref as ref
import picked_ref as pref
from test_gpu_cache import i32, make_q, offsets, random_pool, tables, to_cache
from test_gpu_picked import attend_case, pick_case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PAGE, PAGES = 16, 30


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def scorer(scorer, rows):
    """Queries of each request, at 4 / 2 heads, by which the kernel is chosen: 2 columns a request, 2 x 9, 2 x 40."""
    n = {"token": 1, "some": 9, "many": 40}[scorer]
    return [n] * -(-rows // n)


def whole(q, dtype):
    """Values of a query's elements as the selection takes them: NaN as 0, an infinity as the largest value."""
    v = q.double().cpu().numpy() if dtype == "bf16" else ref.E4M3[q.cpu().numpy()]
    return np.where(np.isnan(v), 0.0, np.clip(v, -255 * 2.0 ** 120, 255 * 2.0 ** 120))


def check(select, q, dtype, counts, codes, exps, table=None, budget=5, sink=1, recent=1, report=False):
    """Every request has the same pages and stands at their end."""
    batch, hq, hkv, d = len(counts), q.shape[1], codes.shape[1], q.shape[2]
    table = np.tile(np.arange(PAGES, dtype=np.int32) if table is None else table, (batch, 1))
    lens, off = [PAGE * PAGES] * batch, offsets(counts)
    s = select.Selector(batch, 8, 8, hq, hkv, d, dtype)
    bounds = select.KeyBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), PAGE)
    got = s.cache_pick(bounds, i32(table), i32(lens), q, i32(off), PAGE * PAGES, budget, sink, recent, offsets_h=off)
    if report:
        with pytest.raises(select.LitevlmError) as e:
            s.check_device()
        assert e.value.name == "DEVICE_BOUNDS"
    else:
        s.check_device()
    want = pref.pick(whole(q, dtype), off, lens, table, codes, exps, PAGE, budget, sink, recent, hkv)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    s.close()


def ranges(rng, hkv, d):
    return (rng.integers(-127, 128, (PAGES, hkv, 2, d)).astype(np.int8),
            rng.integers(-3, 3, (PAGES, hkv)).astype(np.int8))


@pytest.mark.parametrize("kernel", ["token", "some", "many"])
@pytest.mark.parametrize("d", [64, 128])
def test_special_bf16_queries(select, kernel, d):
    """Zeros, NaN, infinities, the type's ends, one after the other through all queries of the call."""
    rng = np.random.default_rng(d)
    counts = scorer(kernel, 40)
    x = rng.standard_normal((sum(counts), 4, d))
    x[0::8] = 0.0
    x[1::8, 0, 5], x[1::8, 2, 7] = np.nan, np.nan
    x[2::8, 1, 3], x[2::8, 3, 9] = np.inf, -np.inf
    x[3::8] *= 2.0 ** -130
    x[4::8] *= 2.0 ** 120
    x[5::8] = np.nan
    x[6::8, :, 1:] *= 1e-4
    x[7::8] *= 2.0 ** -118
    check(select, torch.from_numpy(x).to(torch.bfloat16).cuda(), "bf16", counts, *ranges(rng, 2, d))


@pytest.mark.parametrize("kernel", ["token", "some", "many"])
def test_special_e4m3_queries(select, kernel):
    """Codes of NaN (0x7F, 0xFF), zeros of both signs, the largest and the smallest values."""
    rng = np.random.default_rng(3)
    counts = scorer(kernel, 40)
    x = rng.integers(0, 0x7F, (sum(counts), 4, 128)) | rng.choice([0, 0x80], (sum(counts), 4, 128))
    x[0::6] = rng.choice([0, 0x80], x[0::6].shape)
    x[1::6, :, ::5] = 0x7F
    x[2::6, 1::2] = 0xFF
    x[3::6] = rng.choice([0x7F, 0xFF], x[3::6].shape)
    x[4::6] = rng.choice([0x7E, 0xFE, 0x00], x[4::6].shape)
    x[5::6] = rng.choice([0x01, 0x81, 0x07], x[5::6].shape)
    check(select, torch.from_numpy(x.astype(np.uint8)).cuda(), "e4m3", counts, *ranges(rng, 2, 128))


@pytest.mark.parametrize("kernel", ["token", "some", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_query_of_zeros_ties_at_every_page(select, kernel, dtype):
    """Its score is 0 whatever the signs of a page's keys are: pages of keys that are all negative, all positive, zero or
    mixed tie, and the lower ones are picked."""
    rng = np.random.default_rng(4)
    counts = scorer(kernel, 40)
    q = torch.zeros((sum(counts), 4, 128), dtype=torch.bfloat16 if dtype == "bf16" else torch.uint8, device="cuda")
    q[1::2] = -q[1::2] if dtype == "bf16" else 0x80
    codes, exps = ranges(rng, 2, 128)
    for j in range(PAGES):  # the lowest pages, which are picked, are all negative
        codes[j] = (-np.abs(codes[j]) - (codes[j] == 0), np.abs(codes[j]), 0 * codes[j], codes[j])[0 if j < 4 else j % 4]
    codes[8::4, :, 0, 3] = 1  # (some of the others but for a channel)
    check(select, q, dtype, counts, codes, exps)
    # ... and a head of zeros beside heads whose scores are below 0
    if dtype == "bf16":
        q[:, 1::2] = -1.0
        codes[:, :, :] = np.abs(codes) + 1
        codes[3::5] *= -1
        check(select, q, dtype, counts, codes.clip(-127, 127), exps)


@pytest.mark.parametrize("count", [2, 9, 40])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("e4m3", 128)])
def test_the_lower_of_equal_pages(select, count, dtype, d):
    for levels in (1, 2, 3):
        pick_case(select, 4, 2, d, dtype, 16, [900, 700], [count, 1], 9, 1, 1, seed=levels, levels=levels)


@pytest.mark.parametrize("kernel", ["token", "some", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_pages_that_the_pool_has_not_rank_last(select, kernel, dtype):
    rng = np.random.default_rng(5)
    counts = scorer(kernel, 40)
    q, _, _ = make_q(rng, sum(counts), 4, 128, dtype)
    codes, exps = ranges(rng, 2, 128)
    table = rng.permutation(PAGES).astype(np.int32)
    table[[3, 7, 8, 9, 10, 11, 12, 13, 14]] = [-1, PAGES, 99, -5, 2 ** 31 - 1, -1, -1, -1, -1]
    for budget in (5, 25):  # 25: four more than the pages that are there
        check(select, q, dtype, counts, codes, exps, table, budget, 0, 1, report=True)


# ---------------------------------------------------------------------------------------------------------- attend
@pytest.mark.parametrize("hq,hkv,d,dtype", [
    (9, 1, 64, "bf16"), (16, 1, 128, "bf16"), (32, 2, 128, "bf16"), (24, 2, 128, "e4m3"), (16, 1, 128, "e4m3"),
    (17, 1, 128, "bf16"), (40, 2, 64, "bf16"), (33, 1, 128, "e4m3"), (128, 1, 64, "bf16"),
    (4, 4, 128, "e4m3"), (1, 1, 128, "e4m3"),
])
@pytest.mark.parametrize("page,budget", [(16, 1), (16, 7), (16, 60), (64, 16), (256, 3)])
def test_single_tokens_of_many_heads_and_of_single_8_bit_ones(select, hq, hkv, d, dtype, page, budget):
    """More than eight and more than sixteen heads a key head; one head in e4m3: lists taken whole, and in chunks."""
    attend_case(select, hq, hkv, d, dtype, page, [1500, 40, 0, 700], [1, 1, 1, 1], budget, seed=hq + page, strided=hq > 9)
    attend_case(select, hq, hkv, d, dtype, page, [900], [1], budget, seed=budget)


def test_single_tokens_of_many_heads_in_batches_that_fill_the_gpu(select):
    """So many lists that each is taken whole by a CTA."""
    rng = np.random.default_rng(2)
    for hq, hkv, dtype in ((64, 4, "bf16"), (80, 4, "e4m3"), (8, 8, "e4m3")):
        lens = rng.integers(1, 300, 160).tolist()
        attend_case(select, hq, hkv, 128, dtype, 16, lens, [1] * 160, 4, seed=hq)


@pytest.mark.parametrize("hq,hkv,counts", [
    (28, 4, [50, 30]), (4, 4, [300, 129]), (14, 2, [37, 1, 19]), (32, 2, [20, 9]), (300, 1, [2, 1]),
])
@pytest.mark.parametrize("budget", [3, 20])
def test_prompts_of_8_bit_queries(select, hq, hkv, counts, budget):
    lens = [700 + 100 * n for n in range(len(counts))]
    attend_case(select, hq, hkv, 128, "e4m3", 16, lens, counts, budget, seed=budget, strided=True)


@pytest.mark.parametrize("hq,hkv,dtype", [(2, 2, "bf16"), (14, 2, "bf16"), (14, 2, "e4m3"), (28, 4, "bf16")])
def test_nan_keys_reach_only_those_that_see_them(select, hq, hkv, dtype):
    """A key whose scale is NaN makes the queries NaN that see it; others that share a list of pages, or stand before it,
    are as without it."""
    rng = np.random.default_rng(hq)
    g = hq // hkv
    for count in (1, 3, 30):
        lens, counts = [100], [count]
        table, pool = tables(rng, lens, 16)
        c, off = random_pool(rng, pool, hkv, 16, 128), offsets(counts)
        at = 99 if count == 1 else 98  # the position: the last queries see it
        picked = np.tile(np.array([5, 0, 6], np.int32), (count, hkv, 1))
        picked[count * 2 // 3:count - 1] = [4, 1, 2]
        q, qv, scale = make_q(rng, count, hq, 128, dtype)
        want, slack = pref.attend(c, table, lens, qv, off, picked)
        c["k_scales"][table[0, at // 16], 0, at % 16, 3] = 0x7F
        s = select.Selector(1, 8, 8, hq, hkv, 128, dtype)
        got = s.cache_attend_picked(to_cache(select, c), i32(table), i32(lens), q, i32(off), i32(picked), q_scale=scale,
                                    offsets_h=off)
        s.check_device()
        got = got.double().cpu().numpy()
        nan = np.zeros(got.shape, bool)
        for i in range(count):
            nan[i, :g] = at // 16 in picked[i, 0] and at <= 100 - count + i
        assert nan.any()
        np.testing.assert_array_equal(np.isnan(got), nan)
        assert (np.abs(got - want) <= slack)[~nan].all()
        s.close()
