"""Paths of the 4-bit cache's kernels that only unusual shapes take: query heads that alone fill a tile of a decoded
token, weights of few rows whose scores are not kept, and evictions whose keys pass shared memory."""
import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import i32, random_pool, select, tables, to_cache, test_attend_matches_the_definition as attend_matches  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("hq,hkv,d,dtype,lens,counts", [
    (64, 1, 128, "bf16", [300, 1, 0, 77], [1, 1, 1, 1]),     # 64 rows of one token
    (100, 1, 128, "e4m3", [400, 129], [1, 1]),
    (192, 1, 64, "bf16", [260, 33], [1, 1]),                 # more than one row tile of one token
    (129, 3, 64, "bf16", [200, 40], [4, 1]),
    (64, 64, 128, "bf16", [150, 33, 5], [33, 2, 7]),         # tiles of one head of its own
])
@pytest.mark.parametrize("weights", [False, True])
def test_attend_of_many_query_heads(select, hq, hkv, d, dtype, lens, counts, weights):  # noqa: F811
    attend_matches(select, hq, hkv, d, 16, dtype, lens, counts, weights)


@pytest.mark.parametrize("hq,hkv,lens,counts", [
    (128, 128, [60, 90], [20, 17]),     # 20 rows x 128 heads: more rows than scores are kept for
    (256, 256, [130, 300], [9, 2]),
    (280, 140, [140, 3], [16, 1]),
    (2100, 2100, [40], [1]),            # a single row
])
def test_weights_of_few_rows_of_many_heads(select, hq, hkv, lens, counts):  # noqa: F811
    attend_matches(select, hq, hkv, 64, 16, "bf16", lens, counts, True)


@pytest.mark.parametrize("lens,budget,kind", [([450001], 4000, "plain"), ([450001], 400000, "ties"),
                                              ([420000, 17, 399999], 100, "special")])
@pytest.mark.parametrize("inplace", [False, True])
def test_evictions_of_keys_beyond_shared_memory(select, lens, budget, kind, inplace):  # noqa: F811
    """More than 8 x 49152 tokens of a request: weights are read again for every digit."""
    rng = np.random.default_rng(budget)
    page = 256
    table, pool = tables(rng, list(lens) + ([] if inplace else [min(n, budget) for n in lens]), page)
    c = random_pool(rng, pool, 1, page, 64)
    w = np.exp(2 * rng.standard_normal((pool, page)) - 5).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 40).astype(np.float32) / 40
    if kind == "special":
        w = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1.0, 1e-40], np.float32), w.shape)
    cache = to_cache(select, c, w)
    s = select.Selector(len(lens), 8, 8, 1, 1, 64, "bf16")
    from_t, to_t = table[:len(lens)], table[len(lens):, :-(-budget // page)]
    kept, new = s.cache_evict(cache, i32(from_t), i32(lens), max(lens), budget, 4, 60,
                              to_table=None if inplace else i32(to_t))
    s.check_device()
    to_t = from_t if inplace else to_t
    got = {x: getattr(cache, x).cpu().numpy() for x in ("k_codes", "k_scales", "v_codes", "v_scales")}
    for b, n in enumerate(lens):
        pos = np.arange(n)
        want = ref.evict(w[from_t[b][pos // page], pos % page], n, budget, 4, 60)
        assert int(new[b]) == len(want)
        np.testing.assert_array_equal(kept[b].cpu().numpy(), np.concatenate([want, np.full(budget - len(want), -1)]))
        i = np.arange(len(want))
        for x, a in got.items():
            np.testing.assert_array_equal(a[to_t[b][i // page], :, i % page],
                                          c[x][from_t[b][want // page], :, want % page], err_msg=x)
    s.close()


@pytest.mark.parametrize("dtype,scale,in_scale", [
    ("bf16", 2.0 ** -60, 1.0), ("bf16", 2.0 ** 60, 1.0), ("bf16", 1.3e-18, 1.0), ("bf16", 7.7e17, 1.0), ("bf16", 0.3, 1.0),
    ("e4m3", 2.0 ** -60, 2.0 ** 60), ("e4m3", 1.1e-18, 9e17), ("e4m3", 2.0 ** 60, 2.0 ** -60), ("e4m3", 0.7, 0.011)])
def test_append_at_the_ends_of_the_scales(select, dtype, scale, in_scale):  # noqa: F811
    """Values of every magnitude under the largest and smallest scales: codes and block scales byte for byte."""
    rng = np.random.default_rng(int(np.float32(scale).view(np.uint32)) + len(dtype))
    rows, d = 200, 128
    if dtype == "bf16":
        x = rng.standard_normal((rows, 1, d)) * 2.0 ** rng.uniform(-130, 126, (rows, 1, d // 16)).repeat(16, -1)
        x *= 2.0 ** rng.integers(-4, 1, x.shape)
        t = torch.from_numpy(x).to(torch.bfloat16).cuda()
        xv = t.double().cpu().numpy()
    else:
        t = torch.from_numpy(rng.integers(0, 256, (rows, 1, d), dtype=np.uint8)).cuda()
        xv = ref.E4M3[t.cpu().numpy()]
    s = select.Selector(1, 8, 8, 1, 1, d, dtype)
    cache = s.cache(4, 64, k_scale=scale, v_scale=1.0)
    s.cache_append(cache, i32([[2, 0, 3, 1]]), i32([0]), t, t, i32([0, rows]), k_in_scale=in_scale, v_in_scale=1.0)
    s.check_device()
    pos = np.arange(rows)
    at = np.array([2, 0, 3, 1])[pos // 64], pos % 64
    for name, sc, ins in (("k", scale, in_scale), ("v", 1.0, 1.0)):
        codes, scales = ref.quantise(xv, sc, ins)
        np.testing.assert_array_equal(getattr(cache, name + "_scales")[at[0], :, at[1]].cpu().numpy(), scales)
        np.testing.assert_array_equal(getattr(cache, name + "_codes")[at[0], :, at[1]].cpu().numpy(), codes)
    s.close()
