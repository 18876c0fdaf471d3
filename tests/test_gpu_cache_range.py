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
