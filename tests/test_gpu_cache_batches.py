"""Attention over the 4-bit cache by batches that fill the GPU, whose keys are not split, and by whole prompts: every kernel
that a plan can choose, against the 64-bit definition."""
import numpy as np
import pytest

from test_gpu_cache import select, test_attend_matches_the_definition as attend_matches  # noqa: F401

pytestmark = pytest.mark.gpu

# hq, hkv, d, page, dtype, requests, longest, most queries
BATCHES = [
    (64, 8, 128, 32, "bf16", 20, 300, 25),    # tiles of 256 rows
    (64, 8, 64, 16, "bf16", 24, 290, 24),     # ... of 64 channels
    (64, 8, 128, 16, "e4m3", 20, 200, 12),    # tiles of 128 rows
    (64, 16, 64, 16, "bf16", 86, 100, 3),     # tiles of 16 rows
    (64, 16, 128, 32, "e4m3", 60, 130, 2),    # tiles of 8 rows
    (16, 16, 128, 32, "bf16", 60, 150, 1),    # a single row a head
    (16, 4, 64, 64, "bf16", 60, 2100, 1),     # one long request among short ones: weights of many keys a CTA
]


@pytest.mark.parametrize("hq,hkv,d,page,dtype,batch,longest,most", BATCHES)
@pytest.mark.parametrize("weights", [False, True])
def test_attend_of_batches(select, hq, hkv, d, page, dtype, batch, longest, most, weights):  # noqa: F811
    rng = np.random.default_rng(batch + d + most)
    lens = rng.integers(0, min(longest, 300) + 1, batch).tolist()
    lens[batch // 2], lens[0], lens[-1] = longest, 0, 1
    counts = rng.integers(0 if most > 1 else 1, most + 1, batch).tolist()
    counts[batch // 2], counts[1] = most, most
    attend_matches(select, hq, hkv, d, page, dtype, lens, counts, weights)


@pytest.mark.parametrize("hq,hkv,d,lens,counts", [(8, 1, 128, [700, 300], [700, 299]), (4, 2, 64, [513], [513])])
@pytest.mark.parametrize("weights", [False, True])
def test_attend_of_whole_prompts(select, hq, hkv, d, lens, counts, weights):  # noqa: F811
    attend_matches(select, hq, hkv, d, 64, "bf16", lens, counts, weights)
