"""Requests that `cache_reserve` refuses, and what the calls behind it then do: nothing of another request's is touched, and
nothing is counted that is not there."""
import numpy as np
import pytest

import picked_ref as pref
from test_gpu_cache import i32, make_q, numpy_cache, offsets, random_pool, tables, to_cache
from test_gpu_picked import ring_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def reserve(s, table, held, want, free, state, new, page=16):
    off = offsets(new)
    g, st, sl = s.cache_reserve(table, i32(held), i32(want), free, i32(state), page, i32(off), offsets_h=off)
    return g.tolist(), st.tolist(), sl.tolist()


def bounds_reported(select, s):
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    return e.value.name == "DEVICE_BOUNDS"


def test_a_refused_request_names_no_page_of_another_one(select):
    """A request gives pages back, another takes them, the first wants one again and finds none: the entries of the pages
    that it wanted are -1, and rows appended all the same go nowhere."""
    rng = np.random.default_rng(1)
    s = select.Selector(2, 8, 8, 2, 2, 64, "bf16")
    table, free = i32([[4, 1, 2, 7, -1], [0, -1, -1, -1, -1]]), i32([3, -1, -1, -1, -1, -1, -1, -1])
    g, st, _ = reserve(s, table, [64, 16], [30, 16], free, [0, 1], [0, 0])  # pages 2 and 7 go back
    assert g == [30, 16] and st == [0, 3]
    g, st, _ = reserve(s, table, [30, 16], [30, 64], free, st, [0, 48])     # ... and to the second
    assert g == [30, 64] and st == [3, 0] and table[1].tolist() == [0, 3, 2, 7, -1]
    g, st, sl = reserve(s, table, [30, 64], [60, 64], free, st, [30, 0])
    assert g == [30, 64] and st == [3, 0] and sl == [-1] * 30
    assert table.tolist() == [[4, 1, -1, -1, -1], [0, 3, 2, 7, -1]]
    s.check_device()
    cache = to_cache(select, random_pool(rng, 8, 2, 16, 64))
    before = numpy_cache(cache)
    x = torch.from_numpy(rng.standard_normal((2, 30, 2, 64))).to(torch.bfloat16).cuda()
    off = offsets([30, 0])
    s.cache_append(cache, table, i32([30, 64]), x[0], x[1], i32(off), offsets_h=off)
    assert bounds_reported(select, s)  # 28 of the rows had no page
    for name, after in numpy_cache(cache).items():
        if not name.endswith("_scale"):
            np.testing.assert_array_equal(np.delete(after, 1, 0), np.delete(before[name], 1, 0), err_msg=name)
    # once pages are back the request gets its own
    g, st, _ = reserve(s, table, [32, 64], [32, 20], free, st, [0, 0])
    g, st, sl = reserve(s, table, [30, 20], [60, 20], free, st, [30, 0])
    assert g == [60, 20] and table[0, :4].tolist() == [4, 1, 2, 7] and min(sl) >= 0
    s.check_device()
    s.close()


@pytest.mark.parametrize("batch,page,share", [(5, 16, 0.0), (129, 16, 0.5), (300, 64, 0.3), (2500, 32, 0.7)])
def test_refused_requests_of_large_batches(select, batch, page, share):
    """Rows of the table that name pages of others behind a request's last one: those that a refused request wanted are -1,
    all else is as the restatement has it."""
    rng = np.random.default_rng(batch)
    held = rng.integers(0, 900, batch)
    want = np.where(rng.random(batch) < 0.2, rng.integers(0, held + 1), held + rng.integers(0, 300, batch))
    new = np.maximum(want - held, 0)
    table, pool = tables(rng, held.tolist(), page, spare=700)
    width = -(-int(max(held.max(), want.max())) // page) + 2
    full = rng.integers(0, pool, (batch, width)).astype(np.int32)  # what earlier calls left behind
    for b in range(batch):
        n = -(-int(held[b]) // page)
        full[b, :n] = table[b, :n]
    used = {int(x) for x in table.flatten() if x >= 0}
    need = int(np.maximum(-(-want // page) - -(-held // page), 0).sum())
    spare = min(int(need * share), pool - len(used))
    others = rng.permutation([p for p in range(pool) if p not in used])
    head = pool - 3
    free, off = ring_of(rng, others[:spare], pool, head), offsets(new)
    wg, wst, wsl, wt, wf = pref.reserve(full, held, want, free, (head, spare), page, new)
    refused = wg != want
    assert refused.any()
    for b in np.flatnonzero(refused):
        wt[b, -(-int(held[b]) // page):-(-int(want[b]) // page)] = -1
    s = select.Selector(batch, 8, 8, 4, 4, 64, "bf16")
    tg, fg = i32(full), i32(free)
    got = s.cache_reserve(tg, i32(held), i32(want), fg, i32([head, spare]), page, i32(off), offsets_h=off)
    for name, a, b in (("granted", got[0], wg), ("state", got[1], wst), ("slots", got[2], wsl), ("table", tg, wt),
                       ("free", fg, wf)):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    s.check_device()
    s.close()
