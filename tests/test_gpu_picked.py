"""The calls around a paged cache's pages on the GPU against a plain 64-bit restatement: pages and slots given to requests,
ranges of keys, pages picked by them, attention over picked pages, each at the sizes where it can go wrong, and all of
them in a run."""
import numpy as np
import pytest

import cache_ref as ref
import picked_ref as pref
from test_gpu_cache import i32, make_q, numpy_cache, offsets, random_pool, tables, to_cache

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def ring_of(rng, pages, total, head):
    """A ring with these free pages from `head` on."""
    free = np.full(total, -1, np.int32)
    free[(head + np.arange(len(pages))) % total] = pages
    return free


# --------------------------------------------------------------------------------------------------------- reserve
def reserve_case(select, held, want, new, page, spare, extra=3, width=None, seed=0, batch_max=None):
    rng = np.random.default_rng(seed)
    table, pool = tables(rng, held, page, spare=spare + extra)
    most = max([1] + [-(-max(a, b) // page) for a, b in zip(held, want)])
    full = np.full((len(held), width or most), -1, np.int32)
    full[:, :table.shape[1]] = table[:, :full.shape[1]]
    used = {int(x) for x in table.flatten() if x >= 0}
    others = rng.permutation([p for p in range(pool) if p not in used])
    head = int(rng.integers(0, pool))
    free = ring_of(rng, others[:spare], pool, head)
    off = offsets(new)
    s = select.Selector(batch_max or max(1, len(held)), 8, 8, 4, 4, 64, "bf16")
    tg, fg = torch.from_numpy(full.copy()).cuda(), torch.from_numpy(free.copy()).cuda()
    state = i32([head, spare])
    got = s.cache_reserve(tg, i32(held), i32(want), fg, state, page, i32(off), offsets_h=off)
    want_g, want_st, want_sl, want_t, want_f = pref.reserve(full, held, want, free, (head, spare), page, new)
    for name, a, b in (("granted", got[0], want_g), ("state", got[1], want_st), ("slots", got[2], want_sl),
                       ("table", tg, want_t), ("free", fg, want_f)):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    assert state.tolist() == [head, spare]
    s.check_device()
    s.close()
    return want_g


@pytest.mark.parametrize("held,want,new,page,spare", [
    ([0], [1], [1], 16, 1),
    ([0], [0], [0], 16, 0),
    ([16, 15, 0, 40], [17, 16, 33, 40], [1, 1, 33, 0], 16, 9),
    ([100, 64, 3], [0, 10, 200], [0, 0, 197], 64, 5),       # pages that come back are not free for the same call
    ([1, 1, 1, 1], [200, 20, 1, 17], [199, 19, 0, 16], 16, 5),  # the first finds too few, and then nobody takes any
    ([30, 5], [33, 600], [3, 595], 32, 3),                  # the second does
    ([255, 256, 257], [256, 257, 300], [1, 1, 43], 256, 2),
])
def test_reserve_of_small_batches(select, held, want, new, page, spare):
    for seed in range(3):  # heads of the ring, some near its end
        reserve_case(select, held, want, new, page, spare, seed=seed)


@pytest.mark.parametrize("batch,page,share,seed", [(129, 16, 1.0, 1), (300, 64, 0.6, 2), (1024, 32, 1.0, 3),
                                                   (2500, 16, 0.9, 4)])
def test_reserve_of_large_batches(select, batch, page, share, seed):
    rng = np.random.default_rng(seed)
    kind = rng.random(batch)
    held = np.where(kind < 0.3, 0, rng.integers(1, 900, batch))
    want = np.where(kind > 0.8, rng.integers(0, held + 1), held + np.where(kind < 0.3, rng.integers(0, 700, batch),
                                                                            rng.integers(0, 9, batch)))
    new = np.where(kind > 0.8, 0, want - held)
    need = int(np.maximum(-(-want // page) - -(-held // page), 0).sum())
    granted = reserve_case(select, held.tolist(), want.tolist(), new.tolist(), page, max(1, int(need * share)), seed=seed)
    assert (granted == want).all() == (share >= 1.0)


def test_reserve_over_many_steps_keeps_every_page_once(select):
    """Requests come, grow, shrink and go; table and ring together hold every page once after every call."""
    rng = np.random.default_rng(8)
    batch, page, pool, width = 37, 16, 200, 24
    s = select.Selector(batch, 8, 8, 4, 4, 64, "bf16")
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    free = i32(rng.permutation(pool))
    state, held = i32([0, pool]), np.zeros(batch, np.int64)
    for step in range(60):
        u = rng.random(batch)
        want = np.where(u < 0.1, 0, np.where(u < 0.2, held // 2, np.minimum(held + rng.integers(0, 60, batch), width * page)))
        new = np.maximum(want - held, 0)
        off = offsets(new)
        granted, state, slots = s.cache_reserve(table, i32(held), i32(want), free, state, page, i32(off), offsets_h=off)
        held = granted.cpu().numpy().astype(np.int64)
        assert ((held == want) | (want > held)).all()
        t, f, (head, count) = table.cpu().numpy(), free.cpu().numpy(), state.tolist()
        owned = [int(t[b, o]) for b in range(batch) for o in range(-(-int(held[b]) // page))]
        owned += [int(f[(head + i) % pool]) for i in range(count)]
        assert sorted(owned) == list(range(pool)), step
        sl = slots.cpu().numpy()
        for b in range(batch):
            p = np.arange(want[b] - new[b], want[b])
            exp = t[b, p // page].astype(np.int64) * page + p % page if held[b] == want[b] else np.full(len(p), -1)
            np.testing.assert_array_equal(sl[off[b]:off[b + 1]], exp)
    s.check_device()
    s.close()


def test_reserve_reports_what_is_no_page_or_no_length(select):
    s = select.Selector(4, 8, 8, 4, 4, 64, "bf16")

    def call(table, held, want, free, state, new):
        t, f, off = i32(table), i32(free), offsets(new)
        out = s.cache_reserve(t, i32(held), i32(want), f, i32(state), 16, i32(off), offsets_h=off)
        r = [x.cpu().numpy().tolist() for x in (*out, t, f)]
        with pytest.raises(select.LitevlmError) as e:
            s.check_device()
        assert e.value.name == "DEVICE_BOUNDS"
        return r

    # a length beyond the table is cut to it
    g, st, sl, t, f = call([[-1, -1]], [0], [99], [0, 1, 2], [0, 3], [32])
    assert g == [32] and st == [2, 1] and t == [[0, 1]] and sl == list(range(32))
    # a page of the ring that the pool has not: its tokens have no slot
    g, st, sl, t, f = call([[-1, -1]], [0], [17], [77, 1, 2], [0, 3], [17])
    assert sl == [-1] * 16 + [16] and t == [[77, 1]]
    # a state that is none: nothing is taken or given back
    for state in ([5, 1], [-1, 1], [0, 4], [0, -2]):
        g, st, sl, t, f = call([[0, -1], [1, -1]], [16, 16], [17, 0], [2, -1, -1], state, [1, 0])
        assert g[0] == 16 and st == state and sl == [-1] and t == [[0, -1], [1, -1]] and f == [2, -1, -1]
    # a token before position 0
    g, st, sl, t, f = call([[0, -1]], [2], [2], [1, 2], [0, 2], [3])
    assert sl == [-1, 0, 1]
    # a ring without room for what comes back
    g, st, sl, t, f = call([[0, 1]], [32], [0], [2, 1], [0, 1], [0])
    assert st == [0, 2] and f == [2, 0]
    s.close()


# ---------------------------------------------------------------------------------------------------------- bounds
@pytest.mark.parametrize("hkv,d,page,lens,new", [
    (4, 128, 16, [1, 16, 17, 40, 5], [1, 1, 1, 40, 0]),
    (1, 64, 64, [200, 63, 64, 65], [70, 1, 64, 2]),
    (3, 64, 16, [100, 33], [33, 17]),
    (2, 128, 256, [300, 511, 3], [200, 3, 3]),
    (32, 128, 32, [70, 0, 31], [9, 0, 31]),
])
def test_bounds_match_the_definition(select, hkv, d, page, lens, new):
    rng = np.random.default_rng(hkv + d + page)
    table, pool = tables(rng, lens, page)
    c = random_pool(rng, pool, hkv, page, d)
    c["k_scales"] = rng.integers(0, 0x7F, c["k_scales"].shape, dtype=np.uint8)  # the whole range of scales
    c["k_scales"][0] = 0
    c["k_scales"][rng.random(c["k_scales"].shape) < 0.02] = 0x7F  # NaN
    c["k_scales"][rng.random(c["k_scales"].shape) < 0.02] |= 0x80  # a negative scale of another program's cache
    cache, off = to_cache(select, c), offsets(new)
    s = select.Selector(len(lens), 8, 8, hkv, hkv, d, "bf16")
    bounds = s.key_bounds(cache)
    codes, exps = rng.integers(-99, 99, bounds.codes.shape, dtype=np.int8), rng.integers(-9, 9, bounds.exps.shape, dtype=np.int8)
    bounds.codes.copy_(torch.from_numpy(codes)), bounds.exps.copy_(torch.from_numpy(exps))
    s.cache_bounds(cache, bounds, i32(table), i32(lens), i32(off), offsets_h=off)
    s.check_device()
    want_c, want_e = pref.bounds(numpy_cache(cache), table, lens, new, codes, exps)
    np.testing.assert_array_equal(bounds.exps.cpu().numpy(), want_e)
    np.testing.assert_array_equal(bounds.codes.cpu().numpy(), want_c)
    s.close()


def test_bounds_of_many_pages(select):
    """So many that a warp takes several heads of a page."""
    rng = np.random.default_rng(3)
    hkv, d, page = 16, 64, 16
    lens = rng.integers(700, 1400, 48).tolist()
    new = [n - int(x) for n, x in zip(lens, rng.integers(0, 40, 48))]
    table, pool = tables(rng, lens, page)
    c = random_pool(rng, pool, hkv, page, d)
    off = offsets(new)
    s = select.Selector(48, 8, 8, hkv, hkv, d, "bf16")
    cache = to_cache(select, c)
    bounds = s.key_bounds(cache)
    s.cache_bounds(cache, bounds, i32(table), i32(lens), i32(off), offsets_h=off)
    s.check_device()
    want_c, want_e = pref.bounds(c, table, lens, new, np.zeros(bounds.codes.shape, np.int8),
                                 np.zeros(bounds.exps.shape, np.int8))
    np.testing.assert_array_equal(bounds.exps.cpu().numpy(), want_e)
    np.testing.assert_array_equal(bounds.codes.cpu().numpy(), want_c)
    s.close()


def test_bounds_report_bad_lengths_and_pages(select):
    rng = np.random.default_rng(1)
    c = random_pool(rng, 3, 1, 16, 64)
    cache = to_cache(select, c)
    s = select.Selector(3, 8, 8, 1, 1, 64, "bf16")
    bounds = s.key_bounds(cache)
    bounds.codes.fill_(5)
    # a page outside the pool, a length beyond the table, more new tokens than the request has
    s.cache_bounds(cache, bounds, i32([[0, 9], [1, -1], [2, -1]]), i32([20, 99, 7]), i32([0, 20, 40, 60]),
                   offsets_h=np.array([0, 20, 40, 60], np.int32))
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    want, _ = pref.bounds(c, np.array([[0], [1], [2]]), [16, 16, 7], [16, 16, 7], np.full((3, 1, 2, 64), 5, np.int8),
                          np.zeros((3, 1), np.int8))
    np.testing.assert_array_equal(bounds.codes.cpu().numpy(), want)
    s.close()


# ------------------------------------------------------------------------------------------------------------ pick
def pick_case(select, hq, hkv, d, dtype, page, lens, counts, budget, sink, recent, seed=0, levels=None, strided=False,
              max_len=None):
    """levels: codes take so few values that scores tie."""
    rng = np.random.default_rng(seed)
    table, pool = tables(rng, lens, page)
    codes = rng.integers(-127, 128, (pool, hkv, 2, d)).astype(np.int8)
    exps = rng.integers(-6, 3, (pool, hkv)).astype(np.int8)
    if levels:
        codes[:] = rng.integers(0, levels, (pool, hkv, 1, 1))
        exps[:] = 0
    off = offsets(counts)
    q, qv, _ = make_q(rng, int(off[-1]), hq, d, dtype)
    if dtype == "e4m3":
        qv = ref.E4M3[q.cpu().numpy()]
    if strided:
        wide = torch.zeros((q.shape[0], hq + 2, d), dtype=q.dtype, device="cuda")
        wide[:, 1:1 + hq] = q
        q = wide[:, 1:1 + hq]
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, dtype)
    bounds = select.KeyBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), page)
    got = s.cache_pick(bounds, i32(table), i32(lens), q, i32(off), max_len or max(lens + [1]), budget, sink, recent,
                       offsets_h=off)
    s.check_device()
    want = pref.pick(qv, off, lens, table, codes, exps, page, budget, sink, recent, hkv)
    np.testing.assert_array_equal(got.cpu().numpy(), want)
    s.close()


@pytest.mark.parametrize("hq,hkv,d,dtype,page,lens,counts,budget,sink,recent", [
    (4, 4, 64, "bf16", 16, [200, 1, 16, 65], [1, 1, 1, 1], 3, 1, 1),          # one head a key head
    (4, 2, 128, "bf16", 16, [300, 40], [2, 5], 4, 0, 1),                      # two
    (6, 2, 64, "bf16", 32, [999, 100], [1, 9], 5, 2, 2),                      # three
    (4, 1, 128, "e4m3", 16, [500], [3], 7, 0, 0),                             # four
    (14, 2, 64, "bf16", 16, [321, 1000, 7], [4, 11, 7], 6, 1, 2),             # seven
    (16, 2, 128, "e4m3", 64, [3000, 2000], [1, 8], 8, 1, 4),                  # eight
    (18, 2, 128, "bf16", 16, [700], [5], 5, 1, 1),                            # nine: two tiles of columns
    (32, 2, 128, "bf16", 32, [2000, 64], [3, 2], 9, 0, 3),                    # sixteen
    (80, 1, 64, "bf16", 16, [400, 300], [2, 1], 4, 1, 1),                     # eighty: more columns than a CTA's usual
    (128, 1, 128, "bf16", 16, [300], [2], 4, 1, 1),
    (28, 4, 128, "bf16", 64, [9000], [70], 16, 1, 2),                         # a chunk of a prompt
    (4, 4, 64, "bf16", 16, [3000, 129], [300, 65], 16, 1, 2),                 # ... with one head a key head
    (4, 2, 128, "e4m3", 16, [5000, 140], [100, 140], 9, 0, 1),                # two, three, four
    (6, 2, 64, "bf16", 32, [4111], [40], 5, 1, 1),
    (16, 4, 128, "bf16", 16, [2100, 900], [33, 1], 12, 1, 2),
    (18, 2, 128, "bf16", 16, [2500], [20], 7, 1, 1),                          # nine, twenty-four, eighty
    (24, 1, 64, "bf16", 16, [2500, 60], [11, 3], 7, 1, 1),
    (80, 1, 128, "bf16", 16, [2100], [5], 7, 1, 1),
    (128, 1, 128, "e4m3", 16, [2100], [3], 7, 1, 1),
    (2, 2, 64, "bf16", 16, [50, 20], [50, 20], 2, 0, 1),                      # a whole prompt, from the first token on
    (8, 8, 128, "bf16", 16, [9000, 600], [1, 2], 20, 1, 2),                   # more than 512 pages
    (8, 2, 128, "bf16", 16, [70000, 100], [1, 1], 64, 1, 4),                  # more than 4096
    (2, 1, 64, "bf16", 16, [300000], [2], 40, 1, 1),                          # more than 16384
    (4, 2, 64, "bf16", 16, [160, 0, 90], [2, 0, 3], 4, 4, 0),                 # the first pages alone
    (4, 2, 64, "bf16", 16, [160, 40], [3, 6], 4, 1, 3),                       # nothing left to the scores
    (4, 2, 64, "bf16", 16, [5, 3], [8, 3], 1, 0, 0),                          # queries that see no key
    (4, 2, 64, "bf16", 16, [40, 30], [1, 1], 3, 0, 0),                        # all pages
])
def test_pick_matches_the_definition(select, hq, hkv, d, dtype, page, lens, counts, budget, sink, recent):
    pick_case(select, hq, hkv, d, dtype, page, lens, counts, budget, sink, recent, seed=hq * d + page,
              strided=hq % 4 == 0)


@pytest.mark.parametrize("hq,hkv,d,dtype,batch", [(8, 8, 64, "bf16", 70), (14, 2, 64, "bf16", 33), (9, 3, 128, "e4m3", 40),
                                                  (4, 1, 128, "bf16", 129)])
def test_pick_of_batches_whose_lengths_differ(select, hq, hkv, d, dtype, batch):
    rng = np.random.default_rng(batch)
    lens = np.where(rng.random(batch) < 0.2, rng.integers(0, 40, batch), rng.integers(100, 1500, batch)).tolist()
    lens[batch // 2] = 9000
    counts = [1] * batch
    pick_case(select, hq, hkv, d, dtype, 16, lens, counts, 5, 1, 1, seed=batch)
    counts = rng.integers(0, 2, batch).tolist()
    pick_case(select, hq, hkv, d, dtype, 16, lens, counts, 5, 1, 1, seed=batch + 1)
    counts = rng.integers(0, 4, batch).tolist()
    pick_case(select, hq, hkv, d, dtype, 16, lens, counts, 5, 1, 1, seed=batch + 2)


@pytest.mark.parametrize("hq,hkv,d,dtype,batch", [(8, 8, 64, "bf16", 70), (14, 2, 64, "bf16", 33), (8, 2, 128, "e4m3", 40)])
def test_attend_picked_of_batches_whose_lengths_differ(select, hq, hkv, d, dtype, batch):
    rng = np.random.default_rng(batch)
    lens = np.where(rng.random(batch) < 0.2, rng.integers(0, 40, batch), rng.integers(100, 600, batch)).tolist()
    for counts in ([1] * batch, rng.integers(0, 2, batch).tolist(), rng.integers(0, 4, batch).tolist()):
        attend_case(select, hq, hkv, d, dtype, 16, lens, counts, 5, seed=sum(counts))


@pytest.mark.parametrize("lens,budget", [([900], 9), ([9000], 33), ([70001], 100)])
def test_pick_takes_the_lower_of_equal_pages(select, lens, budget):
    for levels in (1, 2, 3):
        pick_case(select, 4, 2, 64, "bf16", 16, lens, [2], budget, 1, 1, seed=levels, levels=levels)


def test_pick_with_a_bound_far_above_the_lengths(select):
    pick_case(select, 4, 2, 128, "bf16", 16, [50, 70], [1, 1], 3, 1, 1, max_len=80)
    rng = np.random.default_rng(3)
    table = np.full((1, 5000), -1, np.int32)
    table[0, :9] = np.arange(9)
    codes, exps = rng.integers(-127, 128, (9, 1, 2, 64)).astype(np.int8), np.zeros((9, 1), np.int8)
    s = select.Selector(1, 8, 8, 2, 1, 64, "bf16")
    q, qv, _ = make_q(rng, 1, 2, 64, "bf16")
    got = s.cache_pick(select.KeyBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), 16), i32(table),
                       i32([140]), q, i32([0, 1]), 80000, 4, 0, 1)
    s.check_device()
    np.testing.assert_array_equal(got.cpu().numpy(), pref.pick(qv, [0, 1], [140], table, codes, exps, 16, 4, 0, 1, 1))
    s.close()


def test_pick_of_special_queries(select):
    """Zeros, NaN (as 0), infinities (as the largest value), values near the type's ends, in queries of one call."""
    rng = np.random.default_rng(12)
    codes, exps = rng.integers(-127, 128, (30, 2, 2, 64)).astype(np.int8), rng.integers(-3, 3, (30, 2)).astype(np.int8)
    table = rng.permutation(30).astype(np.int32)[None]
    x = rng.standard_normal((8, 4, 64))
    x[0] = 0.0
    x[1, 0, 5], x[1, 2, 7] = np.nan, np.nan
    x[2, 1, 3], x[2, 3, 9] = np.inf, -np.inf
    x[3] *= 2.0 ** -130
    x[4] *= 2.0 ** 120
    x[5] = np.nan
    x[6, :, 1:] *= 1e-4
    x[7] *= 2.0 ** -118
    q = torch.from_numpy(x).to(torch.bfloat16).cuda()
    v = q.double().cpu().numpy()
    v = np.where(np.isnan(v), 0.0, np.clip(v, -255 * 2.0 ** 120, 255 * 2.0 ** 120))
    s = select.Selector(1, 8, 8, 4, 2, 64, "bf16")
    got = s.cache_pick(select.KeyBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), 16), i32(table),
                       i32([480]), q, i32([0, 8]), 480, 5, 1, 1)
    s.check_device()
    np.testing.assert_array_equal(got.cpu().numpy(), pref.pick(v, [0, 8], [480], table, codes, exps, 16, 5, 1, 1, 2))
    s.close()


def test_pick_ranks_pages_that_the_pool_has_not_last(select):
    rng = np.random.default_rng(4)
    codes, exps = rng.integers(-127, 128, (20, 1, 2, 64)).astype(np.int8), np.zeros((20, 1), np.int8)
    table = rng.permutation(20).astype(np.int32)[None]
    table[0, [3, 7, 8, 9, 10, 11, 12, 13, 14]] = [-1, 20, 99, -5, 2 ** 31 - 1, -1, -1, -1, -1]
    s = select.Selector(1, 8, 8, 1, 1, 64, "bf16")
    q, qv, _ = make_q(rng, 1, 1, 64, "bf16")
    bounds = select.KeyBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), 16)
    for budget in (5, 14):  # 14: three more than the pages that are there
        got = s.cache_pick(bounds, i32(table), i32([320]), q, i32([0, 1]), 320, budget)
        with pytest.raises(select.LitevlmError) as e:
            s.check_device()
        assert e.value.name == "DEVICE_BOUNDS"
        np.testing.assert_array_equal(got.cpu().numpy(),
                                      pref.pick(qv, [0, 1], [320], table, codes, exps, 16, budget, 0, 0, 1))
    s.close()


# ---------------------------------------------------------------------------------------------------------- attend
def random_lists(rng, lens, off, hkv, budget, page, holes=0.2):
    """Lists with pages in any order, entries that are none between them, pages that the query does not see yet."""
    out = np.full((int(off[-1]), hkv, budget), -1, np.int32)
    for b in range(len(lens)):
        most = -(-lens[b] // page)
        for i in range(off[b], off[b + 1]):
            for h in range(hkv):
                x = rng.permutation(max(most, 1))[:budget].astype(np.int32)
                x[rng.random(len(x)) < holes] = rng.choice([-1, -7, 1 << 30])
                at = rng.permutation(budget)[:len(x)]
                out[i, h, at] = x
    return out


def attend_case(select, hq, hkv, d, dtype, page, lens, counts, budget, seed=0, strided=False, spread=1.0, picked=None):
    rng = np.random.default_rng(seed)
    table, pool = tables(rng, lens, page)
    c = random_pool(rng, pool, hkv, page, d)
    for b, n in enumerate(lens):  # what lies behind the last token may be anything
        if n % page:
            for x in "kv":
                c[x + "_scales"][table[b, n // page], :, n % page:] = 0x7F
    off = offsets(counts)
    q, qv, q_scale = make_q(rng, int(off[-1]), hq, d, dtype)
    if spread != 1.0:
        q, qv = q * spread, qv * spread
    if strided:
        wide = torch.zeros((q.shape[0], hq + 4, d), dtype=q.dtype, device="cuda")
        wide[:, 2:2 + hq] = q
        q = wide[:, 2:2 + hq]
    picked = random_lists(rng, lens, off, hkv, budget, page) if picked is None else picked
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, dtype)
    got = s.cache_attend_picked(to_cache(select, c), i32(table), i32(lens), q, i32(off), i32(picked), q_scale=q_scale,
                                offsets_h=off).double().cpu().numpy()
    s.check_device()
    want, slack = pref.attend(c, table, lens, qv, off, picked)
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) - slack, initial=-np.inf)
    assert worst <= 0, worst
    s.close()


@pytest.mark.parametrize("hq,hkv,d,dtype,page,lens,counts,budget", [
    (4, 4, 64, "bf16", 16, [70, 1, 16, 33], [1, 1, 1, 1], 3),              # a head with keys of its own
    (16, 16, 128, "bf16", 16, [1500], [1], 64),
    (3, 3, 128, "bf16", 256, [1000, 300], [1, 4], 2),
    (2, 2, 128, "e4m3", 32, [500, 0, 64], [2, 0, 1], 9),
    (4, 2, 64, "bf16", 16, [200, 100], [3, 7], 5),                         # two heads
    (28, 4, 128, "bf16", 64, [3000, 70], [1, 2], 12),                      # seven
    (32, 4, 128, "e4m3", 16, [900, 55], [4, 3], 30),                       # eight
    (18, 2, 64, "bf16", 32, [400], [3], 6),                                # nine
    (32, 2, 128, "bf16", 16, [600, 31], [2, 5], 20),                       # sixteen
    (40, 2, 128, "e4m3", 64, [999], [3], 8),                               # twenty
    (8, 8, 128, "bf16", 16, [5, 3], [8, 3], 1),                            # queries that see no key
    (28, 4, 128, "bf16", 16, [40, 400], [40, 60], 6),                      # prompts, from the first token on
    (4, 1, 128, "bf16", 256, [9000], [1], 33),                             # a list split among many CTAs
    (2, 2, 64, "bf16", 128, [9000], [1], 60),
])
def test_attend_picked_matches_the_definition(select, hq, hkv, d, dtype, page, lens, counts, budget):
    attend_case(select, hq, hkv, d, dtype, page, lens, counts, budget, seed=hq + d + page, strided=hq % 8 == 0)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (4, 1, 64, "bf16"), (14, 2, 128, "e4m3"), (5, 1, 64, "bf16")])
@pytest.mark.parametrize("page,budget", [(16, 1), (16, 30), (64, 9)])  # whole lists, and lists in chunks
def test_attend_picked_of_requests_with_few_and_many_rows(select, hq, hkv, d, dtype, page, budget):
    """Rows of a request and key head around 32, 64 and 128 in one call."""
    g = hq // hkv
    counts = [1, 32 // g, 32 // g + 1, 64 // g, 64 // g + 1, 0, 3, 128 // g, 7]
    lens = [700, 900, 40, 333, 1200, 5, 2, 800, 64]
    attend_case(select, hq, hkv, d, dtype, page, lens, counts, budget, seed=budget)
    attend_case(select, hq, hkv, d, dtype, page, lens[:2], [2, 32 // g + 1], budget, seed=budget + 1, strided=True)


@pytest.mark.parametrize("hq,hkv,counts", [(4, 4, [1, 1]), (14, 2, [3, 2]), (28, 4, [50, 30])])
def test_attend_picked_of_lists_that_leave_nothing(select, hq, hkv, counts):
    off, budget = offsets(counts), 4
    lens = [100, 60]
    picked = np.full((int(off[-1]), hkv, budget), -1, np.int32)
    picked[::2, 0] = [9, 50, 1 << 29, -1]   # no page that a query sees
    picked[1::2, hkv - 1, 2] = 0            # one page
    attend_case(select, hq, hkv, 128, "bf16", 16, lens, counts, budget, seed=3, picked=picked)


@pytest.mark.parametrize("hq,hkv,counts", [(8, 2, [0, 3, 0, 1]), (8, 2, [0, 1, 0, 0]), (28, 4, [0, 90, 0, 7]),
                                           (2, 2, [0, 0, 0, 0])])
def test_requests_without_queries_take_no_part(select, hq, hkv, counts):
    lens = [300, 200, 0, 77]
    attend_case(select, hq, hkv, 64, "bf16", 16, lens, counts, 5, seed=1)
    pick_case(select, hq, hkv, 64, "bf16", 16, lens, counts, 3, 1, 1, seed=2)


@pytest.mark.parametrize("hq,hkv,count", [(4, 4, 1), (4, 4, 3), (14, 2, 3), (16, 2, 30)])
def test_attend_picked_over_more_pages_than_a_window(select, hq, hkv, count):
    """More than 65536 pages: the shared lists are made a window of them at a time. The request's pages are the same
    fifty again and again (shared pages are allowed where they are only read)."""
    rng = np.random.default_rng(15)
    page, pages, pool, budget, d = 16, 140000, 50, 6, 64
    n = pages * page - 5
    table = rng.integers(0, pool, (1, pages)).astype(np.int32)
    c, off = random_pool(rng, pool, hkv, page, d), offsets([count])
    q, qv, _ = make_q(rng, count, hq, d, "bf16")
    picked = rng.integers(0, pages - 1, (count, hkv, budget)).astype(np.int32)
    picked[:, :, 0] = pages - 1
    picked[:, :, 1] = rng.integers(65500, 65600, (count, hkv))
    picked[:, :, 2] = rng.integers(0, 3, (count, hkv))
    s = select.Selector(1, 8, 8, hq, hkv, d, "bf16")
    got = s.cache_attend_picked(to_cache(select, c), i32(table), i32([n]), q, i32(off), i32(picked), offsets_h=off)
    s.check_device()
    want, slack = pref.attend(c, table, [n], qv, off, picked)
    assert (np.abs(got.double().cpu().numpy() - want) <= slack).all()
    s.close()


def test_attend_picked_of_flat_and_of_strong_scores(select):
    for spread in (1.0 / 64, 16.0):
        attend_case(select, 8, 8, 128, "bf16", 16, [700, 300], [1, 2], 20, seed=4, spread=spread)
        attend_case(select, 28, 4, 128, "bf16", 16, [700, 300], [5, 30], 20, seed=5, spread=spread)


def test_attend_picked_of_all_pages_is_cache_attend(select):
    """With every page in the lists the two calls agree to the rounding of both outputs (2^-8 each, and 2^-11 each for
    their probabilities)."""
    rng = np.random.default_rng(6)
    hq, hkv, d, page, lens, counts = 28, 4, 128, 32, [300, 77], [3, 5]
    table, pool = tables(rng, lens, page)
    c, off = random_pool(rng, pool, hkv, page, d), offsets(counts)
    cache = to_cache(select, c)
    q, qv, _ = make_q(rng, int(off[-1]), hq, d, "bf16")
    s = select.Selector(2, 8, 8, hq, hkv, d, "bf16")
    lists = np.tile(np.arange(10, dtype=np.int32), (int(off[-1]), hkv, 1))
    a = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), 300, offsets_h=off)
    b = s.cache_attend_picked(cache, i32(table), i32(lens), q, i32(off), i32(lists), offsets_h=off)
    s.check_device()
    _, slack = pref.attend(c, table, lens, qv, off, lists)
    assert (np.abs(a.double().cpu().numpy() - b.double().cpu().numpy()) <= 2 * slack).all()
    s.close()


def test_attend_picked_sees_nan_values_only_where_they_are_seen(select):
    """A NaN value reaches the queries that see its token, and no other."""
    rng = np.random.default_rng(7)
    for hq, hkv in ((2, 2), (14, 2), (28, 4)):
        lens, counts, page = [100], [30], 16
        table, pool = tables(rng, lens, page)
        c, off = random_pool(rng, pool, hkv, page, 128), offsets(counts)
        c["v_scales"][table[0, 5], 0, 9, 3] = 0x7F  # position 89, channels 48 to 63 of key head 0
        picked = np.tile(np.array([5, 0, 6], np.int32), (30, hkv, 1))
        picked[20:] = [6, 1, 2]
        q, _, _ = make_q(rng, 30, hq, 128, "bf16")
        s = select.Selector(1, 8, 8, hq, hkv, 128, "bf16")
        got = s.cache_attend_picked(to_cache(select, c), i32(table), i32(lens), q, i32(off), i32(picked), offsets_h=off)
        s.check_device()
        nan = got.isnan().cpu().numpy()
        want = np.zeros(nan.shape, bool)
        want[19:20, :hq // hkv, 48:64] = True  # query i stands at position 70 + i
        np.testing.assert_array_equal(nan, want)
        s.close()


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 128), (4, 2, 64), (8, 2, 128)])
def test_attend_picked_sees_nan_values_beside_a_request_with_more_rows(select, hq, hkv, d):
    """The same where a request's 30, 60 or 120 rows stand beside one's with more."""
    rng = np.random.default_rng(hq)
    lens, counts, page, g = [100, 90], [30, 128 * hkv // hq], 16, hq // hkv
    table, pool = tables(rng, lens, page)
    c, off = random_pool(rng, pool, hkv, page, d), offsets(counts)
    c["v_scales"][table[0, 5], 0, 9, 3] = 0x7F  # position 89, channels 48 to 63 of key head 0
    picked = np.tile(np.array([5, 0, 6], np.int32), (sum(counts), hkv, 1))
    picked[20:30] = [6, 1, 2]
    picked[30:] = [0, 1, 2]
    q, qv, _ = make_q(rng, sum(counts), hq, d, "bf16")
    s = select.Selector(2, 8, 8, hq, hkv, d, "bf16")
    got = s.cache_attend_picked(to_cache(select, c), i32(table), i32(lens), q, i32(off), i32(picked), offsets_h=off)
    s.check_device()
    got = got.double().cpu().numpy()
    want = np.zeros(got.shape, bool)
    want[19:20, :g, 48:64] = True  # query i of the first stands at position 70 + i
    np.testing.assert_array_equal(np.isnan(got), want)
    c["v_scales"][table[0, 5], 0, 9, 3] = 0x38
    ref_out, slack = pref.attend(c, table, lens, qv, off, picked)
    assert (np.abs(got - ref_out) <= slack)[~want].all()
    s.close()


def test_attend_picked_skips_pages_that_the_pool_has_not(select):
    rng = np.random.default_rng(9)
    table, pool = tables(rng, [100], 16)
    c = random_pool(rng, pool, 2, 16, 64)
    table[0, 2], table[0, 4] = -1, pool
    q, qv, _ = make_q(rng, 1, 4, 64, "bf16")
    picked = np.array([[[0, 2, 4, 5], [2, 4, -1, -1]]], np.int32)
    s = select.Selector(1, 8, 8, 4, 2, 64, "bf16")
    got = s.cache_attend_picked(to_cache(select, c), i32(table), i32([100]), q, i32([0, 1]), i32(picked))
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    want, slack = pref.attend(c, table, [100], qv, [0, 1], picked)
    assert (np.abs(got.double().cpu().numpy() - want) <= slack).all() and (got[0, 2:] == 0).all()
    s.close()


# ------------------------------------------------------------------------------------------------------ in a run
def test_a_decoding_run(select):
    """Prompts, then steps of one token and of drafts: pages reserved, rows appended, ranges renewed, pages picked and
    attended to, everything against the restatement; one request ends and its pages go to another."""
    rng = np.random.default_rng(21)
    hq, hkv, d, page, pool, width, batch = 14, 2, 64, 16, 60, 20, 3
    s = select.Selector(batch, 8, 8, hq, hkv, d, "bf16")
    cache = s.cache(pool, page, k_scale=0.25, v_scale=0.125, weights=False)
    bounds = s.key_bounds(cache)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    free, state = i32(rng.permutation(pool)), i32([0, pool])
    held = np.zeros(batch, np.int64)
    for new, ends in (([200, 90, 17], -1), ([1, 1, 1], -1), ([3, 0, 5], 1), ([1, 64, 1], -1), ([2, 1, 7], -1)):
        if ends >= 0:
            want = held.copy()
            want[ends] = 0
            none = offsets([0] * batch)
            g, state, _ = s.cache_reserve(table, i32(held), i32(want), free, state, page, i32(none), offsets_h=none)
            held = g.cpu().numpy().astype(np.int64)
        new = np.array(new)
        off, want = offsets(new), held + new
        total = int(off[-1])
        granted, state, slots = s.cache_reserve(table, i32(held), i32(want), free, state, page, i32(off), offsets_h=off)
        x = torch.from_numpy(rng.standard_normal((2, total, hkv, d))).to(torch.bfloat16).cuda()
        lens = s.cache_append(cache, table, i32(held), x[0], x[1], i32(off), offsets_h=off)
        s.cache_bounds(cache, bounds, table, lens, i32(off), offsets_h=off)
        q, qv, _ = make_q(rng, total, hq, d, "bf16")
        picked = s.cache_pick(bounds, table, lens, q, i32(off), width * page, 5, 1, 1, offsets_h=off)
        out = s.cache_attend_picked(cache, table, lens, q, i32(off), picked, offsets_h=off)
        s.check_device()
        held = granted.cpu().numpy().astype(np.int64)
        np.testing.assert_array_equal(held, want)
        np.testing.assert_array_equal(lens.cpu().numpy(), held)
        t, c = table.cpu().numpy(), numpy_cache(cache)
        # the slots are where the rows were put
        sl = slots.cpu().numpy()
        code, _ = ref.quantise(x[0].double().cpu().numpy(), 0.25)
        np.testing.assert_array_equal(c["k_codes"][sl // page, :, sl % page], code)
        z = np.zeros((pool, hkv, 2, d), np.int8), np.zeros((pool, hkv), np.int8)
        wc, we = pref.bounds(c, t, held, held, *z)
        mine = np.concatenate([t[b, :-(-held[b] // page)] for b in range(batch)])
        np.testing.assert_array_equal(bounds.codes.cpu().numpy()[mine], wc[mine])
        np.testing.assert_array_equal(bounds.exps.cpu().numpy()[mine], we[mine])
        want_p = pref.pick(qv, off, held, t, wc, we, page, 5, 1, 1, hkv)
        np.testing.assert_array_equal(picked.cpu().numpy(), want_p)
        want_o, slack = pref.attend(c, t, held, qv, off, want_p)
        assert (np.abs(out.double().cpu().numpy() - want_o) <= slack).all()
    s.close()
