"""Rows appended behind a reservation whose answer the host has not seen: a refused request stays as it is, and everybody
else's tokens stay where they are."""
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


def rows_of(rng, n, hkv, d):
    return torch.from_numpy(rng.standard_normal((2, n, hkv, d))).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("hkv,d,dtype,stored", [(2, 64, "bf16", True), (4, 128, "bf16", False), (3, 128, "e4m3", True)])
def test_tokens_behind_the_granted_ones_are_skipped(select, hkv, d, dtype, stored):
    rng = np.random.default_rng(hkv + d)
    lens, counts = [5, 16, 0, 31, 9, 40], [9, 1, 7, 20, 0, 3]
    granted = [14, 16, 0, 40, 9, 10]  # all, none (at a page's end), none of a new request, nine of twenty, nothing new, less
    fit = [9, 0, 0, 9, 0, 0]
    table, pool = tables(rng, [n + f for n, f in zip(lens, fit)], 16)  # (-1 behind what is granted)
    off, total = offsets(counts), sum(counts)
    s = select.Selector(len(lens), 8, 8, hkv, hkv, d, dtype)
    cache = to_cache(select, random_pool(rng, pool, hkv, 16, d), np.full((pool, 16), 7.0, np.float32))
    before = numpy_cache(cache)
    x = rows_of(rng, total, hkv, d)
    if dtype == "e4m3":
        x = x.to(torch.float8_e4m3fn).view(torch.uint8)
    got = s.cache_append(cache, i32(table), i32(lens), x[0], x[1], i32(off), offsets_h=off, stored=stored,
                         granted=i32(granted))
    s.check_device()  # nothing is reported
    new = (got[0] if stored else got).cpu().numpy()
    np.testing.assert_array_equal(new, np.add(lens, fit))
    # the rows that were appended are as without the others
    alone = to_cache(select, before, np.full((pool, 16), 7.0, np.float32))
    keep = np.concatenate([np.arange(off[b], off[b] + fit[b]) for b in range(len(lens))]).astype(np.int32)
    fo = offsets(fit)
    want = s.cache_append(alone, i32(table), i32(lens), x[0], x[1], i32(fo), rows=i32(keep), offsets_h=fo, stored=stored)
    s.check_device()
    a, b = numpy_cache(cache), numpy_cache(alone)
    for k in a:
        np.testing.assert_array_equal(a[k], b[k], err_msg=k)
    assert torch.equal(cache.weights, alone.weights) and (cache.weights == 0).sum() == len(keep)
    if stored:
        at = torch.from_numpy(keep).long().cuda()
        assert torch.equal(got[1][at], want[1]) and torch.equal(got[2][at], want[2])
    s.close()


def test_ranges_of_requests_with_fewer_tokens_than_queries(select):
    """A refused prompt has no tokens, or fewer than the call's: the ranges of all its pages are renewed, with no report."""
    rng = np.random.default_rng(3)
    table, pool = tables(rng, [7, 0, 40], 16)
    c = random_pool(rng, pool, 2, 16, 64)
    s = select.Selector(3, 8, 8, 2, 2, 64, "bf16")
    cache, off, table[1] = to_cache(select, c), offsets([30, 50, 1]), -1
    bounds = s.key_bounds(cache)
    s.cache_bounds(cache, bounds, i32(table), i32([7, 0, 40]), i32(off), offsets_h=off)
    s.check_device()
    z = np.zeros((pool, 2, 2, 64), np.int8), np.zeros((pool, 2), np.int8)
    wc, we = pref.bounds(c, table, [7, 0, 40], [7, 0, 1], *z)
    np.testing.assert_array_equal(bounds.codes.cpu().numpy(), wc)
    np.testing.assert_array_equal(bounds.exps.cpu().numpy(), we)
    # ... and their queries before the first token pick no page and give zeros
    q, _, _ = make_q(rng, 81, 4, 64, "bf16")
    s2 = select.Selector(3, 8, 8, 4, 2, 64, "bf16")
    p = s2.cache_pick(bounds, i32(table), i32([7, 0, 40]), q, i32(off), 48, 2, offsets_h=off)
    o = s2.cache_attend_picked(cache, i32(table), i32([7, 0, 40]), q, i32(off), p, offsets_h=off)
    s2.check_device()
    assert (p[:23] == -1).all() and (p[30:80] == -1).all() and (o[:23] == 0).all() and (o[30:80] == 0).all()
    assert (o[80] != 0).any()
    s.close(), s2.close()


def test_a_captured_step_that_runs_out_of_pages(select):
    """Reserve, append, ranges, selection and attention in one graph. The pages run out; requests that find none wait as
    they are, and go on when another request has ended. Every token that was appended is found where it belongs."""
    rng = np.random.default_rng(1)
    hq, hkv, d, page, pool, width, batch, per = 8, 2, 64, 16, 24, 12, 4, 3  # (three tokens a step)
    s = select.Selector(batch, 8, 8, hq, hkv, d, "bf16")
    off_h = offsets([per] * batch)
    off = i32(off_h)
    c = random_pool(rng, pool, hkv, page, d)
    cache = to_cache(select, c)
    bounds = s.key_bounds(cache)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    free, state, lens = i32(rng.permutation(pool)), i32([0, pool]), i32([0] * batch)
    x, (q, qv, _) = rows_of(rng, batch * per, hkv, d), make_q(rng, batch * per, hq, d, "bf16")

    def step():
        granted, st, slots = s.cache_reserve(table, lens, lens + per, free, state, page, off, offsets_h=off_h)
        new = s.cache_append(cache, table, lens, x[0], x[1], off, offsets_h=off_h, granted=granted)
        s.cache_bounds(cache, bounds, table, new, off, offsets_h=off_h)
        picked = s.cache_pick(bounds, table, new, q, off, width * page, 3, 1, 1, offsets_h=off_h)
        out = s.cache_attend_picked(cache, table, new, q, off, picked, offsets_h=off_h)
        lens.copy_(new)
        state.copy_(st)
        return granted, slots, picked, out

    step()  # (kernels loaded; what it did is taken back)
    for t, v in ((table, -1), (lens, 0)):
        t.fill_(v)
    free.copy_(i32(rng.permutation(pool))), state.copy_(i32([0, pool]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    codes = [ref.quantise(x[i].double().cpu().numpy(), sc) for i, sc in ((0, 0.25), (1, 0.125))]
    held = np.zeros(batch, np.int64)
    waited, model = 0, (table.cpu().numpy(), free.cpu().numpy(), state.tolist())
    for n in range(120):
        if n in (60, 90):  # one ends
            want = held.copy()
            want[(n // 30) % batch] = 0
            none = offsets([0] * batch)
            gr, st, _ = s.cache_reserve(table, lens, i32(want), free, state, page, i32(none), offsets_h=none)
            lens.copy_(gr), state.copy_(st)
            held = want
            model = (table.cpu().numpy(), free.cpu().numpy(), state.tolist())
        g.replay()
        s.check_device()
        wg, wst, wsl, wt, wf = pref.reserve(model[0], held, held + per, model[1], model[2], page, [per] * batch)
        refused = wg == held
        for b in np.flatnonzero(refused):
            wt[b, -(-held[b] // page):-(-(held[b] + per) // page)] = -1
        waited += int(refused.sum())
        for a, b in ((got[0], wg), (got[1], wsl), (table, wt), (free, wf), (state, wst), (lens, wg)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
        held, model = wg.astype(np.int64), (wt, wf, wst.tolist())
        # every page once, every request's tokens in its own
        owned = [int(wt[b, o]) for b in range(batch) for o in range(-(-int(held[b]) // page))]
        owned += [int(wf[(wst[0] + i) % pool]) for i in range(wst[1])]
        assert sorted(owned) == list(range(pool)), n
        if n % 10 == 9:
            now = numpy_cache(cache)
            for b in range(batch):
                pos = np.arange(held[b])
                pg, sl = wt[b, pos // page], pos % page
                for (code, scale), k in zip(codes, "kv"):
                    np.testing.assert_array_equal(now[k + "_codes"][pg, :, sl], code[b * per + pos % per])
                    np.testing.assert_array_equal(now[k + "_scales"][pg, :, sl], scale[b * per + pos % per])
            wc, we = pref.bounds(now, wt, held, held, np.zeros(bounds.codes.shape, np.int8), np.zeros(bounds.exps.shape, np.int8))
            mine = np.array(owned[:sum(-(-int(h) // page) for h in held)], int)
            np.testing.assert_array_equal(bounds.codes.cpu().numpy()[mine], wc[mine])
            # the outputs of those that were served
            served = np.repeat(~refused, per)
            want_p = pref.pick(qv, off_h, held, wt, wc, we, page, 3, 1, 1, hkv)
            np.testing.assert_array_equal(got[2].cpu().numpy()[served], want_p[served])
            want_o, slack = pref.attend(now, wt, held, qv, off_h, want_p)
            assert (np.abs(got[3].double().cpu().numpy() - want_o) <= slack)[served].all()
    assert waited > 50 and (held > 0).all()
    s.close()


def test_refusals(select):
    rng = np.random.default_rng(2)
    table, pool = tables(rng, [20, 20], 16)
    s = select.Selector(2, 8, 8, 2, 2, 64, "bf16")
    cache, lens, off, x = to_cache(select, random_pool(rng, pool, 2, 16, 64)), i32([3, 4]), offsets([1, 1]), rows_of(rng, 2, 2, 64)
    granted = i32([4, 5])

    def call(**kw):
        return s.cache_append(**(dict(cache=cache, table=i32(table), seq_lens=lens, k=x[0], v=x[1], offsets=i32(off), offsets_h=off,
                                      granted=granted) | kw))

    for kw in (dict(granted=granted.long()), dict(granted=granted[:1]), dict(granted=granted.cpu()), dict(new_lens=granted)):
        with pytest.raises(select.LitevlmError) as e:
            call(**kw)
        assert e.value.name == "INVALID_ARG"
    assert call().tolist() == [4, 5]
    # as the lengths' own array: nothing is granted
    assert call(granted=lens).tolist() == [3, 4]
    s.check_device()
    s.close()
