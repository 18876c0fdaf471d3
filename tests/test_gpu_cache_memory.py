"""Whose memory the 4-bit cache's calls use, and for how long: a cache's tensors, workspaces, arrays that overlap."""
import gc

import numpy as np
import pytest

from test_gpu_cache import i32, make_q, offsets, random_pool, select, tables, to_cache  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def refused(select, name, call):  # noqa: F811
    with pytest.raises(select.LitevlmError) as e:
        call()
    assert e.value.name == name, str(e.value)


def test_a_cache_s_tensors_and_scales_are_fixed(select):  # noqa: F811
    """The calls use the addresses that a cache was made with: another tensor is refused, not passed over."""
    rng = np.random.default_rng(1)
    table, pool = tables(rng, [200], 16)
    c, other = random_pool(rng, pool, 2, 16, 64), random_pool(rng, pool, 2, 16, 64)
    cache, two = to_cache(select, c, np.zeros((pool, 16), np.float32)), to_cache(select, other)
    s = select.Selector(1, 8, 8, 4, 2, 64, "bf16")
    q, _, _ = make_q(rng, 1, 4, 64, "bf16")
    a = (i32(table), i32([200]), q, i32([0, 1]), 200)
    want = s.cache_attend(cache, *a, accumulate=True)
    for name, value in (("k_codes", two.k_codes), ("k_scales", two.k_scales), ("v_codes", two.v_codes),
                        ("v_scales", two.v_scales), ("k_scale", 3.0), ("v_scale", 3.0), ("page_size", 32),
                        ("num_pages", 1), ("struct", two.struct)):
        refused(select, "INVALID_ARG", lambda: setattr(cache, name, value))
    assert torch.equal(s.cache_attend(cache, *a), want)
    # the weights are read on every call, so they may be others, of the same form
    cache.weights = None
    refused(select, "INVALID_ARG", lambda: s.cache_attend(cache, *a, accumulate=True))
    for bad in (torch.zeros((pool, 8), device="cuda"), torch.zeros((pool, 16)), torch.zeros((pool, 16), device="cuda").double()):
        refused(select, "INVALID_ARG", lambda: setattr(cache, "weights", bad))
    cache.weights = torch.zeros((pool, 16), device="cuda")
    assert torch.equal(s.cache_attend(cache, *a, accumulate=True), want)
    assert abs(float(cache.weights.double().sum()) - 1.0) < 1e-5
    s.check_device()
    s.close()


def test_a_handle_keeps_one_workspace_and_gives_it_back(select):  # noqa: F811
    rng = np.random.default_rng(2)
    n = 60000
    table, pool = tables(rng, [n], 16)
    cache = to_cache(select, random_pool(rng, pool, 2, 16, 64), np.zeros((pool, 16), np.float32))
    s = select.Selector(1, 8, 8, 32, 2, 64, "bf16")
    q, _, _ = make_q(rng, 2, 32, 64, "bf16")
    t, lens, off, off_h = i32(table), i32([n]), i32([0, 2]), offsets([2])
    out = torch.empty((2, 32, 64), dtype=torch.bfloat16, device="cuda")
    need = select.cache_attend_workspace(s.handle, 1, off_h, n)
    assert need > 10 << 20
    torch.cuda.synchronize()
    gc.collect()  # (what earlier tests left behind is not counted)
    before = torch.cuda.memory_allocated()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for st in streams + streams:
        with torch.cuda.stream(st):
            s.cache_attend(cache, t, lens, q, off, n, accumulate=True, offsets_h=off_h, out=out)
        st.synchronize()
    held = torch.cuda.memory_allocated() - before
    assert need <= held < 2 * need
    s.check_device()
    s.close()
    assert torch.cuda.memory_allocated() <= before


def test_the_workspace_follows_the_rows_of_a_call(select):  # noqa: F811
    """Beside what joins the keys' chunks, weights take 4 bytes a row (up to 32 of the longest request's) or tile of 128
    rows and key of max_len, of the call's rows and not of as many for every request as the longest has."""
    most, hq, hkv = 8192, 32, 8
    s = select.Selector(64, 8, 8, hq, hkv, 128, "bf16")
    space = lambda counts, w: select.cache_attend_workspace(s.handle, len(counts), offsets(counts), most, w)  # noqa: E731
    for counts in ([8] + [1] * 31, [1] * 64, [0] * 63 + [8], [8] * 32):
        rows = sum(counts) * hq // hkv
        assert space(counts, True) - space(counts, False) <= hkv * rows * (4 * most + 4) + 512, counts
    for counts in ([1000] + [1] * 31, [0] * 40 + [9], [100] * 8):
        rows = sum(counts) * hq // hkv
        assert space(counts, True) - space(counts, False) <= hkv * ((rows // 128 + len(counts)) * 4 * most + 4 * rows) + 512
    s.close()


@pytest.mark.parametrize("counts", [[3, 0, 8, 1, 0], [70, 1, 0, 33, 129], [0, 0, 128, 256, 0], [1, 1, 1, 1, 40]])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (6, 2)])
def test_a_request_s_weights_do_not_depend_on_the_others(select, counts, hq, hkv):  # noqa: F811
    """Requests of different numbers of rows, some of none, in a workspace of just the bytes asked for: each request's
    outputs and weights are those of the call alone, up to the rounding of other chunks of keys."""
    rng = np.random.default_rng(sum(counts) + hq)
    lens = [300, 50, 260, 401, 300]
    table, pool = tables(rng, lens, 16)
    w = np.exp(rng.standard_normal((pool, 16)) - 5).astype(np.float32)
    cache = to_cache(select, random_pool(rng, pool, hkv, 16, 64), w)
    s = select.Selector(5, 8, 8, hq, hkv, 64, "bf16")
    off = offsets(counts)
    q, _, _ = make_q(rng, int(off[-1]), hq, 64, "bf16")
    bytes_ = select.cache_attend_workspace(s.handle, 5, off, 401)
    room = torch.full((bytes_ + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    nxt = torch.full((pool, 16), -1.0, device="cuda")
    out = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), 401, weights_out=nxt, offsets_h=off,
                         workspace=room[:bytes_])
    assert (room[bytes_:] == 0xAB).all()
    for b, n in enumerate(lens):
        one = torch.full((pool, 16), -1.0, device="cuda")
        rows = slice(int(off[b]), int(off[b + 1]))
        alone = s.cache_attend(cache, i32(table[b:b + 1]), i32([n]), q[rows], i32([0, counts[b]]), n, weights_out=one)
        # both are off the exact values by at most 2^-8 + 2^-9 of the value and of the rounding of probabilities
        assert torch.allclose(out[rows].float(), alone.float(), rtol=2.0 ** -7, atol=2.0 ** -8)
        live = one >= 0
        assert torch.allclose(nxt[live], one[live], rtol=2.0 ** -12, atol=0)
    s.check_device()
    s.close()


def test_arrays_that_overlap_are_refused(select):  # noqa: F811
    """CTAs read what others write there: queries that a later launch reads again, lengths and drafts of other requests."""
    rng = np.random.default_rng(4)
    lens_h = [200, 37, 90]
    table, pool = tables(rng, [n + 64 for n in lens_h], 16)
    w = np.zeros((pool, 16), np.float32)
    cache = to_cache(select, random_pool(rng, pool, 2, 16, 128), w)
    s = select.Selector(3, 8, 8, 8, 2, 128, "bf16")
    t, off, off_h = i32(table), i32([0, 1, 2, 3]), offsets([1, 1, 1])
    buf = i32([0] + lens_h + [0, 0])
    lens = buf[1:4]
    k = torch.from_numpy(rng.standard_normal((3, 2, 128))).to(torch.bfloat16).cuda()
    q, _, _ = make_q(rng, 4, 8, 128, "bf16")
    bad = "INVALID_ARG"
    for at in (0, 1, 2, 3):
        refused(select, bad, lambda: s.cache_append(cache, t, lens, k, k, off, new_lens=buf[at:at + 3]))
        refused(select, bad, lambda: s.cache_evict(cache, t, lens, 200, 20, new_lens=buf[at:at + 3]))
    assert buf.tolist() == [0] + lens_h + [0, 0]
    refused(select, bad, lambda: s.cache_attend(cache, t, lens, q[:3], off, 200, out=q[:3]))
    refused(select, bad, lambda: s.cache_attend(cache, t, lens, q[:3], off, 200, out=q[1:]))
    wide = torch.zeros((pool + 1, 16), device="cuda")
    cache.weights = wide[:pool]
    refused(select, bad, lambda: s.cache_attend(cache, t, lens, q[:3], off, 200, weights_out=wide[1:]))
    raw = lambda ks, vs: select.cache_append(s.handle, 3, cache.struct, t, t.shape[1], lens, k, 256, k, 256, 3, None, off,  # noqa: E731
                                             off_h, 1.0, 1.0, cache.weights, ks, vs, torch.empty_like(lens),
                                             torch.cuda.current_stream().cuda_stream)
    room = torch.empty((7, 2, 128), dtype=torch.bfloat16, device="cuda")
    for ks, vs in ((k, room[:3]), (room[:3], k), (room[:3], room[2:5])):
        refused(select, bad, lambda: raw(ks, vs))
    raw(room[:3], room[3:6])
    x = i32([1, 2, 3, 0, 0, 0, 0])
    p, u = torch.full((6, 5), 0.2, device="cuda"), torch.zeros(3, device="cuda")
    refused(select, bad, lambda: s.verify(x[:3], p, u, u, off, tokens=x[:6]))
    refused(select, bad, lambda: s.verify(x[4:], p, u, u, off, tokens=x[:6]))
    # beside one another they are taken
    new = s.cache_append(cache, t, lens, k, k, off, new_lens=torch.cat([buf, buf])[6:9])
    assert new.tolist() == [n + 1 for n in lens_h]
    many = torch.cat([q[:3], torch.zeros_like(q[:3])])
    out = s.cache_attend(cache, t, lens, many[:3], off, 200, out=many[3:], weights_out=torch.zeros_like(cache.weights))
    assert torch.equal(out, s.cache_attend(cache, t, lens, q[:3], off, 200))
    s.check_device()
    s.close()


@pytest.mark.parametrize("hq,hkv,t", [(4, 4, 1), (8, 2, 1), (8, 2, 4), (8, 2, 16), (8, 2, 70)])
@pytest.mark.parametrize("weights", [False, True])
def test_requests_without_queries_cost_next_to_nothing(select, hq, hkv, t, weights):  # noqa: F811
    """A few requests with queries among many without: the keys are split as if the others were not there, into a
    workspace of the same size but for their weights, and the outputs have the same bits."""
    rng = np.random.default_rng(hq + t)
    batch, active, n = 130, (0, 77, 129), 2500
    lens = np.full(batch, 20)
    lens[list(active)] = n, 700, n - 333
    table, pool = tables(rng, lens.tolist(), 64)
    w = np.exp(rng.standard_normal((pool, 64)) - 5).astype(np.float32)
    cache = to_cache(select, random_pool(rng, pool, hkv, 64, 128), w)
    counts = np.zeros(batch, np.int64)
    counts[list(active)] = t, max(1, t - 2), t
    few = counts[list(active)]
    off, off3 = offsets(counts), offsets(few)
    q, _, _ = make_q(rng, int(off[-1]), hq, 128, "bf16")
    s = select.Selector(batch, 8, 8, hq, hkv, 128, "bf16")
    for wanted in (False, weights):
        many, alone = (select.cache_attend_workspace(s.handle, len(o) - 1, o, n, wanted) for o in (off, off3))
        more = (batch * 8 + 512) + (wanted and hkv * (batch - 3) * 4 * (n + 32) + 512)
        assert many <= alone + more, (many, alone)
    nxt, one = torch.full((pool, 64), -1.0, device="cuda"), torch.full((pool, 64), -1.0, device="cuda")
    out = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), n, weights_out=nxt if weights else None, offsets_h=off)
    want = s.cache_attend(cache, i32(table[list(active)]), i32(lens[list(active)]), q, i32(off3), n,
                          weights_out=one if weights else None, offsets_h=off3)
    assert torch.equal(out, want)
    if weights:
        live = one >= 0
        # (sums of up to t hq positive terms, which warps share by the call's size: two orders of n terms differ by at
        # most n 2^-23 of the sum, 560 2^-23 < 2^-13)
        assert torch.allclose(nxt[live], one[live], rtol=2.0 ** -13, atol=0)
        for b in (1, 50, 128):  # the others' weights as they are
            pos = np.arange(20)
            at = table[b][pos // 64], pos % 64
            assert (nxt.cpu().numpy()[at] == w[at]).all()
    s.check_device()
    s.close()


def test_what_lies_between_rows_does_not_overlap(select):  # noqa: F811
    """Rows far apart in one buffer: the outputs may lie between two of them, and the sources' number of rows, where an
    index picks them, may be any bound."""
    rng = np.random.default_rng(5)
    table, pool = tables(rng, [100, 40], 16)
    cache = to_cache(select, random_pool(rng, pool, 2, 16, 64), np.zeros((pool, 16), np.float32))
    s = select.Selector(2, 8, 8, 4, 2, 64, "bf16")
    t, lens, off, off_h = i32(table), i32([100, 40]), i32([0, 1, 2]), offsets([1, 1])
    q, _, _ = make_q(rng, 2, 4, 64, "bf16")
    room = torch.zeros((2, 64, 4, 64), dtype=torch.bfloat16, device="cuda")
    room[:, 5] = q
    want = s.cache_attend(cache, t, lens, q, off, 100)
    for at in (0, 3, 6, 60):   # beside the first row or between the two
        assert torch.equal(s.cache_attend(cache, t, lens, room[:, 5], off, 100, out=room[0, at:at + 2]), want)
    assert torch.equal(s.cache_attend(cache, t, lens, room[:, 5], off, 100, out=room[1, 6:8]), want)  # behind the last
    for b, at in ((0, 4), (0, 5), (1, 4), (1, 5)):
        refused(select, "INVALID_ARG", lambda: s.cache_attend(cache, t, lens, room[:, 5], off, 100, out=room[b, at:at + 2]))
    assert torch.equal(room[:, 5], q)
    k = torch.from_numpy(rng.standard_normal((2, 2, 64))).to(torch.bfloat16).cuda()
    new = torch.empty_like(lens)
    below = torch.empty((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    below[2:] = k
    for rows in (2, 2 ** 40, 2 ** 62):
        # values written below their sources (above them every byte may be a source's)
        call = lambda a, b: select.cache_append(s.handle, 2, cache.struct, t, t.shape[1], i32([3, 4]), below[2:], 128,  # noqa: E731
                                                below[2:], 128, rows, i32([1, 0]), off, off_h, 1.0, 1.0, cache.weights, a, b,
                                                new, torch.cuda.current_stream().cuda_stream)
        call(below[:2], None)
        assert torch.equal(below[2:], k)
        refused(select, "INVALID_ARG", lambda: call(below[1:3], None))
        refused(select, "INVALID_ARG", lambda: call(None, below[3:]))
    s.check_device()
    s.close()
