"""The 4-bit K/V cache on the GPU against a plain 64-bit restatement: rows appended, attention that reads them with the
weights it adds up, eviction, drafts verified, each at the sizes where it can go wrong, and all of them in a run."""
import numpy as np
import pytest

import cache_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def tables(rng, lens, page, spare=2):
    """Random distinct pages for every request; -1 behind a request's last page."""
    need = [-(-n // page) for n in lens]
    pool = sum(need) + spare
    perm, table, at = rng.permutation(pool), np.full((len(lens), max(1, max(need))), -1, np.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = perm[at:at + m]
        at += m
    return table, pool


def random_pool(rng, pool, hkv, page, d, k_scale=0.25, v_scale=0.125):
    """A pool of random codes and scales of moderate size; NaN scales (0x7F) are put in by the tests that want them."""
    c = dict(k_scale=k_scale, v_scale=v_scale)
    for x in "kv":
        c[x + "_codes"] = rng.integers(0, 256, (pool, hkv, page, d // 2), dtype=np.uint8)
        c[x + "_scales"] = rng.integers(0x28, 0x40, (pool, hkv, page, d // 16), dtype=np.uint8)
    return c


def to_cache(select, c, weights=None):
    t = [torch.from_numpy(c[x]).cuda() for x in ("k_codes", "k_scales", "v_codes", "v_scales")]
    w = None if weights is None else torch.from_numpy(weights).cuda()
    return select.KVCache(*t, c["k_scale"], c["v_scale"], w)


def numpy_cache(cache):
    return {x: getattr(cache, x).cpu().numpy() for x in ("k_codes", "k_scales", "v_codes", "v_scales")} | {
        "k_scale": cache.k_scale, "v_scale": cache.v_scale}


def make_q(rng, rows, hq, d, dtype):
    x = rng.standard_normal((rows, hq, d)).astype(np.float32)
    if dtype == "bf16":
        t = torch.from_numpy(x).to(torch.bfloat16).cuda()
        return t, t.double().cpu().numpy(), 1.0
    scale = 0.0137
    codes = torch.from_numpy(x / scale / 8).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    return codes, ref.E4M3[codes.cpu().numpy()] * float(np.float32(scale)), scale


# ---------------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("hkv,d,page,dtype,lens,counts", [
    (4, 128, 16, "bf16", [0, 5, 16, 31], [1, 17, 0, 40]),
    (1, 64, 64, "bf16", [3], [1]),
    (3, 64, 32, "bf16", [0, 100], [70, 3]),
    (2, 128, 256, "e4m3", [255, 0], [2, 300]),
])
def test_append_matches_the_definition(select, hkv, d, page, dtype, lens, counts):
    rng = np.random.default_rng(hkv * d + page)
    table, pool = tables(rng, [a + b for a, b in zip(lens, counts)], page)
    off, total = offsets(counts), sum(counts)
    s = select.Selector(len(lens), 8, 8, hkv, hkv, d, dtype)
    cache = s.cache(pool, page, k_scale=0.25, v_scale=0.3)
    cache.weights.fill_(7.0)
    before = numpy_cache(cache)
    # K and V as parts of one fused projection's rows; picked by an index
    src = rng.permutation(total + 9)[:total].astype(np.int32)
    x = rng.standard_normal((total + 9, 2 * hkv, d)) * np.exp(rng.standard_normal((total + 9, 2 * hkv, 1)))
    x[:, :, :16] *= 1e-3
    x[0, :, 16:32] = 0.0
    x[1, :, ::7] = -0.0
    x[2] = np.round(x[2] * 4) / 4  # ties
    in_scale = 1.0 if dtype == "bf16" else 0.0231
    if dtype == "bf16":
        t = torch.from_numpy(x).to(torch.bfloat16).cuda()
        xv = t.double().cpu().numpy()
    else:
        t = torch.from_numpy(x.astype(np.float32) / in_scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
        xv = ref.E4M3[t.cpu().numpy()]
    got = s.cache_append(cache, i32(table), i32(lens), t[:, :hkv], t[:, hkv:], i32(off), rows=i32(src),
                         k_in_scale=in_scale, v_in_scale=in_scale, offsets_h=off, stored=True)
    s.check_device()
    new_lens, stored = got[0].cpu().numpy(), got[1:]
    np.testing.assert_array_equal(new_lens, np.add(lens, counts))
    after, w = numpy_cache(cache), cache.weights.cpu().numpy()
    want, want_w = {k: v.copy() if k[1:] != "_scale" else v for k, v in before.items()}, np.full(w.shape, 7.0, np.float32)
    for b in range(len(lens)):
        for i in range(counts[b]):
            r, p = off[b] + i, lens[b] + i
            pg, sl = table[b, p // page], p % page
            want_w[pg, sl] = 0.0
            for n, x_part, sc in (("k", xv[src[r], :hkv], 0.25), ("v", xv[src[r], hkv:], np.float32(0.3))):
                c, f = ref.quantise(x_part, sc, in_scale)
                want[n + "_codes"][pg, :, sl], want[n + "_scales"][pg, :, sl] = c, f
                st = ref.E2M1[np.stack((c & 15, c >> 4), -1).reshape(hkv, d)] * np.repeat(ref.E4M3[f], 16, -1)
                st = ref.bf16_bits(st.astype(np.float32) * np.float32(sc))
                np.testing.assert_array_equal(stored["kv".index(n)][r].double().cpu().numpy(), st)
    for k in ("k_codes", "k_scales", "v_codes", "v_scales"):
        np.testing.assert_array_equal(after[k], want[k], err_msg=k)
    np.testing.assert_array_equal(w, want_w)
    s.close()


def test_append_of_special_values(select):
    """A NaN makes its block's scale NaN; infinities and values beyond 448 * 6 saturate; tiny ones keep their sign."""
    s = select.Selector(1, 8, 8, 1, 1, 128, "bf16")
    cache = s.cache(1, 16)
    x = torch.zeros((2, 1, 128))
    x[0, 0, 3] = float("nan")
    x[0, 0, 16:18] = torch.tensor([float("inf"), 1.0])
    x[0, 0, 32:34] = torch.tensor([-1e30, 5.0])
    x[0, 0, 48:50] = torch.tensor([1e-9, -1e-9])
    x[0, 0, 64:66] = torch.tensor([-3e38, 3e38])
    x[0, 0, 80] = 2.0 ** -126
    k = x.to(torch.bfloat16).cuda()
    s.cache_append(cache, i32([[0]]), i32([0]), k, -k, i32([0, 2]))
    s.check_device()
    for name, sign in (("k", 1), ("v", -1)):
        c, f = ref.quantise(sign * k.double().cpu().numpy(), 1.0)
        np.testing.assert_array_equal(getattr(cache, name + "_scales")[0, 0, :2].cpu().numpy(), f[:, 0])
        np.testing.assert_array_equal(getattr(cache, name + "_codes")[0, 0, :2].cpu().numpy(), c[:, 0])
    s.close()


def test_append_out_of_range_is_skipped_and_reported(select):
    """Positions behind the table's row, pages outside the pool and source rows outside k are skipped."""
    s = select.Selector(3, 8, 8, 2, 2, 64, "bf16")
    cache = s.cache(4, 16)
    k = torch.ones((6, 2, 64), dtype=torch.bfloat16, device="cuda")
    table = i32([[0], [4], [-1]])
    lens = s.cache_append(cache, table, i32([15, 0, 3]), k, k, i32([0, 2, 4, 6]))
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    assert lens.tolist() == [16, 2, 5]
    hit = torch.nonzero(cache.k_scales.amax((1, 3))).tolist()
    assert hit == [[0, 15]]
    s.cache_append(cache, i32([[1]]), i32([0]), k, k, i32([0, 3]), rows=i32([5, 6, -1]))
    with pytest.raises(select.LitevlmError):
        s.check_device()
    assert torch.nonzero(cache.k_scales.amax((1, 3))).tolist() == [[0, 15], [1, 0]]
    lens = s.cache_append(cache, i32([[1], [2]]), i32([-5, 99]), k, k, i32([0, 1, 1]))
    with pytest.raises(select.LitevlmError):
        s.check_device()
    assert lens.tolist() == [1, 16]
    s.close()


# ---------------------------------------------------------------------------------------------------------- attend
CASES = [
    # hq, hkv, d, page, dtype, lens, queries
    (4, 4, 64, 16, "bf16", [1], [1]),
    (16, 16, 128, 16, "bf16", [17, 1, 64, 333], [1, 1, 1, 1]),
    (28, 4, 128, 32, "bf16", [700, 33], [1, 1]),
    (14, 2, 64, 128, "bf16", [129, 0, 15], [1, 1, 1]),
    (8, 1, 128, 64, "bf16", [65], [1]),
    (9, 3, 64, 256, "bf16", [300, 40], [2, 5]),
    (32, 8, 128, 32, "e4m3", [1000, 77, 16, 515], [8, 0, 3, 1]),
    (28, 4, 128, 16, "bf16", [90, 50], [40, 13]),          # several row tiles
    (4, 4, 128, 64, "bf16", [3, 10, 0], [7, 10, 2]),       # more queries than keys: rows that see nothing
    (2, 2, 64, 16, "bf16", [5000], [1]),                   # many chunks
    (4, 2, 128, 16, "e4m3", [2100, 5], [33, 5]),
    (12, 12, 64, 32, "bf16", [260], [70]),
    (16, 2, 64, 32, "bf16", [600, 1300, 45], [30, 2, 45]),  # 240 rows: two row tiles, the second of them in part
    (7, 1, 128, 16, "e4m3", [900, 300], [90, 1]),
    (8, 2, 128, 256, "bf16", [400, 20, 129], [16, 9, 12]),  # 36 to 64 rows: places of their own
]


@pytest.mark.parametrize("hq,hkv,d,page,dtype,lens,counts", CASES)
@pytest.mark.parametrize("weights", [False, True])
def test_attend_matches_the_definition(select, hq, hkv, d, page, dtype, lens, counts, weights):
    rng = np.random.default_rng(hq * 1000 + d + page)
    table, pool = tables(rng, lens, page)
    c = random_pool(rng, pool, hkv, page, d)
    # whatever lies behind a request's last token does not matter: NaN scales there
    for b, n in enumerate(lens):
        if n % page:
            for x in "kv":
                c[x + "_scales"][table[b, n // page], :, n % page:] = 0x7F
    w = np.exp(2 * rng.standard_normal((pool, page)) - 5).astype(np.float32)
    cache = to_cache(select, c, w)
    off = offsets(counts)
    q, qv, q_scale = make_q(rng, int(off[-1]), hq, d, dtype)
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, dtype)
    # rows of a wider tensor
    wide = torch.zeros((q.shape[0], hq + 2, d), dtype=q.dtype, device="cuda")
    wide[:, 1:-1] = q
    nxt = torch.full_like(cache.weights, -1.0)
    out = s.cache_attend(cache, i32(table), i32(lens), wide[:, 1:-1], i32(off), max(lens), q_scale=q_scale,
                         weights_out=nxt if weights else None, offsets_h=off)
    s.check_device()
    o, wn, slack, slack_w = ref.attend(c, table, lens, qv, off, hq, w if weights else None)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = float((np.abs(got - o) / np.maximum(slack, 1e-30)).max())
    assert worst <= 1.0
    assert (cache.weights.cpu().numpy() == w).all()
    if weights:
        touched = slack_w > 0
        g = nxt.double().cpu().numpy()
        assert (g[~touched] == -1.0).all()
        assert (np.abs(g - wn)[touched] <= slack_w[touched]).all()
        # in place, twice: the same bits as out of place, then added up
        again = s.cache_attend(cache, i32(table), i32(lens), q, i32(off), max(lens), q_scale=q_scale, accumulate=True)
        assert torch.equal(again, out)
        m = torch.from_numpy(touched).cuda()
        assert torch.equal(cache.weights[m], nxt[m])
        assert torch.equal(cache.weights[~m].cpu(), torch.from_numpy(w)[torch.from_numpy(~touched)])
    s.close()


def test_attend_extreme_scores(select):
    """Scores far apart, equal ones, and references that move often; the largest and the smallest queries of bf16."""
    rng = np.random.default_rng(5)
    hq, d, n = 8, 128, 700
    table, pool = tables(rng, [n], 16)
    c = random_pool(rng, pool, 1, 16, d)
    q = np.zeros((1, hq, d), np.float32)
    q[0, 0] = 40 * rng.standard_normal(d)      # a few keys take everything
    q[0, 2] = 2.0 ** -100 * rng.standard_normal(d)
    q[0, 3, 5] = 2.0 ** 9
    q[0, 4] = rng.standard_normal(d) * 2.0 ** rng.integers(-40, 3, d)
    q[0, 5] = -q[0, 0]
    q[0, 6] = rng.standard_normal(d)
    t = torch.from_numpy(q).to(torch.bfloat16).cuda()
    s = select.Selector(1, 8, 8, hq, 1, d, "bf16")
    w = np.zeros((pool, 16), np.float32)
    cache = to_cache(select, c, w)
    out = s.cache_attend(cache, i32(table), i32([n]), t, i32([0, 1]), n, accumulate=True)
    s.check_device()
    o, wn, slack, slack_w = ref.attend(c, table, [n], t.double().cpu().numpy(), offsets([1]), hq, w)
    assert (np.abs(out.double().cpu().numpy() - o) <= slack).all()
    g = cache.weights.double().cpu().numpy()
    assert (np.abs(g - wn)[slack_w > 0] <= slack_w[slack_w > 0]).all()
    s.close()


@pytest.mark.parametrize("t", [6, 40])
def test_attend_nan_reaches_only_the_rows_that_see_it(select, t):
    """A NaN or infinite query channel, a NaN key, a NaN value: rows that do not see them are as without them."""
    rng = np.random.default_rng(6)
    hq, d, n = 4, 128, 100
    table, pool = tables(rng, [n], 16)
    clean = random_pool(rng, pool, 2, 16, d)
    q, qv, _ = make_q(rng, t, hq, d, "bf16")
    s = select.Selector(1, 8, 8, hq, 2, d, "bf16")
    base = s.cache_attend(to_cache(select, clean), i32(table), i32([n]), q, i32([0, t]), n)
    # a NaN value block at the position of query 3, head 1: rows from query 3 on, heads 2 and 3, channels 32..47
    c = {k: v.copy() if hasattr(v, "copy") else v for k, v in clean.items()}
    p = n - t + 3
    c["v_scales"][table[0, p // 16], 1, p % 16, 2] = 0x7F
    out = s.cache_attend(to_cache(select, c), i32(table), i32([n]), q, i32([0, t]), n)
    want = torch.zeros((t, hq, d), dtype=torch.bool)
    want[3:, 2:, 32:48] = True
    assert torch.equal(torch.isnan(out).cpu(), want)
    assert torch.equal(out[~want.cuda()], base[~want.cuda()])
    # a NaN key there: the rows from query 3 on of those heads, and nothing else
    c = {k: v.copy() if hasattr(v, "copy") else v for k, v in clean.items()}
    c["k_scales"][table[0, p // 16], 1, p % 16, 2] = 0x7F
    out = s.cache_attend(to_cache(select, c), i32(table), i32([n]), q, i32([0, t]), n)
    want = torch.zeros((t, hq), dtype=torch.bool)
    want[3:, 2:] = True
    assert torch.equal(torch.isnan(out).all(-1).cpu(), want)
    assert torch.equal(out[~want.cuda()], base[~want.cuda()])
    for bad in (float("nan"), float("inf"), float("-inf")):
        q2 = q.clone()
        q2[1, 2, 7] = bad
        out = s.cache_attend(to_cache(select, clean), i32(table), i32([n]), q2, i32([0, t]), n)
        want = torch.zeros((t, hq), dtype=torch.bool)
        want[1, 2] = True
        assert torch.equal(torch.isnan(out).all(-1).cpu(), want)
        assert torch.equal(out[~want.cuda()], base[~want.cuda()])
    s.check_device()
    s.close()


def test_attend_bad_pages_and_lengths_are_skipped_and_reported(select):
    rng = np.random.default_rng(7)
    hq, d = 4, 64
    c = random_pool(rng, 6, 2, 16, d)
    w = np.ones((6, 16), np.float32)
    cache = to_cache(select, c, w)
    q, qv, _ = make_q(rng, 3, hq, d, "bf16")
    table = np.array([[0, 99, 2], [3, 4, -7], [5, -1, -1]], np.int32)
    s = select.Selector(3, 8, 8, hq, 2, d, "bf16")
    out = s.cache_attend(cache, i32(table), i32([40, 33, -3]), q, i32([0, 1, 2, 3]), 48, accumulate=True)
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    s.check_device()  # cleared
    # as if the skipped tokens were not there
    short = np.array([[0, 2], [3, 4], [5, -1]], np.int32)
    o, wn, slack, slack_w = ref.attend(c, short, [24, 32, 0], qv, offsets([1, 1, 1]), hq, w)
    assert (np.abs(out.double().cpu().numpy() - o) <= slack).all()
    g = cache.weights.double().cpu().numpy()
    assert (np.abs(g - wn) <= np.maximum(slack_w, 0)).all()
    # a length beyond max_len is cut to it
    out = s.cache_attend(cache, i32([[0, 2]]), i32([30]), q[:1], i32([0, 1]), 20)
    with pytest.raises(select.LitevlmError):
        s.check_device()
    o, _, slack, _ = ref.attend(c, np.array([[0, 2]]), [20], qv[:1], offsets([1]), hq)
    assert (np.abs(out.double().cpu().numpy() - o) <= slack).all()
    s.close()


# ----------------------------------------------------------------------------------------------------------- evict
@pytest.mark.parametrize("hkv,d,page,lens,budget,sink,recent,kind", [
    (2, 128, 16, [100, 40, 41, 0, 39], 40, 4, 8, "plain"),
    (1, 64, 64, [1000], 1, 0, 0, "plain"),
    (3, 64, 32, [700, 701], 333, 0, 333, "plain"),
    (2, 128, 128, [4097, 200, 3000], 1500, 5, 100, "ties"),
    (1, 64, 16, [20000], 7777, 1, 5, "ties"),
    (2, 64, 256, [600, 500], 300, 2, 3, "special"),
    (1, 128, 16, [300], 299, 0, 0, "special"),
])
@pytest.mark.parametrize("inplace", [False, True])
def test_evict_matches_the_definition(select, hkv, d, page, lens, budget, sink, recent, kind, inplace):
    rng = np.random.default_rng(budget + page)
    both = list(lens) if inplace else list(lens) + [min(n, budget) for n in lens]
    table, pool = tables(rng, both, page)
    c = random_pool(rng, pool, hkv, page, d)
    w = np.exp(2 * rng.standard_normal((pool, page)) - 5).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 40).astype(np.float32) / 40
    if kind == "special":
        w = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1.0, 1e-40], np.float32), w.shape)
    cache = to_cache(select, c, w)
    from_t = table[:len(lens)]
    to_t = from_t if inplace else table[len(lens):, :max(1, -(-min(max(lens), budget) // page))]
    s = select.Selector(len(lens), 8, 8, hkv, hkv, d, "bf16")
    kept, new_lens = s.cache_evict(cache, i32(from_t), i32(lens), max(lens), budget, sink, recent,
                                   to_table=None if inplace else i32(to_t))
    s.check_device()
    want = {k: v.copy() for k, v in c.items() if hasattr(v, "copy")}
    want_w = w.copy()
    for b, n in enumerate(lens):
        pos = np.arange(n)
        row = w[from_t[b][pos // page], pos % page]
        k = ref.evict(row, n, budget, sink, recent)
        assert kept[b].tolist() == k.tolist() + [-1] * (budget - len(k))
        assert int(new_lens[b]) == len(k)
        i = np.arange(len(k))
        f, t = (from_t[b][k // page], k % page), (to_t[b][i // page], i % page)
        for x in ("k_codes", "k_scales", "v_codes", "v_scales"):
            want[x][t[0], :, t[1]] = c[x][f[0], :, f[1]]
        want_w[t] = w[f]
    for x in ("k_codes", "k_scales", "v_codes", "v_scales"):
        np.testing.assert_array_equal(getattr(cache, x).cpu().numpy(), want[x], err_msg=x)
    np.testing.assert_array_equal(cache.weights.cpu().numpy().view(np.int32), want_w.view(np.int32))
    s.close()


def test_evict_bad_pages_are_skipped_and_reported(select):
    rng = np.random.default_rng(9)
    c = random_pool(rng, 4, 1, 16, 64)
    w = np.ones((4, 16), np.float32)
    cache = to_cache(select, c, w)
    s = select.Selector(1, 8, 8, 1, 1, 64, "bf16")
    kept, lens = s.cache_evict(cache, i32([[0, 77, 1]]), i32([48]), 48, 32)
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    # tokens without a page rank lowest
    assert kept[0].tolist() == list(range(16)) + list(range(32, 48)) and lens.tolist() == [32]
    s.close()


# ---------------------------------------------------------------------------------------------------------- verify
@pytest.mark.parametrize("vocab", [1, 31, 1000, 4097, 50001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafts", [True, False])
def test_verify_matches_the_definition(select, vocab, dtype, drafts):
    rng = np.random.default_rng(vocab)
    counts = [0, 1, 4, 8, 3, 0, 30]
    off, total, batch = offsets(counts), sum(counts), len(counts)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    lg = 3 * rng.standard_normal((total + batch, vocab))
    req = np.repeat(np.arange(batch), counts)
    p = torch.softmax(torch.from_numpy(lg), -1).to(kind)
    q = torch.softmax(torch.from_numpy(lg[np.arange(total) + req] + 0.6 * rng.standard_normal((total, vocab))), -1).to(kind)
    x = np.array([rng.choice(vocab, p=(r / r.sum())) for r in q.double().numpy()], np.int32)
    x[5] = vocab // 2
    p[3] = 0.0                      # nothing to sample
    q[12] = p[12 + req[12]]         # refused only by chance; then p - q has nothing above 0
    u, ul = rng.random(total).astype(np.float32), rng.random(batch).astype(np.float32)
    u[12] = 1.0
    ul[0], ul[2] = 0.0, 1.0
    if vocab > 100:
        p[20, 5] = float("nan")
        q[3, 7] = float("nan")
    s = select.Selector(batch, 8, 8, 4, 4, 128, "bf16")
    acc, tok = s.verify(i32(x), p.cuda(), torch.from_numpy(u).cuda(), torch.from_numpy(ul).cuda(), i32(off),
                        draft_probs=q.cuda() if drafts else None)
    s.check_device()
    pn, qn = p.double().numpy(), q.double().numpy()
    for b in range(batch):
        a, t = ref.verify(x[off[b]:off[b + 1]], pn[off[b] + b:off[b + 1] + b + 1],
                          qn[off[b]:off[b + 1]] if drafts else None, u[off[b]:off[b + 1]], ul[b])
        assert int(acc[b]) == a, b
        assert tok[off[b] + b:off[b + 1] + b + 1].tolist() == t.tolist(), b
    s.close()


def test_verify_borders(select):
    """Draws that fall on a border between two tokens: weights whose sums are exact, every border tried."""
    vocab = 4096
    p = torch.full((vocab + 1, vocab), 1.0 / vocab)  # one request for every border, no drafts
    p = p[:vocab].cuda()
    u = (torch.arange(vocab, dtype=torch.float64) / vocab).float().cuda()
    s = select.Selector(vocab, 8, 8, 4, 4, 128, "bf16")
    off = np.zeros(vocab + 1, np.int32)
    acc, tok = s.verify(torch.empty(0, dtype=torch.int32, device="cuda"), p,
                        torch.empty(0, dtype=torch.float32, device="cuda"), u, i32(off))
    s.check_device()
    assert not acc.any()
    assert torch.equal(tok.cpu(), torch.arange(vocab, dtype=torch.int32))
    s.close()


def test_verify_bad_tokens_are_refused_and_reported(select):
    s = select.Selector(2, 8, 8, 4, 4, 128, "bf16")
    p = torch.full((5, 8), 0.125, device="cuda")
    q = torch.full((3, 8), 0.125, device="cuda")
    acc, tok = s.verify(i32([8, 1, -1]), p, torch.zeros(3, device="cuda"), torch.full((2,), 0.5, device="cuda"),
                        i32([0, 1, 3]), draft_probs=q)
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "DEVICE_BOUNDS"
    assert acc.tolist() == [0, 1] and tok.tolist() == [4, -1, 1, 4, -1]
    s.close()


# ------------------------------------------------------------------------------------------------------- together
def test_a_run_of_the_operators(select):
    """Kept rows of a selection go into the cache; tokens are decoded, with drafts now and then; when the cache passes
    its budget it is cut back by the weights that the steps have added up. Every step against the restatement."""
    rng = np.random.default_rng(11)
    hq, hkv, d, page, batch, vocab = 8, 2, 128, 16, 3, 257
    n_vis, keep = [200, 130, 90], [60, 39, 27]
    s = select.Selector(batch, sum(n_vis), 64, hq, hkv, d, "bf16")
    so, to = offsets(n_vis), offsets([8, 5, 3])
    k = torch.from_numpy(rng.standard_normal((sum(n_vis), hkv, d))).to(torch.bfloat16).cuda()
    v = torch.from_numpy(rng.standard_normal((sum(n_vis), hkv, d))).to(torch.bfloat16).cuda()
    qt = torch.from_numpy(rng.standard_normal((16, hq, d))).to(torch.bfloat16).cuda()
    _, kept, _, kept_h = s.score_topk(qt, i32(to), k, i32(so), keep_k=np.array(keep, np.int32), seq_offsets_h=so,
                                      text_offsets_h=to)
    table, pool = tables(rng, [112] * batch, page)
    cache, tab = s.cache(pool, page), i32(table)
    lens = s.cache_append(cache, tab, i32([0] * batch), k, v, i32(kept_h), rows=kept, offsets_h=kept_h)
    assert lens.tolist() == keep
    n, w = np.array(keep), np.zeros((pool, page))
    w_slack = np.zeros((pool, page))
    for step in range(12):
        t = int(rng.integers(1, 4))
        off = offsets([t] * batch)
        new = [torch.from_numpy(rng.standard_normal((t * batch, h, d))).to(torch.bfloat16).cuda() for h in (hkv, hkv, hq)]
        lens = s.cache_append(cache, tab, lens, new[0], new[1], i32(off))
        n = n + t
        out = s.cache_attend(cache, tab, lens, new[2], i32(off), 112, accumulate=True)
        for b in range(batch):
            pos = np.arange(n[b] - t, n[b])
            w[table[b][pos // page], pos % page] = 0
            w_slack[table[b][pos // page], pos % page] = 0
        o, w, slack, ws = ref.attend(numpy_cache(cache), table, n, new[2].double().cpu().numpy(), off, hq, w)
        w_slack += ws
        assert (np.abs(out.double().cpu().numpy() - o) <= slack).all()
        live = np.zeros(w.shape, bool)
        for b in range(batch):
            pos = np.arange(n[b])
            live[table[b][pos // page], pos % page] = True
        got = cache.weights.double().cpu().numpy()
        assert (np.abs(got - w) <= w_slack)[live].all()
        if t > 1:  # the drafts behind the first token are verified; the cache forgets the refused ones
            p = torch.softmax(torch.from_numpy(rng.standard_normal((t * batch, vocab))), -1).float()
            dq = torch.softmax(torch.from_numpy(rng.standard_normal(((t - 1) * batch, vocab))), -1).float()
            x = rng.integers(0, vocab, (t - 1) * batch).astype(np.int32)
            u = rng.random(((t - 1) * batch)).astype(np.float32)
            ul = rng.random(batch).astype(np.float32)
            do = offsets([t - 1] * batch)
            acc, _ = s.verify(i32(x), p.cuda(), torch.from_numpy(u).cuda(), torch.from_numpy(ul).cuda(), i32(do),
                              draft_probs=dq.cuda())
            for b in range(batch):
                a, _ = ref.verify(x[do[b]:do[b + 1]], p.numpy()[do[b] + b:do[b + 1] + b + 1], dq.numpy()[do[b]:do[b + 1]],
                                  u[do[b]:do[b + 1]], ul[b])
                assert int(acc[b]) == a
            lens = lens - (t - 1) + acc
            n = n - (t - 1) + acc.cpu().numpy()
        if (n > 50).any():
            weights = cache.weights.cpu().numpy()
            kept_idx, lens2 = s.cache_evict(cache, tab, lens, 112, 45, 2, 6)
            for b in range(batch):
                pos = np.arange(n[b])
                row = weights[table[b][pos // page], pos % page]
                kk = ref.evict(row, int(n[b]), 45, 2, 6)
                assert kept_idx[b, :len(kk)].tolist() == kk.tolist()
                moved = np.arange(len(kk))
                for arr in (w, w_slack):
                    arr[table[b][moved // page], moved % page] = arr[table[b][kk // page], kk % page].copy()
            lens = lens2
            n = np.minimum(n, 45)
        assert lens.tolist() == n.tolist()
    s.check_device()
    s.close()
