"""How the 4-bit cache's calls are made: captured and replayed, on streams of their own, two at once, on pools of more
than 4 GiB, empty, wrong, and giving up."""
import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import i32, make_q, numpy_cache, offsets, random_pool, tables, to_cache

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def setup(select, rng, hq=8, hkv=2, d=128, page=16, lens=(200, 37, 90), counts=(1, 1, 1), room=64):
    table, pool = tables(rng, [n + room for n in lens], page)
    c = random_pool(rng, pool, hkv, page, d)
    w = np.exp(rng.standard_normal((pool, page)) - 5).astype(np.float32)
    s = select.Selector(len(lens), 8, 8, hq, hkv, d, "bf16")
    q, qv, _ = make_q(rng, int(sum(counts)), hq, d, "bf16")
    return s, c, w, table, q, qv


def test_a_captured_step_is_replayed_as_lengths_change(select):
    rng = np.random.default_rng(1)
    s, c, w, table, q, _ = setup(select, rng)
    off = offsets([1, 1, 1])
    k = torch.from_numpy(rng.standard_normal((3, 2, 128))).to(torch.bfloat16).cuda()
    args = (i32(table), i32(off))
    one, two = to_cache(select, c, w), to_cache(select, c, w)
    lens, lens2 = i32([200, 37, 90]), i32([200, 37, 90])

    def step(cache, lens):
        new = s.cache_append(cache, args[0], lens, k, k, args[1], offsets_h=off)
        out = s.cache_attend(cache, args[0], new, q, args[1], 264, accumulate=True, offsets_h=off)
        lens.copy_(new)
        return out

    step(to_cache(select, c, w), i32([200, 37, 90]))  # (kernels loaded, workspace of the eager calls made)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(one, lens)
    lens.copy_(i32([200, 37, 90]))
    for n in range(6):
        g.replay()
        want = step(two, lens2)
        assert torch.equal(out, want), n
    assert torch.equal(lens, lens2) and lens.tolist() == [206, 43, 96]
    assert torch.equal(one.weights, two.weights) and torch.equal(one.k_codes, two.k_codes)
    s.check_device()
    s.close()


def test_two_captured_graphs_run_at_once(select):
    """Each graph has a workspace of its own; a split call's chunks would otherwise mix."""
    rng = np.random.default_rng(2)
    cases = []
    for n in (30000, 29000):
        s, c, w, table, q, qv = setup(select, rng, lens=(n,), counts=(1,))
        cache, nxt = to_cache(select, c, w), torch.zeros((c["k_codes"].shape[0], 16), device="cuda")
        a = (cache, i32(table), i32([n]), q, i32([0, 1]), n)
        want = (s.cache_attend(*a, weights_out=nxt, offsets_h=offsets([1])).clone(), nxt.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = s.cache_attend(*a, weights_out=nxt, offsets_h=offsets([1]))
        cases.append((g, out, nxt, want, s, a))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(30):
        for st, (g, *_rest) in zip(streams, cases):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for g, out, nxt, want, s, a in cases:
        assert torch.equal(out, want[0]) and torch.equal(nxt, want[1])
        s.check_device()


def test_calls_on_a_stream_of_their_own(select):
    rng = np.random.default_rng(3)
    s, c, w, table, q, _ = setup(select, rng, lens=(3000, 37, 90))
    cache = to_cache(select, c, w)
    a = (i32(table), i32([3000, 37, 90]))
    off_h = offsets([1, 1, 1])
    want = s.cache_attend(cache, *a, q, i32(off_h), 3000)
    off = i32(off_h)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [s.cache_attend(cache, *a, q, off, 3000, offsets_h=off_h, stream=st) for _ in range(20)]
    raw = [s.cache_attend(cache, *a, q, off, 3000, offsets_h=off_h, stream=st.cuda_stream) for _ in range(3)]
    with torch.cuda.stream(st):
        here = s.cache_attend(cache, *a, q, off, 3000, offsets_h=off_h)
    st.synchronize()
    assert all(torch.equal(o, want) for o in outs + raw + [here])
    new = s.cache_append(cache, *a, torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda"),
                         torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda"), off, offsets_h=off_h, stream=st)
    kept, lens = s.cache_evict(cache, a[0], new, 3001, 30, 2, 3, stream=st)
    st.synchronize()
    assert new.tolist() == [3001, 38, 91] and lens.tolist() == [30, 30, 30]
    s.check_device()
    s.close()


def test_a_pool_of_more_than_4_gib(select):
    """Rows beyond 2^32 bytes of a tensor: appended, read, moved."""
    hkv, d, page = 32, 128, 256
    pages = 8300  # codes: 8300 * 32 * 256 * 64 bytes = 4.05 GiB each of K and V
    s = select.Selector(1, 8, 8, hkv, hkv, d, "bf16")
    shape = (pages, hkv, page)
    t = [torch.empty((*shape, d // n), dtype=torch.uint8, device="cuda") for n in (2, 16, 2, 16)]
    cache = select.KVCache(*t, weights=torch.zeros((pages, page), device="cuda"))
    assert t[0].numel() > 1 << 32
    last, low = pages - 1, 3
    rng = np.random.default_rng(4)
    n = 300
    k = torch.from_numpy(rng.standard_normal((n, hkv, d))).to(torch.bfloat16).cuda()
    v = torch.from_numpy(rng.standard_normal((n, hkv, d))).to(torch.bfloat16).cuda()
    table = i32([[last, last - 1]])
    lens, ks, vs = s.cache_append(cache, table, i32([0]), k, v, i32([0, n]), stored=True)
    q = torch.from_numpy(rng.standard_normal((1, hkv, d))).to(torch.bfloat16).cuda()
    out = s.cache_attend(cache, table, lens, q, i32([0, 1]), n, accumulate=True)
    p = torch.softmax(torch.einsum("hd,nhd->hn", q[0].double(), ks.double()) / d ** 0.5, -1)
    want = torch.einsum("hn,nhd->hd", p, vs.double())
    # the rounding of the output, of the probabilities and of the scores, as in cache_ref
    slack = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -14) * torch.einsum("hn,nhd->hd", p, vs.double().abs()) + 1e-6
    assert ((out[0].double() - want).abs() <= slack).all()
    w = cache.weights[[last, last - 1]].flatten()[:n].double()
    assert ((w - p.mean(0)).abs() <= 1e-4 * p.mean(0) + 1e-9).all()
    kept, _ = s.cache_evict(cache, table, lens, n, 100, 4, 10, to_table=i32([[low]]))
    assert kept[0].tolist() == ref.evict(w.float().cpu().numpy(), n, 100, 4, 10).tolist()
    j = kept[0].long()
    src = torch.tensor([last, last - 1], device="cuda")[j // page], j % page
    for x in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        assert torch.equal(x[low, :, :100].transpose(0, 1), x[src[0], :, src[1]])
    s.check_device()
    s.close()


def test_empty_calls_change_nothing(select):
    rng = np.random.default_rng(5)
    s, c, w, table, q, _ = setup(select, rng)
    cache = to_cache(select, c, w)
    before = numpy_cache(cache)
    t, lens = i32(table), i32([200, 37, 90])
    none = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    new = s.cache_append(cache, t, lens, none, none, i32([0, 0, 0, 0]))
    assert torch.equal(new, lens)
    nxt = torch.full_like(cache.weights, -1.0)
    out = s.cache_attend(cache, t, lens, q[:0], i32([0, 0, 0, 0]), 200, weights_out=nxt)
    assert out.shape[0] == 0
    for b, n in enumerate([200, 37, 90]):  # nobody attends: the weights of the tokens as they are
        pos = np.arange(n)
        at = table[b][pos // 16], pos % 16
        assert (nxt.cpu().numpy()[at] == w[at]).all()
    kept, lens2 = s.cache_evict(cache, t, lens, 200, 300)
    assert lens2.tolist() == [200, 37, 90] and kept[1].tolist() == list(range(37)) + [-1] * 263
    z = torch.empty(0, dtype=torch.int32, device="cuda")
    zt = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    assert s.cache_append(cache, zt, z, none, none, i32([0])).shape[0] == 0
    assert s.cache_attend(cache, zt, z, q[:0], i32([0]), 0).shape[0] == 0
    assert s.cache_evict(cache, zt, z, 0, 5)[1].shape[0] == 0
    acc, tok = s.verify(z, torch.empty((0, 7), device="cuda"), torch.empty(0, device="cuda"),
                        torch.empty(0, device="cuda"), i32([0]))
    assert acc.shape[0] == 0 and tok.shape[0] == 0
    s.check_device()
    after = numpy_cache(cache)
    assert all(np.array_equal(after[x], before[x]) for x in ("k_codes", "k_scales", "v_codes", "v_scales"))
    assert (cache.weights.cpu().numpy() == w).all()
    # the same source row twice
    k = torch.from_numpy(rng.standard_normal((4, 2, 128))).to(torch.bfloat16).cuda()
    _, ks, _ = s.cache_append(cache, t, lens, k, k, i32([0, 2, 2, 3]), rows=i32([3, 3, 0]), stored=True)
    assert torch.equal(ks[0], ks[1]) and not torch.equal(ks[0], ks[2])
    s.check_device()
    s.close()


def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(select):
    rng = np.random.default_rng(6)
    n = 40000  # 80 rows a key head, chunks of several tiles of keys
    s, c, w, table, q, qv = setup(select, rng, lens=(n,), counts=(20,))
    cache = to_cache(select, c, w)
    a = (cache, i32(table), i32([n]), q, i32([0, 20]), n)
    s.set_wait_budget(200000)  # about 0.1 ms
    s.set_debug_flags(select.DEBUG_STALL_ATTEND)
    s.cache_attend(*a)
    with pytest.raises(select.LitevlmError) as e:
        s.check_device()
    assert e.value.name == "TIMEOUT"
    s.set_debug_flags(0)
    s.set_wait_budget(0)
    out = s.cache_attend(*a)
    s.check_device()
    fresh = select.Selector(1, 8, 8, 8, 2, 128, "bf16")
    assert torch.equal(out, fresh.cache_attend(*a))
    s.close()


def test_refusals(select):
    rng = np.random.default_rng(7)
    s, c, w, table, q, _ = setup(select, rng)
    cache = to_cache(select, c, w)
    t, lens, off = i32(table), i32([200, 37, 90]), i32([0, 1, 2, 3])
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")

    def refused(name, call):
        with pytest.raises(select.LitevlmError) as e:
            call()
        assert e.value.name == name, str(e.value)

    bad = "INVALID_ARG"
    att = lambda **kw: s.cache_attend(**(dict(cache=cache, table=t, seq_lens=lens, q=q, offsets=off, max_len=200) | kw))  # noqa: E731
    app = lambda **kw: s.cache_append(**(dict(cache=cache, table=t, seq_lens=lens, k=k, v=k, offsets=off) | kw))  # noqa: E731
    evi = lambda **kw: s.cache_evict(**(dict(cache=cache, table=t, seq_lens=lens, max_len=200, budget=20) | kw))  # noqa: E731
    refused(bad, lambda: att(q=q.float()))
    refused(bad, lambda: att(q=q.cpu()))
    refused(bad, lambda: att(q=q[:2]))
    refused(bad, lambda: att(q=torch.zeros((3, 128, 8), dtype=torch.bfloat16, device="cuda").transpose(1, 2)))
    refused(bad, lambda: att(table=t.long()))
    refused(bad, lambda: att(table=t[:, ::2]))
    refused(bad, lambda: att(seq_lens=lens[:2]))
    refused(bad, lambda: att(max_len=-1))
    refused(bad, lambda: att(max_len=t.shape[1] * 16 + 1))
    refused(bad, lambda: att(q_scale=2.0))
    refused(bad, lambda: att(weights_out=torch.zeros(3, device="cuda")))
    refused(bad, lambda: att(out=torch.zeros((3, 8, 128), device="cuda")))
    refused(bad, lambda: att(offsets=i32([0, 2, 1, 3])))
    refused(bad, lambda: att(cache=None))
    refused("WORKSPACE", lambda: att(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")))
    refused(bad, lambda: att(workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda")[1:]))
    refused(bad, lambda: app(new_lens=lens))
    refused(bad, lambda: app(k_in_scale=0.5))
    refused(bad, lambda: app(v=k[:2]))
    refused(bad, lambda: app(k=k[:2], v=k[:2]))
    refused(bad, lambda: app(rows=i32([0, 1])))
    refused(bad, lambda: app(k=torch.zeros((3, 2, 129), dtype=torch.bfloat16, device="cuda")[:, :, 1:],
                             v=k))
    refused(bad, lambda: evi(budget=0))
    refused(bad, lambda: evi(sink=11, recent=10))
    refused(bad, lambda: evi(sink=-1))
    refused(bad, lambda: evi(max_len=100000))
    refused(bad, lambda: evi(new_lens=lens))
    refused(bad, lambda: evi(to_table=t[:, :1].contiguous()))
    refused(bad, lambda: evi(cache=to_cache(select, c)))
    wrong = select.Selector(2, 8, 8, 8, 2, 128, "bf16")
    refused("WORKSPACE", lambda: wrong.cache_attend(cache, t, lens, q, off, 200))
    other = select.Selector(3, 8, 8, 8, 4, 128, "bf16")
    refused(bad, lambda: other.cache_attend(cache, t, lens, q, off, 200))
    e4m3 = select.Selector(3, 8, 8, 8, 2, 128, "e4m3")
    refused(bad, lambda: e4m3.cache_attend(cache, t, lens, q, off, 200))
    for size in (8, 24, 512):
        z = torch.zeros((2, 2, size, 64), dtype=torch.uint8, device="cuda")
        f = torch.zeros((2, 2, size, 8), dtype=torch.uint8, device="cuda")
        odd = select.KVCache(z, f, z, f)
        refused(bad, lambda: s.cache_append(odd, t, lens, k, k, off))
    for scale in (0.0, -1.0, float("nan"), 2.0 ** 70):
        refused(bad, lambda: app(cache=select.KVCache(cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales,
                                                      scale, 1.0)))
    p, x, u = torch.full((6, 5), 0.2, device="cuda"), i32([1, 2, 3]), torch.zeros(3, device="cuda")
    refused(bad, lambda: s.verify(x, p.half(), u, u, off))
    refused(bad, lambda: s.verify(x, p[:5], u, u, off))
    refused(bad, lambda: s.verify(x.long(), p, u, u, off))
    refused(bad, lambda: s.verify(x, p, u, u, off, draft_probs=p[:3].to(torch.bfloat16)))
    refused(bad, lambda: s.verify(x, p, u[:2], u, off))
    refused(bad, lambda: s.verify(x, p, u, u, off, tokens=x))
    # nothing of all this was enqueued, and the handle still works
    s.check_device()
    att()
    s.check_device()


def test_tensors_of_another_device_than_the_handle_s_are_refused(select):
    rng = np.random.default_rng(8)
    s, c, w, table, q, _ = setup(select, rng)
    cache, t, lens, off = to_cache(select, c, w), i32(table), i32([200, 37, 90]), i32([0, 1, 2, 3])
    k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    p, x, u = torch.full((6, 5), 0.2, device="cuda"), i32([1, 2, 3]), torch.zeros(3, device="cuda")
    assert s.device == torch.cuda.current_device() and s.cache(2, 16).device == s.device
    s.device += 1  # (as if the handle had been made there: the check is the host's)
    for call in (lambda: s.cache_append(cache, t, lens, k, k, off), lambda: s.cache_attend(cache, t, lens, q, off, 200),
                 lambda: s.cache_evict(cache, t, lens, 200, 20), lambda: s.verify(x, p, u, u, off)):
        with pytest.raises(select.LitevlmError) as e:
            call()
        assert e.value.name == "INVALID_ARG", str(e.value)
    s.close()


def test_a_workspace_beyond_every_size_is_refused(select):
    s = select.Selector(65535, 8, 8, 65535, 65535, 128, "bf16")
    off = np.arange(65536, dtype=np.int32)
    with pytest.raises(select.LitevlmError) as e:
        select.cache_attend_workspace(s.handle, 65535, off, 1 << 30)
    assert e.value.name == "UNSUPPORTED", str(e.value)
    s.close()


def test_a_budget_whose_places_pass_32_bits_is_refused(select):
    rng = np.random.default_rng(9)
    s, c, w, table, _, _ = setup(select, rng)
    cache, t, lens, kept, new = to_cache(select, c, w), i32(table), i32([200, 37, 90]), i32([0] * 3), i32([0] * 3)
    for budget in ((1 << 30) + 1, 2 ** 31 - 1):  # (refused by the host: kept_idx is far too small for a launch)
        with pytest.raises(select.LitevlmError) as e:
            select.cache_evict(s.handle, 3, cache.struct, t, t.shape[1], lens, 200, budget, 0, 0, None, 0, cache.weights,
                               kept, new, torch.cuda.current_stream().cuda_stream)
        assert e.value.name == "INVALID_ARG", str(e.value)
    s.check_device()
    s.close()
