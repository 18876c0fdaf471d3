"""How the calls around a paged cache's pages are made: captured and replayed, on streams of their own, two at once, on
pools of more than 4 GiB, empty, wrong, and giving up."""
import numpy as np
import pytest

import picked_ref as pref
from test_gpu_cache import i32, make_q, offsets, random_pool, tables, to_cache

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


class Setup:
    """A cache with its ranges and queries, and the three calls that read them."""

    def __init__(self, select, seed, counts, hq=8, hkv=2, d=128, page=16, lens=(900, 437, 650), budget=6):
        rng = np.random.default_rng(seed)
        self.table, self.pool = tables(rng, lens, page)
        self.c = random_pool(rng, self.pool, hkv, page, d)
        self.cache = to_cache(select, self.c)
        self.s = select.Selector(len(lens), 8, 8, hq, hkv, d, "bf16")
        self.bounds = self.s.key_bounds(self.cache)
        self.t, self.lens, self.n = i32(self.table), i32(lens), list(lens)
        self.off_h = offsets(counts)
        self.off, self.most, self.budget, self.page, self.hkv = i32(self.off_h), max(lens), budget, page, hkv
        self.q, self.qv, _ = make_q(rng, int(self.off_h[-1]), hq, d, "bf16")
        every = offsets(lens)
        self.s.cache_bounds(self.cache, self.bounds, self.t, self.lens, i32(every), offsets_h=every)

    def pick(self, **kw):
        a = dict(bounds=self.bounds, table=self.t, seq_lens=self.lens, q=self.q, offsets=self.off, max_len=self.most,
                 budget=self.budget, sink=1, recent=2, offsets_h=self.off_h) | kw
        return self.s.cache_pick(**a)

    def attend(self, picked=None, **kw):
        a = dict(cache=self.cache, table=self.t, seq_lens=self.lens, q=self.q, offsets=self.off,
                 picked=self.picked if picked is None else picked, offsets_h=self.off_h) | kw
        return self.s.cache_attend_picked(**a)

    def want(self):
        wc, we = pref.bounds(self.c, self.table, self.n, self.n, np.zeros(self.bounds.codes.shape, np.int8),
                             np.zeros(self.bounds.exps.shape, np.int8))
        picked = pref.pick(self.qv, self.off_h, self.n, self.table, wc, we, self.page, self.budget, 1, 2, self.hkv)
        return picked, *pref.attend(self.c, self.table, self.n, self.qv, self.off_h, picked)

    def check(self, picked, out):
        want_p, want_o, slack = self.want()
        np.testing.assert_array_equal(picked.cpu().numpy(), want_p)
        assert (np.abs(out.double().cpu().numpy() - want_o) <= slack).all()


COUNTS = [(1, 1, 1), (3, 0, 2), (40, 1, 33)]  # a tile for each query; of 16 rows; of 128 and more


def test_a_captured_step_is_replayed_as_lengths_change(select):
    """Reserve, append, ranges, selection and attention of a decoding step in one graph."""
    rng = np.random.default_rng(1)
    hq, hkv, d, page, pool, width, batch = 8, 2, 64, 16, 90, 24, 3
    s = select.Selector(batch, 8, 8, hq, hkv, d, "bf16")
    off_h = offsets([1] * batch)
    off = i32(off_h)
    lens0 = [200, 31, 90]
    table0, _ = tables(rng, lens0, page)
    c = random_pool(rng, pool, hkv, page, d)
    k = torch.from_numpy(rng.standard_normal((2, batch, hkv, d))).to(torch.bfloat16).cuda()
    q, _, _ = make_q(rng, batch, hq, d, "bf16")
    spare = rng.permutation(np.arange(int(table0.max()) + 1, pool)).astype(np.int32)

    class World:
        def __init__(self):
            self.cache = to_cache(select, c)
            self.bounds = s.key_bounds(self.cache)
            full = np.full((batch, width), -1, np.int32)
            full[:, :table0.shape[1]] = table0
            ring = np.full(pool, -1, np.int32)
            ring[(pool - 2 + np.arange(len(spare))) % pool] = spare
            self.table, self.free, self.state = i32(full), i32(ring), i32([pool - 2, len(spare)])
            self.lens = i32(lens0)
            every = offsets(lens0)
            s.cache_bounds(self.cache, self.bounds, self.table, self.lens, i32(every), offsets_h=every)

        def step(self):
            granted, state, slots = s.cache_reserve(self.table, self.lens, self.lens + 1, self.free, self.state, page, off,
                                                    offsets_h=off_h)
            new = s.cache_append(self.cache, self.table, self.lens, k[0], k[1], off, offsets_h=off_h)
            s.cache_bounds(self.cache, self.bounds, self.table, new, off, offsets_h=off_h)
            picked = s.cache_pick(self.bounds, self.table, new, q, off, width * page, 5, 1, 1, offsets_h=off_h)
            out = s.cache_attend_picked(self.cache, self.table, new, q, off, picked, offsets_h=off_h)
            self.lens.copy_(new)
            self.state.copy_(state)
            return granted, slots, picked, out

    World().step()  # (kernels loaded, workspace of the eager calls made)
    one, two = World(), World()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = one.step()
    for n in range(40):
        g.replay()
        for a, b in zip(got, two.step()):
            assert torch.equal(a, b), n
    for a, b in ((one.table, two.table), (one.free, two.free), (one.state, two.state), (one.lens, two.lens),
                 (one.bounds.codes, two.bounds.codes)):
        assert torch.equal(a, b)
    assert one.lens.tolist() == [n + 40 for n in lens0] and one.state.tolist()[1] < len(spare)
    s.check_device()
    s.close()


@pytest.mark.parametrize("counts", COUNTS)
def test_two_graphs_at_once_use_workspaces_of_their_own(select, counts):
    a, b = Setup(select, 2, counts), Setup(select, 3, counts)
    b.s = a.s  # (one handle)
    want = []
    for x in (a, b):
        p = x.pick()
        x.picked = p
        want.append((p, x.attend()))
        x.check(*want[-1])
    graphs = []
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p = x.pick()
            graphs.append((g, p, x.attend(p)))
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(20):
        for (g, _, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for (_, p, o), (wp, wo) in zip(graphs, want):
        assert torch.equal(p, wp) and torch.equal(o, wo)
    a.s.check_device()


@pytest.mark.parametrize("counts", COUNTS)
def test_calls_on_streams_of_their_own(select, counts):
    a, b = Setup(select, 4, counts), Setup(select, 5, counts)
    b.s = a.s
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got = []
        for x, st in zip((a, b), streams):
            p = x.pick(stream=st)
            got.append((p, x.attend(p, stream=st)))
    torch.cuda.synchronize()
    for x, g in zip((a, b), got):
        x.check(*g)
    # ... and on the current one, after another
    with torch.cuda.stream(streams[1]):
        p = a.pick()
        o = a.attend(p)
    torch.cuda.synchronize()
    a.check(p, o)
    a.s.check_device()


@pytest.mark.parametrize("counts", COUNTS)
def test_the_same_inputs_give_the_same_bits(select, counts):
    a = Setup(select, 6, counts)
    p = a.pick()
    o = a.attend(p)
    for _ in range(5):
        assert torch.equal(a.pick(), p) and torch.equal(a.attend(p), o)
    a.check(p, o)


@pytest.mark.parametrize("counts", COUNTS)
def test_nothing_else_is_written(select, counts):
    """Outputs inside larger buffers, a workspace of exactly its bytes: what lies around stays as it was."""
    a = Setup(select, 7, counts)
    r, h, b = a.q.shape[0], a.hkv, a.budget
    pbuf = torch.full((r + 2, h, b), -9, dtype=torch.int32, device="cuda")
    obuf = torch.full((r + 2, 8, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    for need, call in ((select.cache_pick_workspace(a.s.handle, 3, a.off_h, a.most, a.page, b),
                        lambda w: a.pick(picked=pbuf[1:-1], workspace=w)),
                       (select.cache_attend_picked_workspace(a.s.handle, 3, a.off_h, a.page, a.t.shape[1], b),
                        lambda w: a.attend(pbuf[1:-1], out=obuf[1:-1], workspace=w))):
        ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        call(ws[256:256 + need])
        torch.cuda.synchronize()
        assert (ws[:256] == 0xA5).all() and (ws[256 + need:] == 0xA5).all()
    for buf, v in ((pbuf, -9), (obuf, 9.0)):
        assert (buf[0] == v).all() and (buf[-1] == v).all()
    a.check(pbuf[1:-1], obuf[1:-1])
    a.s.check_device()


def test_pools_of_more_than_4_gib(select):
    """Pages whose codes lie behind 2^32 bytes, and ranges too."""
    rng = np.random.default_rng(8)
    hq, hkv, d, page = 16, 8, 128, 16
    pages = 2300000  # 4.7 GB of ranges; 18.8 GB of codes each
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    lens = [300, 150]
    table = np.full((2, 19), -1, np.int32)
    table[0] = rng.permutation(np.arange(pages - 19, pages))
    table[1, :10] = rng.permutation(np.arange(2 ** 21 + 1, 2 ** 21 + 11))
    small = random_pool(rng, 29, hkv, page, d)
    at = np.concatenate([table[0], table[1, :10]])
    big = {}
    for n, v in small.items():
        if n.endswith("_scale"):
            big[n] = v
            continue
        big[n] = torch.empty((pages, *v.shape[1:]), dtype=torch.uint8, device="cuda")
        big[n][torch.from_numpy(at).long().cuda()] = torch.from_numpy(v).cuda()
    cache = select.KVCache(big["k_codes"], big["k_scales"], big["v_codes"], big["v_scales"], big["k_scale"], big["v_scale"])
    s = select.Selector(2, 8, 8, hq, hkv, d, "bf16")
    bounds = select.KeyBounds(torch.empty((pages, hkv, 2, d), dtype=torch.int8, device="cuda"),
                              torch.empty((pages, hkv), dtype=torch.int8, device="cuda"), page)
    local = np.full((2, 19), -1, np.int32)  # the same pages in the small pool
    local[0], local[1, :10] = np.arange(19), np.arange(19, 29)
    every = offsets(lens)
    s.cache_bounds(cache, bounds, i32(table), i32(lens), i32(every), offsets_h=every)
    z = np.zeros((29, hkv, 2, d), np.int8), np.zeros((29, hkv), np.int8)
    wc, we = pref.bounds(small, local, lens, lens, *z)
    idx = torch.from_numpy(at).long().cuda()
    np.testing.assert_array_equal(bounds.codes[idx].cpu().numpy(), wc)
    np.testing.assert_array_equal(bounds.exps[idx].cpu().numpy(), we)
    for counts in ((1, 1), (2, 3), (40, 33)):
        off = offsets(counts)
        q, qv, _ = make_q(rng, int(off[-1]), hq, d, "bf16")
        p = s.cache_pick(bounds, i32(table), i32(lens), q, i32(off), 300, 4, 1, 1, offsets_h=off)
        want_p = pref.pick(qv, off, lens, local, wc, we, page, 4, 1, 1, hkv)
        np.testing.assert_array_equal(p.cpu().numpy(), want_p)
        o = s.cache_attend_picked(cache, i32(table), i32(lens), q, i32(off), p, offsets_h=off)
        want_o, slack = pref.attend(small, local, lens, qv, off, want_p)
        assert (np.abs(o.double().cpu().numpy() - want_o) <= slack).all()
    s.check_device()
    s.close()


def test_empty_calls(select):
    a = Setup(select, 9, (1, 1, 1))
    none = np.zeros(4, np.int32)
    q = a.q[:0]
    p = a.pick(q=q, offsets=i32(none), offsets_h=none)
    assert p.shape == (0, 2, 6)
    assert a.attend(p, q=q, offsets=i32(none), offsets_h=none).shape == (0, 8, 128)
    before = a.bounds.codes.clone()
    a.s.cache_bounds(a.cache, a.bounds, a.t, a.lens, i32(none), offsets_h=none)
    assert torch.equal(before, a.bounds.codes)
    t = a.t[:0]
    zero = i32([0])
    g, st, sl = a.s.cache_reserve(t, i32([]), i32([]), i32([3, 4, 5]), i32([1, 2]), 16, zero)
    assert g.shape == (0,) and st.tolist() == [1, 2] and sl.shape == (0,)
    p = a.s.cache_pick(a.bounds, t, i32([]), q, zero, 10, 4)
    assert a.s.cache_attend_picked(a.cache, t, i32([]), q, zero, p).shape == (0, 8, 128)
    a.s.cache_bounds(a.cache, a.bounds, t, i32([]), zero)
    # requests of no tokens
    a.lens.zero_()
    p = a.pick()
    assert (p == -1).all() and (a.attend(p) == 0).all()
    a.s.check_device()


def test_a_wait_that_runs_out_is_reported_and_the_handle_recovers(select):
    a = Setup(select, 10, (40, 33, 20), lens=(9000, 3000, 100))
    p = a.pick()
    o = a.attend(p)
    for flag, call, want in ((select.DEBUG_STALL_PICK, a.pick, p), (select.DEBUG_STALL_ATTEND, lambda: a.attend(p), o)):
        a.s.set_wait_budget(200000)  # about 0.1 ms
        a.s.set_debug_flags(flag)
        call()
        with pytest.raises(select.LitevlmError) as e:
            a.s.check_device()
        assert e.value.name == "TIMEOUT"
        a.s.set_debug_flags(0)
        a.s.set_wait_budget(0)
        assert torch.equal(call(), want)
        a.s.check_device()
    # scores that were never made, whatever memory holds in their place, do not lead out of the lists
    need = select.cache_pick_workspace(a.s.handle, 3, a.off_h, a.most, a.page, a.budget)
    for byte in (0x00, 0x01, 0x7F, 0xFF):
        ws = torch.full((need,), byte, dtype=torch.uint8, device="cuda")
        buf = torch.full((p.shape[0] + 2, *p.shape[1:]), -9, dtype=torch.int32, device="cuda")
        a.s.set_wait_budget(200000)
        a.s.set_debug_flags(select.DEBUG_STALL_PICK)
        a.pick(picked=buf[1:-1], workspace=ws)
        with pytest.raises(select.LitevlmError):
            a.s.check_device()
        assert (buf[0] == -9).all() and (buf[-1] == -9).all()
        a.s.set_debug_flags(0)
        a.s.set_wait_budget(0)
    assert torch.equal(a.pick(), p)


def test_lengths_beyond_the_table_are_cut_and_reported(select):
    a = Setup(select, 11, (2, 1, 1))
    p = a.pick()
    a.lens.copy_(i32([900, 437, 10 ** 9]))
    for call in (lambda: a.pick(), lambda: a.attend(p)):
        call()
        with pytest.raises(select.LitevlmError) as e:
            a.s.check_device()
        assert e.value.name == "DEVICE_BOUNDS"


def test_refusals(select):
    a = Setup(select, 12, (1, 1, 1))
    s = a.s
    p = a.pick()

    def refused(name, call):
        with pytest.raises(select.LitevlmError) as e:
            call()
        assert e.value.name == name, str(e.value)

    bad = "INVALID_ARG"
    byte = dict(dtype=torch.uint8, device="cuda")
    refused(bad, lambda: a.pick(q=a.q.float()))
    refused(bad, lambda: a.pick(q=a.q.cpu()))
    refused(bad, lambda: a.pick(q=a.q[:2]))
    refused(bad, lambda: a.pick(q=torch.zeros((3, 128, 8), dtype=torch.bfloat16, device="cuda").transpose(1, 2)))
    refused(bad, lambda: a.pick(table=a.t.long()))
    refused(bad, lambda: a.pick(table=a.t[:, ::2]))
    refused(bad, lambda: a.pick(seq_lens=a.lens[:2]))
    refused(bad, lambda: a.pick(bounds=a.cache))
    refused(bad, lambda: a.pick(bounds=None))
    refused(bad, lambda: a.pick(max_len=-1))
    refused(bad, lambda: a.pick(max_len=a.t.shape[1] * 16 + 1))
    refused(bad, lambda: a.pick(max_len=(1 << 30) + 1))
    refused(bad, lambda: a.pick(budget=0))
    refused(bad, lambda: a.pick(budget=(1 << 26) + 1))
    refused(bad, lambda: a.pick(budget=3, sink=2, recent=2))
    refused(bad, lambda: a.pick(sink=-1))
    refused(bad, lambda: a.pick(recent=-1))
    refused(bad, lambda: a.pick(picked=p[:2]))
    refused(bad, lambda: a.pick(offsets_h=np.array([0, 2, 1, 3], np.int32)))
    refused("WORKSPACE", lambda: a.pick(workspace=torch.empty(256, **byte)))
    refused(bad, lambda: a.pick(workspace=torch.empty(1 << 24, **byte)[1:]))
    refused(bad, lambda: a.attend(p, q=a.q[:2]))
    refused(bad, lambda: a.attend(p.long()))
    refused(bad, lambda: a.attend(p[:, :1]))
    refused(bad, lambda: a.attend(p[:, :, :0].contiguous()))
    refused(bad, lambda: a.attend(p[:, :, ::2]))
    refused(bad, lambda: a.attend(p, q_scale=2.0))
    refused(bad, lambda: a.attend(p, cache=a.bounds))
    refused(bad, lambda: a.attend(p, out=torch.zeros((3, 8, 128), device="cuda")))
    refused(bad, lambda: a.attend(p, out=a.q))
    refused(bad, lambda: a.attend(p, offsets_h=np.array([0, 2, 1, 3], np.int32)))
    two = Setup(select, 13, (2, 1, 1))
    p2 = two.pick()
    refused("WORKSPACE", lambda: two.attend(p2, workspace=torch.empty(256, **byte)))
    refused(bad, lambda: two.attend(p2, workspace=torch.empty(1 << 24, **byte)[1:]))
    ws = torch.empty(1 << 24, **byte)  # too short, whatever lies behind it
    refused("WORKSPACE", lambda: two.attend(p2, workspace=ws[:256],
                                            out=ws[256:256 + 4 * 8 * 128 * 2].view(torch.bfloat16).view(4, 8, 128)))
    refused(bad, lambda: two.attend(p2, workspace=ws, out=ws[:4 * 8 * 128 * 2].view(torch.bfloat16).view(4, 8, 128)))
    # ranges
    every, evd = a.off_h, a.off
    small = select.KeyBounds(a.bounds.codes[:3].contiguous(), a.bounds.exps[:3].contiguous(), 16)
    refused(bad, lambda: s.cache_bounds(a.cache, small, a.t, a.lens, evd, offsets_h=every))
    refused(bad, lambda: s.cache_bounds(a.cache, select.KeyBounds(a.bounds.codes, a.bounds.exps, 32), a.t, a.lens, evd))
    refused(bad, lambda: s.cache_bounds(a.bounds, a.bounds, a.t, a.lens, evd))
    refused(bad, lambda: s.cache_bounds(a.cache, a.bounds, a.t, a.lens, evd[:3]))
    over = a.cache.k_codes.view(torch.int8).flatten()[:a.bounds.codes.numel()].view(a.bounds.codes.shape)
    refused(bad, lambda: s.cache_bounds(a.cache, select.KeyBounds(over, a.bounds.exps, 16), a.t, a.lens, evd))
    refused(bad, lambda: select.KeyBounds(a.bounds.codes.view(torch.uint8), a.bounds.exps, 16))
    refused(bad, lambda: select.KeyBounds(a.bounds.codes, a.bounds.exps[:2], 16))
    with pytest.raises(select.LitevlmError):
        a.bounds.codes = a.bounds.codes.clone()
    refused(bad, lambda: a.pick(bounds=select.KeyBounds(a.bounds.codes, a.bounds.exps, 24)))
    # pages
    t, n, f, st, off = a.t.clone(), i32([16, 16, 16]), i32(np.arange(9)), i32([0, 9]), i32([0, 0, 0, 0])
    res = lambda **kw: s.cache_reserve(**(dict(table=t, held=n, want=n.clone(), free=f, state=st, page_size=16, offsets=off) | kw))  # noqa: E731
    refused(bad, lambda: res(table=t.long()))
    refused(bad, lambda: res(table=t[:, ::2]))
    refused(bad, lambda: res(held=n[:2]))
    refused(bad, lambda: res(state=i32([0])))
    refused(bad, lambda: res(free=f.long()))
    refused(bad, lambda: res(free=f[:0]))
    refused(bad, lambda: res(page_size=24))
    refused(bad, lambda: res(granted=n))
    refused(bad, lambda: res(new_state=st))
    refused(bad, lambda: res(state=f[:2]))
    refused(bad, lambda: res(slots=torch.zeros(1, dtype=torch.int64, device="cuda")))
    refused(bad, lambda: res(offsets_h=np.array([0, 2, 1, 3], np.int32)))
    # handles
    wrong = select.Selector(2, 8, 8, 8, 2, 128, "bf16")
    refused("WORKSPACE", lambda: wrong.cache_pick(a.bounds, a.t, a.lens, a.q, a.off, a.most, 4))
    refused("WORKSPACE", lambda: wrong.cache_attend_picked(a.cache, a.t, a.lens, a.q, a.off, p))
    other = select.Selector(3, 8, 8, 8, 4, 128, "bf16")
    refused(bad, lambda: other.cache_pick(a.bounds, a.t, a.lens, a.q, a.off, a.most, 4))
    refused(bad, lambda: other.cache_attend_picked(a.cache, a.t, a.lens, a.q, a.off, p))
    e4m3 = select.Selector(3, 8, 8, 8, 2, 128, "e4m3")
    refused(bad, lambda: e4m3.cache_pick(a.bounds, a.t, a.lens, a.q, a.off, a.most, 4))
    many = select.Selector(1, 8, 8, 129, 1, 64, "bf16")
    one = np.array([0, 1], np.int32)
    refused("UNSUPPORTED", lambda: select.cache_pick_workspace(many.handle, 1, one, 1000, 16, 4))
    long = np.array([0, 2 ** 31 - 1], np.int32)
    refused("UNSUPPORTED", lambda: select.cache_pick_workspace(a.s.handle, 1, long, 1000, 16, 4))
    refused("UNSUPPORTED", lambda: select.cache_attend_picked_workspace(a.s.handle, 1, long, 16, 1000, 4))
    # nothing of all this was enqueued, and the handle still works
    s.check_device()
    a.check(a.pick(), a.attend(p))
    s.check_device()


def test_tensors_of_another_device_than_the_handle_s_are_refused(select):
    a = Setup(select, 14, (1, 1, 1))
    p = a.pick()
    a.s.device += 1  # (as if the handle had been made there: the check is the host's)
    off = i32([0, 0, 0, 0])
    for call in (lambda: a.pick(), lambda: a.attend(p),
                 lambda: a.s.cache_bounds(a.cache, a.bounds, a.t, a.lens, off),
                 lambda: a.s.cache_reserve(a.t, a.lens, a.lens, i32([1]), i32([0, 1]), 16, off)):
        with pytest.raises(select.LitevlmError) as e:
            call()
        assert e.value.name == "INVALID_ARG", str(e.value)
