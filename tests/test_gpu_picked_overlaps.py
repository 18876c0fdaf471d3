"""What the calls around a cache's pages write overlaps none of their other arrays: refused before anything is launched."""
import numpy as np
import pytest

from test_gpu_cache import i32
from test_gpu_picked_calls import Setup

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BASE = 1 << 22


@pytest.fixture(scope="module")
def select():
    if not torch.cuda.is_available():
        pytest.fail("the GPU tests need a CUDA device")
    from paper_2506_07416_gb300 import select
    return select


def refused(select, call):
    with pytest.raises(select.LitevlmError) as e:
        call()
    assert e.value.name == "INVALID_ARG" and "overlap" in str(e.value), str(e.value)


def test_bounds(select):
    a = Setup(select, 1, (1, 1, 1))
    s, c, b = a.s, a.cache, a.bounds
    n, m = b.codes.numel(), b.exps.numel()

    def call(codes=None, exps=None, cache=c, table=a.t, lens=a.lens, off=a.off):
        kb = select.KeyBounds(b.codes if codes is None else codes, b.exps if exps is None else exps, 16)
        return s.cache_bounds(cache, kb, table, lens, off, offsets_h=a.off_h)

    for t in (c.k_codes, c.v_codes, c.k_scales, c.v_scales):
        flat = t.view(torch.int8).flatten()
        refused(select, lambda: call(exps=flat[-m:].view(b.exps.shape)))
        if flat.numel() >= n:
            refused(select, lambda: call(codes=flat[:n].view(b.codes.shape)))
    buf = torch.zeros(n + (1 << 16), dtype=torch.int8, device="cuda")
    into = buf[1 << 12:(1 << 12) + n].view(b.codes.shape)
    i = into.view(-1)[:n // 4 * 4].view(torch.int32)
    for kw in (dict(table=i[:a.t.numel()].view(a.t.shape)), dict(lens=i[5:8]), dict(off=i[9:13])):
        list(kw.values())[0].copy_({"table": a.t, "lens": a.lens, "off": a.off}[next(iter(kw))])
        refused(select, lambda: call(codes=into, **kw))
    refused(select, lambda: call(codes=into, exps=into.view(-1)[:m].view(b.exps.shape)))
    # the cache's weights, whenever they were given to it
    w = torch.zeros((c.num_pages, c.page_size), dtype=torch.float32, device="cuda")
    other = select.KVCache(c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.k_scale, c.v_scale, w)
    over = w.view(torch.int8).view(-1)[:m].view(b.exps.shape)
    refused(select, lambda: call(exps=over, cache=other))
    other.weights = None
    call(exps=over, cache=other)
    other.weights = w
    refused(select, lambda: call(exps=over, cache=other))
    # side by side is no overlap
    call(codes=into, exps=buf[(1 << 12) + n:(1 << 12) + n + m].view(b.exps.shape))
    s.check_device()
    s.close()


def inside(buf, at, t):
    """A copy of t at byte `at` of buf."""
    x = buf[at:at + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
    x.copy_(t)
    return x


@pytest.mark.parametrize("counts", [(1, 1, 1), (3, 0, 2), (40, 1, 33)])
def test_pick_and_attend(select, counts):
    a = Setup(select, 2, counts)
    p = a.pick()
    o = a.attend(p)
    b, r = a.bounds, a.q.shape[0]
    pick_need = select.cache_pick_workspace(a.s.handle, 3, a.off_h, a.most, a.page, a.budget)
    need = select.cache_attend_picked_workspace(a.s.handle, 3, a.off_h, a.page, a.t.shape[1], a.budget)
    buf = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    for size, name, call in ((p.numel() * 4, "picked", a.pick), (o.numel() * 2, "out", lambda **kw: a.attend(**({"picked": p} | kw)))):
        for t, key in ((a.t, "table"), (a.lens, "seq_lens"), (a.off, "offsets"), (a.q, "q")):
            # the input at the output's first and last bytes, and just beside them
            n = t.numel() * t.element_size()
            for at, over in ((BASE, True), (BASE + (size - 16) // 16 * 16, True), (BASE + (size + 15) // 16 * 16, False),
                             (BASE - (n + 15) // 16 * 16, False)):
                x = inside(buf, at, t)
                y = buf[BASE:BASE + size].view(torch.int32 if name == "picked" else torch.bfloat16)
                kw = {key: x, name: y.view(p.shape if name == "picked" else o.shape)}
                if over:
                    refused(select, lambda: call(**kw))
                else:
                    assert torch.equal(call(**kw), p if name == "picked" else o)
    for n, call, want in ((pick_need, a.pick, p), (need, lambda **kw: a.attend(**({"picked": p} | kw)), o)):
        if not n:
            continue
        for t, key in ((a.t, "table"), (a.lens, "seq_lens"), (a.off, "offsets"), (a.q, "q"), (p, "picked")):
            at = 1 << 23
            if key == "picked" and call == a.pick:
                x = buf[at:at + p.numel() * 4].view(torch.int32).view(p.shape)
            else:
                x = inside(buf, at, t)
            refused(select, lambda: call(**{key: x}, workspace=buf[at:at + n]))
            refused(select, lambda: call(**{key: x}, workspace=buf[at - (n - 1) // 256 * 256:][:n]))
            assert torch.equal(call(**{key: x}, workspace=buf[at + (1 << 22):][:n]), want)
    # the ranges, and the cache
    over = b.codes.view(torch.uint8).view(-1)
    refused(select, lambda: a.pick(picked=over[:p.numel() * 4].view(torch.int32).view(p.shape)))
    refused(select, lambda: a.pick(bounds=select.KeyBounds(b.codes, inside(buf, BASE, b.exps), 16),
                                   picked=buf[BASE:BASE + p.numel() * 4].view(torch.int32).view(p.shape)))
    for t in (a.cache.k_codes, a.cache.v_codes, a.cache.k_scales, a.cache.v_scales):
        if t.numel() >= o.numel() * 2:
            refused(select, lambda: a.attend(p, out=t.view(-1)[:o.numel() * 2].view(torch.bfloat16).view(o.shape)))
    # rows of q with room between them: what lies there is not q's
    if r > 1:
        wide = torch.zeros((r, 2, 8, 128), dtype=torch.bfloat16, device="cuda")
        wide[:, 0] = a.q
        assert torch.equal(a.attend(p, q=wide[:, 0]), o)
        mid = wide[0, 1].view(torch.uint8).view(-1)
        if 0 < need <= mid.numel():
            assert torch.equal(a.attend(p, q=wide[:, 0], workspace=mid[:need]), o)
    a.check(p, a.attend(p))
    a.s.check_device()
    a.s.close()
