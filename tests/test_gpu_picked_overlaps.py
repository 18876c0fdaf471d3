"""What the calls around a cache's pages write overlaps none of their other arrays: refused before anything is launched."""
import numpy as np
import pytest

from test_gpu_cache import i32
from test_gpu_picked_calls import Setup

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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
