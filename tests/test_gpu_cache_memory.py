"""Whose memory the 4-bit cache's calls use, and for how long: a cache's tensors, workspaces, arrays that overlap."""
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
    assert torch.cuda.memory_allocated() == before
