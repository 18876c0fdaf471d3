"""The calls around a paged cache's pages on the host: the restatement that the GPU tests compare with on worked
examples, the places of the pages that new tokens touch (the kernels' header, compiled here), the structs' layout, and
what is refused without a GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import picked_ref as pref
from paper_2506_07416_gb300 import select

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_07416_gb300", "csrc")


def test_reserve_worked_example():
    """Three requests on pages of 16: one grows into the ring's wrapped end, one finds too few, one gives back."""
    table = np.array([[7, -1, -1], [2, -1, -1], [4, 0, 6]], np.int32)
    free = np.array([5, -1, -1, -1, -1, -1, 1, 3], np.int32)  # 1, 3, 5 from place 6 on
    g, st, sl, t, f = pref.reserve(table, [16, 10, 40], [33, 40, 3], free, [6, 3], 16, [17, 30, 0])
    assert g.tolist() == [33, 10, 3] and st.tolist() == [0, 3]  # two taken, two back
    assert t.tolist() == [[7, 1, 3], [2, -1, -1], [4, 0, 6]]
    assert f.tolist() == [5, 0, 6, -1, -1, -1, 1, 3]
    assert sl.tolist() == list(range(16, 32)) + [48] + [-1] * 30
    # give everything back: the ring then holds every page once
    g, st, sl, t, f = pref.reserve(t, [33, 10, 3], [0, 0, 0], f, st, 16, [0, 0, 0])
    assert st.tolist() == [0, 8] and sorted(f.tolist()) == list(range(8))


def test_bounds_worked_example():
    k = np.zeros((2, 1, 64))
    k[0, 0, :3], k[1, 0, :3] = [3.0, -1.0, 0.5], [2.5, -4.0, 0.25]
    c, e = pref.page_bounds(k)
    assert e.tolist() == [-4]  # 4 = 1/2 * 2^3, unit 2^-4
    assert c[0, 0, :4].tolist() == [48, -16, 8, 0] and c[0, 1, :4].tolist() == [40, -64, 4, 0]
    k[0, 0, 0] = 2688.0  # 21/32 * 2^12: unit 32
    c, e = pref.page_bounds(k)
    assert e.tolist() == [5] and c[0, 0, :3].tolist() == [84, 0, 1] and c[0, 1, :3].tolist() == [0, -1, 0]


def test_ranges_bound_every_key_of_the_page():
    rng = np.random.default_rng(5)
    k = rng.standard_normal((32, 2, 64))
    k = np.round(k * 8) / 8
    c, e = pref.page_bounds(k)
    q = rng.standard_normal((3, 64))
    for h in range(2):
        top = np.abs(q).max()
        r = np.clip(np.round(q * 2.0 ** (7 - np.frexp(top)[1])), -127, 127)
        assert pref.page_scores(q, c[None, h], e[None, h])[0] >= (r @ k[:, h].T).max()


PROGRAM = r'''
#include <cstdio>
#include <cstdlib>
#include "cache_index.h"
int main()
{
    srand(11);
    for (int it = 0; it < 20000; ++it) {
        const int shift = 4 + rand() % 5, batch = 1 + rand() % 20;
        int64_t rows = it % 2 ? (int64_t)(rand() % 1000) << 20 : 0, end = lvs::page_at(rows, 0, shift);
        for (int b = 0; b < batch; ++b) {
            const int64_t t = rand() % 4 ? rand() % 5 : rand() % 3000, before = rand() % 5000, n = before + t;
            const int64_t at = lvs::page_at(rows, b, shift);
            if (at < end) return 1;
            end = at + (t > 0 ? ((n - 1) >> shift) - (before >> shift) + 1 : 0);
            rows += t;
            if (end > lvs::page_at(rows, b + 1, shift)) return 2;
        }
    }
    puts("ok");
    return 0;
}
'''


def test_places_of_the_touched_pages_do_not_overlap(tmp_path):
    src, exe = tmp_path / "touched.cpp", tmp_path / "touched"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.returncode


def test_struct_layout_matches_header(tmp_path):
    fields = [f for f, _ in select.Bounds._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "litevlm_select.h"\nint main(void){printf("%zu'
                   + " %zu" * len(fields) + '\\n", sizeof(litevlm_key_bounds_t)'
                   + "".join(f", offsetof(litevlm_key_bounds_t, {f})" for f in fields) + ");return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(select.Bounds)] + [getattr(select.Bounds, f).offset for f in fields]


def test_calls_need_a_handle():
    L = select.LIB
    N = None
    assert L.litevlm_select_cache_reserve(N, 1, 16, N, 1, N, N, N, 1, N, N, N, N, N, N, N) == 1
    assert L.litevlm_select_cache_bounds(N, 1, N, N, N, 1, N, N, N, N) == 1
    n = ctypes.c_int64(-7)
    assert L.litevlm_select_cache_pick_workspace(N, 1, N, 1, 16, 1, ctypes.byref(n)) == 1
    assert L.litevlm_select_cache_pick(N, 1, N, N, 1, N, N, 0, N, N, 1, 1, 0, 0, N, N, 0, N) == 1
    assert L.litevlm_select_cache_attend_picked_workspace(N, 1, N, 16, 1, 1, ctypes.byref(n)) == 1 and n.value == -7
    assert L.litevlm_select_cache_attend_picked(N, 1, N, N, 1, N, N, 0, N, N, N, 1, 1.0, N, N, 0, N) == 1


def test_the_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(select.LitevlmError) as e:
        select.KeyBounds(torch.zeros((2, 1, 2, 64), dtype=torch.int8), torch.zeros((2, 1), dtype=torch.int8), 16)
    assert e.value.name == "INVALID_ARG" and "CUDA" in str(e.value)
