"""The 4-bit cache's calls on the host: where a token lies and what is out of range (the kernels' own header, compiled
here), the argument checks that need no GPU, and the struct's layout."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2506_07416_gb300 import select

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_07416_gb300", "csrc")

PROGRAM = r'''
#include <cstdio>
#include <cstdlib>
#include "cache_index.h"
int main()
{
    // random tables with entries outside the pool: every row that the header gives lies inside it
    srand(7);
    for (int it = 0; it < 20000; ++it) {
        const int shift = 4 + rand() % 5, page = 1 << shift, width = 1 + rand() % 9, pages = 1 + rand() % 50;
        const int heads = 1 + rand() % 8;
        int32_t table[3 * 9];
        for (int& t : table) t = rand() % (pages + 40) - 20;
        bool bad;
        const int limit = width * page, given = rand() % (2 * limit + 20) - 10;
        const int len = lvs::cache_len(given, limit, bad);
        if (len < 0 || len > limit || bad != (given < 0 || given > limit) || (!bad && len != given)) return 1;
        for (int k = 0; k < 20; ++k) {
            const int64_t b = rand() % 3, pos = rand() % (limit + 3 * page);
            const int32_t p = lvs::cache_page(table, width, pages, shift, b, pos);
            const int64_t i = pos / page;
            const int32_t want = i < width && table[b * width + i] >= 0 && table[b * width + i] < pages
                                     ? table[b * width + i] : -1;
            if (p != want) return 2;
            if (p < 0) continue;
            const int h = rand() % heads;
            const int64_t row = lvs::cache_row(p, heads, h, shift, pos % page);
            if (row < 0 || row >= (int64_t)pages * heads * page) return 3;
            if (row != ((int64_t)p * heads + h) * page + pos % page) return 4;
        }
    }
    // a pool of more than 2^32 bytes
    const int64_t row = lvs::cache_row(2000000, 32, 31, 8, 255);
    if (row != (2000000LL * 32 + 31) * 256 + 255) return 5;
    puts("ok");
    return 0;
}
'''


def test_places_in_the_pool_and_out_of_range_entries(tmp_path):
    src, exe = tmp_path / "places.cpp", tmp_path / "places"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.returncode


def test_cache_struct_layout_matches_header(tmp_path):
    fields = [f for f, _ in select.Cache._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "litevlm_select.h"\nint main(void){printf("%zu'
                   + " %zu" * len(fields) + '\\n", sizeof(litevlm_cache_t)'
                   + "".join(f", offsetof(litevlm_cache_t, {f})" for f in fields) + ");return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(select.Cache)] + [getattr(select.Cache, f).offset for f in fields]


def test_calls_need_a_handle():
    L = select.LIB
    assert L.litevlm_select_cache_append(None, 1, None, None, 1, None, None, 0, None, 0, 0, None, None, None, 1.0, 1.0,
                                         None, None, None, None, None) == 1
    n = ctypes.c_int64(-7)
    assert L.litevlm_select_cache_attend_workspace(None, 1, None, 1, 1, ctypes.byref(n)) == 1 and n.value == -7
    assert L.litevlm_select_cache_attend(None, 1, None, None, 1, None, None, 0, None, None, 1, 1.0, None, None, None,
                                         None, 0, None) == 1
    assert L.litevlm_select_cache_evict(None, 1, None, None, 1, None, 1, 1, 0, 0, None, 0, None, None, None, None) == 1
    assert L.litevlm_select_verify(None, 1, 1, 0, None, None, None, None, None, None, None, None, None, None) == 1


def test_the_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    c = torch.zeros((2, 1, 16, 32), dtype=torch.uint8)
    f = torch.zeros((2, 1, 16, 4), dtype=torch.uint8)
    with pytest.raises(select.LitevlmError) as e:
        select.KVCache(c, f, c, f)
    assert e.value.name == "INVALID_ARG" and "CUDA" in str(e.value)
    with pytest.raises(select.LitevlmError):
        select._want("x", np.zeros(3, np.int32), torch.int32, (3,), 0)
    with pytest.raises(select.LitevlmError):
        select._row_stride("q", torch.zeros((2, 1, 64)), torch.bfloat16, 1, 64, 0)
