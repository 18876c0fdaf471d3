"""The 4-bit cache's sizes at their limits, by the kernels' own header compiled here: chunks of a request's keys, places of
its tiles of rows."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_07416_gb300", "csrc")

PROGRAM = r'''
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "cache_index.h"
int main()
{
    const int32_t most = 1 << 30;  // the longest request that the calls take
    // one chunk for all keys ends behind the last of them, at every length
    if (lvs::kMostKeys < most || lvs::kMostKeys % 64 != 0) return 1;
    for (int32_t seen : {most, most - 1, most - 64, 1, 0, -5})
        if (lvs::chunk_end(seen, 0, lvs::kMostKeys) != seen) return 2;
    // chunks of any length cover every key once and stay within 32 bits
    srand(3);
    for (int it = 0; it < 2000; ++it) {
        const int32_t n = it % 3 ? most - rand() % 1000 : 1 + rand() % 100000;
        const int32_t chunk = ((it % 3 ? most / (1 + rand() % 300) : 1 + rand() % 5000) + 63) & ~63;
        int64_t k0 = 0;
        for (int guard = 0; k0 < n; ++guard) {
            const int64_t end = lvs::chunk_end(n, (int32_t)k0, chunk);
            if (end <= k0 || end > n || (end < n && end != k0 + chunk) || guard > 100000) return 3;
            k0 = end;
        }
        if (k0 != n) return 4;
        if (lvs::chunk_end(n / 2, n, chunk) > n) return 5;  // behind the keys: empty
    }
    // the tiles of 128 rows of every request lie behind those of the last one, and inside those of all
    for (int it = 0; it < 2000; ++it) {
        const int batch = 1 + rand() % 40;
        int64_t rows = 0, end = 0;
        for (int b = 0; b < batch; ++b) {
            const int64_t n = rand() % 4 == 0 ? 0 : (rand() % 4 == 0 ? 128 * (rand() % 9) : rand() % 1000);
            const int64_t at = lvs::tile_at(rows, b);
            if (at < end) return 6;
            end = at + (n + 127) / 128;
            rows += n;
        }
        if (end > lvs::tile_at(rows, batch)) return 7;
    }
    puts("ok");
    return 0;
}
'''


def test_chunks_cover_every_key(tmp_path):
    src, exe = tmp_path / "chunks.cpp", tmp_path / "chunks"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-ftrapv", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stderr)


def test_no_kernel_has_a_limit_of_its_own():
    """The chunk of all keys and the longest request are the header's in every source."""
    for name in ("cache_attend.cu", "cache_attend.cuh", "cache_tile.cu", "api.cu"):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        assert "chunk = INT32_MAX" not in text and "kMostKeys" in text, name
