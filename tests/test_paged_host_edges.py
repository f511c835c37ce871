"""Refusals of the paged-cache calls at the edges of their arguments, without a GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2510_00636_b200 import build

from test_paged_host import INVALID, P, _vary, ctx, ea, shape          # noqa: F401 (fixtures)


def test_rows_that_overlap_what_is_written_are_refused(ea, ctx):       # noqa: F811
    """16 KiB of a pool at 1 MiB and at 2 MiB, four rows of 256 bytes, four slots."""
    L, ref = ea.lib(), ctypes.byref(shape(ea, n_pages=4))
    M, rows = 1 << 20, 4 * 256
    good = [P, 4, 4 * M, 5 * M, 0, 0, M, 2 * M]                        # slots, rows, k, v, k_stride, v_stride, k_pages, v_pages
    for change in ({2: M}, {2: M - rows + 16}, {2: M + 16384 - 16}, {3: 2 * M + 512}, {3: M}, {6: 2 * M}, {6: 2 * M + 16368}, {0: M + 64},
                   {2: M - 1024, 4: 512}):                             # two tokens 512 elements apart end 512 bytes into the pool
        assert L.ea_page_store(ctx, ref, *_vary(good, change), None) == INVALID, change
    good = [P, 4, M, 2 * M, 4 * M, 5 * M]                              # slots, rows, k_pages, v_pages, k, v
    for change in ({4: M}, {5: 2 * M + 16368}, {4: 5 * M}, {4: 5 * M + 512}, {5: P}):
        assert L.ea_page_load(ctx, ref, *_vary(good, change), None) == INVALID, change


def _host_program(tmp_path, source):
    """A program that includes the library's device headers, for the CPU."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(source)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    return exe


def test_division_by_any_head_count(tmp_path):
    """quotient(n, fast_div(d)) is n / d for every 0 <= n < 2^31 and 1 <= d < 2^31: around the multiples, and at random."""
    exe = _host_program(tmp_path, """
        #define __device__
        #define __forceinline__ inline
        #include <stdint.h>
        static inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)(((uint64_t)a * b) >> 32); }
        #include "fast_div.cuh"
        #include <stdio.h>
        static uint64_t s = 1;
        static uint32_t rnd() { s = s * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(s >> 33); }
        int main() {
            const uint32_t top = 0x7fffffffu;
            for (int i = 0; i < 400000; ++i) {
                uint32_t d = i < 31 ? 1u << i : i < 62 ? (1u << (i - 31)) + 1u : i < 93 ? (2u << (i - 62)) - 1u : i < 200 ? top - (i - 93) : rnd() >> (rnd() % 31);
                if (d < 1 || d > top) continue;
                const FastDiv f = fast_div((int)d);
                for (int k = 0; k < 40; ++k) {
                    const uint64_t m = (uint64_t)(rnd() % (top / d + 1)) * d + (k % 3) - 1;
                    const uint32_t n = k < 30 ? (uint32_t)m : k == 30 ? top : k == 31 ? 0 : rnd();
                    if (m > top && k < 30) continue;
                    if (quotient((int)n, f) != (int)(n / d)) { printf("%u / %u\\n", n, d); return 1; }
                }
            }
            return 0;
        }
        """)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


@pytest.mark.parametrize("folder,name", [("csrc", n) for n in ("paged_attn.cuh", "fast_div.cuh", "ptx_sm100.cuh", "paged.h", "paged.cu")] +
                         [("include", "ea.h")])
def test_a_changed_source_makes_the_library_stale(tmp_path, monkeypatch, folder, name):
    """Headers hold device code too: a library older than any of them is not the sources'."""
    for d, attr in ((build.CSRC, "CSRC"), (build.INCLUDE, "INCLUDE")):
        copy = tmp_path / os.path.basename(d)
        shutil.copytree(d, copy)
        monkeypatch.setattr(build, attr, str(copy))
    library = tmp_path / "libea.so"
    library.write_bytes(b"")
    monkeypatch.setattr(build, "LIB_PATH", str(library))
    now = max(p.stat().st_mtime for p in tmp_path.rglob("*") if p.is_file())
    os.utime(library, (now + 10, now + 10))
    assert not build._stale()
    os.utime(tmp_path / folder / name, (now + 20, now + 20))
    assert build._stale()
