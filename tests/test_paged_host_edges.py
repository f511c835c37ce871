"""Refusals of the paged-cache calls at the edges of their arguments, without a GPU."""
import ctypes

import pytest

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
