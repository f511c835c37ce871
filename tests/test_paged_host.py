"""Refusals of the paged-cache calls that need no GPU: every argument check comes before the first CUDA call."""
import ctypes

import pytest

from paper_2510_00636_b200 import build


@pytest.fixture(scope="module")
def ea():
    build.build()
    from paper_2510_00636_b200 import binding
    binding.lib()
    return binding


@pytest.fixture()
def ctx():
    """Stands for a context without a workspace: what passes the argument checks ends at EA_ERR_WORKSPACE (3)."""
    return ctypes.create_string_buffer(4096)


GOOD = dict(n_seqs=2, n_q_heads=8, n_kv_heads=2, head_dim=128, page_rows=16, n_pages=64, max_pages=8)
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 0x1000                                     # an aligned address that is never followed


def shape(ea, **changes):
    return ea.make_paged_shape(**{**GOOD, **changes})


@pytest.mark.parametrize("changes,status", [
    (dict(n_seqs=-1), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_kv_heads=3), INVALID),
    (dict(n_pages=-1), INVALID), (dict(max_pages=-1), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(page_rows=8), UNSUPPORTED),
    (dict(page_rows=48), UNSUPPORTED), (dict(page_rows=0), UNSUPPORTED), (dict(n_seqs=32768), UNSUPPORTED),
    (dict(n_pages=1 << 27), UNSUPPORTED), (dict(max_pages=1 << 27), UNSUPPORTED), (dict(max_pages=(1 << 26) + 1), UNSUPPORTED),
])
def test_shapes_that_do_not_fit_are_refused_by_every_call(ea, ctx, changes, status):
    L, s = ea.lib(), shape(ea, **changes)
    ref = ctypes.byref(s)
    out = ctypes.c_size_t(0)
    assert L.ea_paged_workspace_bytes(ref, 1, ctypes.byref(out)) == status
    assert L.ea_page_plan(ctx, ref, P, P, P, P, P, 0, P, 4, P, None) == status
    assert L.ea_page_slots(ctx, ref, P, P, P, 0, P, 4, P, None) == status
    assert L.ea_page_store(ctx, ref, P, 4, P, P, 0, 0, P, P, None) == status
    assert L.ea_page_load(ctx, ref, P, 4, P, P, P, P, None) == status
    assert L.ea_paged_attention(ctx, ref, P, 0, 4, P, 2, P, P, P, P, 1.0, 1, P, P, None) == status


def test_workspace_bytes(ea):
    assert 0 < ea.ea_paged_workspace_bytes(shape(ea)) < 64 << 20
    many = ea.ea_paged_workspace_bytes(shape(ea, n_seqs=32767))
    assert many >= 3 * 65534 * 4
    with pytest.raises(ea.EAError):
        ea.ea_paged_workspace_bytes(shape(ea), -1)
    assert ea.lib().ea_paged_workspace_bytes(ctypes.byref(shape(ea)), 1, None) == INVALID
    assert ea.lib().ea_paged_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t(0))) == INVALID


def _vary(base, changes):
    args = list(base)
    for i, v in changes.items():
        args[i] = v
    return args


def test_plan_arguments(ea, ctx):
    L, ref = ea.lib(), ctypes.byref(shape(ea))
    good = [P, P, P, P, P, 0, P, 64, P]        # old, new, table, free, n_free, order, slots, capacity, offsets
    assert L.ea_page_plan(None, ref, *good, None) == INVALID
    assert L.ea_page_plan(ctx, None, *good, None) == INVALID
    assert L.ea_page_plan(ctx, ref, *good, None) == WORKSPACE
    for change in ({0: None}, {1: None}, {2: None}, {3: None}, {4: None}, {5: 2}, {5: -1}, {6: None}, {7: -1}, {0: P + 2},
                   {2: P + 1}, {8: P + 3}):
        assert L.ea_page_plan(ctx, ref, *_vary(good, change), None) == INVALID, change
    for change in ({6: None, 7: 0}, {8: None}, {5: 1}):
        assert L.ea_page_plan(ctx, ref, *_vary(good, change), None) == WORKSPACE, change


def test_slots_arguments(ea, ctx):
    L, ref = ea.lib(), ctypes.byref(shape(ea))
    good = [P, P, P, 0, P, 64, P]              # table, first, end, order, slots, capacity, offsets
    assert L.ea_page_slots(None, ref, *good, None) == INVALID
    assert L.ea_page_slots(ctx, ref, *good, None) == WORKSPACE
    for change in ({0: None}, {1: None}, {2: None}, {3: 5}, {4: None}, {5: -2}, {4: P + 2}):
        assert L.ea_page_slots(ctx, ref, *_vary(good, change), None) == INVALID, change


def test_store_and_load_arguments(ea, ctx):
    L, ref = ea.lib(), ctypes.byref(shape(ea))
    good = [P, 4, P, P, 0, 0, P, P]            # slots, rows, k, v, k_stride, v_stride, k_pages, v_pages
    assert L.ea_page_store(None, ref, *good, None) == INVALID
    assert L.ea_page_store(ctx, ref, *_vary(good, {1: 0}), None) == 0
    for change in ({0: None}, {1: -1}, {1: 1 << 31}, {2: None}, {3: None}, {6: None}, {7: None}, {2: P + 8}, {6: P + 2}, {4: -256},
                   {4: 248}, {4: 260}, {5: 128}, {1: 3, 4: 512}, {0: P + 2}):
        assert L.ea_page_store(ctx, ref, *_vary(good, change), None) == INVALID, change
    good = [P, 4, P, P, P, P]
    assert L.ea_page_load(None, ref, *good, None) == INVALID
    assert L.ea_page_load(ctx, ref, *_vary(good, {1: 0}), None) == 0
    for change in ({0: None}, {1: -1}, {2: None}, {3: None}, {4: None}, {5: None}, {5: P + 4}):
        assert L.ea_page_load(ctx, ref, *_vary(good, change), None) == INVALID, change


def test_attention_arguments(ea, ctx):
    L, ref = ea.lib(), ctypes.byref(shape(ea))
    good = [P, 0, 4, P, 2, P, P, P, P, 0.1, 1, P, P]   # q, stride, tokens, offsets, max_q, lens, table, k, v, scale, causal, out, lse
    assert L.ea_paged_attention(None, ref, *good, None) == INVALID
    assert L.ea_paged_attention(ctx, ref, *good, None) == WORKSPACE
    inf = float("inf")
    for change in ({0: None}, {0: P + 8}, {1: 1000}, {1: 1028}, {1: -1024}, {2: -1}, {4: -1}, {4: 5}, {3: None}, {5: None},
                   {6: None}, {7: None}, {8: None}, {9: inf}, {9: float("nan")}, {11: None}, {11: P + 8}, {12: P + 2}):
        assert L.ea_paged_attention(ctx, ref, *_vary(good, change), None) == INVALID, change
    for change in ({12: None}, {1: 1032}, {10: 0}):
        assert L.ea_paged_attention(ctx, ref, *_vary(good, change), None) == WORKSPACE, change
    for change in ({2: 0, 4: 0}, {4: 0}):
        assert L.ea_paged_attention(ctx, ref, *_vary(good, change), None) == 0, change
    assert L.ea_paged_attention(ctx, ctypes.byref(shape(ea, n_seqs=0)), *good, None) == 0
    assert L.ea_paged_attention(ctx, ref, *_vary(good, {2: 1 << 30, 4: 1}), None) == UNSUPPORTED


def test_scales_whose_multiple_of_log2_e_overflows_are_refused(ea, ctx):
    L, ref = ea.lib(), ctypes.byref(shape(ea))
    good = [P, 0, 4, P, 2, P, P, P, P, 2.0e38, 1, P, P]
    assert L.ea_paged_attention(ctx, ref, *good, None) == WORKSPACE
    for scale in (2.5e38, -2.5e38):
        assert L.ea_paged_attention(ctx, ref, *_vary(good, {9: scale}), None) == INVALID


def test_status_string(ea):
    assert ea.lib().ea_status_string(7) == b"EA_ERR_PAGES"
