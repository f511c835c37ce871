"""Paged cache at the edges of its range: scores beyond 32 bits, and what else a call may meet."""
import math

import pytest
import torch

import paged_reference as ref
from test_gpu_paged import Cache, attend, ea, i32, make          # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

INF = float("inf")


def one_hot_lists(ea, d, G, m, n, values, page=16, seed=0):
    """One list of n rows whose scores are whole numbers: k = (x_p, 0, ..), q = (1 or -1, 0, ..), v whole."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pages = ref.ceil_div(n, page)
    shape = ea.make_paged_shape(1, G, 1, d, page, pages, pages)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape, m))
    k, v = (torch.zeros(pages * page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:n, 0] = values(n, gen).to(torch.bfloat16)
    v[:n] = torch.randint(-8, 9, (n, d), generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.zeros(m, G, d, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = torch.randint(0, 2, (m, G), generator=gen, device="cuda").to(torch.bfloat16) * 2 - 1
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, 1, pages)
    return ctx, shape, q, i32([0, m]), m, i32([[n]]), table, k.view(pages, page, d), v.view(pages, page, d)


ANY = lambda n, gen: torch.randint(-3, 4, (n,), generator=gen, device="cuda")                  # noqa: E731
LOW = lambda n, gen: torch.randint(-5, -1, (n,), generator=gen, device="cuda")                 # noqa: E731
CLIMB = lambda n, gen: torch.linspace(-100, 100, n, device="cuda").round()                     # noqa: E731


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 40), (2, 700), (3, 20000), (5, 40), (12, 700), (12, 20000), (70, 3), (70, 700), (70, 20000)])
@pytest.mark.parametrize("values", [ANY, LOW, CLIMB], ids=["any", "low", "climb"])
@pytest.mark.parametrize("scale", [2.0e38, -2.0e38, 1.0e38, -1.0e30, 3.0e9, 1.2e7, -6.0e6])
def test_scores_out_of_range_are_not_answered_and_large_ones_pick_the_largest(ea, d, m, n, values, scale):      # noqa: F811
    """A token whose largest score is 2^30 or more in units of log 2 gets NaN, in either kernel; below, scores that differ do so by
    6e6 at least, and the rows of the largest one share the weight.

    Whole numbers times `scale`.  The rows that share have one weight, 1 or (what the rounding of the largest score leaves) a
    power of two that is rounded to bf16 for the product with V, 2^-8, and not for the sum; out's own rounding is 2^-8 (half a
    step).  Sums of up to 20 000 weights, 16 at a time, and 160 parts: some 1400 roundings of 2^-24 of the mean of |v| at most.
    lse carries six roundings of 2^-24 (two constants, three products, a sum) and that of the logarithm.
    """
    G = 4
    args = one_hot_lists(ea, d, G, m, n, values)
    ctx, q, k, v = args[0], args[2], args[7].view(-1, d)[:n], args[8].view(-1, d)[:n]
    out, lse = ea.ea_paged_attention(*args, scale=scale, want_lse=True)
    ctx.sync_status()
    scale32 = torch.tensor(scale, dtype=torch.float32).double().item()
    x = q[:, :, :1].double() * k[:, 0].double()                                                 # [m, G, n]
    seen = torch.arange(n, device="cuda")[None] <= torch.arange(m, device="cuda")[:, None] + n - m
    s = (scale32 * x).masked_fill(~seen[:, None], -INF)
    best = s.amax(-1, keepdim=True)
    hit = (s == best) & seen[:, None]
    ties = hit.sum(-1)
    far = (ties > 0) & (best[..., 0].abs() * math.log2(math.e) >= 2.0 ** 30)
    assert bool(torch.isnan(out[far]).all()) and bool(torch.isnan(lse[far]).all())
    want, mean = (torch.einsum("mgn,nd->mgd", hit.double(), x.double()) / ties.clamp(min=1)[..., None] for x in (v, v.abs()))
    assert bool(((out.double() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -12 * mean)[~far].all())
    blind = ties == 0
    assert bool((lse[blind] == -INF).all()) and not bool(out[blind].any())
    want_lse = best[..., 0] + torch.log(ties.double())
    near = ~far & ~blind
    err = (lse.double() - want_lse).abs()[near]
    assert bool((err <= 2.0 ** -21 * want_lse[near].abs() + 2.0 ** -20).all())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m", [1, 40])
def test_tokens_whose_scores_are_all_minus_infinity(ea, d, m):                                  # noqa: F811
    """exp(-infinity) over a sum of zeros: not the zeros of a token that sees no row."""
    args = one_hot_lists(ea, d, 4, m, 300, lambda n, gen: torch.full((n,), -INF, device="cuda"))
    args[2][:, :, 0] = 1.0
    args[7].view(-1, d)[:300, 1:] = 1.0
    out, lse = ea.ea_paged_attention(*args, want_lse=True)
    args[0].sync_status()
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("which", ["few rows", "chunk", "plan", "score"])
def test_a_replay_that_overwrites_a_fused_operand_is_recorded(ea, which):                       # noqa: F811
    """The operand of fused statistics lies where paged calls, and scoring calls with statistics, put theirs; the host sees no replay."""
    S, Hq, Hkv, d, n, W = 1, 8, 2, 128, 256, 32
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(*x, generator=gen, device="cuda").to(torch.bfloat16) for x in ((S, Hq, W, d), (S, Hkv, n, d), (S, Hkv, n, d)))
    dense = ea.make_shape(S, Hq, Hkv, d, n, W)
    if which == "plan":
        c = Cache(ea, 5000, 1, 1, 64, 16, 5000, 1)
        lens = [c.lens([0] * 5000), c.lens([9] * 5000)]
        slots, offsets = torch.empty(45000, dtype=torch.int32, device="cuda"), torch.empty(5001, dtype=torch.int32, device="cuda")
    else:
        c = make(ea, (8, 2, 128), 16, [40 if which == "chunk" else 1], [[2000, 3000]])
    ctx = ea.Context(0, max(ea.ea_workspace_bytes(dense), ea.ea_paged_workspace_bytes(c.shape, 40)))
    c.ctx = ctx
    pos = torch.full((S,), n, dtype=torch.int64, device="cuda")
    given = ea.ea_query_stats(ctx, dense, q, pos, 64, 1e6)

    def call():
        if which == "plan":
            ea.ea_page_plan(ctx, c.shape, *lens, c.table, c.free, c.n_free, slots=slots, offsets=offsets)
        elif which == "score":
            ea.ea_score(ctx, dense, k, v, *given, 0.02)
        else:
            attend(ea, c)

    graph = torch.cuda.CUDAGraph()
    if which != "plan":
        call()
    with torch.cuda.graph(graph):
        call()
    ctx.set_fused_stats(True)
    for _ in range(2):
        ea.ea_query_stats(ctx, dense, q, pos, 64, 1e6)
        for _ in range(2):
            scores = ea.ea_score(ctx, dense, k, v, None, None, 0.02)
        ctx.sync_status()
        ea.ea_query_stats(ctx, dense, q, pos, 64, 1e6)
        graph.replay()
        ea.ea_score(ctx, dense, k, v, None, None, 0.02)
        with pytest.raises(ea.EAError) as e:
            ctx.sync_status()
        # (the second plan finds an empty pool and records that; either word is an error)
        assert e.value.status in ((1, 7) if which == "plan" else (1,))
        ctx.sync_status()
    assert torch.equal(scores, ea.ea_score(ctx, dense, k, v, *given, 0.02))
    ctx.sync_status()


@pytest.mark.parametrize("lists", [4, 5000])
@pytest.mark.parametrize("given", [False, True])
def test_an_empty_slot_map_holds_no_rows(ea, lists, given):                                     # noqa: F811
    c = Cache(ea, lists // 2, 2, 2, 64, 16, 2 * lists, 8)
    kw = dict(slots=i32([])) if given else dict(n_slots=0)
    before = [x.clone() for x in (c.table, c.free, c.n_free)]
    none, some = [0] * lists, [0] * (lists - 1) + [17]
    for refused in (lambda: c.plan(none, some, **kw),
                    lambda: ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens(none), c.lens(some), **kw)):
        slots, offsets = refused()
        with pytest.raises(ea.EAError) as e:
            c.ctx.sync_status()
        assert e.value.status == 7 and slots.numel() == 0 and not bool(offsets.any())
        assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.free, c.n_free)))
    assert c.plan(none, some) is None                       # without a map they grow
    c.py.resize(none, some)
    c.same()
    c.plan(some, none, **kw)                                # and shrink with an empty one
    c.py.resize(some, none)
    c.same()
    ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens(some), c.lens(none), **kw)
    c.ctx.sync_status()


def test_outputs_that_overlap_other_buffers_are_refused(ea):                                    # noqa: F811
    c = make(ea, (8, 2, 128), 16, [1, 1], [[200, 300], [40, 50]])
    want, want_lse = attend(ea, c, want_lse=True)
    both = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device="cuda")
    both[:2] = c.q
    held = [x.clone() for x in (c.k, c.v, c.table, c.free, c.n_free)]

    def refused(call):
        with pytest.raises(ea.EAError) as e:
            call()
        assert e.value.status == 1

    c.q = both[:2]
    refused(lambda: attend(ea, c, out=c.q))
    refused(lambda: attend(ea, c, out=both[1:3]))
    refused(lambda: attend(ea, c, out=c.k.view(-1)[:2048].view(2, 8, 128)))
    refused(lambda: attend(ea, c, out=both[2:], lse=both[2:].view(-1)[:32].view(torch.float32).view(2, 8)))
    out, lse = attend(ea, c, out=both[2:], want_lse=True)                        # side by side is no overlap
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    rows, slots = c.k.view(-1, 128), i32([1, 0])
    fresh = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    refused(lambda: ea.ea_page_store(c.ctx, c.shape, slots, rows[:2], fresh, c.k, c.v))
    refused(lambda: ea.ea_page_store(c.ctx, c.shape, slots, fresh, c.v.view(-1, 128)[-2:], c.k, c.v))
    refused(lambda: ea.ea_page_store(c.ctx, c.shape, slots, fresh, fresh, c.k, c.k))
    refused(lambda: ea.ea_page_load(c.ctx, c.shape, slots, c.k, c.v, rows[:2], fresh))
    refused(lambda: ea.ea_page_load(c.ctx, c.shape, slots, c.k, c.v, fresh, fresh))
    longer = c.kv_lens + 1
    refused(lambda: ea.ea_page_plan(c.ctx, c.shape, c.kv_lens, longer, c.table, c.free, c.n_free, slots=c.free))
    refused(lambda: ea.ea_page_plan(c.ctx, c.shape, c.kv_lens, longer, c.table, c.free, c.n_free, n_slots=8, offsets=c.table.view(-1)[:5]))
    refused(lambda: ea.ea_page_slots(c.ctx, c.shape, c.table, c.kv_lens, longer, slots=c.table.view(-1)))
    c.ctx.sync_status()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(held, (c.k, c.v, c.table, c.free, c.n_free)))
    ea.ea_page_plan(c.ctx, c.shape, c.kv_lens, c.kv_lens, c.table, c.free, c.n_free, n_slots=1)     # inputs may be the same
    got, _ = ea.ea_page_load(c.ctx, c.shape, slots, c.k, c.k)                                       # so may pools that are read
    assert torch.equal(got.view(torch.uint8), rows[[1, 0]].view(torch.uint8))
    c.ctx.sync_status()


@pytest.mark.parametrize("order", [0, 1])
def test_a_plan_of_no_sequences_with_any_head_count(ea, order):                                 # noqa: F811
    shape = ea.make_paged_shape(0, 2 ** 30 + 1, 2 ** 30 + 1, 64, 16, 3, 4)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape))
    none = torch.empty(0, 2 ** 30 + 1, dtype=torch.int32, device="cuda")
    slots, offsets = ea.ea_page_plan(ctx, shape, none, none, none.view(0, 2 ** 30 + 1, 1).expand(0, 2 ** 30 + 1, 4).contiguous(), i32([0, 1, 2]),
                                     i32([3]), n_slots=2, order=order)
    ctx.sync_status()
    assert slots.tolist() == [-1, -1] and offsets.tolist() == [0]
