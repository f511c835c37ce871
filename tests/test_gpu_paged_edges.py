"""Paged cache at the edges of its range: scores beyond 32 bits, and what else a call may meet."""
import math
import random

import pytest
import torch

import paged_reference as ref
from test_gpu_paged import Cache, attend, check, ea, i32, make          # noqa: F401 (a fixture)

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


# ---- parts of the kernels that other tests do not reach ------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,m", [(9, 1, 1), (5, 1, 3), (16, 2, 2), (16, 1, 1), (1, 1, 16), (33, 3, 1), (26, 2, 1)])
@pytest.mark.parametrize("page", [16, 128])
def test_nine_to_sixteen_rows_of_a_list(ea, d, Hq, Hkv, m, page):                               # noqa: F811
    """The upper half of the few-row kernel's tile: whole lists, lists shared by many CTAs, and many lists."""
    for lens in ([[40 + 7 * g for g in range(Hkv)], [m] * Hkv, [0] * Hkv], [[60000 + g for g in range(Hkv)]],
                 [[900 + (31 * s + 17 * g) % 300 for g in range(Hkv)] for s in range(70)]):
        for causal in (True, False):
            check(ea, make(ea, (Hq, Hkv, d), page, [m] * len(lens), lens), causal=causal)


@pytest.mark.parametrize("lists,most,page", [(3000, 100, 16), (4096, 40, 16), (40, 9000, 32), (1, 30000, 16)])
def test_plans_without_a_slot_map_over_many_processors(ea, lists, most, page):                  # noqa: F811
    """Pools of more than 1024 pages: growing and shrinking lists mixed, pages pushed, the free count by the CTA that ends last."""
    rng = random.Random(lists)
    c = Cache(ea, lists, 1, 1, 64, page, lists * ref.ceil_div(most, page) + 3, ref.ceil_div(most, page))
    old = [0] * lists
    for _ in range(6):
        new = [rng.choice((o, 0, most, rng.randint(0, most))) for o in old]
        assert c.plan(old, new) is None
        assert c.py.resize(old, new)
        c.same()
        old = new
    c.ctx.sync_status()


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("seqs,each,capacity", [(3, 4000, 40001), (30, 3000, 300003)])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_slot_maps_that_begin_at_any_word(ea, order, seqs, each, capacity, shift):              # noqa: F811
    Hkv, page = 3, 16
    wide = ref.ceil_div(each, page)
    c = Cache(ea, seqs, Hkv, Hkv, 64, page, seqs * Hkv * wide, wide)
    old, new = [0] * (seqs * Hkv), [each - 5 * (r // Hkv) for r in range(seqs * Hkv)]
    got, again = (torch.full((capacity + 8,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    _, offsets = c.plan(old, new, slots=got[shift:shift + capacity], order=order)
    assert c.py.resize(old, new)
    rows, want_offsets = c.py.slots(old, new, Hkv if order else None)
    assert offsets.tolist() == want_offsets
    want = torch.full((capacity + 8,), 77, dtype=torch.int32)
    want[shift:shift + capacity] = -1
    want[shift:shift + len(rows)] = torch.tensor(rows, dtype=torch.int32)
    assert torch.equal(got.cpu(), want)
    ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens(old), c.lens(new), slots=again[shift:shift + capacity], order=order)
    assert torch.equal(again, got)
    c.ctx.sync_status()


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (16, 8, 256)])
@pytest.mark.parametrize("max_q", [3, 64, 300])
def test_a_padded_batch(ea, heads, max_q):                                                      # noqa: F811
    """A captured batch is launched for more tokens, and more sequences, than a step has."""
    S, Hkv = 60, heads[1]
    chunks = [0] * S
    chunks[0], chunks[1], chunks[31], chunks[59] = 1, 3, 1, 2
    lens = [[(700 + 13 * s + 5 * g) if s % 2 else 0 for g in range(Hkv)] for s in range(S)]
    c = make(ea, heads, 16, chunks, lens, n_tokens=400, max_q=max_q)
    c.ctx = ea.Context(0, ea.ea_paged_workspace_bytes(c.shape, max_q))
    out = torch.full((400, heads[0], heads[2]), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((400, heads[0]), 7.0, device="cuda")
    check(ea, c, out=out, lse=lse)
    assert bool((out[7:] == 7).all()) and bool((lse[7:] == 7).all())


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (16, 8, 256)])
def test_one_step_as_a_call_for_each_run_of_sequences(ea, heads):                               # noqa: F811
    """Single tokens in a call of their own beside a prompt's chunk: the same tokens, offsets and outputs, by runs."""
    Hkv = heads[1]
    chunks = [1] * 6 + [130] + [1, 0, 1]
    lens = [[max(m, 1) + (s * 53 + g * 97) % 400 for g in range(Hkv)] for s, m in enumerate(chunks)]
    c = make(ea, heads, 16, chunks, lens, n_tokens=sum(chunks) + 3)
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
    for a, b, max_q in ((0, 6, 1), (6, 7, 130), (7, 10, 1)):
        run = ea.make_paged_shape(b - a, *heads, 16, c.k.shape[0], c.table.shape[2])
        ea.ea_paged_attention(c.ctx, run, c.q, c.q_offsets[a:b + 1], max_q, c.kv_lens[a:b], c.table[a:b], c.k, c.v, out=out, lse=lse)
    c.ctx.sync_status()
    n = sum(chunks)
    exact = ref.attention(c.q, c.q_offsets, c.kv_lens, c.rows_of, c.d ** -0.5, True)
    tol_o, tol_l = ref.attention_tolerance(*exact, int(c.kv_lens.max()))
    assert bool(((out.double() - exact[0]).abs() <= tol_o)[:n].all()) and bool(((lse.double() - exact[1]).abs() <= tol_l)[:n].all())
    assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())


# ---- as they are used ------------------------------------------------------------------------------------------------
def test_a_cache_through_two_compressions_with_generation_in_a_graph(ea):                       # noqa: F811
    """A prompt's cache compressed over all heads of a layer into pages, sixteen tokens generated as replays of one graph, every
    list (they differ in length) scored and compressed again, stored back, and one more token."""
    S, Hq, Hkv, d, n, W, n_kept, page, steps = 2, 8, 2, 128, 512, 16, 192, 16, 16
    G = Hq // Hkv
    gen = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)      # noqa: E731
    q_win, k, v = rnd(S, Hq, W, d), rnd(S, Hkv, n, d), rnd(S, Hkv, n, d)
    dense = ea.make_shape(S, Hq, Hkv, d, n, W)
    wide = ref.ceil_div(Hkv * n_kept + steps, page)
    paged = ea.make_paged_shape(S, Hq, Hkv, d, page, S * Hkv * wide, wide)
    longest = ea.make_shape(1, G, 1, d, wide * page, W)
    ctx = ea.Context(0, max(ea.ea_workspace_bytes(dense), ea.ea_workspace_bytes(longest), ea.ea_paged_workspace_bytes(paged, 1)))
    pos = torch.full((S,), n, dtype=torch.int64, device="cuda")
    scores = ea.ea_score(ctx, dense, k, v, *ea.ea_query_stats(ctx, dense, q_win, pos, 64, 1e6), 0.02)
    idx, head_off, k_out, v_out = ea.ea_select_compact_adaptive(ctx, dense, scores, n_kept, ea.ea_n_floor(n_kept, 0.2), k, v)
    lens = (head_off[:, 1:] - head_off[:, :-1]).to(torch.int32).contiguous()
    table = torch.full((S, Hkv, wide), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.arange(S * Hkv * wide, dtype=torch.int32, device="cuda"), i32([S * Hkv * wide])
    kp, vp = (torch.full((S * Hkv * wide, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zero = torch.zeros_like(lens)
    slots, _ = ea.ea_page_plan(ctx, paged, zero, lens, table, free, n_free, n_slots=S * Hkv * n_kept)
    ea.ea_page_store(ctx, paged, slots, k_out.view(-1, d), v_out.view(-1, d), kp, vp)
    rows = {(s, g): [x[s, int(head_off[s, g]):int(head_off[s, g + 1])] for x in (k_out, v_out)] for s in range(S) for g in range(Hkv)}

    q, kn, vn = (torch.zeros(S, h, d, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    longer, out = torch.empty_like(lens), torch.empty_like(q)
    one, off = torch.empty(S * Hkv, dtype=torch.int32, device="cuda"), torch.empty(S + 1, dtype=torch.int32, device="cuda")

    def step():
        torch.add(lens, 1, out=longer)
        ea.ea_page_plan(ctx, paged, lens, longer, table, free, n_free, order=ea.SLOTS_BY_TOKEN, slots=one, offsets=off)
        ea.ea_page_store(ctx, paged, one, kn, vn, kp, vp)
        ea.ea_paged_attention(ctx, paged, q, off, 1, longer, table, kp, vp, out=out)
        lens.copy_(longer)

    def attended():
        ctx.sync_status()
        exact = ref.attention(q, off, lens, lambda s, g: rows[s, g], d ** -0.5, True)
        assert bool(((out.double() - exact[0]).abs() <= ref.attention_tolerance(*exact, int(lens.max()))[0]).all())

    kept = [x.clone() for x in (lens, table, free, n_free, kp, vp)]
    step()
    for x, y in zip((lens, table, free, n_free, kp, vp), kept):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((lens, table, free, n_free, kp, vp), kept):
        x.copy_(y)
    window = []
    for _ in range(steps):
        for x in (q, kn, vn):
            x.copy_(rnd(*x.shape))
        window.append(q.clone())
        graph.replay()
        for (s, g), pair in rows.items():
            pair[:] = [torch.cat([pair[0], kn[s, g][None]]), torch.cat([pair[1], vn[s, g][None]])]
        attended()
    # the next compression: half of every list, scored with the window of the queries since
    q_win = torch.stack(window, 2)                                                              # [S, Hq, W, d]
    slots, offsets = ea.ea_page_slots(ctx, paged, table, zero, lens, n_slots=int(lens.sum()))
    kd, vd = ea.ea_page_load(ctx, paged, slots, kp, vp)
    ends, half, new = offsets.tolist(), [], {}
    for i, (s, g) in enumerate(sorted(rows)):
        a, b = ends[i], ends[i + 1]
        assert torch.equal(kd[a:b], rows[s, g][0]) and torch.equal(vd[a:b], rows[s, g][1])
        m = b - a
        one_list = ea.make_shape(1, G, 1, d, m, W)
        kr, vr = kd[a:b].view(1, 1, m, d), vd[a:b].view(1, 1, m, d)
        stats = ea.ea_query_stats(ctx, one_list, q_win[s:s + 1, g * G:(g + 1) * G].contiguous(), pos[:1] + steps, 64, 1e6)
        scores = ea.ea_score(ctx, one_list, kr, vr, *stats, 0.02)
        idx, ko, vo = ea.ea_select_compact(ctx, one_list, scores, m // 2, kr, vr)
        top = scores.view(-1).sort(descending=True, stable=True).indices[:m // 2].sort().values
        assert torch.equal(idx.view(-1).long(), top)
        half.append(m // 2)
        new[s, g] = [ko.view(-1, d), vo.view(-1, d)]
        assert torch.equal(new[s, g][0], rows[s, g][0][top]) and torch.equal(new[s, g][1], rows[s, g][1][top])
    rows = new
    fewer = i32(half, S, Hkv)
    before = n_free.item()
    ea.ea_page_plan(ctx, paged, lens, fewer, table, free, n_free)
    slots, _ = ea.ea_page_slots(ctx, paged, table, zero, fewer, n_slots=sum(half))
    ea.ea_page_store(ctx, paged, slots, torch.cat([rows[x][0] for x in sorted(rows)]), torch.cat([rows[x][1] for x in sorted(rows)]), kp, vp)
    assert n_free.item() - before == int(((lens + page - 1) // page - (fewer + page - 1) // page).sum())
    lens.copy_(fewer)
    for x in (q, kn, vn):
        x.copy_(rnd(*x.shape))
    graph.replay()                                          # the same graph over the compressed lists
    for (s, g), pair in rows.items():
        pair[:] = [torch.cat([pair[0], kn[s, g][None]]), torch.cat([pair[1], vn[s, g][None]])]
    attended()
    held = table[table >= 0].tolist()
    assert len(set(held)) == len(held) and not set(held) & set(free[:n_free.item()].tolist())
