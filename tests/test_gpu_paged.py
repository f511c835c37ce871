"""Paged cache on the GPU: page bookkeeping and row moves bit for bit against Python, attention against 64 bits."""
import math
import random

import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ea():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2510_00636_b200 import binding
    binding.lib()
    return binding


def i32(x, *shape):
    t = torch.tensor(x, dtype=torch.int32, device="cuda")
    return t.view(*shape) if shape else t


class Cache:
    """A paged cache on the device beside its Python statement."""

    def __init__(self, ea, seqs, Hq, Hkv, d, page, n_pages, max_pages, max_q=1, seed=0):
        self.ea, self.seqs, self.Hkv, self.d, self.page = ea, seqs, Hkv, d, page
        self.shape = ea.make_paged_shape(seqs, Hq, Hkv, d, page, n_pages, max_pages)
        self.ctx = ea.Context(0, ea.ea_paged_workspace_bytes(self.shape, max_q))
        self.py = ref.Pages(seqs * Hkv, max_pages, n_pages, page)
        random.Random(seed).shuffle(self.py.free)
        self.table = torch.full((seqs, Hkv, max_pages), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = i32(self.py.free), i32([n_pages])

    def lens(self, x):
        return i32(x, self.seqs, self.Hkv)

    def plan(self, old, new, **kw):
        return self.ea.ea_page_plan(self.ctx, self.shape, self.lens(old), self.lens(new), self.table, self.free, self.n_free, **kw)

    def same(self):
        n = self.py.n_free
        assert self.n_free.item() == n
        assert self.free[:n].tolist() == self.py.free[:n]
        assert torch.equal(self.table.cpu().view(-1), torch.tensor(self.py.table, dtype=torch.int32).view(-1))


# ---- plans and slots -------------------------------------------------------------------------------------------------
# a cluster; three launches (many slots); more lists than a CTA scans itself
@pytest.mark.parametrize("seqs,Hkv,page,most,rounds,capacity", [
    (1, 1, 16, 40, 12, 64), (5, 3, 16, 100, 10, 1600), (7, 8, 32, 300, 6, 20000), (3, 4, 128, 9000, 4, 120000),
    (600, 7, 64, 70, 3, 300000), (16383, 4, 16, 20, 2, 1 << 21)])
def test_plans_follow_the_rule(ea, seqs, Hkv, page, most, rounds, capacity):
    rng = random.Random(seqs)
    lists = seqs * Hkv
    c = Cache(ea, seqs, Hkv, Hkv, 64, page, lists * ref.ceil_div(most, page) + 3, ref.ceil_div(most, page) + 1)
    old = [0] * lists
    for step in range(rounds):
        by_token = step % 2 == 1
        if by_token:
            room = [min(most - old[s * Hkv + g] for g in range(Hkv)) for s in range(seqs)]
            gain = [rng.choice((0, 0, min(r, 1), rng.randint(0, r))) for r in room]
            new = [old[r] + gain[r // Hkv] for r in range(lists)]
        else:
            new = [rng.choice((o, 0, most, rng.randint(0, most))) for o in old]
        order = ea.SLOTS_BY_TOKEN if by_token else ea.SLOTS_BY_LIST
        slots, offsets = c.plan(old, new, n_slots=capacity, order=order)
        assert c.py.resize(old, new)
        c.same()
        want, want_off = c.py.slots(old, [max(o, n) for o, n in zip(old, new)], Hkv if by_token else None)
        assert offsets.tolist() == want_off
        got = slots.cpu()
        assert torch.equal(got[:len(want)], torch.tensor(want, dtype=torch.int32)) and bool((got[len(want):] == -1).all())
        # the same rows from the table that stands now
        again, off2 = ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens(old), c.lens(new), n_slots=capacity, order=order)
        assert torch.equal(again, slots) and torch.equal(off2, offsets)
        c.ctx.sync_status()
        old = new


@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("lists", [6, 5000])
def test_a_shrink_that_undoes_a_growth_restores_the_free_list(ea, lists, slots):
    rng = random.Random(1)
    c = Cache(ea, lists, 1, 1, 64, 16, lists * 8, 8)
    old = [rng.randint(0, 60) for _ in range(lists)]
    c.plan([0] * lists, old)
    before = c.table.clone(), c.free.clone(), c.n_free.clone()
    new = [o + rng.randint(0, 60) for o in old]
    kw = dict(n_slots=sum(new) - sum(old)) if slots else {}
    c.plan(old, new, **kw)
    c.plan(new, old, **kw)
    assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.free, c.n_free)))
    c.ctx.sync_status()


@pytest.mark.parametrize("lists", [8, 4200])
@pytest.mark.parametrize("slots", [40, 70000])
def test_plans_that_cannot_be_served_change_nothing(ea, lists, slots):
    Hkv = 2
    n_pages = lists + 4
    c = Cache(ea, lists // Hkv, Hkv, Hkv, 64, 16, n_pages, 3)
    old = [16] * lists
    c.plan([0] * lists, old)
    c.ctx.sync_status()
    before = c.table.clone(), c.free.clone(), c.n_free.clone()

    def bump(**at):
        new = list(old)
        for r, n in at.items():
            new[int(r[1:])] = n
        return new

    wrong = [(bump(r0=48, r1=48, r3=32), {}),                                       # five pages, four free
             (bump(r2=-1), {}), (bump(r5=49), {}),                                  # no such length
             (bump(r0=17), dict(order=ea.SLOTS_BY_TOKEN))]                          # the other head of the token did not grow
    if slots == 40:
        wrong.append((bump(r0=40, r1=40), {}))                                      # more rows than the map holds
    for new, kw in wrong:
        got, offsets = c.plan(old, new, n_slots=slots, **kw)
        with pytest.raises(ea.EAError) as e:
            c.ctx.sync_status()
        assert e.value.status == 7
        assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.free, c.n_free)))
        assert bool((got == -1).all()) and not bool(offsets.any())
    bad_free = i32([n_pages + 1])
    got, offsets = ea.ea_page_plan(c.ctx, c.shape, c.lens(old), c.lens(bump(r0=17)), c.table, c.free, bad_free, n_slots=slots)
    with pytest.raises(ea.EAError):
        c.ctx.sync_status()
    assert torch.equal(c.table, before[0]) and bool((got == -1).all())
    c.plan(old, bump(r0=20, r1=17), n_slots=slots)                                  # and the next one goes through
    c.ctx.sync_status()
    assert c.n_free.item() == 2


def test_slots_of_ranges_and_of_pages_outside_the_pool(ea):
    c = Cache(ea, 2, 2, 1, 64, 16, 8, 4)
    c.plan([0, 0], [50, 20])
    c.py.resize([0, 0], [50, 20])
    c.table[0, 0, 1] = 8
    c.table[1, 0, 1] = -1
    slots, offsets = ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens([15, 18]), c.lens([34, 3]), n_slots=21)
    want, _ = c.py.slots([15, 18], [34, 18])
    for i, p in enumerate(range(15, 34)):
        if p // 16 == 1:
            want[i] = -1
    assert slots.tolist() == want + [-1, -1] and offsets.tolist() == [0, 19, 19]
    c.ctx.sync_status()


def test_an_empty_call(ea):
    c = Cache(ea, 0, 2, 1, 64, 16, 0, 0)
    slots, offsets = c.plan([], [], n_slots=5)
    assert slots.tolist() == [-1] * 5 and offsets.tolist() == [0]
    c.ctx.sync_status()


# ---- rows ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,strided", [(1, False), (37, False), (36, True), (5000, False), (4000, True)])
def test_rows_into_their_slots_and_back(ea, d, rows, strided):
    Hkv, page, n_pages = 4, 16, 400
    shape = ea.make_paged_shape(3, Hkv, Hkv, d, page, n_pages, 100)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape))
    gen = torch.Generator(device="cuda").manual_seed(rows + d)
    pools = [torch.randn(n_pages, page, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    slots = torch.randperm(n_pages * page, generator=gen, device="cuda")[:rows].to(torch.int32)
    slots[rows // 2] = -1
    if strided:                                   # keys and values where a fused projection leaves them, with other strides
        fused = torch.randn(rows // Hkv, 3 * Hkv * d, generator=gen, device="cuda").to(torch.bfloat16)
        new = [fused[:, Hkv * d:2 * Hkv * d].view(-1, Hkv, d), torch.randn(rows // Hkv, Hkv, d, generator=gen, device="cuda").to(torch.bfloat16)]
    else:
        new = [torch.randn(rows, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    want = [p.clone().view(-1, d) for p in pools]
    there = slots >= 0
    for w, x in zip(want, new):
        w[slots[there].long()] = x.reshape(rows, d)[there]
    ea.ea_page_store(ctx, shape, slots, *new, *pools)
    assert all(torch.equal(w, p.view(-1, d)) for w, p in zip(want, pools))
    out = [torch.full((rows, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ea.ea_page_load(ctx, shape, slots, *pools, *out)
    for x, y in zip(out, new):
        assert torch.equal(x[there], y.reshape(rows, d)[there]) and bool((x[~there] == 7.0).all())
    ctx.sync_status()


def test_slots_outside_the_pool_are_skipped_and_reported(ea):
    shape = ea.make_paged_shape(1, 1, 1, 64, 16, 4, 4)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape))
    pools = [torch.zeros(4, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    new = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    slots = i32([3, 64, -2, 2 ** 31 - 1])
    ea.ea_page_store(ctx, shape, slots, new, new, *pools)
    with pytest.raises(ea.EAError) as e:
        ctx.sync_status()
    assert e.value.status == 7 and pools[0].sum().item() == 64 and bool((pools[1].view(-1, 64)[3] == 1).all())
    k, v = ea.ea_page_load(ctx, shape, slots, *pools, new.clone(), new.clone())
    with pytest.raises(ea.EAError):
        ctx.sync_status()
    assert bool((k == 1).all())


# ---- attention -------------------------------------------------------------------------------------------------------
def make(ea, heads, page, chunks, lens, seed=0, n_tokens=None, spare=3, stale=NAN, q_pad=0, max_q=None):
    """A cache of lists of the given lengths on scattered pages; rows behind a list's end and unused pages hold `stale`."""
    Hq, Hkv, d = heads
    S = len(chunks)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = [n for r in lens for n in r]
    max_pages = max([ref.ceil_div(n, page) for n in flat] + [1])
    n_pages = sum(ref.ceil_div(n, page) for n in flat) + spare
    c = Cache(ea, S, Hq, Hkv, d, page, n_pages, max_pages, max(chunks + [1]), seed)
    c.plan([0] * len(flat), flat)
    slots, _ = ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens([0] * len(flat)), c.lens(flat), n_slots=max(1, sum(flat)))
    c.k = torch.full((n_pages, page, d), stale, dtype=torch.bfloat16, device="cuda")
    c.v = torch.full((n_pages, page, d), stale, dtype=torch.bfloat16, device="cuda")
    big = torch.ones(d, device="cuda")
    big[:2] = 4.0
    rows_k = ((torch.randn(sum(flat), d, generator=gen, device="cuda") + 0.3) * big).to(torch.bfloat16)
    rows_v = torch.randn(sum(flat), d, generator=gen, device="cuda").to(torch.bfloat16)
    c.k.view(-1, d)[slots[:sum(flat)].long()] = rows_k
    c.v.view(-1, d)[slots[:sum(flat)].long()] = rows_v
    T = sum(chunks) if n_tokens is None else n_tokens
    q = (torch.randn(T, Hq + q_pad, d, generator=gen, device="cuda") * big).to(torch.bfloat16)
    c.q = q[:, :Hq]
    off = [0]
    for m in chunks:
        off.append(off[-1] + m)
    c.q_offsets, c.max_q = i32(off), max(chunks + [0]) if max_q is None else max_q
    c.kv_lens = c.lens(flat)
    at = [0]
    for n in flat:
        at.append(at[-1] + n)
    c.rows_of = lambda s, g: (rows_k[at[s * Hkv + g]:at[s * Hkv + g + 1]], rows_v[at[s * Hkv + g]:at[s * Hkv + g + 1]])
    return c


def attend(ea, c, **kw):
    return ea.ea_paged_attention(c.ctx, c.shape, c.q, c.q_offsets, c.max_q, c.kv_lens, c.table, c.k, c.v, **kw)


def check(ea, c, scale=None, causal=True, **kw):
    out, lse = attend(ea, c, scale=scale, causal=causal, want_lse=True, **kw)
    c.ctx.sync_status()
    exact = ref.attention(c.q, c.q_offsets, c.kv_lens, c.rows_of, c.d ** -0.5 if scale is None else scale, causal)
    tol_o, tol_l = ref.attention_tolerance(*exact, max(1, int(c.kv_lens.max())))
    n = int(c.q_offsets[-1])
    want_o, want_l = exact[0][:n], exact[1][:n]
    err = (out[:n].double() - want_o).abs()
    assert bool((err <= tol_o[:n]).all()), f"out: {(err / tol_o[:n]).max().item()} of the tolerance"
    empty = torch.isinf(want_l)
    assert torch.equal(empty, lse[:n] == -INF) and bool((out[:n][empty] == 0).all())
    err = (lse[:n].double() - want_l).abs()[~empty]
    assert bool((err <= tol_l[:n][~empty]).all()), f"lse: {(err / tol_l[:n][~empty]).max().item()} of the tolerance"
    return out, lse


HEADS = [(4, 2, 64), (32, 8, 128), (16, 8, 256), (28, 4, 128), (3, 3, 64), (24, 1, 128), (40, 2, 256), (130, 1, 64)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_one_token_per_sequence(ea, heads, page):
    Hkv = heads[1]
    lens = [[(s * 131 + g * 37) % 300 + 1 for g in range(Hkv)] for s in range(5)]
    lens[1] = [1] * Hkv
    lens[2][0] = 129
    lens[3][-1] = 1000
    check(ea, make(ea, heads, page, [1] * 5, lens))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_of_different_lengths(ea, heads, page, causal):
    Hkv = heads[1]
    chunks = [5, 1, 0, 67, 130]
    lens = [[max(m, 1) + (s * 53 + g * 97) % 400 for g in range(Hkv)] for s, m in enumerate(chunks)]
    lens[0] = [5] * Hkv                                      # the chunk is all there is
    check(ea, make(ea, heads, page, chunks, lens), causal=causal)


@pytest.mark.parametrize("heads", [(4, 2, 64), (16, 8, 256), (28, 4, 128)])
@pytest.mark.parametrize("m", [1, 3, 40, 200])
def test_lists_without_rows_and_shorter_than_the_chunk(ea, heads, m):
    Hkv = heads[1]
    lens = [[0] * Hkv, [max(0, m - 1 - g) for g in range(Hkv)], [m + 17] * Hkv, [g % 2 * 130 for g in range(Hkv)]]
    for causal in (True, False):
        check(ea, make(ea, heads, 16, [m] * 4, lens), causal=causal)


@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128), (4, 2, 256)])
@pytest.mark.parametrize("m", [1, 129])
@pytest.mark.parametrize("n", [127, 128, 129, 255, 256, 257, 1023, 1025])
def test_lengths_around_the_tiles(ea, heads, m, n):
    check(ea, make(ea, heads, 32, [min(m, n)], [[n, max(n - 1, m)]]))


@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("m", [1, 2, 300])
def test_long_lists_shared_by_many_processors(ea, heads, m):
    lens = [[20000 + 1111 * g for g in range(heads[1])], [m] * heads[1], [7000] * heads[1]]
    check(ea, make(ea, heads, 64, [m] * 3, lens))


@pytest.mark.parametrize("m", [1, 150])
def test_queries_inside_a_fused_projection_and_tokens_of_no_sequence(ea, m):
    c = make(ea, (8, 2, 128), 16, [m, m], [[200, 333], [170, 160]], n_tokens=2 * m + 9, q_pad=4)
    assert c.q.stride(0) == 12 * 128
    out = torch.full((2 * m + 9, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2 * m + 9, 8), 7.0, device="cuda")
    check(ea, c, out=out, lse=lse)
    assert bool((out[2 * m:] == 7).all()) and bool((lse[2 * m:] == 7).all())
    shifted = make(ea, (8, 2, 128), 16, [m, m], [[200, 333], [170, 160]], n_tokens=2 * m + 9, q_pad=4)
    shifted.q_offsets += 5
    out2, lse2 = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    attend(ea, shifted, out=out2, lse=lse2)
    for o in (out2, lse2):
        assert bool((o[:5] == 7).all()) and bool((o[2 * m + 5:] == 7).all())
    assert not bool((lse2[5:2 * m + 5] == 7).any())


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (16, 8, 256)])
@pytest.mark.parametrize("m", [1, 90])
@pytest.mark.parametrize("scale", [0.0, -0.11, 1.5])
def test_scales_from_flat_to_one_hot(ea, heads, m, scale):
    check(ea, make(ea, heads, 16, [m, m], [[m + 300] * heads[1], [m + 77] * heads[1]]), scale=scale)


@pytest.mark.parametrize("m", [1, 100])
def test_the_maximum_may_come_late_and_be_large(ea, m):
    """Scores that climb along the list by thousands: every block moves the running maximum."""
    c = make(ea, (8, 2, 128), 16, [m], [[1500, 1400]])
    rows = [c.rows_of(0, g) for g in range(2)]
    for g, (k, _) in enumerate(rows):
        k[:, 5] = torch.linspace(-300, 300, k.shape[0], device="cuda").to(torch.bfloat16)
        slots, _ = ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens([0, 0]), c.kv_lens, n_slots=2900)
        lo = 0 if g == 0 else 1500
        c.k.view(-1, 128)[slots[lo:lo + k.shape[0]].long()] = k
    c.q[:, :, 5] = 60.0
    check(ea, c)
    c.q[:, :, 5] = -60.0
    check(ea, c)


@pytest.mark.parametrize("m", [1, 60])
def test_keys_that_are_not_finite_behind_the_causal_border_do_not_matter(ea, m):
    c = make(ea, (8, 2, 128), 16, [m + 1], [[200, 300]])
    want = attend(ea, c, want_lse=True)
    slots, offsets = ea.ea_page_slots(c.ctx, c.shape, c.table, c.lens([199, 299]), c.kv_lens, n_slots=2)
    c.k.view(-1, 128)[slots.long()] = NAN                    # the last token's own keys: only the last token sees them
    got = attend(ea, c, want_lse=True)
    assert all(torch.equal(a[:m], b[:m]) for a, b in zip(want, got)) and bool(torch.isnan(got[0][m:]).all())


@pytest.mark.parametrize("heads,m", [((8, 2, 128), 1), ((4, 2, 64), 70), ((4, 2, 256), 70)])
def test_the_same_call_gives_the_same_bits(ea, heads, m):
    c = make(ea, heads, 16, [m] * 6, [[4000 + 100 * s, m + s] for s in range(6)])
    a = attend(ea, c, want_lse=True)
    for _ in range(3):
        b = attend(ea, c, want_lse=True)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("m", [1, 80])
def test_lengths_offsets_and_pages_that_do_not_fit_are_reported(ea, m):
    def fresh():
        return make(ea, (8, 2, 128), 16, [m, m, m], [[m + 60, m + 33], [m + 64, m + 64], [m + 9, m + 5]], stale=1.0)

    c = fresh()
    good = attend(ea, c, want_lse=True)
    rows = slice(2 * m, 3 * m)
    # the third sequence is served in every case; its key blocks may be split elsewhere when another list's length differs,
    # so it is held to the exact result and not to the bits of the good call
    exact = ref.attention(c.q, c.q_offsets, c.kv_lens, c.rows_of, c.d ** -0.5, True)
    tol_o, tol_l = ref.attention_tolerance(*exact, m + 64)
    for spoil in ("length", "negative", "offsets", "beyond", "page", "page low", "max_q"):
        c = fresh()
        out, lse = (torch.full_like(x, 7.0) for x in good)
        if spoil == "length":
            c.kv_lens[0, 0] = 16 * c.table.shape[2] + 1
        elif spoil == "negative":
            c.kv_lens[1, 1] = -5
        elif spoil == "offsets":
            c.q_offsets[1] = 3 * m + 2
        elif spoil == "beyond":
            c.q_offsets[0] = -1
        elif spoil == "page":
            c.table[0, 1, 1] = c.k.shape[0]
        elif spoil == "page low":
            c.table[1, 0, 0] = -7
        else:
            c.q_offsets[1] = 0                               # the second sequence now has 2 m tokens
        attend(ea, c, out=out, lse=lse)
        with pytest.raises(ea.EAError) as e:
            c.ctx.sync_status()
        assert e.value.status == 7, spoil
        assert bool(((out.double() - exact[0]).abs() <= tol_o)[rows].all()), spoil
        assert bool(((lse.double() - exact[1]).abs() <= tol_l)[rows].all()), spoil
        c.ctx.sync_status()


def test_an_empty_pool(ea):
    shape = ea.make_paged_shape(1, 2, 1, 64, 16, 0, 4)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape))
    q = torch.randn(1, 2, 64, device="cuda").to(torch.bfloat16)
    none = torch.empty(0, 16, 64, dtype=torch.bfloat16, device="cuda")
    args = (ctx, shape, q, i32([0, 1]), 1)
    out, lse = ea.ea_paged_attention(*args, i32([[0]]), i32([[[-1] * 4]]), none, none, want_lse=True)
    ctx.sync_status()
    assert not bool(out.any()) and bool((lse == -INF).all())
    ea.ea_paged_attention(*args, i32([[5]]), i32([[[0] * 4]]), none, none)
    with pytest.raises(ea.EAError):
        ctx.sync_status()


@pytest.mark.parametrize("m", [1, 64])
def test_pages_beyond_32_bit_offsets(ea, m):
    """Pools of more than 2^31 elements (4.3 GB each): the list sits on the last pages."""
    d, page = 128, 128
    n_pages = (1 << 31) // (page * d) + 40
    shape = ea.make_paged_shape(1, 8, 1, d, page, n_pages, 4)
    ctx = ea.Context(0, ea.ea_paged_workspace_bytes(shape, m))
    k, v = (torch.empty(n_pages, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = [torch.randn(400, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    table = i32([[[n_pages - 1, n_pages - 7, n_pages - 2, n_pages - 33]]])
    slots, _ = ea.ea_page_slots(ctx, shape, table, i32([[0]]), i32([[400]]), n_slots=400)
    ea.ea_page_store(ctx, shape, slots, *rows, k, v)
    got = ea.ea_page_load(ctx, shape, slots, k, v)
    assert all(torch.equal(a, b) for a, b in zip(got, rows))
    q = torch.randn(m, 8, d, generator=gen, device="cuda").to(torch.bfloat16)
    off, lens = i32([0, m]), i32([[400]])
    out, lse = ea.ea_paged_attention(ctx, shape, q, off, m, lens, table, k, v, want_lse=True)
    ctx.sync_status()
    exact = ref.attention(q, off, lens, lambda s, g: rows, d ** -0.5, True)
    tol_o, tol_l = ref.attention_tolerance(*exact, 400)
    assert bool(((out.double() - exact[0]).abs() <= tol_o).all()) and bool(((lse.double() - exact[1]).abs() <= tol_l).all())


def test_many_sequences_of_few_rows(ea):
    S = 700
    lens = [[(7 * s + 3 * g) % 19 for g in range(4)] for s in range(S)]
    check(ea, make(ea, (28, 4, 128), 16, [s % 3 for s in range(S)], lens))


@pytest.mark.parametrize("heads", [(4, 2, 64), (12, 3, 128), (4, 2, 256), (30, 2, 256)])
@pytest.mark.parametrize("page", [16, 128])
def test_many_short_lists_of_chunks(ea, heads, page):
    S, Hkv = 90, heads[1]
    chunks = [(5 * s) % 23 for s in range(S)]
    chunks[7] = 40
    lens = [[(31 * s + 77 * g) % 140 for g in range(Hkv)] for s in range(S)]
    check(ea, make(ea, heads, page, chunks, lens))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m", [17, 127, 128, 129, 255, 256, 257, 511, 513])
def test_rows_around_the_tiles(ea, d, m):
    for n in (m, 900):
        check(ea, make(ea, (2, 2, d), 64, [m, 3], [[n, m + 130], [5, 600]]))


@pytest.mark.parametrize("heads", [(5, 1, 64), (5, 1, 128), (5, 1, 256)])
@pytest.mark.parametrize("n", [700, 5000, 60000])
def test_few_lists_joined_from_many_parts(ea, heads, n):
    for m in (4, 30, 100):
        c = make(ea, heads, 64, [m], [[n]])
        out, lse = check(ea, c)
        for _ in range(5):                                   # in whatever order the parts arrive
            again = attend(ea, c, causal=True, want_lse=True)
            assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


# ---- as they are used ------------------------------------------------------------------------------------------------
def test_on_another_stream_and_with_a_workspace_that_is_too_small(ea):
    c = make(ea, (8, 2, 128), 16, [1, 1], [[200, 300], [40, 50]])
    want = attend(ea, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = attend(ea, c)
    side.synchronize()
    assert torch.equal(want, got)
    small = ea.Context(0, 16)
    with pytest.raises(ea.EAError) as e:
        ea.ea_paged_attention(small, c.shape, c.q, c.q_offsets, 1, c.kv_lens, c.table, c.k, c.v)
    assert e.value.status == 3


@pytest.mark.parametrize("first,second", [(((28, 4, 128), 1), ((4, 2, 256), 70)), (((8, 2, 128), 40), ((4, 2, 64), 200))])
def test_two_contexts_on_two_streams_do_not_disturb_each_other(ea, first, second):
    caches = [make(ea, heads, 32, [m, m], [[4000, 1500][:heads[1]] * (heads[1] // 2), [m + 9] * heads[1]], seed=i)
              for i, (heads, m) in enumerate((first, second))]
    alone = [attend(ea, c, want_lse=True) for c in caches]
    streams = [torch.cuda.Stream() for _ in caches]
    torch.cuda.synchronize()
    together = [[], []]
    for _ in range(20):
        for c, st, outs in zip(caches, streams, together):
            with torch.cuda.stream(st):
                outs.append(attend(ea, c, want_lse=True))
    torch.cuda.synchronize()
    for c, want, outs in zip(caches, alone, together):
        c.ctx.sync_status()
        for out, lse in outs:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_binding_refuses_what_does_not_fit(ea):
    c = make(ea, (8, 2, 128), 16, [1, 1], [[20, 30], [40, 50]])
    args = dict(q=c.q, q_offsets=c.q_offsets, max_q=1, kv_lens=c.kv_lens, block_table=c.table, k_pages=c.k, v_pages=c.v)
    for name, bad, error in [("q", c.q.float(), TypeError), ("q", c.q[:, :4], ValueError), ("q", c.q.transpose(0, 1), ValueError),
                             ("q", c.q[0], ValueError), ("q_offsets", c.q_offsets.long(), TypeError),
                             ("q_offsets", c.q_offsets[:2], ValueError), ("kv_lens", c.kv_lens.view(-1), ValueError),
                             ("block_table", c.table[:, :, :-1], (TypeError, ValueError)), ("k_pages", c.k[1:], ValueError),
                             ("v_pages", c.v.cpu(), TypeError), ("out", torch.empty_like(c.q).float(), TypeError),
                             ("lse", torch.empty(2, 4, device="cuda"), ValueError)]:
        with pytest.raises(error):
            ea.ea_paged_attention(c.ctx, c.shape, **{**args, name: bad})
    with pytest.raises(ValueError):
        ea.ea_page_store(c.ctx, c.shape, i32([0, 1]), c.q[:, :2, :], c.q[:1, :2, :], c.k, c.v)
    with pytest.raises(ValueError):
        ea.ea_page_slots(c.ctx, c.shape, c.table, c.kv_lens, c.kv_lens)
    with pytest.raises(ValueError):
        ea.ea_page_plan(c.ctx, c.shape, c.kv_lens, c.kv_lens, c.table, c.free[:-1], c.n_free)


@pytest.mark.parametrize("heads,m", [((8, 2, 128), 1), ((28, 4, 128), 3), ((4, 2, 64), 70), ((4, 2, 256), 70)])
def test_generation_steps_as_replays_of_one_graph(ea, heads, m):
    """plan, store and attention of one step captured once: lengths, tables and pages move on by themselves."""
    Hq, Hkv, d = heads
    S, page, steps = 3, 16, 6
    start = [[30, 47], [16, 1], [100, 15]]
    start = [(r * Hkv)[:Hkv] for r in start]
    c = make(ea, heads, page, [m] * S, start, spare=S * Hkv * (steps * m // page + 2), max_q=m)
    wide = max(n for r in start for n in r) // page + steps * m // page + 2
    c.shape = ea.make_paged_shape(S, Hq, Hkv, d, page, c.k.shape[0], wide)
    table = torch.full((S, Hkv, wide), -1, dtype=torch.int32, device="cuda")
    table[:, :, :c.table.shape[2]] = c.table
    lens, longer = c.kv_lens.clone(), torch.empty_like(c.kv_lens)
    q, kn, vn = (torch.zeros(S * m, h, d, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    slots, offsets = torch.empty(S * m * Hkv, dtype=torch.int32, device="cuda"), torch.empty(S + 1, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(S * m, Hq, device="cuda")

    def step():
        torch.add(lens, m, out=longer)
        ea.ea_page_plan(c.ctx, c.shape, lens, longer, table, c.free, c.n_free, order=ea.SLOTS_BY_TOKEN, slots=slots, offsets=offsets)
        ea.ea_page_store(c.ctx, c.shape, slots, kn, vn, c.k, c.v)
        ea.ea_paged_attention(c.ctx, c.shape, q, offsets, m, longer, table, c.k, c.v, out=out, lse=lse)
        lens.copy_(longer)

    saved = [x.clone() for x in (table, c.free, c.n_free, lens, c.k, c.v)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip((table, c.free, c.n_free, lens, c.k, c.v), saved):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((table, c.free, c.n_free, lens, c.k, c.v), saved):
        x.copy_(y)
    rows = {(s, g): [x.clone() for x in c.rows_of(s, g)] for s in range(S) for g in range(Hkv)}
    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(steps):
        for x in (q, kn, vn):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graph.replay()
        c.ctx.sync_status()
        for (s, g), pair in rows.items():
            for i, x in enumerate((kn, vn)):
                pair[i] = torch.cat([pair[i], x[s * m:(s + 1) * m, g]])
        exact = ref.attention(q, offsets, lens, lambda s, g: rows[s, g], d ** -0.5, True)
        tol_o, tol_l = ref.attention_tolerance(*exact, int(lens.max()))
        assert bool(((out.double() - exact[0]).abs() <= tol_o).all())
        assert bool(((lse.double() - exact[1]).abs() <= tol_l).all())
    held = table[table >= 0].tolist()
    assert len(set(held)) == len(held) and not set(held) & set(c.free[:c.n_free.item()].tolist())


def test_compressed_heads_paged_attended_grown_and_compressed_again(ea):
    """Head-adaptive compression of a prompt's cache, its ragged output into pages, generation over it, and the next
    compression event read back from the pages."""
    S, Hq, Hkv, d, n, W, n_kept, page = 2, 8, 2, 128, 512, 32, 192, 16
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)      # noqa: E731
    q_win, k, v = rnd(S, Hq, W, d), rnd(S, Hkv, n, d), rnd(S, Hkv, n, d)
    dense = ea.make_shape(S, Hq, Hkv, d, n, W)
    max_pages = ref.ceil_div(Hkv * n_kept + 64, page)
    paged = ea.make_paged_shape(S, Hq, Hkv, d, page, S * Hkv * max_pages, max_pages)
    ctx = ea.Context(0, max(ea.ea_workspace_bytes(dense), ea.ea_paged_workspace_bytes(paged, 1)))
    pos = torch.full((S,), n, dtype=torch.int64, device="cuda")
    mu, sigma = ea.ea_query_stats(ctx, dense, q_win, pos, 64, 1e6)
    scores = ea.ea_score(ctx, dense, k, v, mu, sigma, 0.02)
    idx, head_off, k_out, v_out = ea.ea_select_compact_adaptive(ctx, dense, scores, n_kept, ea.ea_n_floor(n_kept, 0.2), k, v)
    lens = (head_off[:, 1:] - head_off[:, :-1]).to(torch.int32).contiguous()
    assert int(lens.sum()) == S * Hkv * n_kept
    table = torch.full((S, Hkv, max_pages), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(S * Hkv * max_pages, dtype=torch.int32, device="cuda")
    n_free = i32([S * Hkv * max_pages])
    kp, vp = (torch.full((S * Hkv * max_pages, page, d), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zero = torch.zeros_like(lens)
    slots, offsets = ea.ea_page_plan(ctx, paged, zero, lens, table, free, n_free, n_slots=S * Hkv * n_kept)
    # the ragged rows lie in list order already
    ea.ea_page_store(ctx, paged, slots, k_out.view(-1, d), v_out.view(-1, d), kp, vp)
    rows = {}
    for s in range(S):
        for g in range(Hkv):
            a, b = int(head_off[s, g]), int(head_off[s, g + 1])
            rows[s, g] = [k_out[s, a:b], v_out[s, a:b]]
            assert torch.equal(rows[s, g][0], k[s, g][idx[s, a:b].long()])
    for _ in range(20):
        q, kn, vn = rnd(S, Hq, d), rnd(S, Hkv, d), rnd(S, Hkv, d)
        longer = lens + 1
        slots, q_off = ea.ea_page_plan(ctx, paged, lens, longer, table, free, n_free, n_slots=S * Hkv, order=ea.SLOTS_BY_TOKEN)
        ea.ea_page_store(ctx, paged, slots, kn, vn, kp, vp)
        lens = longer
        out, lse = ea.ea_paged_attention(ctx, paged, q, q_off, 1, lens, table, kp, vp, want_lse=True)
        for (s, g), pair in rows.items():
            pair[0], pair[1] = torch.cat([pair[0], kn[s, g][None]]), torch.cat([pair[1], vn[s, g][None]])
    ctx.sync_status()
    exact = ref.attention(q, q_off, lens, lambda s, g: rows[s, g], d ** -0.5, True)
    tol_o, tol_l = ref.attention_tolerance(*exact, int(lens.max()))
    assert bool(((out.double() - exact[0]).abs() <= tol_o).all()) and bool(((lse.double() - exact[1]).abs() <= tol_l).all())
    # the next event: one head's rows out of their pages, scored and compacted, pages given back
    total = int(lens.sum())
    slots, offsets = ea.ea_page_slots(ctx, paged, table, zero, lens, n_slots=total)
    kd, vd = ea.ea_page_load(ctx, paged, slots, kp, vp)
    for i, ((s, g), pair) in enumerate(sorted(rows.items())):
        a, b = int(offsets[i]), int(offsets[i + 1])
        assert torch.equal(kd[a:b], pair[0]) and torch.equal(vd[a:b], pair[1])
    before = n_free.item()
    ea.ea_page_plan(ctx, paged, lens, lens // 2, table, free, n_free)
    ctx.sync_status()
    pages = lambda x: int(((x + page - 1) // page).sum())      # noqa: E731
    assert n_free.item() - before == pages(lens) - pages(lens // 2)


def test_a_paged_call_ends_a_fused_operand(ea):
    """Fused statistics leave their operand in the workspace that the paged calls use too."""
    S, Hq, Hkv, d, n, W = 1, 8, 2, 128, 256, 32
    q, k, v = (torch.randn(*x, device="cuda").to(torch.bfloat16) for x in ((S, Hq, W, d), (S, Hkv, n, d), (S, Hkv, n, d)))
    dense = ea.make_shape(S, Hq, Hkv, d, n, W)
    c = make(ea, (8, 2, 128), 16, [1], [[20, 30]])
    ctx = ea.Context(0, max(ea.ea_workspace_bytes(dense), ea.ea_paged_workspace_bytes(c.shape)))
    ctx.set_fused_stats(True)
    ea.ea_query_stats(ctx, dense, q, torch.full((S,), n, dtype=torch.int64, device="cuda"), 64, 1e6)
    ea.ea_score(ctx, dense, k, v, None, None, 0.02)
    c.ctx = ctx
    attend(ea, c)
    with pytest.raises(ea.EAError) as e:
        ea.ea_score(ctx, dense, k, v, None, None, 0.02)
    assert e.value.status == 1
