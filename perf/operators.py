"""Cases for the paged-cache operators, with their plain forms.

A paged cache holds the pairs of every (sequence, KV head), a *list*, in pages of `page` rows: `k_pages`, `v_pages`
bf16 [n_pages, page, d].  Row `p` of a list lies in slot `block_table[list, p // page] * page + p % page`.  After
head-adaptive eviction the heads of one sequence hold different numbers of pairs, so lengths and tables are kept per list.

  plan    block tables and slot maps from lengths: the lists' pages are taken from a free list (or given back to it) and
          the slots of the new rows are written down.  One pass is a growth and its undoing.
  slots   the slots of given ranges of rows, from tables that stand
  store   new rows into their slots
  load    rows out of their slots
  attention   a chunk of new tokens (or one token) per sequence over the pairs of its lists

`run` computes them in elementary torch operations, or with `own` set through the library.
"""
import math

import numpy as np
import torch

own = False

BY_LIST, BY_TOKEN = 0, 1
HEADS = ((4, 2, 64), (32, 8, 128), (16, 8, 256), (28, 4, 128))     # query heads, KV heads, head dimension


def listed():
    return [
        # one generated token in 28 layers of 8 sequences: a growth by one row per list, most of them inside a page
        dict(name="plan one token", op="plan", seqs=224, kv_heads=4, page=16, keys=4607, grow=1, ragged=True),
        # 48 layers admitted after a head-adaptive prefill compression: every list from nothing to its length
        dict(name="plan admission", op="plan", seqs=48, kv_heads=8, page=64, keys=16384, grow=0, ragged=True),
        # all rows of one layer of one sequence, read back before its compression
        dict(name="slots one layer", op="slots", seqs=1, kv_heads=8, page=16, keys=4608, ragged=False),
        # the same for a 36-layer model with a ragged cache
        dict(name="slots 36 layers", op="slots", seqs=36, kv_heads=8, page=32, keys=8192, ragged=True),
        # the new token of 8 sequences in one layer: rows in token order, as the projection leaves them
        dict(name="store one token", op="store", seqs=8, q_heads=28, kv_heads=4, dim=128, page=16, keys=4608, grow=1, ragged=True),
        # compacted rows of 4 layers after a prefill compression at head dimension 256
        dict(name="store compacted", op="store", seqs=4, q_heads=16, kv_heads=8, dim=256, page=64, keys=16384, grow=0, ragged=True),
        # one layer of one sequence out of its pages
        dict(name="load one layer", op="load", seqs=1, q_heads=32, kv_heads=8, dim=128, page=16, keys=4608, ragged=True),
        # seven layers of 8 sequences before a compression event
        dict(name="load 7 layers", op="load", seqs=56, q_heads=28, kv_heads=4, dim=128, page=16, keys=4608, ragged=False),
        # a single stream's next token over a compressed cache: latency
        dict(name="attention one token", op="attention", seqs=1, q_heads=32, kv_heads=8, dim=128, page=16, keys=4096, chunk=1, ragged=False, causal=True),
        # the next token of 32 sequences with a head-adaptive cache, seven query heads per KV head: bandwidth
        dict(name="attention 32 streams", op="attention", seqs=32, q_heads=28, kv_heads=4, dim=128, page=16, keys=16384, chunk=1, ragged=True, causal=True),
        # a mixed step: a chunk of a prompt beside a decoding sequence and a short chunk, head dimension 256
        dict(name="attention mixed", op="attention", seqs=3, q_heads=16, kv_heads=8, dim=256, page=64, keys=16896, chunk=517, ragged=True, causal=True),
        # a prompt's next chunk late in a long context: tensor throughput
        dict(name="attention chunk", op="attention", seqs=1, q_heads=32, kv_heads=8, dim=128, page=64, keys=32768, chunk=2048, ragged=False, causal=True),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("plan", "slots", "store", "load", "attention", "attention", "attention"))
    Hq, Hkv, d = rng.choice(HEADS)
    page = rng.choice((16, 32, 64, 128))
    ragged = rng.random() < 0.6
    if op in ("plan", "slots"):
        seqs = _log(rng, 1, 224)
        keys = _log(rng, 1, min(16384, 6_000_000 // (seqs * Hkv)))
        case = dict(op=op, seqs=seqs, kv_heads=Hkv, page=page, keys=keys, ragged=ragged)
        if op == "plan":
            case["grow"] = rng.choice((0, 1, _log(rng, 1, 200)))
        return case
    if op in ("store", "load"):
        seqs = _log(rng, 1, 56)
        keys = _log(rng, 1, min(16384, 500_000 * 256 // d // (seqs * Hkv)))
        case = dict(op=op, seqs=seqs, q_heads=Hq, kv_heads=Hkv, dim=d, page=page, keys=keys, ragged=ragged)
        if op == "store":
            case["grow"] = rng.choice((0, 1, _log(rng, 1, 200)))
        return case
    chunk = rng.choice((1, 1, _log(rng, 2, 16), _log(rng, 2, 2048)))
    keys = _log(rng, chunk, 131072)
    fits = min(2048 * 32768 * 32 * 128 // (chunk * keys * Hq * d), (1 << 30) // (keys * Hkv * d))
    while fits < 1:
        keys = max(chunk, keys // 2)
        fits = min(2048 * 32768 * 32 * 128 // (chunk * keys * Hq * d), (1 << 30) // (keys * Hkv * d))
    return dict(op="attention", seqs=_log(rng, 1, min(64, fits)), q_heads=Hq, kv_heads=Hkv, dim=d, page=page, keys=keys, chunk=chunk,
                ragged=ragged, causal=rng.random() < 0.8)


def _chunks(case):
    """New tokens of each sequence: all of them in the first, fewer in the others of a ragged batch."""
    m, n = case["chunk"], case["seqs"]
    return [max(1, m - int(((s * 0.6180339887) % 1.0) * m)) if case["ragged"] else m for s in range(n)]


def _lengths(case):
    """Rows of each list [seqs][kv_heads]: the same everywhere, or (ragged) between a quarter and all of `keys`."""
    rows, floor = [], _chunks(case) if "chunk" in case else [1] * case["seqs"]
    for s in range(case["seqs"]):
        part = [((s * case["kv_heads"] + g) * 0.6180339887) % 1.0 for g in range(case["kv_heads"])]
        rows.append([max(floor[s], case["keys"] - (int(0.75 * f * case["keys"]) if case["ragged"] else 0)) for f in part])
    return rows


def _ranges(case):
    """(first, end) row of each list that the case writes: the last `grow` rows, or all of them where `grow` is 0."""
    end = [n + case.get("grow", 0) for r in _lengths(case) for n in r]
    first = [n - case.get("grow", 0) for n in end] if case.get("grow", 0) else [0] * len(end)
    return first, end


def _ceil(a, b):
    return -(-a // b)


def work(case):
    lists, page = case["seqs"] * case["kv_heads"], case["page"]
    if case["op"] == "attention":
        d, Hq, G = case["dim"], case["q_heads"], case["q_heads"] // case["kv_heads"]
        pairs = rows = pages = 0
        for m, lens in zip(_chunks(case), _lengths(case)):
            for n in lens:
                pairs += G * (m * n - (m * (m - 1) // 2 if case["causal"] else 0))
                rows += n
                pages += _ceil(n, page)
        tokens = sum(_chunks(case))
        return {"bytes": rows * d * 4 + tokens * Hq * (d * 4 + 4) + pages * 4 + lists * 4, "flops": 4 * pairs * d}
    first, end = _ranges(case)
    rows = sum(e - f for f, e in zip(first, end))
    if case["op"] == "plan":
        new = sum(_ceil(e, page) - _ceil(f, page) for f, e in zip(first, end))
        held = sum(_ceil(e, page) - f // page for f, e in zip(first, end) if e > f)      # table entries that the slots need
        # the growth reads the lengths, the entries of pages begun before and the free pages, and writes entries and slots;
        # the undoing reads the lengths and the entries, and writes the entries and the free list
        return {"bytes": 4 * (2 * lists + held - new + 2 * new + rows + lists + 2 * lists + 3 * new), "flops": rows}
    if case["op"] == "slots":
        held = sum(_ceil(e, page) - f // page for f, e in zip(first, end) if e > f)
        return {"bytes": 4 * (2 * lists + held + rows + lists), "flops": 2 * rows}
    return {"bytes": rows * (case["dim"] * 8 + 4), "flops": rows}


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    S, Hkv, page = case["seqs"], case["kv_heads"], case["page"]
    lens = _lengths(case)
    first, end = _ranges(case)
    held = [n for r in lens for n in r] if case["op"] != "plan" else first
    held = end if case["op"] in ("store", "slots", "load") else held
    have = torch.tensor([_ceil(n, page) for n in held], device=dev)
    columns = max(_ceil(n, page) for n in end) if case["op"] != "attention" else max(_ceil(n, page) for r in lens for n in r)
    total = sum(_ceil(max(a, b), page) for a, b in zip(held, end))
    pages = total + 64
    # the pages of a list lie anywhere in the pool, as after a while of taking and giving back
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    at = torch.cumsum(have, 0) - have
    col = torch.arange(columns, device=dev)
    mine = col[None, :] < have[:, None]
    table = torch.where(mine, order[(at[:, None] + col[None, :]).clamp(max=pages - 1)], -1).to(torch.int32).view(S, Hkv, columns)
    used = int(have.sum())
    st = dict(case=dict(case), page=page, table=table, pages=pages, columns=columns,
              first=torch.tensor(first, dtype=torch.int32, device=dev).view(S, Hkv),
              end=torch.tensor(end, dtype=torch.int32, device=dev).view(S, Hkv))
    step = case.get("grow", 0) > 0
    st["order"] = BY_TOKEN if step else BY_LIST
    st["n_slots"] = sum(e - f for f, e in zip(first, end))
    if case["op"] == "plan":
        st["free"] = torch.cat([order[used:], torch.full((used,), -1, dtype=torch.int32, device=dev)])
        st["n_free"] = torch.tensor([pages - used], dtype=torch.int32, device=dev)
    if case["op"] in ("store", "load", "attention"):
        d = case["dim"]
        st["k_pages"] = torch.empty(pages, page, d, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
        st["v_pages"] = torch.empty(pages, page, d, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
    if case["op"] in ("store", "load"):
        st["slots"] = _slots(st)[0]
        if case["op"] == "store":
            st["k_new"] = torch.empty(st["n_slots"], d, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
            st["v_new"] = torch.empty(st["n_slots"], d, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
    if case["op"] == "attention":
        # keys and queries share a few outlier channels and have offsets per channel, values a scale per row
        chunks = _chunks(case)
        T, Hq = sum(chunks), case["q_heads"]
        big = torch.ones(d, device=dev)
        big[torch.randperm(d, generator=gen, device=dev)[:2]] = 4.0
        off = 0.5 * torch.randn(d, generator=gen, device=dev)
        st["k_pages"].add_(off).mul_(big)
        st["v_pages"].mul_(torch.exp(0.5 * torch.randn(pages, page, 1, generator=gen, device=dev)))
        q = torch.randn(T, Hq, d, generator=gen, device=dev) + 0.5 * torch.randn(Hq, d, generator=gen, device=dev)
        st["q"] = (q * big).to(torch.bfloat16)
        st["q_offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32, device=dev)
        st["kv_lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        st["max_q"] = max(chunks)
        st["scale"] = 1.0 / math.sqrt(d)
    if own:
        from paper_2510_00636_b200 import binding as ea
        st["ea"] = ea
        st["shape"] = ea.make_paged_shape(S, case.get("q_heads", Hkv), Hkv, case.get("dim", 128), page, pages, columns)
        st["ctx"] = ea.Context(0, ea.ea_paged_workspace_bytes(st["shape"], st["max_q"] if case["op"] == "attention" else 1))
    return st


# ---- the plain forms -----------------------------------------------------------------------------------------------
def _slots(st, table=None):
    """Slots of rows first .. end of every list, and where each list's (or sequence's) begin."""
    table = st["table"] if table is None else table
    page, first = st["page"], st["first"].long().flatten()
    n = st["end"].long().flatten() - first
    S, Hkv = st["first"].shape
    t = torch.arange(st["n_slots"], device=first.device)
    if st["order"] == BY_TOKEN:
        offsets = torch.cat([n.new_zeros(1), torch.cumsum(n.view(S, Hkv)[:, 0], 0)])
        token, head = t // Hkv, t % Hkv
        s = torch.searchsorted(offsets, token, right=True) - 1
        r, j = s * Hkv + head, token - offsets[s]
    else:
        offsets = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)])
        r = torch.searchsorted(offsets, t, right=True) - 1
        j = t - offsets[r]
    p = first[r] + j
    slots = table.view(S * Hkv, -1).long()[r, p // page] * page + p % page
    return slots.to(torch.int32), offsets.to(torch.int32)


def _plan(st, old, new, table, free, n_free):
    """Pages after the lengths change from `old` to `new`: (table, free, n_free)."""
    page, pages, columns = st["page"], st["pages"], st["columns"]
    have, want = ((x.long().flatten()[:, None] + page - 1) // page for x in (old, new))
    col = torch.arange(columns, device=old.device)
    take = ((col >= have) & (col < want)).flatten()
    give = ((col >= want) & (col < have)).flatten().flip(0)             # last list first, last page first
    flat, top = table.flatten().long(), n_free.long()
    n_take, n_give = take.sum(), give.sum()
    k = torch.cumsum(give, 0) - 1
    given = flat.new_zeros(pages + 1).scatter_(0, torch.where(give, k, pages), flat.flip(0))
    i = torch.cumsum(take, 0) - 1
    fresh = free.long()[(top - 1 - (i - n_give)).clamp(0, pages - 1)]
    page_of = torch.where(i < n_give, given[i.clamp(0, pages)], fresh)
    table = torch.where(take, page_of, torch.where(give.flip(0), -1, flat)).to(torch.int32).view_as(table)
    k = torch.arange(pages + 1, device=old.device)
    back = (k >= n_take) & (k < n_give)
    free = torch.cat([free.long(), top]).scatter_(0, torch.where(back, top + k - n_take, pages).clamp(max=pages), given)[:pages]
    return table, free.to(torch.int32), (top - n_take + n_give).to(torch.int32)


def _attention(st):
    case = st["case"]
    S, Hkv, Hq, d = case["seqs"], case["kv_heads"], case["q_heads"], case["dim"]
    G, m, T = Hq // Hkv, st["max_q"], st["q"].shape[0]
    off, lens = st["q_offsets"].long(), st["kv_lens"].long()
    n = off[1:] - off[:-1]
    i = torch.arange(m, device=off.device)
    token = (off[:-1, None] + i).clamp(max=T - 1)                                              # [S, m]
    q = st["q"].float()[token].view(S, m, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(S, Hkv, m * G, d)
    at = st["table"].long().clamp(min=0)
    k = st["k_pages"][at].view(S, Hkv, -1, d).float()
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(st["scale"])
    del k
    pos = torch.arange(p.shape[-1], device=off.device)
    limit = lens[:, :, None].expand(S, Hkv, m)
    if case["causal"]:
        limit = torch.minimum(limit, lens[:, :, None] - n[:, None, None] + i + 1)
    limit = limit.repeat_interleave(G, -1)
    p.masked_fill_(pos >= limit[..., None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = st["v_pages"][at].view(S, Hkv, -1, d).float()
    v = torch.where((pos < lens[:, :, None])[..., None], v, 0.0)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    o = o.view(S, Hkv, m, G, d).permute(0, 2, 1, 3, 4).reshape(S * m, Hq, d)
    lse = lse.view(S, Hkv, m, G).permute(0, 2, 1, 3).reshape(S * m, Hq)
    t = torch.arange(T, device=off.device)
    s = torch.searchsorted(off, t, right=True) - 1
    at = s * m + t - off[s]
    return {"out": o[at].to(torch.bfloat16), "lse": lse[at]}


def run(st):
    op = st["case"]["op"]
    if own:
        return _run_own(st, op)
    if op == "plan":
        table, free, n_free = _plan(st, st["first"], st["end"], st["table"], st["free"], st["n_free"])
        slots, offsets = _slots(st, table)
        table, free, n_free = _plan(st, st["end"], st["first"], table, free, n_free)
        return {"slots": slots, "offsets": offsets, "table": table, "free": free, "n_free": n_free}
    if op == "slots":
        return dict(zip(("slots", "offsets"), _slots(st)))
    if op == "store":
        for pool, rows in ((st["k_pages"], st["k_new"]), (st["v_pages"], st["v_new"])):
            pool.view(-1, pool.shape[-1])[st["slots"].long()] = rows
        return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if op == "load":
        return {"k": st["k_pages"].view(-1, st["k_pages"].shape[-1])[st["slots"].long()],
                "v": st["v_pages"].view(-1, st["v_pages"].shape[-1])[st["slots"].long()]}
    return _attention(st)


def _run_own(st, op):
    ea, ctx, shape = st["ea"], st["ctx"], st["shape"]
    if op == "plan":
        slots, offsets = ea.ea_page_plan(ctx, shape, st["first"], st["end"], st["table"], st["free"], st["n_free"],
                                         n_slots=st["n_slots"], order=st["order"])
        ea.ea_page_plan(ctx, shape, st["end"], st["first"], st["table"], st["free"], st["n_free"])
        return {"slots": slots, "offsets": offsets, "table": st["table"], "free": st["free"], "n_free": st["n_free"]}
    if op == "slots":
        slots, offsets = ea.ea_page_slots(ctx, shape, st["table"], st["first"], st["end"], n_slots=st["n_slots"], order=st["order"])
        return {"slots": slots, "offsets": offsets}
    if op == "store":
        ea.ea_page_store(ctx, shape, st["slots"], st["k_new"], st["v_new"], st["k_pages"], st["v_pages"])
        return {"k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if op == "load":
        k, v = ea.ea_page_load(ctx, shape, st["slots"], st["k_pages"], st["v_pages"])
        return {"k": k, "v": v}
    out, lse = ea.ea_paged_attention(ctx, shape, st["q"], st["q_offsets"], st["max_q"], st["kv_lens"], st["table"],
                                     st["k_pages"], st["v_pages"], scale=st["scale"], causal=st["case"]["causal"], want_lse=True)
    return {"out": out, "lse": lse}


# ---- the definitions, in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("store", "load"):
        return None                                     # copies: nothing is computed
    st = prepare(case, seed)
    if case["op"] in ("plan", "slots"):
        return _exact_pages(case, st)
    chunks, lens = _chunks(case), _lengths(case)
    Hq, Hkv, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    G, T = Hq // Hkv, sum(chunks)
    out = torch.zeros(T, Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    begin = 0
    for s, m in enumerate(chunks):
        for g in range(Hkv):
            n = lens[s][g]
            ids = st["table"][s, g, :_ceil(n, page)].long()
            k = st["k_pages"][ids].reshape(-1, d)[:n].double()
            v = st["v_pages"][ids].reshape(-1, d)[:n].double()
            for a in range(0, m, 256):                  # in pieces of the chunk, to bound the memory
                b = min(m, a + 256)
                seen = torch.arange(n, device="cuda")[None, :] <= torch.arange(n - m + a, n - m + b, device="cuda")[:, None]
                for h in range(g * G, (g + 1) * G):
                    x = st["scale"] * (st["q"][begin + a:begin + b, h].double() @ k.T)
                    if case["causal"]:
                        x = torch.where(seen, x, -math.inf)
                    lse[begin + a:begin + b, h] = torch.logsumexp(x, -1)
                    out[begin + a:begin + b, h] = torch.softmax(x, -1) @ v
        begin += m
    return {"out": out, "lse": lse}


def _exact_pages(case, st):
    page, Hkv = case["page"], case["kv_heads"]
    first, end = _ranges(case)
    table = st["table"].cpu().numpy().reshape(len(first), -1).copy()
    if case["op"] == "plan":
        free = st["free"].cpu().numpy().copy()
        top = int(st["n_free"])
        for r, (f, e) in enumerate(zip(first, end)):
            for c in range(_ceil(f, page), _ceil(e, page)):
                top -= 1
                table[r, c] = free[top]
    rows = []
    for r, (f, e) in enumerate(zip(first, end)):
        p = np.arange(f, e)
        rows.append(table[r, p // page] * page + p % page)
    if st["order"] == BY_TOKEN:                         # the heads of a token side by side
        slots = np.concatenate([np.stack(rows[r:r + Hkv], 1).reshape(-1) for r in range(0, len(rows), Hkv)])
        sizes = [len(rows[r]) for r in range(0, len(rows), Hkv)]
    else:
        slots, sizes = np.concatenate(rows), [len(x) for x in rows]
    answer = {"slots": slots.astype(np.int32), "offsets": np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)}
    if case["op"] == "plan":                            # undone: as before
        answer |= {"table": st["table"], "free": st["free"], "n_free": st["n_free"]}
    return answer
