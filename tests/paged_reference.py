"""Plain statements of the paged-cache operators for the tests: page bookkeeping in Python, attention in 64 bits."""
import math

import torch


def ceil_div(a, b):
    return -(-a // b)


class Pages:
    """Tables and free list as Python lists; ``resize`` is the rule of ``ea_page_plan``, one page at a time."""

    def __init__(self, lists, max_pages, n_pages, page):
        self.table = [[-1] * max_pages for _ in range(lists)]
        self.free = list(range(n_pages))
        self.page, self.n_free = page, n_pages

    def resize(self, old, new):
        have, want = [ceil_div(n, self.page) for n in old], [ceil_div(n, self.page) for n in new]
        takes = [(r, c) for r in range(len(old)) for c in range(have[r], want[r])]
        gives = [(r, c) for r in reversed(range(len(old))) for c in reversed(range(want[r], have[r]))]
        if len(takes) - len(gives) > self.n_free:
            return False
        given = []
        for r, c in gives:
            given.append(self.table[r][c])
            self.table[r][c] = -1
        for i, (r, c) in enumerate(takes):
            if i < len(given):
                self.table[r][c] = given[i]
            else:
                self.n_free -= 1
                self.table[r][c] = self.free[self.n_free]
        for x in given[len(takes):]:
            self.free[self.n_free] = x
            self.n_free += 1
        return True

    def slots(self, first, end, kv_heads=None):
        """By list, or by token with ``kv_heads``: (slots, offsets)."""
        per = [[self.table[r][p // self.page] * self.page + p % self.page for p in range(f, e)]
               for r, (f, e) in enumerate(zip(first, end))]
        out, offsets = [], [0]
        if kv_heads is None:
            for x in per:
                out += x
                offsets.append(len(out))
            return out, offsets
        for r in range(0, len(per), kv_heads):
            for j in range(len(per[r])):
                out += [per[r + g][j] for g in range(kv_heads)]
            offsets.append(len(out) // kv_heads)
        return out, offsets


def attention(q, q_offsets, kv_lens, rows_of, scale, causal):
    """q bf16 [T,Hq,d]; ``rows_of(s, g)`` -> (k, v) bf16 [n,d] of a list.  Per head: out and lse in 64 bits, the mean of |v|
    under the weights (what a relative error of the weights acts on) and the largest sum of |q_c k_c| of a visible score."""
    T, Hq, d = q.shape
    S, Hkv = kv_lens.shape
    G = Hq // Hkv
    out = torch.zeros(T, Hq, d, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    terms = torch.zeros(T, Hq, dtype=torch.float64, device=q.device)
    for s in range(S):
        a, b = int(q_offsets[s]), int(q_offsets[s + 1])
        m = b - a
        for g in range(Hkv):
            n = int(kv_lens[s, g])
            if n == 0 or m == 0:
                continue
            k, v = (x.double() for x in rows_of(s, g))
            x = q[a:b, g * G:(g + 1) * G].double()                                   # [m, G, d]
            y = scale * torch.einsum("mgd,nd->mgn", x, k)
            seen = torch.ones(m, n, dtype=torch.bool, device=q.device)
            if causal:
                seen = torch.arange(n, device=q.device)[None] <= torch.arange(m, device=q.device)[:, None] + n - m
            y = y.masked_fill(~seen[:, None], -math.inf)
            top = y.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            p = torch.exp(y - top)
            total = p.sum(-1, keepdim=True)
            w = p / torch.where(total == 0, 1.0, total)
            out[a:b, g * G:(g + 1) * G] = torch.einsum("mgn,nd->mgd", w, v)
            mag[a:b, g * G:(g + 1) * G] = torch.einsum("mgn,nd->mgd", w, v.abs())
            lse[a:b, g * G:(g + 1) * G] = (top + torch.log(total))[..., 0]
            t = abs(scale) * torch.einsum("mgd,nd->mgn", x.abs(), k.abs())
            terms[a:b, g * G:(g + 1) * G] = t.masked_fill(~seen[:, None], 0.0).amax(-1)
    return out, lse, mag, terms


def attention_tolerance(out, lse, mag, terms, n):
    """Bounds on |out - exact| and |lse - exact|.

    A score is an fp32 sum of exact products: off by at most delta = 2^-20 of the sum of their magnitudes (the accumulation
    order of the tensor cores is not specified; 2^-20 leaves 16 units of the last place for it), and its exponential by
    2^-21 more (the hardware's 2^x and the product with log2 e).  Every weight is then rounded to bf16, off by 2^-8 of itself
    (half a step), while the sum that divides keeps 32 bits: n additions of 2^-24, at most n / 16 of them one after the
    other.  So out is off by (2^-8 + 2 (delta + 2^-21) + n 2^-28 + 2^-20) * mean|v| and half a step of its own rounding, and
    lse by delta + 2^-21 + n 2^-28 and the rounding of its value.
    """
    delta = terms * 2.0 ** -20
    add = n * 2.0 ** -28
    o = (2.0 ** -8 + 2 * (delta + 2.0 ** -21) + add + 2.0 ** -20)[..., None] * mag + 2.0 ** -8 * out.abs() + 1e-30
    finite = torch.where(torch.isinf(lse), 0.0, lse)
    return o, delta + 2.0 ** -21 + add + 2.0 ** -20 * (1 + finite.abs())
