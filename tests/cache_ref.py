"""The paged cache and attention over it in 64 bits, one sequence and one token at a time, with the bounds its tests use."""
import math

import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def quantise(x):
    """(codes of the type as float64 values, fp32 scales) for rows x [..., d] bf16, by the definition; dtype -> codes."""
    def to(dtype):
        scale = (x.double().abs().amax(-1) / TOP[dtype]).float()          # one rounding to 32 bits
        y = torch.zeros(x.shape, dtype=torch.float64)
        live = scale > 0
        y[live] = (x.double()[live] / scale.double()[live][:, None]).float().double().clamp(-TOP[dtype], TOP[dtype])
        if dtype is torch.int8:
            return torch.round(y), scale
        _, e = torch.frexp(y)
        step = torch.pow(2.0, (e.double() - 4).clamp(min=-9))
        return torch.round(y / step) * step, scale
    return to


class Ref:
    """A cache on the CPU, float64 values with holes where nothing was written, and the batch's lists."""

    def __init__(self, n_pages, page, heads, dim, dtype):
        self.page, self.heads, self.dim, self.dtype, self.n_pages = page, heads, dim, dtype, n_pages
        self.code = [torch.zeros(n_pages, page, heads, dim, dtype=torch.float64) for _ in "kv"]
        self.scale = [torch.ones(n_pages, page, heads) for _ in "kv"]

    def place(self, table, pos):
        j = pos // self.page
        if pos < 0 or j >= len(table) or not 0 <= table[j] < self.n_pages:
            return None
        return table[j], pos % self.page

    def write(self, cu, lens, tables, k, v):
        """Returns the places that were written."""
        done = []
        for s in range(len(lens)):
            n = cu[s + 1] - cu[s]
            for i in range(n):
                at = self.place(tables[s], lens[s] - n + i)
                if at is None:
                    continue
                done.append(at)
                for c, x in enumerate((k, v)):
                    row = x[cu[s] + i]
                    if self.dtype is torch.bfloat16:
                        self.code[c][at] = row.double()
                    else:
                        self.code[c][at], self.scale[c][at] = quantise(row)(self.dtype)
        return done

    def held(self, s, lens, tables):
        """Positions with a key, and their K and V [n, heads, dim] in 64 bits."""
        at = [(p, self.place(tables[s], p)) for p in range(max(0, lens[s]))]
        at = [(p, x) for p, x in at if x is not None]
        if not at:
            none = torch.zeros(0, self.heads, self.dim, dtype=torch.float64)
            return torch.zeros(0, dtype=torch.long), none, none
        pg, in_page = (torch.tensor([x[i] for _, x in at]) for i in range(2))
        got = []
        for c in range(2):
            x = self.code[c][pg, in_page]
            got.append(x if self.dtype is torch.bfloat16 else x * self.scale[c][pg, in_page].double()[..., None])
        return torch.tensor([p for p, _ in at]), got[0], got[1]


def attention(ref, cu, lens, tables, prefix, q, scale):
    """(O, LSE, bound of O, bound of LSE); rows of no sequence are NaN.

    Bounds, for O_c = sum_j p_j v_jc and A_c = sum_j p_j |v_jc|.  P is rounded to bf16 once before its product (in 8 bits together
    with the value's scale) and O once at the end: 2^-8 of A and of O.  A score is a sum of d products in 32 bits: d roundings
    of at most 2^-23 (the tensor core may cut instead of rounding) of M = scale * sum |q||k|, and three roundings of the
    factors, (d + 4) 2^-23 M; e^x of it carries that and 2^-21 (argument and exponential) as a relative error, as does the row
    sum; sums of n weights in 32 bits add n 2^-24 / 16 (a warp or a thread never has more than a sixteenth of them in one chain,
    but short rows have: n at most 16) and joins of parts some 2^-20.  LSE carries the errors of the largest score and of the sum
    and three roundings of its own."""
    H = q.shape[1]
    O = torch.full(q.shape, math.nan, dtype=torch.float64)
    L = torch.full((H, q.shape[0]), math.nan, dtype=torch.float64)
    bo, bl = torch.zeros_like(O), torch.zeros_like(L)
    for s in range(len(lens)):
        n = cu[s + 1] - cu[s]
        if n <= 0:
            continue
        pos, K, V = ref.held(s, lens, tables)
        qs = q[cu[s]:cu[s + 1]].double()
        own = lens[s] - n + torch.arange(n)
        seen = (pos[None, :] <= own[:, None]) | (pos < (prefix[s] if prefix is not None else 0))[None, :]
        for h in range(H):
            g = h * ref.heads // H
            x = (qs[:, h] @ K[:, g].T) * scale
            m = (qs[:, h].abs() @ K[:, g].abs().T) * scale
            x = x.masked_fill(~seen, -math.inf)
            some = seen.any(1)
            lse = torch.full((n,), -math.inf, dtype=torch.float64)
            lse[some] = torch.logsumexp(x[some], 1)
            p = torch.zeros_like(x)
            p[some] = torch.exp(x[some] - lse[some][:, None])
            o, a = p @ V[:, g], p @ V[:, g].abs()
            big = (m * seen).amax(1) if len(pos) else torch.zeros(n, dtype=torch.float64)
            rel = 2 * (ref.dim + 4) * 2.0 ** -23 * big + 2.0 ** -20 + (16 + len(pos) / 16) * 2.0 ** -24
            O[cu[s]:cu[s + 1], h], L[h, cu[s]:cu[s + 1]] = o, lse
            bo[cu[s]:cu[s + 1], h] = (2.0 ** -8 * (a + o.abs()) * (1 + 2.0 ** -7)) + rel[:, None] * (a + o.abs()) + 1e-37
            bl[h, cu[s]:cu[s + 1]] = rel + 2.0 ** -21 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2.0 ** -22
    return O, L, bo, bl
