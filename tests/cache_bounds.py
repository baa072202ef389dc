"""Attention over an 8-bit cache in 64 bits, with bounds that follow what is kept in which type.

A key holds codes c (whole numbers or e4m3) times a scale a, a value codes w times a scale b.  For a row with
s_j = scale a_j sum_i q_i c_ji, p_j = e^s_j / sum e^s, A = sum p_j b_j |w_j|:

* q goes to fp16 times a power of two that brings Q, the largest magnitude among the rows that are multiplied together, to 2^14 .. 2^15
  (from 2^-98 on; below, times 2^112, where no bit of bf16 is lost).  bf16 has 8 bits and fp16 11, so only what falls below fp16's
  step of 2^-24 is rounded: by at most 2^-25, which is 2^-39 of 2^14.  A score is off by 2^-39 scale Q a_j sum_i |c_ji|.  (Rows multiplied together: at most those of a sequence
  that share a key head.)
* codes are exact in fp16, products of the two in 32 bits; the sum has d roundings of 2^-23 (a tensor core may cut) of
  M_j = scale a_j sum_i |q_i c_ji|, the factors four more.
* log2 b_j is added to the score (one unit of 2^-23), the sum rounded twice: with G the largest |s_j| log2 e + |log2 b_j|, less
  than 2^-21 G in powers of two, times ln 2 as a relative error of the weight.  The exponential itself: 2^-22, sums as in cache_ref.
* a weight p_j b_j is rounded to fp16 relative to a reference that is at most the largest of the row's: by 2^-11 of itself, or
  2^-25 of the largest where fp16 is at its last step.
* O is rounded to bf16: 2^-8 of itself.
"""
import math

import torch


def attention8(ref, cu, lens, tables, prefix, q, scale, weights=None):
    """(O, LSE, bound of O, bound of LSE).  weights: rounds the weights, relative to the largest, before their product (for the
    oracle's own mistakes)."""
    H, group = q.shape[1], q.shape[1] // ref.heads
    O = torch.full(q.shape, math.nan, dtype=torch.float64)
    L = torch.full((H, q.shape[0]), math.nan, dtype=torch.float64)
    bo, bl = torch.zeros_like(O), torch.zeros_like(L)
    for s in range(len(lens)):
        n = cu[s + 1] - cu[s]
        if n <= 0:
            continue
        at = [(p, ref.place(tables[s], p)) for p in range(max(0, lens[s]))]
        at = [(p, x) for p, x in at if x is not None]
        if not at:
            O[cu[s]:cu[s + 1]], L[:, cu[s]:cu[s + 1]] = 0.0, -math.inf
            continue
        pos = torch.tensor([p for p, _ in at])
        pg, place = (torch.tensor([x[i] for _, x in at]) for i in range(2))
        c, w = (ref.code[i][pg, place] for i in range(2))                  # [keys, heads, d]
        a, b = (ref.scale[i][pg, place].double() for i in range(2))        # [keys, heads]
        qs = q[cu[s]:cu[s + 1]].double()
        own = lens[s] - n + torch.arange(n)
        seen = (pos[None, :] <= own[:, None]) | (pos < (prefix[s] if prefix is not None else 0))[None, :]
        some = seen.any(1)
        for h in range(H):
            g = h // group
            Q = qs[:, g * group:(g + 1) * group].abs().max().item()
            x = ((qs[:, h] @ c[:, g].T) * a[:, g]) * scale
            m = ((qs[:, h].abs() @ c[:, g].abs().T) * a[:, g]) * scale
            off = 2.0 ** -39 * scale * Q * a[:, g] * c[:, g].abs().sum(1) + (ref.dim + 4) * 2.0 ** -23 * m
            G = (x.abs() * seen).amax(1) * 1.4427 + b[:, g].clamp(min=2.0 ** -90).log2().abs().amax()
            rel = torch.expm1(2 * (off * seen).amax(1)) + 2.0 ** -21 * 0.6932 * G + 2.0 ** -21 + (16 + len(at) / 16) * 2.0 ** -24
            x = x.masked_fill(~seen, -math.inf)
            lse = torch.full((n,), -math.inf, dtype=torch.float64)
            lse[some] = torch.logsumexp(x[some], 1)
            p = torch.zeros_like(x)
            p[some] = torch.exp(x[some] - lse[some][:, None])
            u = p * b[:, g]
            top = u.amax(1, keepdim=True)
            if weights is not None:
                u = weights(u / top.clamp(min=1e-300)) * top
            o, A = u @ w[:, g], u @ w[:, g].abs()
            least = 2.0 ** -25 * top * (seen.double() @ w[:, g].abs())
            O[cu[s]:cu[s + 1], h], L[h, cu[s]:cu[s + 1]] = o, lse
            bo[cu[s]:cu[s + 1], h] = 2.0 ** -8 * o.abs() + (1 + 2.0 ** -7) * (2.0 ** -11 * A + least) + rel[:, None] * (A + o.abs()) + 1e-37
            bl[h, cu[s]:cu[s + 1]] = rel + 2.0 ** -21 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2.0 ** -22
    return O, L, bo, bl


def check8(setup, qlens, q, o, lse, prefix=None):
    cu = [sum(qlens[:i]) for i in range(len(qlens) + 1)]
    O, L, bo, bl = attention8(setup.ref, cu, setup.lens, setup.tables, prefix, q, setup.dim ** -0.5)
    n = sum(qlens)
    off = (o[:n].double() - O[:n]).abs() / bo[:n]
    assert off.max() <= 1, f"O off by {off.max():.3g} of its bound"
    dead = torch.isinf(L[:, :n])
    assert torch.equal(torch.isinf(lse[:, :n]) & (lse[:, :n] < 0), dead)
    off = ((lse[:, :n].double() - L[:, :n]).abs() / bl[:, :n])[~dead]
    assert off.numel() == 0 or off.max() <= 1, f"LSE off by {off.max():.3g} of its bound"


def to_half(q):
    """What the kernels make of rows [..., d] of queries that are multiplied together, in 64 bits."""
    big = q.double().abs().amax()
    e = min(max((math.frexp(big.item())[1] - 1) - 14, -112), 113) if big > 0 else 0
    return (q.double() * 2.0 ** -e).half().double() * 2.0 ** e
