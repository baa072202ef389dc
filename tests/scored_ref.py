"""Scored attention from its definition in 64 bits, with bounds on what the kernels' roundings can do to each output.

A *problem* is (query rows, key rows, query positions, key positions, prefix length): one sequence, whatever the tasks it is
cut into.  ``forward`` and ``backward`` walk problems and heads and return fp64 tensors on the CPU and, beside each, an
elementwise bound that counts the roundings the kernels make:

  * a score is an fp32 sum of d exact products, then a few fp32 operations: off by at most ``es``;
  * P is rounded to bf16 once (2^-8 of its value) before the products with V and dO;
  * dS is rounded to bf16 ``ds_roundings`` times before the products with K and Q;
  * outputs are rounded once to their type.
"""
from __future__ import annotations

import math

import torch

BF16 = 2.0 ** -8
FP32 = 2.0 ** -24


def scores(qh, kh, qpos, kpos, prefix, scale, cap=0.0, slope=None, table=None, bucket_of=None, masked=False):
    """(s, dC/dx, bucket numbers or None, error bound) of one head: [Lq, Lk] in fp64, -inf where invisible."""
    x = scale * (qh @ kh.T)
    es = (qh.shape[1] + 8) * FP32 * scale * (qh.abs() @ kh.abs().T)   # fp32 sum of exact products, times scale
    dist = kpos[None, :] - qpos[:, None]
    slope_c = torch.ones_like(x)
    s = x
    if cap > 0:
        t = torch.tanh(x / cap)
        s = cap * t
        slope_c = 1 - t * t
        es = es + cap * 2.0 ** -20        # tanh: 7e-8 relative or 2^-22 absolute, two roundings around it
    bucket = None
    if slope is not None:
        s = s - slope * dist.abs()
        es = es + 4 * FP32 * slope.abs() * dist.abs()
    if table is not None:
        reach = (bucket_of.numel() - 1) // 2
        bucket = bucket_of[dist.clamp(-reach, reach) + reach].long()
        ok = (bucket >= 0) & (bucket < table.numel())
        b = torch.where(ok, table[bucket.clamp(0, table.numel() - 1)], torch.zeros((), dtype=table.dtype))
        bucket = torch.where(ok, bucket, torch.full_like(bucket, -1))
        b = torch.where(b <= -1e30, torch.full_like(b, -math.inf), b)
        s = s + b
        es = es + 4 * FP32 * torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b))
    if masked:
        seen = (kpos < prefix)[None, :] | (dist <= 0)
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
    es = es + 4 * FP32 * torch.where(torch.isfinite(s), s.abs(), torch.zeros_like(s))
    return s, slope_c, bucket, es


def _softmax(s):
    m = s.amax(1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=s.dtype)
    m0 = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    p = torch.exp(s - m0)
    l = p.sum(1, keepdim=True)
    lse = torch.where(l > 0, m0 + torch.log(l), torch.full_like(l, -math.inf)).squeeze(1)
    return torch.where(l > 0, p / l, torch.zeros_like(p)), lse


def _args(score, h):
    one = lambda t: None if t is None else t[..., h].double()  # noqa: E731
    return dict(cap=score.get("cap", 0.0), slope=one(score.get("slopes")), table=one(score.get("table")),
                bucket_of=score.get("bucket_of"), masked=score.get("masked", False))


def forward(problems, q, k, v, scale, score, heads=None):
    q, k, v = (x.double() for x in (q, k, v))
    H = q.shape[1]
    o, o_err = torch.zeros_like(q), torch.zeros_like(q)
    lse, lse_err = torch.zeros(H, q.shape[0], dtype=torch.float64), torch.zeros(H, q.shape[0], dtype=torch.float64)
    for n, (qi, ki, qpos, kpos, prefix) in enumerate(problems):
        for h in (range(H) if heads is None else heads[n]):
            s, _, _, es = scores(q[qi, h], k[ki, h], qpos, kpos, prefix, scale, **_args(score, h))
            p, l = _softmax(s)
            worst = torch.where(torch.isfinite(s), es, torch.zeros_like(es)).amax(1, keepdim=True) if ki.numel() else torch.zeros(len(qi), 1)
            rel = 2 * worst + 2.0 ** -19                       # of P: its score, the LSE, exp2 and the sum
            spread = p @ v[ki, h].abs()
            o[qi, h] = p @ v[ki, h]
            o_err[qi, h] = (BF16 + rel) * spread + BF16 * o[qi, h].abs() + 1e-30
            lse[h, qi] = l
            lse_err[h, qi] = worst.squeeze(1) + 2.0 ** -19 + 4 * FP32 * torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
    return dict(o=o, lse=lse, o_err=o_err, lse_err=lse_err)


def backward(problems, q, k, v, o, lse, d_o, scale, score, heads=None, ds_roundings=1):
    """Gradients for the O (as stored) and LSE given; `lse` fp32."""
    q, k, v, o, d_o, lse = (x.double() for x in (q, k, v, o, d_o, lse))
    H = q.shape[1]
    g = {n: torch.zeros_like(x) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    e = {n: torch.zeros_like(x) for n, x in g.items()}
    table = score.get("table")
    dt = torch.zeros_like(table, dtype=torch.float64) if table is not None else None
    et = torch.zeros_like(dt) if table is not None else None
    for n, (qi, ki, qpos, kpos, prefix) in enumerate(problems):
        if not ki.numel():
            continue
        for h in (range(H) if heads is None else heads[n]):
            qh, kh, vh, oh, doh = q[qi, h], k[ki, h], v[ki, h], o[qi, h], d_o[qi, h]
            s, slope_c, bucket, es = scores(qh, kh, qpos, kpos, prefix, scale, **_args(score, h))
            l = lse[h, qi][:, None]
            p = torch.where(torch.isfinite(l), torch.exp(s - l), torch.zeros_like(s))
            d = (doh * oh).sum(1, keepdim=True)
            gr = p * (doh @ vh.T - d)
            rel = torch.where(torch.isfinite(s), es, torch.zeros_like(es)) + 2.0 ** -19 + 8 * FP32 * torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
            eg = rel * gr.abs() + p * (vh.shape[1] + 8) * FP32 * (doh.abs() @ vh.abs().T + (doh * oh).abs().sum(1, keepdim=True))
            ds = gr * slope_c
            # C' is held in fp16; near |C'| = 0 its error is that of tanh
            eds = eg * slope_c + (ds_roundings * BF16 + 2.0 ** -11 * (score.get("cap", 0.0) > 0)) * ds.abs()
            if score.get("cap", 0.0) > 0:
                eds = eds + gr.abs() * (2.0 ** -20 + 2 * es / score["cap"])
            g["dv"][ki, h] += p.T @ doh
            e["dv"][ki, h] += ((BF16 + rel) * p).T @ doh.abs()
            g["dq"][qi, h] += scale * (ds @ kh)
            e["dq"][qi, h] += scale * (eds + 2.0 ** -16 * ds.abs()) @ kh.abs()
            g["dk"][ki, h] += scale * (ds.T @ qh)
            e["dk"][ki, h] += scale * (eds + 2.0 ** -16 * ds.abs()).T @ qh.abs()
            if table is not None:
                for b in range(table.shape[0]):
                    at = bucket == b
                    dt[b, h] += gr[at].sum()
                    et[b, h] += (eg[at] + 2.0 ** -18 * gr[at].abs()).sum()
    for n in g:
        e[n] = e[n] + BF16 * g[n].abs() + 1e-30
    out = dict(g, **{n + "_err": x for n, x in e.items()})
    if table is not None:
        out.update(dtable=dt, dtable_err=et + 2 * FP32 * dt.abs() + 1e-30)
    return out


def check(got, ref, name):
    """|got - ref| within the bound, -inf where the reference has it; returns the largest share of the bound used."""
    got = got.detach().double().cpu()
    want, bound = ref[name], ref[name + "_err"]
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    assert torch.isfinite(got[~inf]).all(), f"{name}: not finite"
    off = (got - want).abs()[~inf] / bound[~inf]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times the bound"
    return worst
