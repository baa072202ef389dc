"""Cases of the attention operators with scores beyond q.k, and of attention over a shared prefix.

Operators (``case["op"]``):

  ``fwd``        attention whose scores may be capped by a tanh, biased by distance or by a learned bucket of the
                 distance, and masked by a prefix mask inside each sequence of a packed batch: O and LSE.
  ``bwd``        its gradients dQ, dK, dV and, with a bucket bias, the gradient of the bias table.
  ``rows``       the same forward for a few query rows at the end of one long key range that is given in chunks
                 (partial results, joined by the log-sum-exp merge): the single-token form.
  ``prefix_fwd`` / ``prefix_bwd``   attention of a batch whose sequences share one long prefix of keys.

Definitions.  For a visible pair (i, j) of head h, with x = scale * q_i.k_j and d = pos(j) - pos(i):
    s = C(x) - slope_h |d| + table[bucket_of[clamp(d, -R, R) + R]][h],  C(x) = cap * tanh(x / cap) if cap > 0 else x
    O = softmax(s) V,  LSE = log sum exp s
    P = exp(s - LSE),  G = P (dO.V - D),  D = rowsum(dO O),  dV = P^T dO,  dS = G C'(x),  dQ = scale dS K,
    dK = scale dS^T Q,  dtable[b][h] = sum of G over the pairs with that bucket.
"""
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # three short texts, one of a single token: what a call costs at least
        dict(name="bucket_fwd_tiny", op="fwd", lens="17,1,130", heads=2, dim=64, buckets=32, reach=128, cap=0.0, slopes=False, mask=False, prefix=0),
        # a batch of captions through a text encoder with learned relative positions, ragged
        dict(name="bucket_fwd_text", op="fwd", lens="512,512,512,77,512,401,512,300,512,512,1,512,512,255,512,512", heads=12, dim=64,
             buckets=32, reach=128, cap=0.0, slopes=False, mask=False, prefix=0),
        # images generated token by token after a condition of 256 tokens that sees itself whole; capped scores
        dict(name="cap_prefix_fwd", op="fwd", lens="1560,1560,3600", heads=12, dim=128, buckets=0, reach=0, cap=50.0, slopes=False, mask=True, prefix=256),
        # one chunk of a video whose scores fall off with the distance
        dict(name="distance_fwd_long", op="fwd", lens="9450", heads=12, dim=128, buckets=0, reach=0, cap=0.0, slopes=True, mask=False, prefix=0),
        # one new token against eight chunks of a long video
        dict(name="row_fwd_chunks", op="rows", rows=1, chunk=9450, chunks=8, heads=40, dim=128, buckets=0, reach=0, cap=0.0, slopes=True),
        # gradients of the first two and of the capped and the long case
        dict(name="bucket_bwd_tiny", op="bwd", lens="17,1,130", heads=2, dim=64, buckets=32, reach=128, cap=0.0, slopes=False, mask=False, prefix=0),
        dict(name="bucket_bwd_text", op="bwd", lens="512,512,512,77,512,401,512,300,512,512,1,512,512,255,512,512", heads=12, dim=64,
             buckets=32, reach=128, cap=0.0, slopes=False, mask=False, prefix=0),
        dict(name="cap_prefix_bwd", op="bwd", lens="1560,1560,3600", heads=12, dim=128, buckets=0, reach=0, cap=50.0, slopes=False, mask=True, prefix=256),
        dict(name="distance_bwd_long", op="bwd", lens="9450", heads=12, dim=128, buckets=0, reach=0, cap=0.0, slopes=True, mask=False, prefix=0),
        # 64 rollouts from one context, one new token each, each with up to 512 tokens of its own
        dict(name="prefix_fwd_decode", op="prefix_fwd", qlens="1*64", klens="ragged", kmax=512, shared=32760, heads=12, dim=128),
        # eight continuations of ragged length after one context, whole, and their gradients
        dict(name="prefix_fwd_tokens", op="prefix_fwd", qlens="100,1,257,64,130,8,77,300", klens="same", kmax=0, shared=8190, heads=12, dim=128),
        dict(name="prefix_bwd_tokens", op="prefix_bwd", qlens="100,1,257,64,130,8,77,300", klens="same", kmax=0, shared=8190, heads=12, dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["fwd", "fwd", "bwd", "bwd", "rows", "prefix_fwd", "prefix_bwd"])
    dim = rng.choice([64, 128])
    heads = rng.randint(1, 12)
    kind = rng.choice(["bucket", "cap", "distance", "all"])
    buckets, reach, cap, slopes, mask, prefix = 0, 0, 0.0, False, False, 0
    if kind in ("bucket", "all"):
        buckets, reach = rng.randint(2, 64), _log(rng, 1, 600)
    if kind in ("cap", "all"):
        cap, mask, prefix = round(rng.uniform(8.0, 60.0), 2), rng.random() < 0.7, rng.choice([0, 1, rng.randint(2, 700)])
    if kind in ("distance", "all"):
        slopes = True
    if op in ("fwd", "bwd"):
        left, lens = _log(rng, 64, 8190), []
        while left > 0 and len(lens) < 12:
            n = min(left, _log(rng, 1, 8190))
            lens.append(n)
            left -= n
        return dict(op=op, lens=",".join(map(str, lens)), heads=heads, dim=dim, buckets=buckets, reach=reach, cap=cap, slopes=slopes,
                    mask=mask, prefix=prefix)
    if op == "rows":
        rows = _log(rng, 1, 64)
        return dict(op=op, rows=rows, chunk=_log(rng, rows, 9450), chunks=rng.randint(1, 8), heads=rng.randint(1, 40), dim=dim,
                    buckets=buckets, reach=reach, cap=cap, slopes=slopes)
    n = _log(rng, 1, 24)
    if op == "prefix_fwd" and rng.random() < 0.5:
        return dict(op=op, qlens="1*%d" % _log(rng, 1, 96), klens="ragged", kmax=_log(rng, 1, 512), shared=_log(rng, 1, 32760), heads=heads, dim=dim)
    return dict(op=op, qlens=",".join(str(_log(rng, 1, 260)) for _ in range(n)), klens="same", kmax=0, shared=_log(rng, 1, 8190), heads=heads, dim=dim)


def _ints(text):
    if "*" in text:
        a, b = text.split("*")
        return [int(a)] * int(b)
    return [int(x) for x in text.split(",")]


def _own_lens(case, qlens):
    if case["klens"] == "same":
        return list(qlens)
    return [1 + (i * 7919 + 101) % case["kmax"] for i in range(len(qlens))]  # ragged, every length from 1 to kmax equally likely


def _pairs(case):
    """(visible pairs per head, query rows, key rows)."""
    op = case["op"]
    if op in ("fwd", "bwd"):
        lens = _ints(case["lens"])
        if not case["mask"]:
            return sum(n * n for n in lens), sum(lens), sum(lens)
        return sum(min(n, case["prefix"]) * min(n, case["prefix"]) + sum(r + 1 for r in range(min(n, case["prefix"]), n)) for n in lens), sum(lens), sum(lens)
    if op == "rows":
        keys, rows = case["chunk"] * case["chunks"], min(case["rows"], case["chunk"])
        return rows * keys - rows * (rows - 1) // 2, rows, keys
    qlens = _ints(case["qlens"])
    klens = _own_lens(case, qlens)
    return sum(q * (case["shared"] + k) for q, k in zip(qlens, klens)), sum(qlens), case["shared"] + sum(klens)


def work(case):
    pairs, nq, nk = _pairs(case)
    h, d = case["heads"], case["dim"]
    if case["op"].endswith("bwd"):
        # reads Q O dO LSE K V, writes dQ dK dV
        return {"bytes": h * (nq * (8 * d + 4) + nk * 8 * d), "flops": 10 * pairs * d * h}
    return {"bytes": h * (nq * (4 * d + 4) + nk * 4 * d), "flops": 4 * pairs * d * h}


# ------------------------------------------------------------------------------------------------ inputs
def _bucket_of(n, reach):
    """Bucket of every distance -reach .. reach: half of the buckets for each side, exact near, logarithmic further out."""
    side = max(1, n // 2)
    near = max(1, side // 2)
    got = []
    for d in range(-reach, reach + 1):
        a, b = abs(d), 0
        b = a if a < near else min(side - 1, near + int((side - near) * math.log(a / near) / max(1e-9, math.log(max(reach, near + 1) / near))))
        got.append(min(n - 1, b + (side if d > 0 else 0)))
    return got


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 17)
    op, h, d = case["op"], case["heads"], case["dim"]
    _, nq, nk = _pairs(case)

    def normal(rows, times=1.0):
        return (torch.randn(rows, h, d, generator=g, device=dev) * times).to(torch.bfloat16)

    st = dict(op=op, q=normal(nq, 1.5), k=normal(nk), v=normal(nk), scale=1.0 / math.sqrt(d), cap=case.get("cap", 0.0),
              slopes=None, table=None, bucket_of=None, reach=case.get("reach", 0), mask=case.get("mask", False) or op == "rows")
    if case.get("slopes"):
        st["slopes"] = torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device=dev)
    if case.get("buckets"):
        st["table"] = torch.randn(case["buckets"], h, generator=g, device=dev) * 0.7
        st["bucket_of"] = torch.tensor(_bucket_of(case["buckets"], case["reach"]), dtype=torch.int32, device=dev)
    # sequence, position and length of the seen-whole prefix of every row: what says which pairs are visible
    if op in ("fwd", "bwd"):
        lens = _ints(case["lens"])
        n = torch.tensor(lens, device=dev)
        doc = torch.repeat_interleave(torch.arange(len(lens), device=dev), n)
        pos = torch.arange(nq, device=dev) - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)
        st.update(q_doc=doc, k_doc=doc, q_pos=pos, k_pos=pos, prefix=case["prefix"])
    elif op == "rows":
        st.update(q_doc=torch.zeros(nq, dtype=torch.long, device=dev), k_doc=torch.zeros(nk, dtype=torch.long, device=dev),
                  q_pos=torch.arange(nk - nq, nk, device=dev), k_pos=torch.arange(nk, device=dev), prefix=0)
    else:
        qlens = _ints(case["qlens"])
        klens = _own_lens(case, qlens)
        docs = torch.arange(len(qlens), device=dev)
        st.update(q_doc=torch.repeat_interleave(docs, torch.tensor(qlens, device=dev)),
                  k_doc=torch.cat([torch.full((case["shared"],), -1, device=dev), torch.repeat_interleave(docs, torch.tensor(klens, device=dev))]),
                  q_pos=torch.zeros(nq, dtype=torch.long, device=dev), k_pos=torch.zeros(nk, dtype=torch.long, device=dev), prefix=0)
    if op.endswith("bwd"):
        st["d_o"] = normal(nq)
        st["o"], st["lse"] = _plain_fwd(st)
    if own:
        _handle(case, st, dev)
    return st


# ------------------------------------------------------------------------------------------------ plain form
def _plain_scores(st):
    """(scores [H, nq, nk], tanh of the capped ones or None), invisible pairs at -inf."""
    s = torch.matmul(st["q"].permute(1, 0, 2).float(), st["k"].permute(1, 2, 0).float()) * st["scale"]
    t = None
    if st["cap"] > 0:
        t = torch.tanh(s / st["cap"])
        s = st["cap"] * t
    d = st["k_pos"][None, :] - st["q_pos"][:, None]
    if st["slopes"] is not None:
        s = s - st["slopes"][:, None, None] * d.abs()
    if st["table"] is not None:
        s = s + st["table"].t().contiguous()[:, st["bucket_of"].long()[d.clamp(-st["reach"], st["reach"]) + st["reach"]]]
    seen = (st["k_doc"][None, :] == st["q_doc"][:, None]) | (st["k_doc"] < 0)[None, :]
    if st["mask"]:
        seen &= (d <= 0) | (st["k_pos"] < st["prefix"])[None, :]
    return s.masked_fill_(~seen, -math.inf), t


def _plain_fwd(st):
    s, _ = _plain_scores(st)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, st["v"].permute(1, 0, 2).float()) / total
    return o.permute(1, 0, 2).contiguous().to(torch.bfloat16), (m + torch.log(total)).squeeze(-1)


def _plain_bwd(st):
    s, t = _plain_scores(st)
    q, k, v, d_o, o = (st[n].permute(1, 0, 2).float() for n in ("q", "k", "v", "d_o", "o"))
    p = torch.exp(s - st["lse"][:, :, None])
    del s
    g = torch.matmul(d_o, v.transpose(1, 2))
    g = p * (g - (d_o * o).sum(-1, keepdim=True))
    dv = torch.matmul(p.transpose(1, 2), d_o)
    del p
    ds = g if t is None else g * (1.0 - t * t)
    dq = torch.matmul(ds, k) * st["scale"]
    dk = torch.matmul(ds.transpose(1, 2), q) * st["scale"]
    out = [x.permute(1, 0, 2).contiguous().to(torch.bfloat16) for x in (dq, dk, dv)]
    if st["table"] is not None:
        del ds
        # rows and columns are the same tokens here: sums over the diagonals, in 64 bits, then over the distances of a bucket
        n = g.shape[1]
        skew = torch.nn.functional.pad(g.flip(1), (0, n)).reshape(g.shape[0], -1)[:, : n * (2 * n - 1)].reshape(-1, n, 2 * n - 1)
        diag = skew.sum(1, dtype=torch.float64)
        d = torch.arange(-(n - 1), n, device=g.device).clamp(-st["reach"], st["reach"]) + st["reach"]
        table = torch.zeros(st["table"].shape, dtype=torch.float64, device=g.device)
        out.append(table.index_add_(0, st["bucket_of"].long()[d], diag.t()).float())
    return out


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handle(case, st, dev):
    import paper_2608_01150_b200 as Z
    op, h, d = case["op"], case["heads"], case["dim"]
    nq, nk = st["q"].shape[0], st["k"].shape[0]
    cu = lambda lens: [sum(lens[:i]) for i in range(len(lens) + 1)]  # noqa: E731
    if op in ("fwd", "bwd"):
        lens = _ints(case["lens"])
        t = Z.build_tasks(cu(lens), [], nq, nk, h, d)
        if case["mask"]:
            t.set_positions(whole_prefix=[case["prefix"]] * len(lens))
    elif op == "rows":
        c = case["chunk"]
        t = Z.build_tasks([0], [(0, nq, i * c, c, 0) for i in range(case["chunks"])], nq, nk, h, d)
        t.set_positions(shard_pos=[(nk - nq, i * c, 0) for i in range(case["chunks"])])
    else:
        qlens = _ints(case["qlens"])
        t = Z.build_tasks_prefix(cu(qlens), cu(_own_lens(case, qlens)), case["shared"], nq, nk, h, d)
    st["tasks"] = t
    if op in ("fwd", "bwd", "rows"):
        st["score"] = Z.Score(cap=st["cap"], slopes=st["slopes"], bucket_bias=st["table"], bucket_of=st["bucket_of"], masked=bool(st["mask"]))
    empty = lambda *shape, t=torch.bfloat16: torch.empty(*shape, dtype=t, device=dev)  # noqa: E731
    if op.endswith("bwd"):
        st.update(dq=empty(nq, h, d), dk=empty(nk, h, d), dv=empty(nk, h, d), dtable=None)
        if st["table"] is not None:
            st["dtable"] = torch.empty_like(st["table"])
        n = t.scored_workspace_bytes(st["score"]) if op == "bwd" else int(t.info.bwd_workspace_bytes)
        st["ws"] = empty(n, t=torch.uint8)
    else:
        rows = max(1, int(t.info.partial_rows))
        st.update(out_o=empty(nq, h, d), out_lse=empty(h, nq, t=torch.float32), o_part=None, lse_part=None)
        if t.info.partial_rows:
            st.update(o_part=empty(rows, h, d, t=torch.float32), lse_part=empty(h, rows, t=torch.float32))


def _own_run(st):
    import paper_2608_01150_b200 as Z
    t, op = st["tasks"], st["op"]
    if op == "bwd":
        Z.scored_attn_bwd(t, st["score"], st["q"], st["k"], st["v"], st["o"], st["lse"], st["d_o"], st["scale"], st["dq"], st["dk"], st["dv"],
                          st["dtable"], st["ws"])
        return [st[n] for n in ("dq", "dk", "dv", "dtable") if st[n] is not None]
    if op == "prefix_bwd":
        Z.coalesced_attn_bwd(t, st["q"], st["k"], st["v"], st["o"], st["lse"], st["d_o"], st["scale"], st["dq"], st["dk"], st["dv"], st["ws"])
        return [st["dq"], st["dk"], st["dv"]]
    if op == "prefix_fwd":
        Z.coalesced_attn_fwd(t, st["q"], st["k"], st["v"], st["scale"], st["out_o"], st["out_lse"], st["o_part"], st["lse_part"])
    else:
        Z.scored_attn_fwd(t, st["score"], st["q"], st["k"], st["v"], st["scale"], st["out_o"], st["out_lse"], st["o_part"], st["lse_part"])
    if st["o_part"] is not None:
        Z.lse_merge(t, st["o_part"], st["lse_part"], st["out_o"], st["out_lse"])
    return [st["out_o"], st["out_lse"]]


def run(st):
    if own:
        return _own_run(st)
    return _plain_bwd(st) if st["op"].endswith("bwd") else list(_plain_fwd(st))


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """One sequence and one head at a time, straight from the definitions."""
    st = prepare(case, seed)
    op, h = case["op"], case["heads"]
    back = op.endswith("bwd")
    q, k, v = (st[n].double() for n in ("q", "k", "v"))
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    lse_out = torch.zeros(h, q.shape[0], dtype=torch.float64, device=q.device)
    table = st["table"].double() if st["table"] is not None else None
    d_table = torch.zeros_like(table) if table is not None else None
    shared = torch.nonzero(st["k_doc"] < 0).flatten()
    for doc in range(int(st["q_doc"].max()) + 1):
        qi = torch.nonzero(st["q_doc"] == doc).flatten()
        ki = torch.cat([shared, torch.nonzero(st["k_doc"] == doc).flatten()])
        dist = st["k_pos"][ki][None, :] - st["q_pos"][qi][:, None]
        hidden = ~((dist <= 0) | (st["k_pos"][ki] < st["prefix"])[None, :]) if st["mask"] else None
        bucket = st["bucket_of"].long()[torch.clamp(dist, -st["reach"], st["reach"]) + st["reach"]] if table is not None else None
        for i in range(h):
            x = (q[qi, i] @ k[ki, i].T) * st["scale"]
            th = torch.tanh(x / st["cap"]) if st["cap"] > 0 else None
            s = st["cap"] * th if th is not None else x
            if st["slopes"] is not None:
                s = s - st["slopes"][i].double() * dist.abs()
            if table is not None:
                s = s + table[:, i][bucket]
            if hidden is not None:
                s = torch.where(hidden, torch.full_like(s, -math.inf), s)
            if not back:
                lse_out[i, qi] = torch.logsumexp(s, 1)
                out["o"][qi, i] = torch.exp(s - lse_out[i, qi][:, None]) @ v[ki, i]
                continue
            d_o, o = st["d_o"][qi, i].double(), st["o"][qi, i].double()
            p = torch.exp(s - st["lse"][i, qi].double()[:, None])
            gr = p * (d_o @ v[ki, i].T - (d_o * o).sum(1, keepdim=True))
            out["dv"][ki, i] += p.T @ d_o
            if table is not None:
                for b in range(table.shape[0]):
                    d_table[b, i] += gr[bucket == b].sum()
            if th is not None:
                gr = gr * (1 - th * th)
            out["dq"][qi, i] = gr @ k[ki, i] * st["scale"]
            out["dk"][ki, i] += gr.T @ q[qi, i] * st["scale"]
    if not back:
        return [out["o"], lse_out]
    return [out["dq"], out["dk"], out["dv"]] + ([d_table] if table is not None else [])
