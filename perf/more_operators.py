"""Cases of the paged key/value cache: writing it, reading it back, and attention of new tokens over it.

The keys and values of a batch of sequences lie in pages of ``page`` tokens; a table gives each sequence's pages.  A
sequence has ``kv_len`` tokens, the last ``q_len`` of which are new.  The cache holds bf16, or 8 bits (whole numbers or
e4m3) with one 32-bit scale for each token and head.

Operators (``case["op"]``):

  ``write``  the new tokens' keys and values go into their slots, then the rows just written are read back as bf16, as a program
             does that runs the chunk's own attention on what the cache holds: rows (bf16) and the scale of every slot.
  ``read``   whole sequences out of the cache, one behind the other, as bf16.
  ``attn``   attention of the new tokens over the cache, a chunk of tokens or a single one for each sequence: O and LSE.

Definitions.  For a token and head with values x_c, T = 127 (whole numbers) or 448 (e4m3):
    scale = max |x_c| / T,  code_c = round(x_c / scale) to the type, both quotients rounded to 32 bits;  0 if scale is 0.
    Read back, a value is code_c * scale.
For a new token i at position p = kv_len - q_len + i, query head h, key head g = h // (heads / kv_heads):
    it sees keys j <= p and keys j < prefix,  s_j = scale * q_i.k_j,  O = softmax(s) V,  LSE = log sum exp s.
"""
import math

import torch

own = False

TOP = {"int8": 127.0, "e4m3": 448.0}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token for each of 16 sequences: what a write costs at least
        dict(name="write_step", op="write", fmt="int8", qlens="1*16", klens="ragged", kmax=2048, kv_heads=8, dim=128, page=16, head_major=False),
        # three images' tokens, ragged against the pages
        dict(name="write_images", op="write", fmt="e4m3", qlens="1560,1560,3600", klens="same", kmax=0, kv_heads=12, dim=128, page=64, head_major=False),
        # a whole video's tokens, pages of one head's tokens
        dict(name="write_video", op="write", fmt="int8", qlens="32760", klens="same", kmax=0, kv_heads=12, dim=128, page=64, head_major=True),
        # eight ragged sequences for an engine that wants them packed
        dict(name="read_ragged", op="read", fmt="int8", qlens="1,77,512,1,300,33,512,130", klens="ragged", kmax=4096, kv_heads=12, dim=64, page=16, head_major=False),
        # a long sequence beside two images
        dict(name="read_video", op="read", fmt="e4m3", qlens="1*3", klens="32760,3600,1560", kmax=0, kv_heads=12, dim=128, page=64, head_major=False),
        # one new token of one short sequence: what a call costs at least
        dict(name="token_tiny", op="attn", fmt="bf16", qlens="1", klens="300", kmax=0, heads=12, kv_heads=12, dim=64, page=16, head_major=False, prefix=0),
        # one new token for each of 64 sequences of up to 8192 keys, five query heads to a key head
        dict(name="token_batch", op="attn", fmt="bf16", qlens="1*64", klens="ragged", kmax=8192, heads=40, kv_heads=8, dim=128, page=16, head_major=False, prefix=0),
        # the same from a cache in 8 bits
        dict(name="token_batch_e4m3", op="attn", fmt="e4m3", qlens="1*64", klens="ragged", kmax=8192, heads=40, kv_heads=8, dim=128, page=64, head_major=False, prefix=0),
        # one new token behind a long video, as many key heads as query heads
        dict(name="token_long", op="attn", fmt="int8", qlens="1", klens="75600", kmax=0, heads=12, kv_heads=12, dim=128, page=64, head_major=True, prefix=0),
        # a chunk of 512 tokens behind 8190
        dict(name="chunk", op="attn", fmt="bf16", qlens="512", klens="8702", kmax=0, heads=12, kv_heads=12, dim=128, page=64, head_major=False, prefix=0),
        # prompts in chunks beside single tokens, in one call
        dict(name="mixed_int8", op="attn", fmt="int8", qlens="700,1*20,130,1*8,257,3,64", klens="ragged", kmax=4096, heads=16, kv_heads=4, dim=64, page=16,
             head_major=False, prefix=0),
        # an image's tokens, seen whole by one another, behind a long video
        dict(name="chunk_image_e4m3", op="attn", fmt="e4m3", qlens="1560", klens="34320", kmax=0, heads=40, kv_heads=8, dim=128, page=64, head_major=False,
             prefix=34320),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attn", "attn", "attn"])
    dim, page = rng.choice([64, 128]), rng.choice([8, 16, 32, 64, 128, 256])
    fmt = rng.choice(["int8", "e4m3"] if op == "write" else ["bf16", "int8", "e4m3"])
    case = dict(op=op, fmt=fmt, dim=dim, page=page, head_major=rng.random() < 0.3, kmax=0)
    kv_heads = rng.randint(1, 12)
    if op != "attn":
        left, lens = _log(rng, 1, 24000), []
        while left > 0 and len(lens) < 24:
            n = min(left, _log(rng, 1, 24000))
            lens.append(n)
            left -= n
        case.update(qlens=",".join(map(str, lens)), kv_heads=kv_heads, klens=",".join(str(n + _log(rng, 1, 4000) - 1) for n in lens))
        return case
    kind = rng.choice(["tokens", "chunk", "mixed"])
    kv_heads, group = rng.randint(1, 8), rng.choice([1, 1, 2, 3, 4, 5, 8])
    if kind == "tokens":
        n = _log(rng, 1, 96)
        qlens = [rng.choice([1, 1, 1, rng.randint(1, 4)]) for _ in range(n)]
        klens = [q - 1 + _log(rng, 1, max(2, 400000 // n) if n > 4 else 75600) for q in qlens]
    elif kind == "chunk":
        qlens = [_log(rng, 2, 2048)]
        klens = [qlens[0] - 1 + _log(rng, 1, 16380)]
    else:
        qlens = [rng.choice([1, _log(rng, 1, 700)]) for _ in range(rng.randint(2, 24))]
        klens = [q - 1 + _log(rng, 1, 8190) for q in qlens]
    prefix = rng.choice([0, 0, 1, _log(rng, 2, 9450)])
    case.update(qlens=",".join(map(str, qlens)), klens=",".join(map(str, klens)), heads=kv_heads * group, kv_heads=kv_heads, prefix=prefix)
    return case


def _ints(text):
    out = []
    for part in text.split(","):
        a, _, n = part.partition("*")
        out += [int(a)] * int(n or 1)
    return out


def _lens(case):
    """New tokens and all tokens of every sequence."""
    qlens = _ints(case["qlens"])
    if case["klens"] == "same":
        return qlens, list(qlens)
    if case["klens"] == "ragged":  # every length from 1 to kmax equally likely before the new tokens
        return qlens, [q + (i * 7919 + 2741) % case["kmax"] for i, q in enumerate(qlens)]
    return qlens, _ints(case["klens"])


def _pairs(case):
    qlens, klens = _lens(case)
    pairs = 0
    for q, k in zip(qlens, klens):
        pairs += sum(min(k, max(k - q + i + 1, case["prefix"])) for i in range(q))
    return pairs


def work(case):
    qlens, klens = _lens(case)
    nq, nk, hk, d = sum(qlens), sum(klens), case["kv_heads"], case["dim"]
    slot = hk * (2 * d + 8 if case["fmt"] != "bf16" else 4 * d)  # keys and values of a token as they are held
    if case["op"] == "write":  # rows in, slots out; slots in, rows out
        return {"bytes": 2 * nq * (4 * hk * d + slot), "flops": 6 * nq * hk * d}
    if case["op"] == "read":
        return {"bytes": nk * (4 * hk * d + slot), "flops": 2 * nk * hk * d}
    h = case["heads"]
    return {"bytes": nk * slot + nq * h * (4 * d + 4), "flops": 4 * _pairs(case) * d * h}


# ------------------------------------------------------------------------------------------------ inputs
def _quantise(x, fmt):
    """Codes and scales of rows x [..., d] in 32 bits."""
    scale = x.abs().amax(-1)
    scale = scale / torch.full_like(scale, TOP[fmt])  # (by a number, the quotient would be a product with its rounded reciprocal)
    y = x / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None]
    if fmt == "int8":
        return torch.round(y).to(torch.int8), scale
    return y.clamp(-TOP[fmt], TOP[fmt]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 29)
    op, fmt, page, hk, d = case["op"], case["fmt"], case["page"], case["kv_heads"], case["dim"]
    qlens, klens = _lens(case)
    nq = sum(qlens)
    counts = [(k + page - 1) // page for k in klens]
    n_pages = sum(counts) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    pages = torch.full((len(klens), max(counts)), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(counts):
        pages[i, :n] = order[at:at + n]
        at += n
    dtype = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[fmt]
    channel = torch.exp(0.5 * torch.randn(d, generator=g, device=dev))  # some channels of the keys are larger than others

    def rows(n, keys):
        x = torch.randn(n, hk, d, generator=g, device=dev)
        return (x * channel if keys else x).to(torch.bfloat16)

    st = dict(op=op, fmt=fmt, page=page, qlens=qlens, klens=klens, pages=pages, hk=hk, d=d)
    for name in ("k", "v"):
        shape = (n_pages, hk, page, d) if case["head_major"] else (n_pages, page, hk, d)
        pool = torch.zeros(shape, dtype=dtype, device=dev)
        pool = pool.transpose(1, 2) if case["head_major"] else pool
        scale = torch.zeros(n_pages, page, hk, dtype=torch.float32, device=dev) if fmt != "bf16" else None
        if op == "write":
            st["new_" + name] = rows(nq, name == "k")
        else:  # what the steps before this one have left there
            step = max(1, (1 << 26) // (page * hk * d))
            for a in range(0, n_pages, step):
                b = min(n_pages, a + step)
                x = rows((b - a) * page, name == "k").view(b - a, page, hk, d)
                if fmt == "bf16":
                    pool[a:b] = x
                else:
                    codes, scale[a:b] = _quantise(x.float(), fmt)
                    pool[a:b] = codes
        st[name], st[name + "_scale"] = pool, scale
    st["cu_q"] = torch.tensor([sum(qlens[:i]) for i in range(len(qlens) + 1)], dtype=torch.int32, device=dev)
    st["kv_len"] = torch.tensor(klens, dtype=torch.int32, device=dev)
    if op == "attn":
        h = case["heads"]
        st.update(heads=h, scale=1.0 / math.sqrt(d), q=(torch.randn(nq, h, d, generator=g, device=dev) * 1.5).to(torch.bfloat16), prefix=None)
        if case["prefix"]:
            st["prefix"] = torch.full((len(qlens),), case["prefix"], dtype=torch.int32, device=dev)
    else:  # the rows that are read: the new ones, or everything
        n = qlens if op == "write" else klens
        st["first"] = st["kv_len"] - torch.tensor(n, dtype=torch.int32, device=dev)
        st["cu_kv"] = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=dev)
    if own:
        _handle(st, dev)
    return st


# ------------------------------------------------------------------------------------------------ plain form
def _slots(st, seq, first, last):
    """Page and place in it of the tokens first .. last - 1 of a sequence."""
    pos = torch.arange(first, last, device=st["pages"].device)
    return st["pages"][seq].long()[pos // st["page"]], pos % st["page"]


def _held(st, name, seq, first, last):
    """Rows [n, kv_heads, d] of the cache in 32 bits."""
    pg, at = _slots(st, seq, first, last)
    x = st[name].view(torch.uint8)[pg, at].view(st[name].dtype).float() if st["fmt"] == "e4m3" else st[name][pg, at].float()
    return x if st["fmt"] == "bf16" else x * st[name + "_scale"][pg, at][..., None]


def _plain_write(st):
    at = 0
    for i, (q, k) in enumerate(zip(st["qlens"], st["klens"])):
        pg, place = _slots(st, i, k - q, k)
        for name in ("k", "v"):
            x = st["new_" + name][at:at + q]
            if st["fmt"] == "bf16":
                st[name][pg, place] = x
                continue
            codes, scale = _quantise(x.float(), st["fmt"])
            st[name].view(torch.uint8)[pg, place] = codes.view(torch.uint8)
            st[name + "_scale"][pg, place] = scale
        at += q
    return _plain_read(st, st["qlens"]) + [st["k_scale"], st["v_scale"]]


def _plain_read(st, lens):
    return [torch.cat([_held(st, name, i, k - n, k).to(torch.bfloat16) for i, (n, k) in enumerate(zip(lens, st["klens"]))]) for name in ("k", "v")]


def _plain_attn(st):
    out, lses, at = [], [], 0
    group = st["heads"] // st["hk"]
    for i, (n, k) in enumerate(zip(st["qlens"], st["klens"])):
        q = st["q"][at:at + n].float().view(n, st["hk"], group, st["d"]).permute(1, 2, 0, 3).reshape(st["hk"], group * n, st["d"])
        s = torch.matmul(q, _held(st, "k", i, 0, k).permute(1, 2, 0)) * st["scale"]
        key, pos = torch.arange(k, device=s.device), torch.arange(k - n, k, device=s.device).repeat(group)
        hidden = key[None, :] > pos[:, None]
        if st["prefix"] is not None:
            hidden &= key[None, :] >= st["prefix"][i]
        s.masked_fill_(hidden, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s.sub_(m))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, _held(st, "v", i, 0, k).transpose(0, 1)) / total
        out.append(o.view(st["hk"], group, n, st["d"]).permute(2, 0, 1, 3).reshape(n, st["heads"], st["d"]).to(torch.bfloat16))
        lses.append((m + torch.log(total)).view(st["heads"], n))
        at += n
    return [torch.cat(out), torch.cat(lses, 1)]


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handle(st, dev):
    import paper_2608_01150_b200 as Z
    st["cache"] = Z.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
    st["batch"] = Z.CacheBatch(st["cu_q"], st["kv_len"], st["pages"], prefix=st.get("prefix"), max_q=max(st["qlens"]))
    if st["op"] == "attn":
        st["attn"] = Z.build_cached_attn(st["heads"], st["hk"], st["d"])
        st["ws"] = torch.empty(st["attn"].workspace_bytes, dtype=torch.uint8, device=dev)
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["heads"], st["q"].shape[0], dtype=torch.float32, device=dev)
    else:
        n = sum(st["qlens"] if st["op"] == "write" else st["klens"])
        st["rows_k"] = torch.empty(n, st["hk"], st["d"], dtype=torch.bfloat16, device=dev)
        st["rows_v"] = torch.empty_like(st["rows_k"])


def _own_run(st):
    import paper_2608_01150_b200 as Z
    if st["op"] == "attn":
        Z.cached_attn_fwd(st["attn"], st["cache"], st["batch"], st["q"], st["scale"], st["o"], st["lse"], st["ws"])
        return [st["o"], st["lse"]]
    if st["op"] == "write":
        Z.cache_write(st["cache"], st["batch"], st["new_k"], st["new_v"])
    Z.cache_read(st["cache"], st["batch"], st["cu_kv"], st["rows_k"], st["rows_v"], first=st["first"])
    return [st["rows_k"], st["rows_v"]] + ([st["k_scale"], st["v_scale"]] if st["op"] == "write" else [])


def run(st):
    if own:
        return _own_run(st)
    if st["op"] == "write":
        return _plain_write(st)
    return _plain_read(st, st["klens"]) if st["op"] == "read" else _plain_attn(st)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _to_code(y, fmt):
    """Nearest value of the type, ties to even, of 32-bit quotients y."""
    y = y.float().double().clamp(-TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return torch.round(y)
    _, e = torch.frexp(y)
    step = torch.pow(2.0, (e.double() - 4).clamp(min=-9))  # three bits behind the leading one, down to 2^-9
    return torch.round(y / step) * step


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    table, page, fmt = st["pages"].long(), case["page"], case["fmt"]

    def where(i, lo, hi):
        pos = torch.arange(lo, hi, device=table.device)
        return table[i][torch.div(pos, page, rounding_mode="floor")] * page + pos % page

    if case["op"] == "write":
        res, slot = {}, torch.cat([where(i, k - q, k) for i, (q, k) in enumerate(zip(st["qlens"], st["klens"]))])
        for name in ("k", "v"):
            x = st["new_" + name].double()
            scale = (x.abs().max(-1).values / TOP[fmt]).float().double()
            code = torch.zeros_like(x)
            live = scale > 0
            code[live] = _to_code(x[live] / scale[live][:, None], fmt)
            res[name] = code * scale[..., None]
            full = torch.zeros(st[name].shape[0] * page, case["kv_heads"], dtype=torch.float64, device=x.device)
            full[slot] = scale
            res[name + "_scale"] = full.view(-1, page, case["kv_heads"])
        return [res["k"], res["v"], res["k_scale"], res["v_scale"]]
    flat = {}
    for name in ("k", "v"):
        x = st[name].float().reshape(-1, case["kv_heads"], case["dim"])
        flat[name] = (x, st[name + "_scale"].reshape(-1, case["kv_heads"]) if fmt != "bf16" else None)

    def held(name, slot):
        x, scale = flat[name]
        return x[slot].double() if scale is None else x[slot].double() * scale[slot].double()[..., None]

    if case["op"] == "read":
        slot = torch.cat([where(i, 0, k) for i, k in enumerate(st["klens"])])
        return [held("k", slot), held("v", slot)]
    o, lse, at = torch.zeros(st["q"].shape, dtype=torch.float64, device=table.device), [], 0
    for i, (n, k) in enumerate(zip(st["qlens"], st["klens"])):
        slot = where(i, 0, k)
        keys, values = held("k", slot), held("v", slot)
        sees = torch.clamp(torch.clamp(torch.arange(k - n, k, device=slot.device) + 1, min=case["prefix"]), max=k)
        seen = torch.arange(k, device=slot.device)[None, :] < sees[:, None]
        got = torch.empty(case["heads"], n, dtype=torch.float64, device=slot.device)
        for h in range(case["heads"]):
            j = h * case["kv_heads"] // case["heads"]
            s = torch.where(seen, (st["q"][at:at + n, h].double() @ keys[:, j].T) * st["scale"], -math.inf)
            got[h] = torch.logsumexp(s, 1)
            o[at:at + n, h] = torch.softmax(s, 1) @ values[:, j]
        lse.append(got)
        at += n
    return [o, torch.cat(lse, 1)]
