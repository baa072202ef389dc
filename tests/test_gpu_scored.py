"""Scored attention and shared prefixes on the GPU against the definition in 64 bits, with bounds counted from the
roundings (scored_ref): lengths and masks where tiles, windows and buckets can go wrong, and how the calls are used."""
import math

import pytest
import torch

import scored_ref as R
from zl_testlib import SENTINEL

pytestmark = pytest.mark.gpu


def rand(g, *shape, times=1.0):
    return (torch.randn(*shape, generator=g) * times).to(torch.bfloat16)


def make_score(g, H, cap=0.0, slopes=False, buckets=0, reach=0, masked=False, symmetric=False):
    s = dict(cap=cap, masked=masked)
    if slopes:
        s["slopes"] = torch.tensor([0.5 ** (i + 1) for i in range(H)])
    if buckets:
        n = 2 * reach + 1
        if symmetric:       # the same bucket on both sides and again further out: several runs of one bucket in a patch
            of = torch.arange(-reach, reach + 1).abs() % buckets
        else:
            of = torch.clamp(torch.arange(n) * buckets // n, 0, buckets - 1)
        s["table"], s["bucket_of"] = torch.randn(buckets, H, generator=g), of.to(torch.int32)
    return s


def to_score(Z, s):
    c = lambda n: None if s.get(n) is None else s[n].cuda()  # noqa: E731
    return Z.Score(cap=s.get("cap", 0.0), slopes=c("slopes"), bucket_bias=c("table"), bucket_of=c("bucket_of"), masked=s.get("masked", False))


def status_ok(h):
    torch.cuda.synchronize()
    assert h.last_device_status() == (0, 0)


class Run:
    """Forward (+ merge) and backward through the binding, outputs poisoned first."""

    def __init__(self, h, s, q, k, v, scale, packed=False, plain=False):
        import paper_2608_01150_b200 as Z
        self.Z, self.h, self.s, self.scale, self.plain = Z, h, s, scale, plain
        self.q, self.k, self.v = (x.cuda() for x in (q, k, v))
        self.packed = torch.stack([self.q, self.k, self.v], 1).contiguous() if packed else None
        self.score = None if plain else to_score(Z, s)

    def forward(self):
        Z, h = self.Z, self.h
        rows, H, d = self.q.shape
        self.o = torch.full((rows, H, d), SENTINEL, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((H, rows), SENTINEL, dtype=torch.float32, device="cuda")
        pr = int(h.info.partial_rows)
        op = torch.full((pr, H, d), SENTINEL, device="cuda") if pr else None
        lp = torch.full((H, pr), SENTINEL, device="cuda") if pr else None
        if self.plain:
            Z.coalesced_attn_fwd(h, self.q, self.k, self.v, self.scale, self.o, self.lse, op, lp)
        elif self.packed is not None:
            Z.scored_attn_fwd_packed(h, self.score, self.packed, self.scale, self.o, self.lse, op, lp)
        else:
            Z.scored_attn_fwd(h, self.score, self.q, self.k, self.v, self.scale, self.o, self.lse, op, lp)
        if pr:
            Z.lse_merge(h, op, lp, self.o, self.lse)
        status_ok(h)
        return self.o, self.lse

    def backward(self, d_o, o=None, lse=None):
        Z, h = self.Z, self.h
        self.d_o = d_o.cuda()
        o = self.o if o is None else o
        lse = self.lse if lse is None else lse
        full = lambda x: torch.full_like(x, SENTINEL)  # noqa: E731
        out = dict(dq=full(self.q), dk=full(self.k), dv=full(self.v))
        if self.plain:
            ws = torch.full((int(h.info.bwd_workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
            Z.coalesced_attn_bwd(h, self.q, self.k, self.v, o, lse, self.d_o, self.scale, out["dq"], out["dk"], out["dv"], ws)
        else:
            ws = torch.full((h.scored_workspace_bytes(self.score),), 255, dtype=torch.uint8, device="cuda")
            dt = None
            if self.score.bucket_bias is not None:
                dt = out["dtable"] = torch.full_like(self.score.bucket_bias, SENTINEL)
            if self.packed is not None:
                dqkv = full(self.packed)
                Z.scored_attn_bwd_packed(h, self.score, self.packed, o, lse, self.d_o, self.scale, dqkv, dt, ws)
                out.update(dq=dqkv[:, 0], dk=dqkv[:, 1], dv=dqkv[:, 2])
            else:
                Z.scored_attn_bwd(h, self.score, self.q, self.k, self.v, o, lse, self.d_o, self.scale, out["dq"], out["dk"], out["dv"], dt, ws)
        status_ok(h)
        return out


def check_all(run, problems, s, q, k, v, d_o, scale, heads=None, ds_roundings=1):
    o, lse = run.forward()
    f = R.forward(problems, q, k, v, scale, s, heads)
    covered = [torch.cat([p[0] for p in problems])] if heads is None else None
    used = {}
    if covered is not None:
        rows = covered[0]
        used["o"] = R.check(o.cpu()[rows], {"o": f["o"][rows], "o_err": f["o_err"][rows]}, "o")
        used["lse"] = R.check(lse.cpu()[:, rows], {"lse": f["lse"][:, rows], "lse_err": f["lse_err"][:, rows]}, "lse")
    got = run.backward(d_o)
    b = R.backward(problems, q, k, v, o.cpu(), lse.cpu(), d_o, scale, s, heads, ds_roundings)
    for name in got:
        if name == "dtable" or heads is None:
            g = got[name]
            if name in ("dk", "dv"):
                keys = torch.unique(torch.cat([p[1] for p in problems if len(p[0])] or [torch.zeros(0, dtype=torch.long)]))
                used[name] = R.check(g.cpu()[keys], {name: b[name][keys], name + "_err": b[name + "_err"][keys]}, name)
            elif name == "dq":
                used[name] = R.check(g.cpu()[covered[0]], {name: b[name][covered[0]], name + "_err": b[name + "_err"][covered[0]]}, name)
            else:
                used[name] = R.check(g, b, name)
    return used, f, b, got


def whole_problems(lens, prefix):
    out, at = [], 0
    for n, p in zip(lens, prefix):
        i = torch.arange(at, at + n)
        out.append((i, i, torch.arange(n), torch.arange(n), p))
        at += n
    return out


def cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


LENS = [1, 2, 127, 128, 129, 31, 257, 33, 0, 64]
KINDS = {
    "mask": dict(masked=True),
    "cap": dict(cap=7.0),
    "cap_mask": dict(cap=30.0, masked=True),
    "slopes": dict(slopes=True),
    "slopes_mask": dict(slopes=True, masked=True),
    "buckets": dict(buckets=32, reach=128),
    "buckets_mask": dict(buckets=17, reach=40, masked=True),
    "one_bucket": dict(buckets=1, reach=0),
    "symmetric": dict(buckets=5, reach=70, symmetric=True),
    "wide": dict(buckets=64, reach=300),
    "all": dict(cap=9.0, slopes=True, buckets=40, reach=60, masked=True),
}


@pytest.mark.parametrize("d,H", [(64, 3), (128, 2)])
@pytest.mark.parametrize("kind", list(KINDS))
def test_whole_sequences(kind, d, H):
    import paper_2608_01150_b200 as Z
    g = torch.Generator().manual_seed(7 + d)
    s = make_score(g, H, **KINDS[kind])
    T = sum(LENS)
    q, k, v, d_o = rand(g, T, H, d, times=2.0), rand(g, T, H, d), rand(g, T, H, d), rand(g, T, H, d)
    prefix = [0, 5, 1, 64, 0, 31, 130, 7, 4, 63]
    h = Z.build_tasks(cu(LENS), [], T, T, H, d)
    if s["masked"]:
        h.set_positions(whole_prefix=prefix)
    run = Run(h, s, q, k, v, d ** -0.5)
    check_all(run, whole_problems(LENS, prefix), s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("kind", ["mask", "all", "wide"])
def test_long_sequence_many_tiles(kind):
    """Rows whose far keys lie many tiles away, tiles that stop before others, items of unequal work."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 128, 1, [1500, 900]
    g = torch.Generator().manual_seed(11)
    s = make_score(g, H, **KINDS[kind])
    T = sum(lens)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    if s["masked"]:
        h.set_positions(whole_prefix=[300, 0])
    check_all(Run(h, s, q, k, v, d ** -0.5), whole_problems(lens, [300, 0]), s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("cap,times", [(50.0, 1.0), (5.0, 6.0), (0.5, 30.0)])
def test_cap_near_and_far_from_saturation(cap, times):
    """Both forms of the tanh, scores deep in saturation included (dC/dx = 0 there)."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 64, 2, [200]
    g = torch.Generator().manual_seed(5)
    q, k, v, d_o = rand(g, 200, H, d, times=times), rand(g, 200, H, d), rand(g, 200, H, d), rand(g, 200, H, d)
    h = Z.build_tasks([0, 200], [], 200, 200, H, d)
    s = dict(cap=cap)
    check_all(Run(h, s, q, k, v, d ** -0.5), whole_problems(lens, [0]), s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("value", [-math.inf, torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, -1e30])
def test_bucket_entries_that_remove_pairs(value):
    """The farther buckets of one head removed; one sequence short enough to keep all, one row keeps only itself."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 64, 2, [150, 3]
    g = torch.Generator().manual_seed(6)
    s = make_score(g, H, buckets=9, reach=4)
    s["table"][:4, 0] = value
    s["table"][5:, 0] = value       # head 0: only distance 0 stays
    s["table"][8, 1] = value        # head 1: nothing 4 or more behind
    q, k, v, d_o = (rand(g, 153, H, d) for _ in range(4))
    h = Z.build_tasks(cu(lens), [], 153, 153, H, d)
    run = Run(h, s, q, k, v, d ** -0.5)
    _, f, _, got = check_all(run, whole_problems(lens, [0, 0]), s, q, k, v, d_o, d ** -0.5)
    assert torch.equal(run.o[:, 0].cpu(), v[:, 0])
    assert (got["dtable"][:4, 0] == 0).all()


@pytest.mark.parametrize("lens", [[300, 5], [1, 60, 128]])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("by", ["slopes", "table"])
def test_largest_biases_leave_every_row_its_own_key(by, cap, lens):
    """Biases at the documented limits outweigh every product: P is the identity, so O = V and dV = dO to the bit, and what is
    left of dQ and dK is the rounding of dO.V - D (products of bf16 are exact, d additions each, D once more)."""
    import paper_2608_01150_b200 as Z
    d, H, scale, reach = 64, 2, 0.125, 3
    g = torch.Generator().manual_seed(34)
    T = sum(lens)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    s = dict(cap=cap, masked=False)
    if by == "slopes":
        s["slopes"] = torch.tensor([1e18, 1e6])
    else:
        s["table"] = torch.tensor([[-9e29, -1e6], [0.0, 0.0]])
        s["bucket_of"] = (torch.arange(-reach, reach + 1) == 0).to(torch.int32)
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    run = Run(h, s, q, k, v, scale)
    o, lse = run.forward()
    assert torch.equal(o.cpu(), v)
    x = (q.double() * k.double()).sum(-1) * scale
    x = cap * torch.tanh(x / cap) if cap else x
    assert (lse.cpu().double().T - x).abs().max() <= 1e-4  # |x| < 16: 2^-20 for each of a few roundings and the exponent's base
    got = run.backward(d_o)
    assert torch.equal(got["dv"].cpu(), d_o)
    noise = (2 * d + 4) * 2.0 ** -23 * (d_o.double() * v.double()).abs().sum(-1, keepdim=True) * scale
    for name, other in (("dq", k), ("dk", q)):
        assert (got[name].cpu().double().abs() <= noise * other.double().abs() * 1.01 + 1e-30).all()
    if by == "table":  # all of it in the diagonal's bucket
        assert got["dtable"][0].abs().max() == 0
        assert (got["dtable"][1].cpu().double().abs() <= noise.sum(0)[:, 0] / scale).all()


def test_every_pair_removed_leaves_empty_rows():
    import paper_2608_01150_b200 as Z
    d, H, T = 128, 2, 140
    g = torch.Generator().manual_seed(8)
    s = dict(table=torch.tensor([[-math.inf, 0.0]]), bucket_of=torch.zeros(1, dtype=torch.int32))
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, T], [], T, T, H, d)
    run = Run(h, s, q, k, v, d ** -0.5)
    check_all(run, whole_problems([T], [0]), s, q, k, v, d_o, d ** -0.5)
    assert (run.o[:, 0] == 0).all() and torch.isneginf(run.lse[0]).all()


def test_bucket_numbers_outside_the_table_mean_no_bias():
    import paper_2608_01150_b200 as Z
    d, H, T = 64, 1, 100
    g = torch.Generator().manual_seed(9)
    s = make_score(g, H, buckets=3, reach=3)
    s["bucket_of"] = torch.tensor([-1, 2, 0, 3, 1, 1000000, -2 ** 31], dtype=torch.int32)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, T], [], T, T, H, d)
    check_all(Run(h, s, q, k, v, d ** -0.5), whole_problems([T], [0]), s, q, k, v, d_o, d ** -0.5)


# ------------------------------------------------------------------------------------------------- shards
@pytest.mark.parametrize("kind", ["mask", "slopes_mask", "all", "buckets"])
@pytest.mark.parametrize("flags", [0, 1])
def test_chunks_of_one_sequence(kind, flags):
    """A 600-token sequence as 3 query chunks x 4 key chunks beside a whole sequence: some chunks are wholly in a row's
    future, and the positions say so (the KV-space order of the chunks is another).  Fused into one task with flags=1."""
    import paper_2608_01150_b200 as Z
    d, H = 64, 2
    g = torch.Generator().manual_seed(12)
    s = make_score(g, H, **KINDS[kind])
    whole, L, cq, ck, prefix = 50, 600, 200, 150, 20
    order = [0, 1, 2, 3] if flags else [2, 0, 3, 1]       # where key chunk c lies in KV-space
    shards, pos = [], []
    for qi in range(3):
        for c in range(4):
            shards.append((whole + qi * cq, cq, whole + order[c] * ck, ck, 0))
            pos.append((qi * cq, c * ck, prefix))
    T = whole + L
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, whole], shards, T, T, H, d, flags=flags)
    assert (h.info.n_fused_ranges > 0) == bool(flags)
    h.set_positions([3], pos)
    i = torch.arange(whole)
    problems = [(i, i, i, i, 3)]
    keys = torch.cat([torch.arange(whole + order[c] * ck, whole + (order[c] + 1) * ck) for c in range(4)])
    problems.append((torch.arange(whole, T), keys, torch.arange(L), torch.arange(L), prefix))
    check_all(Run(h, s, q, k, v, d ** -0.5), problems, s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("rows", [1, 3])
def test_single_tokens_against_chunks_at_far_positions(rows):
    """One to three new tokens against a long past in five ragged chunks, near the end of the 32-bit positions; the last
    chunk holds keys after some of the rows, one chunk is wholly in the future, one is empty."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 128, 3, [257, 1, 640, 130, 0, 60]
    g = torch.Generator().manual_seed(13)
    s = make_score(g, H, slopes=True, buckets=12, reach=300, masked=True)
    base = 2 ** 31 - 513 - 1088
    K = sum(lens)
    q, k, v, d_o = rand(g, rows, H, d), rand(g, K, H, d), rand(g, K, H, d), rand(g, rows, H, d)
    at, shards, pos = 0, [], []
    for n in lens:
        shards.append((0, rows, at, n, 0))
        pos.append((base + 1000, base + at, 0))
        at += n
    h = Z.build_tasks([0], shards, rows, K, H, d)
    h.set_positions(None, pos)
    problems = [(torch.arange(rows), torch.arange(K), base + 1000 + torch.arange(rows), base + torch.arange(K), 0)]
    check_all(Run(h, s, q, k, v, d ** -0.5), problems, s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("rows,chunk,H,masked", [(1, 5000, 2, True), (1, 5000, 2, False), (17, 2100, 3, True), (64, 1300, 1, False)])
def test_long_chunks_cut_along_the_keys(rows, chunk, H, masked):
    """Few rows against chunks so long that the kernel takes them in pieces: each shard's slot holds its whole partial result,
    the merge the whole result, with the same bits launch after launch and replay after replay."""
    import paper_2608_01150_b200 as Z
    d = 128
    g = torch.Generator().manual_seed(31)
    K = 2 * chunk
    q, k, v = rand(g, rows, H, d), rand(g, K, H, d), rand(g, K, H, d)
    s = dict(masked=masked, slopes=torch.tensor([0.002 * (i + 1) for i in range(H)]))
    h = Z.build_tasks([0], [(0, rows, 0, chunk, 0), (0, rows, chunk, chunk, 0)], rows, K, H, d)
    pos = K - rows if masked else 100
    h.set_positions(None, [(pos, 0, 0), (pos, chunk, 0)])
    run = Run(h, s, q, k, v, d ** -0.5)
    f = R.forward([(torch.arange(rows), torch.arange(K), pos + torch.arange(rows), torch.arange(K), 0)], q, k, v, d ** -0.5, s)
    o, lse = run.forward()
    R.check(o, f, "o")
    R.check(lse, f, "lse")
    # each slot against its own chunk
    pr = int(h.info.partial_rows)
    op, lp = torch.full((pr, H, d), SENTINEL, device="cuda"), torch.full((H, pr), SENTINEL, device="cuda")
    Z.scored_attn_fwd(h, run.score, run.q, run.k, run.v, run.scale, o, lse, op, lp)
    status_ok(h)
    for c in range(2):
        keys = torch.arange(c * chunk, (c + 1) * chunk)
        part = R.forward([(torch.arange(rows), keys, pos + torch.arange(rows), keys, 0)], q, k, v, d ** -0.5, s)
        at, _ = h.partial_slot(c)
        R.check(op[at:at + rows], {"o": part["o"], "o_err": part["o_err"]}, "o")
        R.check(lp[:, at:at + rows], part, "lse")
    first = op.clone(), lp.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Z.scored_attn_fwd(h, run.score, run.q, run.k, run.v, run.scale, o, lse, op, lp)
    for _ in range(3):
        op.fill_(SENTINEL)
        lp.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        for c in range(2):
            at, _ = h.partial_slot(c)
            assert torch.equal(op[at:at + rows], first[0][at:at + rows]) and torch.equal(lp[:, at:at + rows], first[1][:, at:at + rows])
    status_ok(h)


def test_masked_calls_with_an_sm_margin():
    """The dealt lists are for all SMs; with a margin the plain lists run, with the same results."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 64, 2, [700, 300]
    g = torch.Generator().manual_seed(32)
    T = sum(lens)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    s = dict(masked=True)
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    h.set_positions([0, 50])
    run = Run(h, s, q, k, v, d ** -0.5)
    problems = whole_problems(lens, [0, 50])
    check_all(run, problems, s, q, k, v, d_o, d ** -0.5)
    for margin in (140, 146):
        h.set_sm_margin(margin)
        check_all(run, problems, s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("lens,chunks,H", [([700, 1, 300, 130], [], 3), ([60, 128, 5], [], 2), ([], [3000, 2000], 2)])
def test_unmasked_calls_with_an_sm_margin(lens, chunks, H):
    """Which CTA takes an item changes no bit of the forward: all SMs by dealt lists, few SMs in turn."""
    import paper_2608_01150_b200 as Z
    d, scale = 64, 0.125
    g = torch.Generator().manual_seed(33)
    rows, keys = (sum(lens), sum(lens)) if lens else (7, sum(chunks))
    q, d_o = rand(g, rows, H, d), rand(g, rows, H, d)
    k, v = rand(g, keys, H, d), rand(g, keys, H, d)
    s = make_score(g, H, cap=20.0, buckets=8, reach=40)
    if lens:
        h = Z.build_tasks(cu(lens), [], rows, keys, H, d)
        h.set_positions([0] * len(lens))
        problems = whole_problems(lens, [0] * len(lens))
    else:
        h = Z.build_tasks([0], [(0, rows, sum(chunks[:i]), n, 0) for i, n in enumerate(chunks)], rows, keys, H, d)
        h.set_positions(None, [(2900, sum(chunks[:i]), 0) for i in range(len(chunks))])
        problems = [(torch.arange(rows), torch.arange(keys), 2900 + torch.arange(rows), torch.arange(keys), 0)]
    run = Run(h, s, q, k, v, scale)
    check_all(run, problems, s, q, k, v, d_o, scale)
    o, lse = run.o.clone(), run.lse.clone()
    for margin in (8, 145):
        h.set_sm_margin(margin)
        check_all(run, problems, s, q, k, v, d_o, scale)
        assert torch.equal(run.o, o) and torch.equal(run.lse, lse)


def test_rows_that_see_no_chunk_at_all():
    import paper_2608_01150_b200 as Z
    d, H, rows, K = 64, 2, 140, 300
    g = torch.Generator().manual_seed(14)
    s = dict(masked=True, slopes=torch.tensor([0.5, 0.0]))
    q, k, v, d_o = rand(g, rows, H, d), rand(g, K, H, d), rand(g, K, H, d), rand(g, rows, H, d)
    h = Z.build_tasks([0], [(0, rows, 0, K, 0)], rows, K, H, d)
    h.set_positions(None, [(0, 130, 0)])        # rows 0..129 come before every key
    problems = [(torch.arange(rows), torch.arange(K), torch.arange(rows), 130 + torch.arange(K), 0)]
    run = Run(h, s, q, k, v, d ** -0.5)
    _, _, _, got = check_all(run, problems, s, q, k, v, d_o, d ** -0.5)
    assert (run.o[:130] == 0).all() and torch.isneginf(run.lse[:, :130]).all() and (got["dq"][:130] == 0).all()
    assert (got["dk"][10:] == 0).all() and (got["dv"][10:] == 0).all()     # keys that no row sees


# ------------------------------------------------------------------------------------------------- layouts
def test_packed_equals_separate_and_rows_outside_tasks_stay():
    import paper_2608_01150_b200 as Z
    d, H, lens, T = 128, 2, [130, 70], 260                                 # 60 rows that no task covers
    g = torch.Generator().manual_seed(15)
    s = make_score(g, H, **KINDS["all"])
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    h.set_positions([0, 10])
    a, b = Run(h, s, q, k, v, d ** -0.5), Run(h, s, q, k, v, d ** -0.5, packed=True)
    (oa, la), (ob, lb) = a.forward(), b.forward()
    assert torch.equal(oa, ob) and torch.equal(la, lb)
    ga, gb = a.backward(d_o), b.backward(d_o, oa, la)
    for n in ("dk", "dv", "dtable"):
        assert torch.equal(ga[n], gb[n]), n
    for n in ("dq", "dk", "dv"):
        assert (ga[n][200:] == SENTINEL).all() and (gb[n][200:] == SENTINEL).all(), n
    assert (oa[200:] == SENTINEL).all() and (la[:, 200:] == SENTINEL).all()


def test_head_ranges():
    """Two sequences on the same rows with disjoint heads, a third on all: each head's bias is its own, heads without a
    task keep a zero share of the table's gradient."""
    import paper_2608_01150_b200 as Z
    d, H, T = 64, 4, 330
    g = torch.Generator().manual_seed(16)
    s = make_score(g, H, **KINDS["all"])
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    whole = [(0, 130, 0, 1), (0, 130, 2, 1), (130, 200, 0, 3)]
    h = Z.build_tasks_heads(whole, [], None, T, T, H, d)
    h.set_positions([4, 9, 0])
    problems, heads = [], []
    for (off, n, hb, hc), p in zip(whole, [4, 9, 0]):
        i = torch.arange(off, off + n)
        problems.append((i, i, torch.arange(n), torch.arange(n), p))
        heads.append(range(hb, hb + hc))
    run = Run(h, s, q, k, v, d ** -0.5)
    _, f, b, got = check_all(run, problems, s, q, k, v, d_o, d ** -0.5, heads=heads)
    for (off, n, hb, hc) in whole:
        for x, ref in ((run.o, f), (got["dq"], b), (got["dk"], b), (got["dv"], b)):
            name = {id(run.o): "o", id(got["dq"]): "dq", id(got["dk"]): "dk", id(got["dv"]): "dv"}[id(x)]
            sl = (slice(off, off + n), slice(hb, hb + hc))
            R.check(x[sl], {name: ref[name][sl], name + "_err": ref[name + "_err"][sl]}, name)
    assert (run.o[:130, 1] == SENTINEL).all() and (run.o[:, 3] == SENTINEL).all() and (got["dk"][:, 3] == SENTINEL).all()
    assert (got["dtable"][:, 3] == 0).all()


def test_no_score_is_the_plain_call():
    import paper_2608_01150_b200 as Z
    d, H, T = 128, 2, 300
    g = torch.Generator().manual_seed(17)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, 100, T], [], T, T, H, d)
    a, b = Run(h, {}, q, k, v, d ** -0.5), Run(h, {}, q, k, v, d ** -0.5, plain=True)
    (oa, la), (ob, lb) = a.forward(), b.forward()
    assert torch.equal(oa, ob) and torch.equal(la, lb)
    ga, gb = a.backward(d_o), b.backward(d_o)
    assert torch.equal(ga["dk"], gb["dk"]) and torch.equal(ga["dv"], gb["dv"])


def test_rows_behind_four_gigabytes():
    """Keys whose byte offset passes 32 bits and whose element offset passes 31."""
    import paper_2608_01150_b200 as Z
    d, H, K, n = 128, 40, 460000, 300
    g = torch.Generator().manual_seed(18)
    k = torch.zeros(K, H, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    kt, vt, q, d_o = rand(g, n, H, d), rand(g, n, H, d), rand(g, 2, H, d), rand(g, 2, H, d)
    k[K - n:], v[K - n:] = kt.cuda(), vt.cuda()
    s = dict(masked=True, slopes=torch.tensor([0.9 ** i for i in range(H)]))
    h = Z.build_tasks([0], [(0, 2, K - n, n, 0)], 2, K, H, d)
    h.set_positions(None, [(n - 2, 0, 0)])
    run = Run(h, s, q, kt, vt, d ** -0.5)
    run.k, run.v = k, v
    o, lse = run.forward()
    problems = [(torch.arange(2), torch.arange(n), n - 2 + torch.arange(2), torch.arange(n), 0)]
    f = R.forward(problems, q, kt, vt, d ** -0.5, s)
    R.check(o, f, "o")
    R.check(lse, f, "lse")
    got = run.backward(d_o)
    b = R.backward(problems, q, kt, vt, o.cpu(), lse.cpu(), d_o, d ** -0.5, s)
    R.check(got["dq"], b, "dq")
    R.check(got["dk"][K - n:], b, "dk")
    R.check(got["dv"][K - n:], b, "dv")
    assert (got["dk"][K - n - 1] == SENTINEL).all()


# ------------------------------------------------------------------------------------------------- use
def test_same_bits_every_time_and_under_capture():
    """Eager twice, then captured and replayed with other inputs and another table in the same tensors; backward too."""
    import paper_2608_01150_b200 as Z
    d, H, lens = 64, 3, [257, 129, 40]
    T = sum(lens)
    g = torch.Generator().manual_seed(19)
    s = make_score(g, H, **KINDS["all"])
    data = [[rand(g, T, H, d).cuda() for _ in range(4)] + [torch.randn(40, H, generator=g).cuda()] for _ in range(2)]
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    h.set_positions([0, 3, 40])
    sc = to_score(Z, s)
    q, k, v, d_o = (x.clone() for x in data[0][:4])
    sc.bucket_bias.copy_(data[0][4])
    o, dq, dk, dv = (torch.empty_like(q) for _ in range(4))
    lse, dt = torch.empty(H, T, device="cuda"), torch.empty_like(sc.bucket_bias)
    ws = torch.empty(h.scored_workspace_bytes(sc), dtype=torch.uint8, device="cuda")

    def step():
        Z.scored_attn_fwd(h, sc, q, k, v, 0.125, o, lse)
        Z.scored_attn_bwd(h, sc, q, k, v, o, lse, d_o, 0.125, dq, dk, dv, dt, ws)

    def load(i):
        for t, x in zip((q, k, v, d_o, sc.bucket_bias), data[i]):
            t.copy_(x)

    want = []
    for i in (0, 1):
        load(i)
        step()
        torch.cuda.synchronize()
        want.append([x.clone() for x in (o, lse, dk, dv, dt, dq)])
    load(0)
    step()
    torch.cuda.synchronize()
    for a, b in zip(want[0][:5], (o, lse, dk, dv, dt)):
        assert torch.equal(a, b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in (1, 0, 1):
        load(i)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want[i][:5], (o, lse, dk, dv, dt)):
            assert torch.equal(a, b)
        assert torch.allclose(want[i][5].float(), dq.float(), atol=2e-2, rtol=2e-2)     # dQ: order of the fp32 reduce-adds
    status_ok(h)


def test_two_streams_with_their_own_handles_and_workspaces():
    import paper_2608_01150_b200 as Z
    d, H, lens = 128, 2, [300, 200]
    T = sum(lens)
    g = torch.Generator().manual_seed(20)
    runs = []
    for i in range(2):
        s = make_score(g, H, **KINDS["all"])
        q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
        h = Z.build_tasks(cu(lens), [], T, T, H, d)
        h.set_positions([i, 7])
        run = Run(h, s, q, k, v, d ** -0.5)
        run.forward()
        runs.append((run, d_o, run.backward(d_o), run.o, run.lse))
    streams = [torch.cuda.Stream() for _ in runs]
    outs = []
    for (run, d_o, _, o, lse), st in zip(runs, streams):
        with torch.cuda.stream(st):
            ws = torch.empty(run.h.scored_workspace_bytes(run.score), dtype=torch.uint8, device="cuda")
            res = [torch.empty_like(x) for x in (run.q, run.k, run.v)] + [torch.empty_like(run.score.bucket_bias)]
            o2, l2 = torch.empty_like(o), torch.empty_like(lse)
            outs.append((o2, l2, res, ws))
    torch.cuda.synchronize()
    for _ in range(3):
        for (run, _, _, _, _), st, (o2, l2, res, ws) in zip(runs, streams, outs):
            Z.scored_attn_fwd(run.h, run.score, run.q, run.k, run.v, run.scale, o2, l2, stream=st)
            Z.scored_attn_bwd(run.h, run.score, run.q, run.k, run.v, o2, l2, run.d_o, run.scale, *res, ws, stream=st)
    torch.cuda.synchronize()
    for (run, _, want, o, lse), (o2, l2, res, _) in zip(runs, outs):
        assert torch.equal(o, o2) and torch.equal(lse, l2)
        assert torch.equal(want["dk"], res[1]) and torch.equal(want["dv"], res[2]) and torch.equal(want["dtable"], res[3])


def test_positions_can_change_and_leave_plain_calls_alone():
    import paper_2608_01150_b200 as Z
    d, H, T = 64, 2, 400
    g = torch.Generator().manual_seed(21)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, T], [], T, T, H, d)
    plain = Run(h, {}, q, k, v, d ** -0.5, plain=True)
    o0, l0 = plain.forward()
    s = dict(masked=True)
    for prefix in (0, 250, 400):
        h.set_positions([prefix])
        check_all(Run(h, s, q, k, v, d ** -0.5), whole_problems([T], [prefix]), s, q, k, v, d_o, d ** -0.5)
    o1, l1 = plain.forward()
    assert torch.equal(o0, o1) and torch.equal(l0, l1)


@pytest.mark.parametrize("lens", [[400, 900], [130, 70]])
def test_captured_masked_calls_follow_new_positions(lens):
    """Forward and backward captured under one mask, replayed under others: the results of eager calls with those."""
    import paper_2608_01150_b200 as Z
    d, H, T = 64, 2, sum(lens)
    g = torch.Generator().manual_seed(33)
    q, k, v, d_o = (rand(g, T, H, d).cuda() for _ in range(4))
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    h.set_positions([0, 0])
    sc = Z.Score(masked=True)
    o, dq, dk, dv = (torch.empty_like(q) for _ in range(4))
    lse = torch.empty(H, T, device="cuda")
    ws = torch.empty(h.scored_workspace_bytes(sc), dtype=torch.uint8, device="cuda")

    def step():
        Z.scored_attn_fwd(h, sc, q, k, v, 0.125, o, lse)
        Z.scored_attn_bwd(h, sc, q, k, v, o, lse, d_o, 0.125, dq, dk, dv, None, ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for prefix in ([0, 0], [lens[0], 0], [7, lens[1]], [lens[0], lens[1]], [0, 0]):
        h.set_positions(prefix)
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (o, lse, dk, dv)]
        for x in (o, lse, dk, dv):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (o, lse, dk, dv)):
            assert torch.equal(a, b), prefix
    status_ok(h)


def test_refusals_on_the_device():
    import paper_2608_01150_b200 as Z
    h = Z.build_tasks([0, 10], [], 10, 10, 2, 64)
    x = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    lse, f = torch.zeros(2, 10, device="cuda"), torch.zeros(64, device="cuda")
    s = Z.Score(cap=3.0)
    ws = torch.zeros(h.scored_workspace_bytes(s), dtype=torch.uint8, device="cuda")

    def status(fn, *a):
        with pytest.raises(Z.ZlError) as e:
            fn(*a)
        return e.value.status

    assert status(Z.scored_attn_fwd, h, s, 0, x, x, 1.0, x, lse) == 1
    assert status(Z.scored_attn_fwd, h, s, x, x, x, 0.0, x, lse) == 1
    assert status(Z.scored_attn_fwd, h, s, x.data_ptr() + 2, x, x, 1.0, x, lse) == 1
    assert status(Z.scored_attn_fwd, h, Z.Score(masked=True), x, x, x, 1.0, x, lse) == 1
    assert status(Z.scored_attn_fwd, h, Z.Score(slopes=torch.zeros(2)), x, x, x, 1.0, x, lse) == 1             # slopes on the host
    assert status(Z.scored_attn_fwd, h, Z.Score(cap=1e-4), x, x, x, 3e38, x, lse) == 1                          # scale / cap overflows
    assert status(Z.scored_attn_bwd, h, s, x, x, x, x, lse, x, 1.0, x, x, x, f, ws) == 1            # a table's gradient without a table
    assert status(Z.scored_attn_bwd, h, s, x, x, x, x, lse, x, 1.0, x, x, x, None, ws[:-4]) == 4
    assert status(Z.scored_attn_bwd, h, s, x, x, x, x, lse, x, 1.0, x, x, x, None, ws[16:], ws.numel()) == 1
    status_ok(h)


# ------------------------------------------------------------------------------------------------- shared prefix
def prefix_problems(qlens, klens, P):
    out, qa, ka = [], 0, P
    for ql, kl in zip(qlens, klens):
        keys = torch.cat([torch.arange(P), torch.arange(ka, ka + kl)])
        zeros = lambda n: torch.zeros(n, dtype=torch.long)  # noqa: E731
        out.append((torch.arange(qa, qa + ql), keys, zeros(ql), zeros(len(keys)), 0))
        qa, ka = qa + ql, ka + kl
    return out


@pytest.mark.parametrize("qlens,klens,P,H,d", [
    ([1] * 37, [1 + 5 * i for i in range(37)], 700, 2, 128),       # one token each, ragged own keys
    ([1] * 130, [0] * 130, 1025, 1, 64),                            # nothing of their own, two row tiles
    ([100, 1, 0, 257, 64, 130], [100, 1, 9, 257, 0, 300], 640, 2, 128),
    ([3, 129, 128], [3, 129, 128], 1, 3, 64),
    ([5, 40], [70, 0], 0, 2, 128),                                  # no prefix: the second sequence has no key
    ([300], [200], 300, 1, 64),                                     # a batch of one
    ([2, 200, 1], [2, 200, 1], 4000, 1, 128),
])
def test_shared_prefix(qlens, klens, P, H, d):
    import paper_2608_01150_b200 as Z
    g = torch.Generator().manual_seed(22)
    nq, nk = sum(qlens) + 9, P + sum(klens) + 11                    # rows behind the batch stay as they are
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
    run = Run(h, {}, q, k, v, d ** -0.5, plain=True)
    problems = prefix_problems(qlens, klens, P)
    _, f, _, got = check_all(run, problems, {}, q, k, v, d_o, d ** -0.5, ds_roundings=3)
    assert (run.o[sum(qlens):] == SENTINEL).all() and (run.lse[:, sum(qlens):] == SENTINEL).all()
    assert (got["dq"][sum(qlens):] == SENTINEL).all()
    assert (got["dk"][P + sum(klens):] == SENTINEL).all() and (got["dv"][P + sum(klens):] == SENTINEL).all()
    at = P
    for ql, kl in zip(qlens, klens):
        if ql == 0:
            assert (got["dk"][at:at + kl] == SENTINEL).all()
        at += kl


@pytest.mark.parametrize("s", [dict(cap=6.0), dict(masked=True), dict(cap=20.0, masked=True)])
def test_shared_prefix_with_scores(s):
    """Among a sequence's own rows the mask is causal with a prefix of its own; the shared prefix is seen whole."""
    import paper_2608_01150_b200 as Z
    d, H, P, qlens, klens = 128, 2, 520, [30, 1, 140], [50, 1, 140]
    g = torch.Generator().manual_seed(23)
    nq, nk = sum(qlens), P + sum(klens)
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
    own = [(20, 0, 0), (0, 0, 0), (0, 0, 33)]
    if s.get("masked"):
        h.set_positions(shard_pos=own)
    problems, qa, ka = [], 0, P
    for ql, kl, (qp, kp, pre) in zip(qlens, klens, own):
        keys = torch.cat([torch.arange(P), torch.arange(ka, ka + kl)])
        # shared keys at positions before everything
        problems.append((torch.arange(qa, qa + ql), keys, P + qp + torch.arange(ql), torch.cat([torch.arange(P), P + kp + torch.arange(kl)]), P + pre))
        qa, ka = qa + ql, ka + kl
    check_all(Run(h, s, q, k, v, d ** -0.5), problems, s, q, k, v, d_o, d ** -0.5)


def test_shared_prefix_both_backward_kernels_and_a_captured_step():
    import paper_2608_01150_b200 as Z
    d, H, P, lens = 128, 2, 1100, [20, 1, 300]
    g = torch.Generator().manual_seed(24)
    nq, nk = sum(lens), P + sum(lens)
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    problems = prefix_problems(lens, lens, P)
    for kernel in (1, 2):
        h = Z.build_tasks_prefix(cu(lens), cu(lens), P, nq, nk, H, d)
        h.set_bwd_kernel(kernel)
        run = Run(h, {}, q, k, v, d ** -0.5, plain=True)
        _, _, _, want = check_all(run, problems, {}, q, k, v, d_o, d ** -0.5, ds_roundings=3)
    pr = int(h.info.partial_rows)
    op, lp = torch.empty(pr, H, d, device="cuda"), torch.empty(H, pr, device="cuda")
    o, lse = torch.empty_like(run.q), torch.empty(H, nq, device="cuda")
    dq, dk, dv = torch.empty_like(run.q), torch.empty_like(run.k), torch.empty_like(run.k)
    ws = torch.empty(int(h.info.bwd_workspace_bytes), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Z.coalesced_attn_fwd(h, run.q, run.k, run.v, d ** -0.5, o, lse, op, lp)
        Z.lse_merge(h, op, lp, o, lse)
        Z.coalesced_attn_bwd(h, run.q, run.k, run.v, o, lse, run.d_o, d ** -0.5, dq, dk, dv, ws)
    for _ in range(2):
        for t in (o, lse, dk, dv):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, run.o) and torch.equal(lse, run.lse) and torch.equal(dk, want["dk"]) and torch.equal(dv, want["dv"])
    status_ok(h)


def test_shared_prefix_in_phases_and_without_a_workspace():
    """Own parts in a later launch phase than the prefix; the backward in phases and with the library's own scratch."""
    import paper_2608_01150_b200 as Z
    d, H, P, lens = 64, 2, 900, [40, 1, 200]
    g = torch.Generator().manual_seed(25)
    nq, nk = sum(lens), P + sum(lens)
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    problems = prefix_problems(lens, lens, P)
    f = R.forward(problems, q, k, v, d ** -0.5, {})
    h = Z.build_tasks_prefix(cu(lens), cu(lens), P, nq, nk, H, d)
    h.set_fwd_phases(None, [1, 1, 1], 2)
    h.set_bwd_phases(None, [1, 1, 1], 2)
    run = Run(h, {}, q, k, v, d ** -0.5, plain=True)
    pr = int(h.info.partial_rows)
    op, lp = torch.full((pr, H, d), SENTINEL, device="cuda"), torch.full((H, pr), SENTINEL, device="cuda")
    o, lse = torch.empty_like(run.q), torch.empty(H, nq, device="cuda")
    for phase in (1, 0):
        Z.coalesced_attn_fwd_phase(h, phase, run.q, run.k, run.v, d ** -0.5, o, lse, op, lp)
    Z.lse_merge(h, op, lp, o, lse)
    status_ok(h)
    R.check(o, f, "o")
    R.check(lse, f, "lse")
    b = R.backward(problems, q, k, v, o.cpu(), lse.cpu(), d_o, d ** -0.5, {}, ds_roundings=1)
    ws = torch.full((int(h.info.bwd_workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
    dd = d_o.cuda()
    for noalloc in (False, True):
        dq, dk, dv = (torch.full_like(x, SENTINEL) for x in (run.q, run.k, run.v))
        if noalloc:
            Z.coalesced_attn_bwd_noalloc(h, run.q, run.k, run.v, o, lse, dd, d ** -0.5, dq, dk, dv)
        else:
            for phase in (0, 1):
                Z.coalesced_attn_bwd_phase(h, phase, run.q, run.k, run.v, o, lse, dd, d ** -0.5, dq, dk, dv, ws)
        status_ok(h)
        for name, x in (("dq", dq), ("dk", dk), ("dv", dv)):
            R.check(x, b, name)


def test_many_rows_over_a_short_prefix_and_one_row_over_a_long_one():
    """Row blocks of two query tiles, of one, and a handle whose prefix is cut into many chunks."""
    import paper_2608_01150_b200 as Z
    d = 128
    g = torch.Generator().manual_seed(26)
    for H, qlens, klens, P in ((2, [500, 600], [3, 0], 130), (2, [1], [0], 9000), (1, [2], [5], 33000), (2, [1, 1, 1], [128, 129, 1], 5000)):
        nq, nk = sum(qlens), P + sum(klens)
        q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
        h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
        check_all(Run(h, {}, q, k, v, d ** -0.5, plain=True), prefix_problems(qlens, klens, P), {}, q, k, v, d_o, d ** -0.5)
