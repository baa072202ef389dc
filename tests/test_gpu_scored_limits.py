"""Scored attention on the GPU where memory next to a task, numbers at their limits or several calls could reach results:
against the definition in 64 bits, with the bounds of scored_ref."""
import pytest
import torch

import scored_ref as R
from test_gpu_scored import KINDS, Run, check_all, cu, make_score, prefix_problems, rand, status_ok, whole_problems

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- neighbours
def poison(x, rows, every):
    """Huge finite values of both signs: products of two such rows overflow, their sums are NaN."""
    big = torch.full(x.shape[1:], 3e38)
    big.view(-1)[::every] *= -1
    x[rows] = big.to(x.dtype)


@pytest.mark.parametrize("kind", ["cap", "cap_mask", "slopes_mask", "all"])
@pytest.mark.parametrize("d", [64, 128])
def test_finite_neighbours_of_whole_sequences_and_shards_cannot_leak(kind, d):
    """Rows that no task owns, behind ragged sequences, shards and key chunks: tiles read them, results do not."""
    import paper_2608_01150_b200 as Z
    H, T = 2, 330
    g = torch.Generator().manual_seed(41)
    s = make_score(g, H, **KINDS[kind])
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    owned_q = list(range(0, 230)) + list(range(240, 290))
    owned_k = list(range(0, 230)) + list(range(240, 310))
    for x in (q, d_o):
        poison(x, [i for i in range(T) if i not in owned_q], 3)
    for x in (k, v):
        poison(x, [i for i in range(T) if i not in owned_k], 2)
    h = Z.build_tasks([0, 100, 230], [(240, 50, 240, 70, 0)], T, T, H, d)
    h.set_positions([3, 0], [(30, 0, 5)])
    problems = whole_problems([100, 130], [3, 0])
    problems.append((torch.arange(240, 290), torch.arange(240, 310), 30 + torch.arange(50), torch.arange(70), 5))
    check_all(Run(h, s, q, k, v, d ** -0.5), problems, s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("s", [dict(cap=6.0), dict(cap=20.0, masked=True), dict(masked=True)])
def test_finite_neighbours_of_a_shared_prefix_cannot_leak(s):
    """Keys of a sequence without queries lie behind a ragged key tile whose ragged query tile reaches into the next
    sequence: nothing of them arrives in any gradient."""
    import paper_2608_01150_b200 as Z
    d, H, P, qlens, klens = 128, 2, 520, [30, 0, 140], [50, 40, 140]
    g = torch.Generator().manual_seed(42)
    nq, nk = sum(qlens) + 20, P + sum(klens) + 20
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    for x in (k, v):
        poison(x, slice(P + 50, P + 90), 2)
        poison(x, slice(P + sum(klens), nk), 2)
    for x in (q, d_o):
        poison(x, slice(sum(qlens), nq), 3)
    h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
    own = [(20, 0, 0), (0, 0, 0), (0, 0, 33)]
    if s.get("masked"):
        h.set_positions(shard_pos=own)
    problems, qa, ka = [], 0, P
    for ql, kl, (qp, kp, pre) in zip(qlens, klens, own):
        if ql:
            keys = torch.cat([torch.arange(P), torch.arange(ka, ka + kl)])
            problems.append((torch.arange(qa, qa + ql), keys, P + qp + torch.arange(ql),
                             torch.cat([torch.arange(P), P + kp + torch.arange(kl)]), P + pre))
        qa, ka = qa + ql, ka + kl
    check_all(Run(h, s, q, k, v, d ** -0.5), problems, s, q, k, v, d_o, d ** -0.5)


# ------------------------------------------------------------------------------------------------- calls
def test_a_score_made_before_its_module_moves():
    """Made on the CPU, moved, given another table, a cap and a mask later: each call takes what is there."""
    import paper_2608_01150_b200 as Z
    d, H, T = 64, 2, 150
    g = torch.Generator().manual_seed(43)
    s = make_score(g, H, **KINDS["all"])
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    h = Z.build_tasks([0, T], [], T, T, H, d)
    h.set_positions([4])
    run = Run(h, s, q, k, v, d ** -0.5)
    module = torch.nn.Module()
    module.slopes, module.table = torch.nn.Parameter(s["slopes"].clone()), torch.nn.Parameter(s["table"].clone())
    run.score = Z.Score(slopes=module.slopes, bucket_bias=module.table, bucket_of=s["bucket_of"].cuda())
    module.cuda()
    run.score.cap, run.score.masked = s["cap"], True
    check_all(run, whole_problems([T], [4]), s, q, k, v, d_o, d ** -0.5)
    s["table"] = torch.randn(40, H, generator=g)
    module.table.data = s["table"].cuda()
    check_all(run, whole_problems([T], [4]), s, q, k, v, d_o, d ** -0.5)


def test_a_table_gradient_on_the_host_is_refused():
    import paper_2608_01150_b200 as Z
    h = Z.build_tasks([0, 10], [], 10, 10, 2, 64)
    x, lse = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 10, device="cuda")
    s = Z.Score(bucket_bias=torch.zeros(3, 2, device="cuda"), bucket_of=torch.zeros(3, dtype=torch.int32, device="cuda"))
    ws = torch.zeros(h.scored_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    for packed in (False, True):
        args = (torch.zeros(10, 3, 2, 64, dtype=torch.bfloat16, device="cuda"),) if packed else (x, x, x)
        fn = Z.scored_attn_bwd_packed if packed else Z.scored_attn_bwd
        with pytest.raises(Z.ZlError) as e:
            fn(h, s, *args, x, lse, x, 1.0, *(torch.zeros_like(a) for a in args), torch.zeros(3, 2), ws)
        assert e.value.status == 1


@pytest.mark.parametrize("cu_seqlens,shards", [([0], [(0, 0, 0, 10, 0)]), ([0, 0], [])])
def test_the_table_gradient_of_a_handle_without_queries_is_zero(cu_seqlens, shards):
    """A rank without query rows adds nothing to the sum over ranks."""
    import paper_2608_01150_b200 as Z
    h = Z.build_tasks(cu_seqlens, shards, 0, 10, 2, 64)
    x = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    none, lse = x[:0], torch.zeros(2, 0, device="cuda")
    s = Z.Score(bucket_bias=torch.ones(3, 2, device="cuda"), bucket_of=torch.zeros(3, dtype=torch.int32, device="cuda"))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    dt = torch.full((3, 2), 7.0, device="cuda")
    Z.scored_attn_fwd(h, s, none, x, x, 1.0, none, lse)
    Z.scored_attn_bwd(h, s, none, x, x, none, lse, none, 1.0, none, torch.zeros_like(x), torch.zeros_like(x), dt, ws)
    status_ok(h)
    assert (dt == 0).all()


# ------------------------------------------------------------------------------------------------- the cap's accuracy
def tight_scores(qh, kh, qpos, kpos, prefix, scale, cap=0.0, **kw):
    """scored_ref.scores with the header's bound on a capped score: 2^-20 of its own magnitude, whatever the cap and
    whatever other rows hold (scored_ref allows 2^-20 of the cap)."""
    s, slope, bucket, es = loose_scores(qh, kh, qpos, kpos, prefix, scale, cap=cap, **kw)
    capped = cap * torch.tanh(scale * (qh @ kh.T) / cap)
    return s, slope, bucket, es + 2.0 ** -20 * (capped.abs() - cap)


loose_scores = R.scores


@pytest.mark.parametrize("cap", [50.0, 1e3, 1e6])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("L,d", [(160, 64), (100, 128)])
def test_small_scores_beside_saturating_ones(L, d, slopes, cap, monkeypatch):
    """Every third query saturates the cap, in the same warps (and, backward, in the same registers) as queries whose scores are
    near zero: those keep their accuracy.  The saturating queries get no gradient of their own, so that dK and dV are the
    others'."""
    import paper_2608_01150_b200 as Z
    monkeypatch.setattr(R, "scores", tight_scores)
    H = 2
    g = torch.Generator().manual_seed(44)
    q, k, v, d_o = (rand(g, L, H, d) for _ in range(4))
    q[::3] = (q[::3].float() * cap).to(q.dtype)
    d_o[::3] = 0
    s = make_score(g, H, cap=cap, slopes=slopes)
    h = Z.build_tasks([0, L], [], L, L, H, d)
    check_all(Run(h, s, q, k, v, d ** -0.5), whole_problems([L], [0]), s, q, k, v, d_o, d ** -0.5)


@pytest.mark.parametrize("cap,slopes", [(0.5, False), (50.0, False), (0.5, True)])
def test_a_query_of_nan_stays_its_own_and_stays_nan(cap, slopes):
    """No clamp or maximum turns it into a number, and no other row of its warp notices."""
    import paper_2608_01150_b200 as Z
    d, H, L = 64, 2, 200
    g = torch.Generator().manual_seed(45)
    q, k, v = rand(g, L, H, d, times=2.0), rand(g, L, H, d), rand(g, L, H, d)
    s = make_score(g, H, cap=cap, slopes=slopes)
    h = Z.build_tasks([0, L], [], L, L, H, d)
    q[70, 1] = float("nan")
    o, lse = Run(h, s, q, k, v, d ** -0.5).forward()
    assert o[70, 1].isnan().all()
    f = R.forward(whole_problems([L], [0]), torch.nan_to_num(q), k, v, d ** -0.5, s)
    rows = [i for i in range(L) if i != 70]
    R.check(o.cpu()[rows], {"o": f["o"][rows], "o_err": f["o_err"][rows]}, "o")
    R.check(lse.cpu()[:, rows], {"lse": f["lse"][:, rows], "lse_err": f["lse_err"][:, rows]}, "lse")
    assert not o[70, 0].isnan().any()


# ------------------------------------------------------------------------------------------------- shared prefixes
@pytest.mark.parametrize("qlens,klens,P,H,d", [
    ([1] * 37, [1 + 5 * i for i in range(37)], 700, 2, 128), ([1] * 130, [0] * 130, 1025, 1, 64), ([100, 1, 0, 257, 64, 130], [100, 1, 9, 257, 0, 300], 640, 2, 128),
    ([3, 129, 128], [3, 129, 128], 1, 3, 64), ([5, 40], [70, 0], 0, 2, 128), ([300], [200], 300, 1, 64), ([2, 200, 1], [2, 200, 1], 4000, 1, 128)])
def test_shared_prefixes_round_ds_once(qlens, klens, P, H, d):
    """The default backward of these handles, against the bounds of a single rounding between P, dP and the products."""
    import paper_2608_01150_b200 as Z
    g = torch.Generator().manual_seed(46)
    nq, nk = sum(qlens), P + sum(klens)
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
    check_all(Run(h, {}, q, k, v, d ** -0.5, plain=True), prefix_problems(qlens, klens, P), {}, q, k, v, d_o, d ** -0.5, ds_roundings=1)


# ------------------------------------------------------------------------------------------------- no keys at all
@pytest.mark.parametrize("make,kind", [("shards", "plain"), ("shards", "mask"), ("shards", "all"), ("prefix", "plain"), ("prefix", "cap_mask")])
def test_queries_without_any_key_in_the_batch(make, kind):
    """K and V are empty tensors, whose address is NULL: rows get O = 0, LSE = -inf, dQ = 0."""
    import paper_2608_01150_b200 as Z
    d, H, rows = 64, 2, 150
    g = torch.Generator().manual_seed(47)
    q, d_o = rand(g, rows, H, d), rand(g, rows, H, d)
    none = torch.zeros(0, H, d, dtype=torch.bfloat16)
    if make == "shards":
        h = Z.build_tasks([0], [(0, 140, 0, 0, 0), (140, 10, 0, 0, 1)], rows, 0, H, d)
    else:
        h = Z.build_tasks_prefix([0, 140, 150], [0, 0, 0], 0, rows, 0, H, d)
    h.set_positions(None, [(5, 0, 0), (0, 0, 3)])
    s = {} if kind == "plain" else make_score(g, H, **KINDS[kind])
    run = Run(h, s, q, none, none, d ** -0.5, plain=kind == "plain")
    o, lse = run.forward()
    assert (o == 0).all() and torch.isneginf(lse).all()
    got = run.backward(d_o)
    assert (got["dq"] == 0).all() and got["dk"].numel() == 0
    if kind == "all":
        assert (got["dtable"] == 0).all()
