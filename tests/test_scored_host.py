"""Scored attention and shared prefixes without a GPU: bucket maps, positions, refusals, the shared-prefix schedule, and
the 64-bit reference against differences and autograd."""
import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2608_01150_b200 as Z
import scored_ref as R
from paper_2608_01150_b200 import binding as B


# ---------------------------------------------------------------------------------------------- bucket maps
@pytest.mark.parametrize("n,dist,both", [(32, 128, True), (32, 128, False), (4, 2, True), (64, 600, True), (2, 5, False), (6, 17, True)])
def test_bucket_map(n, dist, both):
    got = Z.relative_position_buckets(n, dist, both)
    assert len(got) == 2 * dist + 1 and min(got) >= 0 and max(got) <= n - 1
    side = n // 2 if both else n
    exact = side // 2
    for d in range(-dist, dist + 1):
        a = abs(d) if both else max(0, -d)
        b = got[d + dist] - (side if both and d > 0 else 0)
        if a < exact:
            assert b == a
            continue
        # b is the largest step whose border e * (D / e)^((b - e) / (side - e)) is not beyond a: compared as fractions
        steps = side - exact
        border = lambda k: Fraction(dist, exact) ** k <= Fraction(a, exact) ** steps  # noqa: E731
        k = b - exact
        assert 0 <= k <= steps - 1 and border(k)
        assert k == steps - 1 or not border(k + 1)


def test_bucket_map_border_distances_are_not_rounded_down():
    got = Z.relative_position_buckets(32, 128, True)  # 8 exact, factor 16 over 8 steps: borders 8, 11.3, 16, 22.6, 32, 45.3, 64, 90.5
    of = lambda a: got[128 - a]  # noqa: E731
    assert [of(a) for a in (7, 8, 11, 12, 15, 16, 31, 32, 63, 64, 90, 91, 127, 128)] == [7, 8, 8, 9, 9, 10, 11, 12, 13, 14, 14, 15, 15, 15]


@pytest.mark.parametrize("n,dist,both", [(2, 128, True), (1, 128, False), (32, 8, True), (32, 0, True)])
def test_bucket_map_refusals(n, dist, both):
    with pytest.raises(Z.ZlError):
        Z.relative_position_buckets(n, dist, both)


# ---------------------------------------------------------------------------------------------- refusals
def _call(h, score, **kw):
    """Status of a scored forward with made-up pointers on a handle without a device."""
    d = B.ScoreDesc(score.get("cap", 0.0), score.get("slopes"), score.get("bias"), score.get("of"), score.get("n", 0),
                    score.get("dist", 0), score.get("masked", 0))
    return B.lib().zl_scored_attn_fwd(h.ptr, ctypes.byref(d), 16, 16, 16, ctypes.c_float(1.0), 16, 16, 16, 16, None)


no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: only on handles without a device")


@no_device
@pytest.mark.parametrize("score,status", [
    (dict(cap=-1.0), 1), (dict(cap=math.inf), 1), (dict(cap=1e-5), 1), (dict(cap=2e6), 1), (dict(cap=math.nan), 1), (dict(masked=2), 1),
    (dict(bias=16, of=16, n=0), 1), (dict(bias=16, n=4), 1), (dict(of=16), 1), (dict(n=4), 1),
    (dict(bias=16, of=16, n=65), 3), (dict(bias=16, of=16, n=4, dist=-1), 1), (dict(bias=16, of=16, n=4, dist=(1 << 24) + 1), 1),
    (dict(slopes=2), 1), (dict(masked=1), 1),                            # misaligned; mask without positions
    (dict(cap=30.0), 5), (dict(slopes=16), 5), (dict(bias=16, of=16, n=64, dist=128), 5), (dict(), 5),   # accepted: no device
])
def test_score_refusals(score, status):
    h = Z.build_tasks([0, 10, 30], [], 30, 30, 2, 64)
    assert _call(h, score) == status


@no_device
def test_positions_are_needed_and_checked():
    h = Z.build_tasks([0, 10], [(10, 5, 10, 7, 0), (10, 5, 17, 3, 0)], 20, 20, 1, 128)
    assert _call(h, dict(slopes=16)) == 1 and _call(h, dict(masked=1)) == 1      # shards without positions
    assert _call(h, dict(cap=5.0)) == 5
    for whole, shards in (([-1], [(0, 0, 0)] * 2), ([0], [(-1, 0, 0), (0, 0, 0)]), ([0], [(0, -1, 0), (0, 0, 0)]), ([0], [(0, 0, -1), (0, 0, 0)]),
                          ([0], [(2 ** 31 - 1, 0, 0), (0, 0, 0)]), ([0], [(0, 2 ** 31 - 516, 0), (0, 0, 0)]), ([0], None)):
        with pytest.raises(Z.ZlError):
            h.set_positions(whole, shards)
    for whole, shards in (([0, 0], [(0, 0, 0)] * 2), ([0], [(0, 0, 0)])):
        with pytest.raises(Z.ZlError):
            h.set_positions(whole, shards)
    assert _call(h, dict(masked=1)) == 1                                          # still none
    h.set_positions([3], [(2 ** 31 - 600, 2 ** 31 - 600, 0), (0, 7, 2 ** 31 - 1)])
    assert _call(h, dict(masked=1)) == 5 and _call(h, dict(slopes=16)) == 5


@no_device
def test_positions_of_a_fused_range_have_to_be_one_stretch():
    def build():
        return Z.build_tasks([0], [(0, 5, 0, 7, 0), (0, 5, 7, 3, 0)], 5, 10, 1, 128, flags=Z.BUILD_FUSE_LOCAL_CHUNKS)
    assert build().info.n_fused_ranges == 1
    build().set_positions(None, [(4, 20, 1), (4, 27, 1)])
    for bad in ([(4, 20, 1), (4, 28, 1)], [(4, 20, 1), (5, 27, 1)], [(4, 20, 1), (4, 27, 2)], [(4, 20, 1), (4, 3, 1)]):
        with pytest.raises(Z.ZlError):
            build().set_positions(None, bad)


def test_score_object_refusals():
    t = torch.zeros
    for kw in (dict(slopes=t(2, dtype=torch.float64)), dict(slopes=t(2, 2)), dict(bucket_bias=t(4, 2)), dict(bucket_of=t(5, dtype=torch.int32)),
               dict(bucket_bias=t(4, 2), bucket_of=t(5, dtype=torch.int64)), dict(bucket_bias=t(4, 2), bucket_of=t(4, dtype=torch.int32)),
               dict(bucket_bias=t(2, 4).t(), bucket_of=t(5, dtype=torch.int32))):
        with pytest.raises(Z.ZlError):
            Z.Score(**kw)
    h = Z.build_tasks([0, 10], [], 10, 10, 3, 64)
    with pytest.raises(Z.ZlError):                                                # heads of another handle
        Z.scored_attn_fwd(h, Z.Score(slopes=t(2)), 0, 0, 0, 1.0, 0, 0)
    bias = dict(bucket_bias=t(4, 3), bucket_of=t(5, dtype=torch.int32))
    with pytest.raises(Z.ZlError):
        Z.scored_attn_bwd(h, Z.Score(**bias), 0, 0, 0, 0, 0, 0, 1.0, 0, 0, 0, t(5, 3), t(1))


def test_workspace_counts_cap_and_buckets():
    h = Z.build_tasks([0, 10, 300], [], 300, 300, 3, 64)
    base = int(h.info.bwd_workspace_bytes)
    bias = dict(bucket_bias=torch.zeros(4, 3), bucket_of=torch.zeros(5, dtype=torch.int32))
    assert h.scored_workspace_bytes(Z.Score()) == base
    assert h.scored_workspace_bytes(Z.Score(slopes=torch.zeros(3))) == base
    q_pad, tiles = 128 + 384, 1 + 3
    assert h.scored_workspace_bytes(Z.Score(cap=3.0)) == base + q_pad * 3 * 4
    assert h.scored_workspace_bytes(Z.Score(**bias)) == base + tiles * 3 * Z.MAX_BUCKETS * 4
    assert h.scored_workspace_bytes(Z.Score(cap=3.0, **bias)) == base + q_pad * 3 * 4 + tiles * 3 * Z.MAX_BUCKETS * 4


# ---------------------------------------------------------------------------------------------- shared prefix
def _prefix_handle(qlens, klens, P, H=2, d=64, extra=0):
    cu = lambda x: [0] + list(np.cumsum(x))  # noqa: E731
    return Z.build_tasks_prefix(cu(qlens), cu(klens), P, sum(qlens) + extra, P + sum(klens) + extra, H, d)


@pytest.mark.parametrize("qlens,klens,P,H", [
    ([1] * 64, [17] * 64, 32760, 12), ([3, 0, 300, 1], [5, 9, 0, 700], 1000, 2), ([5], [0], 1, 1), ([1, 2], [3, 4], 0, 3), ([0, 4], [2, 0], 0, 2),
    ([700] * 3, [10] * 3, 513, 40), ([1], [1], 2 ** 20 + 1, 1)])
def test_prefix_schedule_covers_every_pair_once(qlens, klens, P, H):
    h = _prefix_handle(qlens, klens, P, H)
    cu_q, cu_kv = np.cumsum([0] + qlens), np.cumsum([0] + klens)
    n_own = sum(1 for q, k in zip(qlens, klens) if q > 0 and (k > 0 or P == 0))
    n_chunks = h.info.n_tasks - n_own
    assert (n_chunks == 0) == (P == 0) and n_chunks <= max(1, P // 512)
    assert h.info.n_merge_groups == sum(q > 0 for q in qlens)
    # forward: every (task, head, row) once
    rows = {}
    for task, head, r0, n in h.fwd_items():
        rows.setdefault((task, head), []).append((r0, n))
    total = sum(qlens)
    assert len(rows) == h.info.n_tasks * H
    own_q = [q for q, k in zip(qlens, klens) if q > 0 and (k > 0 or P == 0)]
    for (task, head), parts in rows.items():
        want = total if task < n_chunks else own_q[task - n_chunks]
        at = 0
        for r0, n in sorted(parts):
            assert r0 == at and 0 < n <= 256
            at += n
        assert at == want
    # backward: the key tiles of the prefix's chunks and of every own range, once per head
    keys = sum(n for g, head, r0, n in h.bwd_items() if head == 0)
    assert keys == P + sum(k for q, k in zip(qlens, klens) if q > 0)
    # slots: chunks first, one row per query of the batch, then the own parts
    pad = lambda n: -(-n // 128) * 128  # noqa: E731
    at = n_chunks * pad(total)
    for i, (q, k) in enumerate(zip(qlens, klens)):
        off, n = h.partial_slot(i)
        if q > 0 and (k > 0 or P == 0):
            assert (off, n) == (at, pad(q))
            at += pad(q)
        else:
            assert n == 0
    assert h.info.partial_rows == at


def test_prefix_chunks_fill_the_gpu_for_few_rows():
    h = _prefix_handle([1] * 64, [1] * 64, 32760, 12)
    n_prefix = sum(1 for t, _, _, _ in h.fwd_items()) - 64 * 12
    assert 0.9 * 148 <= n_prefix <= 2 * 148   # one or two rounds of the 148 SMs, or nearly


@pytest.mark.parametrize("cu_q,cu_kv,P,tq,tk,H,d", [
    ([0, 5], [0, 5], -1, 5, 5, 1, 64), ([1, 5], [0, 5], 0, 5, 5, 1, 64), ([0, 5], [1, 5], 0, 5, 9, 1, 64), ([0, 5, 4], [0, 1, 2], 0, 5, 9, 1, 64),
    ([0, 5], [0, 5], 0, 4, 5, 1, 64), ([0, 5], [0, 5], 1, 5, 5, 1, 64), ([0, 5], [0, 5], 0, 5, 5, 0, 64), ([0, 5], [0, 5], 0, 5, 5, 1, 96),
    ([0, 5], [0, 2, 5], 0, 5, 5, 1, 64)])
def test_prefix_refusals(cu_q, cu_kv, P, tq, tk, H, d):
    with pytest.raises(Z.ZlError):
        Z.build_tasks_prefix(cu_q, cu_kv, P, tq, tk, H, d)


def test_prefix_of_nothing():
    h = Z.build_tasks_prefix([0], [0], 7, 0, 7, 1, 64)
    assert h.info.n_tasks == 0 and h.info.partial_rows == 0
    h = Z.build_tasks_prefix([0, 0], [0, 3], 7, 0, 10, 1, 64)
    assert h.info.n_tasks == 0


@no_device
def test_prefix_refuses_scores_by_distance():
    h = _prefix_handle([2, 3], [4, 5], 100)
    assert _call(h, dict(slopes=16)) == 3 and _call(h, dict(bias=16, of=16, n=4, dist=2)) == 3
    assert _call(h, dict(cap=4.0)) == 5 and _call(h, dict(masked=1)) == 1
    h.set_positions(shard_pos=[(2, 0, 0), (2, 0, 1)])
    assert _call(h, dict(masked=1)) == 5 and _call(h, dict(slopes=16)) == 3


# ---------------------------------------------------------------------------------------------- the reference itself
@pytest.mark.parametrize("cap,slopes,buckets,masked", [(0, 0, 0, 0), (3.0, 0, 0, 1), (0, 1, 0, 0), (0, 0, 1, 1), (2.0, 1, 1, 1)])
def test_reference_gradients_against_autograd_and_differences(cap, slopes, buckets, masked):
    g = torch.Generator().manual_seed(3)
    H, d, L = 2, 4, 7
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, d_o = rnd(L, H, d), rnd(L, H, d), rnd(L, H, d), rnd(L, H, d)
    score = dict(cap=float(cap), masked=bool(masked))
    if slopes:
        score["slopes"] = rnd(H).abs()
    if buckets:
        score["table"], score["bucket_of"] = rnd(4, H), torch.tensor([0, 1, 2, 3, 1], dtype=torch.int32)
    pos = torch.arange(L)
    problems = [(pos, pos, pos, pos, 2)]

    def loss(q, k, v, table):
        total = 0
        for h in range(H):
            a = R._args(dict(score, **({"table": table} if buckets else {})), h)
            s, _, _, _ = R.scores(q[:, h], k[:, h], pos, pos, 2, 0.7, **a)
            total = total + (torch.softmax(s, 1) @ v[:, h] * d_o[:, h]).sum()
        return total

    f = R.forward(problems, q, k, v, 0.7, score)
    got = R.backward(problems, q, k, v, f["o"], f["lse"], d_o, 0.7, score)
    leaves = [x.clone().requires_grad_() for x in (q, k, v) + ((score["table"],) if buckets else ())]
    loss(*leaves, *([None] if not buckets else [])).backward()
    names = ["dq", "dk", "dv"] + (["dtable"] if buckets else [])
    for name, leaf in zip(names, leaves):
        assert torch.allclose(got[name], leaf.grad, atol=1e-12), name
        at = torch.nonzero(torch.ones_like(leaf))[:: max(1, leaf.numel() // 9)]
        for i in at:                                                              # central differences
            e = torch.zeros_like(leaf)
            e[tuple(i)] = 1e-5
            up = [x.detach() + (e if x is leaf else 0) for x in leaves] + ([] if buckets else [None])
            dn = [x.detach() - (e if x is leaf else 0) for x in leaves] + ([] if buckets else [None])
            assert abs(float((loss(*up) - loss(*dn)) / 2e-5 - got[name][tuple(i)])) < 1e-7
