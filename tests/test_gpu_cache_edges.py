"""The paged cache on the GPU: orders of items, ragged tiles and magnitudes that the plain cases do not reach."""
import pytest
import torch

import cache_ref as R
import paper_2608_01150_b200 as Z
from cache_bounds import check8
from test_cache_state import near_pairs
from test_gpu_cache import BF16, E4M3, INT8, Setup, attend, check, i32, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 64, 1), (BF16, 128, 2), (INT8, 64, 5), (E4M3, 128, 3)])
def test_short_items_behind_items_that_are_cut(dtype, dim, group):
    """Long sequences, most of which lie in several CTAs, each in front of a dozen short ones: a join is followed at once by items that need none.
    Every run gives the same."""
    lens = sum(([700] + [1 + (7 * i + j) % 16 for j in range(12)] for i in range(20)), [])
    s = Setup(dtype, dim, 16, 4, lens)
    s.fill()
    qlens = [1] * len(lens)
    q = rand(s.g, len(lens), 4 * group, dim, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)
    for _ in range(20):
        again = attend(s, qlens, q)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,tokens", [(1, 17), (1, 131), (3, 43), (7, 20), (11, 13), (100, 1), (48, 5)])
def test_tiles_with_rows_that_do_not_exist(dtype, dim, group, tokens):
    """Warps that have rows of a tile and places without one, in one query tile and in two, in items that are cut and whole ones."""
    lens, qlens = [1500, tokens + 30, tokens], [tokens] * 3
    s = Setup(dtype, dim, 16, 2, lens)
    s.fill()
    q = rand(s.g, 3 * tokens + 2, 2 * group, dim, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)


@pytest.mark.parametrize("dtype,dim", [(INT8, 64), (E4M3, 128)])
@pytest.mark.parametrize("rows", [1, 12, 150])
@pytest.mark.parametrize("times", [2.0 ** 30, 2.0 ** 36])
def test_a_channel_of_large_queries_without_keys(dtype, dim, rows, times):
    """A channel whose queries are far above the others' and whose keys are 0: what is lost of the others is what the largest magnitude
    takes, not what the products would say."""
    n = 200 + rows
    s = Setup(dtype, dim, 16, 2, [n])
    k, v = rand(s.g, n, 2, dim), rand(s.g, n, 2, dim)
    k[:, :, 3] = 0.0
    q = rand(s.g, rows, 4, dim)
    q[:, :, 3] = times
    Z.cache_write(s.cache, s.batch([n]), k.cuda(), v.cuda())
    s.ref.write([0, n], [n], s.tables, k, v)
    o, lse = attend(s, [rows], q)
    check8(s, [rows], q, o, lse)


@pytest.mark.parametrize("dtype", [INT8, E4M3])
def test_weights_of_8_bit_values_keep_eleven_bits(dtype):
    """Single tokens over two keys each, whose values cancel: within what fp16 weights leave, an eighth of what bf16 ones would."""
    ref, tables, k, v, q = near_pairs(dtype)
    S = len(tables)
    s = Setup(dtype, 64, 8, 2, [2] * S)
    s.tables, s.ref = tables, ref
    Z.cache_write(s.cache, s.batch([2] * S), k.cuda(), v.cuda())
    o, lse = attend(s, [1] * S, q)
    check8(s, [1] * S, q, o, lse)
    # as chunks: twenty new tokens that all see their two keys and no more
    rows = q.repeat_interleave(20, 0)
    o, lse = attend(s, [20] * S, rows, [2] * S)
    check8(s, [20] * S, rows, o, lse, [2] * S)


@pytest.mark.parametrize("dtype,dim,group", [(INT8, 64, 1), (INT8, 128, 5), (E4M3, 64, 8), (E4M3, 128, 2)])
@pytest.mark.parametrize("prefix", [None, "some"])
def test_8_bit_caches_within_the_bounds_of_what_they_keep(dtype, dim, group, prefix):
    """Single tokens, chunks in one and in two tiles, cut items, against the bounds of exact codes and fp16 weights."""
    qlens = [1, 1, 3, 20, 150, 300, 1]
    lens = [40, 900, 60, 500, 150, 2000, 3000]
    s = Setup(dtype, dim, 32, 2, lens)
    s.fill()
    prefix = None if prefix is None else [0, 5, 60, 490, 2 ** 31 - 1, 7, 1]
    q = rand(s.g, sum(qlens), 2 * group, dim, times=1.5)
    for times in (1.0, 0.05):  # (small scores: what rounds the weights is most of the bound)
        x = (q.float() * times).to(BF16)
        o, lse = attend(s, qlens, x, prefix)
        check8(s, qlens, x, o, lse, prefix)


@pytest.mark.parametrize("dtype", [INT8, E4M3])
@pytest.mark.parametrize("rows", [1, 12, 60, 300])
def test_values_far_apart_within_the_bounds_of_what_they_keep(dtype, rows):
    """One token's values are 2^20 times the others' and looked at a little, one head's are 2^-60 times, one row of values is 0."""
    n, dim = 300, 64
    s = Setup(dtype, dim, 16, 2, [n])
    k, v = rand(s.g, n, 2, dim), rand(s.g, n, 2, dim)
    q = rand(s.g, rows, 4, dim).abs()
    k[17] = -2.0
    v[17] *= 2.0 ** 20
    v[:, 1] *= 2.0 ** -60
    v[40] = 0.0
    Z.cache_write(s.cache, s.batch([n]), k.cuda(), v.cuda())
    s.ref.write([0, n], [n], s.tables, k, v)
    o, lse = attend(s, [rows], q, [n])
    check8(s, [rows], q, o, lse, [n])


@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
def test_chunks_then_tokens_are_the_definitions_and_the_engines(dtype):
    """A prompt in chunks and then token by token, each step over what the steps before it wrote, against the definition; and the engine's masked
    attention of the whole sequence over what is read back, a rounding to bf16 away from it: 2^-8 of every key in a score
    (M = scale * sum |q||k| of its row, weights by a factor of e^(2 * 2^-8 M)) and of every value."""
    H, dim, total, prefix = 4, 64, 333, 50
    s = Setup(dtype, dim, 16, H, [total])
    q, k, v = (rand(s.g, total, H, dim) for _ in range(3))
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    h = Z.build_cached_attn(H, H, dim)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(qd), []
    at = 0
    for n in [50, 130, 64, 1, 3] + [1] * 85:
        b = s.batch([n], lens=[at + n], prefix=[prefix])
        Z.cache_write(s.cache, b, kd[at:at + n], vd[at:at + n])
        part = torch.empty(H, n, device="cuda")
        Z.cached_attn_fwd(h, s.cache, b, qd[at:at + n], dim ** -0.5, o[at:at + n], part, ws)
        lse.append(part)
        at += n
    assert at == total
    held = [torch.empty_like(kd) for _ in "kv"]
    Z.cache_read(s.cache, s.batch([0]), i32([0, total]), held[0], held[1])
    t = Z.build_tasks([0, total], [], total, total, H, dim)
    t.set_positions([prefix])
    o2, lse2 = torch.empty_like(qd), torch.empty(H, total, device="cuda")
    Z.scored_attn_fwd(t, Z.Score(masked=True), qd, held[0], held[1], dim ** -0.5, o2, lse2)
    torch.cuda.synchronize()
    s.ref.write([0, total], [total], s.tables, k, v)
    lse = torch.cat(lse, 1).cpu()
    if dtype is BF16:
        check(s, [total], q, o.cpu(), lse, [prefix])
    else:
        check8(s, [total], q, o.cpu(), lse, [prefix])
    O, L, bo, bl = R.attention(s.ref, [0, total], [total], s.tables, [prefix], q, dim ** -0.5)
    if dtype is not BF16:
        _, K, V = s.ref.held(0, [total], s.tables)
        seen = torch.arange(total)[None, :] < torch.arange(1, total + 1).clamp(min=prefix)[:, None]
        for j in range(H):
            x = (q[:, j].double() @ K[:, j].T * dim ** -0.5).masked_fill(~seen, -torch.inf)
            A = torch.softmax(x, 1) @ V[:, j].abs()
            off = 2.0 ** -8 * (q[:, j].double().abs() @ K[:, j].abs().T * dim ** -0.5 * seen).amax(1)
            bo[:, j] += torch.expm1(2 * off)[:, None] * (A + O[:, j].abs()) + 2.0 ** -8 * A
            bl[j] += off
    assert ((o2.cpu().double() - O).abs() <= bo).all() and ((lse2.cpu().double() - L).abs() <= bl).all()
    assert not (O.abs() <= bo).all(-1).any()  # (no row would pass as zeros)


@pytest.mark.parametrize("dtype,exponents", [(INT8, 9), (E4M3, 20)])
@pytest.mark.parametrize("times", [1.0, 2.0 ** -66, 2.0 ** 80, 2.0 ** -100])
def test_every_quotient_of_a_number_by_a_scale(dtype, exponents, times):
    """All mantissas of a row's largest number, and of the others with every exponent that can reach a code: codes and scales bit for bit
    (times: powers of two within and beyond what the fast quotient takes)."""
    m = 1 + torch.arange(128, dtype=torch.float64) / 128
    x = torch.cat([m * 2.0 ** -e for e in range(exponents)] + [torch.zeros(64)])
    rows = []
    for big in m:
        y = x[x <= big]
        y = torch.cat([y, y.new_zeros(-len(y) % 63)]).view(-1, 63)
        y[:, 1::2] *= -1
        rows.append(torch.cat([big.expand(len(y), 1), y], 1))
    rows = (torch.cat(rows) * times).to(BF16)[:, None]
    n = len(rows)
    s = Setup(dtype, 64, 16, 1, [n])
    Z.cache_write(s.cache, s.batch([n]), rows.cuda(), (-rows).cuda())
    code, scale = R.quantise(rows)(dtype)
    table = i32(s.tables[0]).long()
    for pool, got, sign in zip(s.pools, s.scales, (1.0, -1.0)):
        held = pool.view(torch.uint8)[table].view(dtype).float().reshape(-1, 64)[:n].cpu().double()
        assert torch.equal(held, sign * code[:, 0])
        assert torch.equal(got[table].reshape(-1)[:n].cpu(), scale[:, 0])
