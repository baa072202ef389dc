"""Rows that no task owns: finite values of any magnitude there reach no result, with every backward kernel."""
import pytest
import torch

from test_gpu_scored import Run, check_all, cu, prefix_problems, rand, whole_problems

pytestmark = pytest.mark.gpu


def poison(x, rows, every):
    """3e38 with every `every`-th sign turned: products overflow to either infinity."""
    big = torch.full(x.shape[1:], 3e38)
    big.view(-1)[::every] *= -1
    x[rows] = big.to(x.dtype)


KERNELS = [(64, 0), (64, 1), (128, 0), (128, 1), (128, 2)]


@pytest.mark.parametrize("every", [2, 3, 10 ** 9])
@pytest.mark.parametrize("d,kernel", KERNELS)
def test_whole_sequences_and_chunks(d, kernel, every):
    """Ragged whole sequences of one and several tiles, and query chunks of unequal lengths that share their key chunks (a key
    tile's CTA walks several query ranges), with gaps behind each."""
    import paper_2608_01150_b200 as Z
    H, T = 2, 1400
    g = torch.Generator().manual_seed(51)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    whole = [(0, 100), (120, 130), (260, 257), (530, 64)]
    chunks_q, chunks_k = [(600, 130), (740, 7), (760, 300)], [(600, 150), (770, 300), (1090, 33)]
    shards = [(qo, ql, ko, kl, 0) for qo, ql in chunks_q for ko, kl in chunks_k]
    own_q, own_k = torch.zeros(T, dtype=torch.bool), torch.zeros(T, dtype=torch.bool)
    for off, n in whole + chunks_q:
        own_q[off:off + n] = True
    for off, n in whole + chunks_k:
        own_k[off:off + n] = True
    for x, own, e in ((q, own_q, every), (d_o, own_q, every), (k, own_k, 2), (v, own_k, 3)):
        poison(x, ~own, e)
    h = Z.build_tasks_heads([(off, n, 0, H) for off, n in whole], shards, None, T, T, H, d)
    h.set_bwd_kernel(kernel)
    problems = [(torch.arange(o, o + n), torch.arange(o, o + n), torch.arange(n), torch.arange(n), 0) for o, n in whole]
    keys = torch.cat([torch.arange(o, o + n) for o, n in chunks_k])
    problems += [(torch.arange(o, o + n), keys, torch.arange(n), torch.arange(len(keys)), 0) for o, n in chunks_q]
    check_all(Run(h, {}, q, k, v, d ** -0.5, plain=True), problems, {}, q, k, v, d_o, d ** -0.5, ds_roundings=3)


@pytest.mark.parametrize("d,kernel", KERNELS)
def test_shared_prefix(d, kernel):
    """Keys of a sequence without queries behind a ragged key tile, rows behind the batch."""
    import paper_2608_01150_b200 as Z
    H, P, qlens, klens = 2, 520, [30, 0, 140, 1], [50, 40, 140, 3]
    g = torch.Generator().manual_seed(52)
    nq, nk = sum(qlens) + 20, P + sum(klens) + 20
    q, d_o, k, v = rand(g, nq, H, d), rand(g, nq, H, d), rand(g, nk, H, d), rand(g, nk, H, d)
    for x in (k, v):
        poison(x, slice(P + 50, P + 90), 2)
        poison(x, slice(P + sum(klens), nk), 2)
    for x in (q, d_o):
        poison(x, slice(sum(qlens), nq), 3)
    h = Z.build_tasks_prefix(cu(qlens), cu(klens), P, nq, nk, H, d)
    h.set_bwd_kernel(kernel)
    problems = [p for p in prefix_problems(qlens, klens, P) if len(p[0])]
    check_all(Run(h, {}, q, k, v, d ** -0.5, plain=True), problems, {}, q, k, v, d_o, d ** -0.5, ds_roundings=3)


@pytest.mark.parametrize("d,kernel", KERNELS)
def test_a_neighbouring_sequence_of_huge_values(d, kernel):
    """The second sequence's own results are what its values make of them; the first one's are untouched."""
    import paper_2608_01150_b200 as Z
    H, lens = 2, [140, 90]
    T = sum(lens)
    g = torch.Generator().manual_seed(53)
    q, k, v, d_o = (rand(g, T, H, d) for _ in range(4))
    for x, e in ((q, 3), (k, 2), (v, 2), (d_o, 3)):
        poison(x, slice(140, T), e)
    h = Z.build_tasks(cu(lens), [], T, T, H, d)
    h.set_bwd_kernel(kernel)
    check_all(Run(h, {}, q, k, v, d ** -0.5, plain=True), whole_problems(lens, [0, 0])[:1], {}, q, k, v, d_o, d ** -0.5, ds_roundings=3)
