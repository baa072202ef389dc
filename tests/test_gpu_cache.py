"""The paged cache on the GPU: written, read back and attended to, against the definition in 64 bits (cache_ref)."""
import math

import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

BF16, INT8, E4M3 = torch.bfloat16, torch.int8, torch.float8_e4m3fn
NAN_CODE = {INT8: -128, E4M3: 0x7f}


def cu(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rand(g, *shape, times=1.0):
    return (torch.randn(*shape, generator=g) * times).to(BF16)


class Setup:
    """A cache on the GPU whose unwritten places hold what must not matter, with its reference and the tables of a batch.

    tokens: kv_len of every sequence; its pages are scattered over the cache."""

    def __init__(self, dtype, dim, page, heads, lens, layout="tokens", seed=1, spare=3, max_pages=None):
        g = self.g = torch.Generator().manual_seed(seed)
        need = [max(0, (n + page - 1) // page) for n in lens]
        n_pages = sum(need) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        width = max(need + [1]) if max_pages is None else max_pages
        self.tables, at = [], 0
        for n in need:
            self.tables.append((order[at:at + n] + [-1] * width)[:width])
            at += n
        self.dtype, self.dim, self.page, self.heads, self.lens = dtype, dim, page, heads, list(lens)
        self.ref = R.Ref(n_pages, page, heads, dim, dtype)
        shape = (n_pages, page, heads, dim)
        if layout == "heads":
            pools = [torch.empty(n_pages, heads, page, dim, dtype=dtype, device="cuda").transpose(1, 2) for _ in "kv"]
        elif layout == "together":
            both = torch.empty(n_pages, 2, page, heads, dim, dtype=dtype, device="cuda")
            pools = [both[:, 0], both[:, 1]]
        else:
            pools = [torch.empty(shape, dtype=dtype, device="cuda") for _ in "kv"]
        self.scales = [None, None]
        for p in pools:
            if dtype is BF16:
                p.fill_(math.nan)
            else:
                p.view(torch.int8).fill_(NAN_CODE[dtype])
        if dtype is not BF16:
            self.scales = [torch.full(shape[:3], math.nan, device="cuda") for _ in "kv"]
            if layout == "heads":  # and the scales by heads too
                self.scales = [torch.full((n_pages, heads, page), math.nan, device="cuda").transpose(1, 2) for _ in "kv"]
        self.pools = pools
        import paper_2608_01150_b200 as Z
        self.cache = Z.KvCache(pools[0], pools[1], *self.scales)

    def batch(self, qlens, lens=None, prefix=None, max_q=None):
        import paper_2608_01150_b200 as Z
        return Z.CacheBatch(i32(cu(qlens)), i32(self.lens if lens is None else lens), i32(self.tables), prefix=None if prefix is None else i32(prefix),
                            max_q=max(qlens + [0]) if max_q is None else max_q)

    def fill(self):
        """Every sequence's keys and values, written by one call."""
        import paper_2608_01150_b200 as Z
        n = [max(0, x) for x in self.lens]
        k, v = rand(self.g, sum(n), self.heads, self.dim, times=1.5), rand(self.g, sum(n), self.heads, self.dim)
        Z.cache_write(self.cache, self.batch(n), k.cuda(), v.cuda())
        self.ref.write(cu(n), n, self.tables, k, v)
        return k, v


def attend(setup, qlens, q, prefix=None, handle=None, ws=None, max_q=None, lens=None, stream=None):
    import paper_2608_01150_b200 as Z
    h = handle or Z.build_cached_attn(q.shape[1], setup.heads, setup.dim)
    ws = torch.full((h.workspace_bytes,), 0xff, dtype=torch.uint8, device="cuda") if ws is None else ws
    o = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    Z.cached_attn_fwd(h, setup.cache, setup.batch(qlens, lens, prefix, max_q), q.cuda(), setup.dim ** -0.5, o, lse, ws)
    torch.cuda.synchronize()
    assert h.last_device_status() == (0, 0)
    return o.cpu(), lse.cpu()


def check(setup, qlens, q, o, lse, prefix=None, lens=None):
    O, L, bo, bl = R.attention(setup.ref, cu(qlens), setup.lens if lens is None else lens, setup.tables, prefix, q, setup.dim ** -0.5)
    n = sum(qlens)
    assert not torch.isnan(O[:n]).any() and not torch.isnan(o[:n].float()).any() and not torch.isnan(lse[:, :n]).any()
    off = ((o[:n].double() - O[:n]).abs() / bo[:n])
    assert off.max() <= 1, f"O off by {off.max():.3g} of its bound"
    dead = torch.isinf(L[:, :n])
    assert torch.equal(torch.isinf(lse[:, :n]) & (lse[:, :n] < 0), dead)
    off = ((lse[:, :n].double() - L[:, :n]).abs() / bl[:, :n])[~dead]
    assert off.numel() == 0 or off.max() <= 1, f"LSE off by {off.max():.3g} of its bound"
    assert (o[n:] == 7.0).all() and (lse[:, n:] == 7.0).all()  # rows behind the last sequence


# ------------------------------------------------------------------------------------------------- write and read
@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
@pytest.mark.parametrize("dim,page,heads,layout", [(64, 8, 1, "tokens"), (64, 64, 3, "heads"), (128, 16, 2, "together"), (128, 256, 5, "tokens")])
def test_written_values_are_the_definitions(dtype, dim, page, heads, layout):
    """Codes and scales bit for bit; every other place as it was; read back in whole and in part."""
    import paper_2608_01150_b200 as Z
    lens, qlens = [37, 5, 1, 300, 0, 12], [9, 5, 1, 300, 0, 0]
    s = Setup(dtype, dim, page, heads, lens, layout)
    before = [p.clone() for p in s.pools], [None if x is None else x.clone() for x in s.scales]
    T = sum(qlens) + 4
    qkv = rand(s.g, T, 3, heads, dim)
    qkv[0, 1:] = 0.0                       # a row of zeros
    qkv[1, 1:] = 1e-38                     # subnormal scales
    qkv[2, 1:, :, ::2] = 3e38
    qkv[3, 1:, :, 1:] *= 1e-3              # one element far above the others
    k, v = qkv[:, 1], qkv[:, 2]            # strided rows
    dev = qkv.cuda()
    Z.cache_write(s.cache, s.batch(qlens), dev[:, 1], dev[:, 2])
    done = s.ref.write(cu(qlens), lens, s.tables, k, v)
    assert len(done) == len(set(done)) == sum(qlens)
    pg, at = (torch.tensor([d[i] for d in done]) for i in range(2))
    for c in range(2):
        got = s.pools[c].cpu()
        assert torch.equal(got[pg, at].double() if dtype is not E4M3 else got.float()[pg, at].double(), s.ref.code[c][pg, at])
        keep = torch.ones(got.shape[:2], dtype=torch.bool)
        keep[pg, at] = False
        assert torch.equal(got.view(torch.uint8)[keep], before[0][c].cpu().view(torch.uint8)[keep])
        if dtype is not BF16:
            sc = s.scales[c].cpu()
            assert torch.equal(sc[pg, at], s.ref.scale[c][pg, at]) and torch.isnan(sc[keep]).all()
    # the new rows, one behind the other, then from other positions on, past the ends
    for first, n in ((None, None), ([28, -3, 0, 250, 0, 13], [9, 6, 2, 60, 3, 0])):
        if n is None:
            first, n = [a - b for a, b in zip(lens, qlens)], qlens
        out = [torch.full((sum(n) + 2, heads, dim), 7.0, dtype=BF16, device="cuda") for _ in "kv"]
        Z.cache_read(s.cache, s.batch(qlens), i32([x + 1 for x in cu(n)]), out[0], out[1], first=i32(first))
        for c in range(2):
            want = torch.zeros(sum(n), heads, dim, dtype=torch.float64)
            for i in range(len(n)):
                for j in range(n[i]):
                    p = first[i] + j
                    place = s.ref.place(s.tables[i], p)
                    if 0 <= p < lens[i] and place in done:
                        want[cu(n)[i] + j] = s.ref.code[c][place] * (1.0 if dtype is BF16 else s.ref.scale[c][place].double()[:, None])
                    elif 0 <= p < lens[i]:
                        want[cu(n)[i] + j] = math.nan  # never written: whatever is there
            got = out[c].cpu()
            assert (got[0] == 7.0).all() and (got[-1] == 7.0).all()
            known = ~torch.isnan(want)
            # the product in 32 bits, then bf16: one rounding of each
            off = (got[1:-1].double() - want).abs()[known]
            assert (off <= (2.0 ** -8 + 2.0 ** -23) * want[known].abs() + 1e-40).all()
            if dtype is BF16:
                assert (off == 0).all()


@pytest.mark.parametrize("dtype", [INT8, E4M3])
def test_values_between_two_codes_go_to_the_even_one(dtype):
    """Rows whose largest magnitude is T: the scale is 1 and halves are ties."""
    import paper_2608_01150_b200 as Z
    s = Setup(dtype, 64, 16, 1, [4])
    k = torch.zeros(4, 1, 64)
    k[:, 0, 0] = R.TOP[dtype]
    k[0, 0, 1:33] = torch.arange(-16, 16) + 0.5
    k[1, 0, 1:17] = (torch.arange(16) + 0.5) * 2.0 ** -9       # subnormal steps of e4m3
    k[2, 0, 1:9] = 16 + torch.arange(8) + 0.5
    k = k.to(BF16)
    Z.cache_write(s.cache, s.batch([4]), k.cuda(), k.cuda())
    s.ref.write([0, 4], [4], s.tables, k, k)
    pg = s.tables[0][0]
    assert torch.equal(s.pools[0].cpu().float()[pg, :4].double(), s.ref.code[0][pg, :4])
    assert (s.scales[0][pg, :4] == 1.0).all()


@pytest.mark.parametrize("dtype", [BF16, INT8])
def test_pages_that_do_not_exist_are_left_out(dtype):
    """Dropped pages and numbers outside the cache: not written, read as zeros, seen by nobody; so are positions beyond
    the table and new tokens before position 0."""
    import paper_2608_01150_b200 as Z
    lens, page = [200, 90, 3, 700], 16
    s = Setup(dtype, 64, page, 2, lens, spare=4)
    s.tables[0][2] = -1
    s.tables[0][5] = s.ref.n_pages
    s.tables[1] = [-7] * len(s.tables[1])
    s.tables[3][0] = 2 ** 31 - 1
    s.tables[3][30] = -2 ** 31
    s.tables = [t[:40] for t in s.tables]      # 640 positions
    s.fill()
    qlens = [170, 2, 6, 33]                    # the third sequence has three tokens, its first three rows are before it
    q = rand(s.g, sum(qlens), 4, 64, times=1.5)
    for prefix in (None, [0, 5, 0, 650]):
        o, lse = attend(s, qlens, q, prefix)
        check(s, qlens, q, o, lse, prefix)
        assert (o[172:175] == 0).all() and torch.isinf(lse[:, 170:175]).all()
    out = [torch.full((200, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in "kv"]
    Z.cache_read(s.cache, s.batch(qlens), i32([0, 200, 200, 200, 200]), out[0], out[1])
    assert (out[0][32:48] == 0).all() and (out[1][80:96] == 0).all() and (out[0][48:80] != 0).any()


# ------------------------------------------------------------------------------------------------- attention
GRID = [(BF16, 64, 16, 2, 1), (BF16, 128, 8, 1, 5), (INT8, 64, 64, 3, 2), (INT8, 128, 16, 2, 8), (E4M3, 64, 8, 1, 3), (E4M3, 128, 256, 2, 4)]


@pytest.mark.parametrize("dtype,dim,page,heads,group", GRID)
@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_single_tokens(dtype, dim, page, heads, group, layout):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 0, 500, 1000, 31]
    s = Setup(dtype, dim, page, heads, lens, layout)
    s.fill()
    q = rand(s.g, len(lens) + 2, heads * group, dim, times=1.5)
    o, lse = attend(s, [1] * len(lens), q)
    check(s, [1] * len(lens), q, o, lse)


@pytest.mark.parametrize("dtype,dim,page,heads,group", GRID)
@pytest.mark.parametrize("prefix", [None, "some"])
def test_chunks_beside_single_tokens(dtype, dim, page, heads, group, prefix):
    """New tokens of every number, a sequence without any, one longer than the sequence, rows behind the last."""
    qlens = [130, 1, 0, 3, 16, 17, 257, 2, 64, 40]
    lens = [130, 900, 50, 3, 300, 17, 600, 1, 200, 25]
    s = Setup(dtype, dim, page, heads, lens)
    s.fill()
    prefix = None if prefix is None else [0, 5, 3, 2 ** 31 - 1, 295, -4, 450, 1, 2 ** 31 - 1, 7]
    q = rand(s.g, sum(qlens) + 3, heads * group, dim, times=1.5)
    o, lse = attend(s, qlens, q, prefix)
    check(s, qlens, q, o, lse, prefix)
    assert prefix is not None or (o[490:505] == 0).all()  # the last sequence's tokens before its position 0


@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (INT8, 64), (E4M3, 128)])
@pytest.mark.parametrize("rows", [1, 2, 20, 140])
def test_long_sequences_are_joined_from_many_parts(dtype, dim, rows):
    """A few heads over long keys: every SM has a part.  The same from run to run."""
    lens = [9000, 70]
    s = Setup(dtype, dim, 32, 2, lens)
    s.fill()
    qlens = [rows, 1]
    q = rand(s.g, rows + 1, 4, dim, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)
    again = attend(s, qlens, q)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
def test_growing_scores_move_the_reference(dtype):
    """Keys that grow along the sequence, so that every tile has a new maximum; and rows that are nearly one-hot."""
    dim, n = 128, 700
    s = Setup(dtype, dim, 16, 1, [n, n])
    k, v = rand(s.g, 2 * n, 1, dim), rand(s.g, 2 * n, 1, dim)
    k[:n] = (k[:n].float() * 0.1 + torch.linspace(0, 3, n)[:, None, None]).to(BF16)
    import paper_2608_01150_b200 as Z
    Z.cache_write(s.cache, s.batch([n, n]), k.cuda(), v.cuda())
    s.ref.write([0, n, 2 * n], [n, n], s.tables, k, v)
    qlens = [150, 2]
    q = rand(s.g, 152, 2, dim, times=1.0)
    q[:, 0] = q[:, 0].abs()
    q[150:] *= 8
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)


@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
def test_rows_of_no_sequence_and_of_others_do_not_matter(dtype):
    """Queries behind the last sequence hold NaN and infinities, those of another sequence 2^60 times the rest; tiles read both."""
    lens, qlens = [200, 30, 150], [40, 3, 21]
    s = Setup(dtype, 64, 16, 2, lens)
    s.fill()
    q = rand(s.g, 70, 4, 64, times=1.5)
    q[64:67], q[67:] = math.nan, math.inf
    small = q[:64].clone()
    small[40:43] *= 2.0 ** -60
    q[40:43] *= 2.0 ** 60
    o, lse = attend(s, qlens, q)
    check(s, [40], q[:40], o[:40], lse[:, :40], lens=lens[:1])
    s.tables, tables = s.tables[2:], s.tables
    check(s, [21], q[43:64], o[43:64], lse[:, 43:64], lens=lens[2:])
    s.tables = tables
    o, lse = attend(s, qlens, small)
    check(s, qlens, small, o, lse)


@pytest.mark.parametrize("dtype", [INT8, E4M3])
@pytest.mark.parametrize("rows", [1, 12, 60])
def test_values_of_very_different_scales(dtype, rows):
    """One token's values are 2^20 times the others', and next to nobody looks at it; one head's are 2^-60 times."""
    import paper_2608_01150_b200 as Z
    n, dim = 300, 64
    s = Setup(dtype, dim, 16, 2, [n])
    k, v = rand(s.g, n, 2, dim), rand(s.g, n, 2, dim)
    q = rand(s.g, rows, 4, dim).abs()
    k[17] = -2.0                     # scores some 2^5 below the rest
    v[17] *= 2.0 ** 20
    v[:, 1] *= 2.0 ** -60
    Z.cache_write(s.cache, s.batch([n]), k.cuda(), v.cuda())
    s.ref.write([0, n], [n], s.tables, k, v)
    o, lse = attend(s, [rows], q)
    check(s, [rows], q, o, lse)


@pytest.mark.parametrize("n_seqs", [255, 257, 700])
def test_many_sequences(n_seqs):
    """More sequences than a CTA has threads."""
    lens = [(i * 37) % 90 for i in range(n_seqs)]
    s = Setup(BF16, 64, 16, 1, lens)
    s.fill()
    qlens = [1 if i % 5 else 2 for i in range(n_seqs)]
    q = rand(s.g, sum(qlens), 2, 64, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)


@pytest.mark.parametrize("max_q", [0, 1, 10 ** 6])
def test_max_q_only_chooses_kernels(max_q):
    qlens, lens = [1, 300, 5], [400, 350, 5]
    s = Setup(INT8, 64, 16, 2, lens)
    s.fill()
    q = rand(s.g, sum(qlens), 6, 64, times=1.5)
    o, lse = attend(s, qlens, q, max_q=max_q)
    check(s, qlens, q, o, lse)


@pytest.mark.parametrize("dtype,group,dim", [(BF16, 100, 64), (INT8, 128, 64), (BF16, 40, 128), (E4M3, 9, 128), (INT8, 33, 64)])
def test_many_query_heads_to_a_key_head(dtype, group, dim):
    """Tiles of one, three, fourteen tokens; single tokens that fill a tile, or two columns of eight rows."""
    lens, qlens = [40, 300, 150], [1, 5, 1]
    s = Setup(dtype, dim, 16, 2, lens)
    s.fill()
    q = rand(s.g, 8, 2 * group, dim, times=1.5)
    for max_q in (0, 5):
        o, lse = attend(s, qlens, q, max_q=max_q)
        check(s, qlens, q, o, lse)
    o, lse = attend(s, [1, 1, 1], q)
    check(s, [1, 1, 1], q, o, lse)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_tokens_outermost(dtype):
    """A cache whose pages are strided: token 0 of every page, then token 1, ..."""
    import paper_2608_01150_b200 as Z
    lens, qlens = [40, 200], [1, 150]
    s = Setup(dtype, 64, 8, 2, lens)
    n = s.ref.n_pages
    s.pools = [torch.zeros(8, n, 2, 64, device="cuda").to(dtype).transpose(0, 1) for _ in "kv"]
    if dtype is not BF16:
        s.scales = [torch.zeros(8, 2, n, device="cuda").permute(2, 0, 1) for _ in "kv"]
    s.cache = Z.KvCache(s.pools[0], s.pools[1], *s.scales)
    s.fill()
    q = rand(s.g, 151, 6, 64, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)
    o, lse = attend(s, [1, 1], q[:2])
    check(s, [1, 1], q[:2], o, lse)


def test_caches_without_a_page():
    """No page, or tables without an entry: nobody sees anything, nothing is written, zeros are read."""
    import paper_2608_01150_b200 as Z
    none = torch.zeros(0, 16, 2, 64, dtype=BF16, device="cuda")
    one = torch.zeros(1, 16, 2, 64, dtype=BF16, device="cuda")
    h = Z.build_cached_attn(4, 2, 64)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    k = torch.ones(40, 2, 64, dtype=BF16, device="cuda")
    q = torch.ones(40, 4, 64, dtype=BF16, device="cuda")
    for pool, width in ((none, 3), (one, 0)):
        c = Z.KvCache(pool, pool.clone())
        b = Z.CacheBatch(i32([0, 1, 40]), i32([10, 39]), torch.zeros(2, width, dtype=torch.int32, device="cuda"))
        Z.cache_write(c, b, k, k)
        rows = [torch.full((3, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in "kv"]
        Z.cache_read(c, b, i32([0, 2, 3]), rows[0], rows[1])
        o, lse = torch.full_like(q, 7.0), torch.zeros(4, 40, device="cuda")
        Z.cached_attn_fwd(h, c, b, q, 0.125, o, lse, ws)
        torch.cuda.synchronize()
        assert (o == 0).all() and torch.isinf(lse).all() and (lse < 0).all() and (rows[0] == 0).all() and (rows[1] == 0).all() and (pool == 0).all()
    assert h.last_device_status() == (0, 0)


def test_outputs_over_the_queries_are_refused():
    import paper_2608_01150_b200 as Z
    s = Setup(BF16, 64, 16, 2, [20, 20])
    h = Z.build_cached_attn(4, 2, 64)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    both = torch.zeros(4, 4, 64, dtype=BF16, device="cuda")
    for o in (both[:2], both[1:3]):
        with pytest.raises(Z.ZlError) as e:
            Z.cached_attn_fwd(h, s.cache, s.batch([1, 1]), both[:2], 0.125, o, None, ws)
        assert e.value.status == 1
    Z.cached_attn_fwd(h, s.cache, s.batch([1, 1]), both[:2], 0.125, both[2:], None, ws)


@pytest.mark.parametrize("dtype", [BF16, INT8])
def test_calls_one_behind_the_other(dtype):
    """Writes and attention of chunks beside single tokens, each call needing the one before it and writing over what that has read:
    the same without a pause as with one behind every call."""
    import paper_2608_01150_b200 as Z
    qlens = [300, 1, 1, 40, 1, 1, 1, 1]
    s = Setup(dtype, 128, 16, 4, [1200, 3000, 40, 900, 2000, 17, 2500, 600])
    s.fill()
    n, heads, steps = sum(qlens), 8, 12
    k, v, q = (rand(s.g, steps, n, h, 128, times=1.5).cuda() for h in (4, 4, heads))
    h = Z.build_cached_attn(heads, 4, 128)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    b = s.batch(qlens)
    outs = []
    for pause in (True, False):
        o = torch.zeros(steps, n, heads, 128, dtype=BF16, device="cuda")
        torch.cuda.synchronize()
        for i in range(steps):
            Z.cache_write(s.cache, b, k[i], v[i])
            if pause:
                torch.cuda.synchronize()
            Z.cached_attn_fwd(h, s.cache, b, q[0] if i == 0 else o[i - 1], 128 ** -0.5, o[i], None, ws)  # (reads what the last call wrote)
            if pause:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        outs.append(o)
    assert h.last_device_status() == (0, 0) and torch.equal(outs[0], outs[1])


def test_a_shared_beginning():
    """Two sequences with the same first pages, one of them continued in its own."""
    s = Setup(BF16, 64, 16, 2, [40, 64])
    s.fill()
    s.tables[0][:2] = s.tables[1][:2]
    qlens = [3, 1]
    q = rand(s.g, 4, 2, 64, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)


def test_strided_queries_and_no_lse():
    import paper_2608_01150_b200 as Z
    s = Setup(BF16, 128, 16, 2, [200, 20])
    s.fill()
    qlens = [3, 1]
    qkv = rand(s.g, 4, 8 + 2 + 2, 128, times=1.5)
    dev = qkv.cuda()
    h = Z.build_cached_attn(8, 2, 128)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    o = torch.empty(4, 8, 128, dtype=BF16, device="cuda")
    Z.cached_attn_fwd(h, s.cache, s.batch(qlens), dev[:, :8], 128 ** -0.5, o, None, ws)
    q = qkv[:, :8].contiguous()
    same, lse = attend(s, qlens, q)
    assert torch.equal(o.cpu(), same)
    check(s, qlens, q, same, lse)


def test_places_beyond_32_bits():
    """The last pages of a cache of more than 2^31 elements and 2^32 bytes."""
    import paper_2608_01150_b200 as Z
    dim, page, heads = 128, 16, 2
    n_pages = (2 ** 31 + 2 ** 28) // (page * heads * dim)
    for dtype in (BF16, INT8):
        pools = [torch.empty(n_pages, page, heads, dim, dtype=dtype, device="cuda") for _ in "kv"]
        scales = [None, None] if dtype is BF16 else [torch.empty(n_pages, page, heads, device="cuda") for _ in "kv"]
        s = Setup(dtype, dim, page, heads, [50, 170])
        s.tables = [[n_pages - 1 - p if p >= 0 else p for p in t] for t in s.tables]
        s.cache, s.pools, s.scales = Z.KvCache(pools[0], pools[1], *scales), pools, scales
        kept = s.ref
        mirrored = R.Ref(kept.n_pages, page, heads, dim, dtype)
        k, v = rand(s.g, 220, heads, dim, times=1.5), rand(s.g, 220, heads, dim)
        Z.cache_write(s.cache, s.batch([50, 170]), k.cuda(), v.cuda())
        tables, s.tables = s.tables, [[n_pages - 1 - p if p >= 0 else p for p in t] for t in s.tables]
        mirrored.write([0, 50, 220], [50, 170], s.tables, k, v)
        s.ref, low = mirrored, s.tables
        q = rand(s.g, 151, 4, dim, times=1.5)
        s.tables = tables
        o, lse = attend(s, [1, 150], q)
        s.tables = low
        check(s, [1, 150], q, o, lse)
        del pools, scales, s
        torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------- calls
def test_a_captured_step_follows_the_batch():
    """Write, read and attention in one graph; lengths, tables and tokens change under it.  A second graph shares the
    handle and the workspace."""
    import paper_2608_01150_b200 as Z
    s = Setup(E4M3, 64, 16, 2, [300, 150])
    h = Z.build_cached_attn(6, 2, 64)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    k, v = rand(s.g, 450, 2, 64), rand(s.g, 450, 2, 64)

    def graph_of(qlens):
        n = sum(qlens)
        b = s.batch(qlens, lens=[0, 0], max_q=0)
        t = dict(b=b, k=torch.zeros(n, 2, 64, dtype=BF16, device="cuda"), v=torch.zeros(n, 2, 64, dtype=BF16, device="cuda"),
                 q=torch.zeros(n, 6, 64, dtype=BF16, device="cuda"), o=torch.zeros(n, 6, 64, dtype=BF16, device="cuda"),
                 lse=torch.zeros(6, n, device="cuda"), rk=torch.zeros(n, 2, 64, dtype=BF16, device="cuda"), rv=torch.zeros(n, 2, 64, dtype=BF16, device="cuda"),
                 first=i32([0, 0]))

        def step():
            Z.cache_write(s.cache, b, t["k"], t["v"])
            Z.cache_read(s.cache, b, b.cu_q, t["rk"], t["rv"], first=t["first"])
            Z.cached_attn_fwd(h, s.cache, b, t["q"], 0.125, t["o"], t["lse"], ws)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        return graph, t

    graphs = {(140, 60): graph_of([140, 60]), (1, 1): graph_of([1, 1])}
    lens = [0, 0]
    for qlens in ((140, 60), (1, 1), (1, 1), (140, 60), (1, 1)):
        graph, t = graphs[qlens]
        rows = torch.cat([torch.arange(lens[0], lens[0] + qlens[0]), 300 + torch.arange(lens[1], lens[1] + qlens[1])])
        first, lens = lens, [lens[0] + qlens[0], lens[1] + qlens[1]]
        q = rand(s.g, sum(qlens), 6, 64, times=1.5)
        for name, x in (("k", k[rows]), ("v", v[rows]), ("q", q), ("first", i32(first))):
            t[name].copy_(x)
        t["b"].kv_len.copy_(i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        s.ref.write(cu(qlens), lens, s.tables, k[rows], v[rows])
        check(s, list(qlens), q, t["o"].cpu(), t["lse"].cpu(), lens=lens)
        _, held, _ = s.ref.held(0, lens, s.tables)
        assert (t["rk"][:qlens[0]].cpu().double() - held[first[0]:]).abs().max() <= 2.0 ** -8 * held.abs().max()
    assert h.last_device_status() == (0, 0)


def test_calls_on_other_streams():
    """Two streams with a handle and a workspace each, at the same time; tensors made on the default stream."""
    import paper_2608_01150_b200 as Z
    runs = []
    for seed in (3, 4):
        s = Setup(INT8, 128, 16, 2, [3000, 40], seed=seed)
        s.fill()
        runs.append((s, rand(s.g, 4, 8, 128, times=1.5), Z.build_cached_attn(8, 2, 128), torch.cuda.Stream()))
    alone = [attend(s, [3, 1], q) for s, q, _, _ in runs]
    torch.cuda.synchronize()
    outs = []
    tensors = [(torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda"), q.cuda(), s.batch([3, 1])) for s, q, h, _ in runs]
    torch.cuda.synchronize()
    for (s, q, h, stream), (ws, qd, b) in zip(runs, tensors):
        o, lse = torch.empty_like(qd), torch.empty(8, 4, device="cuda")
        outs.append((o, lse))
        with torch.cuda.stream(stream):
            for _ in range(5):
                Z.cached_attn_fwd(h, s.cache, b, qd, 128 ** -0.5, o, lse, ws)
    torch.cuda.synchronize()
    for (o, lse), (a, b) in zip(outs, alone):
        assert torch.equal(o.cpu(), a) and torch.equal(lse.cpu(), b)


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_token_by_token_is_the_engines_attention(dtype):
    """A prompt in chunks, then single tokens, over the cache, against the engine's masked attention of the whole sequence with
    what the cache holds: both are within their distance of the definition."""
    import paper_2608_01150_b200 as Z
    H, dim, total, prefix = 4, 64, 333, 50
    s = Setup(dtype, dim, 16, H, [total])
    g = s.g
    qkv = [rand(g, total, H, dim) for _ in range(3)]
    q, k, v = (x.cuda() for x in qkv)
    h = Z.build_cached_attn(H, H, dim)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), []
    at = 0
    for n in [50, 130, 64, 1, 3] + [1] * 85:
        b = s.batch([n], lens=[at + n], prefix=[prefix])
        Z.cache_write(s.cache, b, k[at:at + n], v[at:at + n])
        part = torch.empty(H, n, device="cuda")
        Z.cached_attn_fwd(h, s.cache, b, q[at:at + n], 0.125, o[at:at + n], part, ws)
        lse.append(part)
        at += n
    assert at == total
    held = [torch.empty_like(k) for _ in "kv"]
    Z.cache_read(s.cache, s.batch([0]), i32([0, total]), held[0], held[1])
    t = Z.build_tasks([0, total], [], total, total, H, dim)
    t.set_positions([prefix])
    o2, lse2 = torch.empty_like(q), torch.empty(H, total, device="cuda")
    Z.scored_attn_fwd(t, Z.Score(masked=True), q, held[0], held[1], 0.125, o2, lse2)
    torch.cuda.synchronize()
    s.ref.write([0, total], [total], s.tables, qkv[1], qkv[2])
    _, _, bo, bl = R.attention(s.ref, [0, total], [total], s.tables, [prefix], qkv[0], 0.125)
    # cached: the bound; the engine: the same for its own roundings, and in 8 bits the rounding of the values that were read
    # back (2^-8 of every key in a score and of every value)
    kk = 2.0 ** -8 * (qkv[0].double().abs().amax() * dim * 0.125 * qkv[1].double().abs().amax()) if dtype is E4M3 else 0.0
    vmax = qkv[2].double().abs().amax()
    extra = (2 * kk + 2.0 ** -8) * vmax if dtype is E4M3 else 0.0
    assert ((o.cpu().double() - o2.cpu().double()).abs() <= 2 * bo + extra).all()
    assert ((torch.cat(lse, 1).cpu().double() - lse2.cpu().double()).abs() <= 2 * bl + kk).all()


def test_refusals_on_the_gpu():
    import paper_2608_01150_b200 as Z
    s = Setup(BF16, 64, 16, 2, [20])
    b = s.batch([1])
    h = Z.build_cached_attn(4, 2, 64)
    ws = torch.empty(h.workspace_bytes, dtype=torch.uint8, device="cuda")
    q = torch.zeros(1, 4, 64, dtype=BF16, device="cuda")

    def refused(status, q=q, o=None, lse=None, ws=ws, scale=1.0, cache=s.cache, h=h):
        with pytest.raises(Z.ZlError) as e:
            Z.cached_attn_fwd(h, cache, b, q, scale, torch.empty_like(q) if o is None else o, lse, ws)
        assert e.value.status == status
    refused(4, ws=ws[:-256])
    refused(1, ws=ws[8:])
    refused(1, scale=0.0)
    refused(1, q=q.float())
    refused(1, q=q[:, :2])
    refused(1, o=torch.empty(2, 4, 64, dtype=BF16, device="cuda"))
    refused(1, lse=torch.empty(1, 4, device="cuda"))
    refused(1, lse=torch.empty(4, 1))
    refused(1, h=Z.build_cached_attn(4, 4, 64))
    k = torch.zeros(1, 2, 64, dtype=BF16, device="cuda")
    for bad in (k.float(), k[:, :1], k.cpu(), torch.zeros(1, 64, 2, dtype=BF16, device="cuda").transpose(1, 2), k.expand(3, 2, 64)):
        with pytest.raises(Z.ZlError) as e:
            Z.cache_write(s.cache, b, bad, bad)
        assert e.value.status == 1
    with pytest.raises(Z.ZlError):
        Z.cache_read(s.cache, b, i32([0]), k, k)
    with pytest.raises(Z.ZlError):
        Z.cache_read(s.cache, b, i32([0, 1]), k, torch.zeros(1, 2, 128, dtype=BF16, device="cuda")[:, :, ::2])
    # nothing to do is no error
    none = Z.CacheBatch(i32([0]), i32([]), torch.zeros(0, 0, dtype=torch.int32, device="cuda"))
    Z.cache_write(s.cache, none, k[:0], k[:0])
    Z.cache_read(s.cache, none, i32([0]), k, k)
    Z.cached_attn_fwd(h, s.cache, none, q, 1.0, torch.empty_like(q), None, ws)
