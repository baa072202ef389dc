"""The paged cache's descriptions at their limits and when they change, without a GPU."""
import ctypes

import pytest
import torch

import cache_bounds
import cache_ref as R
import paper_2608_01150_b200 as Z
from paper_2608_01150_b200 import binding as B
from test_cache_calls import CUDA, INVALID, batch_desc, cache_desc, no_device, pool


# ---------------------------------------------------------------------------------------------- limits
@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("name", ["page_stride", "token_stride", "head_stride"])
def test_strides_fit_32_bits_in_units_of_16_bytes(fmt, name):
    """2^35 bf16 elements are 2^32 such units: none of them is left in 32 bits."""
    lib, b = B.lib(), batch_desc()
    scales = dict(k_scale=4096, v_scale=4096) if fmt else {}
    c = cache_desc(format=fmt, **scales, **{name: 1 << 35})
    assert lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == INVALID


@no_device
@pytest.mark.parametrize("name", ["page_stride", "token_stride", "head_stride"])
def test_the_largest_strides_are_taken(name):
    lib, c, b = B.lib(), cache_desc(**{name: (1 << 35) - 8}), batch_desc()
    assert lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == CUDA


# ---------------------------------------------------------------------------------------------- changes in place
def refused(call):
    with pytest.raises(Z.ZlError) as e:
        call()
    assert e.value.status == INVALID


def test_a_batch_follows_changes_of_shape_in_place():
    """The address stays, the number of sequences does not."""
    i32 = torch.int32
    cu, lens, pages, prefix = torch.zeros(5, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(4, 3, dtype=i32), torch.zeros(4, dtype=i32)
    b = Z.CacheBatch(cu, lens, pages, prefix)
    now = lambda: b._look(None)[-1]  # noqa: E731
    assert now().n_seqs == 4
    lens.resize_(2)
    refused(now)
    cu.resize_(3), prefix.resize_(2)
    refused(now)  # (the table still has four rows)
    pages.resize_(2, 3)
    assert now().n_seqs == 2 and now().max_pages == 3


@pytest.mark.parametrize("name", ["cu_q", "kv_len", "pages", "prefix"])
@pytest.mark.parametrize("what", ["shape", "type", "strides"])
def test_a_batch_whose_tensors_no_longer_fit_is_refused(name, what):
    i32 = torch.int32
    b = Z.CacheBatch(torch.zeros(5, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(4, 3, dtype=i32), torch.zeros(4, dtype=i32))
    t = getattr(b, name)
    if what == "shape":
        t.data = t.data[:2]
    elif what == "type":
        t.data = t.data.view(torch.float32)
    else:
        t.as_strided_(t.shape, (0,) * t.dim())
    refused(lambda: b._look(None))


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
@pytest.mark.parametrize("what", ["shape", "type", "strides"])
def test_a_cache_whose_tensors_no_longer_fit_is_refused(name, what):
    c = Z.KvCache(*pool(torch.int8))
    t = getattr(c, name)
    before = t.data_ptr()
    if what == "shape":
        t.data = t.data[:3]
    elif what == "type":
        t.data = t.data.view(torch.uint8 if name in "kv" else torch.int32)
    else:
        t.as_strided_(t.shape, (1,) * t.dim())
    assert t.data_ptr() == before
    refused(lambda: c.desc)


def test_a_cache_that_changes_as_a_whole_is_followed():
    k, v, ks, vs = pool(torch.int8)
    c = Z.KvCache(k, v, ks, vs)
    for t in (k, v, ks, vs):
        t.data = t.data[:3]
    assert c.desc.n_pages == 3


# ---------------------------------------------------------------------------------------------- bounds of 8-bit caches
@pytest.mark.parametrize("top", [2.0 ** 120, 1.0, 1.9921875 * 2.0 ** -20, 2.0 ** -98, 2.0 ** -126])
def test_queries_in_fp16_are_off_by_2_to_the_minus_39_of_the_largest(top):
    """All mantissas and every exponent below the largest one's; what is 2^-31 of it or more stays as it is."""
    m = 1 + torch.arange(128, dtype=torch.float64) / 128
    q = torch.cat([m * top * 2.0 ** -i for i in range(1, 60)]).to(torch.bfloat16)
    q = torch.cat([torch.tensor([top], dtype=torch.bfloat16), q, -q])
    got, q = cache_bounds.to_half(q), q.double()
    off = (got - q).abs()
    assert off.max() <= 2.0 ** -39 * top
    assert (off[q.abs() >= 2.0 ** -31 * top] == 0).all()
    if top >= 2.0 ** -80:
        assert off.max() > 2.0 ** -40 * top  # half of it would not do
    if top <= 2.0 ** -98:  # (the last bit of any bf16 is 2^-133, times at least 2^112 a multiple of 2^-24)
        assert (off == 0).all()


def near_pairs(dtype):
    """Sequences of two keys whose values cancel and whose weights are nearly the same: O is small, and what rounding the weights
    leaves is most of its error."""
    g = torch.Generator().manual_seed(7)
    S, heads, dim = 60, 2, 64
    ref = R.Ref(S, 8, heads, dim, dtype)
    k = torch.randn(2 * S, heads, dim, generator=g).to(torch.bfloat16)
    v = torch.randn(S, heads, dim, generator=g).to(torch.bfloat16)
    v = torch.stack([v, -v], 1).reshape(2 * S, heads, dim)
    q = (torch.randn(S, 2 * heads, dim, generator=g) * 0.05).to(torch.bfloat16)
    cu, tables = list(range(0, 2 * S + 1, 2)), [[i] for i in range(S)]
    ref.write(cu, [2] * S, tables, k, v)
    return ref, tables, k, v, q


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_the_bounds_tell_fp16_weights_from_bf16_ones(dtype):
    ref, tables, _, _, q = near_pairs(dtype)
    S = len(tables)

    def worst(weights):
        O, _, bo, _ = cache_bounds.attention8(ref, list(range(S + 1)), [2] * S, tables, None, q, 0.125)
        o = cache_bounds.attention8(ref, list(range(S + 1)), [2] * S, tables, None, q, 0.125, weights)[0]
        return ((o.to(torch.bfloat16).double() - O).abs() / bo).max()

    assert worst(None) <= 1 and worst(lambda u: u.half().double()) <= 1
    assert worst(lambda u: u.to(torch.bfloat16).double()) > 1.5
