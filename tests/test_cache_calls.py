"""What the binding and the library make of the paged cache's arguments, without a GPU."""
import ctypes

import pytest
import torch

import paper_2608_01150_b200 as Z
from paper_2608_01150_b200 import binding as B

no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="calls without a device")
OK, INVALID, UNSUPPORTED, CUDA = 0, 1, 3, 5


def pool(fmt=torch.bfloat16, pages=4, page=16, heads=2, dim=64):
    k = torch.zeros(pages, page, heads, dim).to(fmt)
    sc = [None, None] if fmt is torch.bfloat16 else [torch.zeros(pages, page, heads) for _ in "kv"]
    return k, torch.zeros_like(k), *sc


def batch(n=2, pages=3, prefix=None, max_q=0):
    return Z.CacheBatch(torch.zeros(n + 1, dtype=torch.int32), torch.zeros(n, dtype=torch.int32),
                        torch.zeros(n, pages, dtype=torch.int32), prefix=prefix, max_q=max_q)


def refused(call, status=INVALID):
    with pytest.raises(Z.ZlError) as e:
        call()
    assert e.value.status == status


def cache_desc(**kw):
    f = dict(k=4096, v=8192, k_scale=None, v_scale=None, page_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64,
             scale_page_stride=32, scale_token_stride=2, scale_head_stride=1, n_pages=4,
             page_size=16, n_kv_heads=2, head_dim=64, format=0)
    f.update(kw)
    return B.KvCacheDesc(**f)


def batch_desc(**kw):
    f = dict(cu_q=4096, kv_len=4096, pages=4096, prefix=None, n_seqs=2, max_pages=3, total_q=5, max_q=0)
    f.update(kw)
    return B.CacheBatchDesc(**f)


# ---------------------------------------------------------------------------------------------- what the Python objects refuse
@pytest.mark.parametrize("fmt", [torch.bfloat16, torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("layout", ["tokens", "heads", "together"])
def test_a_cache_describes_its_layout(fmt, layout):
    k, v, ks, vs = pool(fmt, 4, 16, 2, 64)
    if layout == "heads":
        k, v = (torch.zeros(4, 2, 16, 64).to(fmt).transpose(1, 2) for _ in "kv")
    if layout == "together":
        both = torch.zeros(4, 2, 16, 2, 64).to(fmt)
        k, v = both[:, 0], both[:, 1]
    d = Z.KvCache(k, v, ks, vs).desc
    want = dict(tokens=(2048, 128, 64), heads=(2048, 64, 1024), together=(4096, 128, 64))[layout]
    assert (d.page_stride, d.token_stride, d.head_stride) == want
    assert (d.n_pages, d.page_size, d.n_kv_heads, d.head_dim) == (4, 16, 2, 64)
    assert d.k == k.data_ptr() and d.v == v.data_ptr() and (d.k_scale or None) == (ks.data_ptr() if ks is not None else None)


def test_a_cache_follows_its_attributes():
    k, v, ks, vs = pool(torch.int8)
    c = Z.KvCache(k, v, ks, vs)
    other = torch.zeros_like(ks)
    c.k_scale = other
    assert c.desc.k_scale == other.data_ptr()
    c.k = torch.zeros(4, 16, 2, 64)
    refused(lambda: c.desc)


@pytest.mark.parametrize("bad", ["type", "types", "shape", "strides", "rows", "no_scale", "one_scale", "scale_type", "scale_shape", "scale_strides", "bf16_scale"])
def test_unfit_caches_are_refused(bad):
    k, v, ks, vs = pool(torch.int8)
    if bad == "type":
        k, v = k.float(), v.float()
    elif bad == "types":
        v = v.to(torch.float8_e4m3fn)
    elif bad == "shape":
        v = v[:3]
    elif bad == "strides":
        v = torch.zeros(4, 2, 16, 64, dtype=torch.int8).transpose(1, 2)
    elif bad == "rows":
        k, v = (torch.zeros(4, 16, 64, 2, dtype=torch.int8).transpose(2, 3) for _ in "kv")
    elif bad == "no_scale":
        ks = vs = None
    elif bad == "one_scale":
        vs = None
    elif bad == "scale_type":
        ks = ks.double()
    elif bad == "scale_shape":
        ks = ks[:, :, :1].contiguous()
    elif bad == "scale_strides":
        ks = torch.zeros(4, 2, 16).transpose(1, 2)
    elif bad == "bf16_scale":
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    refused(lambda: Z.KvCache(k, v, ks, vs))


@pytest.mark.parametrize("bad", ["cu_len", "cu_type", "len_type", "len_dims", "pages_rows", "pages_type", "pages_strides", "prefix", "max_q"])
def test_unfit_batches_are_refused(bad):
    i32 = torch.int32
    cu, lens, pages, prefix, max_q = torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2, 3, dtype=i32), None, 0
    if bad == "cu_len":
        cu = torch.zeros(2, dtype=i32)
    elif bad == "cu_type":
        cu = cu.long()
    elif bad == "len_type":
        lens = lens.long()
    elif bad == "len_dims":
        lens = lens[None]
    elif bad == "pages_rows":
        pages = torch.zeros(3, 3, dtype=i32)
    elif bad == "pages_type":
        pages = pages.float()
    elif bad == "pages_strides":
        pages = torch.zeros(3, 2, dtype=i32).t()
    elif bad == "prefix":
        prefix = torch.zeros(3, dtype=i32)
    elif bad == "max_q":
        max_q = 2 ** 31
    refused(lambda: Z.CacheBatch(cu, lens, pages, prefix, max_q))


def test_tensors_that_are_not_on_the_gpu_are_refused():
    c, b = Z.KvCache(*pool()), batch()
    x = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    refused(lambda: Z.cache_write(c, b, x, x))
    refused(lambda: Z.cache_read(c, b, torch.zeros(3, dtype=torch.int32), x, x))
    h = Z.build_cached_attn(4, 2, 64)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    refused(lambda: Z.cached_attn_fwd(h, c, b, q, 1.0, q, None, torch.zeros(256, dtype=torch.uint8)))


# ---------------------------------------------------------------------------------------------- what the library refuses
@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), UNSUPPORTED), (dict(format=3), UNSUPPORTED), (dict(format=-1), UNSUPPORTED), (dict(page_size=4), UNSUPPORTED),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=0), INVALID), (dict(page_size=1 << 25), UNSUPPORTED), (dict(n_pages=-1), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(k=None), INVALID), (dict(v=8200), INVALID), (dict(page_stride=2052), INVALID),
    (dict(token_stride=-128), INVALID), (dict(token_stride=32), INVALID), (dict(head_stride=0), INVALID), (dict(page_stride=0), INVALID),
    (dict(format=1), INVALID), (dict(format=2, k_scale=4096), INVALID), (dict(format=1, k_scale=4098, v_scale=4096), INVALID),
    (dict(k_scale=4096), INVALID), (dict(scale_page_stride=-1), INVALID), (dict(format=1, k_scale=4096, v_scale=4096, scale_token_stride=0), INVALID),
    (dict(format=2, k_scale=4096, v_scale=4096, scale_head_stride=0), INVALID), (dict(format=2, k_scale=4096, v_scale=4096, scale_page_stride=0), INVALID),
    (dict(format=1, k_scale=4096, v_scale=4096, token_stride=136), INVALID)])
def test_caches_the_library_refuses(kw, status):
    lib, c, b = B.lib(), cache_desc(**kw), batch_desc()
    assert lib.zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == status
    assert lib.zl_cache_read(ctypes.byref(c), ctypes.byref(b), None, 4096, 5, 4096, 4096, 0) == status


@pytest.mark.parametrize("kw", [dict(n_seqs=-1), dict(max_pages=-1), dict(total_q=-1), dict(max_q=-1), dict(cu_q=None), dict(kv_len=None), dict(pages=None)])
def test_batches_the_library_refuses(kw):
    c, b = cache_desc(), batch_desc(**kw)
    assert B.lib().zl_cache_write(ctypes.byref(c), ctypes.byref(b), 4096, 4096, 128, 0) == INVALID


def test_rows_the_library_refuses():
    lib, c, b = B.lib(), ctypes.byref(cache_desc()), ctypes.byref(batch_desc())
    write = lambda k=4096, v=4096, stride=128, b=b: lib.zl_cache_write(c, b, k, v, stride, 0)  # noqa: E731
    assert write(b=ctypes.byref(batch_desc(max_pages=2 ** 26 + 1))) == UNSUPPORTED  # more than 2^30 positions
    assert write(k=None) == INVALID and write(v=4104) == INVALID and write(stride=132) == INVALID and write(stride=120) == INVALID
    assert lib.zl_cache_write(None, b, 4096, 4096, 128, 0) == INVALID and lib.zl_cache_write(c, None, 4096, 4096, 128, 0) == INVALID
    three = ctypes.byref(cache_desc(n_kv_heads=3, token_stride=192, page_stride=16 * 192))  # 2^32 rows and more
    assert lib.zl_cache_write(three, ctypes.byref(batch_desc(total_q=2 ** 31 - 1)), 4096, 4096, 192, 0) == UNSUPPORTED
    read = lambda cu=4096, total=5, k=4096, v=4096: lib.zl_cache_read(c, b, None, cu, total, k, v, 0)  # noqa: E731
    assert read(cu=None) == INVALID and read(total=-1) == INVALID and read(k=None) == INVALID and read(v=4100) == INVALID
    assert lib.zl_cache_read(three, b, None, 4096, 2 ** 31 - 1, 4096, 4096, 0) == UNSUPPORTED


@pytest.mark.parametrize("args,status", [((0, 1, 64), INVALID), ((4, 0, 64), INVALID), ((5, 2, 64), INVALID), ((-4, -2, 64), INVALID),
                                         ((4, 2, 80), UNSUPPORTED), ((129, 1, 64), UNSUPPORTED), ((2 ** 31, 1, 64), INVALID)])
def test_handles_that_are_refused(args, status):
    refused(lambda: Z.build_cached_attn(*args), status)


def test_attention_calls_the_library_refuses():
    lib, h = B.lib(), Z.build_cached_attn(4, 2, 64)

    def call(c=None, b=None, q=4096, stride=256, scale=1.0, o=65536, lse=None):
        return lib.zl_cached_attn_fwd(h.ptr, ctypes.byref(c or cache_desc()), ctypes.byref(b or batch_desc()), q, stride, scale, o, lse, 4096, 1 << 40, 0)

    assert call(c=cache_desc(n_kv_heads=4)) == INVALID and call(c=cache_desc(head_dim=128, token_stride=256, head_stride=128)) == INVALID
    for scale in (0.0, -1.0, float("inf"), float("nan"), 3e38):
        assert call(scale=scale) == INVALID
    assert call(o=4096) == INVALID and call(o=4096 + 4 * 512 + 496) == INVALID and call(o=4096 - 2560 + 16) == INVALID  # over the queries
    assert call(q=None) == INVALID and call(o=None) == INVALID and call(q=4104) == INVALID and call(stride=252) == INVALID
    assert call(stride=248) == INVALID and call(lse=4098) == INVALID and call(b=batch_desc(kv_len=None)) == INVALID
    assert call(c=cache_desc(format=7)) == UNSUPPORTED and call(b=batch_desc(total_q=2 ** 31 - 1)) == UNSUPPORTED
    assert lib.zl_cached_attn_fwd(None, ctypes.byref(cache_desc()), ctypes.byref(batch_desc()), 4096, 256, 1.0, 4096, None, 4096, 1 << 40, 0) == INVALID


@no_device
def test_calls_without_a_device_say_so():
    lib, c, b = B.lib(), ctypes.byref(cache_desc()), ctypes.byref(batch_desc())
    assert lib.zl_cache_write(c, b, 4096, 4096, 128, 0) == CUDA
    assert lib.zl_cache_read(c, b, None, 4096, 5, 4096, 4096, 0) == CUDA
    h = Z.build_cached_attn(4, 2, 64)
    assert lib.zl_cached_attn_fwd(h.ptr, c, b, 4096, 256, 1.0, 65536, None, 4096, 1 << 40, 0) == CUDA
    assert lib.zl_cached_attn_fwd(h.ptr, c, b, 4096, 256, 1.0, 4096 + 2560, None, 4096, 1 << 40, 0) == CUDA  # right behind the queries
    code, where = ctypes.c_int32(), ctypes.c_int32()
    assert lib.zl_cached_attn_device_status(h.ptr, ctypes.byref(code), ctypes.byref(where)) == CUDA
    h.close()
    h.close()
