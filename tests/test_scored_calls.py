"""What the binding and the library make of a scored call's arguments, without a GPU."""
import pytest
import torch

import paper_2608_01150_b200 as Z
from paper_2608_01150_b200 import binding as B


# ---------------------------------------------------------------------------------------------- a Score follows its attributes
def buckets(n, H, dist):
    return dict(bucket_bias=torch.nn.Parameter(torch.zeros(n, H)), bucket_of=torch.zeros(2 * dist + 1, dtype=torch.int32))


def test_a_score_reads_its_tensors_at_the_call():
    """Moving a module swaps its parameters' storage under a Score that was made before."""
    s = Z.Score(slopes=torch.nn.Parameter(torch.zeros(3)), **buckets(4, 3, 2))
    for name, field in (("slopes", "slopes"), ("bucket_bias", "bucket_bias"), ("bucket_of", "bucket_of")):
        t = getattr(s, name)
        kept = t.data                                   # the old storage stays alive: the new address is another
        t.data = t.data.clone()
        assert t.data_ptr() != kept.data_ptr() and getattr(s.desc, field) == t.data_ptr(), name
        other = t.detach().clone()
        setattr(s, name, other)
        assert getattr(s.desc, field) == other.data_ptr(), name


def test_a_score_follows_its_numbers_and_sizes():
    s = Z.Score(cap=2.0)
    s.cap, s.masked = 3.0, True
    assert s.desc.cap == 3.0 and s.desc.masked == 1
    assert s.desc.n_buckets == 0 and s.desc.max_distance == 0 and not s.desc.bucket_bias and not s.desc.bucket_of
    new = buckets(7, 3, 5)
    s.bucket_bias, s.bucket_of = new["bucket_bias"], new["bucket_of"]
    assert s.desc.n_buckets == 7 and s.desc.max_distance == 5
    h = Z.build_tasks([0, 10], [], 10, 10, 3, 64)
    h.set_positions([0])
    with_table = h.scored_workspace_bytes(s)
    s.bucket_bias = s.bucket_of = None
    assert h.scored_workspace_bytes(s) == with_table - 3 * Z.MAX_BUCKETS * 4


@pytest.mark.parametrize("name,value", [
    ("slopes", torch.zeros(3, dtype=torch.float64)), ("slopes", torch.zeros(3, 1)), ("bucket_bias", torch.zeros(3, 4).t()), ("bucket_bias", None),
    ("bucket_of", None), ("bucket_of", torch.zeros(4, dtype=torch.int32)), ("bucket_of", torch.zeros(5, dtype=torch.int64))])
def test_a_score_with_unfit_attributes_is_refused_at_the_call(name, value):
    s = Z.Score(slopes=torch.zeros(3), **buckets(4, 3, 2))
    h = Z.build_tasks([0, 10], [], 10, 10, 3, 64)
    setattr(s, name, value)
    with pytest.raises(Z.ZlError) as e:
        h.scored_workspace_bytes(s)
    assert e.value.status == 1
    with pytest.raises(Z.ZlError) as e:
        Z.scored_attn_fwd(h, s, 0, 0, 0, 1.0, 0, 0)
    assert e.value.status == 1


def test_a_table_gradient_that_is_not_on_the_gpu_is_refused():
    """It is written by a kernel; shape, type and layout alone do not make its address one that a kernel can use."""
    s = Z.Score(**buckets(4, 3, 2))
    with pytest.raises(Z.ZlError) as e:
        B._check_table(s, torch.zeros(4, 3))
    assert e.value.status == 1 and "GPU" in str(e.value)
    B._check_table(s, None)
    B._check_table(s, 4096)      # raw addresses are the caller's word, as everywhere in the binding
