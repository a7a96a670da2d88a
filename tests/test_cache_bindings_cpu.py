"""What the Python layer refuses before it calls the cache operators."""
import pytest
import torch

import paper_2608_29539_amd as pk

I32, BF16 = dict(dtype=torch.int32), dict(dtype=torch.bfloat16)


@pytest.mark.parametrize("name", ["cu_prefix", "cu_group"])
@pytest.mark.parametrize("bad,why", [
    (torch.tensor([0, 4]), "int64"),                 # torch's own default
    (torch.tensor([0.0, 4.0]), "float32"),
    (torch.tensor([0, 9, 4, 9], **I32)[::2], "contiguous"),
], ids=["int64", "float", "strided"])
def test_prefix_bounds(name, bad, why):
    """Bounds that a kernel would read as other numbers: an int64 [0, 4] is
    [0, 0, 4, 0] as int32, a prefix of no rows."""
    good = dict(cu_prefix=torch.tensor([0, 4], **I32), cu_group=torch.tensor([0, 4], **I32))
    host = dict(cu_prefix_host=[0, 4], cu_group_host=[0, 4])
    pk.Prefix(**good, **host)
    with pytest.raises(TypeError, match=f"{name}.*{why}"):
        pk.Prefix(**{**good, name: bad}, **host)


@pytest.mark.parametrize("bad,why", [(torch.tensor([0, 4]), "int64"),
                                     (torch.tensor([0, 9, 4, 9], **I32)[::2], "contiguous")],
                         ids=["int64", "strided"])
def test_problem_bounds(bad, why):
    prob = pk.Problem(bad, 4, 2, 64, 8, cu_seqlens_host=[0, 4])
    pre = pk.Prefix(torch.tensor([0, 4], **I32), torch.tensor([0, 1], **I32),
                    cu_prefix_host=[0, 4], cu_group_host=[0, 1])
    q, qn, k = (torch.zeros(s, **BF16) for s in ((1, 4, 64), (4, 4, 64), (4, 2, 64)))
    gate, score = torch.zeros(1), torch.zeros(2, 4)
    for call in (lambda: pk.logo_decode_prefix(prob, pre, q, k, k, k, k, gate, threshold=0.5),
                 lambda: pk.logo_cache_score(prob, qn, k),
                 lambda: pk.logo_decode_score(prob, q, k, gate, threshold=0.5),
                 lambda: pk.logo_cache_evict(prob, score, 2, k=k, v=k)):
        with pytest.raises(TypeError, match=f"cu_seqlens.*{why}"):
            call()
