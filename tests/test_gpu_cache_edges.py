"""GPU tests of the cache operators at the ends of what their documentation
allows."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu tests need an MI355X")
    import paper_2608_29539_amd as pk
    pk.library()
    return pk


def bf16(rng, *shape):
    import torch
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(torch.bfloat16)


@pytest.mark.parametrize("lists", [False, True], ids=["output-alone", "lists"])
@pytest.mark.parametrize("d", [64, 128])
def test_prefix_no_cache_has_a_row(pk, d, lists):
    """Without host copies, a batch of empty caches behind empty prefixes
    outputs zeros, and lists its selected sequences."""
    import torch
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    grp = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, 4, 2, d, 8, total_tokens=0, max_seqlen=0)
    pre = pk.Prefix(cu[:3].clone(), grp, total_tokens=0, max_prefix=0, max_group=2)
    q, none = bf16(np.random.default_rng(1), 3, 4, d), torch.empty((0, 2, d), dtype=torch.bfloat16,
                                                                  device="cuda")
    gate = torch.tensor([0.7, 0.2, 0.9], device="cuda")
    out = torch.full((3, 4, d), 5.0, dtype=torch.bfloat16, device="cuda")
    kw = {}
    if lists:
        kw = dict(active=torch.full((3,), -7, dtype=torch.int32, device="cuda"),
                  n_active=torch.full((1,), -7, dtype=torch.int32, device="cuda"))
    pk.logo_decode_prefix(prob, pre, q, none, none, none, none, gate, threshold=0.5, out=out, **kw)
    torch.cuda.synchronize()
    assert bool((out == 0).all())
    if lists:
        assert kw["active"].tolist() == [0, 2, -7] and kw["n_active"].tolist() == [2]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("thr", [-math.inf, math.inf], ids=["global", "local"])
def test_prefix_empty_cache_without_eps(pk, d, thr):
    """Zeros for a sequence without rows also where eps = 0 would divide them
    by zero; its neighbour's output stays."""
    import torch
    rng = np.random.default_rng(2)
    cu, cup = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 0, 5], [0, 0, 30]))
    grp = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, 4, 2, d, 8, total_tokens=5, max_seqlen=5)
    pre = pk.Prefix(cup, grp, total_tokens=30, max_prefix=30, max_group=1)
    q, gate = bf16(rng, 2, 4, d), torch.tensor([0.7, 0.4], device="cuda")
    t = [bf16(rng, n, 2, d) for n in (30, 30, 5, 5)]
    got = {eps: pk.logo_decode_prefix(prob, pre, q, *t, gate, threshold=thr, eps=eps)[0]
           for eps in (0.0, 1e-12)}
    torch.cuda.synchronize()
    assert bool((got[0.0][0] == 0).all())
    assert bool(torch.isfinite(got[0.0]).all()) and bool((got[0.0][1] != 0).any())
    # (1e-12 in a mean square near one moves no bf16 rounding but a tie's)
    assert bool(((got[0.0] - got[1e-12]).float().abs() <= 2.0 ** -7 * got[0.0].float().abs()).all())


def test_workspace_of_one_stored_byte(pk):
    """An expanded workspace has the bytes that are asked for, but not the
    memory: every operator refuses it."""
    import torch
    rng = np.random.default_rng(3)
    n = 20000                                    # (more rows than an eviction's part)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, 2, 2, 64, 8, cu_seqlens_host=[0, n])
    pre = pk.Prefix(cu, one, cu_prefix_host=[0, n], cu_group_host=[0, 1])
    q, qn, k = bf16(rng, 1, 2, 64), bf16(rng, n, 2, 64), bf16(rng, n, 2, 64)
    gate, score = torch.ones(1, device="cuda"), torch.rand((2, n), device="cuda")
    ws = torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 30)
    for call in (lambda: pk.logo_decode_prefix(prob, pre, q, k, k, k, k, gate, threshold=0.5, ws=ws),
                 lambda: pk.logo_cache_score(prob, qn, k, ws=ws),
                 lambda: pk.logo_decode_score(prob, q, k, gate, threshold=0.5, ws=ws),
                 lambda: pk.logo_cache_evict(prob, score, 2, k=k, v=k, ws=ws)):
        with pytest.raises(ValueError, match="ws must be contiguous"):
            call()
