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


def guarded(nbytes):
    import torch
    return torch.full((nbytes + 4096,), 0xA5, dtype=torch.uint8, device="cuda")


def close(got, want, tol):
    e = (got.double() - want.double()).abs()
    print(f"[edges] max difference {float(e.max()):.3g}", flush=True)
    assert bool((e <= tol).all())


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 4, 64)])
@pytest.mark.parametrize("distinct", [False, True], ids=["shared", "own-global"])
def test_prefix_in_a_longer_step_s_workspace(pk, hq, hkv, d, distinct):
    """A workspace given for the loop's longest step serves the shorter ones,
    and nothing is written behind it."""
    import torch
    rng = np.random.default_rng(4)
    P, B = 1500, 4
    lens = [600, 1, 300, 77]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cup, grp = np.array([0, P], np.int32), np.array([0, B], np.int32)
    dcu, dcp, dcg = (torch.from_numpy(t).cuda() for t in (cu, cup, grp))
    N = int(cu[-1])
    prob = pk.Problem(dcu, hq, hkv, d, 256, cu_seqlens_host=cu)
    pre = pk.Prefix(dcp, dcg, cu_prefix_host=cup, cu_group_host=grp)
    q, kp, vp, k, v = (bf16(rng, *s) for s in ((B, hq, d), (P, hkv, d), (P, hkv, d), (N, hkv, d),
                                               (N, hkv, d)))
    kw = dict(q_g=bf16(rng, B, hq, d), k_pre_g=vp, v_pre_g=kp, k_g=v, v_g=k) if distinct else {}
    gate = torch.tensor([0.9, 0.8, 0.1, 0.6], device="cuda")
    args = (prob, pre, q, kp, vp, k, v, gate)
    want = pk.logo_decode_prefix(*args, threshold=0.5, **kw)[0]
    need = pk.logo_decode_prefix_workspace_bytes(prob, pre)
    # the least: a chunk for each of the four key ranges (two of which the
    # window may leave empty)
    least = 4 * B * hq * (d + 2) * 4 + 512
    for nbytes in (need, need - need // 4, need // 2, least):
        ws = guarded(nbytes)
        got = pk.logo_decode_prefix(*args, threshold=0.5, ws=ws[:nbytes], **kw)[0]
        torch.cuda.synchronize()
        assert bool((ws[nbytes:] == 0xA5).all()), nbytes
        # (fp32 sums in another order may round to the next bf16 number)
        close(got, want, 2.0 ** -7 * want.float().abs() + 1e-5)
    with pytest.raises(pk.LogoError, match="WORKSPACE"):
        pk.logo_decode_prefix(*args, threshold=0.5, ws=ws[:256], **kw)


def test_score_in_more_rows_workspace(pk):
    import torch
    rng = np.random.default_rng(5)
    N, hq, hkv, d = 9000, 8, 2, 128
    cu = torch.tensor([0, N], dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, hq, hkv, d, 64, cu_seqlens_host=[0, N])
    q, k = bf16(rng, N, hq, d), bf16(rng, N, hkv, d)
    sel = torch.arange(N - 40, N, dtype=torch.int32, device="cuda")
    kw = dict(sel_idx=sel, cu_sel=torch.tensor([0, 40], dtype=torch.int32, device="cuda"))
    want = pk.logo_cache_score(prob, q, k, **kw)
    need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_CACHE_SCORE, 40)
    least = -(-8 * 40 * hq // 256) * 256
    assert need > 4 * least
    for nbytes in (need, need // 2, least):
        ws = guarded(nbytes)
        got = pk.logo_cache_score(prob, q, k, ws=ws[:nbytes], **kw)
        torch.cuda.synchronize()
        assert bool((ws[nbytes:] == 0xA5).all()), nbytes
        # (the log-sum-exp's terms in other groups: 9000 fp32 additions)
        close(got, want, want * 9000 * 2.0 ** -24)
    with pytest.raises(pk.LogoError, match="WORKSPACE"):
        pk.logo_cache_score(prob, q, k, ws=ws[:least - 256], **kw)


def test_step_in_longer_caches_workspace(pk):
    import torch
    rng = np.random.default_rng(6)
    lens, hq, hkv, d = [3000, 1, 2777], 20, 4, 64
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    prob = pk.Problem(torch.from_numpy(cu).cuda(), hq, hkv, d, 64, cu_seqlens_host=cu)
    q, k = bf16(rng, 3, hq, d), bf16(rng, int(cu[-1]), hkv, d)
    gate = torch.tensor([0.9, 0.9, 0.9], device="cuda")
    want = pk.logo_decode_score(prob, q, k, gate, threshold=0.5)
    need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_DECODE_SCORE)
    logits = -(-4 * (hq * int(cu[-1]) + 1) // 256) * 256
    assert need > logits + 4 * 8 * 3 * hq
    for nbytes in (need, logits + (need - logits) // 2, logits + 512):
        ws = guarded(nbytes)
        got = pk.logo_decode_score(prob, q, k, gate, threshold=0.5, ws=ws[:nbytes])
        torch.cuda.synchronize()
        assert bool((ws[nbytes:] == 0xA5).all()), nbytes
        close(got, want, want * 3000 * 2.0 ** -24)
    with pytest.raises(pk.LogoError, match="WORKSPACE"):
        pk.logo_decode_score(prob, q, k, gate, threshold=0.5, ws=ws[:logits])


def test_evict_into_far_more_room_than_rows(pk):
    """A capacity far above the kept rows (the stride of score_out and
    keep_idx; one head has no second row of them)."""
    import ctypes

    import torch
    L, cap = 300, 1 << 30
    cu = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, 1, 1, 64, 8, cu_seqlens_host=[0, L])
    rng = np.random.default_rng(7)
    k, v, score = bf16(rng, L, 1, 64), bf16(rng, L, 1, 64), torch.rand((1, L), device="cuda")
    want = pk.logo_cache_evict(prob, score, 40, recent=5, k=k, v=v)
    got = {n: torch.zeros_like(t) for n, t in want.items() if t is not None}
    p = {n: ctypes.c_void_p(t.data_ptr()) for n, t in dict(got, k=k, v=v, score=score).items()}
    st = pk.library().logo_cache_evict(
        prob.c, p["score"], 40, 5, p["k"], p["v"], None, None, p["k_out"], p["v_out"], None, None,
        p["score_out"], p["keep_idx"], p["cu_keep"], cap, None, 0,
        ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert st == 0, pk.logo_status_str(st)
    for n in got:
        assert torch.equal(got[n], want[n]), n
