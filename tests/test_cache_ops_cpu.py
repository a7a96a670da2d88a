"""The cache operators without a GPU: their 64-bit references against cases
worked out by hand, sizes that the library answers on the host, and every
refusal (no call here reaches a launch)."""
import ctypes
import os

import numpy as np
import pytest

import _cache_ops as ref
import synth
from test_abi_cpu import (ERR_ARG, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, FAKE, OK,
                          Prob)

MISALIGNED = ctypes.c_void_p(0x1008)


@pytest.fixture(scope="module")
def lib():
    import paper_2608_29539_amd as pk
    if not os.path.exists(pk.library_path()):
        from paper_2608_29539_amd.build import build_library
        build_library()
    return pk.library()


class Pre:
    def __init__(self, prefixes=(100, 30), groups=(1, 1), host=True, **kw):
        import paper_2608_29539_amd.binding as b
        self.cp = np.concatenate([[0], np.cumsum(prefixes)]).astype(np.int32)
        self.cg = np.concatenate([[0], np.cumsum(groups)]).astype(np.int32)
        ptr = [x.ctypes.data_as(ctypes.c_void_p) for x in (self.cp, self.cg)]
        f = dict(num_prefixes=len(prefixes), total_tokens=int(self.cp[-1]),
                 max_prefix=max(prefixes), max_group=max(groups))
        f.update(kw)
        self.s = b._Prefix(f["num_prefixes"], f["total_tokens"], f["max_prefix"], f["max_group"],
                           ptr[0], ptr[1], *(ptr if host else (None, None)))

    @property
    def c(self):
        return ctypes.byref(self.s)


# --- the references ------------------------------------------------------------
def test_evict_reference_by_hand():
    nan = float("nan")
    s = np.array([[3, 1, 3, nan, 2, 9, 9, -0.0, 0.0, -1]], np.float32)
    cu = np.array([0, 10], np.int32)
    kept, ck = ref.evict(s, cu, 4, 1)       # 9 (recent), then 5, 6 and the first 3
    assert kept.tolist() == [[0, 5, 6, 9]] and ck.tolist() == [0, 4]
    kept, _ = ref.evict(s, cu, 7, 0)        # -0 and 0 tie: the lower index
    assert kept.tolist() == [[0, 1, 2, 4, 5, 6, 7]]
    kept, _ = ref.evict(s, cu, 9, 0)        # NaN goes first
    assert kept.tolist() == [[0, 1, 2, 4, 5, 6, 7, 8, 9]]
    kept, _ = ref.evict(s, cu, 3, 8)        # more recent rows than the budget
    assert kept.tolist() == [[7, 8, 9]]


def test_score_reference_by_hand():
    """Two keys, one head: scores 0 and log2(3) in the exp2 domain."""
    d = 64
    k = np.zeros((2, 1, d), np.float32)
    k[1, 0, 0] = 1.0
    q = np.zeros((2, 1, d), np.float32)
    q[1, 0, 0] = 2.0
    bits = [synth.bf16_bits_from_f32(t.reshape(-1)).reshape(t.shape) for t in (q, k)]
    c = np.log2(np.e) / 8
    w = np.exp2(2 * c)
    got, _ = ref.scores_of(*bits, [0, 1], [0, 2], [2])
    np.testing.assert_allclose(got, [[1 + 1 / (1 + w), w / (1 + w)]], rtol=1e-12)
    step, _ = ref.step_scores(bits[0][1:], bits[1], [0, 2], [True])
    np.testing.assert_allclose(step, [[1 / (1 + w), w / (1 + w)]], rtol=1e-12)


# --- sizes ---------------------------------------------------------------------
def test_keep_capacity(lib):
    assert lib.logo_cache_keep_capacity(Prob((100, 50)).c, 60) == 110
    assert lib.logo_cache_keep_capacity(Prob((100, 50)).c, 1 << 30) == 150
    assert lib.logo_cache_keep_capacity(Prob((100, 50), host=False).c, 60) == 120
    assert lib.logo_cache_keep_capacity(Prob((100, 50), host=False).c, 90) == 150
    assert lib.logo_cache_keep_capacity(Prob((100, 50)).c, 0) == -1
    assert lib.logo_cache_keep_capacity(Prob(d=96).c, 5) == -1


def test_workspaces(lib):
    import paper_2608_29539_amd as pk
    p = Prob((1000, 50), hq=8, hkv=2)
    need = lib.logo_workspace_bytes(p.c, pk.LOGO_ENTRY_DECODE_SCORE, 0)
    assert need >= 4 * 8 * 1050
    assert lib.logo_workspace_bytes(p.c, pk.LOGO_ENTRY_CACHE_SCORE, 100) >= 4 * 8 * 100
    assert lib.logo_decode_prefix_workspace_bytes(p.c, Pre().c) > 0
    assert lib.logo_decode_prefix_workspace_bytes(p.c, Pre(groups=(3, 1)).c) == 0
    assert lib.logo_decode_prefix_workspace_bytes(Prob(d=96).c, Pre().c) == 0
    assert lib.logo_decode_prefix_workspace_bytes(p.c, None) == 0


# --- refusals ------------------------------------------------------------------
def test_prefix_refusals(lib):
    p = Prob((10, 20))

    def dec(p=p, x=None, q=FAKE, kp=FAKE, vp=FAKE, k=FAKE, v=FAKE, qg=None, kpg=None, vpg=None,
            kg=None, vg=None, gate=FAKE, mode=0, thr=0.5, thr_dev=None, eps=1e-6, out=FAKE,
            ws=FAKE, ws_bytes=1 << 40):
        x = x or Pre()
        return lib.logo_decode_prefix(p.c, x.c, q, kp, vp, k, v, qg, kpg, vpg, kg, vg, gate, mode,
                                      thr, thr_dev, None, None, eps, out, None, None, ws,
                                      ws_bytes, None)

    for name in ("q", "kp", "vp", "k", "v", "gate", "out"):
        assert dec(**{name: None}) == ERR_NULL, name
    for name in ("q", "kp", "vp", "k", "v", "out"):
        assert dec(**{name: MISALIGNED}) == ERR_ARG, name
    assert dec(qg=MISALIGNED) == ERR_ARG
    assert lib.logo_decode_prefix(p.c, None, *[FAKE] * 5, *[None] * 5, FAKE, 0, 0.5, None, None,
                                  None, 1e-6, FAKE, None, None, FAKE, 1 << 40, None) == ERR_NULL
    # the global branch's caches come together
    full = dict(kpg=FAKE, vpg=FAKE, kg=FAKE, vg=FAKE)
    for name in full:
        assert dec(**{**full, name: None}) == ERR_ARG, name
    assert dec(kg=FAKE, vg=FAKE) == ERR_ARG and dec(kpg=FAKE, vpg=FAKE) == ERR_ARG
    assert dec(mode=1) == ERR_ARG and dec(mode=7) == ERR_ARG
    assert dec(thr=float("nan")) == ERR_ARG
    assert dec(mode=2) == ERR_NULL
    for eps in (-1.0, float("inf"), float("nan")):
        assert dec(eps=eps) == ERR_ARG
    assert dec(x=Pre(groups=(1, 2))) == ERR_SHAPE            # three sequences of two
    assert dec(x=Pre(groups=(2, 0), max_group=1)) == ERR_SHAPE
    assert dec(x=Pre(max_prefix=99)) == ERR_SHAPE
    assert dec(x=Pre(total_tokens=131)) == ERR_SHAPE
    assert dec(x=Pre(num_prefixes=0)) == ERR_SHAPE
    assert dec(x=Pre(max_group=0, host=False)) == ERR_SHAPE
    assert dec(x=Pre(max_group=3, host=False)) == ERR_SHAPE
    assert dec(x=Pre(max_prefix=-1, host=False)) == ERR_SHAPE
    assert dec(x=Pre(max_prefix=(1 << 31) - 40, host=False)) == ERR_UNSUPPORTED
    assert dec(p=Prob((0, 20)), x=Pre((0, 30))) == ERR_SHAPE  # a cache without rows
    assert dec(ws=None) == ERR_WORKSPACE and dec(ws=MISALIGNED) == ERR_WORKSPACE
    need = lib.logo_decode_prefix_workspace_bytes(p.c, Pre().c)
    assert dec(ws_bytes=256) == ERR_WORKSPACE and need > 256
    for nm in ("cu_prefix", "cu_group"):
        x = Pre()
        setattr(x.s, nm, None)
        assert dec(x=x) == ERR_NULL


def test_cache_score_refusals(lib):
    import paper_2608_29539_amd as pk
    p = Prob((100, 50))
    need = lib.logo_workspace_bytes(p.c, pk.LOGO_ENTRY_CACHE_SCORE, 40)

    def sc(p=p, q=FAKE, k=FAKE, sel=FAKE, cu=FAKE, cap=40, lse=None, out=FAKE, ws=FAKE,
           ws_bytes=need):
        return lib.logo_cache_score(p.c, q, k, sel, cu, cap, lse, None, out, ws, ws_bytes, None)

    for name in ("q", "k", "out"):
        assert sc(**{name: None}) == ERR_NULL, name
    assert sc(sel=None) == ERR_NULL and sc(cu=None) == ERR_NULL
    assert sc(cap=-1) == ERR_SHAPE
    assert sc(q=MISALIGNED) == ERR_ARG and sc(k=MISALIGNED) == ERR_ARG
    assert sc(ws=None) == ERR_WORKSPACE and sc(ws_bytes=need - 1) == ERR_WORKSPACE
    assert sc(ws=MISALIGNED) == ERR_WORKSPACE
    assert sc(p=Prob(hq=6, hkv=4)) == ERR_SHAPE and sc(p=Prob(d=32)) == ERR_UNSUPPORTED
    assert sc(p=Prob((0, 0))) == OK                          # nothing to write


def test_decode_score_refusals(lib):
    import paper_2608_29539_amd as pk
    p = Prob((100, 50))
    need = lib.logo_workspace_bytes(p.c, pk.LOGO_ENTRY_DECODE_SCORE, 0)

    def sc(p=p, q=FAKE, k=FAKE, gate=FAKE, mode=0, thr=0.5, thr_dev=None, out=FAKE, ws=FAKE,
           ws_bytes=need):
        return lib.logo_decode_score(p.c, q, k, gate, mode, thr, thr_dev, None, out, ws, ws_bytes,
                                     None)

    for name in ("q", "k", "gate", "out"):
        assert sc(**{name: None}) == ERR_NULL, name
    assert sc(mode=1) == ERR_ARG and sc(thr=float("nan")) == ERR_ARG
    assert sc(mode=2) == ERR_NULL
    assert sc(q=MISALIGNED) == ERR_ARG and sc(k=MISALIGNED) == ERR_ARG
    assert sc(p=Prob((100, 0, 50))) == ERR_SHAPE
    assert sc(ws=None) == ERR_WORKSPACE and sc(ws_bytes=need - 1) == ERR_WORKSPACE
    assert sc(p=Prob((100,), hq=8193 * 2, hkv=2), ws_bytes=1 << 40) == ERR_UNSUPPORTED


def test_evict_refusals(lib):
    p = Prob((100, 50))

    def ev(p=p, score=FAKE, budget=60, recent=10, k=FAKE, v=FAKE, kg=None, vg=None, ko=FAKE,
           vo=FAKE, kgo=None, vgo=None, so=FAKE, idx=FAKE, cu=FAKE, cap=109):
        return lib.logo_cache_evict(p.c, score, budget, recent, k, v, kg, vg, ko, vo, kgo, vgo, so,
                                    idx, cu, cap, FAKE, 1 << 40, None)

    assert ev() == ERR_SHAPE                                 # 60 + 50 rows stay
    for name in ("score", "so", "idx", "cu"):
        assert ev(cap=110, **{name: None}) == ERR_NULL, name
    assert ev(budget=0) == ERR_ARG and ev(budget=-3) == ERR_ARG and ev(recent=-1) == ERR_ARG
    for name in ("k", "v", "ko", "vo"):
        assert ev(cap=110, **{name: None}) == ERR_ARG, name
        assert ev(cap=110, **{name: MISALIGNED}) == ERR_ARG, name
    assert ev(cap=110, kg=FAKE, vg=FAKE) == ERR_ARG
    assert ev(cap=110, kg=FAKE, kgo=FAKE) == ERR_ARG
    assert ev(p=Prob((100, 50), host=False), cap=119) == ERR_SHAPE


def test_binding_refusals():
    """What the Python layer checks before it calls the library."""
    import torch

    import paper_2608_29539_amd as pk
    cu = torch.tensor([0, 4], dtype=torch.int32)
    prob = pk.Problem(cu, 4, 2, 64, 8, cu_seqlens_host=[0, 4])
    bf = dict(dtype=torch.bfloat16)
    q, k, gate = torch.zeros(1, 4, 64, **bf), torch.zeros(4, 2, 64, **bf), torch.zeros(1)
    pre = pk.Prefix(torch.tensor([0, 4], dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32),
                    cu_prefix_host=[0, 4], cu_group_host=[0, 1])
    with pytest.raises(ValueError, match="device tensor"):
        pk.logo_decode_prefix(prob, pre, q, k, k, k, k, gate, threshold=0.5)
    with pytest.raises(ValueError, match="exactly one"):
        pk.logo_decode_prefix(prob, pre, q, k, k, k, k, gate)
    with pytest.raises(ValueError, match="exactly one"):
        pk.logo_decode_score(prob, q, k, gate)
    with pytest.raises(TypeError, match="score"):
        pk.logo_cache_evict(prob, torch.zeros(2, 4, dtype=torch.float64), 2)
    with pytest.raises(ValueError, match="R \\+ 1"):
        pk.Prefix(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="host copies"):
        pk.Prefix(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="R \\+ 1"):
        pk.Prefix(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                  cu_prefix_host=[0, 1, 2], cu_group_host=[0, 1])
